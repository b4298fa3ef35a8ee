// Attention over a cache in 4 bits (layout: q4.cuh) for few query rows per KV head: a decoded token, a short draft.  bfloat16 steps,
// head_dim 64 or 128, up to 64 rows.
//
// With few rows the cache's bytes are what the call takes, and the codes have to be opened at the rate of the memory: 128 tokens of a
// KV head arrive every 0.4 us per SM.  Here they go from shared memory to registers and stay there: opened codes ARE the fragments of
// the warp-wide matrix instruction (m16n8k16, 16 tokens or channels by 8 rows), so nothing is written back.  (Through the tcgen05
// kernel, opened tiles are written to and read from shared memory, which alone takes 1900 cycles per 128 tokens: four sequences of
// 96K to 128K tokens x 4 layers, 4 rows per head, 1630 us.)  Both products are turned over:
//   S^T = K Q^T   [16 tokens x 8 rows]      A = keys, B = queries
//   O^T += V^T P^T  [16 channels x 8 rows]  A = values, B = weights
// A product's summation index may be numbered in any order as long as both factors agree, and so may tokens: with g = lane / 4 and
// t = lane % 4, channels 32 t .. 32 t + 31 of a key belong to lane t (16 bytes of codes, all of whose bits it uses), and of 64 tokens the
// value words of tokens 8 t .. 8 t + 7 and 32 + 8 t .. do.  Step s (of four) takes tokens 8 i + 2 s and 8 i + 2 s + 1 of every group of
// eight: A's row 2 i + e of S^T is token 8 i + 2 s + e, which is where P^T, transposed in registers, needs it.
//
// A warp walks chunks of 64 tokens on its own (one to four pages, copied in bulk into stages of its own), with its own running maximum,
// sums and accumulators; the warps of a CTA meet at the end, KV splits in the merge kernel.
// Precision: weights rounded to bfloat16 for the second product (2^-8 of each at most), their sums taken before that in float32.
#include <type_traits>

#include "attn_tc.cuh"
#include "q4.cuh"

namespace specpv {

namespace {

using namespace tc;

constexpr int kChunk = 64;               // tokens
constexpr int kMaxRows = 64;             // of a KV head; also bounds the step's tokens, which are one chunk
constexpr float kRaise = 60.f;           // log2 of the weight from which references are raised

// rows of a CTA: 8 NT.  More accumulators, fewer warps.
template <int D, int NT>
struct RowsShape {
    static constexpr int kWarps = NT <= 2 ? 12 : 8;
    static constexpr int kStages = 2;
    static constexpr int kStageBytes = kChunk * (D + 8);
    static constexpr int kPitch = D + 4;  // of the accumulators when the warps meet
    static constexpr int kRing = kWarps * kStages * kStageBytes;
    static constexpr int kMeet = kWarps * 8 * NT * kPitch * 4;
    static constexpr int kStepV = D * kChunk * 2;
    static constexpr int kQ = NT > 2 ? 8 * NT * D * 2 : 0;
    static constexpr int kSmemBytes = (kRing > kMeet ? kRing : kMeet) + kStepV + kQ;
};

struct RowsParams {
    const void* q;
    const void* k_new;
    const void* v_new;
    const uint64_t* tree_mask;
    const int32_t* q_lens;
    const void* pool;
    const int32_t* block_table;
    const int32_t* seq_lens;
    void* out;
    float* lse;
    float* part_o;   // [lb][Hkv][splits][R_max][d]
    float* part_ml;  // [lb][Hkv][splits][R_max][2], natural logarithm
    void* workspace;
    int layer0, batch, M_max, mask_words, Hq, Hkv, G, bs, bs_log2, max_blocks, n_pages;
    int n_splits, n_row_groups, out_f32;
    float scale_log2;
    uint32_t q4_mask, q4_ones;  // q4::kMask, q4::kOnes
};

__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {  // an 8 x 8 matrix of 16-bit elements, two of a row to a lane
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ uint4 lds16(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lds8(uint32_t at) {
    uint2 v;
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds4(uint32_t at) {
    uint32_t v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}

template <int D, int NT>
__global__ void __launch_bounds__(32 * RowsShape<D, NT>::kWarps, 1) attn_q4_rows_kernel(const __grid_constant__ RowsParams p) {
    using S = RowsShape<D, NT>;
    constexpr int kWarps = S::kWarps, kThreads = 32 * kWarps, kRows = 8 * NT;
    constexpr int kWords = D / 32;        // of codes per lane and key
    constexpr bool kQInSmem = NT > 2;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ uint64_t full[kWarps][S::kStages];
    __shared__ uint32_t bad_pages[kWarps][S::kStages];
    __shared__ float s_m[kWarps][kRows], s_l[kWarps][kRows], s_factor[kWarps][kRows], s_sum[kRows], s_top[kRows];
    __shared__ int abort_flag, odd;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    int x = blockIdx.x;
    const int rg = x % p.n_row_groups;
    x /= p.n_row_groups;
    const int split = x % p.n_splits;
    x /= p.n_splits;
    const int h = x % p.Hkv, lb = x / p.Hkv, b = lb % p.batch, l = lb / p.batch;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kWarps * S::kStages; ++i) mbar_init(smem_u32(&full[0][0] + i), 1);
        abort_flag = 0;
        odd = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    const uint32_t base = smem_u32(smem), step_v = base + (S::kRing > S::kMeet ? S::kRing : S::kMeet), q_smem = step_v + S::kStepV;
    __syncthreads();
    if (p.n_splits == 1) pdl_trigger();
    pdl_wait();

    const int seq_len = (int)min((long long)max(p.seq_lens[b], 0), (long long)p.max_blocks * p.bs);
    const int M = min(max(p.q_lens ? p.q_lens[b] : p.M_max, 0), p.M_max);
    const int row0 = rg * kRows, rows = min(kRows, M * p.G - row0);
    if (rows <= 0) return;  // (uniform for the CTA)
    // KV range of this split: an equal share of the chunks and of the step's tokens, which come last
    const int ctx_chunks = (seq_len + kChunk - 1) / kChunk;
    const long long positions = ctx_chunks + 1;
    const int begin = (int)(positions * split / p.n_splits), n_chunks = (int)(positions * (split + 1) / p.n_splits) - begin;
    const bool last = split == p.n_splits - 1;
    const int n_ctx = n_chunks - (last ? 1 : 0);

    // ---- copies: chunk i of the warp's (the CTA's chunk warp + i kWarps) into stage i % kStages ----
    const int ppc = kChunk >> p.bs_log2;  // pages per chunk
    const uint32_t page_bytes = (uint32_t)p.bs * (D + 8);
    const char* pool = reinterpret_cast<const char*>(p.pool) + ((size_t)(p.layer0 + l) * p.n_pages * p.Hkv + h) * page_bytes;
    const int32_t* table = p.block_table + (size_t)b * p.max_blocks;
    const uint32_t ring = base + warp * S::kStages * S::kStageBytes;
    auto entry_of = [&](int i) {  // of the lane's page; looked at when it is used
        const int c = warp + i * kWarps, blk = (begin + c) * ppc + lane;
        return lane >= ppc || c >= n_ctx || (long long)blk * p.bs >= seq_len || blk >= p.max_blocks ? -1 : table[blk];
    };
    auto copy = [&](int i, int page) {
        const int c = warp + i * kWarps, blk = (begin + c) * ppc + lane;
        if (c >= n_ctx) return;
        const bool wanted = lane < ppc && (long long)blk * p.bs < seq_len && blk < p.max_blocks, there = wanted && page >= 0 && page < p.n_pages;
        if (wanted && !there) record_fault(p.workspace, SPECPV_ERR_BAD_BLOCK_TABLE, b, blk, page, l);
        const uint32_t bad = __ballot_sync(0xffffffffu, wanted && !there), n = (uint32_t)__popc(__ballot_sync(0xffffffffu, there));
        const uint32_t bar = smem_u32(&full[warp][i & 1]);
        if (lane == 0) {
            bad_pages[warp][i & 1] = bad;
            mbar_expect_tx(bar, n * page_bytes);
        }
        __syncwarp();
        if (there)
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                         ::"r"(ring + (i & 1) * S::kStageBytes + lane * page_bytes), "l"(pool + (size_t)page * p.Hkv * page_bytes), "r"(page_bytes), "r"(bar)
                         : "memory");
        __syncwarp();
    };
    static_assert(S::kStages == 2, "stage = chunk & 1");
    copy(0, entry_of(0));
    copy(1, entry_of(1));
    int next_entry = entry_of(2);

    // ---- the rows' queries as B fragments; the step's values, transposed, in shared memory ----
    uint32_t qf[kQInSmem ? 1 : NT][kQInSmem ? 1 : D / 8];
    auto q_row = [&](int r) {
        const int row = row0 + r;
        return reinterpret_cast<const __nv_bfloat16*>(p.q) + (((size_t)lb * p.M_max + row / p.G) * p.Hq + h * p.G + row % p.G) * D;
    };
    if constexpr (kQInSmem) {  // [row][lane t][D / 8 words], words of a lane 16 bytes at a time, spread over the banks
        for (int i = threadIdx.x; i < kRows * (D / 8); i += kThreads) {
            const int r = i / (D / 8), piece = i % (D / 8);
            uint4 v = make_uint4(0, 0, 0, 0);
            if (r < rows) v = reinterpret_cast<const uint4*>(q_row(r))[piece];
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(q_smem + r * D * 2 + ((piece ^ (r & 7)) << 4)), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
        }
    } else {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (n * 8 + g < rows) v = reinterpret_cast<const uint4*>(q_row(n * 8 + g))[t * (D / 32) + i];
                qf[n][4 * i] = v.x; qf[n][4 * i + 1] = v.y; qf[n][4 * i + 2] = v.z; qf[n][4 * i + 3] = v.w;
            }
    }
    if (last) {
        const __nv_bfloat16* src = reinterpret_cast<const __nv_bfloat16*>(p.v_new) + ((size_t)lb * p.M_max * p.Hkv + h) * D;
        uint16_t* dst = reinterpret_cast<uint16_t*>(smem + (step_v - base));  // [channel][64 tokens], 16-byte pieces swizzled by channel
        bool found = false;
        for (int i = threadIdx.x; i < kChunk * D; i += kThreads) {
            const int a = i / D, c = i % D;
            uint16_t v = 0;
            if (a < M) {
                v = __bfloat16_as_ushort(src[(size_t)a * p.Hkv * D + c]);
                if ((v & 0x7F80u) == 0x7F80u) {  // infinite and NaN values go another way
                    found = true;
                    v = 0;
                }
            }
            dst[c * kChunk + (((a >> 3) ^ (c & 7)) << 3) + (a & 7)] = v;
        }
        if (found) odd = 1;
    }
    if (kQInSmem || last) __syncthreads();

    // ---- where the lane's codes are in a stage (chunks of a page: keys [d / 32][bs][16 bytes], values [bs / 16][d][8 bytes]) ----
    const int bs_mask = p.bs - 1;
    const int k_token = 8 * (g >> 1) + (g & 1);  // of A's row g at step 0; row g + 8 is 32 tokens on; a step is two tokens
    uint32_t k_off[2], k_par[2], v_off[2], v_par[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int kt = k_token + 32 * i, vt = 8 * t + 32 * i;
        const uint32_t kp = (uint32_t)(kt >> p.bs_log2) * page_bytes, vp = (uint32_t)(vt >> p.bs_log2) * page_bytes;
        const int ka = kt & bs_mask, va = vt & bs_mask;
        k_off[i] = kp + (D == 128 ? (uint32_t)(t * p.bs + ka) * 16 : (uint32_t)((t >> 1) * p.bs + ka) * 16 + (t & 1) * 8);
        k_par[i] = kp + (uint32_t)q4::param_at(p.bs, D, 0, ka) * 2;
        v_off[i] = vp + (uint32_t)q4::v_word(p.bs, D, va, g) * 4;
        v_par[i] = vp + (uint32_t)q4::param_at(p.bs, D, 2, va) * 2;
    }
    const uint32_t two_bs = 2u * p.bs;

    float m[NT][2], sum[NT][2], acc[D / 16][NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        m[n][0] = m[n][1] = 0.f;
        sum[n][0] = sum[n][1] = 0.f;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) acc[c][n][0] = acc[c][n][1] = acc[c][n][2] = acc[c][n][3] = 0.f;
    }
    const float scale = p.scale_log2;
    const uint32_t mask = p.q4_mask, ones = p.q4_ones;
    // (Two copies of the code: where a branch chose between opened codes and the step's own rows, every fragment was moved once more.)
    auto work = [&](auto is_step, int i) {
        constexpr bool step = decltype(is_step)::value;
        const int chunk = warp + i * kWarps;
        const uint32_t stage = ring + (i & 1) * S::kStageBytes;
        const int left = step ? M : seq_len - (begin + chunk) * kChunk;  // valid tokens of the chunk, if fewer than 64
        uint32_t bad = 0;
        if (!step) {
            if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&full[warp][i & 1]), (i >> 1) & 1, &abort_flag, p.workspace, 41))) return false;
            bad = bad_pages[warp][i & 1];
        }
        // ---- S^T and the weights, 16 tokens a step ----
        uint32_t pf[4][NT][2];
        float add[NT][2];
        // A row's reference is its largest score in the warp's first chunk, which is looked at once for that before it is worked on.  It
        // is raised when a weight passes 2^60 (float32 sums and bfloat16 weights keep their relative precision at any exponent).
        bool look = i == 0;
        for (bool again = true; again;) {
            again = false;
            float most[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                add[n][0] = add[n][1] = 0.f;
                most[n][0] = most[n][1] = -INFINITY;
            }
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                float c[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n) c[n][0] = c[n][1] = c[n][2] = c[n][3] = 0.f;
                uint32_t k[2][D / 8];  // pairs of channels of rows g and g + 8
                if constexpr (!step) {
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        uint32_t w[kWords];
                        if constexpr (D == 128) {
                            const uint4 v = lds16(stage + k_off[r] + s * 32);
                            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
                        } else {
                            const uint2 v = lds8(stage + k_off[r] + s * 32);
                            w[0] = v.x; w[1] = v.y;
                        }
                        uint32_t sc, of;
                        asm volatile("{\n\t.reg .b16 x, y;\n\tld.shared.b16 x, [%2];\n\tld.shared.b16 y, [%3];\n\tmov.b32 %0, {x, x};\n\tmov.b32 %1, {y, y};\n\t}"
                                     : "=r"(sc), "=r"(of) : "r"(stage + k_par[r] + s * 4), "r"(stage + k_par[r] + two_bs + s * 4) : "memory");
                        if (bad >> ((k_token + 32 * r) >> p.bs_log2) & 1) sc = of = 0;
#pragma unroll
                        for (int i2 = 0; i2 < kWords; ++i2)
#pragma unroll
                            for (int e = 0; e < 4; ++e) k[r][4 * i2 + e] = q4::fma_bf16x2(q4::open_pair(w[i2], e, mask, ones), sc, of);
                    }
                } else {
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int a = k_token + 32 * r + 2 * s;
                        const uint4* src = reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(p.k_new) +
                                                                          (((size_t)lb * p.M_max + a) * p.Hkv + h) * D) + t * kWords;
#pragma unroll
                        for (int i2 = 0; i2 < kWords; ++i2) {
                            const uint4 v = a < M ? src[i2] : make_uint4(0, 0, 0, 0);
                            k[r][4 * i2] = v.x; k[r][4 * i2 + 1] = v.y; k[r][4 * i2 + 2] = v.z; k[r][4 * i2 + 3] = v.w;
                        }
                    }
                }
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        uint32_t b0, b1;
                        if constexpr (kQInSmem) {
                            const int piece = t * kWords + ks / 2;
                            const uint2 v = lds8(q_smem + (n * 8 + g) * D * 2 + ((piece ^ g) << 4) + (ks & 1) * 8);
                            b0 = v.x; b1 = v.y;
                        } else {
                            b0 = qf[n][2 * ks]; b1 = qf[n][2 * ks + 1];
                        }
                        mma_16816(c[n], k[0][2 * ks], k[1][2 * ks], k[0][2 * ks + 1], k[1][2 * ks + 1], b0, b1);
                    }
                }
                // tokens that are not there, or not seen: -infinity
                if (step || left < kChunk) {
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int a = k_token + 32 * r + 2 * s;
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                bool seen = a < left;
                                if (step) {
                                    const int row = row0 + n * 8 + 2 * t + e;
                                    seen = seen && row < row0 + rows && (p.tree_mask[((size_t)b * p.M_max + row / p.G) * p.mask_words] >> a & 1);
                                }
                                if (!seen) c[n][2 * r + e] = -INFINITY;
                            }
                    }
                }
                float top = -INFINITY;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        c[n][e] = fmaf(c[n][e], scale, -m[n][e & 1]);
                        top = fmaxf(top, c[n][e]);
                    }
                if (look) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) most[n][e & 1] = fmaxf(most[n][e & 1], c[n][e]);
                    continue;
                }
                if (__any_sync(0xffffffffu, top > kRaise)) {
                    // references rise to the largest of these tokens; sums and accumulators follow, and the chunk starts over
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float rise = fmaxf(fmaxf(c[n][e], c[n][e + 2]), 0.f);
#pragma unroll
                            for (int o = 4; o < 32; o <<= 1) rise = fmaxf(rise, __shfl_xor_sync(0xffffffffu, rise, o));
                            const float factor = ex2(-rise);
                            m[n][e] += rise;
                            sum[n][e] *= factor;
#pragma unroll
                            for (int d = 0; d < D / 16; ++d) {
                                acc[d][n][e] *= factor;
                                acc[d][n][e + 2] *= factor;
                            }
                        }
                    again = true;
                    break;
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        c[n][e] = ex2(c[n][e]);
                        add[n][e & 1] += c[n][e];
                    }
                    pf[s][n][0] = transposed(pack_bf16(c[n][0], c[n][1]));
                    pf[s][n][1] = transposed(pack_bf16(c[n][2], c[n][3]));
                }
            }
            if (look) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
#pragma unroll
                        for (int o = 4; o < 32; o <<= 1) most[n][e] = fmaxf(most[n][e], __shfl_xor_sync(0xffffffffu, most[n][e], o));
                        m[n][e] = most[n][e] == -INFINITY ? 0.f : most[n][e];
                    }
                look = false;
                again = true;
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            sum[n][0] += add[n][0];
            sum[n][1] += add[n][1];
        }
        // ---- O^T += V^T P^T, 16 channels at a time ----
        uint32_t sc[2][4], of[2][4];
        if (!step) {
#pragma unroll
            for (int i2 = 0; i2 < 2; ++i2) {
                const uint4 a = lds16(stage + v_par[i2]), z = lds16(stage + v_par[i2] + two_bs);
                sc[i2][0] = a.x; sc[i2][1] = a.y; sc[i2][2] = a.z; sc[i2][3] = a.w;
                of[i2][0] = z.x; of[i2][1] = z.y; of[i2][2] = z.z; of[i2][3] = z.w;
            }
            if (left < kChunk || bad) {  // a token that is not there: no scale, no offset, no value
#pragma unroll
                for (int i2 = 0; i2 < 2; ++i2) {
                    const bool gone = bad >> ((8 * t + 32 * i2) >> p.bs_log2) & 1;
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        const int n = gone ? 0 : left - (8 * t + 32 * i2 + 2 * s);
                        const uint32_t keep = n > 1 ? ~0u : n > 0 ? 0xFFFFu : 0u;
                        sc[i2][s] &= keep;
                        of[i2][s] &= keep;
                    }
                }
            }
        }
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
            uint32_t a[4][4];  // [row g | g + 8, first | second tokens][step]
            if constexpr (!step) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {  // (row j & 1, tokens j >> 1)
                    const uint32_t w = lds4(stage + v_off[j >> 1] + d * 128 + (j & 1) * 64);
#pragma unroll
                    for (int s = 0; s < 4; ++s) a[j][s] = q4::fma_bf16x2(q4::open_pair(w, s, mask, ones), sc[j >> 1][s], of[j >> 1][s]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int ch = 16 * d + g + 8 * (j & 1);
                    const uint4 v = lds16(step_v + ch * (kChunk * 2) + (((t + 4 * (j >> 1)) ^ (ch & 7)) << 4));
                    a[j][0] = v.x; a[j][1] = v.y; a[j][2] = v.z; a[j][3] = v.w;
                }
            }
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int n = 0; n < NT; ++n) mma_16816(acc[d][n], a[0][s], a[1][s], a[2][s], a[3][s], pf[s][n][0], pf[s][n][1]);
        }
        __syncwarp();
        if (!step) {
            copy(i + 2, next_entry);
            next_entry = entry_of(i + 3);
        }
        return true;
    };
    int i = 0;
    bool ok = true;
#pragma unroll 1
    for (; ok && warp + i * kWarps < n_ctx; ++i) ok = work(std::false_type(), i);
    if (ok && warp + i * kWarps < n_chunks) work(std::true_type(), i);

    // ---- the warps meet ----
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float v = sum[n][e];
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
            if (g == 0) {
                s_m[warp][n * 8 + 2 * t + e] = m[n][e];
                s_l[warp][n * 8 + 2 * t + e] = v;
            }
        }
    __syncthreads();  // also: every copy has been consumed, the ring is free
    if ((int)threadIdx.x < kRows) {
        const int r = threadIdx.x;
        float top = -INFINITY, total = 0.f;
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s_l[w][r] == 0.f ? -INFINITY : s_m[w][r]);  // (a NaN sum counts)
        for (int w = 0; w < kWarps; ++w) {
            const float f = s_l[w][r] == 0.f ? 0.f : ex2(s_m[w][r] - top);
            s_factor[w][r] = f;
            total += s_l[w][r] * f;
        }
        s_top[r] = top;
        s_sum[r] = total;
    }
    __syncthreads();
    float* meet = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = n * 8 + 2 * t + e;
            const float f = s_factor[warp][r];
            float* to = meet + (warp * kRows + r) * S::kPitch + g;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                to[16 * d] = acc[d][n][e] * f;
                to[16 * d + 8] = acc[d][n][e + 2] * f;
            }
        }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * D; i += kThreads) {
        const int r = i / D, c = i % D, row = row0 + r, j = row / p.G, head = row % p.G;
        float o = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) o += meet[(w * kRows + r) * S::kPitch + c];
        const float total = s_sum[r];
        if (last && odd) {  // infinite and NaN values of the step's tokens that the row sees
            const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(p.v_new) + ((size_t)lb * p.M_max * p.Hkv + h) * D + c;
            const uint64_t seen = p.tree_mask[((size_t)b * p.M_max + j) * p.mask_words];
            for (int a = 0; a < M; ++a) {
                const float y = __bfloat162float(v[(size_t)a * p.Hkv * D]);
                if (!isfinite(y) && (seen >> a & 1)) o += y;
            }
        }
        if (p.n_splits == 1) {
            const size_t at = (((size_t)lb * p.M_max + j) * p.Hq + h * p.G + head) * D + c;
            const float y = total == 0.f ? o : o / total;  // a row that has seen nothing is zero
            if (p.out_f32) reinterpret_cast<float*>(p.out)[at] = y;
            else reinterpret_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(y);
            if (p.lse && c == 0) p.lse[at / D] = total == 0.f ? -INFINITY : fmaf(s_top[r], kLn2, logf(total));
        } else {
            const size_t at = (((size_t)lb * p.Hkv + h) * p.n_splits + split) * ((size_t)p.M_max * p.G) + row;
            p.part_o[at * D + c] = o;
            if (c == 0) {
                // nothing seen: -infinity; a NaN has to survive the merge, which leaves out what weighs nothing
                p.part_ml[at * 2] = total == 0.f ? -INFINITY : total != total ? INFINITY : s_top[r] * kLn2;
                p.part_ml[at * 2 + 1] = total;
            }
        }
    }
    if (abort_flag) __nanosleep(1000000);  // after a wait that gave up, the copies in flight land within microseconds
}

template <int D, int NT>
specpv_status launch_rows_form(const RowsParams& p, int n_ctas, cudaStream_t stream) {
    using S = RowsShape<D, NT>;
    if (!set_smem_limit_once(reinterpret_cast<const void*>(attn_q4_rows_kernel<D, NT>), S::kSmemBytes)) return SPECPV_ERR_CUDA;
    if (launch_pdl(attn_q4_rows_kernel<D, NT>, n_ctas, 32 * S::kWarps, S::kSmemBytes, stream, p) != cudaSuccess) return SPECPV_ERR_CUDA;
    count_launch();
    return SPECPV_OK;
}

}  // namespace

bool attention_q4_rows_wanted(const AttnArgs& a) {
    return a.g.dtype == SPECPV_DTYPE_BF16 && a.M_max * a.g.G <= kMaxRows;
}

specpv_status launch_attention_q4_rows(const AttnArgs& a, cudaStream_t stream) {
    RowsParams p{};
    p.q = a.q; p.k_new = a.k_new; p.v_new = a.v_new; p.tree_mask = a.tree_mask; p.q_lens = a.q_lens; p.pool = a.q4_pool;
    p.block_table = a.block_table; p.seq_lens = a.seq_lens; p.out = a.out; p.lse = a.lse; p.workspace = a.workspace;
    p.layer0 = a.layer0; p.batch = a.batch; p.M_max = a.M_max; p.mask_words = a.mask_words; p.Hq = a.g.Hq; p.Hkv = a.g.Hkv; p.G = a.g.G;
    p.bs = a.g.bs; p.bs_log2 = a.g.bs == 16 ? 4 : a.g.bs == 32 ? 5 : 6;
    p.max_blocks = a.max_blocks; p.n_pages = a.n_pages; p.out_f32 = a.g.out_f32;
    p.scale_log2 = a.g.scale * kLog2e;
    p.q4_mask = q4::kMask; p.q4_ones = q4::kOnes;
    const int R_max = a.M_max * a.g.G, units = a.g.Hkv * a.n_layers * a.batch;
    const int nt = R_max <= 8 ? 1 : R_max <= 16 ? 2 : 4;
    p.n_row_groups = (R_max + 8 * nt - 1) / (8 * nt);
    // KV splits by a cost model in microseconds, one CTA per SM: set-up, the rounds of its warps over their chunks, the meeting, and, with
    // splits, the partial results' round trip and the merge
    const int positions = (a.max_seq_len + kChunk - 1) / kChunk + 1, warps = nt <= 2 ? 12 : 8;
    const long long base = (long long)units * p.n_row_groups;
    const double round = nt == 1 ? 2.2 : nt == 2 ? 2.8 : 3.0;
    const double row_bytes = (double)units * R_max * (a.g.d + 2) * sizeof(float);
    double best = 1e300;
    p.n_splits = 1;
    for (int s = 1; s <= 64 && s <= positions; ++s) {
        if (s > 1 && row_bytes * s > (double)a.partial_bytes) break;
        const long long waves = (base * s + 147) / 148;
        const int chunks = (positions + s - 1) / s;
        double cost = waves * (5.0 + round * ((chunks + warps - 1) / warps));
        if (s > 1) cost += 3.0 + row_bytes * s * 2.0 / 5.3e6;
        if (cost < best) {
            best = cost;
            p.n_splits = s;
        }
    }
    char* ws = reinterpret_cast<char*>(a.workspace) + a.partial_off;
    p.part_o = reinterpret_cast<float*>(ws);
    p.part_ml = reinterpret_cast<float*>(ws + (size_t)units * p.n_splits * R_max * a.g.d * sizeof(float));
    const long long n_ctas = base * p.n_splits;
    if (n_ctas > 0x7FFFFFFF) return SPECPV_ERR_CAPACITY;
    const auto launch = a.g.d == 64 ? (nt == 1 ? launch_rows_form<64, 1> : nt == 2 ? launch_rows_form<64, 2> : launch_rows_form<64, 4>)
                                    : (nt == 1 ? launch_rows_form<128, 1> : nt == 2 ? launch_rows_form<128, 2> : launch_rows_form<128, 4>);
    const specpv_status st = launch(p, (int)n_ctas, stream);
    if (st != SPECPV_OK || p.n_splits == 1) return st;
    return launch_merge_splits(a, p.n_splits, p.part_o, p.part_ml, stream);
}

}  // namespace specpv
