// Attention over a cache in 4 bits (layout: q4.cuh) for few query rows per KV head: a decoded token, a short draft.  bfloat16 steps,
// head_dim 64 or 128, up to 16 rows.
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
// sums and accumulators.  The CTAs, one per SM, take equal shares of all sequences' chunks, whatever their lengths; a share can end one
// sequence's KV head and begin the next.  The warps of a CTA meet at the end of each, the CTAs in the merge kernel.
// Precision: weights rounded to bfloat16 for the second product (2^-8 of each at most), their sums taken before that in float32.
#include <type_traits>

#include "attn_tc.cuh"
#include "q4.cuh"

namespace specpv {

namespace {

using namespace tc;

constexpr int kChunk = 64;               // tokens
// Rows of a KV head; also bounds the step's tokens, which are one chunk.  (us, 65536 tokens x 8 layers, 4 / 8 / 16 rows of 128 here 145 / 146 /
// 241, on the tcgen05 kernel 457 / 483 / 485; 32 rows in one CTA 552, as two CTAs of 16 459, there 486; 4096 tokens x 1 layer 43 / 26, there 16.)
constexpr int kMaxRows = 16;
constexpr float kRaise = 16.f;           // log2 of the weight from which references are raised
// References from here on are coarser than 1.  Scores are then rounded to float32 before the reference, one of them, is taken off: the
// difference of an unrounded product to its own rounding could pass kRaise, at 2^28 and more, and no reference would ever do.
constexpr float kCoarse = 16777216.f;    // 2^24

// rows of a CTA: 8 NT
template <int D, int NT>
struct RowsShape {
    static constexpr int kWarps = NT == 1 ? 12 : 8;
    static constexpr int kStages = 2;  // per warp
    static constexpr int kStageBytes = kChunk * (D + 8);
    static constexpr int kPitch = D + 4;  // of the accumulators when the warps meet
    static constexpr int kRing = kWarps * kStages * kStageBytes;
    static constexpr int kMeet = kWarps * 8 * NT * kPitch * 4;
    static constexpr int kStepV = D * kMaxRows * 2;
    static constexpr int kSmemBytes = (kRing > kMeet ? kRing : kMeet) + kStepV;
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
    float* part_o;   // [lb][Hkv][slots][R_max][d]
    float* part_ml;  // [lb][Hkv][slots][R_max][2], the reference in units of log2, unrounded: the merge takes differences of them
    void* workspace;
    int layer0, batch, M_max, mask_words, Hq, Hkv, G, bs, bs_log2, max_blocks, n_pages;
    int n_layers, n_slots;
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
    constexpr int kTogether = NT == 1 ? 4 : 2;  // steps of 16 tokens whose scores are worked on side by side
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ uint64_t full[kWarps][S::kStages];
    __shared__ uint32_t bad_pages[kWarps][S::kStages];
    __shared__ float s_m[kWarps][kRows], s_l[kWarps][kRows], s_factor[kWarps][kRows], s_sum[kRows], s_top[kRows];
    __shared__ int abort_flag, odd;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kWarps * S::kStages; ++i) mbar_init(smem_u32(&full[0][0] + i), 1);
        abort_flag = 0;
        odd = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    const uint32_t base = smem_u32(smem), step_v = base + (S::kRing > S::kMeet ? S::kRing : S::kMeet);
    __syncthreads();
    pdl_wait();

    // ---- the CTA's share: an equal part of the positions (chunks, and the step's tokens behind them) of all units, which are
    // (layer, sequence, KV head) in that order.  At least so many positions that no unit meets more CTAs than it has slots.
    auto positions_of = [&](int b) {
        return b < p.batch ? (int)((min((long long)max(p.seq_lens[b], 0), (long long)p.max_blocks * p.bs) + kChunk - 1) / kChunk) + 1 : 0;
    };
    int per_head = 0, longest = 0;  // positions of a layer's KV head, all sequences
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
        const int n = positions_of(b0 + lane);
        per_head += __reduce_add_sync(0xffffffffu, n);
        longest = max(longest, __reduce_max_sync(0xffffffffu, n));
    }
    const int total = per_head * p.Hkv * p.n_layers;
    int n_ctas = (int)gridDim.x, share = total / n_ctas;
    if ((long long)share * (p.n_slots - 1) < longest) {
        const int least = (longest + p.n_slots - 2) / (p.n_slots - 1);
        n_ctas = max(1, min(n_ctas, total / least));
        share = total / n_ctas;
    }
    if ((int)blockIdx.x >= n_ctas) return;
    // floor(total c / n_ctas), which lies on a unit's edge wherever it can, and its inverse, the last CTA whose share starts at or
    // before a position (a float32 guess, put right)
    const int more = total - share * n_ctas;
    const float per_position = (float)n_ctas / (float)total;
    auto share_at = [&](int c) { return share * c + more * c / n_ctas; };
    auto cta_of = [&](int at) {
        int c = min((int)((float)at * per_position), n_ctas - 1);
        while (share_at(c) > at) --c;
        while (share_at(c + 1) <= at) ++c;
        return c;
    };
    int at = share_at(blockIdx.x);
    const int share_end = share_at(blockIdx.x + 1);
    uint32_t fills = 0;  // chunks that the warp has taken from its stages so far
    while (at < share_end) {
        // ---- the unit at `at`, and the part of it that is the CTA's ----
        const int l = at / (per_head * p.Hkv);
        int in_layer = at - l * per_head * p.Hkv, b = 0, n_positions = 0;
        for (int b0 = 0; n_positions == 0; b0 += 32) {  // (ends: in_layer lies within one of the sequences)
            const int n = positions_of(b0 + lane);
            int upto = n;  // inclusive sums over the lanes
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += v;
            }
            const unsigned beyond = __ballot_sync(0xffffffffu, upto * p.Hkv > in_layer);
            const int found = beyond ? __ffs(beyond) - 1 : 31;
            const int before = __shfl_sync(0xffffffffu, upto - n, found);
            if (beyond) {
                in_layer -= before * p.Hkv;
                b = b0 + found;
                n_positions = __shfl_sync(0xffffffffu, n, found);
            } else {
                in_layer -= __shfl_sync(0xffffffffu, upto, 31) * p.Hkv;
                if (b0 + 32 >= p.batch) return;
            }
        }
        const int h = in_layer / n_positions, begin = in_layer % n_positions, lb = l * p.batch + b;
        const int n_chunks = min(n_positions - begin, share_end - at);
        const int unit_at = at - begin;
        const int first_cta = cta_of(unit_at), n_parts = cta_of(unit_at + n_positions - 1) - first_cta + 1, part = (int)blockIdx.x - first_cta;
        at += n_chunks;

        const int seq_len = (int)min((long long)max(p.seq_lens[b], 0), (long long)p.max_blocks * p.bs);
        const int M = min(max(p.q_lens ? p.q_lens[b] : p.M_max, 0), p.M_max);
        const int rows = M * p.G;
        if (rows <= 0) continue;  // (uniform for the CTA)
        const bool last = begin + n_chunks == n_positions;  // the step's tokens are here
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
        const uint32_t fills0 = fills;
        auto copy = [&](int i, int page) {
            const int c = warp + i * kWarps, blk = (begin + c) * ppc + lane;
            if (c >= n_ctx) return;
            const bool wanted = lane < ppc && (long long)blk * p.bs < seq_len && blk < p.max_blocks, there = wanted && page >= 0 && page < p.n_pages;
            if (wanted && !there) record_fault(p.workspace, SPECPV_ERR_BAD_BLOCK_TABLE, b, blk, page, l);
            const uint32_t bad = __ballot_sync(0xffffffffu, wanted && !there), n = (uint32_t)__popc(__ballot_sync(0xffffffffu, there));
            const uint32_t slot = (fills0 + i) % S::kStages, bar = smem_u32(&full[warp][slot]);
            if (lane == 0) {
                bad_pages[warp][slot] = bad;
                mbar_expect_tx(bar, n * page_bytes);
            }
            __syncwarp();
            if (there)
                asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                             ::"r"(ring + slot * S::kStageBytes + lane * page_bytes), "l"(pool + (size_t)page * p.Hkv * page_bytes), "r"(page_bytes), "r"(bar)
                             : "memory");
            __syncwarp();
        };
        constexpr int kStages = S::kStages;
        static_assert(kStages == 1 || kStages == 2, "stage = chunk % kStages");
#pragma unroll
        for (int i = 0; i < kStages; ++i) copy(i, entry_of(i));
        int next_entry = entry_of(kStages);

        // ---- the rows' queries as B fragments; the step's values, transposed, in shared memory ----
        uint32_t qf[NT][D / 8];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int r = n * 8 + g;
            const uint4* src = reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(p.q) +
                                                              (((size_t)lb * p.M_max + r / p.G) * p.Hq + h * p.G + r % p.G) * D) + t * (D / 32);
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (r < rows) v = src[i];
                qf[n][4 * i] = v.x; qf[n][4 * i + 1] = v.y; qf[n][4 * i + 2] = v.z; qf[n][4 * i + 3] = v.w;
            }
        }
        if (last) {
            const __nv_bfloat16* src = reinterpret_cast<const __nv_bfloat16*>(p.v_new) + ((size_t)lb * p.M_max * p.Hkv + h) * D;
            uint16_t* dst = reinterpret_cast<uint16_t*>(smem + (step_v - base));  // [token / 8][channel][8 tokens]
            bool found = false;
            for (int i = threadIdx.x; i < kMaxRows * D; i += kThreads) {
                const int a = i / D, c = i % D;
                uint16_t v = 0;
                if (a < M) {
                    v = __bfloat16_as_ushort(src[(size_t)a * p.Hkv * D + c]);
                    if ((v & 0x7F80u) == 0x7F80u) {  // infinite and NaN values go another way
                        found = true;
                        v = 0;
                    }
                }
                dst[((a >> 3) * D + c) * 8 + (a & 7)] = v;
            }
            if (found) odd = 1;
            __syncthreads();
        }

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
            k_par[i] = kp + (uint32_t)q4::param_at(p.bs, D, 0, ka & ~7) * 2;  // of the group of eight
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
        auto any_coarse = [&](const float (&reference)[NT][2]) {
            bool any = false;  // (of an infinite one nothing can be told apart: its row is NaN, and others' copy need not change)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) any |= fabsf(reference[n][e]) >= kCoarse && fabsf(reference[n][e]) < INFINITY;
            return __any_sync(0xffffffffu, any) != 0;
        };
        const uint32_t mask = p.q4_mask, ones = p.q4_ones;
        // (Copies of the code: where a branch chose between opened codes and the step's own rows, every fragment was moved once more.  A branch
        // that told coarse references apart cost 6 % over long caches, a copy 1 %: 445 -> 474, 450 us for four sequences of 96K to 128K x 4 layers.)
        enum Outcome { kGaveUp, kDone, kTooCoarse };  // kTooCoarse: a reference has to be coarse, and nothing has been done
        auto work = [&](auto is_step, auto is_coarse, int i) {
            constexpr bool step = decltype(is_step)::value, coarse = decltype(is_coarse)::value;
            const int chunk = warp + i * kWarps;
            const uint32_t slot = (fills0 + i) % kStages, stage = ring + slot * S::kStageBytes;
            const int left = step ? M : seq_len - (begin + chunk) * kChunk;  // valid tokens of the chunk, if fewer than 64
            uint32_t bad, step_sees[NT][2];  // the lane's rows: a bit per token of the step
            if constexpr (step) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int row = n * 8 + 2 * t + e;
                        step_sees[n][e] = row < rows ? (uint32_t)p.tree_mask[((size_t)b * p.M_max + row / p.G) * p.mask_words] : 0u;
                    }
            }
            if constexpr (!step) {
                if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&full[warp][slot]), (fills0 + i) / kStages & 1, &abort_flag, p.workspace, 41))) return kGaveUp;
                bad = bad_pages[warp][slot];
                if (bad || left < kChunk) {
                    // Tokens behind a bad page id have no scales and offsets, nor (values) have those past the end: zeros.
                    for (int a = lane; a < kChunk; a += 32) {
                        const int page = a >> p.bs_log2, at = a & (p.bs - 1);
                        const bool gone = bad >> page & 1;
                        uint16_t* par = reinterpret_cast<uint16_t*>(smem + (stage - base) + page * page_bytes);
                        if (gone) par[q4::param_at(p.bs, D, 0, at)] = par[q4::param_at(p.bs, D, 1, at)] = 0;
                        if (gone || a >= left) par[q4::param_at(p.bs, D, 2, at)] = par[q4::param_at(p.bs, D, 3, at)] = 0;
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // before the stage is filled again
                    __syncwarp();
                }
            }
            // ---- S^T and the weights, 16 tokens a step ----
            uint32_t pf[4][NT][2];
            float add[NT][2];
            uint32_t k_scale[2][4], k_offset[2][4];  // of tokens 2 s and 2 s + 1 of the lane's eight
            const uint32_t half = g & 1 ? 0x3232 : 0x1010;
            if constexpr (!step) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const uint4 a = lds16(stage + k_par[r]), z = lds16(stage + k_par[r] + two_bs);
                    k_scale[r][0] = a.x; k_scale[r][1] = a.y; k_scale[r][2] = a.z; k_scale[r][3] = a.w;
                    k_offset[r][0] = z.x; k_offset[r][1] = z.y; k_offset[r][2] = z.z; k_offset[r][3] = z.w;
                }
            }
            // A row's reference is its largest score in the warp's first chunk (looked at once more where its scores are not all in
            // registers together).  It is raised when a weight passes 2^16: float32 sums and bfloat16 weights
            // keep their relative precision at any exponent, and values as large as 2^100 are not carried past float32.
            bool look = i == 0;
            auto reference = [&](float most) {
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
                return most == -INFINITY ? 0.f : most;  // (nothing seen)
            };
            for (bool again = true; again;) {
                again = false;
                float most[NT][2];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    add[n][0] = add[n][1] = 0.f;
                    most[n][0] = most[n][1] = -INFINITY;
                }
#pragma unroll
                for (int s0 = 0; s0 < 4; s0 += kTogether) {
                    float cs[kTogether][NT][4];
#pragma unroll
                    for (int s = s0; s < s0 + kTogether; ++s) {
                        float (&c)[NT][4] = cs[s - s0];
#pragma unroll
                        for (int n = 0; n < NT; ++n) c[n][0] = c[n][1] = c[n][2] = c[n][3] = step && 2 * s >= left ? -INFINITY : 0.f;
                        if (step && 2 * s >= left) continue;  // none of the step's tokens is in this one
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
                                const uint32_t sc = __byte_perm(k_scale[r][s], 0, half), of = __byte_perm(k_offset[r][s], 0, half);
#pragma unroll
                                for (int i2 = 0; i2 < kWords; ++i2)
#pragma unroll
                                    for (int e = 0; e < 4; ++e) k[r][4 * i2 + e] = q4::fma_bf16x2(q4::open_pair(w[i2], e, mask, ones), sc, of);
                            }
                        } else {
#pragma unroll
                            for (int i2 = 0; i2 < D / 8; ++i2) k[1][i2] = 0;  // (tokens from 32 on: there are none)
                            {
                                constexpr int r = 0;
                                const int a = k_token + 2 * s;
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
                        for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
                            for (int n = 0; n < NT; ++n)
                                mma_16816(c[n], k[0][2 * ks], k[1][2 * ks], k[0][2 * ks + 1], k[1][2 * ks + 1], qf[n][2 * ks], qf[n][2 * ks + 1]);
                        // tokens that are not there, or not seen: -infinity
                        if (step || left < kChunk) {
                            asm volatile("" ::: "memory");  // a branch
#pragma unroll
                            for (int r = 0; r < 2; ++r) {
                                const int a = k_token + 32 * r + 2 * s;
#pragma unroll
                                for (int n = 0; n < NT; ++n)
#pragma unroll
                                    for (int e = 0; e < 2; ++e) {
                                        bool seen = a < left;
                                        if constexpr (step) seen = seen && (step_sees[n][e] >> (a & 31) & 1);  // (left is at most 16)
                                        if (!seen) c[n][2 * r + e] = -INFINITY;
                                    }
                            }
                        }
                    }
                    float top = -INFINITY, rounded[NT][2];  // the rows' largest rounded scores
                    if constexpr (coarse) {
#pragma unroll
                        for (int n = 0; n < NT; ++n) rounded[n][0] = rounded[n][1] = -INFINITY;
                    }
#pragma unroll
                    for (int s = 0; s < kTogether; ++s)
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                if constexpr (coarse) {
                                    cs[s][n][e] = __fmul_rn(cs[s][n][e], scale);
                                    rounded[n][e & 1] = fmaxf(rounded[n][e & 1], cs[s][n][e]);
                                    cs[s][n][e] = __fsub_rn(cs[s][n][e], m[n][e & 1]);
                                } else {
                                    cs[s][n][e] = fmaf(cs[s][n][e], scale, -m[n][e & 1]);
                                }
                                top = fmaxf(top, cs[s][n][e]);
                            }
                    if (look) {
#pragma unroll
                        for (int s = 0; s < kTogether; ++s)
#pragma unroll
                            for (int n = 0; n < NT; ++n)
#pragma unroll
                                for (int e = 0; e < 4; ++e) most[n][e & 1] = fmaxf(most[n][e & 1], cs[s][n][e]);
                        if constexpr (kTogether < 4) {
                            continue;
                        } else {  // the whole chunk is here: no second pass
#pragma unroll
                            for (int n = 0; n < NT; ++n)
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    m[n][e] = reference(most[n][e]);
#pragma unroll
                                    for (int s = 0; s < kTogether; ++s) {
                                        cs[s][n][e] -= m[n][e];
                                        cs[s][n][e + 2] -= m[n][e];
                                    }
                                }
                            if (!coarse && any_coarse(m)) return kTooCoarse;
                            look = false;
                        }
                    } else if (__any_sync(0xffffffffu, top > kRaise)) {
                        // references rise to the largest of these tokens; sums and accumulators follow, and the chunk starts over
                        float risen[NT][2];
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                float rise = coarse ? rounded[n][e] : 0.f;
                                if constexpr (!coarse) {
#pragma unroll
                                    for (int s = 0; s < kTogether; ++s) rise = fmaxf(rise, fmaxf(cs[s][n][e], cs[s][n][e + 2]));
                                }
#pragma unroll
                                for (int o = 4; o < 32; o <<= 1) rise = fmaxf(rise, __shfl_xor_sync(0xffffffffu, rise, o));
                                risen[n][e] = coarse ? fmaxf(m[n][e], rise) : m[n][e] + rise;
                            }
                        if (!coarse && any_coarse(risen)) return kTooCoarse;
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const float factor = ex2(m[n][e] - risen[n][e]);
                                m[n][e] = risen[n][e];
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
                    for (int s = 0; s < kTogether; ++s)
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            float (&c)[4] = cs[s][n];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                c[e] = ex2(c[e]);
                                add[n][e & 1] += c[e];
                            }
                            pf[s0 + s][n][0] = transposed(pack_bf16(c[0], c[1]));
                            pf[s0 + s][n][1] = transposed(pack_bf16(c[2], c[3]));
                        }
                }
                if (look) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e) m[n][e] = reference(most[n][e]);
                    if (!coarse && any_coarse(m)) return kTooCoarse;
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
                        uint4 v = make_uint4(0, 0, 0, 0);  // (tokens 8 t .. of the first 32; there are at most 16)
                        if (j < 2 && t < 2) v = lds16(step_v + (t * D + 16 * d + g + 8 * j) * 16);
                        a[j][0] = v.x; a[j][1] = v.y; a[j][2] = v.z; a[j][3] = v.w;
                    }
                }
#pragma unroll
                for (int s = 0; s < 4; ++s)
                    if (!step || 2 * s < left) {
#pragma unroll
                        for (int n = 0; n < NT; ++n) mma_16816(acc[d][n], a[0][s], a[1][s], a[2][s], a[3][s], pf[s][n][0], pf[s][n][1]);
                    }
            }
            __syncwarp();
            if (!step) {
                copy(i + kStages, next_entry);
                next_entry = entry_of(i + kStages + 1);
            }
            return kDone;
        };
        int i = 0;
        Outcome outcome = kDone;
        auto walk = [&](auto is_coarse) {
#pragma unroll 1
            for (; warp + i * kWarps < n_ctx; ++i)
                if ((outcome = work(std::false_type(), is_coarse, i)) != kDone) return;
            if (warp + i * kWarps < n_chunks) outcome = work(std::true_type(), is_coarse, i);
        };
        walk(std::false_type());
        if (outcome == kTooCoarse) {  // from this chunk on; a first one is looked at anew
            if (i == 0)
#pragma unroll
                for (int n = 0; n < NT; ++n) m[n][0] = m[n][1] = 0.f;
            walk(std::true_type());
        }
        fills = fills0 + i;

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
            const int r = i / D, c = i % D, j = r / p.G;
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
            const size_t to = (((size_t)lb * p.Hkv + h) * p.n_slots + part) * ((size_t)p.M_max * p.G) + r;
            p.part_o[to * D + c] = o;
            if (c == 0) {
                // nothing seen: -infinity; a NaN has to survive the merge, which leaves out what weighs nothing
                p.part_ml[to * 2] = total == 0.f ? -INFINITY : total != total ? INFINITY : s_top[r];
                p.part_ml[to * 2 + 1] = total;
            }
        }
        if (last)  // slots that no CTA fills
            for (int i = threadIdx.x; i < (p.n_slots - n_parts) * rows; i += kThreads) {
                const size_t to = (((size_t)lb * p.Hkv + h) * p.n_slots + n_parts + i / rows) * ((size_t)p.M_max * p.G) + i % rows;
                p.part_ml[to * 2] = -INFINITY;
                p.part_ml[to * 2 + 1] = 0.f;
            }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // before copies into where the warps met
        __syncthreads();
        if (last) {
            if (threadIdx.x == 0) odd = 0;
            __syncthreads();
        }
        if (abort_flag) break;
    }
    pdl_trigger();
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
    p.block_table = a.block_table; p.seq_lens = a.seq_lens; p.workspace = a.workspace;
    p.layer0 = a.layer0; p.batch = a.batch; p.M_max = a.M_max; p.mask_words = a.mask_words; p.Hq = a.g.Hq; p.Hkv = a.g.Hkv; p.G = a.g.G;
    p.bs = a.g.bs; p.bs_log2 = a.g.bs == 16 ? 4 : a.g.bs == 32 ? 5 : 6;
    p.max_blocks = a.max_blocks; p.n_pages = a.n_pages; p.n_layers = a.n_layers;
    p.scale_log2 = a.g.scale * kLog2e;
    p.q4_mask = q4::kMask; p.q4_ones = q4::kOnes;
    const int R_max = a.M_max * a.g.G, units = a.g.Hkv * a.n_layers * a.batch;
    const int positions = (a.max_seq_len + kChunk - 1) / kChunk + 1;
    if ((long long)units * positions >= 1LL << 30) return SPECPV_ERR_CAPACITY;
    // One CTA per SM, each with at least a chunk for every warp, or, for one sequence, for every scheduler of the SM (2047 tokens, one
    // layer, 4 rows 10.7 -> 10.1 us; two sequences of 1000 and 3000 tokens, whose shares then meet more units, 16.2 -> 16.8).  Where the units are alike a number of CTAs that the units divide
    // makes shares that lie in one unit each; else every SM has the same to do, but a unit more or two to begin and end, 4 us each.
    // (A position takes some 0.29 us, 0.45 with 16 rows.)
    const int warps = R_max <= 8 ? 12 : 8;
    const double us = R_max <= 8 ? 0.29 : 0.45, begin_us = 4.0;
    const int least = a.batch == 1 ? 4 : warps, most = (positions + least - 1) / least;  // CTAs of a unit
    long long n_ctas = (long long)units * most < 148 ? (long long)units * most : 148;
    if (a.batch == 1 && units <= 148) {
        const int k = 148 / units < most ? 148 / units : most;
        const double together = (double)units * positions / n_ctas * us + begin_us * (2.0 + (double)units / n_ctas), apart = (double)positions / k * us + begin_us;
        if (apart <= together) n_ctas = (long long)units * k;
    }
    const long long all = (long long)units * positions;
    const size_t slot_bytes = (size_t)units * R_max * (a.g.d + 2) * sizeof(float);
    const long long share = all / n_ctas > 1 ? all / n_ctas : 1;
    long long slots = (positions + share - 1) / share + 1;
    if (a.batch > 1) slots = slots * 2;  // shorter sequences leave more CTAs to a longer one
    if (slots > 64) slots = 64;
    if (slots > (long long)(a.partial_bytes / slot_bytes)) slots = (long long)(a.partial_bytes / slot_bytes);
    if (slots < 2) return SPECPV_ERR_CAPACITY;
    p.n_slots = (int)slots;
    char* ws = reinterpret_cast<char*>(a.workspace) + a.partial_off;
    p.part_o = reinterpret_cast<float*>(ws);
    p.part_ml = reinterpret_cast<float*>(ws + (size_t)units * slots * R_max * a.g.d * sizeof(float));
    const bool one = R_max <= 8;
    const auto launch = a.g.d == 64 ? (one ? launch_rows_form<64, 1> : launch_rows_form<64, 2>) : (one ? launch_rows_form<128, 1> : launch_rows_form<128, 2>);
    const specpv_status st = launch(p, (int)n_ctas, stream);
    return st != SPECPV_OK ? st : launch_merge_splits(a, p.n_slots, p.part_o, p.part_ml, stream);
}

}  // namespace specpv
