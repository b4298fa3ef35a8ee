// Eviction by accumulated attention weight: the account of the weight that every cached token has received, and the eviction of the
// tokens with the smallest accounts, after which the others close up.
#include <math.h>

#include <type_traits>

#include "aux_kernels.cuh"
#include "tc_common.cuh"

namespace specpv {

namespace {

// ---------------------------------------------------------------------------------------------
// Account: acc[t] += sum over the accepted rows i and the query heads g of the KV head of exp(scale q_ig . k_t - lse_ig), for the
// tokens t that row i sees.  The keys are read once, at the rate of the memory (that is the bound), straight into the registers that
// the warp-wide matrix instruction takes them from: a warp owns 16 tokens at a time, S^T [16 tokens x 8 rows] = K Q^T.  The sum over
// channels may be taken in any order, so lane (g, t) keeps the 16 bytes at 16 (4 j + t) of tokens g and g + 8 as they come.  The
// rows' queries wait in shared memory in the same order, 16 bytes a lane.  The instruction truncates its sums, so that it sums over 32
// channels only and the rest is added in float32: the weights of 5000 tokens, 16 rows x 4 are off by 5.4e-7 and 6.8e-7 of themselves (64 and 128
// channels; 5.9e-7 and 9.9e-7 with two chains over half the channels each).
// (98309 tokens x 8 heads x 12 layers, 28 rows: 522 us a pass, 0.73 of the copy rate; 505 with the longer chains, a third more than 522 with 16
// channels to a sum.)
// float32: both factors as two terms of 11 bits, three products (m16n8k8), which leaves 2^-21 of a product, summed by the instruction
// over 16 channels only (1.5e-6 of a weight was lost with one chain of 128 channels, 0.9e-6 now); bound by forming the
// terms and by the products (4261 tokens x 8 heads x 8 layers, 20 rows 77 us, 21 for its bytes; with terms formed per row tile and every
// element tested for infinity 145).  A token's sum over the rows is formed in a fixed order: the same at every run.
// ---------------------------------------------------------------------------------------------
constexpr int kAccWarps = 8;
constexpr int kAccTokens = 16;      // of a warp at a time
constexpr int kAccPassRows = 128;   // rows per launch; more rows take several
constexpr int kSharers = 3;         // row tiles that share a tile's terms (float32)

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_tf32(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ bool is_odd(uint32_t x) { return (x & 0x7F800000u) == 0x7F800000u; }  // infinite or NaN
// x as two terms of 11 bits.  With kCareful an infinity or NaN is the first alone, and what the other factor's second term meets is
// then 0 (met_by_rest): its products are those with the other's first term, which has the sign and is zero only where the factor is.
template <bool kCareful>
__device__ __forceinline__ void two_terms(uint32_t x, uint32_t& hi, uint32_t& lo) {
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(hi) : "f"(__uint_as_float(x)));
    const float rest = __uint_as_float(x) - __uint_as_float(hi);
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(lo) : "f"(rest));
    if (kCareful && is_odd(x)) {
        hi = x;
        lo = 0;
    }
}
template <bool kCareful>
__device__ __forceinline__ uint32_t met_by_rest(uint32_t hi) { return kCareful && is_odd(hi) ? 0u : hi; }

template <typename T, int D>
__global__ void __launch_bounds__(32 * kAccWarps) accumulate_kernel(AccumulateParams p) {
    pdl_begin(p.pdl);
    constexpr int kPieces = D * (int)sizeof(T) / 64;  // 16-byte pieces of a token per lane
    constexpr bool kF32 = sizeof(T) == 4;
    extern __shared__ __align__(16) unsigned char acc_smem[];
    const int h = blockIdx.y, lb = blockIdx.z, b = lb % p.batch, l = lb / p.batch;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int seq_len = min(max(p.seq_lens[b], 0), p.max_blocks * p.bs);
    const int n = min(max(p.n_accepted[b], 0), p.A_max);
    const int n_tiles = (seq_len + kAccTokens - 1) / kAccTokens;
    const int tile0 = blockIdx.x * p.tiles_per_cta, tile1 = min(tile0 + p.tiles_per_cta, n_tiles);
    const int rows = min(p.row1, n * p.G) - p.row0, row_tiles = (rows + 7) / 8;
    if (tile0 >= tile1 || rows <= 0) return;
    constexpr int kTerms = kF32 ? 2 : 1;
    uint4* s_q = reinterpret_cast<uint4*>(acc_smem);  // [term][row tile][piece][lane]
    const int term_stride = row_tiles * kPieces * 32;
    float* s_lse = reinterpret_cast<float*>(s_q + kTerms * term_stride);  // [row], in the unit of the products; [row], what that lost
    int* s_end = reinterpret_cast<int*>(s_lse + 2 * row_tiles * 8);  // tokens that the row sees: none, if it adds nothing
    __shared__ uint32_t s_idle;  // bit per row tile: such rows are among it
    __shared__ int s_odd;        // a query's element is infinite or NaN (float32)
    static_assert(kAccPassRows / 8 <= 32, "a bit per row tile");
    const float scale = p.scale * 1.4426950408889634f;
    if (threadIdx.x == 0) s_idle = s_odd = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < row_tiles * 8; i += 32 * kAccWarps) {
        const int r = p.row0 + i, a = r / p.G;
        float lse = 0.f, rest = 0.f;
        int row = -1, end = -1;
        if (i < rows) {
            row = p.accepted ? p.accepted[(size_t)b * p.A_max + a] : a;
            if (row < 0 || row >= p.M_max) {
                if (h == 0 && blockIdx.x == 0 && r % p.G == 0) record_fault(p.workspace, SPECPV_ERR_INVALID_ARG, b, a, row, l);
                row = -1;
            } else {
                const float natural = p.lse[((size_t)lb * p.M_max + row) * p.Hq + h * p.G + r % p.G];
                if (natural != -INFINITY) {
                    lse = natural / p.scale;
                    if (isfinite(lse)) {
                        rest = (float)(((double)lse - (double)natural / (double)p.scale) * (double)scale);
                    } else {  // a scale too small for the quotient, or no number
                        lse = 0.f;
                        rest = -natural * 1.4426950408889634f;
                    }
                    end = seq_len - n + a + 1;
                }
            }
        }
        if (end < 0) atomicOr(&s_idle, 1u << (i >> 3));
        s_lse[i] = lse;
        s_lse[row_tiles * 8 + i] = rest;
        s_end[i] = end;
        const uint4* src = reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(p.q) + (((size_t)lb * p.M_max + max(row, 0)) * p.Hq + h * p.G + r % p.G) * D);
#pragma unroll
        for (int j = 0; j < kPieces; ++j)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                uint4 v = row < 0 ? make_uint4(0, 0, 0, 0) : src[j * 4 + x], rest;
                uint4* to = s_q + ((i >> 3) * kPieces + j) * 32 + (i & 7) * 4 + x;
                if constexpr (kF32) {
                    if (is_odd(v.x) || is_odd(v.y) || is_odd(v.z) || is_odd(v.w)) s_odd = 1;
                    two_terms<true>(v.x, v.x, rest.x);
                    two_terms<true>(v.y, v.y, rest.y);
                    two_terms<true>(v.z, v.z, rest.z);
                    two_terms<true>(v.w, v.w, rest.w);
                    to[term_stride] = rest;
                }
                *to = v;
            }
    }
    __syncthreads();
    const uint32_t idle = s_idle;
    const uint4* k_pool = reinterpret_cast<const uint4*>(p.k_pool) + ((size_t)(p.layer0 + l) * p.n_pages * p.Hkv + h) * p.bs * (D * sizeof(T) / 16);
    const size_t page_stride = (size_t)p.Hkv * p.bs * (D * sizeof(T) / 16);
    const int32_t* table = p.block_table + (size_t)b * p.max_blocks;
    float* acc = p.acc + (((size_t)(p.layer0 + l) * p.batch + b) * p.Hkv + h) * (size_t)p.max_blocks * p.bs;
    // tiles of 16 tokens divide a page (of 16, 32 or 64): page and place by shifts
    auto entry_of = [&](int tile) { return tile < tile1 ? table[tile >> p.tiles_log2] : -1; };
    auto fetch = [&](int tile, int page, uint4 (&x)[2][kPieces]) {  // keys of tokens g and g + 8; whether they are there
        if (tile >= tile1) return false;
        if (page < 0 || page >= p.n_pages) {
            if (lane == 0) record_fault(p.workspace, SPECPV_ERR_BAD_BLOCK_TABLE, b, tile >> p.tiles_log2, page, l);
            return false;
        }
        const int at = (tile & ((1 << p.tiles_log2) - 1)) * kAccTokens + g;
        const uint4* src = k_pool + page * page_stride + at * (int)(D * sizeof(T) / 16) + t;
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int j = 0; j < kPieces; ++j) x[r][j] = src[r * 8 * (D * sizeof(T) / 16) + j * 4];
        return true;
    };
    int tile = tile0 + warp;
    uint4 buf[2][2][kPieces];
    bool there = fetch(tile, entry_of(tile), buf[0]);
    int entry = entry_of(tile + kAccWarps);
    // `now` holds the tile's keys, `next` receives those of the warp's next tile meanwhile
    auto work = [&](const uint4 (&now)[2][kPieces], uint4 (&next)[2][kPieces]) {
        const int token = tile * kAccTokens + g;
        float* mine = acc + token + 8 * t;  // of lanes t = 0 and 1
        const bool writes = there && t < 2 && token + 8 * t < seq_len;
        const float before = writes ? *mine : 0.f;
        there = fetch(tile + kAccWarps, entry, next);
        entry = entry_of(tile + 2 * kAccWarps);
        const bool all_seen = (tile + 1) * kAccTokens <= seq_len - n;
        float sum[2] = {0.f, 0.f};
        auto weigh = [&](int rt, const float (&c)[4]) {
            const float2 lse = *reinterpret_cast<const float2*>(s_lse + rt * 8 + 2 * t);
            // the difference first: where a weight counts it is small, and so then is what the factor's rounding takes from it
            const float2 rest = *reinterpret_cast<const float2*>(s_lse + (row_tiles + rt) * 8 + 2 * t);
            float w[4] = {tc::ex2(fmaf(c[0] - lse.x, scale, rest.x)), tc::ex2(fmaf(c[1] - lse.y, scale, rest.y)),
                          tc::ex2(fmaf(c[2] - lse.x, scale, rest.x)), tc::ex2(fmaf(c[3] - lse.y, scale, rest.y))};
            if (!all_seen || (idle >> rt & 1)) {  // (by choice, not by a weight of 0: the key may be infinite)
                const int2 end = *reinterpret_cast<const int2*>(s_end + rt * 8 + 2 * t);
                if (token >= end.x) w[0] = 0.f;
                if (token >= end.y) w[1] = 0.f;
                if (token + 8 >= end.x) w[2] = 0.f;
                if (token + 8 >= end.y) w[3] = 0.f;
            }
            sum[0] += w[0] + w[1];
            sum[1] += w[2] + w[3];
        };
        if constexpr (!kF32) {
#pragma unroll 1
            for (int rt = 0; rt < row_tiles; ++rt) {
                float c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < kPieces; ++j) {
                    const uint4 q = s_q[(rt * kPieces + j) * 32 + lane];
                    float part[4] = {0.f, 0.f, 0.f, 0.f};  // of 32 channels
                    mma_bf16(part, now[0][j].x, now[1][j].x, now[0][j].y, now[1][j].y, q.x, q.y);
                    mma_bf16(part, now[0][j].z, now[1][j].z, now[0][j].w, now[1][j].w, q.z, q.w);
#pragma unroll
                    for (int e = 0; e < 4; ++e) c[e] += part[e];
                }
                weigh(rt, c);
            }
        } else {
            auto products = [&](auto careful) {
                constexpr bool kCareful = decltype(careful)::value;
#pragma unroll 1
                for (int rt0 = 0; rt0 < row_tiles; rt0 += kSharers) {  // the keys' terms are formed once for these
                    float c[kSharers][4], c1[kSharers][4];
#pragma unroll
                    for (int u = 0; u < kSharers; ++u)
#pragma unroll
                        for (int e = 0; e < 4; ++e) c[u][e] = c1[u][e] = 0.f;
#pragma unroll
                    for (int j = 0; j < kPieces; ++j) {
                        const uint32_t k0[4] = {now[0][j].x, now[0][j].y, now[0][j].z, now[0][j].w}, k1[4] = {now[1][j].x, now[1][j].y, now[1][j].z, now[1][j].w};
                        uint32_t hi[2][4], rest[2][4], met[2][4];
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            two_terms<kCareful>(k0[x], hi[0][x], rest[0][x]);
                            two_terms<kCareful>(k1[x], hi[1][x], rest[1][x]);
                            met[0][x] = met_by_rest<kCareful>(hi[0][x]);
                            met[1][x] = met_by_rest<kCareful>(hi[1][x]);
                        }
#pragma unroll
                        for (int u = 0; u < kSharers; ++u) {
                            if (rt0 + u >= row_tiles) break;
                            const uint4* at = s_q + ((rt0 + u) * kPieces + j) * 32 + lane;
                            const uint4 qh = at[0], ql = at[term_stride];
                            const uint4 qm = make_uint4(met_by_rest<kCareful>(qh.x), met_by_rest<kCareful>(qh.y), met_by_rest<kCareful>(qh.z), met_by_rest<kCareful>(qh.w));
                            float part[4] = {0.f, 0.f, 0.f, 0.f};
                            mma_tf32(c1[u], rest[0][0], rest[1][0], rest[0][1], rest[1][1], qm.x, qm.y);
                            mma_tf32(part, hi[0][0], hi[1][0], hi[0][1], hi[1][1], qh.x, qh.y);
                            mma_tf32(c1[u], met[0][0], met[1][0], met[0][1], met[1][1], ql.x, ql.y);
                            mma_tf32(part, hi[0][2], hi[1][2], hi[0][3], hi[1][3], qh.z, qh.w);
#pragma unroll
                            for (int e = 0; e < 4; ++e) c[u][e] += part[e];
                            mma_tf32(c1[u], rest[0][2], rest[1][2], rest[0][3], rest[1][3], qm.z, qm.w);
                            mma_tf32(c1[u], met[0][2], met[1][2], met[0][3], met[1][3], ql.z, ql.w);
                        }
                    }
#pragma unroll
                    for (int u = 0; u < kSharers; ++u) {
                        if (rt0 + u >= row_tiles) break;
#pragma unroll
                        for (int e = 0; e < 4; ++e) c[u][e] += c1[u][e];
                        weigh(rt0 + u, c[u]);
                    }
                }
            };
            float z = 0.f;  // NaN if one of the keys' elements is infinite or NaN
#pragma unroll
            for (int j = 0; j < kPieces; ++j)
#pragma unroll
                for (int r = 0; r < 2; ++r)
                    z = fmaf(__uint_as_float(now[r][j].x), 0.f, fmaf(__uint_as_float(now[r][j].y), 0.f, fmaf(__uint_as_float(now[r][j].z), 0.f, fmaf(__uint_as_float(now[r][j].w), 0.f, z))));
            if (__any_sync(0xffffffffu, z != z) || s_odd)
                products(std::true_type());
            else
                products(std::false_type());
        }
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
            sum[0] += __shfl_xor_sync(0xffffffffu, sum[0], o);
            sum[1] += __shfl_xor_sync(0xffffffffu, sum[1], o);
        }
        if (writes) *mine = before + (t ? sum[1] : sum[0]);
        tile += kAccWarps;
    };
#pragma unroll 1
    while (tile < tile1) {
        work(buf[0], buf[1]);
        if (tile >= tile1) break;
        work(buf[1], buf[0]);
    }
}

// ---------------------------------------------------------------------------------------------
// Close-up: rank j of a KV head's kept tokens (ascending, so idx[j] >= j) moves to place j, in place.  A unit is the keys, the values or
// the accounts of one (layer, sequence, KV head).  Keys and values are worked through in rounds of ranks, by a cluster of CTAs side by
// side: a round is read whole before any of it is written (a cluster barrier between), and then nothing is overwritten that is still to
// be read, because place j, as a source, belongs to a rank <= j.  For the same reason the next round's rows are requested before this
// one's are written; where they are is known by then: one thread per row has asked for its index three rounds ahead and for the
// table entries two ahead, so that no request waits for another.  Rows that stay are neither read nor written.  Bound by memory: every
// moved row is read and written once (4096 of 4352 tokens, 8 heads x 32 layers: 224 us with the selection, 0.74 of the copy rate; with
// each round's look-ups behind the round before 436).  grid = (cluster x 3 KV heads, layers x seqs).
// ---------------------------------------------------------------------------------------------
constexpr int kCloseThreads = 256;
constexpr int kCloseLoads = 8;  // 16-byte loads in flight per thread and round
constexpr int kAccLoads = 16;   // accounts per thread and round
constexpr uint32_t kNoRow = 0xFFFFFFFFu;

__global__ void __launch_bounds__(kCloseThreads, 2) close_up_kernel(EvictParams p) {
    asm volatile("griddepcontrol.launch_dependents;\n\tgriddepcontrol.wait;" ::: "memory");
    __shared__ uint2 s_rows[2][kCloseThreads];  // from, to; of the rounds of either parity
    uint32_t rank, n_ctas;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n_ctas));
    const int unit = blockIdx.x / n_ctas, h = unit % p.Hkv, kind = unit / p.Hkv;  // 0 keys, 1 values, 2 accounts
    const int lb = blockIdx.y, b = lb % p.batch, l = lb / p.batch, tid = threadIdx.x;
    const int capacity = p.max_blocks * p.bs, seq_len = min(max(p.seq_lens[b], 0), capacity);
    if (seq_len <= p.keep) return;  // (the whole cluster)
    const int32_t* idx = p.idx + (((size_t)l * p.batch + b) * p.Hkv + h) * p.keep;
    const int32_t* table = p.block_table + (size_t)b * p.max_blocks;
    const int first = p.sink;  // the ranks before it stay
    if (kind == 2) {
        if (rank) return;  // (no cluster barrier on this path)
        float* acc = p.acc + (((size_t)l * p.batch + b) * p.Hkv + h) * (size_t)capacity;
        for (int j0 = first; j0 < p.keep; j0 += kCloseThreads * kAccLoads) {
            float a[kAccLoads];
#pragma unroll
            for (int u = 0; u < kAccLoads; ++u) {
                const int j = j0 + u * kCloseThreads + tid;
                a[u] = j < p.keep ? acc[idx[j]] : 0.f;
            }
            __syncthreads();
#pragma unroll
            for (int u = 0; u < kAccLoads; ++u) {
                const int j = j0 + u * kCloseThreads + tid;
                if (j < p.keep) acc[j] = a[u];
            }
        }
        __syncthreads();
        for (int j = p.keep + tid; j < seq_len; j += kCloseThreads) acc[j] = 0.f;  // the accounts of the tokens to come
        return;
    }
    uint4* pool = reinterpret_cast<uint4*>(kind ? p.v_pool : p.k_pool);
    const int chunks = p.row_bytes / 16, step = kCloseThreads / chunks;  // 16-byte pieces of a row, rows side by side
    const int piece = tid % chunks, lane_row = tid / chunks, per_cta = step * kCloseLoads, per_round = per_cta * (int)n_ctas;
    const uint32_t row0 = ((uint32_t)l * p.n_pages * p.Hkv + h) * p.bs, page_rows = (uint32_t)p.Hkv * p.bs;
    // a thread's row of a round: rank j, -1 where there is none
    auto rank_of = [&](int round) {
        const int j = first + round * per_round + (int)rank * per_cta + tid;
        return tid < per_cta && j < p.keep ? j : -1;
    };
    auto index_of = [&](int round) {
        const int j = rank_of(round);
        return j >= 0 ? idx[j] : -1;
    };
    struct Pages { int from, to; };
    auto pages_of = [&](int round, int token) {
        const int j = rank_of(round);
        Pages e{0, 0};
        if (j >= 0) {
            e.from = table[token / p.bs];
            e.to = table[j / p.bs];
        }
        return e;
    };
    auto publish = [&](int round, int token, Pages e) {  // where the row goes from and to
        const int j = rank_of(round);
        uint2 r = make_uint2(kNoRow, kNoRow);
        if (j >= 0 && j != token) {
            const bool from_ok = e.from >= 0 && e.from < p.n_pages, to_ok = e.to >= 0 && e.to < p.n_pages;
            if (from_ok && to_ok)
                r = make_uint2(row0 + (uint32_t)e.from * page_rows + token % p.bs, row0 + (uint32_t)e.to * page_rows + j % p.bs);
            else
                record_fault(p.workspace, SPECPV_ERR_BAD_BLOCK_TABLE, b, (from_ok ? j : token) / p.bs, from_ok ? e.to : e.from, l);
        }
        s_rows[round & 1][tid] = r;
    };
    uint32_t to[kCloseLoads];
    uint4 buf[2][kCloseLoads];
    auto load = [&](int round, uint4 (&x)[kCloseLoads]) {
#pragma unroll
        for (int u = 0; u < kCloseLoads; ++u) {
            const uint2 r = s_rows[round & 1][u * step + lane_row];
            to[u] = r.y;
            if (r.x != kNoRow) x[u] = pool[(size_t)r.x * chunks + piece];
        }
    };
    const int n_rounds = (p.keep - first + per_round - 1) / per_round;
    // three rounds of look-ups under way
    const int t0 = index_of(0), t1 = index_of(1);
    int token2 = index_of(2), token3 = index_of(3);
    const Pages e0 = pages_of(0, t0), e1 = pages_of(1, t1);
    Pages pages2 = pages_of(2, token2);
    publish(0, t0, e0);
    publish(1, t1, e1);
    __syncthreads();
    load(0, buf[0]);
    __syncthreads();  // every thread has taken round 0's rows: round 2's come to their place
    auto round = [&](int i, uint4 (&now)[kCloseLoads], uint4 (&next)[kCloseLoads]) {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");  // this round's rows have been read
        uint32_t dst[kCloseLoads];
#pragma unroll
        for (int u = 0; u < kCloseLoads; ++u) dst[u] = to[u];
        load(i + 1, next);
        publish(i + 2, token2, pages2);  // (every thread has taken round i's rows from this place: the barrier below, of the round before, or the one above)
        pages2 = pages_of(i + 3, token3);
        token2 = token3;
        token3 = index_of(i + 4);
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
#pragma unroll
        for (int u = 0; u < kCloseLoads; ++u)
            if (dst[u] != kNoRow) pool[(size_t)dst[u] * chunks + piece] = now[u];
        __syncthreads();  // the rows of round i + 2 are there, those of round i + 1 taken
    };
    for (int i = 0; i < n_rounds; i += 2) {
        round(i, buf[0], buf[1]);
        if (i + 1 < n_rounds) round(i + 1, buf[1], buf[0]);
    }
}

constexpr int kLensThreads = 128;
__global__ void __launch_bounds__(kLensThreads) evict_lens_kernel(EvictParams p) {
    pdl_begin(p.pdl);
    const int b = blockIdx.x * kLensThreads + threadIdx.x;
    if (b < p.batch && p.seq_lens[b] > p.keep) p.seq_lens[b] = p.keep;
}

}  // namespace

#define SPECPV_LAUNCH(...)                                                     \
    do {                                                                       \
        if (launch_pdl_if(__VA_ARGS__) != cudaSuccess) return SPECPV_ERR_CUDA; \
        count_launch();                                                        \
    } while (0)

template <typename T, int D>
static specpv_status launch_accumulate_typed(AccumulateParams p, int n_layers, int max_seq_len, cudaStream_t stream) {
    // Tiles per warp: the waves of CTAs, two on an SM (counted so for float32 with 128 channels as well, of which one fits), times what one takes,
    // of which a start is about two and a half tiles (32 layers x 8 heads x 4261 tokens, 20 rows: 73 us with 14 tiles per warp, 66 with the 17 chosen).
    const long long tiles = (max_seq_len + kAccTokens - 1) / kAccTokens, heads = (long long)p.Hkv * n_layers * p.batch;
    int per_warp = 1;
    double best = 1e300;
    for (int w = 1; w <= 48; ++w) {
        const long long ctas = heads * ((tiles + kAccWarps * w - 1) / (kAccWarps * w));
        const double cost = (double)((ctas + 2 * 148 - 1) / (2 * 148)) * (w + 2.5);
        if (cost < best) {
            best = cost;
            per_warp = w;
        }
    }
    p.tiles_per_cta = per_warp * kAccWarps;
    p.tiles_log2 = p.bs == 64 ? 2 : p.bs == 32 ? 1 : 0;
    const dim3 grid((unsigned)((tiles + p.tiles_per_cta - 1) / p.tiles_per_cta), p.Hkv, n_layers * p.batch);
    const int all_rows = p.A_max * p.G;
    for (p.row0 = 0; p.row0 < all_rows; p.row0 += kAccPassRows) {
        p.row1 = p.row0 + kAccPassRows;
        const int row_tiles = ((all_rows < p.row1 ? all_rows : p.row1) - p.row0 + 7) / 8;
        constexpr int kRowBytes = D * (int)sizeof(T) * (sizeof(T) == 4 ? 2 : 1) + 12;
        const size_t smem = (size_t)row_tiles * 8 * kRowBytes;
        if (!tc::set_smem_limit_once(reinterpret_cast<const void*>(accumulate_kernel<T, D>), kAccPassRows * kRowBytes)) return SPECPV_ERR_CUDA;
        SPECPV_LAUNCH((accumulate_kernel<T, D>), grid, 32 * kAccWarps, smem, stream, p);
    }
    return SPECPV_OK;
}

specpv_status launch_accumulate(const AccumulateParams& p, int n_layers, int max_seq_len, int dtype, int d, cudaStream_t stream) {
    if (max_seq_len <= 0) return SPECPV_OK;
    if (dtype == SPECPV_DTYPE_F32)
        return d == 64 ? launch_accumulate_typed<float, 64>(p, n_layers, max_seq_len, stream) : launch_accumulate_typed<float, 128>(p, n_layers, max_seq_len, stream);
    return d == 64 ? launch_accumulate_typed<__nv_bfloat16, 64>(p, n_layers, max_seq_len, stream) : launch_accumulate_typed<__nv_bfloat16, 128>(p, n_layers, max_seq_len, stream);
}

specpv_status launch_evict(const EvictParams& p, int n_layers, cudaStream_t stream) {
    // CTAs of a unit: enough to fill the SMs three times over
    const long long units = 2LL * p.Hkv * n_layers * p.batch;
    unsigned cluster = 1;
    while (cluster < 8 && units * cluster < 3 * 148) cluster *= 2;
    cudaLaunchAttribute attr[2]{};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(cluster * 3 * p.Hkv, n_layers * p.batch);
    cfg.blockDim = kCloseThreads;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, close_up_kernel, p) != cudaSuccess) return SPECPV_ERR_CUDA;
    count_launch();
    SPECPV_LAUNCH(evict_lens_kernel, dim3((p.batch + kLensThreads - 1) / kLensThreads), kLensThreads, 0, stream, p);
    return SPECPV_OK;
}

}  // namespace specpv
