// Keeping a cache in 4 bits (layout: q4.cuh): rows are quantised as they are appended (paper Section 3.2 / 3.3, the commit of a step's
// accepted tokens, or a chunk of the prefill), and selected blocks are opened into an ordinary partial cache (Section 3.3, "refresh the
// partial KV cache").
#include <math.h>

#include "aux_kernels.cuh"
#include "q4.cuh"

namespace specpv {

namespace {

// ---------------------------------------------------------------------------------------------
// Commit: a CTA owns one (layer, sequence, KV head, page touched), so that the words that old and new tokens share (a value's word is
// eight tokens of a channel) have one writer.  A warp quantises a row at a time: its lanes hold the channels, the smallest and
// largest are found by shuffles.  Key words are formed by shuffles among eight channels; value codes meet in shared memory, where a
// thread per channel puts eight tokens' codes together with those that the word held.  The page's summary is then taken from its
// codes, the new ones among them.  grid = (pages touched, KV heads, layers x seqs).
// ---------------------------------------------------------------------------------------------
constexpr int kCommitThreads = 256;
constexpr int kCommitWarps = kCommitThreads / 32;

template <typename T, int D>
__device__ __forceinline__ void load_row(const void* src, size_t row, int lane, float (&x)[D / 32]) {
    if constexpr (sizeof(T) == 4) {
        const float* p = reinterpret_cast<const float*>(src) + row * D + lane * (D / 32);
#pragma unroll
        for (int i = 0; i < D / 32; ++i) x[i] = p[i];
    } else {
        const uint32_t* p = reinterpret_cast<const uint32_t*>(reinterpret_cast<const __nv_bfloat16*>(src) + row * D + lane * (D / 32));
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
            const uint32_t w = p[i];
            x[2 * i] = q4::lower(w);
            x[2 * i + 1] = q4::upper(w);
        }
    }
}
template <typename T, int D>
__device__ __forceinline__ void store_values(void* dst, size_t row, int lane, const uint32_t (&codes)[D / 32], const q4::Row& r) {
    if (!dst) return;
    T* p = reinterpret_cast<T*>(dst) + row * D + lane * (D / 32);
#pragma unroll
    for (int i = 0; i < D / 32; i += 2) {
        const uint32_t v = q4::fma_bf16x2(0x41804180u | codes[i] << 3 | codes[i + 1] << 19, q4::twice(r.scale16), q4::twice(r.offset16));
        if constexpr (sizeof(T) == 4) {
            p[i] = q4::lower(v);
            p[i + 1] = q4::upper(v);
        } else {
            *reinterpret_cast<uint32_t*>(p + i) = v;
        }
    }
}

template <int D>
__device__ __forceinline__ q4::Row quantise_row(const float (&x)[D / 32], uint32_t (&codes)[D / 32]) {
    float lo = x[0], hi = x[0];
    bool finite = true;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        lo = fminf(lo, x[i]);
        hi = fmaxf(hi, x[i]);
        finite &= isfinite(x[i]);
    }
    asm volatile("redux.sync.min.f32 %0, %1, 0xffffffff;" : "=f"(lo) : "f"(lo));
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(hi) : "f"(hi));
    const q4::Row r = q4::row_of(lo, hi, __all_sync(0xffffffffu, finite));
    q4::codes_of(r, x, codes);
    return r;
}

template <typename T, int D>
__global__ void __launch_bounds__(kCommitThreads) commit_q4_kernel(CommitQ4Params p) {
    pdl_begin(p.pdl);
    constexpr int C = D / 32;              // channels per lane
    constexpr int kColumns = D / 8;        // key words per token
    constexpr int kTokenLanes = kCommitThreads / kColumns;
    __shared__ unsigned char s_v[64][D];   // value codes of the page's new tokens
    __shared__ float s_max[kTokenLanes][D + 4], s_min[kTokenLanes][D + 4];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int h = blockIdx.y, lb = blockIdx.z, b = lb % p.batch, l = lb / p.batch;
    const int n = min(max(p.n_accepted[b], 0), p.A_max), seq_len = max(p.seq_lens[b], 0);
    if ((size_t)seq_len + n > (size_t)p.max_blocks * p.bs) {
        if (threadIdx.x == 0 && blockIdx.x == 0 && h == 0 && n > 0) record_fault(p.workspace, SPECPV_ERR_CAPACITY, b, seq_len, n, l);
        return;
    }
    const int block = seq_len / p.bs + blockIdx.x, page_t0 = block * p.bs;
    const int t0 = max(seq_len, page_t0), t1 = min(seq_len + n, page_t0 + p.bs);  // tokens appended to this page
    if (t0 >= t1) return;
    const int page = p.block_table[(size_t)b * p.max_blocks + block];
    if (page < 0 || page >= p.n_pages) {
        if (threadIdx.x == 0) record_fault(p.workspace, SPECPV_ERR_BAD_BLOCK_TABLE, b, block, page, l);
        return;
    }
    unsigned char* base = reinterpret_cast<unsigned char*>(p.pool) +
                          (((size_t)(p.layer0 + l) * p.n_pages + page) * p.Hkv + h) * q4::page_bytes(p.bs, D);
    uint32_t* words = reinterpret_cast<uint32_t*>(base);
    uint16_t* params = reinterpret_cast<uint16_t*>(base);
    // the next token's rows are in flight while this one's are worked on
    float k_next[C], v_next[C];
    int row_next = -1;
    auto fetch = [&](int t) {
        if (t >= t1) return;
        const int a = t - seq_len;
        row_next = p.accepted ? p.accepted[(size_t)b * p.A_max + a] : a;
        if (row_next < 0 || row_next >= p.M_max) return;
        const size_t src = ((size_t)lb * p.M_max + row_next) * p.Hkv + h;
        load_row<T, D>(p.k_new, src, lane, k_next);
        load_row<T, D>(p.v_new, src, lane, v_next);
    };
    bool lost = false;
    fetch(t0 + warp);
    for (int t = t0 + warp; t < t1; t += kCommitWarps) {
        const int a = t - seq_len, row = row_next, at = t - page_t0;
        float k[C], v[C];
#pragma unroll
        for (int i = 0; i < C; ++i) {
            k[i] = k_next[i];
            v[i] = v_next[i];
        }
        fetch(t + kCommitWarps);
        if (row < 0 || row >= p.M_max) {  // the token keeps what its place held
            if (lane == 0) record_fault(p.workspace, SPECPV_ERR_INVALID_ARG, b, a, row, l);
#pragma unroll
            for (int i = 0; i < C; ++i) s_v[at][lane * C + i] = 0xFF;
            lost = true;
            continue;
        }
        const size_t out = ((size_t)lb * p.A_max + a) * p.Hkv + h;
        uint32_t kc[C], vc[C];
        const q4::Row kr = quantise_row<D>(k, kc), vr = quantise_row<D>(v, vc);
        store_values<T, D>(p.k_values, out, lane, kc, kr);
        store_values<T, D>(p.v_values, out, lane, vc, vr);
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            w |= kc[i] << q4::element_shift((lane * C + i) & 7);
            s_v[at][lane * C + i] = (unsigned char)vc[i];
        }
#pragma unroll
        for (int o = 1; o < 8 / C; o <<= 1) w |= __shfl_xor_sync(0xffffffffu, w, o);
        if (lane % (8 / C) == 0) words[q4::k_word(p.bs, at, lane * C)] = q4::rotated(w);
        if (lane < 4) {
            const uint16_t x = lane == 0 ? kr.scale16 : lane == 1 ? kr.offset16 : lane == 2 ? vr.scale16 : vr.offset16;
            params[q4::param_at(p.bs, D, lane, at)] = x;
        }
    }
    const bool skipped = __syncthreads_or(lost);
    // value words of the touched groups of eight tokens
    const int g0 = (t0 - page_t0) / 8, g1 = (t1 - 1 - page_t0) / 8;
    for (int i = threadIdx.x; i < (g1 - g0 + 1) * D; i += kCommitThreads) {
        const int g = g0 + i / D, c = i % D, at0 = g * 8;
        uint32_t* to = words + q4::v_word(p.bs, D, at0, c);
        const bool whole = page_t0 + at0 >= t0 && page_t0 + at0 + 8 <= t1 && !skipped;  // nothing of the old word stays
        uint32_t w = whole ? 0u : q4::unrotated(*to);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int t = page_t0 + at0 + e;
            if (t >= t0 && t < t1) {
                const uint32_t code = s_v[at0 + e][c];
                if (code < 16u) w = (w & ~(15u << q4::element_shift(e))) | code << q4::element_shift(e);
            }
        }
        *to = q4::rotated(w);
    }
    if (!p.kmax) return;
    // Eq. 1 over the page's tokens (their codes were written by this CTA or stood there): a thread takes eight channels of every
    // kTokenLanes-th token
    const int column = threadIdx.x % kColumns, tl = threadIdx.x / kColumns, n_valid = min(p.bs, seq_len + n - page_t0);
    float mx[8], mn[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        mx[e] = -INFINITY;
        mn[e] = INFINITY;
    }
    for (int t = tl; t < n_valid; t += kTokenLanes) {
        const uint32_t w = words[q4::k_word(p.bs, t, column * 8)];
        const uint32_t s = q4::twice(params[q4::param_at(p.bs, D, 0, t)]), o = q4::twice(params[q4::param_at(p.bs, D, 1, t)]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t v = q4::fma_bf16x2(q4::open_pair(w, i), s, o);
            mx[2 * i] = fmaxf(mx[2 * i], q4::lower(v));
            mn[2 * i] = fminf(mn[2 * i], q4::lower(v));
            mx[2 * i + 1] = fmaxf(mx[2 * i + 1], q4::upper(v));
            mn[2 * i + 1] = fminf(mn[2 * i + 1], q4::upper(v));
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        s_max[tl][column * 8 + e] = mx[e];
        s_min[tl][column * 8 + e] = mn[e];
    }
    __syncthreads();
    if ((int)threadIdx.x < D) {
        const int c = threadIdx.x;
        float a = s_max[0][c], z = s_min[0][c];
#pragma unroll
        for (int i = 1; i < kTokenLanes; ++i) {
            a = fmaxf(a, s_max[i][c]);
            z = fminf(z, s_min[i][c]);
        }
        const size_t o = ((((size_t)(p.layer0 + l) * p.batch + b) * p.Hkv + h) * p.max_blocks + block) * D + c;
        reinterpret_cast<T*>(p.kmax)[o] = from_float<T>(a);
        reinterpret_cast<T*>(p.kmin)[o] = from_float<T>(z);
    }
}

constexpr int kLensThreads = 128;
__global__ void __launch_bounds__(kLensThreads) commit_q4_lens_kernel(CommitQ4Params p) {
    pdl_begin(p.pdl);
    const int b = blockIdx.x * kLensThreads + threadIdx.x;
    if (b >= p.batch) return;
    const int n = min(max(p.n_accepted[b], 0), p.A_max), seq_len = max(p.seq_lens[b], 0);
    if ((size_t)seq_len + n <= (size_t)p.max_blocks * p.bs) p.seq_lens[b] = seq_len + n;
}

// ---------------------------------------------------------------------------------------------
// Gather: a CTA opens one selected block of a KV head into the partial cache.  A key word is 16 bytes of a bfloat16 row: lanes
// take the words of a row, and two rows' words are 32 bytes apart only by the 32 channels, so that both sides are full sectors.
// Values: a thread takes eight channels of 16 tokens (64 contiguous bytes) and stores 16 bytes of each of the 16 rows.
// grid = (budget blocks, KV heads, layers x seqs).
// ---------------------------------------------------------------------------------------------
constexpr int kGatherThreads = 128;

template <typename T>
__device__ __forceinline__ void store8(T* p, const uint32_t (&v)[4]) {  // eight elements, 16-byte aligned
    if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint4*>(p) = make_uint4(v[0], v[1], v[2], v[3]);
    } else {
        *reinterpret_cast<uint4*>(p) = make_uint4(v[0] << 16, v[0] & 0xFFFF0000u, v[1] << 16, v[1] & 0xFFFF0000u);
        *reinterpret_cast<uint4*>(p + 4) = make_uint4(v[2] << 16, v[2] & 0xFFFF0000u, v[3] << 16, v[3] & 0xFFFF0000u);
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(kGatherThreads) gather_q4_kernel(GatherQ4Params p) {
    pdl_begin(p.pdl);
    const int s = blockIdx.x, h = blockIdx.y, lb = blockIdx.z, b = lb % p.batch, l = lb / p.batch;
    const int count = p.count[b], seq_len = max(p.seq_lens[b], 0), nb = (seq_len + p.bs - 1) / p.bs;
    // the last selected block is the sequence's last block, of which the valid tokens are kept
    if (s == 0 && h == 0 && l == 0 && threadIdx.x == 0) p.partial_lens[b] = count > 0 ? (count - 1) * p.bs + (seq_len - (nb - 1) * p.bs) : 0;
    if (s >= count) return;
    const int block = p.idx[(((size_t)l * p.batch + b) * p.Hkv + h) * p.budget_blocks + s];
    if (block < 0 || block >= nb || block >= p.full_max_blocks || s >= p.part_max_blocks) {
        if (threadIdx.x == 0) record_fault(p.workspace, SPECPV_ERR_INVALID_ARG, b, s, block, l);
        return;
    }
    const int from = p.full_table[(size_t)b * p.full_max_blocks + block], to = p.part_table[(size_t)b * p.part_max_blocks + s];
    if (from < 0 || from >= p.full_pages || to < 0 || to >= p.part_pages) {
        if (threadIdx.x == 0) record_fault(p.workspace, SPECPV_ERR_BAD_BLOCK_TABLE, b, block, from, to);
        return;
    }
    const int n_valid = min(p.bs, seq_len - block * p.bs);
    const unsigned char* base = reinterpret_cast<const unsigned char*>(p.pool) + (((size_t)l * p.full_pages + from) * p.Hkv + h) * q4::page_bytes(p.bs, D);
    const uint32_t* words = reinterpret_cast<const uint32_t*>(base);
    const uint16_t* params = reinterpret_cast<const uint16_t*>(base);
    const size_t out = (((size_t)l * p.part_pages + to) * p.Hkv + h) * p.bs * D;
    T* k = reinterpret_cast<T*>(p.part_k) + out;
    T* v = reinterpret_cast<T*>(p.part_v) + out;
    constexpr int kBatch = 4;  // words in flight per thread
    for (int i0 = threadIdx.x; i0 < n_valid * (D / 8); i0 += kBatch * kGatherThreads) {
        uint32_t w[kBatch], scale[kBatch], offset[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int i = i0 + u * kGatherThreads, t = i / (D / 8), c = i % (D / 8) * 8;
            if (t < n_valid) {
                w[u] = words[q4::k_word(p.bs, t, c)];
                scale[u] = params[q4::param_at(p.bs, D, 0, t)];
                offset[u] = params[q4::param_at(p.bs, D, 1, t)];
            }
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int i = i0 + u * kGatherThreads, t = i / (D / 8), c = i % (D / 8) * 8;
            if (t >= n_valid) break;
            uint32_t x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = q4::fma_bf16x2(q4::open_pair(w[u], e), scale[u] * 0x10001u, offset[u] * 0x10001u);
            store8(k + (size_t)t * D + c, x);
        }
    }
    for (int i = threadIdx.x; i < p.bs / 16 * (D / 8); i += kGatherThreads) {
        const int t0 = i / (D / 8) * 16, c = i % (D / 8) * 8;
        if (t0 >= n_valid) break;
        uint32_t w[8][2];  // [channel][eight tokens]
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint4 x = *reinterpret_cast<const uint4*>(words + q4::v_word(p.bs, D, t0, c + 2 * j));
            w[2 * j][0] = x.x;
            w[2 * j][1] = x.y;
            w[2 * j + 1][0] = x.z;
            w[2 * j + 1][1] = x.w;
        }
        uint32_t scales[8], offsets[8];  // of pairs of tokens
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint4 x = *reinterpret_cast<const uint4*>(params + q4::param_at(p.bs, D, 2, t0 + 8 * j));
            const uint4 y = *reinterpret_cast<const uint4*>(params + q4::param_at(p.bs, D, 3, t0 + 8 * j));
            scales[4 * j] = x.x; scales[4 * j + 1] = x.y; scales[4 * j + 2] = x.z; scales[4 * j + 3] = x.w;
            offsets[4 * j] = y.x; offsets[4 * j + 1] = y.y; offsets[4 * j + 2] = y.z; offsets[4 * j + 3] = y.w;
        }
#pragma unroll
        for (int pair = 0; pair < 8; ++pair) {  // tokens t0 + 2 pair and the next
            const int t = t0 + 2 * pair;
            const uint32_t scale = scales[pair], offset = offsets[pair];
            uint32_t even[4], odd[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t a = q4::fma_bf16x2(q4::open_pair(w[2 * j][pair / 4], pair % 4), scale, offset);
                const uint32_t z = q4::fma_bf16x2(q4::open_pair(w[2 * j + 1][pair / 4], pair % 4), scale, offset);
                even[j] = __byte_perm(a, z, 0x5410);
                odd[j] = __byte_perm(a, z, 0x7632);
            }
            if (t < n_valid) store8(v + (size_t)t * D + c, even);
            if (t + 1 < n_valid) store8(v + (size_t)(t + 1) * D + c, odd);
        }
    }
}

}  // namespace

#define SPECPV_LAUNCH(...)                                                     \
    do {                                                                       \
        if (launch_pdl_if(__VA_ARGS__) != cudaSuccess) return SPECPV_ERR_CUDA; \
        count_launch();                                                        \
    } while (0)

specpv_status launch_commit_q4(const CommitQ4Params& p, int n_layers, int dtype, int d, bool advance, cudaStream_t stream) {
    const dim3 grid((p.A_max + p.bs - 1) / p.bs + 1, p.Hkv, n_layers * p.batch);
    if (dtype == SPECPV_DTYPE_F32)
        SPECPV_LAUNCH((d == 64 ? commit_q4_kernel<float, 64> : commit_q4_kernel<float, 128>), grid, kCommitThreads, 0, stream, p);
    else
        SPECPV_LAUNCH((d == 64 ? commit_q4_kernel<__nv_bfloat16, 64> : commit_q4_kernel<__nv_bfloat16, 128>), grid, kCommitThreads, 0, stream, p);
    if (advance) SPECPV_LAUNCH(commit_q4_lens_kernel, dim3((p.batch + kLensThreads - 1) / kLensThreads), kLensThreads, 0, stream, p);
    return SPECPV_OK;
}

specpv_status launch_gather_q4(const GatherQ4Params& p, int n_layers, int dtype, int d, cudaStream_t stream) {
    const dim3 grid(p.budget_blocks, p.Hkv, n_layers * p.batch);
    if (dtype == SPECPV_DTYPE_F32)
        SPECPV_LAUNCH((d == 64 ? gather_q4_kernel<float, 64> : gather_q4_kernel<float, 128>), grid, kGatherThreads, 0, stream, p);
    else
        SPECPV_LAUNCH((d == 64 ? gather_q4_kernel<__nv_bfloat16, 64> : gather_q4_kernel<__nv_bfloat16, 128>), grid, kGatherThreads, 0, stream, p);
    return SPECPV_OK;
}

}  // namespace specpv
