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
// eight tokens of a channel) have one writer.  A lane holds eight channels of a row: half a warp, or a quarter, quantises a key and the
// next its value, a token (two with 64 channels) per warp at a time; the smallest and largest element meet in shuffles, in bfloat16 as
// one pair.  A key's eight channels are a word as they are; a value's go to shared memory as such a word, and a thread then turns
// the words of eight tokens over into words of eight channels, with those of tokens that the page held before.  The page's summary is
// taken from the new keys in registers and the old ones' codes.  Bound by instructions (2048 rows x 8 heads x 16 layers of 128
// channels: 102 us against 47 for its bytes, 300 instructions a token; with four channels a lane and values gathered byte by byte 165).
// grid = (pages touched, KV heads, layers x seqs).
// ---------------------------------------------------------------------------------------------
constexpr int kCommitThreads = 256;
constexpr int kCommitWarps = kCommitThreads / 32;

template <typename T>
struct Eight {};  // channels of a row
template <>
struct Eight<__nv_bfloat16> {
    uint4 x;
};
template <>
struct Eight<float> {
    float4 x, y;
};
__device__ __forceinline__ void load8(const __nv_bfloat16* p, Eight<__nv_bfloat16>& r) { r.x = *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void load8(const float* p, Eight<float>& r) {
    r.x = *reinterpret_cast<const float4*>(p);
    r.y = *reinterpret_cast<const float4*>(p + 4);
}
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {  // of a number and NaN the number
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t min_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t max_nan_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t min_nan_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// The elements in float32, and the smallest and largest of the kLanes lanes' that share a row; an infinite or NaN one makes `hi` or
// `lo` infinite or NaN.
template <int kLanes>
__device__ __forceinline__ void range_of(const Eight<__nv_bfloat16>& r, float (&x)[8], float& lo, float& hi) {
    const uint32_t w[4] = {r.x.x, r.x.y, r.x.z, r.x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = q4::lower(w[i]);
        x[2 * i + 1] = q4::upper(w[i]);
    }
    const uint32_t h = max_nan_bf16x2(max_nan_bf16x2(w[0], w[1]), max_nan_bf16x2(w[2], w[3]));
    const uint32_t l = min_nan_bf16x2(min_nan_bf16x2(w[0], w[1]), min_nan_bf16x2(w[2], w[3]));
    uint32_t m = max_nan_bf16x2(__byte_perm(h, l, 0x5410) ^ 0x80000000u, __byte_perm(h, l, 0x7632) ^ 0x80000000u);  // (largest, -smallest)
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1) m = max_nan_bf16x2(m, __shfl_xor_sync(0xffffffffu, m, o));
    hi = q4::lower(m);
    lo = -q4::upper(m);
}
template <int kLanes>
__device__ __forceinline__ void range_of(const Eight<float>& r, float (&x)[8], float& lo, float& hi) {
    x[0] = r.x.x; x[1] = r.x.y; x[2] = r.x.z; x[3] = r.x.w; x[4] = r.y.x; x[5] = r.y.y; x[6] = r.y.z; x[7] = r.y.w;
    bool finite = true;
    lo = hi = x[0];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        lo = fminf(lo, x[i]);
        hi = fmaxf(hi, x[i]);
        finite &= isfinite(x[i]);
    }
    if (!finite) hi = INFINITY;
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
}

__device__ __forceinline__ void store8(__nv_bfloat16* p, const uint32_t (&v)[4]) {  // eight elements, 16-byte aligned
    *reinterpret_cast<uint4*>(p) = make_uint4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void store8(float* p, const uint32_t (&v)[4]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(v[0] << 16, v[0] & 0xFFFF0000u, v[1] << 16, v[1] & 0xFFFF0000u);
    *reinterpret_cast<uint4*>(p + 4) = make_uint4(v[2] << 16, v[2] & 0xFFFF0000u, v[3] << 16, v[3] & 0xFFFF0000u);
}

// Words (as before their rotation) of eight tokens, a code per channel, into words of eight channels, a code per token.  Element e
// of a word is its digit e / 2 + 4 (e % 2): with rows and columns in that order it is the plain transpose of 8 x 8 digits of four bits.
__device__ __forceinline__ void turn_over(const uint32_t (&token)[8], uint32_t (&channel)[8]) {
    uint32_t a[8], b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e / 2 + 4 * (e % 2)] = token[e];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        b[i] = __byte_perm(a[i], a[i + 4], 0x5410);
        b[i + 4] = __byte_perm(a[i], a[i + 4], 0x7632);
    }
#pragma unroll
    for (int i = 0; i < 8; i += i % 4 == 1 ? 3 : 1) {  // 0, 1, 4, 5
        a[i] = __byte_perm(b[i], b[i + 2], 0x6240);
        a[i + 2] = __byte_perm(b[i], b[i + 2], 0x7351);
    }
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        b[i] = (a[i] & 0x0F0F0F0Fu) | (a[i + 1] << 4 & 0xF0F0F0F0u);
        b[i + 1] = (a[i] >> 4 & 0x0F0F0F0Fu) | (a[i + 1] & 0xF0F0F0F0u);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) channel[e] = b[e / 2 + 4 * (e % 2)];
}

template <typename T, int D>
__global__ void __launch_bounds__(kCommitThreads, 3) commit_q4_kernel(CommitQ4Params p) {
    pdl_begin(p.pdl);
    constexpr int kLanes = D / 8;                    // per row
    constexpr int kTokens = 16 / kLanes;             // per warp at a time
    constexpr int kStep = kCommitWarps * kTokens;    // per CTA
    constexpr int kGroups = kCommitThreads / kLanes;
    constexpr int kPad = D == 128 ? 2 : 1;           // two groups of eight tokens (four with 64 channels) are in different banks
    __shared__ uint32_t s_v[64][kLanes + kPad];      // value codes of the page's new tokens, a word per eight channels
    __shared__ __align__(8) unsigned char s_there[64];
    __shared__ __align__(16) uint32_t s_max[kGroups][D / 2], s_min[kGroups][D / 2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int column = lane % kLanes, c0 = column * 8, is_v = lane / kLanes & 1, sub = warp * kTokens + lane / (2 * kLanes);
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
    // A lane of the first 64 / kStep holds the row of a token of each round (which a token's lanes then take from it); the next round's
    // rows are in flight while this one's are worked on.
    constexpr int kRounds = 64 / kStep;
    int rows = -1;
    {
        const int t = t0 + warp * kTokens + lane % kTokens + lane / kTokens * kStep;
        if (lane < kRounds * kTokens && t < t1) rows = p.accepted ? p.accepted[(size_t)b * p.A_max + (t - seq_len)] : t - seq_len;
    }
    const T* src = reinterpret_cast<const T*>(is_v ? p.v_new : p.k_new) + ((size_t)lb * p.M_max * p.Hkv + h) * D + c0;
    T* values = reinterpret_cast<T*>(is_v ? p.v_values : p.k_values);
    const size_t row_stride = (size_t)p.Hkv * D;
    Eight<T> next{};
    int row_next = -1;
    auto fetch = [&](int round) {
        row_next = __shfl_sync(0xffffffffu, rows, round * kTokens + lane / (2 * kLanes));
        if (row_next >= 0 && row_next < p.M_max) load8(src + row_next * row_stride, next);
    };
    uint32_t mx[4], mn[4];  // of this lane's key channels
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        mx[i] = 0xFF80FF80u;
        mn[i] = 0x7F807F80u;
    }
    bool lost = false;
    fetch(0);
    for (int round = 0; t0 + warp * kTokens + round * kStep < t1; ++round) {
        const int t = t0 + sub + round * kStep, at = t - page_t0, row = row_next;
        const bool there = t < t1 && row >= 0 && row < p.M_max;
        const Eight<T> now = next;
        fetch(round + 1 < kRounds ? round + 1 : 0);
        float x[8], lo, hi;
        range_of<kLanes>(now, x, lo, hi);
        const q4::Row r = q4::row_of(lo, hi);
        const uint32_t w = q4::word_of(r, x), turned = q4::rotated(w);
        uint32_t value[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) value[i] = q4::fma_bf16x2(q4::open_pair(turned, i), q4::twice(r.scale16), q4::twice(r.offset16));
        if (there) {
            if (values) store8(values + ((size_t)lb * p.A_max + (t - seq_len)) * row_stride + (size_t)h * D + c0, value);
            if (is_v) {
                s_v[at][column] = w;
                if (column == 0) s_there[at] = 1;
            } else {
                words[q4::k_word(p.bs, at, c0)] = turned;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    mx[i] = max_bf16x2(mx[i], value[i]);
                    mn[i] = min_bf16x2(mn[i], value[i]);
                }
            }
            if (column < 2) params[q4::param_at(p.bs, D, 2 * is_v + column, at)] = column ? r.offset16 : r.scale16;
        } else if (t < t1) {  // the token keeps what its place held
            if (lane % (2 * kLanes) == 0) record_fault(p.workspace, SPECPV_ERR_INVALID_ARG, b, t - seq_len, row, l);
            if (is_v && column == 0) s_there[at] = 0;
            lost = true;
        }
    }
    const bool skipped = __syncthreads_or(lost);
    // value words of the touched groups of 16 tokens: neighbours take eight tokens each and exchange halves, so that each stores the 32
    // bytes of four channels
    const int g0 = (t0 - page_t0) / 16, g1 = (t1 - 1 - page_t0) / 16;
    for (int i0 = 0; i0 < (g1 - g0 + 1) * 2 * kLanes; i0 += kCommitThreads) {
        const int i = i0 + (int)threadIdx.x, half = i & 1, g = g0 + i / (2 * kLanes), c = i / 2 % kLanes;
        const bool mine = g <= g1;
        const int at0 = g * 16 + 8 * half;
        uint32_t token[8], channel[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) token[e] = mine ? s_v[at0 + e][c] : 0u;
        turn_over(token, channel);
        uint32_t* to = words + q4::v_word(p.bs, D, g * 16, c * 8 + 4 * half);  // [channel][eight tokens]
        uint32_t out[4][2];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t other = __shfl_xor_sync(0xffffffffu, half ? channel[e] : channel[e + 4], 1);
            out[e][0] = q4::rotated(half ? other : channel[e]);
            out[e][1] = q4::rotated(half ? channel[e + 4] : other);
        }
        if (!mine) continue;
        const bool whole = page_t0 + g * 16 >= t0 && page_t0 + g * 16 + 16 <= t1 && !skipped;  // nothing of the old words stays
        if (!whole) {
            uint32_t fresh[2] = {0, 0};
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int t = page_t0 + g * 16 + e;
                if (t >= t0 && t < t1 && s_there[g * 16 + e]) fresh[e / 8] |= 15u << q4::element_shift(e % 8);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    const uint32_t m = q4::rotated(fresh[z]);
                    out[e][z] = (out[e][z] & m) | (to[2 * e + z] & ~m);
                }
        }
#pragma unroll
        for (int e = 0; e < 4; e += 2)
            *reinterpret_cast<uint4*>(to + 2 * e) = make_uint4(out[e][0], out[e][1], out[e + 1][0], out[e + 1][1]);
    }
    if (!p.kmax) return;
    // Eq. 1 over the page's tokens: those that it held before, by their codes (all of them, where a new one kept what its place held)
    for (int t = threadIdx.x / kLanes; t < (skipped ? t1 : t0) - page_t0; t += kGroups) {
        const uint32_t w = words[q4::k_word(p.bs, t, c0)];
        const uint32_t s = q4::twice(params[q4::param_at(p.bs, D, 0, t)]), o = q4::twice(params[q4::param_at(p.bs, D, 1, t)]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t v = q4::fma_bf16x2(q4::open_pair(w, i), s, o);
            mx[i] = max_bf16x2(mx[i], v);
            mn[i] = min_bf16x2(mn[i], v);
        }
    }
    *reinterpret_cast<uint4*>(&s_max[threadIdx.x / kLanes][column * 4]) = make_uint4(mx[0], mx[1], mx[2], mx[3]);
    *reinterpret_cast<uint4*>(&s_min[threadIdx.x / kLanes][column * 4]) = make_uint4(mn[0], mn[1], mn[2], mn[3]);
    __syncthreads();
    if ((int)threadIdx.x < D) {  // two channels' largest, or smallest
        const int pair = threadIdx.x % (D / 2);
        const bool smallest = threadIdx.x >= D / 2;
        uint32_t a = smallest ? s_min[0][pair] : s_max[0][pair];
#pragma unroll
        for (int i = 1; i < kGroups; ++i) a = smallest ? min_bf16x2(a, s_min[i][pair]) : max_bf16x2(a, s_max[i][pair]);
        T* to = reinterpret_cast<T*>(smallest ? p.kmin : p.kmax) +
                ((((size_t)(p.layer0 + l) * p.batch + b) * p.Hkv + h) * p.max_blocks + block) * D + 2 * pair;
        to[0] = from_float<T>(q4::lower(a));
        to[1] = from_float<T>(q4::upper(a));
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
// Gather: a CTA of two warps opens the keys, another the values, of one selected block of a KV head into the partial cache: CTAs of their
// own, so that neither waits for the other's loads.  Keys: a thread takes a word, 16 bytes of a bfloat16 row; lanes take the words of a
// row.  Values: a thread takes eight channels of eight tokens and stores 16 bytes of each of the eight rows.  Bound by HBM where there
// are many blocks (64 blocks of 64 tokens x 8 heads x 32 layers, 128 channels: 111 us, 92 % of the copy rate), by latency where there are few (128
// blocks of 16 tokens, 64 channels: 10.4 us; with four warps for keys and values in turn 12.6).
// grid = (2 x budget blocks, KV heads, layers x seqs).
// ---------------------------------------------------------------------------------------------
constexpr int kGatherThreads = 64;

template <typename T, int D>
__global__ void __launch_bounds__(kGatherThreads) gather_q4_kernel(GatherQ4Params p) {
    pdl_begin(p.pdl);
    const int s = blockIdx.x >> 1, h = blockIdx.y, lb = blockIdx.z, b = lb % p.batch, l = lb / p.batch;
    const bool values = blockIdx.x & 1;
    const int count = p.count[b], seq_len = max(p.seq_lens[b], 0), nb = (seq_len + p.bs - 1) / p.bs;
    // the last selected block is the sequence's last block, of which the valid tokens are kept
    if (blockIdx.x == 0 && h == 0 && l == 0 && threadIdx.x == 0) p.partial_lens[b] = count > 0 ? (count - 1) * p.bs + (seq_len - (nb - 1) * p.bs) : 0;
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
    if (!values) {
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
        return;
    }
    for (int i = threadIdx.x; i < p.bs / 8 * (D / 8); i += kGatherThreads) {
        const int t0 = i / (D / 8) * 8, c = i % (D / 8) * 8;
        if (t0 >= n_valid) break;
        uint32_t w[8];  // of the channels
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = words[q4::v_word(p.bs, D, t0, c + j)];
        const uint4 x = *reinterpret_cast<const uint4*>(params + q4::param_at(p.bs, D, 2, t0));
        const uint4 y = *reinterpret_cast<const uint4*>(params + q4::param_at(p.bs, D, 3, t0));
        const uint32_t scales[4] = {x.x, x.y, x.z, x.w}, offsets[4] = {y.x, y.y, y.z, y.w};  // of pairs of tokens
#pragma unroll
        for (int pair = 0; pair < 4; ++pair) {  // tokens t0 + 2 pair and the next
            const int t = t0 + 2 * pair;
            const uint32_t scale = scales[pair], offset = offsets[pair];
            uint32_t even[4], odd[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t a = q4::fma_bf16x2(q4::open_pair(w[2 * j], pair), scale, offset);
                const uint32_t z = q4::fma_bf16x2(q4::open_pair(w[2 * j + 1], pair), scale, offset);
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
    const dim3 grid(2 * p.budget_blocks, p.Hkv, n_layers * p.batch);
    if (dtype == SPECPV_DTYPE_F32)
        SPECPV_LAUNCH((d == 64 ? gather_q4_kernel<float, 64> : gather_q4_kernel<float, 128>), grid, kGatherThreads, 0, stream, p);
    else
        SPECPV_LAUNCH((d == 64 ? gather_q4_kernel<__nv_bfloat16, 64> : gather_q4_kernel<__nv_bfloat16, 128>), grid, kGatherThreads, 0, stream, p);
    return SPECPV_OK;
}

}  // namespace specpv
