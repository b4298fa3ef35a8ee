// Eviction by accumulated attention weight: the account of the weight that every cached token has received, and the eviction of the
// tokens with the smallest accounts, after which the others close up.
#include <math.h>

#include "aux_kernels.cuh"
#include "tc_common.cuh"

namespace specpv {

namespace {

// ---------------------------------------------------------------------------------------------
// Account: acc[t] += sum over the accepted rows i and the query heads g of the KV head of exp(scale q_ig . k_t - lse_ig), for the
// tokens t that row i sees.  The sum over rows is formed by one thread per token, in row order, so that the result is the same
// at every run.  Plain form: a thread owns a token, eight query rows at a time wait in shared memory as float32 and are read as
// broadcasts.  grid = (groups of 128 tokens, KV heads, layers x seqs).
// ---------------------------------------------------------------------------------------------
constexpr int kAccTokens = 128;
constexpr int kAccRows = 8;

__device__ __forceinline__ void widen4(const float* p, float4& v) { v = *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ void widen4(const __nv_bfloat16* p, float4& v) {
    const uint2 w = *reinterpret_cast<const uint2*>(p);
    v = make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xFFFF0000u));
}

template <typename T, int D>
__global__ void __launch_bounds__(kAccTokens) accumulate_simt_kernel(AccumulateParams p) {
    pdl_begin(p.pdl);
    __shared__ __align__(16) float s_q[kAccRows][D];
    __shared__ float s_lse[kAccRows];
    __shared__ int s_end[kAccRows];  // tokens that the row sees; 0 for a row that adds nothing
    const int h = blockIdx.y, lb = blockIdx.z, b = lb % p.batch, l = lb / p.batch;
    const int seq_len = min(max(p.seq_lens[b], 0), p.max_blocks * p.bs);
    const int n = min(max(p.n_accepted[b], 0), p.A_max);
    const int t = blockIdx.x * kAccTokens + threadIdx.x;
    if (blockIdx.x * kAccTokens >= seq_len || n == 0) return;
    int page = -1;
    if (t < seq_len) {
        page = p.block_table[(size_t)b * p.max_blocks + t / p.bs];
        if (page < 0 || page >= p.n_pages) {
            record_fault(p.workspace, SPECPV_ERR_BAD_BLOCK_TABLE, b, t / p.bs, page, l);
            page = -1;
        }
    }
    const T* k = reinterpret_cast<const T*>(p.k_pool) + ((((size_t)(p.layer0 + l) * p.n_pages + max(page, 0)) * p.Hkv + h) * p.bs + t % p.bs) * D;
    float total = 0.f;
    for (int r0 = 0; r0 < n * p.G; r0 += kAccRows) {
        __syncthreads();  // the rows before have been read
        for (int i = threadIdx.x; i < kAccRows * (D / 4); i += kAccTokens) {
            const int r = r0 + i / (D / 4), c = i % (D / 4) * 4, a = r / p.G;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            float lse = 0.f;
            int end = 0;
            if (a < n) {
                const int row = p.accepted ? p.accepted[(size_t)b * p.A_max + a] : a;
                if (row >= 0 && row < p.M_max) {
                    const size_t q = ((size_t)lb * p.M_max + row) * p.Hq + h * p.G + r % p.G;
                    widen4(reinterpret_cast<const T*>(p.q) + q * D + c, v);
                    lse = p.lse[q];
                    end = lse == -INFINITY ? 0 : seq_len - n + a + 1;
                } else if (c == 0 && h == 0 && blockIdx.x == 0 && r % p.G == 0) {
                    record_fault(p.workspace, SPECPV_ERR_INVALID_ARG, b, a, row, l);
                }
            }
            *reinterpret_cast<float4*>(&s_q[i / (D / 4)][c]) = v;
            if (c == 0) {
                s_lse[i / (D / 4)] = lse;
                s_end[i / (D / 4)] = end;
            }
        }
        __syncthreads();
        if (page < 0) continue;
        float4 sum[kAccRows];
#pragma unroll
        for (int j = 0; j < kAccRows; ++j) sum[j] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int c = 0; c < D; c += 4) {
            float4 x;
            widen4(k + c, x);
#pragma unroll
            for (int j = 0; j < kAccRows; ++j) {
                const float4 q = *reinterpret_cast<const float4*>(&s_q[j][c]);
                sum[j].x = fmaf(q.x, x.x, sum[j].x);
                sum[j].y = fmaf(q.y, x.y, sum[j].y);
                sum[j].z = fmaf(q.z, x.z, sum[j].z);
                sum[j].w = fmaf(q.w, x.w, sum[j].w);
            }
        }
#pragma unroll
        for (int j = 0; j < kAccRows; ++j)
            if (t < s_end[j]) total += expf(((sum[j].x + sum[j].y) + (sum[j].z + sum[j].w)) * p.scale - s_lse[j]);
    }
    if (page >= 0) p.acc[(((size_t)(p.layer0 + l) * p.batch + b) * p.Hkv + h) * (size_t)p.max_blocks * p.bs + t] += total;
}

// ---------------------------------------------------------------------------------------------
// Close-up: rank j of a KV head's kept tokens (ascending, so idx[j] >= j) moves to place j, in place.  A unit is the keys or the values
// of one (layer, sequence, KV head); it is worked through in chunks of ranks, each read whole before any of it is written: place j, as
// a source, belongs to a rank <= j, so nothing that is still to be read is overwritten, and later chunks may be read ahead.  Ranks
// that stay (a prefix) are skipped.  grid = (2 KV heads, layers x seqs).
// ---------------------------------------------------------------------------------------------
constexpr int kCloseThreads = 256;
constexpr int kCloseLoads = 8;  // 16-byte loads in flight per thread

__global__ void __launch_bounds__(kCloseThreads) close_up_kernel(EvictParams p) {
    pdl_begin(p.pdl);
    const int h = blockIdx.x % p.Hkv, values = blockIdx.x / p.Hkv, lb = blockIdx.y, b = lb % p.batch, l = lb / p.batch;
    const int capacity = p.max_blocks * p.bs, seq_len = min(max(p.seq_lens[b], 0), capacity);
    if (seq_len <= p.keep) return;
    const int32_t* idx = p.idx + (((size_t)l * p.batch + b) * p.Hkv + h) * p.keep;
    const int32_t* table = p.block_table + (size_t)b * p.max_blocks;
    // the first rank that moves
    int first = 0;
    for (int lo = 0, hi = p.keep; lo < hi;) {
        const int mid = (lo + hi) / 2;
        if (idx[mid] == mid) first = lo = mid + 1;
        else hi = mid;
    }
    uint4* pool = reinterpret_cast<uint4*>(values ? p.v_pool : p.k_pool);
    const int chunks = p.row_bytes / 16, per_chunk = kCloseThreads * kCloseLoads / chunks;  // 16-byte pieces of a row, ranks at a time
    const int piece = threadIdx.x % chunks, lane_row = threadIdx.x / chunks, step = kCloseThreads / chunks;
    auto place = [&](int t) -> long long {  // of token t, in 16-byte pieces; -1 behind a bad page id
        const int page = table[t / p.bs];
        if (page < 0 || page >= p.n_pages) {
            if (piece == 0) record_fault(p.workspace, SPECPV_ERR_BAD_BLOCK_TABLE, b, t / p.bs, page, l);
            return -1;
        }
        return ((((long long)l * p.n_pages + page) * p.Hkv + h) * p.bs + t % p.bs) * chunks + piece;
    };
    for (int j0 = first; j0 < p.keep; j0 += per_chunk) {
        uint4 buf[kCloseLoads];
        long long to[kCloseLoads];
#pragma unroll
        for (int u = 0; u < kCloseLoads; ++u) {
            const int j = j0 + u * step + lane_row;
            to[u] = -1;
            if (j < p.keep) {
                const long long from = place(idx[j]);
                if (from >= 0) {
                    to[u] = place(j);
                    buf[u] = pool[from];
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kCloseLoads; ++u)
            if (to[u] >= 0) pool[to[u]] = buf[u];
    }
    if (values) return;
    float* acc = p.acc + (((size_t)l * p.batch + b) * p.Hkv + h) * (size_t)capacity;
    for (int j0 = first; j0 < p.keep; j0 += kCloseThreads) {
        const int j = j0 + threadIdx.x;
        const float a = j < p.keep ? acc[idx[j]] : 0.f;
        __syncthreads();
        if (j < p.keep) acc[j] = a;
    }
    __syncthreads();
    for (int j = p.keep + threadIdx.x; j < seq_len; j += kCloseThreads) acc[j] = 0.f;  // the accounts of the tokens to come
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

specpv_status launch_accumulate(const AccumulateParams& p, int n_layers, int max_seq_len, int dtype, int d, cudaStream_t stream) {
    if (max_seq_len <= 0) return SPECPV_OK;
    const dim3 grid((max_seq_len + kAccTokens - 1) / kAccTokens, p.Hkv, n_layers * p.batch);
    if (dtype == SPECPV_DTYPE_F32)
        SPECPV_LAUNCH((d == 64 ? accumulate_simt_kernel<float, 64> : accumulate_simt_kernel<float, 128>), grid, kAccTokens, 0, stream, p);
    else
        SPECPV_LAUNCH((d == 64 ? accumulate_simt_kernel<__nv_bfloat16, 64> : accumulate_simt_kernel<__nv_bfloat16, 128>), grid, kAccTokens, 0, stream, p);
    return SPECPV_OK;
}

specpv_status launch_evict(const EvictParams& p, int n_layers, cudaStream_t stream) {
    SPECPV_LAUNCH(close_up_kernel, dim3(2 * p.Hkv, n_layers * p.batch), kCloseThreads, 0, stream, p);
    SPECPV_LAUNCH(evict_lens_kernel, dim3((p.batch + kLensThreads - 1) / kLensThreads), kLensThreads, 0, stream, p);
    return SPECPV_OK;
}

}  // namespace specpv
