// The cache in 4 bits: layout of a page, and what its codes stand for.
//
// A page holds, per KV head, bs (d + 8) bytes: key codes, value codes, and four rows of bs bfloat16 numbers, the tokens' key
// scales, key offsets, value scales and value offsets.  Code n (0 .. 15) stands for bfloat16((16 + n) * scale + offset), rounded
// once: the four bits, put into the upper mantissa bits of a bfloat16 in [16, 32), ARE 16 + n, so that two codes are opened by one
// logical operation and one packed multiply-add.  The value is a bfloat16 by definition: the attention over such a cache, the
// partial cache taken out of it and the block summaries all see the same numbers.
//   key codes    [d / 32][bs][16 bytes]    a token's 32 channels side by side: lanes that own a token read 16 bytes each, without
//                                          bank conflicts
//   value codes  [bs / 16][d][8 bytes]     a channel's 16 tokens side by side: the same for lanes that own a channel
// A 32-bit word holds eight consecutive elements (channels of a key, tokens of a value): element 2 i in bits 4 i .. 4 i + 3, element
// 2 i + 1 in bits 16 + 4 i .., and the word is then rotated left by three bits, which puts element pair 0 at the mantissa bits as
// it stands, pairs 1 and 2 a shift away and pair 3 a rotation.
#pragma once
#include "common.cuh"

namespace specpv {
namespace q4 {

__host__ __device__ inline size_t page_bytes(int bs, int d) { return (size_t)bs * (d + 8); }  // of one KV head
// 32-bit words from the head of a page: channels c .. c + 7 of token t's key, tokens t .. t + 7 of channel c's value
__host__ __device__ inline int k_word(int bs, int t, int c) { return ((c >> 5) * bs + t) * 4 + ((c & 31) >> 3); }
__host__ __device__ inline int v_word(int bs, int d, int t, int c) { return bs * d / 8 + ((t >> 4) * d + c) * 2 + ((t & 15) >> 3); }
// bfloat16 numbers from the head of a page: `which` 0 key scale, 1 key offset, 2 value scale, 3 value offset
__host__ __device__ inline int param_at(int bs, int d, int which, int t) { return bs * d / 2 + which * bs + t; }

// elements 2 i and 2 i + 1 of a word as bfloat16 16 + n
__device__ __forceinline__ uint32_t open_pair(uint32_t w, int i) {
    const uint32_t x = i == 0 ? w : i == 1 ? w >> 4 : i == 2 ? w >> 8 : __funnelshift_r(w, w, 12);
    return (x & 0x00780078u) | 0x41804180u;
}
// The same where it is what a kernel does most: with both constants in registers (or the kernel's parameters) one instruction takes
// the bits and puts them in place; of two immediates it could hold only one.  `mask` and `ones` are kMask and kOnes, as the compiler must
// not know.
constexpr uint32_t kMask = 0x00780078u, kOnes = 0x41804180u;
__device__ __forceinline__ uint32_t open_pair(uint32_t w, int i, uint32_t mask, uint32_t ones) {
    const uint32_t x = i == 0 ? w : i == 1 ? w >> 4 : i == 2 ? w >> 8 : __funnelshift_r(w, w, 12);
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(x), "r"(mask), "r"(ones));  // (x & mask) | ones
    return r;
}
__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
__device__ __forceinline__ uint32_t twice(uint16_t x) { return (uint32_t)x | (uint32_t)x << 16; }
__device__ __forceinline__ float lower(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float upper(uint32_t pair) { return __uint_as_float(pair & 0xFFFF0000u); }

// place of element e in a word before its rotation, and the rotation
__device__ __forceinline__ int element_shift(int e) { return 4 * (e >> 1) + 16 * (e & 1); }
__device__ __forceinline__ uint32_t rotated(uint32_t w) { return __funnelshift_l(w, w, 3); }

// A row's scale and offset from its smallest and largest element, and the code of an element.  A row whose range or offset bfloat16
// cannot hold is stored as NaN, and so is one whose `lo` or `hi` is infinite or NaN.
struct Row {
    float scale, base;  // in float32, for the codes; base = what code 0 stands for before its rounding
    uint16_t scale16, offset16;
};
// (x - base) / scale is the IEEE quotient, in float32 to nearest.  So is RN(q + r i) with i a reciprocal of the divisor b good to 2^-22 of
// itself, q = RN(a i) and r = a - q b: the dividend a has 24 significant bits and b at most 8 (it is a bfloat16), so that r, 2^-21 of a at
// most and a multiple of the last places of q and b, has 12 bits and is exact; q + r i is then a / b but for 2^-43 of it, and
// nearer than 2^-33 of itself a / b comes to no number half-way between two of float32: such a number has 25 bits, its product with b a
// last place 2^-33 of it or more, and is not a, which would have 25 bits as well.  Outside of kLeast .. kMost, where the reciprocal or the remainder
// may underflow, they are divided.
constexpr float kLeast = 1e-30f, kMost = 1e30f;
__device__ __forceinline__ float reciprocal(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float quotient(float a, float b, float inv) {
    const float q = __fmul_rn(a, inv);
    return __fmaf_rn(__fmaf_rn(-q, b, a), inv, q);
}
__device__ __forceinline__ Row row_of(float lo, float hi) {
    Row r;
    const float range = __fsub_rn(hi, lo);
    const __nv_bfloat16 s = __float2bfloat16_rn(__fmul_rn(range, 1.f / 15.f));
    r.scale = __bfloat162float(s);
    const __nv_bfloat16 c = __float2bfloat16_rn(__fsub_rn(lo, 16.f * r.scale));  // (16 s is exact)
    const float offset = __bfloat162float(c);
    r.base = __fadd_rn(offset, 16.f * r.scale);
    r.scale16 = __bfloat16_as_ushort(s);
    r.offset16 = __bfloat16_as_ushort(c);
    if (!isfinite(r.scale) || !isfinite(offset) || !isfinite(r.base)) {
        r.scale = r.base = __int_as_float(0x7FC00000);
        r.scale16 = r.offset16 = 0x7FC0;
    }
    return r;
}
// The codes of eight elements as a word before its rotation: the nearest integers of (x - base) / scale, ties to even, 0 to 15.
__device__ __forceinline__ uint32_t word_of(const Row& r, const float (&x)[8]) {
    constexpr float kWhole = 12582912.f;  // 1.5 2^23: what is added to it is rounded to an integer, its last bits
    constexpr uint32_t kWholeBits = 0x4B400000u;
    const float inv = reciprocal(r.scale);
    float m[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) m[i] = __fadd_rn(fminf(fmaxf(quotient(__fsub_rn(x[i], r.base), r.scale, inv), 0.f), 15.f), kWhole);
    if (!(r.scale > kLeast && r.scale < kMost)) {  // (rows of equal elements, and NaN, among these)
#pragma unroll
        for (int i = 0; i < 8; ++i)  // 0 / 0: fmaxf takes the 0
            m[i] = __fadd_rn(fminf(fmaxf(__fdiv_rn(__fsub_rn(x[i], r.base), r.scale), 0.f), 15.f), kWhole);
    }
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) w += (__float_as_uint(m[e]) - kWholeBits) << element_shift(e);
    return w;
}

}  // namespace q4
}  // namespace specpv
