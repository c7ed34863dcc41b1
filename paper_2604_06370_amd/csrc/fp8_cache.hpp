// The 8-bit base cache: page layout, and the pieces of a wave that quantise, read and transpose rows.
//
// A row (the 128 values of K or V of one token and KV head) is 128 e4m3 codes and one exponent byte b:
// value = code * 2^(b - 127).  With amax the largest magnitude among the row's finite values, E = b - 127
// is the smallest integer in [-117, 119] with amax <= 448 * 2^E, and code = RNE(clamp(x * 2^-E, +-448));
// values that are not finite become NaN.  The scale is a power of two, so that scaling rounds nothing
// (one rounding per value, at most 2^-4 of it or half of the smallest code, 2^-10 * 2^E), and every value that the cache stands for
// is exact in bf16: four significant bits, and at least 2^(-9 - 117) = 2^-126 in magnitude.
//
// Page (fp8_page_bytes): [Hkv][2][2048] codes, K then V of each head, then [Hkv][2][16] exponent bytes (byte
// t: token t of the page), then up to 127 bytes of padding.  A block's codes are in the order of the matrix-core
// fragments, 16 bytes per lane:
//   K (token t, dim i)  (i/64)*1024 + (t + 16*((i%16)/4))*16 + 8*((i/32)%2) + 4*((i%32)/16) + i%4
//   V (token t, dim i)  (i/64)*1024 + (i%16 + 16*(t/4))*16 + 8*((i/32)%2) + 4*((i/16)%2) + t%4
#pragma once

#include <hip/hip_runtime.h>

#include "mfma.hpp"

namespace fkvk {

constexpr int kF8Block = 2048;        // codes of one (page, head, K|V)
constexpr int kF8HeadBytes = 4096;    // K and V codes of one (page, head)
constexpr int kF8ExpMin = 10, kF8ExpMax = 246;  // exponent bytes that are written

__host__ __device__ constexpr int64_t f8_page_bytes(int hkv) {
    return (int64_t)hkv * kF8HeadBytes + ((int64_t)hkv * 32 + 127) / 128 * 128;
}
// Exponent bytes of head h of a page: K's 16, then V's 16.
__host__ __device__ constexpr int64_t f8_exp_off(int hkv, int h) { return (int64_t)hkv * kF8HeadBytes + (int64_t)h * 32; }

// 2^(b - 127) of an exponent byte (b = 0, a page that was never written: 0; its codes are 0 as well)
__device__ __forceinline__ float f8_scale(uint32_t b) { return __uint_as_float(b << 23); }

// Four codes of a word as bf16 pairs, times a power of two (exact).
__device__ __forceinline__ u32x2 f8_to_bf16(uint32_t w, float scale) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
    const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true);
    return u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}
// Eight codes (16x16x32 operand of the bf16 products).
__device__ __forceinline__ u32x4 f8_to_bf16x8(uint32_t lo, uint32_t hi, float scale) {
    const u32x2 a = f8_to_bf16(lo, scale), b = f8_to_bf16(hi, scale);
    return u32x4{a.x, a.y, b.x, b.y};
}

// The four operands (16x16x32, bf16) of a block's codes as a lane holds them: two 16-byte pieces, two operands each.
__device__ __forceinline__ void f8_fragments(const u32x4 (&raw)[2], float scale, u32x4 (&out)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = f8_to_bf16x8(raw[i / 2][2 * (i % 2)], raw[i / 2][2 * (i % 2) + 1], scale);
}

// ---- a wave over four tokens (slots 4 w .. 4 w + 3 of a page) of one head: lane 16 k + c holds dims 4 c .. 4 c + 3
// (`lo`) and 64 + 4 c .. + 3 (`hi`, their rotate-half partners) of token 4 w + k ----

// Byte offsets of that lane's words: `lo` here, `hi` 1024 further.
__device__ __forceinline__ int f8_k_word(int t, int c) { return (t + 16 * (c & 3)) * 16 + (c >> 2) * 4; }
// V words hold one dim of four tokens: after f8_transpose lane 16 k + c has dim 4 c + k of tokens 4 w .. + 3.
__device__ __forceinline__ int f8_v_word(int w, int k, int c) { return (4 * (c & 3) + k + 16 * w) * 16 + (c >> 2) * 4; }

// Transpose of 4x4 bytes over the lanes l, l + 16, l + 32, l + 48 (its own inverse).
__device__ __forceinline__ uint32_t f8_transpose(uint32_t d, int k) {
    const uint32_t p = __shfl_xor(d, 32);
    const uint32_t r = k < 2 ? __builtin_amdgcn_perm(p, d, 0x05040100u) : __builtin_amdgcn_perm(d, p, 0x07060302u);
    const uint32_t s = __shfl_xor(r, 16);
    return (k & 1) == 0 ? __builtin_amdgcn_perm(s, r, 0x06020400u) : __builtin_amdgcn_perm(r, s, 0x07030501u);
}

// A 64-bit value rounded to 32 bits towards odd: a second rounding, to a code, then gives what one rounding
// of the 64-bit value gives.  Finite values only; beyond fp32 they become its largest.
__device__ __forceinline__ float f8_round_to_odd(double x) {
    x = fmin(fmax(x, -3.4028234663852886e38), 3.4028234663852886e38);
    const float f = (float)x;
    const double back = (double)f;
    uint32_t b = __float_as_uint(f);
    if (back != x) b = (fabs(back) > fabs(x) ? b - 1 : b) | 1u;
    return __uint_as_float(b);
}

// The lane's eight values of a row (16 lanes) as codes, and the row's exponent byte.
struct F8Row {
    uint32_t lo, hi, exp;
};
__device__ __forceinline__ F8Row f8_quantise(const float (&x)[8], const bool (&fine)[8]) {
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fine[i] ? fabsf(x[i]) : 0.f);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
    const uint32_t bits = __float_as_uint(amax);
    int b = (int)(bits >> 23) - ((bits & 0x7fffffu) <= 0x600000u ? 8 : 7);  // 448 = 1.75 * 2^8
    b = b < kF8ExpMin ? kF8ExpMin : (b > kF8ExpMax ? kF8ExpMax : b);
    const float inv = __uint_as_float((uint32_t)(254 - b) << 23);
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = fine[i] ? fminf(fmaxf(x[i] * inv, -448.f), 448.f) : __uint_as_float(0x7fc00000u);
    F8Row r;
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
    r.lo = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], w, true);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(q[4], q[5], 0, false);
    r.hi = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[6], q[7], w, true);
    r.exp = (uint32_t)b;
    return r;
}

}  // namespace fkvk
