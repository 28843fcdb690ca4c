// The 8-bit paged K/V cache and appending with the rotation: what its kernels share.
//
// A block is one page (16 positions) of one KV head.  Finished blocks hold e4m3
// codes x / s with one scale s a block, a power of two: the smallest that brings the
// block's largest magnitude to 448 or less (not below 2^-100).  e4m3 has the same
// four significant bits at every magnitude, so a scale that is no power of two
// would gain nothing but a rounding of its own.  A block with a value that is not
// finite has the scale NaN and codes 0.
//
// The codes lie as the tensor cores read them, in core matrices of 8 rows x 16
// bytes, so that a page goes to shared memory by plain bulk copies and is an
// operand as it lands:
//   K (the reduction runs over dims):   [slot / 8][dim / 16][slot % 8][dim % 16]
//   V (the reduction runs over slots):  [dim][slot]
// Rows of the unfinished page stay in bf16 in the tail, a ring of tail_pages pages
// a sequence that always holds the last rows written (a draft call's chain's rows, which
// nobody has committed, take the place of older ones too): each value is rounded to 8
// bits once, with its block's final scale, however many calls append the block.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"

namespace osp {

constexpr int KV8_MIN_EXP = -100;

// cos and sin of pos * inv_freq.  freq is inv_freq / 2 pi as a 64-bit fraction of a turn:
// the product modulo 2^64 drops whole turns exactly, which in double costs five
// instructions of a pipe that is 1/64 as wide.  What is left is a quarter turn's number
// and an angle of at most pi / 4, as a float and its remainder, for which the Taylor
// series suffice (terms left out: under 2^-29 of the sine, 2^-33 of the cosine).  Off the
// exact values by 1.2e-8 (sine) and 1.9e-8 (cosine) rms, correctly rounded ones by
// 1.1e-8 and 1.7e-8: a cached value rounds as the exact one does, but for chance.
__device__ __forceinline__ void rope_cs_fix(uint64_t freq, int pos, float &c, float &s) {
    const uint64_t t = freq * (uint64_t)pos;
    const uint32_t q = (uint32_t)((t + (1ull << 61)) >> 62) & 3;
    const int r = (int)((int64_t)(t - ((uint64_t)q << 62)) >> 31);   // 2^-33 turns, at most 2^30
    const float x = (float)r, low = (float)(r - (int)x);
    constexpr float u = (float)(6.283185307179586 / 8589934592.0), ul = (float)(6.283185307179586 / 8589934592.0 - (double)u);
    const float a = x * u, al = fmaf(x, u, -a) + fmaf(x, ul, low * u), a2 = a * a;
    float p = fmaf(a2, 1.f / 362880.f, -1.f / 5040.f);
    p = a2 * fmaf(a2, fmaf(a2, p, 1.f / 120.f), -1.f / 6.f);
    float w = fmaf(a2, fmaf(a2, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f);
    w = a2 * fmaf(a2, fmaf(a2, w, 1.f / 24.f), -0.5f);
    const float sn = a + fmaf(a, p, al), cn = 1.f + fmaf(-a, al, w);
    c = q & 1 ? sn : cn;
    s = q & 1 ? cn : sn;
    if (q == 1 || q == 2) c = -c;
    if (q & 2) s = -s;
}

// Two floats an instruction.
typedef unsigned long long f2;
__device__ __forceinline__ f2 mk2(float x, float y) {
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void un2(f2 v, float &x, float &y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ f2 fma2(f2 x, f2 y, f2 z) {
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(x), "l"(y), "l"(z));
    return r;
}
__device__ __forceinline__ f2 mul2(f2 x, f2 y) {
    f2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
    return r;
}
__device__ __forceinline__ f2 add2(f2 x, f2 y) {
    f2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
    return r;
}

// bf16(x1) : bf16(x0), rounded to nearest even; NaN stays NaN
__device__ __forceinline__ uint32_t kv8_bf2(float x0, float x1) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(x1), "f"(x0));
    return r;
}
// e4m3(x1) : e4m3(x0), rounded to nearest even
__device__ __forceinline__ uint32_t e4m3x2(float x0, float x1) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(x1), "f"(x0));
    return r;
}
// four of them, the first in the low byte
__device__ __forceinline__ uint32_t e4m3x4(float x0, float x1, float x2, float x3) {
    uint32_t r;
    asm("{\n.reg .b16 a, b;\ncvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\ncvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\nmov.b32 %0, {a, b};\n}"
        : "=r"(r) : "f"(x0), "f"(x1), "f"(x2), "f"(x3));
    return r;
}
// the two values of a pair of codes
__device__ __forceinline__ float2 e4m3x2_f(uint32_t pair) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)pair));
    float lo, hi;
    asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\ncvt.f32.f16 %0, a;\ncvt.f32.f16 %1, b;\n}" : "=f"(lo), "=f"(hi) : "r"(h));
    return make_float2(lo, hi);
}

// The largest bf16 magnitude of a block as its scale's exponent: smallest k >= -100
// with a <= 448 * 2^k = 1.75 * 2^(k + 8).
__device__ __forceinline__ int kv8_exp(uint32_t mag) {
    const int e = (int)(mag >> 7) - 127 - 8 + ((mag & 0x7f) > 0x60 ? 1 : 0);
    return e < KV8_MIN_EXP ? KV8_MIN_EXP : e;
}
__device__ __forceinline__ float kv8_pow2(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }

struct KvRopeArgs {
    const void *k_rows, *v_rows;   // [layers][total_rows] rows row_stride elements apart, each [Hkv][hd]
    int rows_f32, rotate;
    int64_t total_rows, row_stride;
    const int32_t *n_rows;         // [B]
    const int32_t *page_table;
    int32_t *seq_len;
    int B, layers, layer0, Hkv, hd, max_pages, n_pages;
    int32_t *status;
    uint64_t freq[64];
    // bf16 cache
    uint16_t *k_pages, *v_pages;
    // 8-bit cache
    uint8_t *k8, *v8;
    float *k_scale, *v_scale;
    uint16_t *k_tail, *v_tail;
    int tail_pages;
};
cudaError_t launch_kv_rope(const KvRopeArgs &a, bool eight, bool advance, int sms, cudaStream_t s);

// Quantises the pages that positions pos0[b] .. pos0[b] + nnew[b] - 1 of valid
// sequences finish, from the tail (every layer).
struct Kv8PackArgs {
    int B, L, Hkv, hd, max_pages, n_pages, tail_pages, max_new;
    const int *valid, *pos0, *nnew;
    const int32_t *page_table;
    uint8_t *k8, *v8;
    float *k_scale, *v_scale;
    const uint16_t *k_tail, *v_tail;
};
cudaError_t launch_kv8_pack(const Kv8PackArgs &a, cudaStream_t s);

}  // namespace osp
