// Conversions of e4m3 codes (sm_100a has them as instructions on pairs) and the power-of-two scales of an 8-bit pool.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "ptx.cuh"

namespace ekv {

static constexpr int kScaleMinExp = -112, kScaleMaxExp = 120;
static constexpr float kMaxScale = 1.329227995784916e36f;  // 2^120

// two codes (low byte first) -> two f16, exactly (e4m3 is a subset of f16; NaN stays NaN)
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint16_t v) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(v));
    return r;
}
// the same for the low / high half of a word of four codes
__device__ __forceinline__ uint32_t e4m3_lo(uint32_t w) { return e4m3x2_to_f16x2((uint16_t)(w & 0xffffu)); }
__device__ __forceinline__ uint32_t e4m3_hi(uint32_t w) { return e4m3x2_to_f16x2((uint16_t)(w >> 16)); }

__device__ __forceinline__ float2 f16x2_to_float2(uint32_t h) {
    float2 r;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.f32.f16 %0, lo;\n\tcvt.f32.f16 %1, hi;\n\t}" : "=f"(r.x), "=f"(r.y) : "r"(h));
    return r;
}
// two floats -> two codes (lo in the low byte), round to nearest even, beyond 448 held to 448, NaN to NaN
__device__ __forceinline__ uint32_t floats_to_e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

// bit 7 of each byte that is a NaN code (magnitude 0x7f)
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
// the same codes with 0 in place of NaN
__device__ __forceinline__ uint32_t without_nan_codes(uint32_t w) { return w & ~((nan_codes(w) >> 7) * 0xffu); }
__device__ __forceinline__ uint4 without_nan_codes(const uint4 &v) {
    return make_uint4(without_nan_codes(v.x), without_nan_codes(v.y), without_nan_codes(v.z), without_nan_codes(v.w));
}

// 2^-e for a scale 2^e (a normal power of two): by its bits, no reciprocal
__device__ __forceinline__ float pow2_inverse(float s) { return __uint_as_float((254u << 23) - (__float_as_uint(s) & 0x7f800000u)); }

// the smallest 2^e, -112 <= e <= 120, with a <= 448 * 2^e; a: magnitude bits of a finite bf16
__device__ __forceinline__ float scale_of_bf16_bits(uint32_t a) {
    const int e = (int)(a >> 7) - 127 - ((a & 0x7fu) <= 0x60u ? 8 : 7);  // 448 = 1.75 * 2^8; 0x60 is a mantissa of .75
    const int c = e < kScaleMinExp ? kScaleMinExp : (e > kScaleMaxExp ? kScaleMaxExp : e);
    return __uint_as_float((uint32_t)(c + 127) << 23);
}

// 2^k that brings a positive finite magnitude a into [2^13, 2^14); 1 for 0 and for what is not finite
__device__ __forceinline__ float to_f16_range(float a) {
    const int e = (int)(__float_as_uint(a) >> 23) & 0xff;
    const int k = (e == 0xff || a == 0.f) ? 0 : min(13 - (e - 127), 126);
    return __uint_as_float((uint32_t)(k + 127) << 23);
}

// ---- what decode and the few-rows kernel share: P V with both operands in f16 -----------------------------------
// V's codes are exact in f16, so one conversion instruction makes an operand of them, if V's scale 2^e_V goes elsewhere.  It goes
// into P, and so that f16's range does not matter, a row keeps two references: m for its scores x (log2), which its sum of
// weights p = 2^(x - m) is relative to, and M for x + e_V, i.e. for its contributions to O, which P = 2^(x + e_V - M + kPUp) =
// p * 2^(e_V + m - M + kPUp) is relative to: one more exponential a block and row, none a score.  P then has 11 bits while a
// contribution is within 2^-20 of the row's largest one, and an absolute error of 2^-31 of that below (bf16 would have 8 bits at
// any distance, and V would need three instructions more for two codes).
//   kPUp    against f16's small end; P is at most 2^(kPUp + kLazy) = 2^14
//   kLazy   how far (log2) a score may lie above a reference before the reference is raised and l, O scaled
//   kNoRef  references of a row without a score yet; no finite score is below
static constexpr float kPUp = 6.f, kLazy = 8.f, kNoRef = -3.0e38f;

struct RowRef {
    float m, M, l;
    // 2^(e + m - M + kPUp), kept finite: beyond 2^120 the weights it goes with are below 2^-106 (P is at most 2^14)
    __device__ __forceinline__ float p_factor(float e) const { return fast_exp2(fminf((m - M) + (e + kPUp), 120.f)); }
    // what O is to be multiplied by to be relative to m, like l
    __device__ __forceinline__ float o_factor() const { return fast_exp2((M - m) - kPUp); }
};
// e_V of a V scale (a power of two; -127 for a scale of 0, whose codes the kernels take as 0)
__device__ __forceinline__ float scale_exponent(float scale) { return (float)((int)((__float_as_uint(scale) >> 23) & 0xffu) - 127); }

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
// D(16x8, f32) += A(16x16, f16, row) * B(16x8, f16, col)
__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

}  // namespace ekv
