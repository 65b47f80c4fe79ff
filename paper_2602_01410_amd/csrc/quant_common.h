// Elements of a block of 32: its scale, the conversions to FP8 / FP4 codes and back, their errors; and the random numbers of
// stochastic rounding.  Shared by the kernels that
// quantize a stored tensor (quant_kernels.hip) and those that quantize what they compute (norm_kernels.hip).
#pragma once
#include "snip_internal.h"

namespace snip {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short short2_t __attribute__((ext_vector_type(2)));
typedef float float2_t __attribute__((ext_vector_type(2)));
typedef unsigned short ushort2_t __attribute__((ext_vector_type(2)));

template <int FMT> struct Fmt;
template <> struct Fmt<kFP8> { static constexpr int emax = 8; static constexpr unsigned mmax = 0x60; };  // 448 = 1.75 * 2^8
template <> struct Fmt<kFP4> { static constexpr int emax = 2; static constexpr unsigned mmax = 0x40; };  // 6   = 1.5  * 2^2

// Source loads.  A source line is read once and never again, so its load carries the streaming hint (measured:
// quantize ROW 4.7 -> 5.8 TB/s, COL 4.0 -> 4.75 TB/s of algorithmic bytes on a 361 MB tensor).  Where the one-pass kernel
// for both orientations reads every line twice, the second time out of cache, both of its reads are plain loads
// (with the hint on either one the kernel got 4-6 % slower).
typedef unsigned v4u_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 ld16(const uint16_t* p)
{
    const v4u_t v = __builtin_nontemporal_load(reinterpret_cast<const v4u_t*>(p));
    return make_uint4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ unsigned ld4(const uint16_t* p)
{
    return __builtin_nontemporal_load(reinterpret_cast<const unsigned*>(p));
}

__device__ __forceinline__ unsigned pk_max_u16(unsigned a, unsigned b)
{
    return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(ushort2_t, a),
                                                                  __builtin_bit_cast(ushort2_t, b)));
}
__device__ __forceinline__ unsigned pk_min_u16(unsigned a, unsigned b)
{
    return __builtin_bit_cast(unsigned, __builtin_elementwise_min(__builtin_bit_cast(ushort2_t, a),
                                                                  __builtin_bit_cast(ushort2_t, b)));
}

// Maximum over the four lanes of a quad (DPP quad_perm [1,0,3,2] then [2,3,0,1]).
__device__ __forceinline__ unsigned quad_max(unsigned m)
{
    unsigned t = (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true);
    m = m > t ? m : t;
    t = (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true);
    return m > t ? m : t;
}

// E8M0 byte from the 15 magnitude bits of the block maximum; 0xFF for Inf/NaN.
template <int FMT, int RULE>
__device__ __forceinline__ unsigned scale_byte(unsigned amax_bits)
{
    // (rule 0: adding 0x7F - mmax carries into the exponent where the mantissa exceeds mmax)
    int b = (int)amax_bits + ((RULE == 0 ? 0x7F - (int)Fmt<FMT>::mmax : 0) - (Fmt<FMT>::emax << 7));
    b = b < 0 ? 0 : b;
    return amax_bits >= 0x7F80u ? 0xFFu : (unsigned)b >> 7;
}

// The conversion instructions read only the exponent field of their scale operand; the
// mantissa bit set here keeps byte 0 (2^-127) from being an all-zero word.
__device__ __forceinline__ float scale_operand(unsigned byte)
{
    return __uint_as_float((byte << 23) | 0x00400000u);
}

// Clamp both bf16 halves of w to magnitude <= 448 * 2^(byte-127) (floor rule, FP8 only).
__device__ __forceinline__ unsigned clamp_fp8(unsigned w, unsigned byte)
{
    const unsigned lim = ((byte + 8u) << 7) | 0x60u;
    const unsigned mag = pk_min_u16(w & 0x7FFF7FFFu, lim | (lim << 16));
    return mag | (w & 0x80008000u);
}

// A register with unspecified content, at no cost: the packing conversions below replace their destination piece by
// piece (two halves for FP8, four bytes for FP4) and keep the rest, so the value they start from never survives;
// starting from zero would cost a move per destination.
__device__ __forceinline__ unsigned any_value()
{
    unsigned r;
    asm volatile("" : "=v"(r));
    return r;
}

// Two bf16 pairs (4 elements) -> 4 FP8 bytes.
template <int RULE>
__device__ __forceinline__ unsigned enc8(unsigned w0, unsigned w1, float sc, unsigned byte)
{
    if (RULE == 1) { w0 = clamp_fp8(w0, byte); w1 = clamp_fp8(w1, byte); }
    short2_t r = __builtin_bit_cast(short2_t, any_value());
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, w0), sc, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, w1), sc, true);
    return __builtin_bit_cast(unsigned, r);
}

// Four bf16 pairs (8 elements) -> 8 FP4 nibbles, element 0 in the lowest nibble.
__device__ __forceinline__ unsigned enc4(unsigned w0, unsigned w1, unsigned w2, unsigned w3, float sc)
{
    unsigned r = any_value();
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w0), sc, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w1), sc, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w2), sc, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w3), sc, 3);
    return r;
}

// s0 += x_lo^2 + x_hi^2 for a bf16 pair (one instruction: the products are exact, the sum is rounded once)
__device__ __forceinline__ void acc_sq(unsigned w, float& s0)
{
    asm("v_dot2c_f32_bf16 %0, %1, %1" : "+v"(s0) : "v"(w));
}
__device__ __forceinline__ void acc_err(float2_t q, unsigned w, float& s0, float& se)
{
    const float xl = __uint_as_float(w << 16), xh = __uint_as_float(w & 0xFFFF0000u);
    const float dl = q[0] - xl, dh = q[1] - xh;
    se = fmaf(dl, dl, se);
    se = fmaf(dh, dh, se);
    acc_sq(w, s0);
}

// Error sums of 8 source elements w[0..3] against their FP8 codes c[0..1].
__device__ __forceinline__ void err8(const unsigned* w, unsigned c0, unsigned c1, float sc,
                                     float& s0, float& se)
{
    acc_err(__builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c0, sc, false), w[0], s0, se);
    acc_err(__builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c0, sc, true),  w[1], s0, se);
    acc_err(__builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c1, sc, false), w[2], s0, se);
    acc_err(__builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c1, sc, true),  w[3], s0, se);
}
__device__ __forceinline__ void err4(const unsigned* w, unsigned c, float sc,
                                     float& s0, float& se)
{
    acc_err(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, sc, 0), w[0], s0, se);
    acc_err(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, sc, 1), w[1], s0, se);
    acc_err(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, sc, 2), w[2], s0, se);
    acc_err(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, sc, 3), w[3], s0, se);
}

// The same on elements unpacked to fp32, which is what the statistics work on: unpacked once, an element serves the block's
// maximum, the conversions to both formats and both errors, and nothing has to be re-paired.  Against packed pairs (masked for
// the maximum, re-paired for the conversions, unpacked for the errors) quant_both_kernel with all sums takes 1361 vector
// instructions per tile instead of 1483 (FP4), and us per call: statistics of both directions [16384 x 11008] 134.7 -> 121.4, [16384 x
// 4096] 49.1 -> 44.8, of rows 83 -> 78; quantize with all sums [16384 x 11008] FP4 174 -> 169, FP8 197 -> 194, [8192 x 4096] 41.3 ->
// 39.6 and 43.6 -> 42.
__device__ __forceinline__ void unpack2(unsigned w, float& lo, float& hi)
{
    lo = __uint_as_float(w << 16);
    hi = __uint_as_float(w & 0xFFFF0000u);
}
// max(m, |a|, |b|); a NaN stays a NaN
__device__ __forceinline__ float max3_abs(float m, float a, float b)
{
    float r;
    asm("v_maximum3_f32 %0, %1, |%2|, |%3|" : "=v"(r) : "v"(m), "v"(a), "v"(b));
    return r;
}
template <int N> __device__ __forceinline__ float max_abs(const float* x)
{
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < N; i += 2) m = max3_abs(m, x[i], x[i + 1]);
    return m;
}
// 4 elements -> 4 FP8 bytes, 8 elements -> 8 FP4 nibbles (`byte`: the scale; floor rule: magnitudes clamped to 448 * 2^(byte-127))
template <int RULE>
__device__ __forceinline__ unsigned enc8x4(const float* x, float sc, unsigned byte)
{
    float t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float lim = __uint_as_float(((byte + 8u) << 23) | 0x600000u);
        t[i] = RULE == 1 ? __builtin_amdgcn_fmed3f(x[i], -lim, lim) : x[i];
    }
    short2_t r = __builtin_bit_cast(short2_t, any_value());
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, t[0], t[1], sc, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, t[2], t[3], sc, true);
    return __builtin_bit_cast(unsigned, r);
}
__device__ __forceinline__ unsigned enc4x8(const float* x, float sc)
{
    unsigned r = any_value();
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], sc, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], sc, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], sc, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], sc, 3);
    return r;
}
__device__ __forceinline__ void acc_err2(float2_t q, const float* x, float& se)
{
    const float d0 = q[0] - x[0], d1 = q[1] - x[1];
    se = fmaf(d0, d0, se);
    se = fmaf(d1, d1, se);
}
__device__ __forceinline__ void err8x4(const float* x, unsigned c, float sc, float& se)
{
    acc_err2(__builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, sc, false), x, se);
    acc_err2(__builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, sc, true), x + 2, se);
}
__device__ __forceinline__ void err4x8(const float* x, unsigned c, float sc, float& se)
{
    acc_err2(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, sc, 0), x, se);
    acc_err2(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, sc, 1), x + 2, se);
    acc_err2(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, sc, 2), x + 4, se);
    acc_err2(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, sc, 3), x + 6, se);
}
// Error sums of N elements (a multiple of 8) of one block under both formats, am: magnitude bits of the block's maximum.
template <int N, int RULE>
__device__ __forceinline__ void both_errors(const float* x, unsigned am, float& se4, float& se8)
{
    const unsigned b8 = scale_byte<kFP8, RULE>(am), b4 = scale_byte<kFP4, RULE>(am);
    const float sc8 = scale_operand(b8), sc4 = scale_operand(b4);
#pragma unroll
    for (int k = 0; k < N; k += 8) {
        err8x4(x + k, enc8x4<RULE>(x + k, sc8, b8), sc8, se8);
        err8x4(x + k + 4, enc8x4<RULE>(x + k + 4, sc8, b8), sc8, se8);
        err4x8(x + k, enc4x8(x + k, sc4), sc4, se4);
    }
}
__device__ __forceinline__ unsigned magnitude_bits(float m) { return __float_as_uint(m) >> 16; }

// Magnitude bits of the largest of the 8 bf16 values in v (one lane's share of a block).
__device__ __forceinline__ unsigned amax8(const uint4& v)
{
    unsigned m = pk_max_u16(pk_max_u16(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu),
                            pk_max_u16(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu));
    const unsigned lo = m & 0xFFFFu, hi = m >> 16;
    return lo > hi ? lo : hi;
}

// Threefry-2x32, 20 rounds (Salmon et al., SC'11): adds, rotates and XORs only, which suits a VALU whose
// 32-bit multiplies run at quarter rate.
__device__ __forceinline__ unsigned rotl32(unsigned v, int r) { return (v << r) | (v >> (32 - r)); }
__device__ __forceinline__ void threefry2x32_20(unsigned c0, unsigned c1, unsigned k0, unsigned k1,
                                                unsigned& o0, unsigned& o1)
{
    constexpr int R[8] = {13, 15, 26, 6, 17, 29, 16, 24};
    const unsigned ks[3] = {k0, k1, 0x1BD11BDAu ^ k0 ^ k1};
    unsigned x0 = c0 + ks[0], x1 = c1 + ks[1];
#pragma unroll
    for (int r = 0; r < 20; ++r) {
        x0 += x1;
        x1 = rotl32(x1, R[r % 8]) ^ x0;
        if (r % 4 == 3) {
            const int inj = r / 4 + 1;
            x0 += ks[inj % 3];
            x1 += ks[(inj + 1) % 3] + (unsigned)inj;
        }
    }
    o0 = x0; o1 = x1;
}

}  // namespace
}  // namespace snip
