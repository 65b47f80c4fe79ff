// One AdamW step over many tensors, moments in 32 or in 8 bits.
//     g = grad * grad_scale;   m = b1 m + (1 - b1) g;   v = b2 v + (1 - b2) g^2
//     p = p (1 - lr decay) - lr / (1 - b1^t) * m / (sqrt(v / (1 - b2^t)) + eps)
// One streaming pass over each tensor, bound by memory: 26 to 30 bytes per element with moments of 32 bits (8 each for p, m and v,
// 2 or 4 for the gradient, 2 for the bf16 copy that the next quantize reads), 14 to 18 with 8 bits.
//
// Moments of 8 bits, in groups of 128 elements with an fp32 scale each:
//   m        E4M3 numbers, rounded to nearest; the scale takes the largest to 448.  A scale that is no power of two lets a whole group
//            decay without a change of its codes.  A step moves a number only where (1 - b1) |g - m| exceeds half its distance to the next one, |m| / 16
//            at most: noise in the gradients does (1 - b1 is 0.1), but m can stop 0.63 |m| from a gradient that no longer changes.
//   sqrt(v)  unsigned numbers of 4 exponent and 4 mantissa bits with gradual underflow (bits 13 to 6 of a half); the scale takes
//            the largest to 1.9375.  The root halves the range in the exponent, so that 2^-15.. of the largest root is 2^-30.. of v.  Rounded
//            stochastically: b2 changes v by a small part of a code's distance per step, which rounding to nearest would undo at every
//            step.  What is not zero stays so: a root of zero beside a moment that is not would make a step of m / eps.
// Measured, us per step and TB/s: 7B-shaped block 994-1053 (5.4-5.7) and, 8 bits, 581-601 (5.6); 1B-shaped block of 67 M elements 335-350 (5.6) and 185
// (5.8); 263 k elements 6.1, launch by launch.  A copy at this card's best mix of reads and writes reaches 5.6.
//
// Both are formed with one rounding per written operation (no contraction, and __builtin_sqrtf, which rounds correctly where
// __fsqrt_rn is the hardware's approximation), so that codes are a function of the formulas alone.
#include "snip_internal.h"
#include "quant_common.h"

namespace snip {
namespace {

constexpr int kStepThreads = 256;
// Elements of a workgroup, a multiple of the scale groups' 128: a workgroup for each 2048.  us per step of a 7B-shaped block (202 M elements), moments of
// 32 / 8 bits, all accesses streaming: 1114 / 607; with 8192 elements 1185 / 658, with 2048 workgroups that take turns of 8192 1241 / 737, of 32768 1294 / 757.
constexpr int kStepChunk = kStepThreads * 8;

// Vectors at the elements' own alignment: tensors may start anywhere.
typedef float f4_t __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned u4_t __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned u2_t __attribute__((ext_vector_type(2), aligned(1)));

// NT: streaming.  With moments of 8 bits it pays (7B- / 1B-shaped block 607 / 187 us, plain 601 / 202), with 32 it does not (1114 / 349 us, plain
// 1053 / 350).
template <bool NT, class V> __device__ __forceinline__ V get(const V* p) { return NT ? __builtin_nontemporal_load(p) : *p; }
template <bool NT, class V> __device__ __forceinline__ void put(V* p, V v)
{
    if (NT) __builtin_nontemporal_store(v, p);
    else    *p = v;
}

template <bool NT> __device__ __forceinline__ void load8f(const float* p, int left, float (&f)[8])
{
    if (left >= 8) {
        const f4_t a = get<NT>((const f4_t*)p), b = get<NT>((const f4_t*)p + 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[i] = a[i]; f[4 + i] = b[i]; }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = i < left ? p[i] : 0.f;
    }
}
template <bool NT> __device__ __forceinline__ void store8f(float* p, int left, const float (&f)[8])
{
    if (left >= 8) {
        put<NT>((f4_t*)p, f4_t{f[0], f[1], f[2], f[3]});
        put<NT>((f4_t*)p + 1, f4_t{f[4], f[5], f[6], f[7]});
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = f[i];
    }
}
template <bool NT> __device__ __forceinline__ void load8h(const uint16_t* p, int left, float (&f)[8])
{
    if (left >= 8) {
        const u4_t v = get<NT>((const u4_t*)p);
#pragma unroll
        for (int i = 0; i < 4; ++i) unpack2(v[i], f[2 * i], f[2 * i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = i < left ? __uint_as_float((unsigned)p[i] << 16) : 0.f;
    }
}
__device__ __forceinline__ void store8h(uint16_t* p, int left, const float (&f)[8])
{
    u4_t v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(unsigned, bf16x2{(__bf16)f[2 * i], (__bf16)f[2 * i + 1]});
    if (left >= 8) { *(u4_t*)p = v; return; }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) p[i] = (uint16_t)(v[i / 2] >> (16 * (i & 1)));
}
__device__ __forceinline__ void load8c(const uint8_t* p, int left, unsigned& lo, unsigned& hi)
{
    if (left >= 8) { const u2_t v = get<true>((const u2_t*)p); lo = v[0]; hi = v[1]; return; }
    lo = hi = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) (i < 4 ? lo : hi) |= (unsigned)p[i] << (8 * (i & 3));
}
__device__ __forceinline__ void store8c(uint8_t* p, int left, unsigned lo, unsigned hi)
{
    if (left >= 8) { put<true>((u2_t*)p, u2_t{lo, hi}); return; }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) p[i] = (uint8_t)((i < 4 ? lo : hi) >> (8 * (i & 3)));
}

// Largest over the 16 lanes that share a scale, in each of them; a NaN stays one.
template <int CTRL> __device__ __forceinline__ float max_with(float m)
{
    return max3_abs(m, m, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(m), CTRL, 0xF, 0xF, true)));
}
__device__ __forceinline__ float group_max(float m)
{
    m = max_with<0x121>(m);      // row_ror:1, 2, 4, 8
    m = max_with<0x122>(m);
    m = max_with<0x124>(m);
    return max_with<0x128>(m);
}
// The scale that takes `largest` to `most`, and its reciprocal; none for a group below the normal numbers.
__device__ __forceinline__ float group_scale(float largest, float one_over_most, float& inverse)
{
    float s = largest * one_over_most;
    s = s < 0x1p-126f ? 0.f : s;
    inverse = s == 0.f ? 0.f : __fdiv_rn(1.f, s);
    return s;
}

__device__ __forceinline__ unsigned root_code(float t, unsigned rnd16)
{
    const unsigned c = (__float_as_uint(t * 0x1p-112f) + (rnd16 << 3)) >> 19;
    return t > 0.f ? (c < 1u ? 1u : c > 255u ? 255u : c) : 0u;
}
__device__ __forceinline__ float root_value(unsigned c) { return __uint_as_float(c << 19) * 0x1p112f; }

template <bool SMALL>
__global__ __launch_bounds__(kStepThreads) void adamw_step_kernel(const AdamwStepArgs a)
{
#pragma clang fp contract(off)
    const int lane = threadIdx.x & 63;
    const unsigned my_first = a.first[lane < kStepTensors ? lane : kStepTensors - 1];
    const float gs = a.grad_scale ? *a.grad_scale : 1.f;
    for (unsigned chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
        // the last tensor that starts at or before this chunk
        const unsigned long long before = __builtin_amdgcn_ballot_w64(lane < a.count && my_first <= chunk);
        const int at = 63 - __builtin_clzll(before);
        const AdamwStepTensor& t = a.t[at];
        const int64_t base = (int64_t)(chunk - a.first[at]) * kStepChunk;
        const int64_t e = base + threadIdx.x * 8;
        if (e - lane * 8 < t.n) {                                              // wave-uniform
            const int64_t rest = t.n - e;
            const int left = rest >= 8 ? 8 : rest > 0 ? (int)rest : 0;
            const int64_t at8 = left > 0 ? e : 0;
            float p[8], g[8], m[8], v[8];
            load8f<SMALL>(t.p + at8, left, p);
            if (t.g_bf16) load8h<SMALL>((const uint16_t*)t.g + at8, left, g);
            else          load8f<SMALL>((const float*)t.g + at8, left, g);
            if (SMALL) {
                unsigned mc[2], vc[2];
                load8c((const uint8_t*)t.m + at8, left, mc[0], mc[1]);
                load8c((const uint8_t*)t.v + at8, left, vc[0], vc[1]);
                const float ms = t.m_scale[at8 >> 7], vs = t.v_scale[at8 >> 7];
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    const float2_t d = (i & 2) ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(mc[i / 4], 1.f, true)
                                               : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(mc[i / 4], 1.f, false);
                    m[i] = d[0] * ms;
                    m[i + 1] = d[1] * ms;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float r = root_value((vc[i / 4] >> (8 * (i & 3))) & 0xFFu) * vs;
                    v[i] = r * r;
                }
            } else {
                load8f<SMALL>((const float*)t.m + at8, left, m);
                load8f<SMALL>((const float*)t.v + at8, left, v);
            }
            float r[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float gi = g[i] * gs;
                m[i] = a.beta1 * m[i] + a.rest1 * gi;
                v[i] = a.beta2 * v[i] + a.rest2 * (gi * gi);
                r[i] = __builtin_sqrtf(v[i]);
                p[i] = p[i] * t.keep - __fdiv_rn(a.step_size * m[i], r[i] * a.root_scale + a.eps);
            }
            store8f<SMALL>(t.p + at8, left, p);
            if (t.copy) store8h(t.copy + at8, left, p);
            if (SMALL) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i >= left) m[i] = r[i] = 0.f;
                float mi, ri;
                const float ms = group_scale(group_max(max_abs<8>(m)), (float)(1.0 / 448.0), mi);
                const float vs = group_scale(group_max(max_abs<8>(r)), (float)(1.0 / 1.9375), ri);
                unsigned mc[2], vc[2] = {0, 0}, o[4];
                const uint64_t quad = (uint64_t)at8 >> 2;
                threefry2x32_20((unsigned)quad, t.index, a.seed.x, a.seed.y, o[0], o[1]);
                threefry2x32_20((unsigned)quad + 1, t.index, a.seed.x, a.seed.y, o[2], o[3]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    m[i] *= mi;
                    vc[i / 4] |= root_code(r[i] * ri, (i & 1) ? o[i / 2] >> 16 : o[i / 2] & 0xFFFFu) << (8 * (i & 3));
                }
                mc[0] = enc8x4<0>(m, 1.f, 127);
                mc[1] = enc8x4<0>(m + 4, 1.f, 127);
                if (left > 0) {
                    store8c((uint8_t*)t.m + at8, left, mc[0], mc[1]);
                    store8c((uint8_t*)t.v + at8, left, vc[0], vc[1]);
                    if ((lane & 15) == 0) { t.m_scale[at8 >> 7] = ms; t.v_scale[at8 >> 7] = vs; }
                }
            } else {
                store8f<SMALL>((float*)t.m + at8, left, m);
                store8f<SMALL>((float*)t.v + at8, left, v);
            }
        }
    }
}

}  // namespace

int64_t adamw_step_chunks(int64_t n) { return (n + kStepChunk - 1) / kStepChunk; }

hipError_t launch_adamw_step(const AdamwStepArgs& a, bool small, hipStream_t s)
{
    if (a.chunks == 0) return hipSuccess;
    const dim3 grid((unsigned)(a.chunks < kMostBlocks ? a.chunks : kMostBlocks));
    if (small) hipLaunchKernelGGL(adamw_step_kernel<true>, grid, dim3(kStepThreads), 0, s, a);
    else       hipLaunchKernelGGL(adamw_step_kernel<false>, grid, dim3(kStepThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace snip
