// Few tokens against quantized weights: y[t][n] = sum_k x[t][k] w[n][k] with x in bf16 as it is and w = code * 2^(scale - 127), FP4 or
// FP8 with a scale per 32 elements.  What a model answers with: every weight is read once for a handful of tokens, so the floor is
// the weights' bytes (0.53 or 1.03 per weight) over the memory's rate.
//
// Codes become bf16 (exact: at most four significant bits, the scale is a power of two) and go to v_mfma_f32_16x16x32_bf16 with fp32
// accumulators, 16 rows of w by 16 tokens at a time: on the vector unit four tokens would already take longer than the weights' way from
// memory.  A lane owns one block of 32 elements of one row (16 bytes of FP4, 32 of FP8) in each span of 128: the four lanes of a
// row take the span's four blocks, and matrix instruction j contracts elements 8 j .. 8 j + 7 of all four, for which a lane
// reads the same elements of x.  So a block has one lane's scale, codes come in the widest loads and nothing is exchanged.
// The waves of a workgroup share the rows and split the spans; their sums meet in LDS and are added in wave order.
#include "snip_internal.h"
#include "quant_common.h"

namespace snip {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ bf16x8 join(const bf16x2 (&p)[4])
{
    return bf16x8{p[0][0], p[0][1], p[1][0], p[1][1], p[2][0], p[2][1], p[3][0], p[3][1]};
}
// Elements 8 j .. 8 j + 7 of a lane's block.
template <int FMT> struct Block;
template <> struct Block<kFP4> {
    uint4 c;
    __device__ __forceinline__ void load(const uint8_t* p) { c = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void clear() { c = make_uint4(0, 0, 0, 0); }
    template <int J> __device__ __forceinline__ bf16x8 elements(float sc) const
    {
        const unsigned w = J == 0 ? c.x : J == 1 ? c.y : J == 2 ? c.z : c.w;
        const bf16x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 1),
                             __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 3)};
        return join(p);
    }
};
template <> struct Block<kFP8> {
    uint4 c, d;
    __device__ __forceinline__ void load(const uint8_t* p) { c = *reinterpret_cast<const uint4*>(p); d = *reinterpret_cast<const uint4*>(p + 16); }
    __device__ __forceinline__ void clear() { c = d = make_uint4(0, 0, 0, 0); }
    template <int J> __device__ __forceinline__ bf16x8 elements(float sc) const
    {
        const unsigned lo = J == 0 ? c.x : J == 1 ? c.z : J == 2 ? d.x : d.z, hi = J == 0 ? c.y : J == 1 ? c.w : J == 2 ? d.y : d.w;
        const bf16x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, sc, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, sc, true),
                             __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, sc, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, sc, true)};
        return join(p);
    }
};

// The sums of this wave's spans: acc[r][t] += rows 16 r .. of the workgroup's, tokens 16 t ...
template <int FMT, int TT, int RT>
__device__ __forceinline__ void gemv_spans(const GemvArgs& a, const GemvWeight& w, int row0, int token0, int wave, int waves, f32x4 (&acc)[RT][TT])
{
    const int lane = threadIdx.x & 63, quarter = lane >> 4;
    const int nb = a.k / kBlock, spans = (nb + 3) / 4;
    const uint8_t *codes[RT], *scales[RT];
    const uint16_t* x[TT];
    constexpr int BYTES = FMT == kFP4 ? 16 : 32;             // of a block
    // rows and tokens past the last one repeat it; what comes of them is not stored
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int64_t row = min(row0 + r * 16 + (lane & 15), w.n - 1);
        codes[r] = w.codes + row * nb * BYTES;
        scales[r] = w.scales + row * nb;
    }
#pragma unroll
    for (int t = 0; t < TT; ++t) x[t] = a.x + (int64_t)min(token0 + t * 16 + (lane & 15), a.m - 1) * a.ldx;
    for (int s = wave; s < spans; s += waves) {
        const int b = s * 4 + quarter;
        Block<FMT> c[RT];
        float sc[RT];
        bf16x8 v[TT][4];
        if (b < nb) {
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                c[r].load(codes[r] + (int64_t)b * BYTES);
                sc[r] = scale_operand(scales[r][b]);
            }
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) v[t][j] = *reinterpret_cast<const bf16x8*>(x[t] + b * kBlock + j * 8);
        } else {
            // a span that the row does not fill: nothing of x comes in either (it may be infinite)
#pragma unroll
            for (int r = 0; r < RT; ++r) { c[r].clear(); sc[r] = 1.f; }
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) v[t][j] = __builtin_bit_cast(bf16x8, make_uint4(0, 0, 0, 0));
        }
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const bf16x8 e[4] = {c[r].template elements<0>(sc[r]), c[r].template elements<1>(sc[r]), c[r].template elements<2>(sc[r]),
                                 c[r].template elements<3>(sc[r])};
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(e[j], v[t][j], acc[r][t], 0, 0, 0);
        }
    }
}

// Workgroup: 16 RT rows of one weight by 16 TT tokens, WS waves.
template <int TT, int RT, int WS>
__global__ __launch_bounds__(WS * 64) void gemv_kernel(const GemvArgs a)
{
    __shared__ f32x4 sums[WS][RT * TT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int i = 0;
    while (i + 1 < a.count && (int)blockIdx.x >= a.w[i + 1].first) ++i;
    const GemvWeight& w = a.w[i];
    const int row0 = ((int)blockIdx.x - w.first) * 16 * RT, token0 = blockIdx.y * 16 * TT;
    f32x4 acc[RT][TT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < TT; ++t) acc[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (w.fmt == kFP4) gemv_spans<kFP4, TT, RT>(a, w, row0, token0, wave, WS, acc);
    else               gemv_spans<kFP8, TT, RT>(a, w, row0, token0, wave, WS, acc);
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < TT; ++t) sums[wave][r * TT + t][lane] = acc[r][t];
    __syncthreads();
    for (int p = wave; p < RT * TT; p += WS) {
        f32x4 s = sums[0][p][lane];
#pragma unroll
        for (int k = 1; k < WS; ++k) s += sums[k][p][lane];
        const int row = row0 + p / TT * 16 + (lane >> 4) * 4, token = token0 + p % TT * 16 + (lane & 15);
        if (token >= a.m || row >= w.n) continue;
        if (a.out_fp32) {
            float* const to = (float*)w.y + token * w.ldy + row;
            if (row + 4 <= w.n) *reinterpret_cast<f32x4*>(to) = s;
            else
                for (int k = 0; k < 4 && row + k < w.n; ++k) to[k] = s[k];
        } else {
            uint16_t* const to = (uint16_t*)w.y + token * w.ldy + row;
            const uint2 q = make_uint2(__builtin_bit_cast(unsigned, bf16x2{(__bf16)s[0], (__bf16)s[1]}), __builtin_bit_cast(unsigned, bf16x2{(__bf16)s[2], (__bf16)s[3]}));
            if (row + 4 <= w.n) *reinterpret_cast<uint2*>(to) = q;
            else
                for (int k = 0; k < 4 && row + k < w.n; ++k) to[k] = (uint16_t)((k < 2 ? q.x : q.y) >> (16 * (k & 1)));
        }
    }
}

template <int TT, int RT, int WS> hipError_t launch(GemvArgs& a, hipStream_t s)
{
    int64_t blocks = 0;
    for (int i = 0; i < a.count; ++i) {
        a.w[i].first = (int)blocks;
        blocks += (a.w[i].n + 16 * RT - 1) / (16 * RT);
    }
    hipLaunchKernelGGL((gemv_kernel<TT, RT, WS>), dim3((unsigned)blocks, (a.m + 16 * TT - 1) / (16 * TT)), dim3(WS * 64), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_gemv(GemvArgs a, hipStream_t s)
{
    if (a.count == 0 || a.m == 0) return hipSuccess;
    if (a.m <= 16) return launch<1, 1, 4>(a, s);
    if (a.m <= 32) return launch<2, 1, 4>(a, s);
    return launch<4, 1, 4>(a, s);
}

}  // namespace snip
