// RMS norm with the residual's addition and quantized outputs, and its gradient.
//     h = bf16(x + r);   rstd = 1 / sqrt(mean(h^2) + eps);   y = h w rstd
// y is rounded once: to bf16, and from fp32 to the FP8 / FP4 codes of 32-element blocks along rows (the operand of the forward
// GEMM) or down columns (of the weight-gradient GEMM).  Bound by memory: 2 (4 with r) bytes per element read, 2 written for h,
// 1 or 0.5 for the codes of each orientation.
//
// Rows: a row's elements stay in registers between the sum of squares and the outputs, so x and r are read once.  Columns need
// the norms of 32 rows first: norm_col_kernel runs behind the row kernel and reads h again, with rstd.
//
// Measured (graph replays on three sets of tensors; bf16 x and residual, h stored), us and TB/s of the least bytes: [16384 x 4096] FP8 along rows 86 (5.4),
// down columns 111, both 126 (4.3), bf16 y 95 (5.6); [4096 x 2048] 13.2 (4.5), 18, 21 (3.2); [1 x 4096] 2.6; FP4 down columns 97 and 18, with
// FP8 along rows 116 and 20.6.  The row kernel is bound by memory from some thousand rows on, the column kernel (40 us of the 126 for 203 MB, FP4 34) by h's
// way back from the last-level cache, as far as it is there, and from memory; few rows by the launch and one chain load - sum - gain - store.  Widths
// off a multiple of 8 are read twice, the second time from cache, at two to three times the floor ([4096 x 9001] 79 us).  Loads that stream (past
// the caches) would keep h there but cost small calls their residual: [4096 x 2048] 13.1 -> 16.5.
#include "snip_internal.h"
#include "quant_common.h"

namespace snip {
namespace {

// Scale byte of a block by the bits of its largest magnitude in fp32; 0xFF for Inf/NaN.
template <int FMT>
__device__ __forceinline__ unsigned scale_byte_f32(unsigned amax, int rule)
{
    int b = (int)amax + ((rule == 0 ? 0x7FFFFF - ((int)Fmt<FMT>::mmax << 16) : 0) - (Fmt<FMT>::emax << 23));
    b = b < 0 ? 0 : b;
    return amax >= 0x7F800000u ? 0xFFu : (unsigned)b >> 23;
}

__device__ __forceinline__ unsigned pack_bf16(float lo, float hi)
{
    return __builtin_bit_cast(unsigned, bf16x2{(__bf16)lo, (__bf16)hi});
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8])
{
    return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}
__device__ __forceinline__ void unpack8(const uint4& v, float (&f)[8])
{
    unpack2(v.x, f[0], f[1]); unpack2(v.y, f[2], f[3]); unpack2(v.z, f[4], f[5]); unpack2(v.w, f[6], f[7]);
}

// Eight consecutive elements of a row from column `col` on, zeros from `cols` on.  RAGGED: cols is not a multiple of 8, and nothing
// behind the row's last element is touched; otherwise col + 8 <= cols.
template <bool RAGGED, bool NT = false>
__device__ __forceinline__ uint4 load8(const uint16_t* row, int64_t col, int64_t cols)
{
    if (NT) {
        const v4u_t v = __builtin_nontemporal_load(reinterpret_cast<const v4u_t*>(row + col));
        return make_uint4(v[0], v[1], v[2], v[3]);
    }
    if (!RAGGED || col + 8 <= cols) return *reinterpret_cast<const uint4*>(row + col);
    unsigned w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (col + i < cols) w[i / 2] |= (unsigned)row[col + i] << (16 * (i & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <bool RAGGED>
__device__ __forceinline__ void store8(uint16_t* row, int64_t col, int64_t cols, const uint4& v)
{
    if (!RAGGED || col + 8 <= cols) { *reinterpret_cast<uint4*>(row + col) = v; return; }
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (col + i < cols) row[col + i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
}
template <bool RAGGED>
__device__ __forceinline__ void load_gain(const void* gain, bool fp32, int64_t col, int64_t cols, float (&f)[8])
{
    if (!fp32) { unpack8(load8<RAGGED>((const uint16_t*)gain, col, cols), f); return; }
    const float* g = (const float*)gain + col;
    if (!RAGGED || col + 8 <= cols) {
        const float4 a = *reinterpret_cast<const float4*>(g), b = *reinterpret_cast<const float4*>(g + 4);
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = col + i < cols ? g[i] : 0.f;
    }
}

// y = (h w) rstd: with bf16 gains the first product is exact.
__device__ __forceinline__ float normed(float h, float w, float rstd) { return h * w * rstd; }

// Codes of a block's quarter (eight elements of a lane, a quad owns the block); returns the scale byte.
template <int FMT>
__device__ __forceinline__ unsigned quant_quarter(const float (&y)[8], int rule, unsigned& c0, unsigned& c1)
{
    const unsigned byte = scale_byte_f32<FMT>(quad_max(__float_as_uint(max_abs<8>(y))), rule);
    const float sc = scale_operand(byte);
    if (FMT == kFP8) {
        c0 = rule == 0 ? enc8x4<0>(y, sc, byte) : enc8x4<1>(y, sc, byte);
        c1 = rule == 0 ? enc8x4<0>(y + 4, sc, byte) : enc8x4<1>(y + 4, sc, byte);
    } else {
        c0 = enc4x8(y, sc);
        c1 = 0;
    }
    if (byte == 0xFFu) { c0 = 0; c1 = 0; }
    return byte;
}

__device__ __forceinline__ float rstd_of(float sum_sq, int cols, float eps) { return 1.f / __builtin_sqrtf(sum_sq / (float)cols + eps); }

// Outputs of eight elements of row `row`.  All lanes of a wave come here (a block's maximum is exchanged between lanes); those
// past the last column have zeros.
template <bool RAGGED>
__device__ __forceinline__ void norm_outputs(const NormArgs& a, int64_t row, int64_t col, const uint4& h, float rstd)
{
    float f[8], w[8];
    unpack8(h, f);
    const bool in = col < a.cols;
    if (in) load_gain<RAGGED>(a.gain, a.gain_fp32, col, a.cols, w);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = normed(f[i], w[i], rstd);
    if (a.y && in) store8<RAGGED>(a.y + row * a.ldy, col, a.cols, pack8(f));
    if (!RAGGED && a.codes_r) {                             // (its columns are a multiple of 32)
        unsigned c0, c1;
        const unsigned byte = a.fmt_r == kFP8 ? quant_quarter<kFP8>(f, a.rule, c0, c1) : quant_quarter<kFP4>(f, a.rule, c0, c1);
        const int64_t at = row * a.cols + col;
        if (in) {
            if (a.fmt_r == kFP8) *reinterpret_cast<uint2*>(a.codes_r + at) = make_uint2(c0, c1);
            else                 *reinterpret_cast<unsigned*>(a.codes_r + at / 2) = c0;
            if ((threadIdx.x & 3) == 0) a.scales_r[at / kBlock] = (uint8_t)byte;
        }
        if (a.g4_r) {
            // the bytes of four blocks, of this quad and the next three (zeros past the last column)
            unsigned p = in ? byte : 0u;
            p |= (unsigned)__builtin_amdgcn_update_dpp(0, (int)p, 0x104, 0xF, 0xF, true) << 8;        // lane + 4
            p |= (unsigned)__builtin_amdgcn_update_dpp(0, (int)p, 0x108, 0xF, 0xF, true) << 16;       // lane + 8
            if (in && (threadIdx.x & 15) == 0) *reinterpret_cast<unsigned*>(a.g4_r + ((col >> 7) * a.pitch_r + row) * 4) = p;
        }
    }
}

// One row by W waves, CH groups of eight elements per lane; cols is a multiple of 8.
template <int W, int CH>
__global__ __launch_bounds__(W == 1 ? 256 : W * 64) void norm_row_kernel(NormArgs a)
{
    constexpr int RPB = W == 1 ? 4 : 1;                     // rows a workgroup works on at a time
    __shared__ float sums[2][W];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane_in_row = W == 1 ? threadIdx.x & 63 : threadIdx.x;
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * RPB + (W == 1 ? wave : 0); row < a.rows; row += (int64_t)gridDim.x * RPB, turn ^= 1) {
        uint4 h[CH];
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int64_t col = ((int64_t)j * W * 64 + lane_in_row) * 8;
            h[j] = col < a.cols ? load8<false>(a.x + row * a.ldx, col, a.cols) : make_uint4(0, 0, 0, 0);
        }
        if (a.r) {
            uint4 r[CH];
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const int64_t col = ((int64_t)j * W * 64 + lane_in_row) * 8;
                r[j] = col < a.cols ? load8<false>(a.r + row * a.ldr, col, a.cols) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const int64_t col = ((int64_t)j * W * 64 + lane_in_row) * 8;
                float f[8], g[8];
                unpack8(h[j], f);
                unpack8(r[j], g);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] += g[i];
                h[j] = pack8(f);
                if (a.sum && col < a.cols) store8<false>(a.sum + row * a.lds, col, a.cols, h[j]);
            }
        }
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < CH; ++j) { acc_sq(h[j].x, s); acc_sq(h[j].y, s); acc_sq(h[j].z, s); acc_sq(h[j].w, s); }
        s = wave_sum(s);
        if (W > 1) {
            if ((threadIdx.x & 63) == 0) sums[turn][wave] = s;
            __syncthreads();                                // (the other half of `sums` may still be read)
            s = 0.f;
#pragma unroll
            for (int i = 0; i < W; ++i) s += sums[turn][i];
        }
        const float rstd = rstd_of(s, a.cols, a.eps);
        if (a.rstd && lane_in_row == 0) a.rstd[row] = rstd;
        if (a.y || a.codes_r)
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                if ((int64_t)j * W * 512 >= a.cols) break;
                norm_outputs<false>(a, row, ((int64_t)j * W * 64 + lane_in_row) * 8, h[j], rstd);
            }
    }
}

// The same for rows of any length, by W waves: read twice, the second time as stored or added again (and out of cache unless the
// row is very long).
template <int W, bool RAGGED>
__global__ __launch_bounds__(W * 64) void norm_any_row_kernel(NormArgs a)
{
    constexpr int STEP = W * 512;
    __shared__ float sums[2][W];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        float s = 0.f;
        auto element8 = [&](int64_t col, const uint16_t* r) {
            uint4 h = load8<RAGGED>(a.x + row * a.ldx, col, a.cols);
            if (r) {
                float f[8], g[8];
                unpack8(h, f);
                unpack8(load8<RAGGED>(r + row * a.ldr, col, a.cols), g);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] += g[i];
                h = pack8(f);
            }
            return h;
        };
        for (int64_t col = threadIdx.x * 8; col < a.cols; col += STEP) {
            const uint4 h = element8(col, a.r);
            if (a.sum) store8<RAGGED>(a.sum + row * a.lds, col, a.cols, h);
            acc_sq(h.x, s); acc_sq(h.y, s); acc_sq(h.z, s); acc_sq(h.w, s);
        }
        s = wave_sum(s);
        if ((threadIdx.x & 63) == 0) sums[turn][threadIdx.x >> 6] = s;
        __syncthreads();
        s = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) s += sums[turn][i];
        const float rstd = rstd_of(s, a.cols, a.eps);
        if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
        if (a.y || a.codes_r)
            for (int64_t c0 = 0; c0 < a.cols; c0 += STEP) {
                const int64_t col = c0 + threadIdx.x * 8;
                // a lane reads back what it has stored itself
                uint4 h = make_uint4(0, 0, 0, 0);
                if (col < a.cols) h = a.sum ? load8<RAGGED>(a.sum + row * a.lds, col, a.cols) : element8(col, a.r);
                norm_outputs<RAGGED>(a, row, col, h, rstd);
            }
    }
}

// Column blocks of y = h w rstd.  A workgroup's unit is 128 columns by one 128-byte line of every stored row (four row blocks
// of FP8 codes, eight of FP4); a wave takes a row block at a time, a lane two columns, so that a block's maximum stays in the
// lane.  The codes are turned through LDS and leave in whole lines.
template <int FMT>
__global__ __launch_bounds__(256) void norm_col_kernel(NormArgs a, const uint16_t* __restrict__ h, int64_t ldh)
{
    constexpr int RBU = FMT == kFP8 ? 4 : 8;                // row blocks of a unit
    constexpr int WORDS = FMT == kFP8 ? 8 : 4;              // dwords of codes of a block
    constexpr int CHUNKS = RBU * WORDS / 4;                 // 16-byte chunks of a stored row in the unit: 8
    __shared__ uint4 stage[128 * CHUNKS];
    __shared__ uint8_t bytes[RBU][128];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int cols = a.cols, ncg = (cols + 127) / 128, nrb = a.rows / kBlock;
    const int units = ncg * ((nrb + RBU - 1) / RBU);
    const int64_t out_row = FMT == kFP8 ? a.rows : a.rows / 2;
    for (int u = blockIdx.x; u < units; u += gridDim.x) {
        // from the end: the last rows of h are the ones most likely still in cache
        const int last = units - 1 - u, ru = last / ncg, c0 = (last - ru * ncg) * 128, c = c0 + 2 * lane;
        const int nb = min(nrb - ru * RBU, RBU);
        const bool in = c < cols;
        float w0 = 0.f, w1 = 0.f;
        if (in) {
            if (a.gain_fp32) { w0 = ((const float*)a.gain)[c]; w1 = ((const float*)a.gain)[c + 1]; }
            else unpack2(*((const unsigned*)a.gain + c / 2), w0, w1);
        }
        for (int k = wave; k < nb; k += 4) {
            const int64_t row0 = (int64_t)(ru * RBU + k) * kBlock;
            float y[2][32];
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const unsigned v = in ? __builtin_nontemporal_load(reinterpret_cast<const unsigned*>(h + (row0 + i) * ldh + c)) : 0u;
                unpack2(v, y[0][i], y[1][i]);
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const float rstd = a.rstd[row0 + i];
                y[0][i] = normed(y[0][i], w0, rstd);
                y[1][i] = normed(y[1][i], w1, rstd);
            }
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const unsigned byte = scale_byte_f32<FMT>(__float_as_uint(max_abs<32>(y[s])), a.rule);
                const float sc = scale_operand(byte);
                unsigned q[WORDS];
#pragma unroll
                for (int i = 0; i < WORDS; ++i) {
                    if (FMT == kFP8) q[i] = a.rule == 0 ? enc8x4<0>(y[s] + 4 * i, sc, byte) : enc8x4<1>(y[s] + 4 * i, sc, byte);
                    else             q[i] = enc4x8(y[s] + 8 * i, sc);
                    if (byte == 0xFFu) q[i] = 0;
                }
                // chunk i of stored row n lies at i ^ ((n / 2) & 7): lanes of a wave write to different banks
                uint4* const line = stage + (2 * lane + s) * CHUNKS;
#pragma unroll
                for (int i = 0; i < WORDS / 4; ++i)
                    line[(k * (WORDS / 4) + i) ^ (lane & 7)] = make_uint4(q[4 * i], q[4 * i + 1], q[4 * i + 2], q[4 * i + 3]);
                bytes[k][2 * lane + s] = (uint8_t)byte;
            }
        }
        __syncthreads();
#pragma unroll
        for (int it = 0; it < 128 * CHUNKS / 256; ++it) {
            const int n = it * (256 / CHUNKS) + threadIdx.x / CHUNKS, chunk = threadIdx.x % CHUNKS;
            if (c0 + n < cols && chunk / (WORDS / 4) < nb)
                *reinterpret_cast<uint4*>(a.codes_c + (c0 + n) * out_row + (int64_t)ru * 128 + chunk * 16) = stage[n * CHUNKS + (chunk ^ ((n >> 1) & 7))];
        }
        // scale bytes: a dword for four row blocks, zeros past the last one
        const int n = threadIdx.x & 127, g = threadIdx.x >> 7;
        if (g * 4 < nb && c0 + n < cols) {
            unsigned d = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (g * 4 + k < nb) d |= (unsigned)bytes[(g * 4 + k) & (RBU - 1)][n] << (8 * k);
            const int rb = ru * RBU + g * 4;
            uint8_t* const to = a.scales_c + (int64_t)(c0 + n) * nrb + rb;
            if ((nrb & 3) == 0) *reinterpret_cast<unsigned*>(to) = d;
            else
                for (int k = 0; k < 4 && rb + k < nrb; ++k) to[k] = (uint8_t)(d >> (8 * k));
            if (a.g4_c) *reinterpret_cast<unsigned*>(a.g4_c + ((int64_t)(rb / 4) * a.pitch_c + c0 + n) * 4) = d;
        }
        __syncthreads();
    }
}

template <int W, int CH> void launch_row(const NormArgs& a, hipStream_t s)
{
    const int64_t groups = W == 1 ? ((int64_t)a.rows + 3) / 4 : a.rows;
    constexpr int threads = W == 1 ? 256 : W * 64;
    hipLaunchKernelGGL((norm_row_kernel<W, CH>), dim3((unsigned)(groups < most_blocks(threads) ? groups : most_blocks(threads))), dim3(threads), 0, s, a);
}
template <int W, bool RAGGED> void launch_any_row(const NormArgs& a, hipStream_t s)
{
    hipLaunchKernelGGL((norm_any_row_kernel<W, RAGGED>), dim3((unsigned)(a.rows < most_blocks(W * 64) ? a.rows : most_blocks(W * 64))), dim3(W * 64), 0, s, a);
}

// ---- gradient ------------------------------------------------------------------------------------------------------------------
// With g = dy w and h normed by rstd:   dx = rstd (g - h rstd^2 mean(g h)) + dsum,   dw = sum over rows of dy h rstd.
// 6 (8 with dsum) bytes per element.  Measured with dsum, us and TB/s: [8192 x 8192] 98 (5.5), [16384 x 4096] 96 (5.6), [4096 x 2048] 16.1 (4.2);
// without [1501 x 2056] 10.2; [1 x 4096] 4.7, two launches; dx alone, without dsum, [1501 x 2056] 5.7 (with
// dw 10.1), [4096 x 2048] 10.3 (13.9).  Bound by memory where there are many rows.  A lane owns the same columns of every row
// that its workgroup takes, so that the sums of dw stay in registers until the workgroup's rows are done; then they go to a row of
// `partials`, and grad_sum_kernel adds those in a fixed order.

__device__ __forceinline__ void grad8(const float (&g)[8], const float (&h)[8], const uint4* dsum, float rstd, float coef, float (&dx)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) dx[i] = rstd * fmaf(-coef, h[i], g[i]);
    if (dsum) {
        float d[8];
        unpack8(*dsum, d);
#pragma unroll
        for (int i = 0; i < 8; ++i) dx[i] += d[i];
    }
}

template <int W, int CH, bool NT>
__global__ __launch_bounds__(W == 1 ? 256 : W * 64) void norm_grad_kernel(NormGradArgs a)
{
    constexpr int RPB = W == 1 ? 4 : 1;
    __shared__ float sums[2][W];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane_in_row = W == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int64_t first = (int64_t)blockIdx.x * RPB + (W == 1 ? wave : 0);
    float w[CH][8], dw[CH][8];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        const int64_t col = ((int64_t)j * W * 64 + lane_in_row) * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) w[j][i] = dw[j][i] = 0.f;
        if (col < a.cols) load_gain<false>(a.gain, a.gain_fp32, col, a.cols, w[j]);
    }
    int turn = 0;
    for (int64_t row = first; row < a.rows; row += (int64_t)gridDim.x * RPB, turn ^= 1) {
        const float rstd = a.rstd[row];
        uint4 vy[CH], vh[CH], vd[CH];
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int64_t col = ((int64_t)j * W * 64 + lane_in_row) * 8;
            const bool in = col < a.cols;
            vy[j] = vh[j] = vd[j] = make_uint4(0, 0, 0, 0);
            if (in) {
                vy[j] = load8<false, NT>(a.dy + row * a.lddy, col, a.cols);
                vh[j] = load8<false, NT>(a.h + row * a.ldh, col, a.cols);
                if (a.dsum) vd[j] = load8<false, NT>(a.dsum + row * a.ldds, col, a.cols);
            }
        }
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            float y[8], h[8];
            unpack8(vy[j], y);
            unpack8(vh[j], h);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s = fmaf(y[i] * w[j][i], h[i], s);
                dw[j][i] = fmaf(y[i], h[i] * rstd, dw[j][i]);
            }
        }
        s = wave_sum(s);
        if (W > 1) {
            if ((threadIdx.x & 63) == 0) sums[turn][wave] = s;
            __syncthreads();
            s = 0.f;
#pragma unroll
            for (int i = 0; i < W; ++i) s += sums[turn][i];
        }
        const float coef = s * rstd / (float)a.cols * rstd;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int64_t col = ((int64_t)j * W * 64 + lane_in_row) * 8;
            if (col >= a.cols) break;
            float y[8], h[8], dx[8];
            unpack8(vy[j], y);
            unpack8(vh[j], h);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] *= w[j][i];
            grad8(y, h, a.dsum ? &vd[j] : nullptr, rstd, coef, dx);
            store8<false>(a.dx + row * a.lddx, col, a.cols, pack8(dx));
        }
    }
    if (!a.partials) return;
    if (W == 1) {
        // the four rows' sums become one, in the order of the waves (those without a row have zeros); with a row of partial sums per wave [2048 x 512] took 11.4 us
        // and [16384 x 512] 19.5, now 6.5 and 15.3
        __shared__ float4 joined[W == 1 ? 3 : 1][CH][2][64];
        if (wave > 0)
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                joined[wave - 1][j][0][lane_in_row] = make_float4(dw[j][0], dw[j][1], dw[j][2], dw[j][3]);
                joined[wave - 1][j][1][lane_in_row] = make_float4(dw[j][4], dw[j][5], dw[j][6], dw[j][7]);
            }
        __syncthreads();
        if (wave > 0) return;
        for (int k = 0; k < 3; ++k)
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const float4 p = joined[k][j][0][lane_in_row], q = joined[k][j][1][lane_in_row];
                dw[j][0] += p.x; dw[j][1] += p.y; dw[j][2] += p.z; dw[j][3] += p.w;
                dw[j][4] += q.x; dw[j][5] += q.y; dw[j][6] += q.z; dw[j][7] += q.w;
            }
    }
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        const int64_t col = ((int64_t)j * W * 64 + lane_in_row) * 8;
        if (col >= a.cols) break;
        float4* const to = reinterpret_cast<float4*>(a.partials + blockIdx.x * a.pitch + col);
        to[0] = make_float4(dw[j][0], dw[j][1], dw[j][2], dw[j][3]);
        to[1] = make_float4(dw[j][4], dw[j][5], dw[j][6], dw[j][7]);
    }
}

// Rows of any length: read twice, the sums of dw kept in the workgroup's row of `partials`.
template <int W, bool RAGGED>
__global__ __launch_bounds__(W * 64) void norm_grad_any_kernel(NormGradArgs a)
{
    __shared__ float sums[2][W];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const float rstd = a.rstd[row];
        float s = 0.f;
        auto load_gh = [&](int64_t col, float (&y)[8], float (&h)[8], float (&w)[8]) {
            unpack8(load8<RAGGED>(a.dy + row * a.lddy, col, a.cols), y);
            unpack8(load8<RAGGED>(a.h + row * a.ldh, col, a.cols), h);
            load_gain<RAGGED>(a.gain, a.gain_fp32, col, a.cols, w);
        };
        for (int64_t col = threadIdx.x * 8; col < a.cols; col += W * 512) {
            float y[8], h[8], w[8];
            load_gh(col, y, h, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) s = fmaf(y[i] * w[i], h[i], s);
        }
        s = wave_sum(s);
        if ((threadIdx.x & 63) == 0) sums[turn][threadIdx.x >> 6] = s;
        __syncthreads();
        s = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) s += sums[turn][i];
        const float coef = s * rstd / (float)a.cols * rstd;
        for (int64_t col = threadIdx.x * 8; col < a.cols; col += W * 512) {
            float y[8], h[8], w[8], dx[8];
            load_gh(col, y, h, w);
            if (a.partials) {
                float4* const to = reinterpret_cast<float4*>(a.partials + blockIdx.x * a.pitch + col);       // (pitch is a multiple of 8)
                float4 t0 = make_float4(0.f, 0.f, 0.f, 0.f), t1 = t0;
                if (row != blockIdx.x) { t0 = to[0]; t1 = to[1]; }
                to[0] = make_float4(fmaf(y[0], h[0] * rstd, t0.x), fmaf(y[1], h[1] * rstd, t0.y), fmaf(y[2], h[2] * rstd, t0.z), fmaf(y[3], h[3] * rstd, t0.w));
                to[1] = make_float4(fmaf(y[4], h[4] * rstd, t1.x), fmaf(y[5], h[5] * rstd, t1.y), fmaf(y[6], h[6] * rstd, t1.z), fmaf(y[7], h[7] * rstd, t1.w));
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] *= w[i];
            uint4 d;
            if (a.dsum) d = load8<RAGGED>(a.dsum + row * a.ldds, col, a.cols);
            grad8(y, h, a.dsum ? &d : nullptr, rstd, coef, dx);
            store8<RAGGED>(a.dx + row * a.lddx, col, a.cols, pack8(dx));
        }
    }
}

// dw[c] = sum of partials[p][c] over p < n: 32 columns by 32 shares of the rows, added in a fixed order, the shares in double.
__global__ __launch_bounds__(1024) void grad_sum_kernel(const float* __restrict__ partials, int n, int64_t pitch, int cols, float* __restrict__ dw)
{
    __shared__ float shares[32][33];
    const int g = threadIdx.x >> 5;
    for (int c0 = blockIdx.x * 32; c0 < cols; c0 += gridDim.x * 32) {
        const int c = c0 + (threadIdx.x & 31);
        float s = 0.f;
        if (c < cols)
#pragma unroll 4
            for (int p = g; p < n; p += 32) s += partials[p * pitch + c];
        shares[g][threadIdx.x & 31] = s;
        __syncthreads();
        if (g == 0 && c < cols) {
            double t = 0.0;
            for (int i = 0; i < 32; ++i) t += shares[i][threadIdx.x];
            dw[c] = (float)t;
        }
        __syncthreads();
    }
}

// Waves of a row (0: rows are read twice, by 4 or 16 waves) and workgroups, by the numbers of columns and rows.
struct GradForm { int waves, groups, blocks; };
inline GradForm grad_form(int64_t rows, int64_t cols)
{
    const int64_t groups = (cols + 7) / 8;
    GradForm f;
    // us with fewer / more waves: 512 columns 1 / 4 rows 1024 5.3 / 6.7, 16384 15.3 / 31.0; 1024 columns 1 / 4 rows 64 5.2 / 4.9, 512 5.6 / 6.6, 16384 29.8 / 43.4;
    // 2048 columns 1 / 4 rows 64 6.4 / 5.2, 1024 9.7 / 9.1, 16384 54.8 / 53.6; two groups per lane of 4 waves / one of 8 [1 x 4096] 5.2 / 4.8, [1501 x 2056] 11.0 /
    // 10.2, [16384 x 4096] 98 / 94; four of 4 / one of 16 [1 x 8192] 6.4 / 5.4, [1024 x 8192] 19.6 / 17.7, [8192 x 8192] 98 / 99.
    f.waves = cols % 8 != 0 || groups > 2048 ? 0 : groups <= 64 || (groups <= 128 && rows > 256) ? 1 : groups <= 256 ? 4 : groups <= 512 ? 8 : 16;
    f.groups = groups > 1024 || (f.waves == 1 && groups > 64) ? 2 : 1;
    // Each workgroup's row of partial sums is written and read again: up to 512 of them (two workgroups per compute unit), 256 of 16 waves.  us with 256 /
    // 512: [4096 x 2048] 21.0 / 16.4, [1501 x 2056] 11.0 / 10.2, [16384 x 4096] 102 / 94; [16384 x 8192], 16 waves, 184.5 / 184.6, [4096 x 16384] 104 / 113.
    // Rows that are read twice wait for memory more often than they are limited by it: [4000 x 1001] 61 / 36 / 25.
    const int64_t most = f.waves == 0 ? (groups <= 1024 ? 1024 : 512) : f.waves == 16 ? 256 : 512, want = f.waves == 1 ? (rows + 3) / 4 : rows;
    f.blocks = (int)(want < most ? want : most);
    return f;
}
inline int64_t grad_pitch(int64_t cols) { return (cols + 7) / 8 * 8; }

}  // namespace

hipError_t launch_rms_norm(const NormArgs& a, hipStream_t s)
{
    if (a.rows == 0) return hipSuccess;
    const int groups = (a.cols + 7) / 8;
    // Waves and groups of eight per lane, by the columns and, where a row's own chain of latencies counts, by the rows.  us of row kernels with FP8
    // codes, fewer against more waves: [16384 x 512] 1 x 1 / 4 x 1 13.0 / 21.9; 1024 columns 1 x 2 / 4 x 1 rows 1 3.0 / 2.6, 512 3.6 / 3.3, 1024 3.9 /
    // 4.0, 16384 25.7 / 30.8; 2048 columns 1 x 4 / 4 x 1 rows 1 4.4 / 2.7, 1024 6.5 / 4.9, 16384 47.4 / 46.5; 4096 columns 4 x 2 / 8 x 1 rows 1 3.4 / 2.8, 512 5.5 /
    // 5.1, 2048 12.9 / 13.3; 8192 columns 8 x 2 / 16 x 1 (4 x 4) rows 1 3.5 / 3.3 (5.1), 512 8.4 / 8.0, 1024 12.9 / 13.9 (13.4), 16384 165 / 173 (166).  Read
    // twice, bf16 output, 4 / 16 waves: [1 x 4097] 5.3 / 4.0, [256 x 2049] 5.2 / 4.6, [512 x 2049] 6.1 / 7.3, [256 x 1001] 4.4 / 4.4, [4096 x 9001] 79 / 104,
    // [4096 x 20001] 164 / 160.
    const bool few = a.rows <= 512;
    if (a.cols % 8 != 0) {
        if (groups > 2048 || (groups > 128 && a.rows <= 256)) launch_any_row<16, true>(a, s);
        else                                                  launch_any_row<4, true>(a, s);
    }
    else if (groups <= 64) launch_row<1, 1>(a, s);
    else if (groups <= 128 && !few) launch_row<1, 2>(a, s);
    else if (groups <= 256) launch_row<4, 1>(a, s);
    else if (groups <= 512 && few) launch_row<8, 1>(a, s);
    else if (groups <= 512) launch_row<4, 2>(a, s);
    else if (groups <= 1024 && few) launch_row<16, 1>(a, s);
    else if (groups <= 1024) launch_row<8, 2>(a, s);
    else if (groups <= 2048) launch_row<16, 2>(a, s);
    else if (groups <= 4096) launch_row<16, 4>(a, s);
    else launch_any_row<16, false>(a, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.codes_c) return e;
    const uint16_t* h = a.r ? a.sum : a.x;
    const int64_t ldh = a.r ? a.lds : a.ldx;
    const int rbu = a.fmt_c == kFP8 ? 4 : 8;
    const int64_t units = (int64_t)((a.cols + 127) / 128) * ((a.rows / kBlock + rbu - 1) / rbu);
    const dim3 grid((unsigned)(units < kMostBlocks ? units : kMostBlocks));
    if (a.fmt_c == kFP8) hipLaunchKernelGGL(norm_col_kernel<kFP8>, grid, dim3(256), 0, s, a, h, ldh);
    else                 hipLaunchKernelGGL(norm_col_kernel<kFP4>, grid, dim3(256), 0, s, a, h, ldh);
    return hipGetLastError();
}

size_t norm_workspace_needed(int64_t rows, int64_t cols)
{
    return (size_t)grad_form(rows, cols).blocks * (size_t)grad_pitch(cols) * sizeof(float);
}
// The most that any call of at most these extents needs: 1024 workgroups up to 8192 columns (rows that are read twice), 512 beyond.
size_t norm_workspace_bytes(int64_t rows, int64_t cols)
{
    const int64_t narrow = (rows < 1024 ? rows : 1024) * (cols < 8192 ? grad_pitch(cols) : 8192), wide = (rows < 512 ? rows : 512) * grad_pitch(cols);
    return (size_t)(narrow > wide ? narrow : wide) * sizeof(float);
}

hipError_t launch_rms_norm_backward(NormGradArgs a, hipStream_t s)
{
    const GradForm f = grad_form(a.rows, a.cols);
    a.pitch = grad_pitch(a.cols);
    const dim3 grid(f.blocks);
    const bool wide = (a.cols + 7) / 8 > 1024;
    // Streaming loads where the call's tensors exceed the 256 MB of the last-level cache, in which the ones before left them otherwise: us [16384 x
    // 4096] (537 MB) 102 -> 97, [4096 x 2048] (67 MB) 20.6, with them 23.9.
    const bool streams = (int64_t)a.rows * a.cols * (a.dsum ? 8 : 6) > (int64_t)256 << 20;
#define SNIP_GRAD(W, CH) \
    do { \
        if (streams) hipLaunchKernelGGL((norm_grad_kernel<W, CH, true>), grid, dim3(W == 1 ? 256 : W * 64), 0, s, a); \
        else         hipLaunchKernelGGL((norm_grad_kernel<W, CH, false>), grid, dim3(W == 1 ? 256 : W * 64), 0, s, a); \
    } while (0)
    if (a.rows == 0) ;
    else if (f.waves == 0 && a.cols % 8 == 0) hipLaunchKernelGGL((norm_grad_any_kernel<16, false>), grid, dim3(1024), 0, s, a);
    else if (f.waves == 0 && wide) hipLaunchKernelGGL((norm_grad_any_kernel<16, true>), grid, dim3(1024), 0, s, a);
    else if (f.waves == 0) hipLaunchKernelGGL((norm_grad_any_kernel<4, true>), grid, dim3(256), 0, s, a);
    else if (f.waves == 1 && f.groups == 1) SNIP_GRAD(1, 1);
    else if (f.waves == 1) SNIP_GRAD(1, 2);
    else if (f.waves == 4) SNIP_GRAD(4, 1);
    else if (f.waves == 8) SNIP_GRAD(8, 1);
    else if (f.groups == 1) SNIP_GRAD(16, 1);
    else SNIP_GRAD(16, 2);
#undef SNIP_GRAD
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.dgain) return e;
    const int groups = (a.cols + 31) / 32, most = (int)most_blocks(1024);
    hipLaunchKernelGGL(grad_sum_kernel, dim3(groups < most ? groups : most), dim3(1024), 0, s, a.partials, f.blocks, a.pitch, a.cols, a.dgain);
    return hipGetLastError();
}

}  // namespace snip
