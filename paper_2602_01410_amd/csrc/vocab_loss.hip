// The loss over the vocabulary, softmax cross entropy or distillation from a teacher's top logits, and its gradients, without the logits
// ever being stored.  With z = x w^T, s = z / tau, q the wanted probabilities (one entry of 1, or softmax(teacher / tau) over k entries):
//     lse = log sum_v exp s_v      loss = tau^2 sum_j q_j (log q_j - s_idx_j + lse)
//     dz = dloss tau (exp(s - lse) - q)      dx = dz w      dw = dz^T x
//
// All of it is one matrix product in bf16 (v_mfma_f32_32x32x16_bf16, C[i][j] = sum_r A[i][r] B[j][r], both operands contiguous along r)
// with four ways to take the result out of the accumulators:
//   stats   A = w, B = x: of every token the tile's largest z and the sum of exp(s - largest), and z of the entries that the loss names;
//           a second kernel joins the tiles.  A token's logits lie in the registers of two lanes, so the sums need no shuffles.
//   dz      the same product anew, a piece of the vocabulary at a time: dz in bf16, as [token][entry] and as [entry][token]
//   dx      A = w^T of the piece, B = dz, split over the vocabulary where there are few tiles: partial sums in fp32, joined at the end
//   dw      A = x^T, B = dz^T
#include "gemm_common.h"
#include <algorithm>

namespace snip {
namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
enum Out { kStats, kDz, kDx, kDw };

struct Entries {                 // what the loss names, of every token
    const int* index;            // [tokens][pitch], -1: nothing
    const float* q;
    int k, pitch;
};

struct ProductArgs {
    const uint16_t *a, *b;
    int64_t lda, ldb;            // elements
    int I, J, R;
    int tiles_i, tiles_j, split; // stages of a split (blockIdx.y)
    float alpha;                 // 1 / tau
    Entries e;
    int v0, vocab;               // entry of A's first row
    float2* tile_stats;          // stats: [tiles_i][J]
    float* z;                    // stats: [J][pitch]
    const float* lse;            // dz
    const float* coef;           // dz: dloss tau of every token, zero for those that take no part
    uint16_t *dz, *dzt;          // dz: [J][lddz], [.][lddzt]
    int64_t lddz, lddzt;
    int jpad;                    // dz: columns of dzt to be written
    float* sum; int64_t ldsum, split_stride; int add;      // dx
    void* c; int64_t ldc; int c_fp32;                      // dw (and add)
};

// TM x TN outputs of a workgroup, WM x WN of a wave, NST stages of 64 contraction elements in LDS.
template <int TM_, int TN_, int WM_, int WN_, int NST_> struct Tile {
    static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, NST = NST_, MB = WM / 32, NB = WN / 32;
    static constexpr int WGM = TM / WM, WGN = TN / WN, NW = WGM * WGN, NT = NW * 64;
    static constexpr int SLOT = (TM + TN) * 128, LDS = NST * SLOT, COPIES = (TM + TN) / 8 / NW;      // 1 KB copies of a wave and stage
    static_assert((TM + TN) / 8 % NW == 0 && LDS <= 160 * 1024, "tile");
};

__device__ __forceinline__ unsigned pack2(float a, float b) { return __builtin_bit_cast(unsigned, bf16x2{(__bf16)a, (__bf16)b}); }
__device__ __forceinline__ uint16_t to_bf16(float a) { return __builtin_bit_cast(uint16_t, (__bf16)a); }

// Calls f(n, j, m, quad, part, entry) for every entry the loss names in this wave's block: of lane's column n the logit acc[m][4 quad + part].
template <class T, class F>
__device__ __forceinline__ void named(const Entries& e, int i_base, int j_base, int J, int r32, int g, F f)
{
#pragma unroll
    for (int n = 0; n < T::NB; ++n) {
        const int j = j_base + n * 32 + r32;
        const int* list = e.index + (int64_t)(j < J ? j : J - 1) * e.pitch;
        for (int x = 0; x < e.k; ++x) {
            const int at = list[x] - i_base;
            if (j < J && at >= 0 && at < T::WM && ((at >> 2) & 1) == g) f(n, j, x, at >> 5, ((at & 31) >> 3) * 4 + (at & 3));
        }
    }
}

template <class T, int OUT>
__global__ __launch_bounds__(T::NT) void product_kernel(const ProductArgs p)
{
    __shared__ __attribute__((aligned(1024))) uint8_t lds[T::LDS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / T::WGN, wn = wave % T::WGN, r32 = lane & 31, g = lane >> 5;
    int ti, tj;
    tile_of(blockIdx.x, p.tiles_i * p.tiles_j, p.tiles_i, p.tiles_j, ti, tj);
    const int i0 = ti * T::TM, j0 = tj * T::TN;
    const int all = (p.R + 63) / 64;
    const int first = OUT == kDx ? blockIdx.y * p.split : 0, last = OUT == kDx ? min(all, first + p.split) : all;

    const v4i ra = buffer_desc((const uint8_t*)(p.a + i0 * p.lda), (unsigned)(((min(T::TM, p.I - i0) - 1) * p.lda + p.R) * 2));
    const v4i rb = buffer_desc((const uint8_t*)(p.b + j0 * p.ldb), (unsigned)(((min(T::TN, p.J - j0) - 1) * p.ldb + p.R) * 2));
    const unsigned lds0 = lds_addr(lds);
    // copy c of this wave: 8 rows of 128 bytes
    unsigned off[T::COPIES];
    int chunk[T::COPIES];
#pragma unroll
    for (int c = 0; c < T::COPIES; ++c) {
        const int row = (wave * T::COPIES + c) * 8 + lane / 8;
        chunk[c] = (lane % 8) ^ ((row >> 1) & 7);
        off[c] = (unsigned)((row < T::TM ? row * p.lda : (row - T::TM) * p.ldb) * 2) + chunk[c] * 16;
    }
    auto issue = [&](int s) {
        const unsigned to = lds0 + (s - first) % T::NST * T::SLOT + wave * T::COPIES * 1024;
#pragma unroll
        for (int c = 0; c < T::COPIES; ++c) {
            const unsigned o = chunk[c] * 8 + s * 64 < p.R ? off[c] : kNoSource;
            if ((wave * T::COPIES + c) * 8 < T::TM) blds16(ra, o, s * 128, to + c * 1024);
            else                                    blds16(rb, o, s * 128, to + c * 1024);
        }
    };
    v16f acc[T::MB][T::NB];
#pragma unroll
    for (int m = 0; m < T::MB; ++m)
#pragma unroll
        for (int n = 0; n < T::NB; ++n)
#pragma unroll
            for (int k = 0; k < 16; ++k) acc[m][n][k] = 0.f;
#pragma unroll
    for (int s = 0; s < T::NST - 1; ++s)
        if (first + s < last) issue(first + s);
    for (int s = first; s < last; ++s) {
        // the copies of later stages that are under way
        if (last - s >= T::NST - 1) SNIP_WAIT_VM((T::NST - 2) * T::COPIES);
        else                        SNIP_WAIT_VM(0);
        SNIP_BAR();
        if (s + T::NST - 1 < last) issue(s + T::NST - 1);
        const uint8_t* slot = lds + (s - first) % T::NST * T::SLOT;
        const uint8_t* ta = slot + wm * T::WM * 128 + r32 * 128;
        const uint8_t* tb = slot + T::TM * 128 + wn * T::WN * 128 + r32 * 128;
        const int f = (r32 >> 1) & 7;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            bf16x8 fa[T::MB], fb[T::NB];
            const int at = ((ks * 2 + g) ^ f) * 16;
#pragma unroll
            for (int m = 0; m < T::MB; ++m) fa[m] = *reinterpret_cast<const bf16x8*>(ta + m * 32 * 128 + at);
#pragma unroll
            for (int n = 0; n < T::NB; ++n) fb[n] = *reinterpret_cast<const bf16x8*>(tb + n * 32 * 128 + at);
#pragma unroll
            for (int m = 0; m < T::MB; ++m)
#pragma unroll
                for (int n = 0; n < T::NB; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[m], fb[n], acc[m][n], 0, 0, 0);
        }
    }
    // In registers, lane (r32, g) of block (m, n) holds C[32 m + 8 q + 4 g + t][32 n + r32] in acc[m][n][4 q + t].
    const int iw = i0 + wm * T::WM, jw = j0 + wn * T::WN;

    if constexpr (OUT == kStats) {
        named<T>(p.e, p.v0 + iw, jw, p.J, r32, g, [&](int n, int j, int x, int m, int at) {
            float z = 0.f;
#pragma unroll
            for (int mm = 0; mm < T::MB; ++mm)
#pragma unroll
                for (int nn = 0; nn < T::NB; ++nn)
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        if (nn == n && mm == m && k == at) z = acc[mm][nn][k];
            p.z[(int64_t)j * p.e.pitch + x] = z;
        });
        if (iw + T::WM > p.I) {
#pragma unroll
            for (int m = 0; m < T::MB; ++m)
#pragma unroll
                for (int k = 0; k < 16; ++k)
                    if (iw + m * 32 + 8 * (k >> 2) + 4 * g + (k & 3) >= p.I) {
#pragma unroll
                        for (int n = 0; n < T::NB; ++n) acc[m][n][k] = -INFINITY;
                    }
        }
        __syncthreads();
        float2* shared = reinterpret_cast<float2*>(lds);             // [WGM][TN]
        const float c = p.alpha * kLog2e;
#pragma unroll
        for (int n = 0; n < T::NB; ++n) {
            float top = -INFINITY;
#pragma unroll
            for (int m = 0; m < T::MB; ++m)
#pragma unroll
                for (int k = 0; k < 16; ++k) top = fmaxf(top, acc[m][n][k]);
            top = fmaxf(top, __shfl_xor(top, 32));
            const float base = top == -INFINITY ? 0.f : top;
            float sum = 0.f;
#pragma unroll
            for (int m = 0; m < T::MB; ++m)
#pragma unroll
                for (int k = 0; k < 16; ++k) sum += __builtin_amdgcn_exp2f((acc[m][n][k] - base) * c);
            sum += __shfl_xor(sum, 32);
            if (g == 0) shared[wm * T::TN + wn * T::WN + n * 32 + r32] = make_float2(top, sum);
        }
        __syncthreads();
        for (int j = threadIdx.x; j < T::TN; j += T::NT) {
            if (j0 + j >= p.J) break;
            float2 v = shared[j];
#pragma unroll
            for (int w = 1; w < T::WGM; ++w) {
                const float2 o = shared[w * T::TN + j];
                const float top = fmaxf(v.x, o.x), base = top == -INFINITY ? 0.f : top;
                v = make_float2(top, v.y * __builtin_amdgcn_exp2f((v.x - base) * c) + o.y * __builtin_amdgcn_exp2f((o.x - base) * c));
            }
            p.tile_stats[(int64_t)ti * p.J + j0 + j] = v;
        }
    }
    if constexpr (OUT == kDz) {
#pragma unroll
        for (int n = 0; n < T::NB; ++n) {
            const int j = jw + n * 32 + r32;
            const float lse = j < p.J ? p.lse[j] : 0.f;
#pragma unroll
            for (int m = 0; m < T::MB; ++m)
#pragma unroll
                for (int k = 0; k < 16; ++k) acc[m][n][k] = __builtin_amdgcn_exp2f(fmaf(acc[m][n][k], p.alpha, -lse) * kLog2e);
        }
        named<T>(p.e, p.v0 + iw, jw, p.J, r32, g, [&](int n, int j, int x, int m, int at) {
            const float q = p.e.q[(int64_t)j * p.e.pitch + x];
#pragma unroll
            for (int mm = 0; mm < T::MB; ++mm)
#pragma unroll
                for (int nn = 0; nn < T::NB; ++nn)
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        if (nn == n && mm == m && k == at) acc[mm][nn][k] -= q;
        });
#pragma unroll
        for (int n = 0; n < T::NB; ++n) {
            const int j = jw + n * 32 + r32;
            const float coef = j < p.J ? p.coef[j] : 0.f;
#pragma unroll
            for (int m = 0; m < T::MB; ++m)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int i = iw + m * 32 + 8 * q + 4 * g;
                    float v[4];
#pragma unroll
                    for (int t = 0; t < 4; ++t) v[t] = coef == 0.f || i + t >= p.I ? 0.f : acc[m][n][4 * q + t] * coef;
                    if (j < p.J && i < p.lddz) *reinterpret_cast<uint2*>(p.dz + j * p.lddz + i) = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
                    if (p.dzt && j < p.jpad) {
#pragma unroll
                        for (int t = 0; t < 4; ++t)
                            if (i + t < p.I) p.dzt[(i + t) * p.lddzt + j] = to_bf16(v[t]);
                    }
                }
        }
    }
    if constexpr (OUT == kDx) {
        float* sum = p.sum + blockIdx.y * p.split_stride;
#pragma unroll
        for (int n = 0; n < T::NB; ++n) {
            const int j = jw + n * 32 + r32;
#pragma unroll
            for (int m = 0; m < T::MB; ++m)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int i = iw + m * 32 + 8 * q + 4 * g;
                    if (j >= p.J || i >= p.I) continue;                     // (I is a multiple of 8)
                    float4* to = reinterpret_cast<float4*>(sum + j * p.ldsum + i);
                    float4 v = make_float4(acc[m][n][4 * q], acc[m][n][4 * q + 1], acc[m][n][4 * q + 2], acc[m][n][4 * q + 3]);
                    if (p.add) {
                        const float4 o = *to;
                        v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
                    }
                    *to = v;
                }
        }
    }
    if constexpr (OUT == kDw) {
#pragma unroll
        for (int n = 0; n < T::NB; ++n) {
            const int j = jw + n * 32 + r32;
#pragma unroll
            for (int m = 0; m < T::MB; ++m)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int i = iw + m * 32 + 8 * q + 4 * g;
                    if (j >= p.J || i >= p.I) continue;
                    float4 v = make_float4(acc[m][n][4 * q], acc[m][n][4 * q + 1], acc[m][n][4 * q + 2], acc[m][n][4 * q + 3]);
                    if (p.c_fp32) {
                        float4* to = reinterpret_cast<float4*>((float*)p.c + j * p.ldc + i);
                        if (p.add) {
                            const float4 o = *to;
                            v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
                        }
                        *to = v;
                    } else {
                        uint2* to = reinterpret_cast<uint2*>((uint16_t*)p.c + j * p.ldc + i);
                        if (p.add) {
                            const uint2 o = *to;
                            v.x += __uint_as_float(o.x << 16); v.y += __uint_as_float(o.x & 0xFFFF0000u);
                            v.z += __uint_as_float(o.y << 16); v.w += __uint_as_float(o.y & 0xFFFF0000u);
                        }
                        *to = make_uint2(pack2(v.x, v.y), pack2(v.z, v.w));
                    }
                }
        }
    }
}

// What the loss names, a wave per token: entries (-1 where there is nothing: outside the vocabulary, or q = 0), q, the entropy term sum q log q,
// and for the gradient dloss tau, zero where no entry counts.
template <bool I64>
__global__ __launch_bounds__(256) void entries_kernel(const void* __restrict__ indices, const void* __restrict__ teacher, bool teacher_fp32, int tokens, int vocab,
                                                      int k, int pitch, float tau, const float* __restrict__ dloss, int* __restrict__ index, float* __restrict__ q,
                                                      float* __restrict__ entropy, float* __restrict__ coef)
{
    const int lane = threadIdx.x & 63;
    const float alpha = 1.f / tau;
    for (int t = blockIdx.x * 4 + (threadIdx.x >> 6); t < tokens; t += gridDim.x * 4) {
        auto number = [&](int j) {
            const int64_t v = I64 ? ((const int64_t*)indices)[(int64_t)t * k + j] : ((const int*)indices)[(int64_t)t * k + j];
            return v >= 0 && v < vocab ? (int)v : -1;
        };
        auto wanted = [&](int j) {
            if (!teacher) return 0.f;
            const int64_t at = (int64_t)t * k + j;
            return (teacher_fp32 ? ((const float*)teacher)[at] : __uint_as_float((unsigned)((const uint16_t*)teacher)[at] << 16)) * alpha;
        };
        float top = -INFINITY;
        bool any = false;
        for (int j = lane; j < k; j += 64)
            if (number(j) >= 0) {
                const float u = wanted(j);
                any = any || !(u == -INFINITY);
                top = fmaxf(top, u);
            }
        for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
        any = __builtin_amdgcn_ballot_w64(any) != 0;
        const float base = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
        for (int j = lane; j < k; j += 64)
            if (number(j) >= 0) sum += expf(wanted(j) - base);
        for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
        const float log_sum = logf(sum);
        float ent = 0.f;
        for (int j = lane; j < pitch; j += 64) {
            int v = j < k && any ? number(j) : -1;
            float w = 0.f;
            if (v >= 0) {
                const float l = wanted(j) - base - log_sum;
                w = expf(l);
                if (w == 0.f) v = -1;
                else ent += w * l;
            }
            index[(int64_t)t * pitch + j] = v;
            q[(int64_t)t * pitch + j] = w;
        }
        for (int d = 32; d > 0; d >>= 1) ent += __shfl_xor(ent, d);
        if (lane == 0) {
            if (entropy) entropy[t] = ent;
            if (coef) coef[t] = any ? (dloss ? dloss[t] : 1.f) * tau : 0.f;
        }
    }
}

// The tiles' sums joined and the loss formed: 16 tokens of a workgroup, 16 threads of a token.
__global__ __launch_bounds__(256) void join_kernel(const float2* __restrict__ tile_stats, int tiles, int tokens, float alpha, float tau, Entries e, const float* __restrict__ z,
                                                   const float* __restrict__ entropy, float* __restrict__ loss, float* __restrict__ lse)
{
    __shared__ float2 shared[16][17];
    const int tok = threadIdx.x & 15, part = threadIdx.x >> 4, t = blockIdx.x * 16 + tok;
    const float c = alpha * kLog2e;
    auto join = [&](float2 v, float2 o) {
        const float top = fmaxf(v.x, o.x), base = top == -INFINITY ? 0.f : top;
        return make_float2(top, v.y * __builtin_amdgcn_exp2f((v.x - base) * c) + o.y * __builtin_amdgcn_exp2f((o.x - base) * c));
    };
    float2 v = make_float2(-INFINITY, 0.f);
    if (t < tokens)
        for (int i = part; i < tiles; i += 16) v = join(v, tile_stats[(int64_t)i * tokens + t]);
    shared[part][tok] = v;
    __syncthreads();
    if (part != 0 || t >= tokens) return;
    for (int i = 1; i < 16; ++i) v = join(v, shared[i][tok]);
    const float l = fmaf(v.x, alpha, logf(v.y));
    if (lse) lse[t] = l;
    if (!loss) return;
    float sum = 0.f;
    bool any = false;
    for (int j = 0; j < e.k; ++j) {
        const int64_t at = (int64_t)t * e.pitch + j;
        if (e.index[at] >= 0) {
            sum = fmaf(e.q[at], fmaf(-z[at], alpha, l), sum);
            any = true;
        }
    }
    loss[t] = any ? (sum + entropy[t]) * tau * tau : 0.f;
}

// out[c][r] = in[r][c] of a bf16 matrix, zeros for r in [rows, rows_pad) (a multiple of 8, as cols is) and for rows whose `keep` is zero.
__global__ __launch_bounds__(256) void transpose_kernel(const uint16_t* __restrict__ in, int64_t ld, int rows, int cols, const float* __restrict__ keep, uint16_t* __restrict__ out,
                                                        int64_t ldo, int rows_pad)
{
    __shared__ uint16_t tile[64][66];
    const int r0 = blockIdx.x * 64, c0 = blockIdx.y * 64;
    for (int i = threadIdx.x; i < 64 * 8; i += 256) {
        const int r = i / 8, c = i % 8 * 8;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (r0 + r < rows && c0 + c < cols && !(keep && keep[r0 + r] == 0.f)) v = *reinterpret_cast<const uint4*>(in + (r0 + r) * ld + c0 + c);
        const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) *reinterpret_cast<unsigned*>(&tile[r][c + 2 * k]) = w[k];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 64 * 8; i += 256) {
        const int c = i / 8, r = i % 8 * 8;
        if (c0 + c >= cols || r0 + r >= rows_pad) continue;
        unsigned w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = tile[r + 2 * k][c] | (unsigned)tile[r + 2 * k + 1][c] << 16;
        *reinterpret_cast<uint4*>(out + (c0 + c) * ldo + r0 + r) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// dx: the partial sums of the splits, rounded; zeros for tokens that take no part.
__global__ __launch_bounds__(256) void dx_kernel(const float* __restrict__ sums, int splits, int64_t stride, int tokens, int cols, const float* __restrict__ coef,
                                                 uint16_t* __restrict__ dx, int64_t ld)
{
    const int chunks = cols / 8;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < (int64_t)tokens * chunks; u += (int64_t)gridDim.x * 256) {
        const int64_t t = u / chunks;
        const int c = (int)(u % chunks) * 8;
        float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (coef[t] != 0.f)
            for (int i = 0; i < splits; ++i) {
                const float4* s = reinterpret_cast<const float4*>(sums + i * stride + t * cols + c);
                const float4 a = s[0], b = s[1];
                f[0] += a.x; f[1] += a.y; f[2] += a.z; f[3] += a.w; f[4] += b.x; f[5] += b.y; f[6] += b.z; f[7] += b.w;
            }
        *reinterpret_cast<uint4*>(dx + t * ld + c) = make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
    }
}

template <bool FP32> __global__ __launch_bounds__(256) void zero_kernel(void* out, int64_t rows, int cols, int64_t ld)
{
    const int chunks = cols / 8;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < rows * chunks; u += (int64_t)gridDim.x * 256) {
        uint4* p = reinterpret_cast<uint4*>((uint8_t*)out + (u / chunks * ld + u % chunks * 8) * (FP32 ? 4 : 2));
        p[0] = make_uint4(0, 0, 0, 0);
        if (FP32) p[1] = make_uint4(0, 0, 0, 0);
    }
}

using Big = Tile<256, 256, 128, 64, 2>;
using Few = Tile<128, 32, 32, 32, 4>;

template <class T, int OUT> hipError_t launch_product(ProductArgs p, int splits, hipStream_t s)
{
    p.tiles_i = (p.I + T::TM - 1) / T::TM;
    p.tiles_j = (p.J + T::TN - 1) / T::TN;
    hipLaunchKernelGGL((product_kernel<T, OUT>), dim3((unsigned)(p.tiles_i * p.tiles_j), (unsigned)splits), dim3(T::NT), 0, s, p);
    return hipGetLastError();
}
template <int OUT> hipError_t pick_product(const ProductArgs& p, int splits, bool few, hipStream_t s)
{
    return few ? launch_product<Few, OUT>(p, splits, s) : launch_product<Big, OUT>(p, splits, s);
}

constexpr int64_t up(int64_t n, int64_t m) { return (n + m - 1) / m * m; }
size_t to256(size_t n) { return (n + 255) / 256 * 256; }
int64_t entries_pitch(int64_t k) { return k == 1 ? 1 : up(k, 4); }
bool few_tokens(int64_t tokens) { return tokens <= 64; }

// The backward call's pieces of the vocabulary and splits of dx.
struct Plan { int64_t tp, piece, splits; };
constexpr int64_t kPieceElements = 1 << 26, kLeastPiece = 4096, kMostPiece = 16384, kSplitElements = 1 << 25;
Plan plan_of(const VocabLossArgs& a)
{
    Plan r;
    r.tp = up(a.tokens, 32);
    r.piece = std::min(up(a.vocab, 256), std::min(kMostPiece, std::max(kLeastPiece, kPieceElements / r.tp / 256 * 256)));
    // splits: as long as the partial sums stay within kSplitElements, and of 512 entries at least
    r.splits = std::max<int64_t>(1, std::min(kSplitElements / (a.tokens * a.cols), r.piece / 512));
    return r;
}

struct Space {
    uint8_t* p;
    size_t used = 0;
    template <class T> T* take(size_t n)
    {
        T* r = (T*)(p + used);
        used += to256(n * sizeof(T));
        return r;
    }
};
struct Forward { int* index; float *q, *entropy, *z; float2* stats; size_t bytes; };
Forward forward_space(const VocabLossArgs& a)
{
    Space s{(uint8_t*)a.workspace};
    const size_t n = (size_t)a.tokens * entries_pitch(a.k), tm = few_tokens(a.tokens) ? Few::TM : Big::TM;
    Forward f;
    f.index = s.take<int>(n); f.q = s.take<float>(n); f.z = s.take<float>(n); f.entropy = s.take<float>(a.tokens);
    f.stats = s.take<float2>((a.vocab + tm - 1) / tm * a.tokens);
    f.bytes = s.used;
    return f;
}
struct Backward { int* index; float *q, *coef, *sums; uint16_t *xt, *wt, *dz, *dzt; size_t bytes; };
Backward backward_space(const VocabLossArgs& a, const Plan& pl)
{
    Space s{(uint8_t*)a.workspace};
    const size_t n = (size_t)a.tokens * entries_pitch(a.k);
    Backward b;
    b.index = s.take<int>(n); b.q = s.take<float>(n); b.coef = s.take<float>(a.tokens);
    b.xt = s.take<uint16_t>(a.cols * pl.tp); b.wt = s.take<uint16_t>(a.cols * pl.piece);
    b.dz = s.take<uint16_t>(a.tokens * pl.piece); b.dzt = s.take<uint16_t>(pl.piece * pl.tp);
    b.sums = s.take<float>((size_t)a.tokens * a.cols * pl.splits);
    b.bytes = s.used;
    return b;
}

void launch_entries(const VocabLossArgs& a, int* index, float* q, float* entropy, float* coef, hipStream_t s)
{
    const int64_t blocks = (a.tokens + 3) / 4;
    hipLaunchKernelGGL(a.index64 ? entries_kernel<true> : entries_kernel<false>, dim3((unsigned)(blocks < kMostBlocks ? blocks : kMostBlocks)), dim3(256), 0, s, a.indices, a.teacher,
                       a.teacher_fp32 != 0, (int)a.tokens, (int)a.vocab, (int)a.k, (int)entries_pitch(a.k), a.tau, a.dloss, index, q, entropy, coef);
}

}  // namespace

size_t vocab_loss_needed(const VocabLossArgs& a) { return forward_space(a).bytes; }
size_t vocab_loss_backward_needed(const VocabLossArgs& a) { return backward_space(a, plan_of(a)).bytes; }

// Bounds of the above that grow with every extent.
size_t vocab_loss_bytes(int64_t tokens, int64_t vocab, int64_t k)
{
    const size_t n = (size_t)tokens * entries_pitch(k);
    // the tiles of few tokens are half as high
    const size_t stats = std::max((size_t)((vocab + Few::TM - 1) / Few::TM) * std::min<int64_t>(tokens, 64), (size_t)((vocab + Big::TM - 1) / Big::TM) * tokens);
    return 3 * to256(n * 4) + to256((size_t)tokens * 4) + to256(stats * 8);
}
size_t vocab_loss_backward_bytes(int64_t tokens, int64_t cols, int64_t vocab, int64_t k)
{
    const size_t n = (size_t)tokens * entries_pitch(k);
    const int64_t tp = up(tokens, 32), vp = up(vocab, 256);
    const int64_t piece = std::min(vp, kMostPiece), dz = std::min(tp * piece, std::max(kPieceElements, tp * kLeastPiece));
    const int64_t sums = std::min(std::max(tokens * cols, kSplitElements), tokens * cols * std::max<int64_t>(1, piece / 512));
    return 2 * to256(n * 4) + to256((size_t)tokens * 4) + to256((size_t)(cols * tp) * 2) + to256((size_t)(cols * piece) * 2) + 2 * to256((size_t)dz * 2) + to256((size_t)sums * 4);
}

hipError_t launch_vocab_loss(const VocabLossArgs& a, hipStream_t s)
{
    if (a.tokens == 0) return hipSuccess;
    const Forward f = forward_space(a);
    launch_entries(a, f.index, f.q, f.entropy, nullptr, s);
    ProductArgs p = {};
    p.a = a.w; p.lda = a.ldw; p.I = (int)a.vocab; p.b = a.x; p.ldb = a.ldx; p.J = (int)a.tokens; p.R = (int)a.cols;
    p.alpha = 1.f / a.tau; p.e = {f.index, f.q, (int)a.k, (int)entries_pitch(a.k)}; p.vocab = (int)a.vocab;
    p.tile_stats = f.stats; p.z = f.z;
    const bool few = few_tokens(a.tokens);
    const hipError_t e = pick_product<kStats>(p, 1, few, s);
    if (e != hipSuccess) return e;
    const int tm = few ? Few::TM : Big::TM;
    hipLaunchKernelGGL(join_kernel, dim3((unsigned)((a.tokens + 15) / 16)), dim3(256), 0, s, f.stats, (int)((a.vocab + tm - 1) / tm), (int)a.tokens, p.alpha, a.tau, p.e, f.z, f.entropy,
                       a.loss, a.lse);
    return hipGetLastError();
}

hipError_t launch_vocab_loss_backward(const VocabLossArgs& a, hipStream_t s)
{
    if (a.tokens == 0 && !a.dw) return hipSuccess;
    if (a.tokens == 0) {
        const int64_t blocks = (a.vocab * (a.cols / 8) + 255) / 256;
        if (!a.add)
            hipLaunchKernelGGL(a.dw_fp32 ? zero_kernel<true> : zero_kernel<false>, dim3((unsigned)(blocks < kMostBlocks ? blocks : kMostBlocks)), dim3(256), 0, s, a.dw, a.vocab,
                               (int)a.cols, a.lddw);
        return hipGetLastError();
    }
    const Plan pl = plan_of(a);
    const Backward b = backward_space(a, pl);
    launch_entries(a, b.index, b.q, nullptr, b.coef, s);
    const bool few = few_tokens(a.tokens);
    auto transpose = [&](const uint16_t* in, int64_t ld, int64_t rows, const float* keep, uint16_t* out, int64_t ldo, int64_t pad) {
        hipLaunchKernelGGL(transpose_kernel, dim3((unsigned)((pad + 63) / 64), (unsigned)((a.cols + 63) / 64)), dim3(256), 0, s, in, ld, (int)rows, (int)a.cols, keep, out, ldo, (int)pad);
    };
    if (a.dw) transpose(a.x, a.ldx, a.tokens, b.coef, b.xt, pl.tp, pl.tp);
    hipError_t e = hipSuccess;
    for (int64_t v0 = 0; v0 < a.vocab && e == hipSuccess; v0 += pl.piece) {
        const int64_t here = std::min(pl.piece, a.vocab - v0), padded = up(here, 64);
        const uint16_t* w = a.w + v0 * a.ldw;
        ProductArgs p = {};
        p.a = w; p.lda = a.ldw; p.I = (int)here; p.b = a.x; p.ldb = a.ldx; p.J = (int)a.tokens; p.R = (int)a.cols;
        p.alpha = 1.f / a.tau; p.e = {b.index, b.q, (int)a.k, (int)entries_pitch(a.k)}; p.v0 = (int)v0; p.vocab = (int)a.vocab;
        p.lse = a.lse_in; p.coef = b.coef; p.dz = b.dz; p.lddz = pl.piece; p.dzt = a.dw ? b.dzt : nullptr; p.lddzt = pl.tp; p.jpad = (int)pl.tp;
        if ((e = pick_product<kDz>(p, 1, few, s)) != hipSuccess) break;
        if (a.dx) {
            transpose(w, a.ldw, here, nullptr, b.wt, pl.piece, padded);
            ProductArgs d = {};
            d.a = b.wt; d.lda = pl.piece; d.I = (int)a.cols; d.b = b.dz; d.ldb = pl.piece; d.J = (int)a.tokens; d.R = (int)padded;
            d.split = (int)((up(here, 64) / 64 + pl.splits - 1) / pl.splits);
            d.sum = b.sums; d.ldsum = a.cols; d.split_stride = a.tokens * a.cols; d.add = v0 > 0;
            if ((e = pick_product<kDx>(d, (int)pl.splits, few, s)) != hipSuccess) break;
        }
        if (a.dw) {
            ProductArgs d = {};
            d.a = b.xt; d.lda = pl.tp; d.I = (int)a.cols; d.b = b.dzt; d.ldb = pl.tp; d.J = (int)here; d.R = (int)pl.tp;
            d.c = a.dw_fp32 ? (void*)((float*)a.dw + v0 * a.lddw) : (void*)((uint16_t*)a.dw + v0 * a.lddw);
            d.ldc = a.lddw; d.c_fp32 = a.dw_fp32; d.add = a.add;
            e = pick_product<kDw>(d, 1, false, s);
        }
    }
    if (e != hipSuccess || !a.dx) return e;
    const int64_t blocks = (a.tokens * (a.cols / 8) + 255) / 256;
    hipLaunchKernelGGL(dx_kernel, dim3((unsigned)(blocks < kMostBlocks ? blocks : kMostBlocks)), dim3(256), 0, s, b.sums, (int)pl.splits, a.tokens * a.cols, (int)a.tokens, (int)a.cols,
                       b.coef, a.dx, a.lddx);
    return hipGetLastError();
}

}  // namespace snip
