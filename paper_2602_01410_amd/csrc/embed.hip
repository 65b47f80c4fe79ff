// Rows of an embedding, and their gradient summed over the tokens in sorted order.
//     y[t] = scale w[ids[t]]            dw[v] = scale sum over t with ids[t] = v of dy[t]   (+ what dw holds)
// Both move bytes and do nothing else: T rows read and written; T rows of dy read and the table's gradient written.
//
// The gradient is formed without atomics on memory, so that its sums have one order.  Few tokens find each other themselves (embed_few_kernel); more take three
// launches (16384 tokens of 4096 columns into fp32 [32000]: 17 + 143 + 9 us; 658 MB, of which a fill alone would store the 524 of the table in 76 us):
//   sort      a workgroup for each range of token numbers looks through all of ids twice: it counts its numbers (and those below its
//             range, which gives its place in the order), then puts the places of its tokens in order.  A wave takes a stretch of ids, so
//             tokens of one number stay in their order.  T * ranges reads, from L2: 16384 ids of 8 bytes and 250 ranges are 65 MB.  Latency bounds it: one read of
//             the ids, counts in LDS, sums over waves and numbers, places.  Beyond, the reads do, which grow with tokens x numbers: 65536 x 128000 46 us of 133 for rows of 512
//             columns, 2^20 x 256000 1550 of 1950, where an order by digits, which reads them a few times in all, would be the better one.
//   rows      parts of the rows with more than kLong tokens (the most frequent words, a tenth of a text each), kLong tokens at a time and first, so that they run
//             beside the rest (launched before it they took 20 us of their own); and a wave for each 512 columns of every other row of the table: zeros, or the sum of
//             its tokens; where the gradient is added to, of the rows that have tokens.  Memory bounds it: 4.6 TB/s.  A wave that takes 2 to 8 segments of its row one
//             after the other: 148 to 196 us, against 144 of this form at that time, stores past the caches 205.
//   long      long rows from their parts: a chain of five loads.
#include "snip_internal.h"
#include "quant_common.h"
#include <type_traits>

namespace snip {
namespace {

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kMostRange = 512;          // token numbers of a workgroup of the sort
constexpr int kLong = 64;                // tokens of a row from which on it is summed in parts, and the tokens of a part
constexpr int kHeld = 16;                // loads of 64 ids that a wave of the sort has under way; up to 64 of them for each wave ids are read once
constexpr int kSegment = 512;            // columns of a wave: 8 per lane
// Up to so many tokens a workgroup of every token looks for the others itself.  Added to 32000 x 4096, us, here and sorted: 16 tokens 2.9 and 11, 1003 8.3 and 17
// (all of one number 9.5 and 18), 2048 18 and 25 (11 and 22); 4096 (without the list's limit) 93 and 38.
constexpr int kFewTokens = 2048;

template <bool I64> __device__ __forceinline__ int token(const void* ids, int64_t t, int vocab)      // -1: none
{
    if (I64) {
        const int64_t v = ((const int64_t*)ids)[t];
        return v >= 0 && v < vocab ? (int)v : -1;
    }
    const int v = ((const int*)ids)[t];
    return v >= 0 && v < vocab ? v : -1;
}

__device__ __forceinline__ void load8(const float* p, float (&f)[8])
{
    const float4 a = ((const float4*)p)[0], b = ((const float4*)p)[1];
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ __forceinline__ void load8(const uint16_t* p, float (&f)[8])
{
    const uint4 v = *(const uint4*)p;
    unpack2(v.x, f[0], f[1]); unpack2(v.y, f[2], f[3]); unpack2(v.z, f[4], f[5]); unpack2(v.w, f[6], f[7]);
}
__device__ __forceinline__ void store8(float* p, const float (&f)[8])
{
    ((float4*)p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    ((float4*)p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ unsigned pack2(float a, float b) { return __builtin_bit_cast(unsigned, bf16x2{(__bf16)a, (__bf16)b}); }
__device__ __forceinline__ void store8(uint16_t* p, const float (&f)[8])
{
    *(uint4*)p = make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
}

// `lanes` (64 or 256) threads share a row.  Bound by memory: 16384 rows of 4096 in fp32 52 us, 403 MB with rows that come again from caches; one row 2.1 us, a launch
// and two loads in turn.
template <class T, bool I64>
__global__ __launch_bounds__(256) void embed_kernel(const T* __restrict__ w, int vocab, int cols, int64_t ldw, const void* __restrict__ ids,
                                                    int64_t tokens, float scale, uint16_t* __restrict__ y, int64_t ldy, int lanes)
{
    const int per = 256 / lanes, me = threadIdx.x % lanes;
    for (int64_t t = (int64_t)blockIdx.x * per + threadIdx.x / lanes; t < tokens; t += (int64_t)gridDim.x * per) {
        const int v = token<I64>(ids, t, vocab);
        const T* row = w + (int64_t)(v < 0 ? 0 : v) * ldw;
#pragma unroll 4
        for (int c = me * 8; c < cols; c += lanes * 8) {
            float f[8];
            load8(row + c, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = v < 0 ? 0.f : f[i] * scale;
            store8(y + t * ldy + c, f);
        }
    }
}

// start[v]: place in `order` of the first token of number v, start[vocab] the number of tokens that have one.
template <bool I64>
__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(const void* __restrict__ ids, int tokens, int vocab, int range,
                                                                  int* __restrict__ start, int* __restrict__ order)
{
    __shared__ int counts[kSortWaves][kMostRange];
    __shared__ int sums[kSortWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int base = blockIdx.x * range, here = vocab - base < range ? vocab - base : range;
    const int64_t stretch = ((int64_t)tokens + kSortThreads - 1) / kSortThreads * 64;
    const int64_t from = wave * stretch, to = from + stretch < tokens ? from + stretch : tokens;
    for (int i = threadIdx.x; i < kSortWaves * range; i += kSortThreads) counts[i / range][i % range] = 0;
    __syncthreads();
    int below = 0;
    int held[kHeld];
    auto fetch = [&](int64_t t0) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int64_t t = t0 + i * 64 + lane;
            held[i] = t < to ? token<I64>(ids, t, vocab) : -1;
        }
    };
    for (int64_t t0 = from; t0 < to; t0 += kHeld * 64) {
        fetch(t0);
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int v = held[i];
            below += v >= 0 && v < base;
            if (v >= base && v - base < here) atomicAdd(&counts[wave][v - base], 1);
        }
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) below += __shfl_xor(below, d);
    if (lane == 0) sums[wave] = below;
    __syncthreads();
    int first = 0;
#pragma unroll
    for (int i = 0; i < kSortWaves; ++i) first += sums[i];
    __syncthreads();
    // places: all numbers below, then within a number the waves in turn (range <= kSortThreads)
    const int me = threadIdx.x;
    int total = 0;
    if (me < range)
        for (int i = 0; i < kSortWaves; ++i) total += counts[i][me];
    int inc = total;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(inc, d);
        if (lane >= d) inc += o;
    }
    if (lane == 63) sums[wave] = inc;
    __syncthreads();
    int at = first + inc - total;
    for (int i = 0; i < wave; ++i) at += sums[i];
    if (me < here) {
        start[base + me] = at;
        if (base + me == vocab - 1) start[vocab] = at + total;
        for (int i = 0; i < kSortWaves; ++i) {
            const int n = counts[i][me];
            counts[i][me] = at;
            at += n;
        }
    }
    __syncthreads();
    for (int64_t t0 = from; t0 < to; t0 += kHeld * 64) {
        if (stretch > kHeld * 64) fetch(t0);
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int v = held[i];
            const bool mine = v >= base && v - base < here;
            // of the lanes of one number: the first one, the number of them, this one's place among them
            int lead = lane, many = 0, rank = 0;
            unsigned long long left = __builtin_amdgcn_ballot_w64(mine);
            while (left) {
                const int l = __builtin_ctzll(left);
                const bool same = mine && v == __builtin_amdgcn_readlane(v, l);
                const unsigned long long with = __builtin_amdgcn_ballot_w64(same);
                if (same) { lead = l; many = __builtin_popcountll(with); rank = __builtin_popcountll(with & ((1ull << lane) - 1)); }
                left &= ~with;
            }
            // (LDS serves a wave in order, so nothing waits for the place of the numbers before)
            const int place = mine && lane == lead ? atomicAdd(&counts[wave][v - base], many) : 0;
            const int at = __shfl(place, lead) + rank;
            if (mine) order[at] = (int)(t0 + i * 64 + lane);
        }
    }
}

// Eight columns of a lane: from a on, or (APART) four from a and four from b on, so that a wave's stores of fp32 are whole runs (136 us
// and 144, in turn on one machine).
struct Columns { int a, b; };
template <bool APART> __device__ __forceinline__ uint4 load_row(const uint16_t* row, Columns c)
{
    if (!APART) return *(const uint4*)(row + c.a);
    const uint2 lo = *(const uint2*)(row + c.a), hi = *(const uint2*)(row + c.b);
    return make_uint4(lo.x, lo.y, hi.x, hi.y);
}

// Sum of dy's rows order[from ... to), 64 of them at most, in their order.
template <int B, bool APART> __device__ __forceinline__ void sum_batch(const uint16_t* __restrict__ dy, int64_t ld, int rows, int i, Columns c, float (&sum)[8])
{
    uint4 raw[B];
#pragma unroll
    for (int b = 0; b < B; ++b) raw[b] = load_row<APART>(dy + (int64_t)__builtin_amdgcn_readlane(rows, i + b) * ld, c);
#pragma unroll
    for (int b = 0; b < B; ++b) {
        float f[8];
        unpack2(raw[b].x, f[0], f[1]); unpack2(raw[b].y, f[2], f[3]); unpack2(raw[b].z, f[4], f[5]); unpack2(raw[b].w, f[6], f[7]);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[k] += f[k];
    }
}
template <bool APART = false>
__device__ __forceinline__ void sum_rows(const uint16_t* __restrict__ dy, int64_t ld, const int* __restrict__ order, int from, int to, Columns c, float (&sum)[8])
{
    const int n = to - from, lane = threadIdx.x & 63;
    if (n == 0) return;
    const int rows = order[from + (lane < n ? lane : n - 1)];
    int i = 0;
    for (; i + 16 <= n; i += 16) sum_batch<16, APART>(dy, ld, rows, i, c, sum);
    if (n & 8) { sum_batch<8, APART>(dy, ld, rows, i, c, sum); i += 8; }
    if (n & 4) { sum_batch<4, APART>(dy, ld, rows, i, c, sum); i += 4; }
    if (n & 2) { sum_batch<2, APART>(dy, ld, rows, i, c, sum); i += 2; }
    if (n & 1) sum_batch<1, APART>(dy, ld, rows, i, c, sum);
}

// Sum of the places [j kLong, (j + 1) kLong) of the order, for the rows with more than kLong tokens: two of them at most have tokens there, that of the first
// place (partial sum 0) and, if it is another one, that of the last (1).
template <bool I64>
__device__ __forceinline__ void sum_part(const uint16_t* __restrict__ dy, int64_t ld, int cols, int vocab, const void* __restrict__ ids, const int* __restrict__ start,
                                         const int* __restrict__ order, int j, int c, float* __restrict__ partials)
{
    const int all = start[vocab], p0 = j * kLong, at = c < cols ? c : 0;      // (every lane holds a row's number)
    if (p0 >= all) return;
    const int p1 = all - p0 < kLong ? all : p0 + kLong;
    const int v0 = token<I64>(ids, order[p0], vocab), v1 = token<I64>(ids, order[p1 - 1], vocab);
#pragma unroll
    for (int slot = 0; slot < 2; ++slot) {
        const int v = slot ? v1 : v0;
        if (slot && v1 == v0) break;
        const int s = start[v], e = start[v + 1];
        if (e - s <= kLong) continue;
        float sum[8] = {};
        sum_rows(dy, ld, order, s > p0 ? s : p0, e < p1 ? e : p1, Columns{at, 0}, sum);
        if (c < cols) store8(partials + ((int64_t)j * 2 + slot) * cols + c, sum);
    }
}
template <class T> __device__ __forceinline__ void store_row(T* p, float (&sum)[8], float scale, bool add)
{
    float old[8] = {};
    if (add) load8(p, old);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = fmaf(sum[i], scale, old[i]);
    store8(p, sum);
}
__device__ __forceinline__ void store_half(float* p, const float* sum, float scale, bool add)
{
    const float4 old = add ? *(const float4*)p : make_float4(0.f, 0.f, 0.f, 0.f);
    *(float4*)p = make_float4(fmaf(sum[0], scale, old.x), fmaf(sum[1], scale, old.y), fmaf(sum[2], scale, old.z), fmaf(sum[3], scale, old.w));
}

// A wave for each 512 columns of `parts` parts of long rows and of, behind them, each row of the table or (BY_TOKEN, a gradient that is added to) each
// place in the order, which has something to do where a number's tokens begin.
template <class T, bool BY_TOKEN, bool I64>
__global__ __launch_bounds__(256) void embed_rows_kernel(const uint16_t* __restrict__ dy, int64_t ld, int cols, int vocab, int tokens, const void* __restrict__ ids, float scale,
                                                         const int* __restrict__ start, const int* __restrict__ order, float* __restrict__ partials, int parts,
                                                         T* __restrict__ dw, int64_t lddw, int segments)
{
    constexpr bool APART = sizeof(T) == 4;
    const int64_t units = ((int64_t)parts + (BY_TOKEN ? tokens : vocab)) * segments;
    for (int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); u < units; u += (int64_t)gridDim.x * 4) {
        int v = __builtin_amdgcn_readfirstlane((int)(u / segments));
        const int segment = (int)(u % segments) * kSegment, lane = threadIdx.x & 63;
        if (v < parts) { sum_part<I64>(dy, ld, cols, vocab, ids, start, order, v, segment + lane * 8, partials); continue; }
        v -= parts;
        if (BY_TOKEN) {
            const int place = v;
            if (place >= start[vocab]) continue;
            v = __builtin_amdgcn_readfirstlane(token<I64>(ids, order[place], vocab));
            if (start[v] != place) continue;
        }
        const int s = __builtin_amdgcn_readfirstlane(start[v]), e = __builtin_amdgcn_readfirstlane(start[v + 1]);
        if (e - s > kLong) continue;
        float sum[8] = {};
        T* row = dw + (int64_t)v * lddw;
        const int a = segment + lane * (APART ? 4 : 8), b = a + kSegment / 2;
        sum_rows<APART>(dy, ld, order, s, e, Columns{a < cols ? a : 0, b < cols ? b : 0}, sum);
        if constexpr (!APART) {
            if (a < cols) store_row(row + a, sum, scale, BY_TOKEN);
        } else {
            if (a < cols) store_half(row + a, sum, scale, BY_TOKEN);
            if (b < cols) store_half(row + b, sum + 4, scale, BY_TOKEN);
        }
    }
}

// The long rows from their partial sums: that which begins among the places of block j, if there is one; it goes on behind them.
template <class T, bool I64>
__global__ __launch_bounds__(64) void embed_long_kernel(int cols, int vocab, const void* __restrict__ ids, float scale, const int* __restrict__ start, const int* __restrict__ order,
                                                        const float* __restrict__ partials, T* __restrict__ dw, int64_t lddw, bool add)
{
    const int all = start[vocab], p0 = blockIdx.x * kLong, p1 = p0 + kLong, c = blockIdx.y * kSegment + threadIdx.x * 8;
    if (p1 >= all || c >= cols) return;
    const int v = token<I64>(ids, order[p1 - 1], vocab), s = start[v], e = start[v + 1], last = (e - 1) / kLong;
    if (s < p0 || e - s <= kLong) return;
    float sum[8] = {};
#pragma unroll 4
    for (int j = blockIdx.x; j <= last; ++j) {
        float f[8];
        load8(partials + ((int64_t)j * 2 + (j * kLong < s)) * cols + c, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += f[i];
    }
    store_row(dw + (int64_t)v * lddw + c, sum, scale, add);
}

// Few tokens: a workgroup for each token and 2048 columns looks through all ids itself and lists the tokens of its number in their order.  Up to kLong of
// them are summed by the first one's workgroup, a wave for each 512 columns.  Of more, every one's workgroup takes SLICE columns, and SLICE / 8 threads each
// kLong of the tokens, whose sums are added in turn.  The table is zero before, or added to.
template <class T, bool I64, int FEW>
__global__ __launch_bounds__(256) void embed_few_kernel(const uint16_t* __restrict__ dy, int64_t ld, int cols, int vocab, int tokens, const void* __restrict__ ids, float scale,
                                                        T* __restrict__ dw, int64_t lddw, bool add)
{
    constexpr int HELD = FEW / 256, GROUPS = FEW / kLong, SLICE = 256 / GROUPS * 8;
    __shared__ int list[FEW];
    __shared__ int counts[4], befores[4];
    __shared__ __attribute__((aligned(16))) float sums[GROUPS][SLICE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), me = blockIdx.x;
    const int v = token<I64>(ids, me, vocab);
    const unsigned long long lower = (1ull << lane) - 1;
    int held[HELD];
    auto place = [&](int i) { return wave * (FEW / 4) + i * 64 + lane; };
#pragma unroll
    for (int i = 0; i < HELD; ++i) held[i] = place(i) < tokens ? token<I64>(ids, place(i), vocab) : -1;
    if (v < 0) return;
    unsigned long long same[HELD];
    int n = 0, before = 0;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        same[i] = __builtin_amdgcn_ballot_w64(held[i] == v);
        n += __builtin_popcountll(same[i]);
        before += __builtin_popcountll(__builtin_amdgcn_ballot_w64(held[i] == v && place(i) < me));
    }
    if (lane == 0) { counts[wave] = n; befores[wave] = before; }
    __syncthreads();
    int at = 0, all = 0, rank = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        at += w < wave ? counts[w] : 0;
        all += counts[w];
        rank += befores[w];
    }
    if (all <= kLong ? rank != 0 : blockIdx.y != 0) return;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        if (same[i] >> lane & 1) list[at + __builtin_popcountll(same[i] & lower)] = place(i);
        at += __builtin_popcountll(same[i]);
    }
    __syncthreads();
    T* row = dw + (int64_t)v * lddw;
    if (all <= kLong) {
        const int c = (blockIdx.y * 4 + wave) * kSegment + lane * 8;
        float sum[8] = {};
        sum_rows(dy, ld, list, 0, all, Columns{c < cols ? c : 0, 0}, sum);
        if (c < cols) store_row(row + c, sum, scale, add);
        return;
    }
    const int group = threadIdx.x / (SLICE / 8), mine = threadIdx.x % (SLICE / 8) * 8, many = all - group * kLong < kLong ? all - group * kLong : kLong;
    for (int64_t c0 = (int64_t)rank * SLICE; c0 < cols; c0 += (int64_t)all * SLICE) {
        const int c = (int)c0 + mine;
        float sum[8] = {};
        if (c < cols)
            for (int i = 0; i < many; i += 16) {
                uint4 raw[16];
#pragma unroll
                for (int b = 0; b < 16; ++b) raw[b] = *(const uint4*)(dy + list[group * kLong + (i + b < many ? i + b : many - 1)] * ld + c);
#pragma unroll
                for (int b = 0; b < 16; ++b) {
                    float f[8];
                    unpack2(raw[b].x, f[0], f[1]); unpack2(raw[b].y, f[2], f[3]); unpack2(raw[b].z, f[4], f[5]); unpack2(raw[b].w, f[6], f[7]);
#pragma unroll
                    for (int k = 0; k < 8; ++k) sum[k] += i + b < many ? f[k] : 0.f;
                }
            }
        store8(&sums[group][mine], sum);
        __syncthreads();
        if (group == 0 && c < cols) {
            for (int g = 1; g < GROUPS && g * kLong < all; ++g) {
                float f[8];
                load8(&sums[g][mine], f);
#pragma unroll
                for (int k = 0; k < 8; ++k) sum[k] += f[k];
            }
            store_row(row + c, sum, scale, add);
        }
        __syncthreads();
    }
}

template <class T> __global__ __launch_bounds__(256) void embed_zero_kernel(T* __restrict__ dw, int64_t rows, int cols, int64_t ld)
{
    const float zero[8] = {};
    const int chunks = cols / 8;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < rows * chunks; u += (int64_t)gridDim.x * 256) store8(dw + u / chunks * ld + u % chunks * 8, zero);
}

int sort_range(int64_t vocab)
{
    int r = 16;
    while (r < kMostRange && r * 256 < vocab) r *= 2;
    return r;
}
size_t to256(size_t n) { return (n + 255) / 256 * 256; }
dim3 blocks_of(int64_t n) { return dim3((unsigned)(n < kMostBlocks ? n : kMostBlocks)); }

template <class T> hipError_t launch_grad(const EmbedGradArgs& a, T* dw, hipStream_t s)
{
    const int segments = (a.cols + kSegment - 1) / kSegment, parts = (int)((a.tokens + kLong - 1) / kLong);
    const int vocab = (int)a.vocab, tokens = (int)a.tokens;
    if (a.tokens <= kFewTokens) {
        if (!a.add) hipLaunchKernelGGL(embed_zero_kernel<T>, blocks_of((a.vocab * (a.cols / 8) + 255) / 256), dim3(256), 0, s, dw, a.vocab, a.cols, a.lddw);
        if (tokens > 0)
            hipLaunchKernelGGL((tokens <= kFewTokens / 2 ? a.ids64 ? embed_few_kernel<T, true, kFewTokens / 2> : embed_few_kernel<T, false, kFewTokens / 2>
                                                         : a.ids64 ? embed_few_kernel<T, true, kFewTokens> : embed_few_kernel<T, false, kFewTokens>),
                               dim3((unsigned)tokens, (unsigned)((segments + 3) / 4)), dim3(256), 0, s, a.dy, a.ld, a.cols, vocab, tokens, a.ids, a.scale, dw, a.lddw, a.add);
        return hipGetLastError();
    }
    uint8_t* ws = (uint8_t*)a.workspace;
    int* start = (int*)ws;
    int* order = (int*)(ws + to256((size_t)(a.vocab + 1) * 4));
    float* partials = (float*)(ws + to256((size_t)(a.vocab + 1) * 4) + to256((size_t)a.tokens * 4));
    const int range = sort_range(a.vocab);
    hipLaunchKernelGGL(a.ids64 ? embed_sort_kernel<true> : embed_sort_kernel<false>, dim3((unsigned)((a.vocab + range - 1) / range)), dim3(kSortThreads), 0, s,
                       a.ids, tokens, vocab, range, start, order);
    const dim3 grid = blocks_of(((parts + (a.add ? a.tokens : a.vocab)) * segments + 3) / 4);
    auto rows = [&](auto* kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a.dy, a.ld, a.cols, vocab, tokens, a.ids, a.scale, start, order, partials, parts, dw, a.lddw, segments); };
    if (a.add) a.ids64 ? rows(embed_rows_kernel<T, true, true>) : rows(embed_rows_kernel<T, true, false>);
    else       a.ids64 ? rows(embed_rows_kernel<T, false, true>) : rows(embed_rows_kernel<T, false, false>);
    hipLaunchKernelGGL((a.ids64 ? embed_long_kernel<T, true> : embed_long_kernel<T, false>), dim3((unsigned)parts, (unsigned)segments), dim3(64), 0, s, a.cols, vocab, a.ids, a.scale, start,
                       order, partials, dw, a.lddw, a.add);
    return hipGetLastError();
}

}  // namespace

// [vocab + 1] starts, [tokens] order, [blocks][2][cols] partial sums
size_t embed_workspace_bytes(int64_t tokens, int64_t cols, int64_t vocab)
{
    return to256((size_t)(vocab + 1) * 4) + to256((size_t)tokens * 4) + (size_t)((tokens + kLong - 1) / kLong) * 2 * (size_t)cols * 4;
}

hipError_t launch_embed(const EmbedArgs& a, hipStream_t s)
{
    if (a.tokens == 0) return hipSuccess;
    const int lanes = a.cols > 1024 ? 256 : 64;
    const int64_t blocks = (a.tokens + 256 / lanes - 1) / (256 / lanes);
    const dim3 grid((unsigned)(blocks < kMostBlocks ? blocks : kMostBlocks));
    auto go = [&](auto w, auto* kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, w, (int)a.vocab, a.cols, a.ldw, a.ids, a.tokens, a.scale, a.y, a.ldy, lanes); };
    if (a.w_fp32) go((const float*)a.w, a.ids64 ? embed_kernel<float, true> : embed_kernel<float, false>);
    else          go((const uint16_t*)a.w, a.ids64 ? embed_kernel<uint16_t, true> : embed_kernel<uint16_t, false>);
    return hipGetLastError();
}

hipError_t launch_embed_backward(const EmbedGradArgs& a, hipStream_t s)
{
    if (a.dw_fp32) return launch_grad(a, (float*)a.dw, s);
    return launch_grad(a, (uint16_t*)a.dw, s);
}

}  // namespace snip
