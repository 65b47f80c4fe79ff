// Few tokens against quantized weights: y[t][n] = sum_k x[t][k] w[n][k] with x in bf16 as it is and w = code * 2^(scale - 127), FP4 or
// FP8 with a scale per 32 elements.  What a model answers with: every weight is read once for a handful of tokens, so the floor is
// the weights' bytes (0.53 or 1.03 per weight) over the memory's rate, 7.4 TB/s of reads.
//
// Codes become bf16 (exact down to 2^-126: at most four significant bits, the scale is a power of two) and go to v_mfma_f32_16x16x32_bf16 with fp32
// accumulators, 16 rows of w by 16 tokens at a time: on the vector unit four tokens would already take longer than the weights' way from
// memory.  A lane multiplies one block of 32 elements of one row (16 bytes of FP4, 32 of FP8) in each span of 128: the four lanes of a
// row take the span's four blocks, and matrix instruction j contracts elements 8 j .. 8 j + 7 of all four, for which a lane
// reads the same elements of x.  So a block has one lane and one scale.
//
// Measured (graph replays on four sets of weights), us per call and TB/s: FP4, one token 2 x [28672 x 8192] 50 (5.0), 3 x [4096 x 4096] 8.4 (3.2), [4096
// x 11008] 8.1 (3.0), [512 x 512] 2.3; 16, 32, 48, 64 tokens 2 x [28672 x 8192] 63, 63, 73, 82 (4.0, 4.0, 3.5, 3.1; on other machines 59 to 80 and 86); FP8, one token
// 85 (5.7), 48 tokens 109 (4.5).  One token is bound by memory's latency (8 waves on a compute unit, each with 4 KB under way, wait most of the time; twice as much under way is
// no faster), 48 tokens by LDS and matrix cores taking turns on a span (two waves per SIMD; every wave reads x of all tokens for its two row tiles, 96 KB per
// span and workgroup), small problems by the launch.
#include "snip_internal.h"
#include "quant_common.h"
#include "x_pieces.h"

namespace snip {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned u1_any __attribute__((aligned(1)));
constexpr int kSlot = 128 + 16;            // 16-byte units of LDS through which a wave's codes and scales go to their lanes

__device__ __forceinline__ bf16x8 join(const bf16x2 (&p)[4])
{
    return bf16x8{p[0][0], p[0][1], p[1][0], p[1][1], p[2][0], p[2][1], p[3][0], p[3][1]};
}
// Elements 8 j .. 8 j + 7 of a lane's block.
template <int FMT> struct Block;
template <> struct Block<kFP4> {
    v4u_t c;
    template <class F> __device__ __forceinline__ void get(F piece) { c = piece(0); }
    __device__ __forceinline__ void load(const uint8_t* p) { c = *reinterpret_cast<const v4u_t*>(p); }
    __device__ __forceinline__ void clear() { c = v4u_t{0, 0, 0, 0}; }
    template <int J> __device__ __forceinline__ bf16x8 elements(float sc) const
    {
        const unsigned w = c[J];
        const bf16x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 1),
                             __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 3)};
        return join(p);
    }
};
template <> struct Block<kFP8> {
    v4u_t c, d;
    template <class F> __device__ __forceinline__ void get(F piece) { c = piece(0); d = piece(1); }
    __device__ __forceinline__ void load(const uint8_t* p) { c = *reinterpret_cast<const v4u_t*>(p); d = *reinterpret_cast<const v4u_t*>(p + 16); }
    __device__ __forceinline__ void clear() { c = d = v4u_t{0, 0, 0, 0}; }
    template <int J> __device__ __forceinline__ bf16x8 elements(float sc) const
    {
        const unsigned lo = J < 2 ? c[2 * J & 3] : d[2 * J & 3], hi = J < 2 ? c[(2 * J + 1) & 3] : d[(2 * J + 1) & 3];
        const bf16x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, sc, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, sc, true),
                             __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, sc, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, sc, true)};
        return join(p);
    }
};

// Four rows of a token's output.
__device__ __forceinline__ void store_rows(const GemvArgs& a, const GemvWeight& w, int row, int token, const f32x4& s)
{
    if (token >= a.m || row >= w.n) return;
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

// What the workgroup's waves wrote to LDS is there; loads from memory stay under way.
__device__ __forceinline__ void lds_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

constexpr int HELD = 8;                    // 16-byte pieces of x that a thread holds on their way to LDS
constexpr int64_t kLdsX = 126 * 1024;      // bytes of x in LDS, beside sums (16 KB) and slots (18 KB)

// Workgroup: WR x WS waves, `per` tiles of 16 RT WR rows of one weight, one after the other.  The WR waves of a share have 16 RT rows each
// and the share's spans in common, whose elements of x they keep in LDS: all of them, or `chunk` spans at a time (then per is 1).  A wave
// has RT U blocks per lane under way: as soon as a span's codes are used, those of U spans later are asked for, the next tile's behind the
// last ones.  The WS shares' sums of a tile meet in LDS and are added in order.
template <int FMT, int TT, int RT, int U, int RING, int WR, int WS, bool ALL>
__device__ __forceinline__ void gemv_tiles(const GemvArgs& a, const GemvWeight& w, int block, int token0, uint4* lds)
{
    static_assert(RING == U || !ALL, "the next tile is aimed at before this one's last codes are asked for");
    constexpr int BYTES = FMT == kFP4 ? 16 : 32;             // of a block
    constexpr int THREADS = WR * 64;                         // of a share
    constexpr int ROWS = 16 * RT * WR;
    const int lane = threadIdx.x & 63, quarter = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int share = wave / WR, wr = wave % WR, tid = threadIdx.x % THREADS;
    const int nb = a.k / kBlock, chunk = a.chunk;
    const int chunks = ((nb + 3) / 4 + WS * chunk - 1) / (WS * chunk), begin = share * chunks * chunk;       // in spans
    const int tokens = min(16 * TT, a.m - token0);
    // Where codes are asked for next: rows past the last one repeat it (what comes of them is not stored), blocks past a row's last one repeat
    // that (they meet zeros of x).
    const uint8_t *codes, *scales;
    unsigned row_at[RT];                                     // block 0 of a lane's row behind that of the wave's first
    auto aim = [&](int tile) {
        const int64_t row0 = (int64_t)tile * ROWS + wr * 16 * RT, first = row0 < w.n ? row0 : w.n - 1;
        codes = w.codes + first * nb * BYTES;
        scales = w.scales + first * nb;
#pragma unroll
        for (int r = 0; r < RT; ++r) row_at[r] = (unsigned)min(r * 16 + (lane >> 2), (int)(w.n - 1 - first)) * nb;
    };
    // Codes are asked for in the order of memory, four lanes to the 64 bytes (FP8: twice) of a row's span: with a lane loading the block that
    // it needs every lane is an access of its own to the cache, which took longer than memory.  They go to their lanes through a slot of the
    // wave's in LDS (whose operations are done in order: no wait between a span's use of it and the next one's).
    constexpr int PIECES = BYTES / 16;                       // loads per lane and span
    v4u_t c[RT][RING][PIECES];
    const int piece_of = lane & 3, row_of = lane >> 2;
    auto fetch = [&](int u, int span) {
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const int b = min(span * 4 + (i * 4 + piece_of) / PIECES, nb - 1);
                c[r][u][i] = *reinterpret_cast<const v4u_t*>(codes + (uint64_t)(row_at[r] + b) * BYTES + (i * 4 + piece_of) % PIECES * 16);
            }
    };
    v4u_t* const slot = reinterpret_cast<v4u_t*>(lds + wave * kSlot);
    // piece p of row n lies where 16 rows' pieces of one lane quarter lie in different banks (FP8: at most two in one)
    auto place_of = [](int n, int p) { return PIECES == 1 ? n * 4 + (p ^ (n >> 2 & 3)) : n * 8 + (p ^ (n & 7)); };
    auto turn = [&](int r, int u) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) slot[place_of(row_of, i * 4 + piece_of)] = c[r][u][i];
        __builtin_amdgcn_wave_barrier();                     // (lanes read what others wrote)
        Block<FMT> to;
        to.get([&](int i) { return slot[place_of(lane & 15, quarter * PIECES + i)]; });
        __builtin_amdgcn_wave_barrier();
        return to;
    };
    // The scale bytes of a row come 16 at a time, four per lane, a round of U spans ahead, and to all lanes of the row through LDS as well.  Where the
    // row ends within the 16 or before them they are read one by one, and bytes past its last block are zero: the codes that repeat the last block
    // there are then small, where the scale of another block could make them infinite (times x's zeros: NaN).
    constexpr int G = U / 4;
    v4u_t sc[RT][G];
    unsigned sc_next[RT][G];
    const int full = nb / 16;
    auto fetch_scales = [&](int span) {
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int at = span / 4 + g;
            if (at < full) {
#pragma unroll
                for (int r = 0; r < RT; ++r) sc_next[r][g] = *reinterpret_cast<const u1_any*>(scales + row_at[r] + at * 16 + piece_of * 4);
            } else {
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    unsigned d = 0;
                    for (int i = 0; i < 4; ++i)
                        if (at * 16 + piece_of * 4 + i < nb) d |= (unsigned)scales[row_at[r] + at * 16 + piece_of * 4 + i] << (8 * i);
                    sc_next[r][g] = d;
                }
            }
        }
    };
    auto turn_scales = [&] {
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int g = 0; g < G; ++g) {
                reinterpret_cast<unsigned*>(slot + 128)[lane] = sc_next[r][g];
                __builtin_amdgcn_wave_barrier();
                sc[r][g] = slot[128 + (lane & 15)];
                __builtin_amdgcn_wave_barrier();
            }
    };
    // x in LDS: 16-byte piece i of a token's 16 * chunk at i ^ (token & 15), so that 16 tokens' pieces lie in different banks
    const int per = 16 * chunk, pieces = tokens * per;
    uint4* const xs = lds + WR * WS * kSlot;
    uint4* const mine = xs + share * (ALL ? 1 : 2) * pieces;
    f32x4* const sums = reinterpret_cast<f32x4*>(ALL ? xs + WS * pieces : xs);       // (chunks: in their place, when all are used)        // [2][share][wave in share][RT TT][lane]
    const unsigned one_over_per = 0xFFFFFFFFu / (unsigned)per + 1;           // p / per as a product: p < 2^16
    constexpr int STAGED = 8;                                              // pieces of a thread at a time: their loads wait together
    auto stage = [&](int ch) {
        const int64_t k0 = (int64_t)(begin + ch * chunk) * 128;
        for (int p0 = tid; p0 < pieces; p0 += STAGED * THREADS) {
            uint4 v[STAGED];
            int to[STAGED];
#pragma unroll
            for (int h = 0; h < STAGED; ++h) {
                const int p = p0 + h * THREADS, token = (int)__umulhi(p, one_over_per), i = p - token * per;
                const int64_t k = k0 + i * 8;
                to[h] = token * per + (i ^ (token & 15));
                v[h] = make_uint4(0, 0, 0, 0);
                if (p < pieces && k < a.k) v[h] = *reinterpret_cast<const uint4*>(a.x + (int64_t)(token0 + token) * a.ldx + k);
            }
#pragma unroll
            for (int h = 0; h < STAGED; ++h)
                if (p0 + h * THREADS < pieces) mine[to[h]] = v[h];
        }
    };
    // Chunks: a thread holds its HELD pieces of the next one while this one is used (no condition on the loads: nothing may come between the
    // codes' and their waits).
    uint4 held[HELD];
    auto hold = [&](int ch) {
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            const int p = min(tid + h * THREADS, pieces - 1), token = (int)__umulhi(p, one_over_per), i = p - token * per;
            const int at = min(x_piece(begin, ch, chunk, i), x_pieces(a.k) - 1);
            held[h] = *reinterpret_cast<const uint4*>(a.x + (int64_t)(token0 + token) * a.ldx + piece_element(at));
        }
    };
    auto put = [&](int ch) {
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            const int p = min(tid + h * THREADS, pieces - 1), token = (int)__umulhi(p, one_over_per), i = p - token * per;
            if (x_piece(begin, ch, chunk, i) >= x_pieces(a.k)) held[h] = make_uint4(0, 0, 0, 0);
            mine[(ch & 1) * pieces + token * per + (i ^ (token & 15))] = held[h];
        }
    };
    const uint4* x[TT][4];
#pragma unroll
    for (int t = 0; t < TT; ++t) {
        const int token = min(t * 16 + (lane & 15), tokens - 1);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[t][j] = mine + token * per + ((quarter * 4 + j) ^ (token & 15));
    }
    f32x4 acc[RT][TT];
    constexpr int D = TT == 1 ? 4 : TT == 2 ? 2 : 1;         // how many matrix instructions ahead elements of x are read
    const int tiles = (w.n + ROWS - 1) / ROWS, first_tile = block * a.per, end_tile = min(first_tile + a.per, tiles);
    aim(first_tile);
    fetch_scales(begin);
#pragma unroll
    for (int u = 0; u < RING; ++u) fetch(u, begin + u);
    stage(0);
    __syncthreads();
    turn_scales();
    constexpr bool EARLY = RT == 1;                          // (two rows' tiles leave no registers for it)
    Block<FMT> now_c[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
        if (EARLY) now_c[r] = turn(r, 0);
    for (int tile = first_tile; tile < end_tile; ++tile) {
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int t = 0; t < TT; ++t) acc[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int ch = 0; ch < chunks; ++ch) {
            if (!ALL) hold(ch + 1);
            const int at = ALL ? 0 : (ch & 1) * pieces;
            for (int s = 0; s < chunk; s += U) {
                const int now = begin + ch * chunk + s;
                int next = now + U, stride = 1;
                if (ch + 1 == chunks && s + U >= chunk) {    // behind the tile: the next one, or, once more, blocks that have just come
                    next = begin;
                    if (tile + 1 < end_tile) aim(tile + 1);
                    else { next = now; stride = 0; }
                }
                fetch_scales(next);
                bf16x8 v[D + 1][TT];
#pragma unroll
                for (int q = 0; q < D; ++q)
#pragma unroll
                    for (int t = 0; t < TT; ++t) v[q][t] = __builtin_bit_cast(bf16x8, x[t][q % 4][at + (s + q / 4) * 16]);
                if (EARLY) fetch(0, RING < U ? now + RING : next);               // span 0's codes have gone to their lanes
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    // This span's codes, or early the next one's, go to their lanes, and those of RING spans behind are asked for (not moved down to
                    // their use).
                    Block<FMT> next_c[RT];
                    const int n1 = EARLY ? u + 1 : u, in = n1 + RING;
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int r = 0; r < RT; ++r) (EARLY ? next_c[r] : now_c[r]) = turn(r, n1 % RING);
                    if (n1 < U) fetch(n1 % RING, in < U ? now + in : next + (in - U) * stride);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int q = u * 4 + j, n = q + D;
                        if (n < U * 4)
#pragma unroll
                            for (int t = 0; t < TT; ++t) v[n % (D + 1)][t] = __builtin_bit_cast(bf16x8, x[t][n % 4][at + (s + n / 4) * 16]);
                        bf16x8 e[RT];
#pragma unroll
                        for (int r = 0; r < RT; ++r) {
                            const float f = scale_operand((sc[r][u / 4][u % 4] >> (8 * quarter)) & 0xFFu);
                            e[r] = j == 0 ? now_c[r].template elements<0>(f) : j == 1 ? now_c[r].template elements<1>(f)
                                 : j == 2 ? now_c[r].template elements<2>(f) : now_c[r].template elements<3>(f);
                        }
#pragma unroll
                        for (int r = 0; r < RT; ++r)
#pragma unroll
                            for (int t = 0; t < TT; ++t) acc[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(e[r], v[q % (D + 1)][t], acc[r][t], 0, 0, 0);
                    }
#pragma unroll
                    for (int r = 0; r < RT; ++r)
                        if (EARLY) now_c[r] = next_c[r];
                }
                turn_scales();
            }
            if (!ALL) {
                // into the other buffer, which all have read before the last barrier; codes under way are not waited for
                put(ch + 1);
                lds_barrier();
            }
        }
        auto store = [&](int of, int p, const f32x4& s) {
            store_rows(a, w, tile * ROWS + of * 16 * RT + p / TT * 16 + quarter * 4, token0 + p % TT * 16 + (lane & 15), s);
        };
        if (WS == 1) {
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int t = 0; t < TT; ++t) store(wr, r * TT + t, acc[r][t]);
        } else {
            constexpr int PARTS = WR * RT * TT;
            f32x4* const here = sums + (ALL ? tile & 1 : 0) * WS * PARTS * 64;
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int t = 0; t < TT; ++t) here[((share * WR + wr) * RT * TT + r * TT + t) * 64 + lane] = acc[r][t];
            lds_barrier();                                   // (the other half of `sums` may still be read)
            for (int p = wave; p < PARTS; p += WR * WS) {
                f32x4 s = here[p * 64 + lane];
#pragma unroll
                for (int k = 1; k < WS; ++k) s += here[(k * PARTS + p) * 64 + lane];
                store(p / (RT * TT), p % (RT * TT), s);
            }
        }
    }
}

template <int TT, int RT, int U, int WR, int WS, bool ALL>
__global__ __launch_bounds__(WR * WS * 64, 2) void gemv_kernel(const GemvArgs a)
{
    extern __shared__ uint4 lds[];
    int i = 0;
    while (i + 1 < a.count && (int)blockIdx.x >= a.w[i + 1].first) ++i;
    const GemvWeight& w = a.w[i];
    const int block = (int)blockIdx.x - w.first, token0 = blockIdx.y * 16 * TT;
    if (w.fmt == kFP4) gemv_tiles<kFP4, TT, RT, U, U, WR, WS, ALL>(a, w, block, token0, lds);
    else               gemv_tiles<kFP8, TT, RT, 4, 4 / RT, WR, WS, ALL>(a, w, block, token0, lds);
}

// Small problems: 16 rows by up to 16 tokens, eight waves that take every eighth span, codes and x straight from memory.  Little code, as a
// launch fetches it anew, and no wait but the loads' own.
constexpr int kSmallWaves = 8;
template <int FMT>
__device__ __forceinline__ f32x4 small_sums(const GemvArgs& a, const GemvWeight& w, int row0, int token0, int wave, int lane)
{
    constexpr int BYTES = FMT == kFP4 ? 16 : 32;
    const int nb = a.k / kBlock, quarter = lane >> 4;
    const int64_t row = min(row0 + (lane & 15), w.n - 1);
    const uint8_t* const codes = w.codes + row * nb * BYTES;
    const uint8_t* const scales = w.scales + row * nb;
    const uint16_t* const x = a.x + (int64_t)min(token0 + (lane & 15), a.m - 1) * a.ldx;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s = wave; s * 4 < nb; s += kSmallWaves) {
        const int b = s * 4 + quarter;
        Block<FMT> c;
        c.clear();
        float sc = 1.f;
        bf16x8 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = __builtin_bit_cast(bf16x8, make_uint4(0, 0, 0, 0));
        if (b < nb) {                                        // (nothing of x beyond the row: it may be infinite)
            c.load(codes + (int64_t)b * BYTES);
            sc = scale_operand(scales[b]);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const bf16x8*>(x + b * kBlock + j * 8);
        }
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(c.template elements<0>(sc), v[0], acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(c.template elements<1>(sc), v[1], acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(c.template elements<2>(sc), v[2], acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(c.template elements<3>(sc), v[3], acc, 0, 0, 0);
    }
    return acc;
}
__global__ __launch_bounds__(kSmallWaves * 64) void gemv_small_kernel(const GemvArgs a)
{
    __shared__ f32x4 sums[kSmallWaves][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int i = 0;
    while (i + 1 < a.count && (int)blockIdx.x >= a.w[i + 1].first) ++i;
    const GemvWeight& w = a.w[i];
    const int row0 = ((int)blockIdx.x - w.first) * 16, token0 = blockIdx.y * 16;
    sums[wave][lane] = w.fmt == kFP4 ? small_sums<kFP4>(a, w, row0, token0, wave, lane) : small_sums<kFP8>(a, w, row0, token0, wave, lane);
    __syncthreads();
    if (wave == 0) {
        f32x4 s = sums[0][lane];
#pragma unroll
        for (int k = 1; k < kSmallWaves; ++k) s += sums[k][lane];
        store_rows(a, w, row0 + (lane >> 4) * 4, token0 + (lane & 15), s);
    }
}

template <int TT, int RT, int U, int WR, int WS, bool ALL> hipError_t launch(GemvArgs& a, hipStream_t s, int most = 0)
{
    constexpr int ROWS = 16 * RT * WR;
    const int tokens = a.m < 16 * TT ? a.m : 16 * TT, spans = (a.k / kBlock + 3) / 4;
    const int own = ((spans + WS - 1) / WS + U - 1) / U * U, fit = HELD * WR * 4 / tokens / U * U;
    a.chunk = ALL || own < fit ? own : fit;
    if (a.chunk <= 0) return hipErrorInvalidValue;
    int64_t tiles = 0;
    for (int i = 0; i < a.count; ++i) tiles += (a.w[i].n + ROWS - 1) / ROWS;
    a.per = !ALL ? 1 : (int)((tiles + most - 1) / most);
    int64_t blocks = 0;
    for (int i = 0; i < a.count; ++i) {
        a.w[i].first = (int)blocks;
        blocks += ((a.w[i].n + ROWS - 1) / ROWS + a.per - 1) / a.per;
    }
    const size_t x = (size_t)(ALL ? 1 : 2) * WS * tokens * a.chunk * 256, sums = WS > 1 ? (size_t)2 * WS * WR * RT * TT * 1024 : 0;
    const size_t lds = (size_t)WR * WS * kSlot * 16 + (ALL ? x + sums : x > sums ? x : sums);
    if (lds > 160 * 1024) return hipErrorInvalidValue;
    hipLaunchKernelGGL((gemv_kernel<TT, RT, U, WR, WS, ALL>), dim3((unsigned)blocks, (a.m + 16 * TT - 1) / (16 * TT)), dim3(WR * WS * 64), lds, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_gemv(GemvArgs a, hipStream_t s)
{
    if (a.count == 0 || a.m == 0) return hipSuccess;
    int64_t tiles = 0;                                       // of 16 rows
    for (int i = 0; i < a.count; ++i) tiles += (a.w[i].n + 15) / 16;
    const int64_t spans = (a.k / kBlock + 3) / 4;
    // Up to 24 spans in up to 8000 / spans workgroups: us with the small kernel / the others: 1 token [512 x 512] 2.3 / 4.2, [4096 x 2048] 3.5 / 4.3,
    // [4096 x 4096] (not taken) 5.6 / 5.1, 9 tokens 2 x [1003 x 2080] 3.8 / 6.3, 3 x [4096 x 2048] (not) 9.0 / 6.8, 24 tokens [4096 x 2048] (not) 6.9 / 6.1.
    const int64_t small = tiles * ((a.m + 15) / 16);
    if (spans <= 24 && small * spans <= 8000) {
        int blocks = 0;
        for (int i = 0; i < a.count; ++i) {
            a.w[i].first = blocks;
            blocks += (a.w[i].n + 15) / 16;
        }
        hipLaunchKernelGGL(gemv_small_kernel, dim3(blocks, (a.m + 15) / 16), dim3(kSmallWaves * 64), 0, s, a);
        return hipGetLastError();
    }
    // Up to 16 tokens whose x fits LDS as a whole: eight waves on 16 rows where there are few of them, on 32 where there are many (a share's part of x is
    // read for two tiles, and a workgroup per compute unit goes through several).  us, 16 / 32 rows: 1 token [4096 x 4096] 4.8 / 5.3, [4096 x
    // 11008] 8.1 / 9.7, 3 x [4096 x 4096] 11.0 / 8.3, 2 x [28672 x 8192] 50.4 / 48.9, 8 tokens 3 x [4096 x 4096] 12.6 / 9.0.
    auto whole = [&](int shares) { return a.m <= 16 && shares * a.m * (((spans + shares - 1) / shares + 3) / 4 * 4) * 256 <= kLdsX; };
    if (tiles <= 512 && whole(8)) return launch<1, 1, 4, 1, 8, true>(a, s, 512);
    if (tiles > 512 && whole(4)) return launch<1, 1, 4, 2, 4, true>(a, s, 256);
    // Otherwise x comes in chunks.  Of the tiles (256, 128, 64 or 32 rows, 16 to 64 tokens) the one with the most workgroups that still run at once, one
    // per compute unit: us with 256 / 128 / 64 / 32 rows, 16 tokens: 2 x [28672 x 8192] 62 / 68 / 79 / 93, 2 x [11008 x 4096] 19 / 15 / 21 / 24, 3 x
    // [4096 x 4096] 18 / 14 / 11 / 16, [4096 x 11008] 46 / 31 / 21 / 16; 48 tokens 2 x [28672 x 8192] in tiles of 256 rows by 48 / 32 / 16
    // tokens 77 / 109 / 134, 3 x [4096 x 4096] of 128 rows 27 / 19.4 / 25, [4096 x 11008] of 64 rows by 16 21.
    // It is not the best form everywhere: a tile whose tokens are not all there counts like a full one, and rereading the weights can cost less than idle compute
    // units or fewer rows.  Taken / best of them: 48 tokens 3 x [4096 x 4096] 19.4 / 18.3 (256 rows by 16), 2 x [11008 x 4096] 28.5 (128 by 48) / 26.0 (256 by 32), 64 tokens
    // 3 x [4096 x 4096] 27.6 (128 by 48) / 18.5 (256 by 16), 2 x [11008 x 4096] 32.6 (128 by 64) / 26.1 (256 by 32).
    const int cus = gemm_compute_units();
    int64_t most = 0;
    int form = 0, tt = 0;                                    // rows of a workgroup's tile: 256, 128, 64, 32
    for (int t = a.m <= 16 ? 1 : a.m <= 32 ? 2 : a.m <= 48 ? 3 : 4; t >= 1; --t)
        for (int rows = 16; rows >= 2 * t; rows /= 2) {
            const int64_t wgs = ((tiles + rows - 1) / rows) * ((a.m + 16 * t - 1) / (16 * t));
            if (wgs > most && (wgs <= cus || most == 0)) { most = wgs; form = rows; tt = t; }
            if (rows == 8 && t > 2) break;
        }
#define SNIP_GEMV(ROWS, TT, ...) if (form == ROWS && tt == TT) return launch<TT, __VA_ARGS__, false>(a, s)
    SNIP_GEMV(16, 1, 2, 4, 8, 1); SNIP_GEMV(16, 2, 2, 4, 8, 1); SNIP_GEMV(16, 3, 2, 4, 8, 1); SNIP_GEMV(16, 4, 2, 4, 8, 1);
    SNIP_GEMV(8, 1, 1, 4, 8, 1); SNIP_GEMV(8, 2, 1, 4, 8, 1); SNIP_GEMV(8, 3, 1, 4, 8, 1); SNIP_GEMV(8, 4, 1, 4, 8, 1);
    SNIP_GEMV(4, 1, 1, 4, 4, 2); SNIP_GEMV(4, 2, 1, 4, 4, 2);
    SNIP_GEMV(2, 1, 1, 4, 2, 4);
#undef SNIP_GEMV
    return hipErrorInvalidValue;
}

}  // namespace snip
