// The loss over the vocabulary, softmax cross entropy or distillation from a teacher's top logits, and its gradients, without the logits
// ever being stored.  With z = x w^T, s = z / tau, q the wanted probabilities (one entry of 1, or softmax(teacher / tau) over k entries):
//     lse = log sum_v exp s_v      loss = tau^2 sum_j q_j (log q_j - s_idx_j + lse)
//     dz = dloss tau (exp(s - lse) - q)      dx = dz w      dw = dz^T x
//
// All of it is one matrix product in bf16 (v_mfma_f32_16x16x32_bf16, C[i][j] = sum_r A[i][r] B[j][r]) with four ways to take the result out
// of the accumulators:
//   stats   A = w, B = x: of every token the tile's largest z and the sum of exp(s - largest), and z of the entries that the loss names;
//           a second kernel joins the tiles.  A token's logits lie in the registers of four lanes, so the sums need two shuffles.
//   dz      the same product anew, a piece of the vocabulary at a time: dz in bf16, [token][entry]
//   dx      A = w^T of the piece, B = dz, split over the vocabulary where there are few tiles: partial sums in fp32, joined at the end
//   dw      A = x^T, B = dz^T
// An operand that is contiguous along its other index ("turned": w^T, x^T, dz^T) comes into LDS as it lies in memory and is turned by the reads
// (ds_read_b64_tr_b16: of each 16 lanes, lane l gets element l of four rows), so nothing is transposed in memory.
#include "gemm_common.h"
#include <algorithm>
#include <type_traits>
#include <utility>

namespace snip {
namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
enum Out { kStats, kDz, kDx, kDw };
constexpr int kGroup = 16;       // tokens of a list of named entries: those of a block's columns

struct ProductArgs {
    const uint16_t *a, *b;
    int64_t lda, ldb;            // elements
    int I, J, R;
    const int* count;            // gradients: tokens that take part, J of dz and dx and R of dw
    int tiles_i, tiles_j, split; // stages of a split (blockIdx.y)
    float alpha;                 // 1 / tau
    // What the loss names: a target of every token, or lists of kGroup tokens each, a run for each tile of the vocabulary in turn: token of the group and entry
    // of the tile (16 bits each), and the place in `z` or q itself
    const void* targets; int target64;
    const int* starts; const int2* items; int64_t items_pitch; int vocab_tiles;
    int v0, vocab;               // entry of A's first row
    float2* tile_stats;          // stats: [tiles_i][J], (largest s log2 e, sum of 2^(s log2 e - that))
    float* z;                    // stats: of every named entry, by its place
    const float* lse;            // dz
    const float* part;           // dz: dloss tau of every token in units of *unit, zero for those that take no part
    const float* unit;           // dw
    void* c; int64_t ldc, split_stride; int c_fp32, add;   // dz, dx (fp32), dw
};

// TM x TN outputs of a workgroup of four waves, WM x WN of a wave.  LDS is a ring of SLOTS slots, a stage (64 contraction elements) of A and B
// in turn; an odd number needs slots of one size.
//   Large    bound by the matrix cores and the clock that the power leaves: a wave reads 32 KB from LDS a stage, for 128 MFMAs.  8192 x 4096 against
//            128000 5.9 to 6.0 ms, 1.44 PFLOP/s (the product alone, by the vendor's library, 5.8 ms); its gradient, 32000, 4.5 to 4.6 ms, 1.42.  Matrix cores busy 69 to 75 %
//            of the cycles, at 1.9 GHz; bank conflicts of 100 cycles a launch at most.
//   Middle   two workgroups of a compute unit, for problems with too few large tiles and for 65 to 128 tokens: bound by the copies' latency, 1.1 us a stage.
//   Few, Low up to 64 tokens: bound by w, which is read once; 64 tokens of 4096 against 128000 197 us, 5.3 TB/s, 37 of 2048 against 32000 21 us in the last-level cache.
template <int TM_, int TN_, int WM_, int WN_, int SLOTS_, int PER_CU_> struct Tile {
    static constexpr bool LARGE = PER_CU_ == 1;
    static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, SLOTS = SLOTS_, PER_CU = PER_CU_, MB = WM / 16, NB = WN / 16, NM = MB * NB;      // 16 x 16 blocks of a wave
    static constexpr int WGM = TM / WM, WGN = TN / WN, NT = 256;
    static constexpr int SA = TM * 128, SB = TN * 128, PAIR = SA + SB, LDS = SLOTS / 2 * PAIR + SLOTS % 2 * SA;
    static constexpr int CA = TM / 32, CB = TN / 32;             // 1 KB copies of a wave and stage
    static constexpr int DA = (SLOTS + 1) / 2, DB = SLOTS / 2;   // how many stages ahead copies are issued
    // copies that may be under way when the next stage has to be there: those behind it
    static constexpr int BEHIND = (DB - 2) * (CA + CB) + (SLOTS % 2 ? CA : 0), BEHIND_FIRST = (DA - 2) * CA + (DB - 1) * CB;
    static_assert(WGM * WGN == 4 && (SLOTS % 2 == 0 || SA == SB) && DB >= 2 && LDS * PER_CU <= 160 * 1024, "tile");
};
using Large = Tile<256, 256, 128, 128, 5, 1>;
using Middle = Tile<128, 128, 64, 64, 5, 2>;
using Few64 = Tile<128, 64, 64, 32, 6, 2>;
using Few32 = Tile<128, 32, 32, 32, 8, 2>;
using Low64 = Tile<64, 64, 32, 32, 10, 2>;
using Low32 = Tile<64, 32, 32, 16, 12, 2>;

__device__ __forceinline__ unsigned pack2(float a, float b) { return __builtin_bit_cast(unsigned, bf16x2{(__bf16)a, (__bf16)b}); }

// Two copies of 1 KB, one behind the other in LDS, or one.  The instruction's offset counts in memory and in LDS, so the second lane offset is given
// 1024 too low and the descriptor starts 1024 bytes early (kEarly).  A single M0 and its wait state for both; a copy holds up the wave that
// issues it, and with it the matrix core.
constexpr unsigned kEarly = 1024;
__device__ __forceinline__ void copy2(v4i rsrc, unsigned o0, unsigned o1, unsigned soff, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %4\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %2, %3 offen lds\n\tbuffer_load_dwordx4 %1, %2, %3 offen offset:1024 lds"
                 : : "v"(o0), "v"(o1), "s"(rsrc), "s"(soff), "s"(lds) : "memory", "m0");
}
__device__ __forceinline__ void copy1(v4i rsrc, unsigned o0, unsigned soff, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" : : "v"(o0), "s"(rsrc), "s"(soff), "s"(lds) : "memory", "m0");
}
// (scalar arithmetic only: a descriptor from vector registers would need five wait states in front of the copies)
__device__ __forceinline__ v4i early_desc(const uint16_t* p, unsigned bytes)
{
    const uint64_t a = (uint64_t)p - kEarly;
    v4i r;
    r[0] = (int)(unsigned)a;
    r[1] = (int)((unsigned)(a >> 32) & 0xFFFFu);
    r[2] = (int)(bytes + kEarly);
    r[3] = 0x00020000;
    return r;
}

// One operand of a tile: ROWS indices from `row0` on, of which a wave multiplies W from wave_row on.  C copies of this wave and stage.
// Not turned, a stage is ROWS rows of 128 bytes; 16-byte chunk c of row r lies at c ^ (r / 2 % 8), so that 16 lanes that read one chunk of 16 rows meet
// all banks.  Turned it is 64 rows of ROWS elements; chunk c of row r lies at c ^ (r % 4 * 4) ^ (r / 8 % 2 * 2), so that the 16 rows that a turning
// read takes 32 bytes of, eight apart in fours, meet all banks twice (of 64 elements, two rows to all banks: c ^ (r / 2 % 2 * 4) ^ (r / 8 % 2 * 2)).
template <int ROWS, int W, bool TURNED, bool SINGLE> struct Operand {
    static constexpr int C = ROWS / 32, PAIR = !SINGLE && C % 2 == 0 ? 2 : 1, UNITS = C / PAIR, BLOCKS = W / 16, READS = BLOCKS * (TURNED ? 2 : 1);
    static_assert(!TURNED || ROWS >= 64, "chunks enough to spread");
    const uint16_t* p;
    int64_t ld;
    int rows, R;                 // of the tile, of the contraction
    unsigned off[C];
    int chunk[2];                // not turned: of even and odd copies
    int at[TURNED ? BLOCKS : 2];
    v4i rsrc;

    __device__ __forceinline__ void start(const uint16_t* base, int64_t ld_, int row0, int all, int R_, int wave_row, int lane, int wave)
    {
        // (whole chunks: what is behind an end that is none is zero in one operand at least, or of outputs that are not stored)
        ld = ld_; rows = (min(ROWS, all - row0) + 7) & ~7; R = TURNED ? R_ : (R_ + 7) & ~7;
        const int r16 = lane & 15, g = lane >> 4;
        if constexpr (!TURNED) {
            p = base + row0 * ld;
            rsrc = early_desc(p, (unsigned)(((min(ROWS, all - row0) - 1) * ld + R) * 2));
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int row = (wave * C + c) * 8 + lane / 8;
                chunk[c & 1] = (lane % 8) ^ ((row >> 1) & 7);
                off[c] = (unsigned)(row * ld * 2) + chunk[c & 1] * 16 + early(c);
            }
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) at[ks] = (wave_row + r16) * 128 + (((ks * 4 + g) ^ (r16 >> 1)) * 16);
        } else {
            p = base + row0;
            constexpr int PER_ROW = ROWS / 8, RPC = 64 / PER_ROW;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int row = (wave * C + c) * RPC + lane / PER_ROW;
                off[c] = (unsigned)(row * ld * 2) + ((lane % PER_ROW) ^ spread(row)) * 16 + early(c);
            }
            // of each 16 lanes, four point to 32 bytes of a row; sixteens of a wave are 8 rows apart
            const int row = 8 * g + (lane >> 2 & 3);
#pragma unroll
            for (int m = 0; m < BLOCKS; ++m) at[m] = row * ROWS * 2 + ((((wave_row / 16 + m) * 2 + (lane >> 1 & 1)) ^ spread(row)) * 16) + (lane & 1) * 8;
        }
    }
    static __device__ __forceinline__ int spread(int row) { return ROWS == 64 ? (row >> 1 & 1) * 4 ^ (row >> 3 & 1) * 2 : (row & 3) * 4 ^ (row >> 3 & 1) * 2; }
    static __device__ __forceinline__ constexpr unsigned early(int c) { return kEarly - (PAIR == 2 && c % 2 ? 1024 : 0); }
    // before the copies of stage s; past the contraction's end they bring zeros
    __device__ __forceinline__ void stage(int s)
    {
        if constexpr (TURNED) {
            const int here = min(64, R - s * 64);
            rsrc = here > 0 ? early_desc(p + (int64_t)s * 64 * ld, (unsigned)(((here - 1) * ld + rows) * 2)) : early_desc(p, 0);
        } else if (s * 64 + 64 > R) {                               // chunks past the end of a row lose their source
#pragma unroll
            for (int c = 0; c < C; ++c) off[c] = chunk[c & 1] * 8 + s * 64 < R ? off[c] : kNoSource;
        }
    }
    // (within the descriptor's size: see copy_ranges.h)
    __device__ __forceinline__ unsigned uniform(int s) const { return TURNED ? 0u : (unsigned)min(s, (R - 1) / 64) * 128u; }
    __device__ __forceinline__ void copy(int u, int s, unsigned to)
    {
        if constexpr (PAIR == 2) copy2(rsrc, off[2 * u], off[2 * u + 1], uniform(s), to + u * 2048);
        else                     copy1(rsrc, off[u], uniform(s), to + u * 1024);
    }
    __device__ __forceinline__ void read(int i, int ks, const uint8_t* slot, bf16x8 (&f)[BLOCKS]) const
    {
        if constexpr (!TURNED) {
            f[i] = *reinterpret_cast<const bf16x8*>(slot + at[ks] + i * 2048);
        } else {
            typedef const __attribute__((address_space(3))) s16x4* place;
            const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(place)(slot + at[i / 2] + (ks * 32 + i % 2 * 4) * ROWS * 2));
            uint2 w = __builtin_bit_cast(uint2, v);
            uint4 old = __builtin_bit_cast(uint4, f[i / 2]);
            if (i % 2 == 0) { old.x = w.x; old.y = w.y; } else { old.z = w.x; old.w = w.y; }
            f[i / 2] = __builtin_bit_cast(bf16x8, old);
        }
    }
};

template <int N, class F, int... I> __device__ __forceinline__ void unroll_for_(F f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>()), ...); }
template <int N, class F> __device__ __forceinline__ void unroll_for(F f) { unroll_for_<N>(f, std::make_integer_sequence<int, N>()); }

// acc += A B^T of a 16 x 16 block.  The large tile's accumulators fill their 256 registers; written as assembly they stay in place, where the compiler
// moved up to 200 of them in every stage (its hazard waits in front of the first and behind the last of these are in multiply).
template <class T> __device__ __forceinline__ void mfma(v4f& acc, const bf16x8& a, const bf16x8& b)
{
    if constexpr (T::LARGE) asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
    else                          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, acc, 0, 0, 0);
}

// The same with copy `c` of the large tile behind it: M0 is set in front, and the MFMA is its wait state; so the copy takes two issue slots of the four
// that an MFMA leaves.
template <int CTO> __device__ __forceinline__ void mfma_copy(v4f& acc, const bf16x8& a, const bf16x8& b, v4i rsrc, unsigned off, unsigned soff, unsigned to)
{
    asm volatile("s_add_u32 m0, %6, %7\n\tv_mfma_f32_16x16x32_bf16 %0, %1, %2, %0\n\tbuffer_load_dwordx4 %3, %4, %5 offen lds"
                 : "+a"(acc) : "v"(a), "v"(b), "v"(off), "s"(rsrc), "s"(soff), "s"(to), "i"(CTO) : "memory", "m0", "scc");
}

// The products of a tile, stages [first, last) of the contraction, 64 elements each.
// A stage is two steps; between the MFMAs of a step the wave reads the operands of the next one from LDS (the second step of a stage those of the
// next stage's first) and issues copies.  A barrier a stage, in front of its second step: every wave has the whole stage in registers
// then, so its two slots are free, and the next stage has arrived.  With five slots B of stage s + 2 follows A of stage s in the ring and A of
// stage s + 3 follows B: the copies have 1 to 1.5 stages (A) and 0.75 to 1 (B) to arrive.
// `before` and `behind` are called before and behind the first copies: loads for later.  (What waits for a copy waits for every load before it, and behind copies a load
// makes the wait for the first stage one for later copies.)
template <class T, bool TA, bool TB, class F, class G>
__device__ __forceinline__ void multiply(const ProductArgs& p, uint8_t* lds, int i0, int j0, int first, int last, int lane, int wave, v4f (&acc)[T::MB][T::NB], F before, G behind)
{
    before();
    __builtin_amdgcn_sched_barrier(0);
    const int wm = wave / T::WGN, wn = wave % T::WGN;
    Operand<T::TM, T::WM, TA, T::LARGE> a;
    Operand<T::TN, T::WN, TB, T::LARGE> b;
    a.start(p.a, p.lda, i0, p.I, p.R, wm * T::WM, lane, wave);
    b.start(p.b, p.ldb, j0, p.J, p.R, wn * T::WN, lane, wave);
    const unsigned lds0 = lds_addr(lds), share_a = lds0 + wave * T::CA * 1024, share_b = lds0 + wave * T::CB * 1024;
    auto ahead = [](unsigned slot) { return slot + T::PAIR >= (unsigned)T::LDS ? slot + T::PAIR - T::LDS : slot + T::PAIR; };      // of the next stage
    bf16x8 fa[2][T::MB], fb[2][T::NB];
    constexpr int READS = a.READS + b.READS;
    constexpr auto reads_by = [](int i) { const int n = (i * 4 * READS + 3 * T::NM - 1) / (3 * T::NM); return n < READS ? n : READS; };      // in front of MFMA i
    auto read = [&](int j, int ks, unsigned sa, unsigned sb) {
        if (j < b.READS) b.read(j, ks, lds + sb, fb[ks & 1]);
        else             a.read(j - b.READS, ks, lds + sa, fa[ks & 1]);
    };
#pragma unroll
    for (int m = 0; m < T::MB; ++m)
#pragma unroll
        for (int n = 0; n < T::NB; ++n) acc[m][n] = v4f{0.f, 0.f, 0.f, 0.f};
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (T::LARGE) asm volatile("s_nop 7");
    __builtin_amdgcn_sched_barrier(0);
    // all slots but A's last: its copies are those of the first stage below.  (Copies go on past the end, with zeros that nobody reads: without tests, and the
    // numbers of copies under way stay the same.)
#pragma unroll
    for (int i = 0; i < T::SLOTS; ++i) {
        if (i == 2 * (T::DA - 1)) continue;
        const int s = first + i / 2;
        const unsigned slot = i / 2 * T::PAIR + i % 2 * T::SA;
        if (i % 2 == 0) {
            a.stage(s);
#pragma unroll
            for (int u = 0; u < a.UNITS; ++u) a.copy(u, s, share_a + slot);
        } else {
            b.stage(s);
#pragma unroll
            for (int u = 0; u < b.UNITS; ++u) b.copy(u, s, share_b + slot);
        }
    }
    behind();
    SNIP_WAIT_VM(T::BEHIND_FIRST);
    SNIP_BAR();
    unsigned sa = 0, sb = T::SA, to_a = (T::DA - 1) * T::PAIR;
#pragma unroll
    for (int j = 0; j < READS; ++j) read(j, 0, sa, sb);
    for (int s = first; s < last; ++s) {
        const unsigned na = ahead(sa), nb = ahead(sb);
        // A of stage s - 1 + DA goes into the slot that the stage before left, B of stage s + DB into one of this stage's
        const int next_a = s - 1 + T::DA, next_b = s + T::DB;
        const unsigned lds_a = share_a + to_a, lds_b = share_b + (T::SLOTS % 2 ? sa : sb), at_a = a.uniform(next_a), at_b = b.uniform(next_b);
        a.stage(next_a);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            if (ks == 1) {
                __builtin_amdgcn_s_waitcnt(0xC07F);                 // lgkmcnt(0)
                SNIP_WAIT_VM(T::BEHIND);
                SNIP_BAR();
                asm volatile("" ::: "memory");                      // (no read of the next stage before the barrier)
                b.stage(next_b);
            }
            // A's copies are spread over the first step, B's over the first half of the second
            constexpr int EVERY_A = T::NM / a.UNITS, EVERY_B = T::NM / 2 / b.UNITS;
            unroll_for<T::NM>([&](auto index) {
                constexpr int i = decltype(index)::value;
                v4f& c = acc[i / T::NB][i % T::NB];
                if constexpr (T::LARGE) {
                    constexpr int ua = i % EVERY_A == EVERY_A / 2 ? i / EVERY_A : -1, ub = i % EVERY_B == EVERY_B / 2 && i < T::NM / 2 ? i / EVERY_B : -1;
                    if (ks == 0 && ua >= 0)      mfma_copy<(ua < 0 ? 0 : ua) * 1024>(c, fa[ks][i / T::NB], fb[ks][i % T::NB], a.rsrc, a.off[ua < 0 ? 0 : ua], at_a, lds_a);
                    else if (ks == 1 && ub >= 0) mfma_copy<(ub < 0 ? 0 : ub) * 1024>(c, fa[ks][i / T::NB], fb[ks][i % T::NB], b.rsrc, b.off[ub < 0 ? 0 : ub], at_b, lds_b);
                    else                         mfma<T>(c, fa[ks][i / T::NB], fb[ks][i % T::NB]);
                } else {
                    mfma<T>(c, fa[ks][i / T::NB], fb[ks][i % T::NB]);
                }
                __builtin_amdgcn_sched_barrier(0);
                // the reads behind the first three quarters of the MFMAs
#pragma unroll
                for (int j = reads_by(i); j < reads_by(i + 1); ++j) { if (ks == 0) read(j, 1, sa, sb); else read(j, 0, na, nb); }
                if constexpr (!T::LARGE) {
#pragma unroll
                    for (int u = 0; u < a.UNITS; ++u)
                        if (ks == 0 && (2 * u + 1) * T::NM / 2 / a.UNITS == i) a.copy(u, next_a, lds_a);
#pragma unroll
                    for (int u = 0; u < b.UNITS; ++u)
                        if (ks == 1 && (2 * u + 1) * T::NM / 4 / b.UNITS == i) b.copy(u, next_b, lds_b);
                }
                __builtin_amdgcn_sched_barrier(0);
            });
        }
        to_a = T::SLOTS % 2 ? sb : sa;
        sa = na;
        sb = nb;
    }
    // the last copies have to be there before LDS holds something else, and before the workgroup's end
    SNIP_WAIT_VM(0);
    __builtin_amdgcn_s_waitcnt(0xC07F);
    SNIP_BAR();
    asm volatile("" ::: "memory");
    // (a result is there 18 wait states behind its MFMA)
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (T::LARGE) asm volatile("s_nop 15\n\ts_nop 15");
    __builtin_amdgcn_sched_barrier(0);
}

// In registers, lane 16 g + r of block (m, n) holds C[16 m + 4 g + t][16 n + r] in acc[m][n][t].

// Stored from there: fp32 as it lies, 64 bytes of a row of the result by four lanes; bf16 of two blocks (m, m + 1), where lanes 16 apart swap halves so
// that each has eight numbers in a row, again 64 bytes by four lanes.  (Through LDS in whole lines, before: 5.6 us of a tile of 256 x 256 behind its last product.)
__device__ __forceinline__ void swap_rows(unsigned& a, unsigned& b)          // lanes 16 ... 31 and 48 ... 63 of a with those 16 before of b
{
    const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    a = r[0];
    b = r[1];
}
__device__ __forceinline__ v4u eight(v4f v, v4f w)
{
    v4u u = {pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(w[0], w[1]), pack2(w[2], w[3])};
    { unsigned a = u[0], b = u[2]; swap_rows(a, b); u[0] = a; u[2] = b; }
    { unsigned a = u[1], b = u[3]; swap_rows(a, b); u[1] = a; u[3] = b; }
    return u;
}
__device__ __forceinline__ int eight_at(int m, int g) { return (m + (g & 1)) * 16 + (g >> 1) * 8; }

// A wave's result leaves through its own part of LDS, 16 columns (rows of the result in memory) of WM numbers at a time: stores are whole runs then, and
// an element that the loss names is found by its place.  16-byte chunk c of column r lies at c ^ r.
template <class T> struct Stage {
    static constexpr int ROWB = T::WM * 4, CPR = ROWB / 16, PART = T::LDS / 4 / 1024 * 1024, AREA = 16 * ROWB;
    static_assert(2 * AREA <= PART, "a wave's part: two areas in turn");
    uint8_t *own, *reg;
    int lane, r16, g;
    __device__ __forceinline__ Stage(uint8_t* lds, int wave, int lane_) : own(lds + wave * PART), reg(own), lane(lane_), r16(lane_ & 15), g(lane_ >> 4) {}
    __device__ __forceinline__ float* at(int col, int row) { return reinterpret_cast<float*>(reg + col * ROWB + (((row >> 2) ^ (col & (CPR - 1))) * 16)) + (row & 3); }
    __device__ __forceinline__ void turn(int n) { reg = own + n % 2 * AREA; }
    __device__ __forceinline__ void put(int m, v4f v) { *reinterpret_cast<v4f*>(at(r16, m * 16 + g * 4)) = v; }
    // calls sink(column, row of the first, eight numbers of a column)
    template <class F> __device__ __forceinline__ void take(F sink)
    {
        constexpr int LANES = T::WM / 8, RPI = 64 / LANES;
#pragma unroll
        for (int it = 0; it < 16 / RPI; ++it) {
            const int col = it * RPI + lane / LANES, row = lane % LANES * 8;
            const float4 u = *reinterpret_cast<const float4*>(at(col, row)), v = *reinterpret_cast<const float4*>(at(col, row + 4));
            const float f[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
            sink(col, row, f);
        }
    }
};

// The elements of this wave's block that the loss names.
template <class T> struct Names {
    const ProductArgs& p;
    int lane, row0, col0, group0;            // of the wave's block; its first group of tokens
    int from[T::NB], to[T::NB];              // runs of the groups' lists, and of each the first 64 items
    int mine[T::NB], mine_place[T::NB];
    int64_t target[T::NB];                   // of the lane's columns, as they are
    __device__ __forceinline__ Names(const ProductArgs& p_, int lane_) : p(p_), lane(lane_) {}
    __device__ __forceinline__ const int2* items(int n) const { return p.items + (group0 + n) * p.items_pitch; }
    __device__ __forceinline__ void load(int ti, int tj, int wm, int wn)
    {
        row0 = wm * T::WM; col0 = wn * T::WN; group0 = (tj * T::TN + col0) / kGroup;
        if (p.targets) {
            row0 += p.v0 + ti * T::TM;
#pragma unroll
            for (int n = 0; n < T::NB; ++n) {
                const int j = min(tj * T::TN + col0 + n * 16 + (lane & 15), p.J - 1);
                target[n] = p.target64 ? ((const int64_t*)p.targets)[j] : (int64_t)((const int*)p.targets)[j];
            }
            return;
        }
        // (scalar loads, which the copies behind them do not hold up)
#pragma unroll
        for (int n = 0; n < T::NB; ++n) {
            const bool is = (group0 + n) * kGroup < p.J;
            const auto* run = (const __attribute__((address_space(4))) int*)(p.starts + (int64_t)(is ? group0 + n : 0) * (p.vocab_tiles + 1) + p.v0 / T::TM + ti);
            from[n] = run[0]; to[n] = is ? run[1] : from[n];
        }
    }
    __device__ __forceinline__ void load_items()
    {
        if (p.targets) return;
#pragma unroll
        for (int n = 0; n < T::NB; ++n) {
            if (from[n] >= to[n]) continue;
            const int2 item = items(n)[min(from[n] + lane, to[n] - 1)];
            mine[n] = item.x; mine_place[n] = item.y;
        }
    }
    // Whether there are some in columns 16 n ... 16 n + 15.
    __device__ __forceinline__ bool some(int n, int tj) const
    {
        bool found = false;
        of(n, tj, [&]() { found = true; }, [](int, int, int) {});
        return found;
    }
    // Those of columns 16 n ... 16 n + 15: calls f(column, row, item), a lane for each, with the item of a list or, of targets, the token; `any` before, if there are some.
    template <class G, class F> __device__ __forceinline__ void of(int n, int tj, G any, F f) const
    {
        if (p.targets) {
            const int j = tj * T::TN + col0 + n * 16 + lane;
            const int64_t row = target[n] - row0;
            const bool is = lane < 16 && j < p.J && target[n] < p.vocab && row >= 0 && row < T::WM;
            if (__builtin_amdgcn_ballot_w64(is) == 0) return;
            any();
            if (is) f(lane, (int)row, j);
            return;
        }
        bool first = true;
        for (int e = from[n]; e < to[n]; e += 64) {
            int at = mine[n], place = mine_place[n];
            asm volatile("" : "+v"(at), "+v"(place));               // (numbers, not places in scratch memory)
            if (e != from[n]) {
                const int2 item = items(n)[min(e + lane, to[n] - 1)];
                at = item.x; place = item.y;
            }
            const int row = (at >> 16) - row0;
            const bool is = e + lane < to[n] && row >= 0 && row < T::WM;
            if (__builtin_amdgcn_ballot_w64(is) == 0) continue;
            if (first) any();
            first = false;
            if (is) f(at & 0xFFFF, row, place);
        }
    }
};

__device__ __forceinline__ v4u packed(const float (&f)[8]) { return v4u{pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7])}; }

// Accumulators of the large tile come out of their registers here, not sooner: 256 of them would not fit beside.
template <class T> __device__ __forceinline__ v4f held(v4f& acc)
{
    if constexpr (T::LARGE) asm volatile("" : "+a"(acc));
    return acc;
}

// What is subtracted from the exponents of a sum of powers of two: the largest of them.  Where that is infinite, nothing: infinity less infinity is no number,
// and the sum is 0 or infinity as it stands.
__device__ __forceinline__ float reference(float top) { return fabsf(top) == INFINITY ? 0.f : top; }
// From 2^30 on half a step of the largest exponent, by which its product was rounded, is 32 and more: the largest term itself, 2^that, may be anything.  A sum
// there is worth less than a step whatever it is, 1 to the vocabulary: 1, unless it is no number or the sum of nothing.
__device__ __forceinline__ float far_sum(float top, float sum) { return fabsf(top) >= 1073741824.f && top != -INFINITY && sum == sum ? 1.f : sum; }
// Two sums of powers of two, each (largest exponent, sum of 2^(exponent - reference)).
__device__ __forceinline__ float2 join2(float2 v, float2 o)
{
    const float top = fmaxf(v.x, o.x), base = reference(top);
    return make_float2(top, v.y * __builtin_amdgcn_exp2f(v.x - base) + o.y * __builtin_amdgcn_exp2f(o.x - base));
}

// Tile `tile` of split `split`.
template <class T, int OUT>
__device__ __forceinline__ void product(const ProductArgs& given, uint8_t* lds, int tile, int split)
{
    ProductArgs p = given;
    if constexpr (OUT == kDz || OUT == kDx) {
        p.J = __builtin_amdgcn_readfirstlane(*p.count);
        p.tiles_j = (p.J + T::TN - 1) / T::TN;
        if (tile >= p.tiles_i * p.tiles_j) return;
    }
    if constexpr (OUT == kDw) p.R = __builtin_amdgcn_readfirstlane(*p.count);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / T::WGN, wn = wave % T::WGN, r16 = lane & 15, g = lane >> 4;
    int ti, tj;
    tile_of(tile, p.tiles_i * p.tiles_j, p.tiles_i, p.tiles_j, ti, tj);
    const int i0 = ti * T::TM, j0 = tj * T::TN;
    const int all = (p.R + 63) / 64, first = OUT == kDx ? split * p.split : 0, last = OUT == kDx ? min(all, first + p.split) : all;
    const float unit = OUT == kDw ? *p.unit : 1.f;
    v4f acc[T::MB][T::NB];
    const int iw = i0 + wm * T::WM, jw = j0 + wn * T::WN;
    Names<T> names(p, lane);
    float lse[T::NB], part[T::NB];                                  // dz, of the lane's columns
    multiply<T, (OUT == kDx || OUT == kDw), OUT == kDw>(p, lds, i0, j0, first, last, lane, wave, acc, [&]() {
        if constexpr (OUT == kDz) names.load(ti, tj, wm, wn);
        if constexpr (OUT == kDz) {
#pragma unroll
            for (int n = 0; n < T::NB; ++n) {
                const int j = min(jw + n * 16 + r16, p.J - 1);
                lse[n] = p.lse[j];
                part[n] = p.part[j];
            }
        }
    }, [&]() {
        if constexpr (OUT == kStats) names.load(ti, tj, wm, wn);
        if constexpr (OUT == kStats || OUT == kDz) names.load_items();
    });

    Stage<T> stage(lds, wave, lane);
    if constexpr (OUT == kStats) {
#pragma unroll
        for (int n = 0; n < T::NB; ++n) {
            stage.turn(n);
            names.of(n, tj, [&]() {
#pragma unroll
                for (int m = 0; m < T::MB; ++m) stage.put(m, held<T>(acc[m][n]));
            }, [&](int col, int row, int place) { p.z[place] = *stage.at(col, row); });
        }
        __syncthreads();
        float2* shared = reinterpret_cast<float2*>(lds);             // [WGM][TN]
        const float c = p.alpha * kLog2e;
        auto sums = [&](auto cut) {                                  // cut: rows past the vocabulary's end do not count
#pragma unroll
            for (int n = 0; n < T::NB; ++n) {
                int rows = p.I - iw - 4 * g;
                auto counts = [&](int m, int k) { return !decltype(cut)::value || m * 16 + k < rows; };
                v4f v[T::MB];
                float top = -INFINITY, tops[2] = {-INFINITY, -INFINITY}, part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int m = 0; m < T::MB; ++m) {
                    v[m] = held<T>(acc[m][n]);
                    if (decltype(cut)::value) asm volatile("" : "+v"(rows));      // (kept for all blocks, the comparisons would spill)
#pragma unroll
                    for (int k = 0; k < 4; ++k) tops[k & 1] = fmaxf(tops[k & 1], counts(m, k) ? v[m][k] : -INFINITY);
                }
                top = fmaxf(tops[0], tops[1]);
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32)) * c;
                const float base = reference(top);
#pragma unroll
                for (int m = 0; m < T::MB; ++m) {
                    if (decltype(cut)::value) asm volatile("" : "+v"(rows));
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float e = __builtin_amdgcn_exp2f(fmaf(v[m][k], c, -base));
                        part[k] += counts(m, k) ? e : 0.f;
                    }
                }
                float sum = (part[0] + part[1]) + (part[2] + part[3]);
                sum += __shfl_xor(sum, 16);
                sum += __shfl_xor(sum, 32);
                if (g == 0) shared[wm * T::TN + wn * T::WN + n * 16 + r16] = make_float2(top, far_sum(top, sum));
            }
        };
        if (iw + T::WM > p.I) sums(std::true_type());
        else                  sums(std::false_type());
        __syncthreads();
        for (int j = threadIdx.x; j < T::TN; j += T::NT) {
            if (j0 + j >= p.J) break;
            float2 v = shared[j];
#pragma unroll
            for (int w = 1; w < T::WGM; ++w) v = join2(v, shared[w * T::TN + j]);
            p.tile_stats[(int64_t)ti * p.J + j0 + j] = v;
        }
    }
    if constexpr (OUT == kDz) {
        // (rounded to bf16 soon: a product of the logit with the rounded constant is exact enough)
        const float c = p.alpha * kLog2e;
#pragma unroll
        for (int n = 0; n < T::NB; ++n) {
            // (a weight that is zero makes dz zero, whatever lse holds)
            const float mine = jw + n * 16 + r16 < p.J ? part[n] : 0.f, base = mine == 0.f ? INFINITY : lse[n] * kLog2e;
            auto powers = [&](int m) {
                v4f v = held<T>(acc[m][n]);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = __builtin_amdgcn_exp2f(fmaf(v[k], c, -base));
                return v;
            };
            // (the pitch covers whole tiles)
            if (!names.some(n, tj)) {
                uint16_t* to = (uint16_t*)p.c + (jw + n * 16 + r16) * p.ldc + iw;
                auto direct = [&](auto cut) {                        // cut: rows past the piece's end are zero
#pragma unroll
                    for (int m = 0; m < T::MB; m += 2) {
                        auto weighted = [&](int m) {
                            v4f v = powers(m);
#pragma unroll
                            for (int k = 0; k < 4; ++k) v[k] = decltype(cut)::value && iw + m * 16 + g * 4 + k >= p.I ? 0.f : v[k] * mine;
                            return v;
                        };
                        const v4u u = eight(weighted(m), weighted(m + 1));
                        if (jw + n * 16 + r16 < p.J) *reinterpret_cast<v4u*>(to + eight_at(m, g)) = u;
                    }
                };
                if (iw + T::WM > p.I) direct(std::true_type());
                else                  direct(std::false_type());
                continue;
            }
            stage.turn(n);
#pragma unroll
            for (int m = 0; m < T::MB; ++m) stage.put(m, powers(m));
            names.of(n, tj, []() {}, [&](int col, int row, int q) { *stage.at(col, row) -= p.targets ? 1.f : __int_as_float(q); });
            stage.take([&](int col, int row, const float (&f)[8]) {
                const float coef = __shfl(mine, col);
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = iw + row + e >= p.I ? 0.f : f[e] * coef;
                if (jw + n * 16 + col < p.J) *reinterpret_cast<v4u*>((uint16_t*)p.c + (jw + n * 16 + col) * p.ldc + iw + row) = packed(v);
            });
        }
    }
    if constexpr (OUT == kDx || OUT == kDw) {
        // (I is a multiple of 8)
        auto whole = [&](auto fp32, auto add) {
#pragma unroll
            for (int n = 0; n < T::NB; ++n) {
                const int j = jw + n * 16 + r16;
                auto scaled = [&](int m) {
                    v4f v = held<T>(acc[m][n]);
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = OUT == kDw ? v[k] * unit : v[k];
                    return v;
                };
                if constexpr (decltype(fp32)::value) {
                    float* to = (float*)p.c + (OUT == kDx ? split * p.split_stride : 0) + j * p.ldc + iw + g * 4;
                    v4f old[T::MB];
                    auto is = [&](int m) { return j < p.J && iw + m * 16 + g * 4 < p.I; };
                    if constexpr (decltype(add)::value) {
#pragma unroll
                        for (int m = 0; m < T::MB; ++m) old[m] = is(m) ? *reinterpret_cast<const v4f*>(to + m * 16) : v4f{0.f, 0.f, 0.f, 0.f};
                    }
#pragma unroll
                    for (int m = 0; m < T::MB; ++m) {
                        v4f v = scaled(m);
                        if constexpr (decltype(add)::value) v += old[m];
                        if (is(m)) *reinterpret_cast<v4f*>(to + m * 16) = v;
                    }
                } else {
                    uint16_t* to = (uint16_t*)p.c + j * p.ldc + iw;
                    v4u old[T::MB / 2];
                    auto is = [&](int m) { return j < p.J && iw + eight_at(m, g) < p.I; };
                    if constexpr (decltype(add)::value) {
#pragma unroll
                        for (int m = 0; m < T::MB; m += 2) old[m / 2] = is(m) ? *reinterpret_cast<const v4u*>(to + eight_at(m, g)) : v4u{0u, 0u, 0u, 0u};
                    }
#pragma unroll
                    for (int m = 0; m < T::MB; m += 2) {
                        v4f v = scaled(m), w = scaled(m + 1);
                        if constexpr (decltype(add)::value) {
                            // (one rounding: the old numbers come to the products' places first)
                            v4u o = old[m / 2];
                            { unsigned a = o[0], b = o[2]; swap_rows(a, b); o[0] = a; o[2] = b; }
                            { unsigned a = o[1], b = o[3]; swap_rows(a, b); o[1] = a; o[3] = b; }
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                v[2 * k] += __uint_as_float(o[k] << 16); v[2 * k + 1] += __uint_as_float(o[k] & 0xFFFF0000u);
                                w[2 * k] += __uint_as_float(o[2 + k] << 16); w[2 * k + 1] += __uint_as_float(o[2 + k] & 0xFFFF0000u);
                            }
                        }
                        const v4u u = eight(v, w);
                        if (is(m)) *reinterpret_cast<v4u*>(to + eight_at(m, g)) = u;
                    }
                }
            }
        };
        if constexpr (OUT == kDx) {
            if (p.add) whole(std::true_type(), std::true_type());
            else       whole(std::true_type(), std::false_type());
        } else if (p.c_fp32) {
            if (p.add) whole(std::true_type(), std::true_type());
            else       whole(std::true_type(), std::false_type());
        } else {
            if (p.add) whole(std::false_type(), std::true_type());
            else       whole(std::false_type(), std::false_type());
        }
    }
}

template <class T, int OUT>
__global__ __launch_bounds__(T::NT, T::PER_CU) void product_kernel(const ProductArgs p)
{
    __shared__ __attribute__((aligned(1024))) uint8_t lds[T::LDS];
    product<T, OUT>(p, lds, blockIdx.x, blockIdx.y);
}
// dx (tiles x splits) and dw, which need dz alone, in one launch where neither has large tiles: what one leaves idle the other takes.
template <class X, class W>
__global__ __launch_bounds__(256, 2) void pair_kernel(const ProductArgs dx, int splits, const ProductArgs dw)
{
    __shared__ __attribute__((aligned(1024))) uint8_t lds[X::LDS > W::LDS ? X::LDS : W::LDS];
    const int tiles = dx.tiles_i * dx.tiles_j, b = blockIdx.x, split = __builtin_amdgcn_readfirstlane(b / tiles);
    if (split < splits) product<X, kDx>(dx, lds, b - split * tiles, split);
    else                product<W, kDw>(dw, lds, b - splits * tiles, 0);
}

__device__ __forceinline__ float logit(const void* teacher, bool fp32, int64_t at)
{
    return fp32 ? ((const float*)teacher)[at] : __uint_as_float((unsigned)((const uint16_t*)teacher)[at] << 16);
}
__device__ __forceinline__ float over_wave(float v) { for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d); return v; }
__device__ __forceinline__ float top_of_wave(float v) { for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d)); return v; }

// dloss tau of a token, zero where it takes no part: of targets, or given.
struct Weights {
    const void* targets; int target64, vocab;
    const float *dloss, *given;
    __device__ __forceinline__ int64_t target(int t) const { return target64 ? ((const int64_t*)targets)[t] : (int64_t)((const int*)targets)[t]; }
    __device__ __forceinline__ float operator()(int t) const
    {
        if (!targets) return given[t];
        const int64_t at = target(t);
        return at >= 0 && at < vocab ? (dloss ? dloss[t] : 1.f) : 0.f;
    }
};

// The gradients' products run over the tokens that take part alone, in their order: of a dialogue whose prompt is not learned they are half.  `place`: of a
// token among them, or -1.  8192 x 4096 against 32000: 4.60 ms with all, 3.23 without 40 % of them, 1.38 without 80 %.
// The largest weight that is finite, or 1, is the unit that dz is held in.  dz is rounded to bf16, and at the entry that is wanted it is near -1 times the
// token's weight.  Where all weights are equal (a mean) the weight is 1 in this unit, so that p - q itself is rounded, near -1 where bf16's relative step is smallest.
// Relative error of dw in bf16, its own rounding included, weights from 0.5 to 1.5: 0.0025 -> 0.0022; equal ones 0.0024 -> 0.0017.
template <int NT> struct Live { int before[NT], waves[NT / 64]; unsigned bits[NT]; float tops[NT / 64]; };
// Of tokens t0 ... t0 + 8 NT - 1, eight of a thread: their number, and `top` raised to their largest weight.
template <int NT> __device__ __forceinline__ int find_live(const Weights& w, int t0, int tokens, Live<NT>& s, float& top)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    unsigned bits = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int t = t0 + (int)threadIdx.x * 8 + i;
        const float g = t < tokens ? w(t) : 0.f, v = fabsf(g);
        bits |= g != 0.f ? 1u << i : 0u;
        top = v < INFINITY ? fmaxf(top, v) : top;
    }
    const int n = __builtin_popcount(bits);
    int inc = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(inc, d);
        if (lane >= d) inc += o;
    }
    top = top_of_wave(top);
    __syncthreads();
    if (lane == 63) { s.waves[wave] = inc; s.tops[wave] = top; }
    __syncthreads();
    int before = inc - n, all = 0;
    for (int i = 0; i < NT / 64; ++i) {
        before += i < wave ? s.waves[i] : 0;
        all += s.waves[i];
        top = fmaxf(top, s.tops[i]);
    }
    s.before[threadIdx.x] = before;
    s.bits[threadIdx.x] = bits;
    __syncthreads();
    return all;
}
template <int NT> __device__ __forceinline__ int place_of(const Live<NT>& s, int i)
{
    const unsigned bits = s.bits[i / 8];
    return bits >> i % 8 & 1 ? s.before[i / 8] + __builtin_popcount(bits & ((1u << i % 8) - 1)) : -1;
}
__global__ __launch_bounds__(1024) void order_kernel(const Weights w, int tokens, int* __restrict__ place, int* __restrict__ count, float* __restrict__ unit)
{
    __shared__ Live<1024> live;
    float top = 0.f;
    int before = 0;
    for (int t0 = 0; t0 < tokens; t0 += 8192) {
        const int here = find_live<1024>(w, t0, tokens, live, top);
        for (int i = threadIdx.x; i < 8192 && t0 + i < tokens; i += 1024) {
            const int at = place_of(live, i);
            place[t0 + i] = at < 0 ? -1 : before + at;
        }
        before += here;
    }
    if (threadIdx.x == 0) { *count = before; *unit = top > 0.f ? top : 1.f; }
}
// What the products read of the tokens that take part, one after the other, by a wave for each: x, lse, the weight in that unit, the target or (of a
// distillation) the token itself.  `find`: every workgroup finds the places itself (a launch less), up to kFind tokens.
constexpr int kFind = 2048;
__global__ __launch_bounds__(256) void part_kernel(const uint16_t* __restrict__ x, int64_t ld, int tokens, int cols, const Weights w, const float* __restrict__ lse, bool find,
                                                   int* __restrict__ place, int* __restrict__ count, float* __restrict__ unit, float* __restrict__ part, float* __restrict__ part_lse,
                                                   int* __restrict__ part_at, uint16_t* __restrict__ out)
{
    __shared__ Live<256> live;
    const int lane = threadIdx.x & 63;
    float u = 0.f;
    if (find) {
        const int all = find_live<256>(w, 0, tokens, live, u);
        u = u > 0.f ? u : 1.f;
        if (blockIdx.x == 0 && threadIdx.x == 0) { *count = all; *unit = u; }
    } else {
        u = *unit;
    }
    for (int t = blockIdx.x * 4 + (threadIdx.x >> 6); t < tokens; t += gridDim.x * 4) {
        const int to = __builtin_amdgcn_readfirstlane(find ? place_of(live, t) : place[t]);
        if (find && lane == 0) place[t] = to;
        if (to < 0) continue;
        const float g = __fdiv_rn(w(t), u);
        if (lane == 0) {
            part[to] = g;
            part_lse[to] = lse[t];
            part_at[to] = w.targets ? (int)w.target(t) : t;
        }
        // (a weight that is zero in this unit makes dz zero, whatever x holds)
        for (int c = lane * 8; c < cols; c += 512)
            *reinterpret_cast<uint4*>(out + (int64_t)to * cols + c) = g == 0.f ? make_uint4(0, 0, 0, 0) : *reinterpret_cast<const uint4*>(x + t * ld + c);
    }
}

constexpr unsigned kFree = 0xFFFFFFFFu, kTwice = 0x80000000u;
__device__ __forceinline__ int place_in_table(int v, int mask) { return (int)((unsigned)v * 2654435761u >> 16) & mask; }
// What a distillation's gradient needs of every token, a wave for each: entries (-1 where there is nothing: outside the vocabulary, q = 0, or one named
// before, which has its q added) and q, and dloss tau, zero where no entry counts.  Bound by latency: 515 x 16 entries 5 us, 4096 x 32 9-12,
// 4096 x 1024 45, 209 where most tokens name something twice (all entries compared with all: 1574).
template <bool I64>
__global__ __launch_bounds__(256) void entries_kernel(const void* __restrict__ indices, const void* __restrict__ teacher, bool teacher_fp32, int tokens, int vocab,
                                                      int k, float tau, const float* __restrict__ dloss, int* __restrict__ index, float* __restrict__ q, float* __restrict__ weight)
{
    __shared__ int numbers[4][1024];
    __shared__ float wants[4][1024];
    __shared__ unsigned table[4][2048];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float alpha = 1.f / tau;
    int mask = 63;
    while (mask < 2 * k - 1) mask = 2 * mask + 1;
    for (int t = blockIdx.x * 4 + wave; t < tokens; t += gridDim.x * 4) {
        const int64_t row = (int64_t)t * k;
        float top = -INFINITY;
        bool any = false;
        for (int j = lane; j < k; j += 64) {
            const int64_t v = I64 ? ((const int64_t*)indices)[row + j] : ((const int*)indices)[row + j];
            const float u = logit(teacher, teacher_fp32, row + j) * alpha;
            const bool is = v >= 0 && v < vocab;
            numbers[wave][j] = is ? (int)v : -1;
            wants[wave][j] = u;
            any = any || (is && !(u == -INFINITY));
            if (is) top = fmaxf(top, u);
        }
        top = top_of_wave(top);
        any = __builtin_amdgcn_ballot_w64(any) != 0;
        const float base = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
        for (int j = lane; j < k; j += 64)
            if (numbers[wave][j] >= 0) sum += expf(wants[wave][j] - base);
        sum = over_wave(sum);
        const float log_sum = logf(sum);
        for (int j = lane; j < k; j += 64) {
            float w = 0.f;
            if (any && numbers[wave][j] >= 0) w = expf(wants[wave][j] - base - log_sum);
            if (w == 0.f) numbers[wave][j] = -1;
            wants[wave][j] = w;
        }
        // those named twice are found with a table (open addressing, twice as many places as entries), and the wave looks through all entries for each of them
        for (int j = lane; j <= mask; j += 64) table[wave][j] = kFree;
        for (int j = lane; j < k; j += 64) {
            const int v = numbers[wave][j];
            if (v < 0) continue;
            int at = place_in_table(v, mask);
            for (;; at = (at + 1) & mask) {
                const unsigned old = atomicCAS(&table[wave][at], kFree, (unsigned)v);
                if (old == kFree) break;
                if ((old & ~kTwice) != (unsigned)v) continue;
                atomicOr(&table[wave][at], kTwice);
                break;
            }
        }
        for (int j0 = 0; j0 < k; j0 += 64) {
            const int j = j0 + lane;
            int v = j < k ? numbers[wave][j] : -1;
            float w = j < k ? wants[wave][j] : 0.f;
            bool twice = false;
            if (v >= 0) {
                int at = place_in_table(v, mask);
                while ((table[wave][at] & ~kTwice) != (unsigned)v) at = (at + 1) & mask;
                twice = (table[wave][at] & kTwice) != 0;
            }
            const int named = v;
            for (unsigned long long left = __builtin_amdgcn_ballot_w64(twice); left; left &= left - 1) {
                const int l = __builtin_ctzll(left), of = __builtin_amdgcn_readlane(named, l);
                float all = 0.f;
                int first = k;
                for (int i = lane; i < k; i += 64)
                    if (numbers[wave][i] == of) { all += wants[wave][i]; first = min(first, i); }
                all = over_wave(all);
                for (int d = 32; d > 0; d >>= 1) first = min(first, __shfl_xor(first, d));
                if (lane == l) { w = first < j ? 0.f : all; v = first < j ? -1 : v; }
            }
            if (j < k) { index[row + j] = v; q[row + j] = w; }
        }
        if (lane == 0) weight[t] = any ? dloss ? dloss[t] * tau : tau : 0.f;
    }
}

// Lists of the entries by tile: a workgroup for each kGroup tokens counts the entries of every vocabulary tile (1 << log_tm entries), forms their places
// and writes them, with q or, without, with their place among all.  The order within a tile's run varies; two items of
// one element do not meet: without q they have places of their own, with q entries_kernel has left one.  Latency bounds it: 37 x 8 entries 5 us, 4096 x 64 7,
// 4096 x 1024 24 (a list for all tokens of a tile: 23 and 290, and its tiles looked through as much as sixteen times the items).
constexpr int kMostTiles = 1 << 14, kHeldEntries = kGroup;         // entries of each of 1024 threads: a token has up to 1024
template <bool I64>
__global__ __launch_bounds__(1024) void lists_kernel(const void* __restrict__ index, const float* __restrict__ q, const int* __restrict__ from, const int* __restrict__ count,
                                                     int tokens, int vocab, int k, int log_tm, int tiles, int* __restrict__ starts, int2* __restrict__ items)
{
    __shared__ int counts[kMostTiles];
    __shared__ int sums[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (count) tokens = *count;
    const int t0 = blockIdx.x * kGroup, here = min(kGroup, tokens - t0) * k;
    if (here <= 0) return;
    const int64_t base = (int64_t)t0 * k;
    // entries 1024 j + thread: -1 for those that name nothing, their tokens of the group, and where they lie
    int held[kHeldEntries], token[kHeldEntries];
    unsigned source[kHeldEntries];
    float wanted[kHeldEntries];
    const int step = 1024 / k, step_rest = 1024 % k;               // (one division, not one for each entry)
    int t = (int)threadIdx.x / k, rest = (int)threadIdx.x % k;
#pragma unroll
    for (int j = 0; j < kHeldEntries; ++j) {
        token[j] = t;
        if (j * 1024 < here) source[j] = j * 1024 + (int)threadIdx.x >= here ? 0u : from ? (unsigned)from[t0 + t] * k + rest : (unsigned)(base + t * k + rest);
        t += step;
        rest += step_rest;
        if (rest >= k) { rest -= k; ++t; }
    }
#pragma unroll
    for (int j = 0; j < kHeldEntries; ++j) {
        held[j] = -1;
        if (j * 1024 >= here) continue;
        const int64_t v = I64 ? ((const int64_t*)index)[source[j]] : (int64_t)((const int*)index)[source[j]];
        held[j] = j * 1024 + (int)threadIdx.x < here && v >= 0 && v < vocab ? (int)v : -1;
        if (q) wanted[j] = q[source[j]];
    }
    for (int i = threadIdx.x; i < tiles; i += 1024) counts[i] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kHeldEntries; ++j)
        if (held[j] >= 0) atomicAdd(&counts[held[j] >> log_tm], 1);
    __syncthreads();
    int* out = starts + (int64_t)blockIdx.x * (tiles + 1);
    int before = 0;
    for (int i0 = 0; i0 < tiles; i0 += 1024) {
        const int i = i0 + threadIdx.x, n = i < tiles ? counts[i] : 0;
        int inc = n;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(inc, d);
            if (lane >= d) inc += o;
        }
        if (lane == 63) sums[wave] = inc;
        __syncthreads();
        int at = before + inc - n, all = 0;
        for (int w = 0; w < 16; ++w) {
            if (w < wave) at += sums[w];
            all += sums[w];
        }
        if (i < tiles) { out[i] = at; counts[i] = at; }
        before += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) out[tiles] = before;
#pragma unroll
    for (int j = 0; j < kHeldEntries; ++j) {
        const int v = held[j];
        if (v < 0) continue;
        const int at = atomicAdd(&counts[v >> log_tm], 1);
        items[base + at] = make_int2((v & ((1 << log_tm) - 1)) << 16 | token[j], q ? __float_as_int(wanted[j]) : (int)source[j]);
    }
}

// The tiles' sums joined and the loss formed: TOK tokens of a workgroup, 256 / TOK threads of a token.  8192 tokens of 500 tiles 9 us (33 MB); 4096 with 64 entries 14.
template <int TOK>
__global__ __launch_bounds__(256) void join_kernel(const float2* __restrict__ tile_stats, int tiles, int tokens, int vocab, float alpha, float tau, const void* __restrict__ targets,
                                                   int target64, const void* __restrict__ teacher, bool teacher_fp32, int k, const float* __restrict__ z, float* __restrict__ loss,
                                                   float* __restrict__ lse)
{
    constexpr int PARTS = 256 / TOK;
    __shared__ float2 shared[PARTS][TOK + 1];
    const int tok = threadIdx.x % TOK, part = threadIdx.x / TOK, t = blockIdx.x * TOK + tok;
    const bool here = t < tokens;
    // (what the loss names is fetched beside the sums)
    int64_t target = -1;
    float at_target = 0.f;
    if (here && !teacher) {
        target = target64 ? ((const int64_t*)targets)[t] : (int64_t)((const int*)targets)[t];
        at_target = z[t];
    }
    // of a distillation the first 64 entries of the tokens that this wave will take (`targets` are the entries' numbers)
    constexpr int OWN = TOK / 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    auto entry = [&](int64_t at, float& u) {
        const int64_t v = target64 ? ((const int64_t*)targets)[at] : (int64_t)((const int*)targets)[at];
        u = logit(teacher, teacher_fp32, at) * alpha;
        return v >= 0 && v < vocab && !(u == -INFINITY);
    };
    bool named[OWN];
    float u_of[OWN], z_of[OWN];
#pragma unroll
    for (int o = 0; o < OWN; ++o) {
        const int token = blockIdx.x * TOK + wave + o * 4;
        named[o] = false;
        u_of[o] = z_of[o] = 0.f;
        if (!teacher || token >= tokens || lane >= k) continue;
        named[o] = entry((int64_t)token * k + lane, u_of[o]);
        z_of[o] = z[(int64_t)token * k + lane];
    }
    float2 v = make_float2(-INFINITY, 0.f);
    for (int i0 = part; i0 < tiles; i0 += 8 * PARTS) {
        float2 o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = here && i0 + i * PARTS < tiles ? tile_stats[(int64_t)(i0 + i * PARTS) * tokens + t] : make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int i = 0; i < 8; ++i) v = join2(v, o[i]);
    }
    shared[part][tok] = v;
    __syncthreads();
#pragma unroll
    for (int n = PARTS / 2; n > 0; n >>= 1) {
        if (part < n) shared[part][tok] = v = join2(v, shared[part + n][tok]);
        __syncthreads();
    }
    v = shared[0][tok];
    const float l = fmaf(v.x, kLn2, logf(v.y));
    if (lse && part == 0 && here) lse[t] = l;
    if (!loss) return;
    if (!teacher) {
        if (part == 0 && here) loss[t] = target >= 0 && target < vocab ? l - at_target : 0.f;
        return;
    }
    // a wave for each token: q, and with it the loss
#pragma unroll
    for (int o = 0; o < OWN; ++o) {
        const int token = blockIdx.x * TOK + wave + o * 4;
        if (token >= tokens) break;
        const int64_t row = (int64_t)token * k;
        const float2 all = shared[0][wave + o * 4];
        const float of_token = fmaf(all.x, kLn2, logf(all.y));
        float top = fmaxf(-INFINITY, named[o] ? u_of[o] : -INFINITY), u, total = 0.f;
        bool any = named[o];
        for (int j = lane + 64; j < k; j += 64)
            if (entry(row + j, u)) { top = fmaxf(top, u); any = true; }
        top = top_of_wave(top);
        const float base = top == -INFINITY ? 0.f : top;
        float sum = named[o] ? expf(u_of[o] - base) : 0.f;
        for (int j = lane + 64; j < k; j += 64)
            if (entry(row + j, u)) sum += expf(u - base);
        const float log_sum = logf(over_wave(sum));
        auto add = [&](float u, float at) {
            const float log_q = u - base - log_sum, q = expf(log_q);
            // (a q that is zero has no part, whatever its logit)
            if (q != 0.f) total = fmaf(q, log_q + fmaf(-at, alpha, of_token), total);
        };
        if (named[o]) add(u_of[o], z_of[o]);
        for (int j = lane + 64; j < k; j += 64)
            if (entry(row + j, u)) add(u, z[row + j]);
        total = over_wave(total);
        const bool wanted = __builtin_amdgcn_ballot_w64(any) != 0;       // (of all lanes: a ballot sees those that run it)
        if (lane == 0) loss[token] = wanted ? total * tau * tau : 0.f;
    }
}

// dx: the partial sums of the splits, rounded; zeros for tokens that take no part.  8192 x 4096 in one split, 201 MB, 33 us: memory.  150 of 250 x 2080 in 28 splits, 35 MB,
// 18 us: loads in turn, which a thread adds up, in 254 workgroups.
__global__ __launch_bounds__(256) void dx_kernel(const float* __restrict__ sums, int splits, int64_t stride, int tokens, int cols, const int* __restrict__ place,
                                                 const float* __restrict__ unit, uint16_t* __restrict__ dx, int64_t ld)
{
    const float scale = *unit;
    const int chunks = cols / 8;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < (int64_t)tokens * chunks; u += (int64_t)gridDim.x * 256) {
        const int64_t t = u / chunks;
        const int c = (int)(u % chunks) * 8;
        float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        const int64_t at = place[t];
        if (at >= 0)
            for (int i = 0; i < splits; ++i) {
                const float4* s = reinterpret_cast<const float4*>(sums + i * stride + at * cols + c);
                const float4 a = s[0], b = s[1];
                f[0] += a.x; f[1] += a.y; f[2] += a.z; f[3] += a.w; f[4] += b.x; f[5] += b.y; f[6] += b.z; f[7] += b.w;
            }
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] *= scale;
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

constexpr int64_t up(int64_t n, int64_t m) { return (n + m - 1) / m * m; }
size_t to256(size_t n) { return (n + 255) / 256 * 256; }

enum class Shape { kLarge, kMiddle, kFew64, kFew32, kLow64, kLow32 };
constexpr int tile_rows(Shape s) { return s == Shape::kLarge ? 256 : s == Shape::kLow64 || s == Shape::kLow32 ? 64 : 128; }
constexpr int tile_cols(Shape s) { return s == Shape::kLarge ? 256 : s == Shape::kMiddle ? 128 : s == Shape::kFew64 || s == Shape::kLow64 ? 64 : 32; }
constexpr int64_t stages_of(int64_t n) { return (n + 63) / 64; }
constexpr int64_t tiles_of(Shape s, int64_t I, int64_t J) { return up(I, tile_rows(s)) / tile_rows(s) * (up(J, tile_cols(s)) / tile_cols(s)); }
// About how long `units` tiles of so many stages take, us: a stage and what comes before and behind them, for as many at a time as the chip holds.  Measured: 256 x
// 256 1.45-1.6 us a stage and 8 (8192 x 4096 against 128000: 64 stages, 100 us a tile; dw of 250 tokens: 4 stages, 14.4), 128 x 128 by two workgroups of a
// compute unit 1.1-1.4 and 2.5 (515 x 1024 against 8191: 16 stages, 21; dw of 250 tokens: 7.1).
constexpr int64_t kUnits = 256, kLastLevelCache = 256 << 20;
double tile_time(Shape s, int64_t units, int64_t stages)
{
    return s == Shape::kLarge ? (double)((units + kUnits - 1) / kUnits) * (1.5 * stages + 8.4) : (double)((units + 2 * kUnits - 1) / (2 * kUnits)) * (1.2 * stages + 2.5);
}
Shape faster(int64_t I, int64_t J, int64_t R)
{
    return tile_time(Shape::kLarge, tiles_of(Shape::kLarge, I, J), stages_of(R)) < tile_time(Shape::kMiddle, tiles_of(Shape::kMiddle, I, J), stages_of(R)) ? Shape::kLarge : Shape::kMiddle;
}
// Tiles as narrow as tokens are few.
Shape few(int64_t tokens, bool low) { return tokens <= 32 ? low ? Shape::kLow32 : Shape::kFew32 : tokens <= 64 ? low ? Shape::kLow64 : Shape::kFew64 : Shape::kMiddle; }
// The tile for I x J outputs of a contraction of R, J of them tokens.  Few tokens: 64 rows where tiles of 128 are no more than one for each compute unit (16 tokens, loss of
// 32000 x 2048: 34.0 us, 128 rows 37.3; of 50257 x 1024, 1.5 for each: 27.7 and 26.5).
Shape shape_for(int64_t I, int64_t J, int64_t R)
{
    return J <= 128 ? few(J, up(I, 128) / 128 <= kUnits) : faster(I, J, R);
}

template <class T, int OUT> hipError_t launch_product(ProductArgs p, int splits, hipStream_t s)
{
    p.tiles_i = (p.I + T::TM - 1) / T::TM;
    p.tiles_j = (p.J + T::TN - 1) / T::TN;
    hipLaunchKernelGGL((product_kernel<T, OUT>), dim3((unsigned)(p.tiles_i * p.tiles_j), (unsigned)splits), dim3(T::NT), 0, s, p);
    return hipGetLastError();
}
// Stages of dw's tiles up to which it shares a launch with dx.  us of a call, shared and not: 515 x 1024 against 8191 (4608) 65.6 and 73, 16 x 2048 against 32000 (4000)
// 113 and 118, 250 x 1024 against 50257 (12576) 153 and 158; 500 x 1024 against 50257 (25152) 244 and 240.
constexpr int64_t kPairStages = 1 << 14;
template <class X> hipError_t launch_pair(ProductArgs dx, int splits, ProductArgs dw, hipStream_t s)
{
    dx.tiles_i = (dx.I + X::TM - 1) / X::TM; dx.tiles_j = (dx.J + X::TN - 1) / X::TN;
    dw.tiles_i = (dw.I + Middle::TM - 1) / Middle::TM; dw.tiles_j = (dw.J + Middle::TN - 1) / Middle::TN;
    hipLaunchKernelGGL((pair_kernel<X, Middle>), dim3((unsigned)(dx.tiles_i * dx.tiles_j * splits + dw.tiles_i * dw.tiles_j)), dim3(256), 0, s, dx, splits, dw);
    return hipGetLastError();
}
hipError_t launch_pair(const ProductArgs& dx, Shape shape, int splits, const ProductArgs& dw, hipStream_t s)
{
    switch (shape) {
    case Shape::kFew64: return launch_pair<Few64>(dx, splits, dw, s);
    case Shape::kFew32: return launch_pair<Few32>(dx, splits, dw, s);
    case Shape::kLow64: return launch_pair<Low64>(dx, splits, dw, s);
    case Shape::kLow32: return launch_pair<Low32>(dx, splits, dw, s);
    default:            return launch_pair<Middle>(dx, splits, dw, s);
    }
}
template <int OUT> hipError_t launch_product(const ProductArgs& p, Shape shape, int splits, hipStream_t s)
{
    if (shape == Shape::kLarge) return launch_product<Large, OUT>(p, splits, s);
    if constexpr (OUT != kDw) {
        if (shape == Shape::kFew64) return launch_product<Few64, OUT>(p, splits, s);
        if (shape == Shape::kFew32) return launch_product<Few32, OUT>(p, splits, s);
        if (shape == Shape::kLow64) return launch_product<Low64, OUT>(p, splits, s);
        if (shape == Shape::kLow32) return launch_product<Low32, OUT>(p, splits, s);
    }
    return launch_product<Middle, OUT>(p, splits, s);
}

// The backward call's pieces of the vocabulary, and the tiles and splits of dx.  They go by all tokens: how many take part is known on the device only, so where most do not,
// dx has fewer splits than its tiles would bear.
// Pieces are as large as 2^28 elements of dz, 537 MB, allow: with half of that dx is read and added to once more, 1 % of a step of 8192 tokens against 128000 entries.
struct Plan { int64_t piece, splits; Shape dx; };
constexpr int64_t kPieceElements = 1 << 28, kLeastPiece = 4096, kMostPiece = 1 << 17, kSplitElements = 1 << 25;
// Splits of `here` entries, none of them empty, that are no more than `most`.
int64_t splits_of(int64_t here, int64_t most)
{
    const int64_t per = (stages_of(here) + most - 1) / most;
    return (stages_of(here) + per - 1) / per;
}
Plan plan_of(const VocabLossArgs& a)
{
    Plan r;
    r.piece = std::min(up(a.vocab, 256), std::min(kMostPiece, std::max(kLeastPiece, kPieceElements / a.tokens / 256 * 256)));
    // splits of dx: those of 512 entries at least whose products and partial sums (written, read: 4 TB/s) take least, within kSplitElements
    const int64_t first = std::min(r.piece, a.vocab), most = std::max<int64_t>(1, std::min({kSplitElements / (a.tokens * a.cols), r.piece / 512, (int64_t)256}));
    double least = 0;
    r.splits = 0;
    auto consider = [&](Shape s) {
        const int64_t tiles = tiles_of(s, a.cols, a.tokens), at_a_time = s == Shape::kLarge ? kUnits : 2 * kUnits;
        for (int64_t halves : {0, 1, 2, 4, 6}) {                     // rounds of workgroups, in halves
            const int64_t splits = splits_of(first, std::max<int64_t>(1, std::min(most, halves * at_a_time / (2 * tiles))));
            const double t = tile_time(s, tiles * splits, (stages_of(first) + splits - 1) / splits) + (double)(a.tokens * a.cols * splits) * 8 / 4e6;
            if (r.splits == 0 || t < least) { least = t; r.splits = splits; r.dx = s; }
        }
    };
    if (a.tokens <= 128) {
        // (w of the piece comes from the last-level cache, where dz's pass has left it, or as it did there from memory.  16 tokens, 64 and 128 rows, us of the call:
        // 50257 x 768 56 and 67, 128000 x 1024 124 and 132; 128000 x 2048 239 and 232, 128000 x 4096 452 and 432)
        consider(few(a.tokens, first * a.cols * 2 <= kLastLevelCache));
    } else {
        consider(Shape::kLarge);
        consider(Shape::kMiddle);
    }
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
// Lists of a distillation's entries (without a teacher there are none).
struct Lists { int* starts; int2* items; };
Lists lists_space(const VocabLossArgs& a, Shape shape, Space& s)
{
    Lists l = {};
    if (!a.distill) return l;
    l.items = s.take<int2>((size_t)a.tokens * a.k);
    l.starts = s.take<int>((up(a.tokens, kGroup) / kGroup) * (up(a.vocab, tile_rows(shape)) / tile_rows(shape) + 1));
    return l;
}
size_t lists_bytes(int64_t tokens, int64_t vocab, int64_t k)
{
    return to256((size_t)tokens * k * 8) + to256((size_t)(up(tokens, kGroup) / kGroup) * (up(vocab, 64) / 64 + 1) * 4);
}
struct Forward { Lists l; float* z; float2* stats; Shape shape; size_t bytes; };
Forward forward_space(const VocabLossArgs& a)
{
    Space s{(uint8_t*)a.workspace};
    Forward f;
    f.shape = shape_for(a.vocab, a.tokens, a.cols);
    f.l = lists_space(a, f.shape, s);
    f.z = s.take<float>((size_t)a.tokens * a.k);
    f.stats = s.take<float2>((size_t)(up(a.vocab, tile_rows(f.shape)) / tile_rows(f.shape)) * a.tokens);
    f.bytes = s.used;
    return f;
}
struct Backward { Lists l; int* index; float *q, *weight; int *place, *at, *count; float *part, *lse, *unit, *sums; uint16_t *x, *dz; Shape shape; size_t bytes; };
Backward backward_space(const VocabLossArgs& a, const Plan& pl)
{
    Space s{(uint8_t*)a.workspace};
    Backward b;
    b.shape = shape_for(std::min(pl.piece, a.vocab), a.tokens, a.cols);
    b.l = lists_space(a, b.shape, s);
    const size_t named = a.distill ? (size_t)a.tokens * a.k : 0;
    b.index = s.take<int>(named); b.q = s.take<float>(named); b.weight = s.take<float>(a.distill ? a.tokens : 0);
    b.place = s.take<int>(a.tokens); b.at = s.take<int>(a.tokens); b.count = s.take<int>(1);
    b.part = s.take<float>(a.tokens); b.lse = s.take<float>(a.tokens); b.unit = s.take<float>(1);
    b.x = s.take<uint16_t>(a.tokens * a.cols);
    b.dz = s.take<uint16_t>(a.tokens * pl.piece);
    b.sums = s.take<float>((size_t)a.tokens * a.cols * pl.splits);
    b.bytes = s.used;
    return b;
}

template <bool I64> void launch_lists(const VocabLossArgs& a, const void* index, const float* q, const int* from, const int* count, const Lists& l, Shape shape, hipStream_t s)
{
    const int64_t tm = tile_rows(shape);
    hipLaunchKernelGGL(lists_kernel<I64>, dim3((unsigned)(up(a.tokens, kGroup) / kGroup)), dim3(1024), 0, s, index, q, from, count, (int)a.tokens, (int)a.vocab, (int)a.k, tm == 256 ? 8 : tm == 128 ? 7 : 6,
                       (int)((a.vocab + tm - 1) / tm), l.starts, l.items);
}
void name_entries(ProductArgs& p, const VocabLossArgs& a, const Lists& l, Shape shape)
{
    p.alpha = 1.f / a.tau; p.vocab = (int)a.vocab;
    if (!a.distill) { p.targets = a.indices; p.target64 = a.index64; return; }
    p.starts = l.starts; p.items = l.items; p.items_pitch = kGroup * a.k; p.vocab_tiles = (int)(up(a.vocab, tile_rows(shape)) / tile_rows(shape));
}

}  // namespace

size_t vocab_loss_needed(const VocabLossArgs& a) { return forward_space(a).bytes; }
size_t vocab_loss_backward_needed(const VocabLossArgs& a) { return backward_space(a, plan_of(a)).bytes; }

// Bounds of the above that grow with every extent.
size_t vocab_loss_bytes(int64_t tokens, int64_t vocab, int64_t k)
{
    return lists_bytes(tokens, vocab, k) + to256((size_t)tokens * k * 4) + to256((size_t)std::max(up(vocab, 128) / 128 * tokens, std::min(up(vocab, 64) / 64, 2 * kUnits) * std::min<int64_t>(tokens, 64)) * 8);
}
size_t vocab_loss_backward_bytes(int64_t tokens, int64_t cols, int64_t vocab, int64_t k)
{
    const int64_t piece = std::min(up(vocab, 256), kMostPiece), dz = std::min(tokens * piece, std::max(kPieceElements, tokens * kLeastPiece));
    const int64_t sums = std::min(std::max(tokens * cols, kSplitElements), tokens * cols * std::max<int64_t>(1, piece / 512));
    return lists_bytes(tokens, vocab, k) + 2 * to256((size_t)tokens * k * 4) + 5 * to256((size_t)tokens * 4) + 512 + to256((size_t)(tokens * cols) * 2) + to256((size_t)dz * 2) + to256((size_t)sums * 4);
}

hipError_t launch_vocab_loss(const VocabLossArgs& a, hipStream_t s)
{
    if (a.tokens == 0) return hipSuccess;
    const Forward f = forward_space(a);
    if (a.distill) a.index64 ? launch_lists<true>(a, a.indices, nullptr, nullptr, nullptr, f.l, f.shape, s) : launch_lists<false>(a, a.indices, nullptr, nullptr, nullptr, f.l, f.shape, s);
    ProductArgs p = {};
    p.a = a.w; p.lda = a.ldw; p.I = (int)a.vocab; p.b = a.x; p.ldb = a.ldx; p.J = (int)a.tokens; p.R = (int)a.cols;
    name_entries(p, a, f.l, f.shape);
    p.tile_stats = f.stats; p.z = f.z;
    const hipError_t e = launch_product<kStats>(p, f.shape, 1, s);
    if (e != hipSuccess) return e;
    const int tok = a.tokens >= 2048 ? 16 : 4;
    hipLaunchKernelGGL(tok == 16 ? join_kernel<16> : join_kernel<4>, dim3((unsigned)((a.tokens + tok - 1) / tok)), dim3(256), 0, s, f.stats,
                       (int)((a.vocab + tile_rows(f.shape) - 1) / tile_rows(f.shape)), (int)a.tokens, (int)a.vocab, p.alpha, a.tau, a.indices, a.index64, a.distill ? a.teacher : nullptr,
                       a.teacher_fp32 != 0, (int)a.k, f.z, a.loss, a.lse);
    return hipGetLastError();
}

hipError_t launch_vocab_loss_backward(const VocabLossArgs& a, hipStream_t s)
{
    if (a.tokens == 0) {
        const int64_t blocks = (a.vocab * (a.cols / 8) + 255) / 256;
        if (a.dw && !a.add)
            hipLaunchKernelGGL(a.dw_fp32 ? zero_kernel<true> : zero_kernel<false>, dim3((unsigned)(blocks < kMostBlocks ? blocks : kMostBlocks)), dim3(256), 0, s, a.dw, a.vocab,
                               (int)a.cols, a.lddw);
        return hipGetLastError();
    }
    const Plan pl = plan_of(a);
    const Backward b = backward_space(a, pl);
    const int64_t token_blocks = (a.tokens + 3) / 4;
    const dim3 grid((unsigned)(token_blocks < kMostBlocks ? token_blocks : kMostBlocks));
    if (a.distill)
        hipLaunchKernelGGL(a.index64 ? entries_kernel<true> : entries_kernel<false>, grid, dim3(256), 0, s, a.indices, a.teacher, a.teacher_fp32 != 0, (int)a.tokens, (int)a.vocab,
                           (int)a.k, a.tau, a.dloss, b.index, b.q, b.weight);
    const Weights weights = {a.distill ? nullptr : a.indices, a.index64, (int)a.vocab, a.dloss, b.weight};
    const bool find = a.tokens <= kFind;
    if (!find) hipLaunchKernelGGL(order_kernel, dim3(1), dim3(1024), 0, s, weights, (int)a.tokens, b.place, b.count, b.unit);
    hipLaunchKernelGGL(part_kernel, grid, dim3(256), 0, s, a.x, a.ldx, (int)a.tokens, (int)a.cols, weights, a.lse_in, find, b.place, b.count, b.unit, b.part, b.lse, b.at, b.x);
    if (a.distill) launch_lists<false>(a, b.index, b.q, b.at, b.count, b.l, b.shape, s);
    for (int64_t v0 = 0; v0 < a.vocab; v0 += pl.piece) {
        const int64_t here = std::min(pl.piece, a.vocab - v0);
        const uint16_t* w = a.w + v0 * a.ldw;
        ProductArgs p = {};
        p.a = w; p.lda = a.ldw; p.I = (int)here; p.b = b.x; p.ldb = a.cols; p.J = (int)a.tokens; p.R = (int)a.cols; p.v0 = (int)v0; p.count = b.count;
        name_entries(p, a, b.l, b.shape);
        if (!a.distill) { p.targets = b.at; p.target64 = 0; }
        p.lse = b.lse; p.part = b.part; p.c = b.dz; p.ldc = pl.piece;
        hipError_t e = launch_product<kDz>(p, b.shape, 1, s);
        if (e != hipSuccess) return e;
        ProductArgs x = {}, d = {};
        if (a.dx) {
            // dz is zero up to a whole tile, w has no row past the piece
            x.a = w; x.lda = a.ldw; x.I = (int)a.cols; x.b = b.dz; x.ldb = pl.piece; x.J = (int)a.tokens; x.R = (int)here;
            x.split = (int)((up(here, 64) / 64 + pl.splits - 1) / pl.splits);
            x.c = b.sums; x.ldc = a.cols; x.split_stride = a.tokens * a.cols; x.add = v0 > 0; x.count = b.count;
        }
        if (a.dw) {
            d.a = b.x; d.lda = a.cols; d.I = (int)a.cols; d.b = b.dz; d.ldb = pl.piece; d.J = (int)here; d.R = (int)a.tokens;
            d.c = a.dw_fp32 ? (void*)((float*)a.dw + v0 * a.lddw) : (void*)((uint16_t*)a.dw + v0 * a.lddw);
            d.ldc = a.lddw; d.c_fp32 = a.dw_fp32; d.add = a.add; d.unit = b.unit; d.count = b.count;
        }
        const Shape of_dw = faster(a.cols, here, a.tokens);
        if (a.dx && a.dw && pl.dx != Shape::kLarge && of_dw == Shape::kMiddle && tiles_of(of_dw, a.cols, here) * stages_of(a.tokens) <= kPairStages) {
            e = launch_pair(x, pl.dx, (int)pl.splits, d, s);
        } else {
            if (a.dx) e = launch_product<kDx>(x, pl.dx, (int)pl.splits, s);
            if (e == hipSuccess && a.dw) e = launch_product<kDw>(d, of_dw, 1, s);
        }
        if (e != hipSuccess) return e;
    }
    if (!a.dx) return hipSuccess;
    const int64_t blocks = (a.tokens * (a.cols / 8) + 255) / 256;
    hipLaunchKernelGGL(dx_kernel, dim3((unsigned)(blocks < kMostBlocks ? blocks : kMostBlocks)), dim3(256), 0, s, b.sums, (int)pl.splits, a.tokens * a.cols, (int)a.tokens, (int)a.cols,
                       b.place, b.unit, a.dx, a.lddx);
    return hipGetLastError();
}

}  // namespace snip
