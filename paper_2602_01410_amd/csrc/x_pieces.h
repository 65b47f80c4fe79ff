// Places in a token's row of the few-token kernel's input (gemv.hip), apart from the kernel so that they can be checked without a GPU.
//
// They are counted in pieces of 16 bytes (8 elements): rows have less than 2^31 elements, and chunks run past a row's end, by up to the spans of
// all shares and, where the next chunk is brought in advance, one chunk more.  In elements that passes 32 bits.
#pragma once
#ifdef __HIPCC__
#define SNIP_X_HD __host__ __device__
#else
#define SNIP_X_HD
#endif

namespace snip {

constexpr int kPieceElements = 8;
SNIP_X_HD constexpr int x_pieces(int k) { return k / kPieceElements; }                                   // of a row; k is a multiple of 32
// Piece `i` of chunk `ch` of `chunk` spans (128 elements each) of the share that begins at span `begin`.
SNIP_X_HD constexpr int x_piece(int begin, int ch, int chunk, int i) { return (begin + ch * chunk) * (128 / kPieceElements) + i; }
SNIP_X_HD constexpr long long piece_element(int piece) { return (long long)piece * kPieceElements; }

}  // namespace snip
