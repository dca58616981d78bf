// Attention of new tokens over a paged cache where many rows share a cache head's keys and values (tree_attention.hip has the mathematics).
//
// Above some tens of rows the matrix units bound the call, and what would have to be read, converted and laid out
// for every 16 rows is done once for 64 QT of them: a workgroup's four wavefronts take 16 QT rows each and walk through the keys together;
// 64 keys and values at a time lie in LDS as bf16, two blocks deep, in the order of the operands and with their 16-byte chunks
// exchanged so that the 16 lanes of a quarter read from all banks.  (Reads of 16 bytes a lane are served across quarters, and for the values two quarters'
// chunks fall together: SQ_LDS_BANK_CONFLICT is 4.4e6 at the figures below, about one pass more for each read of a value operand.)  Codes are laid down less a zero within their range (integers up to 255, which
// bf16 holds), so that per row and key only the steps are left to multiply: with a zero of -offset / step that is all there is to a
// value; where that lies outside the range (a row without a sign change) or between two codes, the rest, value - step (c - zero), is
// added to the scores and the results of the block apart.
//
// Measured: 48 tokens of 8 sequences of 1000 to 16000 tokens, 32 query and 8 cache heads of 128, 8 bits (192 rows a cache head, one tile): 117 us, 456
// TFLOP/s with the join (111 with the sums of the weights as they are before they are rounded, and results a third less exact); in 16 bits
// 138, in 4 115.  What bounds it: of a wavefront's time 31 % are vector instructions (a score's
// exponential, factors and packing, a code's conversion), twice that with the two wavefronts of a SIMD; a quarter waits to issue, a third
// for LDS, memory and the barrier of every 64 keys.  What a call takes beside its 64 keys a turn, some 35 us, is mostly the partial results:
// 53 MiB written, and read again by the join (14 us).
#include "tree_attention_wide.h"

namespace conqur {
namespace tree {

namespace {

template <int BITS, int W>
hipError_t launch_rows(const TreeArgs& a, int qt, dim3 grid, hipStream_t s) {
  if (qt == 1) return launch_wide_as<BITS, W, 1, kMasks>(a, grid, s);
  if constexpr (BITS < 16 || W < 128) {
    if (qt == 3) return launch_wide_as<BITS, W, 3, kMasks>(a, grid, s);
  }
  return launch_wide_as<BITS, W, 2, kMasks>(a, grid, s);
}

}  // namespace

hipError_t launch_wide(const TreeArgs& a, int qt, dim3 grid, hipStream_t s) {
  if (a.cache.width == 128)
    return a.cache.bits == 16 ? launch_rows<16, 128>(a, qt, grid, s) : a.cache.bits == 8 ? launch_rows<8, 128>(a, qt, grid, s) : launch_rows<4, 128>(a, qt, grid, s);
  return a.cache.bits == 16 ? launch_rows<16, 64>(a, qt, grid, s) : a.cache.bits == 8 ? launch_rows<8, 64>(a, qt, grid, s) : launch_rows<4, 64>(a, qt, grid, s);
}

}  // namespace tree
}  // namespace conqur
