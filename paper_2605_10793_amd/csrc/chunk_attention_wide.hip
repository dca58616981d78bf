// The kernel of many rows of tree_attention_wide.h for chunks of new tokens (chunk_attention.hip).
#include "tree_attention_wide.h"

namespace conqur {
namespace tree {

namespace {

template <int BITS, int W, int KIND>
hipError_t launch_rows(const TreeArgs& a, int qt, dim3 grid, hipStream_t s) {
  if (qt == 1) return launch_wide_as<BITS, W, 1, KIND>(a, grid, s);
  if constexpr (BITS < 16 || W < 128) {
    if (qt == 3) return launch_wide_as<BITS, W, 3, KIND>(a, grid, s);
  }
  return launch_wide_as<BITS, W, 2, KIND>(a, grid, s);
}
template <int BITS, int W>
hipError_t launch_kind(const TreeArgs& a, int qt, dim3 grid, hipStream_t s) {
  return a.cap_log2 != 0.0f || a.slopes ? launch_rows<BITS, W, kOptions>(a, qt, grid, s) : launch_rows<BITS, W, kChunk>(a, qt, grid, s);
}

}  // namespace

hipError_t launch_chunk_wide(const TreeArgs& a, int qt, dim3 grid, hipStream_t s) {
  if (a.cache.width == 128)
    return a.cache.bits == 16 ? launch_kind<16, 128>(a, qt, grid, s) : a.cache.bits == 8 ? launch_kind<8, 128>(a, qt, grid, s) : launch_kind<4, 128>(a, qt, grid, s);
  return a.cache.bits == 16 ? launch_kind<16, 64>(a, qt, grid, s) : a.cache.bits == 8 ? launch_kind<8, 64>(a, qt, grid, s) : launch_kind<4, 64>(a, qt, grid, s);
}

}  // namespace tree
}  // namespace conqur
