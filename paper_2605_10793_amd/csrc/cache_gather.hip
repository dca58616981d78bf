// Moving tokens of a paged cache into other pages: forks of sequences, tokens that a sequence keeps, states of beams.
//
// Nothing is computed: bound by HBM.  A workgroup takes one head of 64 neighbouring slots of the target (they lie at multiples of 64 of their sequence), whose
// tokens come from anywhere in the source.  Keys go in 16 bytes a lane; values lie with the tokens of a page side by side, so a lane takes four
// neighbouring target tokens of a V row: four reads of one entry each, one where the four lie side by side in the source too, and one store.
#include "packed_attention.h"

namespace conqur {

bool cache_fine(const conqur_cache& c);

namespace {

struct GatherArgs {
  conqur_cache cache;
  const int32_t* tokens;
  const int32_t* start;
  const int32_t* table;
  const int32_t* to_table;
  int64_t table_stride, to_stride;
  int64_t count;
  int columns, to_columns, sequences;
};

constexpr int kSlots = 64;

// UNIT: bytes of a token in a V row.
template <typename UNIT>
__global__ void __launch_bounds__(256) k_gather(const GatherArgs a) {
  __shared__ int64_t s_from[kSlots], s_to[kSlots];          // page * heads + head and slot of each target, as (row of 1 token in the pool) or -1
  const int heads = (int)a.cache.heads, head = blockIdx.x % heads, tid = threadIdx.x;
  auto edge = [&](int i) {
    const int v = a.start[i];
    return v < 0 ? 0 : v > a.count ? (int)a.count : v;
  };
  const int id = blockIdx.x / heads;
  // (rows before the first sequence have no parts: its parts are numbered from its own edge on)
  const int b = packed::sequence_of_part(id, a.sequences, 6, 1, edge);
  const int first = edge(b), count = edge(b + 1) - first, part = id - ((first >> 6) + b);
  if (part < 0 || part * kSlots >= count) return;
  const int page_tokens = (int)a.cache.page_tokens, shift = 31 - __builtin_clz(page_tokens);
  if (tid < kSlots) {
    const int i = part * kSlots + tid;
    int64_t from = -1, to = -1;
    if (i < count) {
      const int32_t token = a.tokens[first + i];
      const int64_t column = token < 0 ? a.columns : token >> shift, to_column = i >> shift;
      if (column < a.columns && to_column < a.to_columns) {
        const int32_t page = a.table[b * a.table_stride + column], to_page = a.to_table[b * a.to_stride + to_column];
        if (page >= 0 && (uint64_t)page < a.cache.pages && to_page >= 0 && (uint64_t)to_page < a.cache.pages) {
          from = ((int64_t)page * heads + head) * page_tokens + (token & (page_tokens - 1));
          to = ((int64_t)to_page * heads + head) * page_tokens + (i & (page_tokens - 1));
        }
      }
    }
    s_from[tid] = from;
    s_to[tid] = to;
  }
  __syncthreads();

  const int width = (int)a.cache.width, row = width * (int)a.cache.bits / 8, chunks = row / 16, v_rows = a.cache.bits == 4 ? width / 2 : width;
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  for (int x = tid; x < kSlots * chunks; x += 256) {
    const int t = x / chunks, c = x % chunks;
    const int64_t from = s_from[t], to = s_to[t];
    if (from < 0) continue;
    const u32x4 v = *reinterpret_cast<const u32x4*>(static_cast<const unsigned char*>(a.cache.k) + from * row + c * 16);
    *reinterpret_cast<u32x4*>(static_cast<unsigned char*>(a.cache.k) + to * row + c * 16) = v;
  }
  if (a.cache.bits != 16 && tid < 2 * kSlots) {
    const int t = tid & (kSlots - 1);
    float2* const pairs = reinterpret_cast<float2*>(tid < kSlots ? a.cache.k_scale : a.cache.v_scale);
    if (s_from[t] >= 0) pairs[s_to[t]] = pairs[s_from[t]];
  }

  // Four target tokens of V rows tid / 16, 16 further, ...
  typedef UNIT units __attribute__((ext_vector_type(4)));
  const int t0 = (tid & 15) * 4;
  UNIT* const v = static_cast<UNIT*>(a.cache.v);
  int64_t at[4];
  bool every = true, side_by_side = true;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t x = s_from[t0 + j];
    every = every && x >= 0;
    side_by_side = side_by_side && x >= 0 && x == s_from[t0] + j;
    at[j] = x < 0 ? -1 : (x >> shift) * v_rows * page_tokens + (x & (page_tokens - 1));
  }
  const int64_t to0 = s_to[t0];
  side_by_side = side_by_side && at[0] % 4 == 0 && ((s_from[t0] ^ s_from[t0 + 3]) >> shift) == 0;
  if (side_by_side) {
    const UNIT* from = v + at[0] + (int64_t)(tid >> 4) * page_tokens;
    UNIT* to = v + (to0 >> shift) * v_rows * page_tokens + (to0 & (page_tokens - 1)) + (int64_t)(tid >> 4) * page_tokens;
    for (int d = tid >> 4; d < v_rows; d += 64, from += 64 * page_tokens, to += 64 * page_tokens) {
      units x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (d + 16 * j < v_rows) x[j] = *reinterpret_cast<const units*>(from + 16 * j * page_tokens);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (d + 16 * j < v_rows) *reinterpret_cast<units*>(to + 16 * j * page_tokens) = x[j];
    }
  } else if (every) {
    UNIT* to = v + (to0 >> shift) * v_rows * page_tokens + (to0 & (page_tokens - 1)) + (int64_t)(tid >> 4) * page_tokens;
    int64_t by = (int64_t)(tid >> 4) * page_tokens;
    for (int d = tid >> 4; d < v_rows; d += 32, by += 32 * page_tokens, to += 32 * page_tokens) {
      units x[2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (d + 16 * i < v_rows) {
#pragma unroll
          for (int j = 0; j < 4; ++j) x[i][j] = v[at[j] + by + 16 * i * page_tokens];
        }
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (d + 16 * i < v_rows) *reinterpret_cast<units*>(to + 16 * i * page_tokens) = x[i];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (at[j] < 0) continue;
      const int64_t t = s_to[t0 + j], to = (t >> shift) * v_rows * page_tokens + (t & (page_tokens - 1));
      for (int d = tid >> 4; d < v_rows; d += 16) v[to + (int64_t)d * page_tokens] = v[at[j] + (int64_t)d * page_tokens];
    }
  }
}

}  // namespace
}  // namespace conqur

using namespace conqur;

extern "C" conqur_status conqur_cache_gather(const conqur_gather_call* c, void* stream) {
  if (!c || !cache_fine(c->cache) || c->count >= 1ull << 31 || c->sequences < 1 || c->sequences > 65535) return CONQUR_EINVAL;
  if (c->table_columns < 1 || c->to_columns < 1 || c->table_columns >= 1u << 31 || c->to_columns >= 1u << 31) return CONQUR_EINVAL;
  if (c->count == 0) return CONQUR_OK;
  auto fine = [](const void* p) { return p && reinterpret_cast<uintptr_t>(p) % 4 == 0; };
  if (!fine(c->tokens) || !fine(c->start) || !fine(c->table) || !fine(c->to_table)) return CONQUR_EINVAL;
  if (c->table_stride < (int64_t)(c->sequences > 1 ? c->table_columns : 0) || c->to_stride < (int64_t)(c->sequences > 1 ? c->to_columns : 0)) return CONQUR_EINVAL;
  if (c->table_stride >= 1ll << 40 || c->to_stride >= 1ll << 40) return CONQUR_EINVAL;
  const uint64_t blocks = (c->count / kSlots + c->sequences + 1) * c->cache.heads;
  if (blocks >= 1ull << 31) return CONQUR_EINVAL;
  GatherArgs a = {c->cache, c->tokens, c->start, c->table, c->to_table, c->table_stride, c->to_stride, (int64_t)c->count, (int)c->table_columns,
                  (int)c->to_columns, (int)c->sequences};
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (c->cache.bits == 16)
    k_gather<uint16_t><<<dim3((uint32_t)blocks), 256, 0, s>>>(a);
  else
    k_gather<uint8_t><<<dim3((uint32_t)blocks), 256, 0, s>>>(a);
  return hipGetLastError() == hipSuccess ? CONQUR_OK : CONQUR_EHIP;
}
