// Moving tokens of a paged cache into other pages: forks of sequences, tokens that a sequence keeps, states of beams.
//
// Nothing is computed: bound by HBM, in 4 bits by the vector instructions that find 64 tokens' places for 9 KiB, too (62 to 66 % of the SIMDs' time), or by the chain of
// reads (starts, token, page, entry) behind which a token's values are found.  A workgroup takes 64
// neighbouring slots of the target (they lie at multiples of 64 of their sequence), whose tokens come from anywhere in the source, of one head, and has all of
// them under way before it stores any (one after the other, keys, pairs, values: 83 us for 77, 32 sequences that keep three quarters of 501 to 8000 tokens in 4 bits; several heads to a workgroup cost more than finding the tokens
// anew for each).  Keys go in 16 bytes a lane; values lie with the tokens of a page side by side, so a lane takes four
// neighbouring target tokens of a V row: four reads of one entry each, one where the four lie side by side in the source too, or (codes) close to each other, and one
// store.  (Codes, one read for four close ones: 67 us for 72, those sequences in 4 bits, 115 for 140 in 8; for 16 bits, two reads, 236 for 240, is left out.)
#include "../../include/conqur.h"
#include "common.h"

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
  int from;                  // number of the launch's first part
};

constexpr int kSlots = 64, kShift = 6, kFours = kSlots / 4;      // targets of a workgroup

template <int BITS, int W>
__global__ void __launch_bounds__(256) k_gather(const GatherArgs a) {
  typedef std::conditional_t<BITS == 16, uint16_t, uint8_t> Unit;          // a token in a V row
  typedef Unit units __attribute__((ext_vector_type(4)));
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  constexpr int kRow = W * BITS / 8, kChunks = kRow / 16, kVRows = BITS == 4 ? W / 2 : W;
  constexpr int kKeys = kSlots * kChunks / 256 ? kSlots * kChunks / 256 : 1, kValues = kVRows * kFours / 256;
  __shared__ int64_t s_from[kSlots], s_to[kSlots];          // of each target: (page * heads + head) * page_tokens + slot, in its source and its target, or -1
  const int heads = (int)a.cache.heads, head = blockIdx.x % heads, tid = threadIdx.x;
  auto edge = [&](int i) {
    const int v = a.start[i];
    return v < 0 ? 0 : v > a.count ? (int)a.count : v;
  };
  const int id = a.from + (int)(blockIdx.x / heads);
  // (rows before the first sequence have no parts: its parts are numbered from its own edge on)
  int first, next;
  const int b = sequence_of_part(id, a.sequences, kShift, 1, edge, &first, &next);
  const int count = next - first, part = id - ((first >> kShift) + b);
  if (part < 0 || part * kSlots >= count) return;
  const int page_tokens = (int)a.cache.page_tokens, shift = 31 - __builtin_clz(page_tokens);
  if (tid < kSlots) {
    const int i = part * kSlots + tid;
    int64_t from = -1, to = -1;
    if (i < count) {
      const int64_t to_column = i >> shift;
      const int32_t token = a.tokens[first + i], to_page = to_column < a.to_columns ? a.to_table[b * a.to_stride + to_column] : -1;
      const int64_t column = token < 0 ? a.columns : token >> shift;
      const int32_t page = column < a.columns ? a.table[b * a.table_stride + column] : -1;
      if (page >= 0 && (uint64_t)page < a.cache.pages && to_page >= 0 && (uint64_t)to_page < a.cache.pages) {
        from = (((int64_t)page * heads + head) << shift) + (token & (page_tokens - 1));
        to = (((int64_t)to_page * heads + head) << shift) + (i & (page_tokens - 1));
      }
    }
    s_from[tid] = from;
    s_to[tid] = to;
  }
  __syncthreads();

  // Four target tokens of some V rows, the threads' 256 / kFours apart.
  const int t0 = (tid & (kFours - 1)) * 4;
  Unit* const v = static_cast<Unit*>(a.cache.v);
  auto in_v = [&](int64_t x) { return (((x >> shift) * kVRows + tid / kFours) << shift) + (x & (page_tokens - 1)); };
  int64_t at[4];
  bool every = true, side_by_side = true;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t x = s_from[t0 + j];
    every = every && x >= 0;
    side_by_side = side_by_side && x >= 0 && x == s_from[t0] + j;
    at[j] = x < 0 ? -1 : in_v(x);
  }
  side_by_side = side_by_side && at[0] % 4 == 0 && ((s_from[t0] ^ s_from[t0 + 3]) >> shift) == 0;
  units values[kValues];
  // Codes of four tokens that lie within 16 of a page, as those of a sequence that drops some do, come with one read for the four.
  int64_t window = 0;
  bool near = false;
  if constexpr (BITS != 16) {
    const int64_t low = min(min(s_from[t0], s_from[t0 + 1]), min(s_from[t0 + 2], s_from[t0 + 3])), high = max(max(s_from[t0], s_from[t0 + 1]), max(s_from[t0 + 2], s_from[t0 + 3]));
    const int slot = (int)(low & (page_tokens - 1)) & ~3, from = slot < page_tokens - 16 ? slot : page_tokens - 16;      // (pages hold 16 tokens or more)
    near = every && (low >> shift) == (high >> shift) && (int)(high & (page_tokens - 1)) - from < 16;
    window = in_v((low >> shift << shift) + from);
  }
  if (near && !side_by_side) {
    u32x4 all[kValues];
#pragma unroll
    for (int i = 0; i < kValues; ++i) __builtin_memcpy(&all[i], __builtin_assume_aligned(v + window + ((int64_t)(i * (256 / kFours)) << shift), 4), 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int byte = (int)(at[j] - window);
#pragma unroll
      for (int i = 0; i < kValues; ++i) {
        const uint32_t a = byte & 4 ? all[i][1] : all[i][0], b = byte & 4 ? all[i][3] : all[i][2];
        values[i][j] = (Unit)((byte & 8 ? b : a) >> (byte & 3) * 8);
      }
    }
  } else if (side_by_side) {
#pragma unroll
    for (int i = 0; i < kValues; ++i) values[i] = *reinterpret_cast<const units*>(v + at[0] + ((int64_t)(i * (256 / kFours)) << shift));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (at[j] >= 0) {
#pragma unroll
        for (int i = 0; i < kValues; ++i) values[i][j] = v[at[j] + ((int64_t)(i * (256 / kFours)) << shift)];
      }
  }
  // 16 bytes of a key.
  u32x4 keys[kKeys];
#pragma unroll
  for (int i = 0; i < kKeys; ++i) {
    const int x = tid + 256 * i, t = x / kChunks;
    if (x < kSlots * kChunks && s_from[t] >= 0) keys[i] = *reinterpret_cast<const u32x4*>(static_cast<const unsigned char*>(a.cache.k) + s_from[t] * kRow + x % kChunks * 16);
  }
  // A pair of each side.
  float2 pair;
  float2* const pairs = reinterpret_cast<float2*>(tid < kSlots ? a.cache.k_scale : a.cache.v_scale);
  static_assert(2 * kSlots <= 256, "");
  const bool has_pair = BITS != 16 && tid < 2 * kSlots && s_from[tid & (kSlots - 1)] >= 0;
  if (has_pair) pair = pairs[s_from[tid & (kSlots - 1)]];

#pragma unroll
  for (int i = 0; i < kKeys; ++i) {
    const int x = tid + 256 * i, t = x / kChunks;
    if (x < kSlots * kChunks && s_from[t] >= 0) *reinterpret_cast<u32x4*>(static_cast<unsigned char*>(a.cache.k) + s_to[t] * kRow + x % kChunks * 16) = keys[i];
  }
  if (has_pair) pairs[s_to[tid & (kSlots - 1)]] = pair;
  if (every) {
    Unit* const to = v + in_v(s_to[t0]);
#pragma unroll
    for (int i = 0; i < kValues; ++i) *reinterpret_cast<units*>(to + ((int64_t)(i * (256 / kFours)) << shift)) = values[i];
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (at[j] >= 0) {
        Unit* const to = v + in_v(s_to[t0 + j]);
#pragma unroll
        for (int i = 0; i < kValues; ++i) to[(int64_t)(i * (256 / kFours)) << shift] = values[i][j];
      }
  }
}

template <int BITS>
void launch(const GatherArgs& a, uint32_t blocks, hipStream_t s) {
  if (a.cache.width == 128)
    k_gather<BITS, 128><<<blocks, 256, 0, s>>>(a);
  else
    k_gather<BITS, 64><<<blocks, 256, 0, s>>>(a);
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
  const uint64_t parts = c->count / kSlots + c->sequences + 1;
  GatherArgs a = {c->cache, c->tokens, c->start, c->table, c->to_table, c->table_stride, c->to_stride, (int64_t)c->count, (int)c->table_columns,
                        (int)c->to_columns, (int)c->sequences, 0};
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const uint64_t most = ((1ull << 24) - 1) / c->cache.heads;          // parts of a launch, whose threads 32 bits count
  for (uint64_t from = 0; from < parts; from += most) {
    const uint32_t blocks = (uint32_t)((parts - from < most ? parts - from : most) * c->cache.heads);
    a.from = (int)from;
    if (c->cache.bits == 16)
      launch<16>(a, blocks, s);
    else if (c->cache.bits == 8)
      launch<8>(a, blocks, s);
    else
      launch<4>(a, blocks, s);
    if (hipGetLastError() != hipSuccess) return CONQUR_EHIP;
  }
  return CONQUR_OK;
}
