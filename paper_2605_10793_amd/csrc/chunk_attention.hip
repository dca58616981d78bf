// Attention of a chunk of new tokens of each sequence, any number of them, over a paged cache that holds them already.
//
//   u_ij = scale q_i k_j, s_ij = cap tanh(u_ij / cap) (cap 0: u_ij) - slope |i - j|, seen are max(0, first_i, i - window + 1) <= j < min(length, last_i)
//   o_i = sum_j e^(s_ij - m_i) v_j / sum_j e^(s_ij - m_i)
//
// i, j: places in the sequence.  Few rows of a cache head (its query heads times the new tokens) are bound by HBM and take the kernel of
// tree_attention_few.h, many the one of tree_attention_wide.h, with bounds in the place of masks: blocks of 64 keys that all rows see take the way of committed
// tokens there, the others the way with every case.
#include "tree_attention_few.h"

using namespace conqur;
using namespace conqur::tree;

namespace {

// Sixteens of rows that a wavefront takes straight from memory (more would not fit its registers).
constexpr int few_tiles(int bits, int width, bool options) { return bits == 16 || (bits == 8 && width == 128 && options) ? 1 : 2; }

template <int BITS, int W, int KIND>
hipError_t launch(const TreeArgs& a, int qt, dim3 grid, hipStream_t s) {
  constexpr int kMostTiles = few_tiles(BITS, W, KIND == kOptions);
  const bool one_page = a.cache.page_tokens >= (uint32_t)kBlock;
  if (qt == 1 && one_page)
    k_tree<BITS, W, 1, true, KIND><<<grid, 64 * kWaves, 0, s>>>(a);
  else if (qt == 1)
    k_tree<BITS, W, 1, false, KIND><<<grid, 64 * kWaves, 0, s>>>(a);
  else if (one_page)
    k_tree<BITS, W, kMostTiles, true, KIND><<<grid, 64 * kWaves, 0, s>>>(a);
  else
    k_tree<BITS, W, kMostTiles, false, KIND><<<grid, 64 * kWaves, 0, s>>>(a);
  return hipGetLastError();
}
template <int BITS, int W>
hipError_t launch(const TreeArgs& a, int qt, dim3 grid, hipStream_t s) {
  return a.cap_log2 != 0.0f || a.slopes ? launch<BITS, W, kOptions>(a, qt, grid, s) : launch<BITS, W, kChunk>(a, qt, grid, s);
}

constexpr int64_t kMaxStride = 1ll << 40;
constexpr uint64_t kMostRoom = 512ull << 20;          // bytes of workspace that a call may take to be cut into more runs than fill the device

struct Plan {
  bool wide;
  int qt, tile_rows, row_tiles, row_shift, splits, min_blocks, tail, tile_by_tile;
  uint64_t tiles;            // row tiles of all sequences at most
  int64_t context;
};

// What `splits` runs leave there: a row's sum of values, its maximum and sum of weights, of two pieces each, or of one where there is one sequence.
uint64_t room_of(const conqur_chunk_call& c, const Plan& p, int64_t splits) {
  return (uint64_t)c.cache.heads * p.row_tiles * (c.batch.sequences > 1 ? 2 : 1) * splits * p.tile_rows * (c.cache.width + 2) * sizeof(float);
}

Plan plan_of(const conqur_chunk_call& c) {
  Plan p;
  const int64_t room = (int64_t)c.batch.table_columns * c.cache.page_tokens;
  p.context = (int64_t)(c.max_context < (uint64_t)room ? c.max_context : (uint64_t)room);
  const int64_t rows = (int64_t)c.max_query * (c.q.heads / c.cache.heads);
  // (17 to 32 rows of codes take two tiles of 16 where one of 32 does not fit: 28 rows of 8 bits with a bias 104 us, in the kernel of many rows 317.)
  p.wide = rows > (c.cache.bits == 16 ? 16 : 32);
  p.qt = rows <= 16 ? 1 : few_tiles((int)c.cache.bits, (int)c.cache.width, c.cap != 0.0f || c.slopes);
  if (p.wide) {
    // Rows of a wavefront in sixteens: as few as pad the rows least, but for more than three full wavefronts' all that its registers hold (3108 rows of 8 bits: 16 a
    // wavefront 1433 us, 32 990, 48 870).
    const int most = c.cache.bits == 16 && c.cache.width == 128 ? 2 : 3;
    int64_t least = 1ll << 62;
    for (int qt = rows > 192 ? most : 1; qt <= most; ++qt) {
      const int64_t padded = (rows + 64 * qt - 1) / (64 * qt) * qt;
      if (padded <= least) {
        least = padded;
        p.qt = qt;
      }
    }
  }
  p.tile_rows = 16 * p.qt * (p.wide ? kWaves : 1);
  p.row_tiles = (int)((rows + p.tile_rows - 1) / p.tile_rows);
  p.row_shift = 31 - __builtin_clz(p.tile_rows);
  p.tiles = p.row_tiles == 1 ? c.batch.sequences : ((c.tokens * (c.q.heads / c.cache.heads)) >> p.row_shift) + c.batch.sequences;
  const int64_t groups = (int64_t)c.cache.heads * p.row_tiles, sequences = c.batch.sequences;
  const int64_t blocks = p.context > kBlock ? (p.context + kBlock - 1) / kBlock : 1;
  p.min_blocks = kWaves;
  p.tile_by_tile = 0;
  // As many runs as fill the device, or a few times that: the smallest number whose last turn leaves less than a tenth of it idle (17 tiles of 8 heads, 30011
  // tokens in 8 bits: 3 runs 870 us with 408 workgroups, 7 runs 650), or the best of those whose parts take no more than kMostRoom and are written and read in
  // the time that is saved, at 400 operations a byte.  (Without regard to that, 8256 tokens of one sequence by themselves took 784 us with parts of 786 MiB, and now 691 with none;
  // 2112 120, now 89.  Over 30000, 8256 take 5.08 ms with parts of 393 MiB, 5.52 with none.  24600 tokens, 8 bits, over 40000: 28.5 ms with none, 27.4 with 1563 MiB.)
  const int64_t most = (blocks * sequences + p.min_blocks - 1) / p.min_blocks, fill = kSlots / groups < 1 ? 1 : kSlots / groups;
  auto share_of = [&](int64_t s) { return (double)(groups * s) / (double)((groups * s + kSlots - 1) / kSlots * kSlots); };
  const double work = 4.0 * c.cache.width * c.q.heads * (double)c.tokens * ((double)p.context - 0.5 * (double)(c.max_query < p.context ? c.max_query : p.context));
  int64_t splits = fill;
  for (int64_t s = fill + 1; s <= 16 && share_of(splits) < 0.9; ++s) {
    const uint64_t room = room_of(c, p, s);
    if (share_of(s) > share_of(splits) && room <= kMostRoom && work * (1.0 - share_of(fill) / share_of(s)) > 400.0 * (double)room) splits = s;
  }
  if (splits > most) splits = most;
  // Row tiles are all cut into as many runs, and the first of them has every sequence, the others only those with as many new tokens.  Where a call's tokens make fewer
  // tiles than so many sequences could, there are as many runs as give the first tile the share of the device that it has of all of them, and they are taken
  // first; other tiles' are not shorter than a quarter of them, or 16 blocks.  16 bits, 640 new tokens of one of 64 sequences of 8000 and one of the others: 4400 us, 611 so (1405
  // without an order); 512 of 4 of them 3890 and 846; 300 of one of 64 of 1000, one of which has 60000: 635 and 149.
  if (p.row_tiles > 1 && splits > 1) {
    const int64_t held = (int64_t)(kMostRoom / room_of(c, p, 1)), uneven = kSlots * sequences / ((int64_t)c.cache.heads * (int64_t)p.tiles);
    const int64_t n = uneven < held ? (uneven < most ? uneven : most) : (held < most ? held : most);
    if (n > splits) {
      splits = n;
      const int64_t quarter = blocks * sequences / splits / 4;
      if (quarter > p.min_blocks) p.min_blocks = (int)(quarter < 16 ? quarter : 16);
      p.tile_by_tile = 1;
    }
  }
  if (splits > kMaxSplits) splits = kMaxSplits;
  const int64_t workgroups = (int64_t)c.cache.heads * (sequences * p.row_tiles < (int64_t)p.tiles ? sequences * p.row_tiles : (int64_t)p.tiles);
  // (Short sequences: a wavefront that takes two blocks, of codes for up to 16 rows four, one after the other costs less than the join: a token of one sequence of 500 tokens, 4 bits, 11.7 us for
  // 14.5, 16 bits, capped, 17.2 for 17.9; 3 tokens of 4 of 1000, 8 bits, width 64, 11.8 for 17.8; but one token at 777 in 16 bits, capped, 21.8 for 16.1,
  // 8 tokens at 900 in 4 bits 22.0 for 18.9.)
  // (Nor is it worth cutting 16 blocks where a quarter of the workgroups that the device holds have them, or 32 where half have: 8 tokens of 32 sequences of 300 to 1000, 4 bits,
  // 21.9 us for 38.7, one token of 16 of them, 16 bits, 23.0 for 26.5; 4 tokens of 32 of 2000, 8 bits with a bias, 33.2 for 39.7.)
  const int64_t short_blocks = p.wide ? kWaves : (c.cache.bits == 16 || rows > 16 ? 2 : 4) * kWaves;
  const bool alone = splits < 2 || blocks <= short_blocks || (blocks <= 32 && workgroups >= (p.wide ? kSlots : kSlots / 2)) || (!p.wide && blocks <= 16 && workgroups >= kSlots / 4) ||
                     (blocks <= 128 && workgroups >= 4 * kSlots);
  p.tail = p.wide || (c.cache.bits != 16 && blocks * sequences >= 8 * splits) ? 4 : 0;
  p.splits = alone || sequences > kMaxScan || (blocks + p.tail) * sequences + 2 * kMaxSplits >= 1ll << 31 ? 0 : (int)splits;
  return p;
}

bool call_fine(const conqur_chunk_call* c) {
  if (!c || !cache_fine(c->cache) || !batch_fine(c->batch) || c->tokens >= 1ull << 31 || c->max_context >= 1ull << 31) return false;
  if (!scores_fine(c->scale, c->cap) || c->window >= 1u << 31 || c->max_query < 1) return false;
  if (c->q.heads < 1 || c->q.heads % c->cache.heads || c->q.heads / c->cache.heads > 64 || c->out.heads != c->q.heads) return false;
  return c->max_query * (c->q.heads / c->cache.heads) < 1ull << 24;
}

bool rows_fine(const conqur_heads& h, uint32_t width, uint64_t tokens, bool output) {
  if (!h.data || reinterpret_cast<uintptr_t>(h.data) % 2) return false;
  if (h.token_stride < 0 || h.token_stride >= kMaxStride || h.head_stride < 0 || h.head_stride >= kMaxStride) return false;
  if (!output) return true;
  const __int128 w = width, ts = h.token_stride, hs = h.head_stride, heads = h.heads, n = tokens;
  if ((heads > 1 && hs < w) || (n > 1 && ts < w)) return false;
  return !(heads > 1 && n > 1 && ts < (heads - 1) * hs + w && hs < (n - 1) * ts + w);
}

}  // namespace

hipError_t conqur::tree::launch_chunk_few(const TreeArgs& a, int qt, dim3 grid, hipStream_t s) {
  if (a.cache.width == 128)
    return a.cache.bits == 16 ? launch<16, 128>(a, qt, grid, s) : a.cache.bits == 8 ? launch<8, 128>(a, qt, grid, s) : launch<4, 128>(a, qt, grid, s);
  return a.cache.bits == 16 ? launch<16, 64>(a, qt, grid, s) : a.cache.bits == 8 ? launch<8, 64>(a, qt, grid, s) : launch<4, 64>(a, qt, grid, s);
}

extern "C" uint64_t conqur_chunk_attention_workspace(const conqur_chunk_call* call) {
  if (!call_fine(call)) return 0;
  const Plan p = plan_of(*call);
  return room_of(*call, p, p.splits);
}

extern "C" conqur_status conqur_chunk_attention(const conqur_chunk_call* c, void* stream) {
  if (!call_fine(c)) return CONQUR_EINVAL;
  if (c->tokens == 0) return CONQUR_OK;
  if (!rows_fine(c->q, c->cache.width, c->tokens, false) || !rows_fine(c->out, c->cache.width, c->tokens, true)) return CONQUR_EINVAL;
  if (reinterpret_cast<uintptr_t>(c->first) % 4 || reinterpret_cast<uintptr_t>(c->last) % 4 || reinterpret_cast<uintptr_t>(c->slopes) % 4) return CONQUR_EINVAL;
  const Plan p = plan_of(*c);
  const uint64_t need = room_of(*c, p, p.splits);
  if (need && (!c->workspace || reinterpret_cast<uintptr_t>(c->workspace) % 16 || c->workspace_bytes < need)) return CONQUR_EINVAL;
  const uint64_t workgroups = c->cache.heads * (p.splits ? (uint64_t)p.row_tiles : p.tiles);
  if (workgroups >= 1u << 24) return CONQUR_EINVAL;          // (of 256 threads, which 32 bits count)
  TreeArgs a = {};
  a.cache = c->cache;
  a.batch = c->batch;
  a.q = static_cast<const bf16_bits*>(c->q.data);
  a.out = static_cast<bf16_bits*>(c->out.data);
  a.q_ts = c->q.token_stride;
  a.q_hs = c->q.head_stride;
  a.out_ts = c->out.token_stride;
  a.out_hs = c->out.head_stride;
  a.q_wide = reinterpret_cast<uintptr_t>(c->q.data) % 16 == 0 && a.q_ts % 8 == 0 && a.q_hs % 8 == 0;
  a.out_wide = reinterpret_cast<uintptr_t>(c->out.data) % 8 == 0 && a.out_ts % 4 == 0 && a.out_hs % 4 == 0;
  a.tokens = (int64_t)c->tokens;
  a.context = p.context;
  a.splits = p.splits;
  a.min_blocks = p.min_blocks;
  a.tile_by_tile = p.tile_by_tile;
  a.tail = p.splits ? p.tail : 0;
  a.max_query = (int)c->max_query;
  a.group = (int)(c->q.heads / c->cache.heads);
  a.tile_rows = p.tile_rows;
  a.row_tiles = p.row_tiles;
  a.row_shift = p.row_shift;
  a.tile_inverse = (uint32_t)(((1ull << 32) + p.tile_rows - 1) / p.tile_rows);
  a.part = static_cast<float*>(c->workspace);
  a.part_ml = reinterpret_cast<float2*>(a.part + need / sizeof(float) / (c->cache.width + 2) * c->cache.width);
  a.scale_log2 = c->scale * 1.4426950408889634f;
  a.chunk = 1;
  a.window = (int)c->window;
  a.looks = c->zero_rest ? (int)((c->tokens - 1) / rows_of_look((int)c->batch.sequences) + 1) : 0;
  a.workgroups = (int)workgroups * (p.splits ? p.splits : 1);
  a.first = c->first;
  a.last = c->last;
  a.slopes = c->slopes;
  a.cap_log2 = c->cap * 1.4426950408889634f;
  a.cap_in = c->cap == 0.0f ? 0.0f : 2.0f / c->cap;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const dim3 grid((uint32_t)workgroups, p.splits ? p.splits : 1);
  hipError_t e = p.wide ? launch_chunk_wide(a, p.qt, grid, s) : launch_chunk_few(a, p.qt, grid, s);
  if (e == hipSuccess && p.splits > 1) e = launch_join(a, p.wide, s);
  return e == hipSuccess ? CONQUR_OK : CONQUR_EHIP;
}
