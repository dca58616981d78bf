// Attention of a few new tokens per sequence (a tree of drafted tokens, a chain, or one token) over a paged cache of bf16 values or
// of 8- or 4-bit zero-point codes.
//
//   s_rj = scale q_r k_j over the tokens j that row r sees, m_r = max_j s_rj, o_r = sum_j e^(s_rj - m_r) v_j / sum_j e^(s_rj - m_r)
//
// in one pass over the cache, with running maxima and sums (in base 2).  The rows of one cache head are its query heads times
// the new tokens; the cache is read once for all of them, so that few rows are bound by HBM and some hundred by the matrix units.
//
// Both products run transposed, S^T = K Q^T and O^T = V^T P^T (16x16x32 bf16 MFMA): a column is a query row, hence a lane holds
// scores of one row only, the softmax needs two lane exchanges a block, factors on O^T are the lane's own, and the layout in which
// S^T leaves the first product is, keys taken in the right order, the layout that P^T has to have in the second: weights never leave
// the registers.  Of a block of 64 keys a lane of quarter g holds keys 16 g to 16 g + 15; V lies with the tokens of a page side by
// side, so that these are 16 neighbouring values of an entry, read straight into an operand.
//
// Codes enter the products as bf16 integers (exact: 128 + code for 4 bits, code for 8), with K's step and offset applied to the
// scores and V's to the weights:
//   q k_j = step_j (q c_j) + offset_j sum q,   sum_j p_j v_j = sum_j w_j c_j + sum_j w_j offset_j / step_j,   w = p step
// The second sum, a scalar a row, takes the weights as they are rounded for the first: so the rounding of a weight is multiplied
// by the value, as with bf16 values, and not by the code (whose zero may lie far from the values' own).  The sum of the weights that
// divides the result takes them so too, over step, so that a row with one large weight gets that token's value unharmed.
//
// The kernel below is for few rows, bound by HBM: each of a workgroup's four wavefronts takes 64 keys at a time by itself, from memory straight into
// operands, and has the next 64 under way; their results meet in LDS at the end.  Measured, 32 query and 8 cache heads of 128: a
// token of 64 sequences of 501 to 8190 tokens, 16 bits, 204 to 210 us (5.4 to 5.6 TB/s); in 8 bits 121 us (5.0 TB/s), in 4 bits 86 us (3.7 TB/s, as
// much work as in 16 bits for a third of the bytes); 5 tokens of 2 sequences of 131000 tokens, 4 bits, 20 rows a cache head, 88 us (3.3
// TB/s): there the conversions, exponentials and the two products of a wavefront, two wavefronts a SIMD, are what takes the time.  One token of one
// sequence of 777 tokens 13.9 us, two launches of a chain of dependent reads.
#include "tree_attention_few.h"

using namespace conqur;
using namespace conqur::tree;

namespace {

// Joins a row's pieces.  WAVES = 1: a wavefront a row, for up to 64 pieces; 4: a workgroup a row, for up to 256.  W / 4
// lanes read a piece's result as 16-byte vectors, 256 / W pieces at a time, and the first ones are under way before the maxima are.
template <int W, int WAVES>
__global__ void __launch_bounds__(256) k_tree_join(const TreeArgs) {
  const Args a = kernel_args();
  constexpr int kLanes = W / 4, kAt = 64 / kLanes;      // lanes of a piece, pieces of a wavefront at a time
  constexpr int kFirst = 4;                             // vectors a lane takes ahead
  __shared__ float s_f[256];
  __shared__ float s_red[2][4];
  __shared__ __attribute__((aligned(16))) float s_o[4][W];

  const int b = blockIdx.y;
  const Sequence sq = sequence_of(a, b);
  const int64_t heads = a->cache.heads;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t id = WAVES == 1 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x;
  const int row = (int)(id / heads), head = (int)(id % heads);
  if (row >= sq.count * a->group) return;
  const int row_tile = row / a->tile_rows;
  const Layout layout(a, row_tile * a->tile_rows, lane);
  int from = 0, to = 0;
  layout.range(b, &from, &to);
  const int p0 = from / layout.each, chunks = (to - 1) / layout.each - p0 + 1;
  if (chunks <= 1) return;
  // the first piece may be its workgroup's last, the others are their workgroups' first
  const int slot0 = 2 * p0 + (from > p0 * layout.each);
  auto at = [&](int c) { return part_at(a, head, row_tile, c ? 2 * (p0 + c) : slot0, row - row_tile * a->tile_rows); };
  const int first = (WAVES == 1 ? 0 : wave * kAt) + lane / kLanes;
  constexpr int kNext = WAVES * kAt;
  const int entry = lane % kLanes * 4;

  f32x4 v[kFirst];
#pragma unroll
  for (int i = 0; i < kFirst; ++i)
    if (first + i * kNext < chunks) v[i] = *reinterpret_cast<const f32x4*>(a->part + at(first + i * kNext) * W + entry);
  const int mine = WAVES == 1 ? lane : (int)threadIdx.x;
  const float2 ml = mine < chunks ? a->part_ml[at(mine)] : make_float2(-INFINITY, 0.0f);
  float m = wave_max(ml.x);
  if constexpr (WAVES > 1) {
    if (lane == 0) s_red[0][wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(s_red[0][0], s_red[0][1]), fmaxf(s_red[0][2], s_red[0][3]));
  }
  const float f = ml.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml.x - m);
  float l = wave_sum(ml.y * f);
  if constexpr (WAVES > 1) {
    if (lane == 0) s_red[1][wave] = l;
    s_f[threadIdx.x] = f;
    __syncthreads();
    l = (s_red[1][0] + s_red[1][1]) + (s_red[1][2] + s_red[1][3]);
  }
  auto factor = [&](int c) { return WAVES == 1 ? __shfl(f, c) : s_f[c]; };
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
  auto add = [&](const f32x4& x, float w) {
    if (w != 0.0f) o += x * w;
  };
#pragma unroll
  for (int i = 0; i < kFirst; ++i) {
    const int c = first + i * kNext;
    const float w = factor(c & 255);
    if (c < chunks) add(v[i], w);
  }
  for (int c0 = kFirst * kNext; c0 < chunks; c0 += kNext) {
    const int c = c0 + first;
    const float w = factor(c & 255);
    if (c < chunks) add(*reinterpret_cast<const f32x4*>(a->part + at(c) * W + entry), w);
  }
#pragma unroll
  for (int off = kLanes; off < 64; off *= 2)
#pragma unroll
    for (int r = 0; r < 4; ++r) o[r] += __shfl_xor(o[r], off);
  if constexpr (WAVES > 1) {
    if (lane < kLanes) *reinterpret_cast<f32x4*>(&s_o[wave][lane * 4]) = o;
    __syncthreads();
    if (wave) return;
    o = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i) o += *reinterpret_cast<const f32x4*>(&s_o[i][lane % kLanes * 4]);
  }
  if (lane >= kLanes) return;
  store_row4(a, sq, head, row, lane * 4, o, l);
}

// Joins the pieces of 16 rows as the workgroups of many rows leave them (their registers' layout): a wavefront takes two of the result's tiles of
// 16 entries, a lane four entries of one row.
template <int W>
__global__ void __launch_bounds__(W * 2) k_tree_join_tiles(const TreeArgs) {
  const Args a = kernel_args();
  const int b = blockIdx.z, head = blockIdx.y, row0 = blockIdx.x * 16;
  const Sequence sq = sequence_of(a, b);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
  if (row0 >= sq.count * a->group) return;
  const int row_tile = row0 / a->tile_rows, in_tile = row0 - row_tile * a->tile_rows;
  const Layout layout(a, row_tile * a->tile_rows, lane);
  int from = 0, to = 0;
  layout.range(b, &from, &to);
  const int p0 = from / layout.each, pieces = (to - 1) / layout.each - p0 + 1;
  if (pieces <= 1) return;
  auto at = [&](int c) { return part_at(a, head, row_tile, c ? 2 * (p0 + c) : 2 * p0 + (from > p0 * layout.each), in_tile); };

  float m = -INFINITY;
#pragma unroll 4
  for (int c = 0; c < pieces; ++c) m = fmaxf(m, a->part_ml[at(c) + col].x);
  f32x4 o[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
  float l = 0.0f;
#pragma unroll 4
  for (int c = 0; c < pieces; ++c) {
    const float2 ml = a->part_ml[at(c) + col];
    const float* const p = a->part + at(c) * W + wave * 512 + lane * 4;
    const f32x4 v0 = *reinterpret_cast<const f32x4*>(p), v1 = *reinterpret_cast<const f32x4*>(p + 256);
    const float f = ml.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml.x - m);
    l += ml.y * f;
    if (f != 0.0f) {
      o[0] += v0 * f;
      o[1] += v1 * f;
    }
  }
  if (row0 + col >= sq.count * a->group) return;
#pragma unroll
  for (int i = 0; i < 2; ++i) store_row4(a, sq, head, row0 + col, (wave * 2 + i) * 16 + g * 4, o[i], l);
}

template <int W>
hipError_t join_pieces(const TreeArgs& a, bool wide, hipStream_t s) {
  const int64_t rows = (int64_t)a.max_query * a.group * a.cache.heads;
  if (wide)
    k_tree_join_tiles<W><<<dim3((a.max_query * a.group + 15) / 16, a.cache.heads, a.batch.sequences), W * 2, 0, s>>>(a);
  // A wavefront a row, or four where there are few rows and they have many pieces (one sequence of 30000 tokens: 33.3 us with four, 40.5 with one;
  // 16 of 2000 to 9000 tokens, 16 rows a head: 39.8 with one, 42.6 with four).
  else if (a.splits <= 64 && a.splits <= 8 * (int64_t)a.batch.sequences)
    k_tree_join<W, 1><<<dim3((uint32_t)((rows + 3) / 4), a.batch.sequences), 256, 0, s>>>(a);
  else
    k_tree_join<W, 4><<<dim3((uint32_t)rows, a.batch.sequences), 256, 0, s>>>(a);
  return hipGetLastError();
}

constexpr int64_t kMaxStride = 1ll << 40;

struct Plan {
  bool wide;
  int qt, tile_rows, row_tiles, splits, min_blocks, tail;
  int64_t context;
};

// How a call is cut: a cache head's rows into tiles, the sequences' blocks into runs.
Plan plan_of(const conqur_tree_call& c) {
  Plan p;
  const int64_t room = (int64_t)c.batch.table_columns * c.cache.page_tokens;
  p.context = (int64_t)(c.max_context < (uint64_t)room ? c.max_context : (uint64_t)room);
  const int rows = (int)(c.max_query * (c.q.heads / c.cache.heads));
  // 17 to 32 rows: of codes, a wavefront's registers hold 64 keys and values and two tiles of results (16 sequences of 3000 to 6000 tokens, 32
  // rows a head, 4 bits: 48 us, laid out in LDS 78; 8 of 4000 to 9000, 20 rows, 8 bits: 47 for 62); of bf16 they do not, and LDS is quicker (the
  // same two 77 us for 90 and 66 for 70).  All before new tokens counted for more, which took each of these a tenth down.
  p.wide = rows > (c.cache.bits == 16 ? 16 : 32);
  // Rows of a wavefront in sixteens: as few as pad the rows least; 48 rows of bf16 values 128 wide do not fit its registers.
  p.qt = rows <= 16 ? 1 : 2;
  if (p.wide) {
    const int most = c.cache.bits == 16 && c.cache.width == 128 ? 2 : 3;
    for (int qt = 1, least = 1 << 30; qt <= most; ++qt) {
      const int padded = (rows + 64 * qt - 1) / (64 * qt) * qt;
      if (padded <= least) {
        least = padded;
        p.qt = qt;
      }
    }
  }
  p.tile_rows = 16 * p.qt * (p.wide ? kWaves : 1);
  p.row_tiles = (rows + p.tile_rows - 1) / p.tile_rows;
  const int64_t groups = (int64_t)c.cache.heads * p.row_tiles, sequences = c.batch.sequences;
  const int64_t blocks = p.context > kBlock ? (p.context + kBlock - 1) / kBlock : 1;
  p.min_blocks = kWaves;
  int64_t splits = kSlots / groups;
  const int64_t most = (blocks * sequences + p.min_blocks - 1) / p.min_blocks;
  if (splits > most) splits = most;
  if (splits > kMaxSplits) splits = kMaxSplits;
  if (splits < 1) splits = 1;
  // A workgroup for each sequence, which needs no join and finds its work at once, where no sequence is so long that it would be waited for: up to 4
  // blocks (one of 200 tokens: 12.1 us for 13.8 in runs); up to 32 if they fill the device (8 heads, 64 sequences of 20 to 1000 tokens in 4 bits
  // 18.4 us for 36.8, of 600 to 2000 in 16 bits 76.5 for 78.9); up to 128 if they do so four times (256 of 500 to 4000 in 8 bits 240 for 279, of
  // 500 to 8000 in 16 bits 811 for 772).  Longer ones gain from runs: 128 of 500 to 15000 in 16 bits 716 us for 831, 64 of 501 to 8190 209 for 230.
  // More sequences than a wavefront can look through, or more blocks than 31 bits count, take that way too.
  const int64_t workgroups = sequences * groups;
  const bool alone = blocks <= kWaves || (blocks <= 32 && workgroups >= kSlots) || (blocks <= 128 && workgroups >= 4 * kSlots);
  // The new tokens, with their masks, take a workgroup as long as some four blocks of committed ones, so they count for as many, where a run is long
  // enough to be cut (48 tokens of 8 sequences of 4096, 8 bits: 70 us for 77; 20 of 16 of 3000 to 6000, 4 bits, 80 rows a head: 87 for 96, both before the
  // sums took rounded weights, which made it 92; one of 64 of
  // 501 to 8190, 4 bits: 87 for 92).  Few rows of bf16 values wait for memory, not for them (215 us either way).
  p.tail = p.wide || (c.cache.bits != 16 && blocks * sequences >= 8 * splits) ? 4 : 0;
  p.splits = alone || sequences > kMaxScan || (blocks + p.tail) * sequences + 2 * kMaxSplits >= 1ll << 31 ? 0 : (int)splits;      // (a run's end is counted too)
  return p;
}

uint64_t workspace_of(const conqur_tree_call& c, const Plan& p) {
  return (uint64_t)c.cache.heads * p.row_tiles * 2 * p.splits * p.tile_rows * (c.cache.width + 2) * sizeof(float);
}

bool call_fine(const conqur_tree_call* c) {
  if (!c || !cache_fine(c->cache) || !batch_fine(c->batch) || c->tokens >= (1ull << 31)) return false;
  if (c->max_query < 1 || c->max_query > (uint32_t)kMaxQuery || !isfinite(c->scale)) return false;
  if (c->q.heads < 1 || c->q.heads % c->cache.heads || c->q.heads / c->cache.heads > 64 || c->out.heads != c->q.heads) return false;
  return c->max_context < (1ull << 31);
}

bool rows_fine(const conqur_heads& h, uint32_t width, uint64_t tokens, bool output) {
  if (!h.data || reinterpret_cast<uintptr_t>(h.data) % 2) return false;
  if (h.token_stride < 0 || h.token_stride >= kMaxStride || h.head_stride < 0 || h.head_stride >= kMaxStride) return false;
  if (!output) return true;
  const __int128 w = width, ts = h.token_stride, hs = h.head_stride, heads = h.heads, n = tokens;
  if ((heads > 1 && hs < w) || (n > 1 && ts < w)) return false;
  return !(heads > 1 && n > 1 && ts < (heads - 1) * hs + w && hs < (n - 1) * ts + w);
}

template <int BITS, int W>
hipError_t launch(const TreeArgs& a, const Plan& p, hipStream_t s) {
  const dim3 grid((uint32_t)(a.cache.heads * p.row_tiles), p.splits ? p.splits : a.batch.sequences);
  hipError_t e;
  if (p.wide) {
    e = launch_wide(a, p.qt, grid, s);
  } else {
    constexpr int kMostTiles = BITS == 16 ? 1 : 2;
    const bool one_page = a.cache.page_tokens >= (uint32_t)kBlock;
    if (p.qt == 1 && one_page)
      k_tree<BITS, W, 1, true, kMasks><<<grid, 64 * kWaves, 0, s>>>(a);
    else if (p.qt == 1)
      k_tree<BITS, W, 1, false, kMasks><<<grid, 64 * kWaves, 0, s>>>(a);
    else if (one_page)
      k_tree<BITS, W, kMostTiles, true, kMasks><<<grid, 64 * kWaves, 0, s>>>(a);
    else
      k_tree<BITS, W, kMostTiles, false, kMasks><<<grid, 64 * kWaves, 0, s>>>(a);
    e = hipGetLastError();
  }
  return e != hipSuccess || p.splits <= 1 ? e : launch_join(a, p.wide, s);
}

}  // namespace

hipError_t conqur::tree::launch_join(const TreeArgs& a, bool wide, hipStream_t s) {
  return a.cache.width == 128 ? join_pieces<128>(a, wide, s) : join_pieces<64>(a, wide, s);
}

extern "C" uint64_t conqur_tree_attention_workspace(const conqur_tree_call* call) {
  if (!call_fine(call)) return 0;
  return workspace_of(*call, plan_of(*call));
}

extern "C" conqur_status conqur_tree_attention(const conqur_tree_call* c, void* stream) {
  if (!call_fine(c)) return CONQUR_EINVAL;
  if (c->tokens == 0) return CONQUR_OK;
  if (!rows_fine(c->q, c->cache.width, c->tokens, false) || !rows_fine(c->out, c->cache.width, c->tokens, true)) return CONQUR_EINVAL;
  if (reinterpret_cast<uintptr_t>(c->mask) % 8) return CONQUR_EINVAL;
  const Plan p = plan_of(*c);
  const uint64_t need = workspace_of(*c, p);
  if (need && (!c->workspace || reinterpret_cast<uintptr_t>(c->workspace) % 16 || c->workspace_bytes < need)) return CONQUR_EINVAL;
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
  a.mask = c->mask;
  a.tokens = (int64_t)c->tokens;
  a.context = p.context;
  a.splits = p.splits;
  a.min_blocks = p.min_blocks;
  a.tail = p.splits ? p.tail : 0;
  a.max_query = (int)c->max_query;
  a.group = (int)(c->q.heads / c->cache.heads);
  a.tile_rows = p.tile_rows;
  a.row_tiles = p.row_tiles;
  a.part = static_cast<float*>(c->workspace);
  a.part_ml = reinterpret_cast<float2*>(a.part + (uint64_t)c->cache.heads * p.row_tiles * 2 * p.splits * p.tile_rows * c->cache.width);
  a.scale_log2 = c->scale * 1.4426950408889634f;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  hipError_t e;
  if (c->cache.width == 128)
    e = c->cache.bits == 16 ? launch<16, 128>(a, p, s) : c->cache.bits == 8 ? launch<8, 128>(a, p, s) : launch<4, 128>(a, p, s);
  else
    e = c->cache.bits == 16 ? launch<16, 64>(a, p, s) : c->cache.bits == 8 ? launch<8, 64>(a, p, s) : launch<4, 64>(a, p, s);
  return e == hipSuccess ? CONQUR_OK : CONQUR_EHIP;
}
