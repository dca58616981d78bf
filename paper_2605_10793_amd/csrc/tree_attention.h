// What the kernels of the tree attention share: a call's arguments, how the work is cut, the operands' formats.
#pragma once
#include <math.h>

#include <type_traits>
#include <utility>

#include "../../include/conqur.h"
#include "kernels.h"

namespace conqur {

bool cache_fine(const conqur_cache& c);
bool batch_fine(const conqur_batch& b);

namespace tree {

constexpr int kWaves = 4;
constexpr int kBlock = 64;                        // keys a wavefront takes at a time
constexpr int kMaxQuery = 64;
constexpr int kMaxSplits = 256;                   // pieces of a sequence that one workgroup joins
constexpr int kScanChunks = 8;
constexpr int kRun = 16384;                        // keys after which blocks that were put off are made up for
constexpr float kRise = 16.0f;                    // by how much (log2) scores may exceed the maximum they are taken against, before it and all results are raised
constexpr int kSlots = 512;                       // workgroups the device holds: two of 4 wavefronts on each of 256 compute units
constexpr int kMaxScan = 64 * kScanChunks;        // sequences that a workgroup finds its pieces among

struct TreeArgs {
  conqur_cache cache;
  conqur_batch batch;
  const bf16_bits* q;
  bf16_bits* out;
  int64_t q_ts, q_hs, out_ts, out_hs;
  const uint64_t* mask;
  int64_t tokens, context;
  // A cache head's rows are cut into row tiles of tile_rows.  splits = 0: a workgroup for each sequence.  Otherwise the blocks of all sequences,
  // one behind the other, are dealt to `splits` workgroups in equal runs of at least min_blocks, whatever the sequences' lengths; a workgroup
  // has up to two pieces that are not whole sequences, its first and its last, whose results go to its slots 0 and 1:
  float* part;               // [cache head][row tile][workgroup][slot][row][width] sums
  float2* part_ml;           // [cache head][row tile][workgroup][slot][row] maxima, sums of weights
  int splits, min_blocks;
  int tail;                  // blocks that a sequence's end, its new tokens, counts for beside its own
  int max_query, group, tile_rows, row_tiles;
  int q_wide, out_wide;
  float scale_log2;
  // Of a chunk of new tokens (kinds kChunk and kOptions): keys by bounds, a window, a cap in base 2 and 2 / cap in base 2, a bias by distance.
  int chunk, window;
  int looks, workgroups;     // rows that get no result get zeros: how often zero_rows looks at some (0: they stay as they are), workgroups of the launch
  int tile_by_tile;          // of the runs, all of the first row tile come first
  // With no runs, row tiles of all sequences are numbered one behind the other.
  uint32_t tile_inverse;     // 2^32 / tile_rows, rounded up: of rows (fewer than 2^24) it makes tiles
  int row_shift;             // more than kMaxScan sequences: 2^row_shift rows (a tile's at most) to a number
  const int32_t* first;
  const int32_t* last;
  const float* slopes;
  float cap_log2, cap_in;
};

// What a row sees and how: a tree's masks; bounds and windows; those with capped scores or a bias by distance.
enum { kMasks = 0, kChunk = 1, kOptions = 2 };

// The arguments as a kernel reads them, where they lie: each call gives an address that the compiler takes for a new one, so that what a part of a
// kernel needs of them is read there and not kept in (some hundred) registers from the kernel's beginning.
typedef const __attribute__((address_space(4))) TreeArgs* Args;
__device__ __forceinline__ Args kernel_args() {
  Args p = (Args)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return p;
}

typedef const __attribute__((address_space(4))) int32_t* Scalars;      // memory that no kernel writes while this one runs
struct Sequence {
  int64_t first, prefix, length;     // first row of q, committed tokens, tokens in sight
  int count;
};

template <typename P>
__device__ __forceinline__ Sequence sequence_from(Args a, P start, P prefix) {
  Sequence s;
  auto clamp_to = [&](int v) { return v < 0 ? (int64_t)0 : (int64_t)v > a->tokens ? a->tokens : (int64_t)v; };
  s.first = clamp_to(start[0]);
  const int64_t n = clamp_to(start[1]) - s.first;
  s.prefix = prefix[0] < 0 ? 0 : prefix[0];
  s.length = s.prefix + (n < 0 ? 0 : n);
  if (s.length > a->context) s.length = a->context;
  s.count = n < 0 ? 0 : n > a->max_query ? a->max_query : (int)n;
  return s;
}
// b the same for a whole wavefront (what follows from it then stays out of the vector registers), or each lane's own.
__device__ __forceinline__ Sequence sequence_of(Args a, int b) {
  b = __builtin_amdgcn_readfirstlane(b);
  return sequence_from(a, (Scalars)(uintptr_t)(a->batch.start + b), (Scalars)(uintptr_t)(a->batch.prefix + b));
}
__device__ __forceinline__ Sequence sequence_of_lane(Args a, int b) { return sequence_from(a, a->batch.start + b, a->batch.prefix + b); }

// A value that the compiler takes for a new one: what is made of it is made anew, not kept in registers from one use, far off, to the next.
__device__ __forceinline__ int anew(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// The lane, counted anew: threadIdx.x need not be kept for it.
__device__ __forceinline__ int lane_anew() {
  int none = 0;
  asm volatile("" : "+s"(none));
  return (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, (uint32_t)none));
}

// Keys that a row tile which begins at row0 (below the sequence's rows) may see: from 64 times the first block on, up to the end.  In a chunk whose tokens see
// no later ones, the tile's last token bounds it; its first one's window leaves blocks out.
__device__ __forceinline__ int64_t tile_end(Args a, const Sequence& s, int row0) {
  if (!a->chunk || a->last) return s.length;
  const int rows = s.count * a->group, row = row0 + a->tile_rows < rows ? row0 + a->tile_rows - 1 : rows - 1;
  const int64_t end = s.prefix + (uint32_t)row / (uint32_t)a->group + 1;
  return end < s.length ? end : s.length;
}
__device__ __forceinline__ int first_block(Args a, const Sequence& s, int row0) {
  if (!a->chunk || a->window == 0) return 0;
  const int64_t from = s.prefix + (uint32_t)row0 / (uint32_t)a->group + 1 - a->window;
  return from > 0 ? (int)((from < s.length ? from : s.length) / kBlock) : 0;
}
// Blocks of a sequence for a row tile that begins at row0: none if it has no such rows, otherwise one at least (which writes zeros if nothing is seen).
__device__ __forceinline__ int blocks_in(Args a, const Sequence& s, int row0) {
  if (row0 >= s.count * a->group) return 0;
  const int64_t end = tile_end(a, s, row0);
  const int n = (end > kBlock ? (int)((end + kBlock - 1) / kBlock) : 1) - first_block(a, s, row0);
  return (n > 1 ? n : 1) + a->tail;
}

// Keys [x, y) that new token `node` of a chunk sees; (0, 0): none.
__device__ __forceinline__ int2 chunk_keys(Args a, const Sequence& s, int node) {
  const int64_t place = s.prefix + node;
  int64_t lo = 0, hi = place + 1;
  if (a->first) lo = a->first[s.first + node];
  if (a->last) hi = a->last[s.first + node];
  if (lo < 0) lo = 0;
  if (a->window && place - a->window + 1 > lo) lo = place - a->window + 1;
  if (hi > s.length) hi = s.length;
  return lo < hi ? make_int2((int)lo, (int)hi) : make_int2(0, 0);
}
// Bits j of 16: whether lo <= pos + j < hi.
__device__ __forceinline__ uint32_t between(int64_t pos, int2 keys) {
  const int64_t lo = keys.x - pos, hi = keys.y - pos;
  const int from = lo < 0 ? 0 : lo > 16 ? 16 : (int)lo, to = hi < 0 ? 0 : hi > 16 ? 16 : (int)hi;
  return to > from ? ((1u << to) - 1) & ~((1u << from) - 1) : 0;
}
template <typename Op>
__device__ __forceinline__ int wave_reduce_int(int v, Op op) {
  const auto a = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
  const int w = op((int)a[0], (int)a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap((uint32_t)w, (uint32_t)w, false, false);
  const uint32_t x = row16_reduce((uint32_t)op((int)b[0], (int)b[1]), [&](uint32_t x, uint32_t y) { return (uint32_t)op((int)x, (int)y); });
  return __builtin_amdgcn_readfirstlane((int)x);
}
__device__ __forceinline__ int wave_min(int v) { return wave_reduce_int(v, [](int a, int b) { return a < b ? a : b; }); }
__device__ __forceinline__ int wave_max_int(int v) { return wave_reduce_int(v, [](int a, int b) { return a > b ? a : b; }); }
// A score in base 2, capped.
__device__ __forceinline__ float capped(float y, float cap_log2, float cap_in) {
  return fmaf(-2.0f * cap_log2, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(y * cap_in)), cap_log2);
}

// Sum over the lanes up to a lane.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);      // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // lane 15 of rows 0 and 2 to rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);      // lane 31 to rows 2 and 3
  return v;
}

// The blocks of all sequences one behind the other, as one wavefront sees them: lane l holds the ends of sequences l, 64 + l, ...
struct Layout {
  int end[kScanChunks];      // last block + 1 of the lane's sequences
  int all;                   // blocks of all
  int each;                  // of a workgroup
  __device__ __forceinline__ Layout(Args a, int row0, int lane) {
    all = 0;
#pragma unroll
    for (int c = 0; c < kScanChunks; ++c) {
      end[c] = all;
      if (c * 64 < (int)a->batch.sequences) {
        const int b = c * 64 + lane;
        end[c] = all + wave_scan(b < (int)a->batch.sequences ? blocks_in(a, sequence_of_lane(a, b), row0) : 0);
        all = __builtin_amdgcn_readlane(end[c], 63);
      }
    }
    each = (all + a->splits - 1) / a->splits;
    if (each < a->min_blocks) each = a->min_blocks;
  }
  // The sequence that holds block x < all, and where it begins and ends.
  __device__ __forceinline__ void find(Args a, int x, int* b, int* from, int* to) const {
    int before = 0;
#pragma unroll
    for (int c = 0; c < kScanChunks; ++c) {
      if (c * 64 < (int)a->batch.sequences) {
        const int last = __builtin_amdgcn_readlane(end[c], 63);
        if (x >= before && x < last) {
          const int i = __popcll(__ballot(end[c] <= x));
          *b = c * 64 + i;
          *to = __builtin_amdgcn_readlane(end[c], i);
          *from = i ? __builtin_amdgcn_readlane(end[c], i - 1) : before;
        }
        before = last;
      }
    }
  }
  __device__ __forceinline__ void range(int b, int* from, int* to) const {
    int before = 0;
#pragma unroll
    for (int c = 0; c < kScanChunks; ++c) {
      if (b >> 6 == c) {
        *to = __builtin_amdgcn_readlane(end[c], b & 63);
        *from = b & 63 ? __builtin_amdgcn_readlane(end[c], (b & 63) - 1) : before;
      }
      before = __builtin_amdgcn_readlane(end[c], 63);
    }
  }
};

// Where a row's results of a piece are.
__device__ __forceinline__ int64_t part_at(Args a, int head, int row_tile, int slot, int row_in_tile) {
  const int one = a->batch.sequences == 1;          // (which has first pieces only)
  return (((int64_t)head * a->row_tiles + row_tile) * (2 * a->splits >> one) + (slot >> one)) * a->tile_rows + row_in_tile;
}

// Pages of a block's four groups of 16 keys, -1 where there is none; the same for a whole wavefront.
struct Pages {
  int32_t at[4];
  __device__ __forceinline__ bool missing() const { return (at[0] | at[1] | at[2] | at[3]) < 0; }
  __device__ __forceinline__ int32_t pick(int u) const {
    const int32_t a0 = at[0], a1 = at[1], a2 = at[2], a3 = at[3];
    const int32_t lo = u & 1 ? a1 : a0, hi = u & 1 ? a3 : a2;
    return u & 2 ? hi : lo;
  }
};

// The sequence (-1: none) and the row tile of it that is the id-th of all sequences' row tiles, wherever their rows lie, for up to kMaxScan sequences, each of
// which has a tile more where its rows end with one (64 prompts of 512: 371 us, 383 without).  All starts are read at once.  By a whole wavefront; the same for
// all lanes.
__device__ __forceinline__ void place_among(Args a, int id, int* b, int* row_tile) {
  const int lane = (int)threadIdx.x & 63, sequences = (int)a->batch.sequences, tokens = (int)a->tokens, most = a->max_query, group = a->group;
  const uint32_t inverse = a->tile_inverse;
  const int32_t* const start = a->batch.start;
  int x[kScanChunks], y[kScanChunks];
#pragma unroll
  for (int c = 0; c < kScanChunks; ++c)
    if (c * 64 < sequences) {
      x[c] = start[min(c * 64 + lane, sequences)];
      y[c] = start[min(c * 64 + lane + 1, sequences)];
    }
  *b = -1;
  int before = 0;
#pragma unroll
  for (int c = 0; c < kScanChunks; ++c) {
    if (c * 64 < sequences && *b < 0) {
      const int n = min(max(y[c], 0), tokens) - min(max(x[c], 0), tokens);
      const int tiles = c * 64 + lane < sequences ? (int)__umulhi((uint32_t)(min(max(n, 0), most) * group), inverse) + 1 : 0;
      const int end = before + wave_scan(tiles), all = __builtin_amdgcn_readlane(end, 63);
      if (id < all) {
        const int i = __popcll(__ballot(end <= id));
        *b = c * 64 + i;
        *row_tile = id - (i ? __builtin_amdgcn_readlane(end, i - 1) : before);
      }
      before = all;
    }
  }
}

// The head and the row tile of a workgroup, and, if there are no runs, its sequence (-1: none).  A chunk's heads come first, so that with eight of them, or a
// multiple, a cache head's workgroups share an L2 (four chunks of 700 to 1024 tokens over 16 bits: 412 us for 421); with no runs, sequences have the row tiles
// that their own tokens make, for one prompt among many single tokens would give each of them a prompt's (2000 tokens and 255 single ones over 500 to 2500: 352 us
// for 505; 64 prompts of 512: 374 for 452).  Up to kMaxScan sequences' tiles are counted, for their starts may fall (500 of 40 tokens over up to 60: 288 us,
// 283 if numbered by their starts, as those of more are).
template <int KIND>
__device__ __forceinline__ void place_of(Args a, int* head, int* row_tile, int* b, int* run) {
  *run = blockIdx.y;
  if constexpr (KIND == kMasks) {
    *head = blockIdx.x / a->row_tiles, *row_tile = blockIdx.x % a->row_tiles, *b = blockIdx.y;
  } else {
    const int heads = (int)a->cache.heads, id = (int)blockIdx.x / heads;
    *head = (int)blockIdx.x % heads, *row_tile = id, *b = 0;
    if (a->splits) {
      if (a->tile_by_tile) {
        const int at = (int)blockIdx.y * a->row_tiles + id;
        *row_tile = at / a->splits, *run = at % a->splits;
      }
      return;
    }
    if (a->row_tiles == 1) {
      *b = id, *row_tile = 0;
      return;
    }
    if ((int)a->batch.sequences <= kMaxScan) {
      place_among(a, id, b, row_tile);
      return;
    }
    int first, next;
    *b = sequence_of_part(
        id, (int)a->batch.sequences, a->row_shift, a->group,
        [&](int i) {
          const int v = a->batch.start[i];
          return v < 0 ? 0 : v > a->tokens ? (int)a->tokens : v;
        },
        &first, &next);
    *row_tile = id - ((int)(((int64_t)first * a->group) >> a->row_shift) + *b);
    if (*row_tile < 0 || *row_tile >= a->row_tiles) *b = -1;
  }
}

// What a workgroup has to do, piece by piece: blocks [first, last) of sequence b.
struct Pieces {
  int run;                   // number of the workgroup's
  int x, stop;               // in the blocks of all sequences
  int b, first, last, slot;
  bool whole;
  // False: nothing left.  Begins with the workgroup's own run, or, if there are none, its sequence in b.  Called by whole wavefronts, with the same results in all of them.
  __device__ __forceinline__ bool next(Args a, int row0, bool begin) {
    if (a->splits == 0) {
      if (!begin || b < 0) return false;
      first = 0;
      last = blocks_in(a, sequence_of(a, b), row0);
      whole = true;
      return last > 0;
    }
    if (begin) {
      const Layout l(a, row0, lane_anew());
      x = run * l.each;
      stop = l.all - x < l.each ? l.all : x + l.each;
      if (x >= stop) return false;
      int from = 0, to = 0;
      l.find(a, x, &b, &from, &to);
      first = x - from;
      last = (to < stop ? to : stop) - from;
      whole = first == 0 && from + last == to;
      slot = 2 * run;
      x = from + last;
      return true;
    }
    // What follows begins with the next sequence that has blocks.
    if (x >= stop) return false;
    int n = 0;
    while (n == 0) {
      if (++b >= (int)a->batch.sequences) return false;
      n = blocks_in(a, sequence_of(a, b), row0);
    }
    first = 0;
    last = n < stop - x ? n : stop - x;
    whole = last == n;
    slot = 2 * run + 1;
    x += last;
    return true;
  }
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ bf16x8 as_frag(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const u32x4 v = {a, b, c, d};
  return __builtin_bit_cast(bf16x8, v);
}
__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Over the four lanes l, l + 16, l + 32, l + 48 of a column.
template <typename Op>
__device__ __forceinline__ float column_reduce(float v, Op op) {
  const uint32_t u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const uint32_t w = __float_as_uint(op(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const auto b = __builtin_amdgcn_permlane16_swap(w, w, false, false);
  return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float column_sum(float v) { return column_reduce(v, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ float column_max(float v) { return column_reduce(v, [](float a, float b) { return fmaxf(a, b); }); }

// Lane E of every row of 16 to the whole row.
template <int E>
__device__ __forceinline__ float row_bcast(float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x150 + E, 0xf, 0xf, true));
}
template <typename F, int... I>
__device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F&& f) {
  each_of(f, std::make_integer_sequence<int, N>{});
}

// How a cache's format meets the operands.
template <int BITS, int W>
struct Format {
  static constexpr int kRow = BITS == 16 ? 2 * W : W * BITS / 8;    // bytes of a key
  static constexpr int kVRows = BITS == 4 ? W / 2 : W;              // rows of V in a page
  static constexpr int kVSize = BITS == 16 ? 2 : 1;                 // bytes of a token in such a row
  static constexpr int kWords = W * BITS / 128;                     // words of a key in each of the four lanes that share it
  static constexpr int kVTiles = kVRows / 16;                       // tiles of 16 V rows
  static constexpr int kVWords = 4 * kVSize;                        // words of a lane's 16 tokens in a V row
};

// Entry of the row that element j of the contraction's operand i holds in quarter g.
template <int BITS, int W>
__device__ __forceinline__ int entry_of(int i, int g, int j) {
  if constexpr (BITS == 16) return (i * 4 + g) * 8 + j;
  if constexpr (BITS == 8) return W == 128 ? ((i / 2) * 4 + g) * 16 + (i % 2) * 8 + j : g * 16 + i * 8 + j;
  // 4 bits: bytes in the order 0, 2, 1, 3 within a word; first the low halves' operands, then the high halves'
  const int byte = (j & 4) | ((j & 1) << 1) | ((j >> 1) & 1);
  return W == 128 ? (i / 2) * 64 + g * 16 + (i % 2) * 8 + byte : i * 32 + g * 8 + byte;
}

// Bytes 0 and 1 (2 and 3) of a word as bf16 integers.
__device__ __forceinline__ uint32_t bytes_to_bf16(uint32_t x, int hi) {
  const float a = (float)((x >> (hi ? 16 : 0)) & 0xff), b = (float)((x >> (hi ? 24 : 8)) & 0xff);
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302);
}
// 128 + code for the low (shift 0, 8) or high (4, 12) halves of bytes 0 and 2 (0, 4) or 1 and 3 (8, 12).
__device__ __forceinline__ uint32_t nibbles_to_bf16(uint32_t x, int shift) { return ((x >> shift) & 0x000f000fu) | 0x43004300u; }

template <int BITS>
__device__ __forceinline__ constexpr float shifted() { return BITS == 4 ? 128.0f : 0.0f; }      // what an operand holds above the code

// Takes the running maximum m to where the highest of new scores, `top` above it, is (none: -inf): what was and what is new fall by the returned amount.
__device__ __forceinline__ float raise(float& m, float top) {
  const bool unset = m == -INFINITY;
  const float by = unset ? (top == -INFINITY ? 0.0f : top) : fmaxf(top, 0.0f);
  m = unset ? top : m + by;
  return by;
}
// The factor on sums over the scores before that; before the first of them they are 0 and `by` may be anything.
__device__ __forceinline__ float m_factor(float by) { return __builtin_amdgcn_exp2f(-fmaxf(by, 0.0f)); }

// Two halves of a word that hold infinities or NaNs.
__device__ __forceinline__ bool any_nonfinite(uint32_t x) { return (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u; }

// Four neighbouring entries of a row's result, sums o over l.
__device__ __forceinline__ void store_row4(Args a, const Sequence& sq, int head, int row, int entry, f32x4 o, float l) {
  bf16_bits* out = a->out + (sq.first + row / a->group) * a->out_ts + (int64_t)(head * a->group + row % a->group) * a->out_hs + entry;
  const float inv = 1.0f / l;
  const uint32_t x = l == 0.0f ? 0 : f32x2_to_bf16x2(o[0] * inv, o[1] * inv), y = l == 0.0f ? 0 : f32x2_to_bf16x2(o[2] * inv, o[3] * inv);
  if (a->out_wide) {
    *reinterpret_cast<u32x2*>(out) = u32x2{x, y};
  } else {
    out[0] = (bf16_bits)x;
    out[1] = (bf16_bits)(x >> 16);
    out[2] = (bf16_bits)y;
    out[3] = (bf16_bits)(y >> 16);
  }
}

// Zeros to the rows of out that get no result: of no sequence, or beyond max_query of one.  All workgroups' wavefronts in turn look at some rows at a time, a
// lane at each, and write those of no sequence together: 8 rows of up to kMaxScan sequences, which may lie anywhere, if the sequences' own rows are not
// all that there are; 64 of more sequences, which are in the order of their rows.  (By one workgroup of a key head, entry by entry: 64 single tokens over 300 with 4000
// such rows behind them 1221 us, now 30, 22 without them; 16 rows at a time by the first workgroups' wavefronts 39.  512 single tokens without such rows: 148, now 152.)
__host__ __device__ __forceinline__ int rows_of_look(int sequences) { return sequences <= kMaxScan ? 8 : 64; }
__device__ __forceinline__ void zero_rows(Args a) {
  const int lane = (int)threadIdx.x & 63, sequences = (int)a->batch.sequences, tokens = (int)a->tokens, workgroups = a->workgroups, end = a->looks;
  int at = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) * workgroups + (int)blockIdx.x * (a->splits ? a->splits : 1) + (int)blockIdx.y;
  if (at >= end) return;
  const bool anywhere = sequences <= kMaxScan;
  const int each = rows_of_look(sequences);
  int first[kScanChunks], count[kScanChunks], have = 0;
  if (anywhere) {
#pragma unroll
    for (int c = 0; c < kScanChunks; ++c) {
      if (c * 64 < sequences) {
        const int b = c * 64 + lane, x = a->batch.start[min(b, sequences)], y = a->batch.start[min(b + 1, sequences)];
        first[c] = min(max(x, 0), tokens);
        count[c] = min(max(min(max(y, 0), tokens) - first[c], 0), a->max_query);
      }
    }
#pragma unroll
    for (int c = 0; c < kScanChunks; ++c)
      if (c * 64 < sequences) have += count[c];
    if (__builtin_amdgcn_readlane(wave_scan(have), 63) == tokens) return;
  }
  for (; at < end; at += workgroups * kWaves) {
    const int row = at * each + lane;
    bool none = lane < each && row < tokens;
    if (anywhere) {
#pragma unroll
      for (int c = 0; c < kScanChunks; ++c)
        for (int i = 0; i < min(64, sequences - c * 64); ++i)
          none = none && (uint32_t)(row - __builtin_amdgcn_readlane(first[c], i)) >= (uint32_t)__builtin_amdgcn_readlane(count[c], i);
    } else {
      int from = 0;                        // the last sequence that begins at the row or before it
      for (int n = sequences; n > 1;) {
        const int half = n / 2;
        if (a->batch.start[from + half] <= row) from += half;
        n -= half;
      }
      const Sequence s = sequence_of_lane(a, from);
      none = none && (uint32_t)(row - (int)s.first) >= (uint32_t)s.count;
    }
    const int width = (int)a->cache.width, shift = 31 - __builtin_clz(width), entries = (int)a->cache.heads * a->group * width;
    for (uint64_t which = __ballot(none); which; which &= which - 1) {
      bf16_bits* const out = a->out + (int64_t)(at * each + __builtin_ctzll(which)) * a->out_ts;
      for (int x = lane * 4; x < entries; x += 256) {
        bf16_bits* const to = out + (int64_t)(x >> shift) * a->out_hs + (x & (width - 1));
        if (a->out_wide) {
          *reinterpret_cast<u32x2*>(to) = u32x2{0, 0};
        } else {
          to[0] = to[1] = to[2] = to[3] = 0;
        }
      }
    }
  }
}

// Rows of more than some tens (tree_attention_wide.hip): 64 qt rows a workgroup.
hipError_t launch_wide(const TreeArgs& a, int qt, dim3 grid, hipStream_t s);
// A chunk's (chunk_attention.hip, chunk_attention_wide.hip).
hipError_t launch_join(const TreeArgs& a, bool wide, hipStream_t s);
hipError_t launch_chunk_few(const TreeArgs& a, int qt, dim3 grid, hipStream_t s);
hipError_t launch_chunk_wide(const TreeArgs& a, int qt, dim3 grid, hipStream_t s);

}  // namespace tree
}  // namespace conqur
