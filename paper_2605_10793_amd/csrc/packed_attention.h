// What the kernels of attention over packed sequences share: arguments, how the work is cut, which keys a row sees, tiles of rows in LDS.
#pragma once
#include <limits.h>
#include <math.h>

#include <type_traits>
#include <utility>

#include "../../include/conqur.h"
#include "kernels.h"

namespace conqur {
namespace packed {

constexpr int kWaves = 4;
constexpr int kTile = 64;                         // keys, or rows, that lie in LDS at a time
constexpr int kRows = 32 * kWaves;                // rows of a workgroup: query heads of a key head, token by token
constexpr float kRise = 16.0f;                    // by how much (log2) scores may exceed the maximum they are taken against, before it and all results are raised
enum { kBiased = 1, kCapped = 2 };                // OPTIONS of the kernels: a bias by distance, capped scores; both (of the gradients: kCapped, too)
constexpr float kLog2e = 1.4426950408889634f;

struct Rows {
  bf16_bits* data;
  int64_t ts, hs;            // elements
};

struct PackedArgs {
  Rows q, k, v, out;
  Rows q_grad, k_grad, v_grad, out_grad;
  float* lse;                // [token][query head], natural logarithms; may be null
  const int32_t* start;
  const int32_t* first;      // of each token; may be null
  const int32_t* last;
  const float* slopes;       // of each query head; may be null
  int64_t tokens;
  int sequences, heads, group, width, window;      // heads: of keys; window 0: none
  int rest;                  // rows of no sequence are written, too: zeros
  float scale, scale_log2, cap_log2, cap_in;       // cap_log2 = cap log2 e (0: none), cap_in = 2 log2 e scale / cap
  // Of the backward pass.  Rows are numbered token * group + query head of the key head.
  float2* stat;              // [key head][row] logarithm (base 2) of the row's sum (+inf: there is none), sum over its gradient times its result; with a cap or
                             // slopes four floats: the row's slope (base 2) and token behind them
  int2* seen;                // [row] first key and last + 1
  int4* span;                // [32 rows of an item] lowest first, highest last, highest first, lowest last (a row that sees nothing: highest first is INT_MAX)
  float* part;               // [part of the rows][64 keys][key head][32 of them][dk, dv]: sums over the part, as registers hold them
  int parts;                 // in which the rows that see 64 keys are taken
  // Of keys that several workgroups share (splits > 1): what each made of its own, as registers hold it, and four numbers a row.
  float* shared;             // [split][128 rows][key head][wavefront] ...
  float4* shared_row;        // [split][128 rows][key head][row]
  int splits;
};

// The arguments as a kernel reads them, where they lie: what a part of a kernel needs of them is read there and not kept in registers.
typedef const __attribute__((address_space(4))) PackedArgs* Args;
__device__ __forceinline__ Args kernel_args() {
  Args p = (Args)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return p;
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// Sequences are numbered from 1 on; 0 is the rows before the first and `sequences` + 1 those behind the last.
__device__ __forceinline__ int edge_of(Args a, int i) {
  if (i <= 0) return 0;
  const int64_t tokens = a->tokens;
  if (i > a->sequences + 1) return (int)tokens;
  const int v = a->start[i - 1];
  return v < 0 ? 0 : v > tokens ? (int)tokens : v;
}

struct Item {
  int first, count;      // rows of the call that are the sequence's tokens
  int part, parts;
  int number;            // of the sequence
  int base;              // number of its first part
  bool rest;             // of no sequence
  __device__ __forceinline__ bool find(Args a, int id, int shift, int of) {
    int next;
    number = sequence_of_part(id, a->sequences + 2, shift, of, [&](int i) { return edge_of(a, i); }, &first, &next);
    count = next - first;
    if (count < 0) count = 0;
    rest = number == 0 || number == a->sequences + 1;
    base = (int)(((int64_t)first * of) >> shift) + number;
    parts = (int)(((int64_t)count * of + (1 << shift) - 1) >> shift);
    part = id - base;
    return part >= 0 && part < parts && !(rest && !a->rest);
  }
};

// Keys [lo, hi) that token p of a sequence sees.
__device__ __forceinline__ int2 keys_of(Args a, const Item& s, int p) {
  int lo = 0, hi = p + 1;
  if (a->first) lo = a->first[s.first + p];
  if (a->last) hi = a->last[s.first + p];
  if (lo < 0) lo = 0;
  if (a->window && p - a->window + 1 > lo) lo = p - a->window + 1;
  if (hi > s.count) hi = s.count;
  if (s.rest) hi = 0;
  return hi > lo ? make_int2(lo, hi) : make_int2(0, 0);
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

// Over the two lanes that share a column of a 32x32 product.
template <typename Op>
__device__ __forceinline__ float halves(float v, Op op) {
  const uint32_t u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return op(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ bf16x8 frag_of(uint32_t a, uint32_t b, uint32_t c, uint32_t d) { return __builtin_bit_cast(bf16x8, u32x4{a, b, c, d}); }
// Row (of a product's result) that register r of a lane in half h holds.
__device__ __forceinline__ constexpr int row_of(int r, int h) { return 8 * (r / 4) + 4 * h + r % 4; }

template <typename F, int... I>
__device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F&& f) {
  each_of(f, std::make_integer_sequence<int, N>{});
}

// The lane, counted anew: what is made of it is made where it is used, not kept in registers from one use, far off, to the next.
__device__ __forceinline__ int lane_anew() {
  int none = 0;
  asm volatile("" : "+s"(none));
  return (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, (uint32_t)none));
}

// A value that the compiler takes for a new one: constants on top of it become an instruction's offset.
__device__ __forceinline__ uint32_t anew(uint32_t v) {
  asm volatile("" : "+v"(v));
  return v;
}

// 64 rows of KS * 16 entries in LDS, rows of kPitch bytes.  Chunk c (16 bytes) of a row lies at c ^ f(row): f takes 16 neighbouring rows (8 of pairs of rows
// of 128 bytes) to different places, for operands whose lanes read a chunk of a row each, and four neighbouring rows to different quarters, for those
// that are turned round on the way (ds_read_b64_tr_b16: 16 lanes read 4 rows of 16 entries and receive 4 rows' values of one entry each).
template <int KS>
struct Tile {
  static constexpr int kPitch = KS <= 4 ? 128 : 256;
  static constexpr int kChunks = kPitch / 16;
  static constexpr int kRowsAt = 64 / kChunks;             // rows that a wavefront fetches with one load
  static constexpr int kLoads = kTile / kRowsAt / kWaves;
  static constexpr int kBytes = kTile * kPitch;
  static constexpr int kTiles = (KS + 1) / 2;              // 32 entries each
  static __device__ __forceinline__ int f(int row) {
    return kChunks == 16 ? ((row & 3) << 2 | ((row >> 2) & 3)) : (((row >> 1) & 1) << 2 | ((row >> 2) & 3));
  }
  // Operands from LDS.  A lane's places in a tile that lies at a multiple of 256 bytes are made once; more rows or tiles behind it are a constant (BEHIND).
  // Of a lane: row (lane & 31), entries 16 s + 8 h to 16 s + 8 h + 7.
  static __device__ __forceinline__ uint32_t row_at(int lane) { return (lane & 31) * kPitch + ((((lane >> 5) ^ f(lane & 31))) << 4); }
  struct RowsAt {
    uint32_t at[KS];
    __device__ __forceinline__ explicit RowsAt(uint32_t x) {
#pragma unroll
      for (int s = 0; s < KS; ++s) at[s] = anew(x ^ (uint32_t)(s << 5));
    }
    template <int BEHIND>
    __device__ __forceinline__ bf16x8 get(int s) const { return *(const __attribute__((address_space(3))) bf16x8*)(uintptr_t)(at[s] + BEHIND); }
  };
  // Turned round: lane's entry 32 t + (lane & 31), rows {4 h .. 4 h + 3, 8 + 4 h .. 8 + 4 h + 3}.
  static __device__ __forceinline__ uint32_t turned_at(int lane) {
    const int l = lane & 15, half = lane >> 5, part = (lane >> 4) & 1, row = 4 * half + (l >> 2);
    return row * kPitch + (((2 * part + ((l & 3) >> 1)) ^ f(row)) << 4) + (l & 1) * 8;
  }
  struct TurnedAt {
    uint32_t at[2 * kTiles];
    __device__ __forceinline__ explicit TurnedAt(uint32_t x) {
#pragma unroll
      for (int t = 0; t < 2 * kTiles; ++t) at[t] = anew(x ^ (uint32_t)(t << 5));
    }
    template <int BEHIND>
    __device__ __forceinline__ bf16x8 get(int t) const {
      typedef __attribute__((address_space(3))) s16x4* P;
      const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)(at[2 * t] + BEHIND));
      const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)(at[2 * t + 1] + BEHIND + 8 * kPitch));
      const u32x2 p = __builtin_bit_cast(u32x2, a), q = __builtin_bit_cast(u32x2, b);
      return frag_of(p[0], p[1], q[0], q[1]);
    }
  };
};

// N products whose operands come from LDS: RING of them are on their way ahead of the products that take them, and nothing but arithmetic passes from one to
// the next (the compiler would hold more of them than there are registers).  load(i), use(i, operand): i as a constant.
constexpr int kArithmetic = 0x6;
template <int FROM, int TO, typename F>
__device__ __forceinline__ void each_from(F&& f) {
  each<TO - FROM>([&](auto i) { f(std::integral_constant<int, FROM + decltype(i)::value>{}); });
}
template <int N, int RING = 4, typename Load, typename Use>
__device__ __forceinline__ void in_turn(Load load, Use use) {
  decltype(load(std::integral_constant<int, 0>{})) ring[RING];
  each<(N < RING ? N : RING)>([&](auto i) { ring[decltype(i)::value] = load(i); });
  each<N>([&](auto i) {
    constexpr int I = decltype(i)::value;
    use(i, ring[I % RING]);
    if constexpr (I + RING < N) ring[I % RING] = load(std::integral_constant<int, I + RING>{});
    __builtin_amdgcn_sched_barrier(kArithmetic);
  });
}

__device__ __forceinline__ uint32_t lds_of(const void* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) unsigned char*)p; }

// 16 bytes a lane from memory to LDS, 64 lanes side by side: what lies `lane_offset` (each lane's) and `offset` behind `from`.  In assembly, because the
// compiler lets reads that turn rows round wait for all that is on its way to LDS, wherever it goes; wait_loads() and a barrier say when it is there.
__device__ __forceinline__ void send16(u32x4 from, uint32_t lds, int lane_offset, int offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               :
               : "s"(lds), "v"(lane_offset), "s"(from), "s"(offset)
               : "memory", "m0");
}
__device__ __forceinline__ u32x4 memory_at(const void* p) {
  const uint64_t x = (uint64_t)(uintptr_t)p;
  return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)x), (uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32) & 0xffff), 0x7fffffffu, 0x00020000u};
}

// Sends for ROWS rows of one head to a tile, from `rows` on; rows behind `count` are the last one again, as are chunks behind the width.
template <int KS, int ROWS = kTile>
__device__ __forceinline__ void send_tile(const bf16_bits* rows, int stride, int count, uint32_t lds, int wave) {
  using T = Tile<KS>;
  constexpr int kLoads = ROWS / T::kRowsAt / kWaves;
  static_assert(kLoads > 0, "");
  const u32x4 from = memory_at(rows);
  const int lane = lane_anew();
  const int in = lane / T::kChunks, c0 = (lane % T::kChunks) ^ T::f(wave * kLoads * T::kRowsAt + in);
  auto chunk = [&](int i) {
    int c = c0 ^ T::f(i * T::kRowsAt);
    if (KS * 2 < T::kChunks) c = c < KS * 2 ? c : KS * 2 - 1;
    return c * 16;
  };
  static_assert(kLoads * T::kRowsAt <= 16, "f of a sum is the exclusive or of its parts'");
  if (count >= ROWS) {
    const int at = in * stride;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r0 = (wave * kLoads + i) * T::kRowsAt;
      send16(from, lds + r0 * T::kPitch, at + chunk(i), r0 * stride);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r0 = (wave * kLoads + i) * T::kRowsAt, r = r0 + in < count ? r0 + in : count - 1;
      send16(from, lds + r0 * T::kPitch, r * stride + chunk(i), 0);
    }
  }
}

template <int N>
__device__ __forceinline__ void wait_loads() {          // until no more than the N last loads of the wavefront are under way
  static_assert(N < 16, "");
  __builtin_amdgcn_s_waitcnt(0x0F70 | N);
  asm volatile("" ::: "memory");
}
// A barrier that leaves loads under way; LDS accesses before it are done.
__device__ __forceinline__ void pipeline_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Operands of 32 rows, straight from memory: lane's row, entries 16 s + 8 h on.
template <int KS>
__device__ __forceinline__ void load_rows(bf16x8 (&f)[KS], const bf16_bits* row, int h) {
#pragma unroll
  for (int s = 0; s < KS; ++s) f[s] = *reinterpret_cast<const bf16x8*>(row + 16 * s + 8 * h);
}

// Entries 0, 1 or 2 of what a word holds that is neither finite nor ...: words with those halves that are infinities or NaNs taken out.
__device__ __forceinline__ uint32_t finite_only(uint32_t x) {
  if ((x & 0x7f80u) == 0x7f80u) x &= 0xffff0000u;
  if ((x & 0x7f800000u) == 0x7f800000u) x &= 0x0000ffffu;
  return x;
}
__device__ __forceinline__ bf16x8 finite_only(bf16x8 f) {
  u32x4 x = __builtin_bit_cast(u32x4, f);
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = finite_only(x[j]);
  return __builtin_bit_cast(bf16x8, x);
}
// A wavefront's EACH rows of a tile: infinities and NaNs become zeros.  64 / EACH neighbouring lanes share a row; they receive whether it had any.
template <int KS, int EACH>
__device__ __forceinline__ bool clear_nonfinite(uint32_t tile, int wave, int lane) {
  using T = Tile<KS>;
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  typedef __attribute__((address_space(3))) u32x4* P;
  constexpr int kLanes = 64 / EACH, kEach = T::kPitch / kLanes / 16;
  const uint32_t at = tile + (wave * EACH + lane / kLanes) * T::kPitch + lane % kLanes * (T::kPitch / kLanes);
  u16x2 most = {0, 0};
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const u32x4 x = *(P)(uintptr_t)(at + 16 * i);
#pragma unroll
    for (int j = 0; j < 4; ++j) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, x[j] & 0x7fff7fffu));
  }
  const uint64_t found = __ballot(most[0] >= 0x7f80 || most[1] >= 0x7f80);
  if (found) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      u32x4 x = *(P)(uintptr_t)(at + 16 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = finite_only(x[j]);
      *(P)(uintptr_t)(at + 16 * i) = x;
    }
  }
  return (found >> (lane / kLanes * kLanes)) & ((1 << kLanes) - 1);
}

// The largest of 16 and one more, whatever their sign; a NaN loses.  (For fmaxf of fmaxf the compiler first makes each argument canonical, an instruction more for
// each; between two pieces of assembly it leaves a pause.)
__device__ __forceinline__ float max17(const float (&s)[16], float more) {
  float x;
  asm("v_max3_f32 %0, %1, %2, %3\n\tv_max3_f32 %0, %0, %4, %5\n\tv_max3_f32 %0, %0, %6, %7\n\tv_max3_f32 %0, %0, %8, %9\n\t"
      "v_max3_f32 %0, %0, %10, %11\n\tv_max3_f32 %0, %0, %12, %13\n\tv_max3_f32 %0, %0, %14, %15\n\tv_max3_f32 %0, %0, %16, %17"
      : "=&v"(x)
      : "v"(s[0]), "v"(s[1]), "v"(s[2]), "v"(s[3]), "v"(s[4]), "v"(s[5]), "v"(s[6]), "v"(s[7]), "v"(s[8]), "v"(s[9]), "v"(s[10]), "v"(s[11]), "v"(s[12]), "v"(s[13]),
        "v"(s[14]), "v"(s[15]), "v"(more));
  return x;
}

// A score in base 2 from a product q k, less the bias and `base`; `r` receives 1 / (1 + e^(2 u / cap)), from which 1 - tanh^2 = 4 r (1 - r) follows.
__device__ __forceinline__ float capped(float dot, float cap_log2, float cap_in, float base, float* r) {
  *r = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(dot * cap_in));
  return fmaf(-2.0f * cap_log2, *r, cap_log2 - base);
}

// The part [*begin, *end) of a workgroup's keys, `tile` at a time, that is workgroup blockIdx.y's of gridDim.y.
__device__ __forceinline__ void share_keys(int* begin, int* end, int tile) {
  if (gridDim.y == 1 || *begin >= *end) return;
  const int tiles = (*end - *begin + tile - 1) / tile, per = (tiles + (int)gridDim.y - 1) / (int)gridDim.y;
  *begin += (int)blockIdx.y * per * tile;
  *end = min(*end, *begin + per * tile);
}
// Where a wavefront's registers go: N float4 a lane.
template <int N>
__device__ __forceinline__ f32x4* shared_of(Args a, int split, int wave) {
  return reinterpret_cast<f32x4*>(a->shared) + (((int64_t)split * gridDim.x + blockIdx.x) * kWaves + wave) * (N * 64) + ((int)threadIdx.x & 63);
}
__device__ __forceinline__ float4* shared_row_of(Args a, int split, int row) {
  return a->shared_row + ((int64_t)split * gridDim.x + blockIdx.x) * kRows + row;
}

// Four neighbouring entries of a row's result.
__device__ __forceinline__ void store4(bf16_bits* to, f32x4 x, bool wide) {
  const uint32_t a = f32x2_to_bf16x2(x[0], x[1]), b = f32x2_to_bf16x2(x[2], x[3]);
  if (wide) {
    *reinterpret_cast<u32x2*>(to) = u32x2{a, b};
  } else {
    to[0] = (bf16_bits)a;
    to[1] = (bf16_bits)(a >> 16);
    to[2] = (bf16_bits)b;
    to[3] = (bf16_bits)(b >> 16);
  }
}
__device__ __forceinline__ bool wide8(const bf16_bits* p, int64_t ts, int64_t hs) {
  return ((uintptr_t)p & 7) == 0 && (ts & 3) == 0 && (hs & 3) == 0;
}

// A row's entries as a lane holds them, times `by`; `to`: the lane's first.
template <int KS>
__device__ __forceinline__ void store_row(bf16_bits* to, const f32x16 (&x)[(KS + 1) / 2], float by, bool wide) {
  auto all = [&](bool w) {
#pragma unroll
    for (int t = 0; t < (KS + 1) / 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (32 * t + 8 * r < KS * 16) store4(to + 32 * t + 8 * r, f32x4{x[t][4 * r], x[t][4 * r + 1], x[t][4 * r + 2], x[t][4 * r + 3]} * by, w);
  };
  if (wide)
    all(true);
  else
    all(false);
}

// The 32 entries t of a row.
template <int KS>
__device__ __forceinline__ void store_tile(bf16_bits* to, int t, const f32x16& x, float by, bool wide) {
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (32 * t + 8 * r < KS * 16) store4(to + 32 * t + 8 * r, f32x4{x[4 * r], x[4 * r + 1], x[4 * r + 2], x[4 * r + 3]} * by, wide);
}

// Items of the rows, and of the keys, of a call.
static inline int64_t row_items(const PackedArgs& a) { return a.tokens * a.group / kRows + a.sequences + 2; }
static inline int64_t key_items(const PackedArgs& a) { return a.tokens / kTile + a.sequences + 2; }

hipError_t launch_forward(const PackedArgs& a, hipStream_t s);
hipError_t launch_backward(const PackedArgs& a, hipStream_t s);

}  // namespace packed
}  // namespace conqur
