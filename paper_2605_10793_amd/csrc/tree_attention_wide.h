// The kernel of many rows (tree_attention_wide.hip says how it works and what it measured).
#pragma once
#include "tree_attention.h"

namespace conqur {
namespace tree {

namespace {

constexpr int kRing = 4;                   // operands on their way from LDS ahead of the products that take them (8 sequences of 16384 tokens: 181 us for 190 as the compiler has it)
constexpr int kArithmetic = 0x6;           // what may pass the fences between products: vector and scalar arithmetic
constexpr float kTiny = 1e-30f;            // steps below it are not divided by
constexpr int kDepth = 4;                  // blocks whose steps and zeros are in LDS

template <int BITS, int W>
struct Wide {
  using F = Format<BITS, W>;
  // 64 keys are taken in units of 16 bytes, kKParts a key; their values in units of kVKeys tokens, kVParts a V row.
  static constexpr int kKParts = F::kRow / 16;
  static constexpr int kVKeys = 16 / F::kVSize;
  static constexpr int kVParts = kBlock / kVKeys;
  static constexpr int kKAll = kBlock * kKParts, kVAll = F::kVRows * kVParts;
  // A thread's share; where there are only 128 of each, two wavefronts take the keys and two the values.
  static constexpr bool kApart = kKAll < 256;
  static constexpr int kUnits = kApart ? 1 : kKAll / 256;
  static_assert(kKAll == kVAll && (kApart ? kKAll == 128 : kKAll % 256 == 0), "units");
  static constexpr int kChunks = W / 8;                                  // 16-byte chunks of a key in LDS
  static constexpr int kTile = kBlock * W * 2;                           // bytes of 64 keys, and of their values, as bf16
  static constexpr int kRaw = 2 * kKAll * 16 + 16 * kBlock;              // bytes of 64 keys and values as the cache has them, and of their pairs
  static constexpr int kPairs = 6 * kBlock;                              // K's steps, zeros and rests, V's steps, zeros and rests
  // LDS: bf16 keys and values, two blocks of them or (codes) one, and two blocks of codes on their way; pairs; flags, blocks put off.
  static constexpr int kPairAt = BITS == 16 ? 4 * kTile : 2 * kTile + 2 * kRaw;
  static constexpr int kFlagAt = kPairAt + (BITS == 16 ? 0 : kDepth * kPairs * 4);
  static constexpr int kShared = kFlagAt + 2 * kDepth * 4 + kRun / kBlock * 2;
};

// 16 bytes a lane from memory to LDS, 64 lanes side by side, `first` being lane 0's place; in the second form `from` is the same for all lanes.
__device__ __forceinline__ void to_lds(const unsigned char* from, unsigned char* first) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)first, 16, 0, 0);
}
__device__ __forceinline__ void offset_to_lds(const unsigned char* from, int offset, unsigned char* first) {
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(from), 0, 0x7fffffff, 0x00020000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)first, 16, offset, 0, 0, 0);
}

template <int N>
__device__ __forceinline__ void wait_loads() {          // until no more than the N last loads of the wavefront are under way
  static_assert(N < 16, "");
  __builtin_amdgcn_s_waitcnt(0x0F70 | N);
  asm volatile("" ::: "memory");
}
// A barrier that leaves loads under way, which __syncthreads would wait for; LDS accesses before it are done.
__device__ __forceinline__ void pipeline_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

__device__ __forceinline__ u32x4 join(u32x2 a, u32x2 b) { return u32x4{a[0], a[1], b[0], b[1]}; }

// 8 bytes of LDS, and the 8 that lie 512 behind (in assembly: for a plain read the compiler would first wait for all that is on its way to LDS).
__device__ __forceinline__ u32x4 read_two(const unsigned char* p) {
  const uint32_t at = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) unsigned char*)p;
  u32x2 a, b;
  asm volatile("ds_read_b64 %0, %2\n\tds_read_b64 %1, %2 offset:512\n\ts_waitcnt lgkmcnt(0)" : "=&v"(a), "=&v"(b) : "v"(at) : "memory");
  return join(a, b);
}

// Byte of chunk c of key row (t, i) and of V row d; 256 (128) bytes of neighbouring rows lie on different banks.
template <int W>
__device__ __forceinline__ int key_at(int t, int i, int c) {
  return (t * 16 + i) * W * 2 + ((W == 128 ? c ^ i : c ^ (i >> 1)) << 4);
}
__device__ __forceinline__ int value_at(int d, int c) { return d * kBlock * 2 + ((c ^ ((d >> 1) & 7)) << 4); }

// Four codes (bytes of x) less z, as bf16.
__device__ __forceinline__ u32x2 less_zero(uint32_t x, float z) {
  return u32x2{f32x2_to_bf16x2((float)(x & 0xff) - z, (float)((x >> 8) & 0xff) - z), f32x2_to_bf16x2((float)((x >> 16) & 0xff) - z, (float)(x >> 24) - z)};
}
__device__ __forceinline__ u32x2 less_zeros(uint32_t x, f32x4 z) {
  return u32x2{f32x2_to_bf16x2((float)(x & 0xff) - z[0], (float)((x >> 8) & 0xff) - z[1]),
               f32x2_to_bf16x2((float)((x >> 16) & 0xff) - z[2], (float)(x >> 24) - z[3])};
}

template <int BITS, int W, int QT, int KIND>
__global__ void __launch_bounds__(64 * kWaves, 2) k_tree_wide(const TreeArgs) {
  Args a = kernel_args();
  using F = Format<BITS, W>;
  using D = Wide<BITS, W>;
  constexpr int kOps = W / 32, kTiles = W / 16;
  constexpr bool kCodes = BITS != 16;
  extern __shared__ __attribute__((aligned(16))) unsigned char shared[];
  auto s_k = [&](int block) { return shared + (kCodes ? 0 : (block & 1) * 2 * D::kTile); };
  auto s_v = [&](int block) { return s_k(block) + D::kTile; };
  auto s_raw = [&](int block) { return shared + 2 * D::kTile + (block & 1) * D::kRaw; };
  auto s_pair = [&](int block) { return reinterpret_cast<float*>(shared + D::kPairAt) + (block & (kDepth - 1)) * D::kPairs; };
  int* const s_flag = reinterpret_cast<int*>(shared + D::kFlagAt);          // of a pair's slot: K's tokens, V's tokens have rests
  uint16_t* const s_later = reinterpret_cast<uint16_t*>(s_flag + 2 * kDepth);

  int head, row_tile;
  Pieces piece;
  place_of<KIND>(a, &head, &row_tile, &piece.b, &piece.run);
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int row0 = (row_tile * kWaves + wave) * 16 * QT;
  if constexpr (KIND != kMasks) {
    if (a->looks) zero_rows(a);
  }
  for (bool first = true; piece.next(a, row_tile * 64 * QT, first); first = false) {
  int tid, lane, col, g;
  auto number = [&] {
    a = kernel_args();
    lane = lane_anew();
    tid = wave * 64 + lane;
    col = lane & 15;
    g = lane >> 4;
  };
  number();
  const int b = piece.b;
  const Sequence sq = sequence_of(a, b);
  const int rows = sq.count * a->group;
  const bool idle = row0 >= rows;        // still loads and meets the barriers
  const int tile_row0 = row_tile * 64 * QT;
  const int64_t base_key = KIND == kMasks ? 0 : (int64_t)first_block(a, sq, tile_row0) * kBlock, limit = KIND == kMasks ? sq.length : tile_end(a, sq, tile_row0);
  const int64_t piece_to = base_key + (int64_t)piece.last * kBlock;
  int64_t piece_from = base_key + (int64_t)piece.first * kBlock, piece_end = piece_to < limit ? piece_to : limit;
  // A chunk: the keys of each row, and those that all rows of the workgroup see.  A row that sees nothing is taken to see all, and gets zeros at the end.
  int low_all = 0, high_all = 0, low_any = 0, high_any = 0;
  float slope[QT], place[QT];
  if constexpr (KIND != kMasks) {
    high_all = low_any = INT_MAX;
#pragma unroll
    for (int x = 0; x < QT; ++x) {
      const int other = tile_row0 + x * 64 + lane;
      const int2 k = chunk_keys(a, sq, (uint32_t)(other < rows ? other : 0) / (uint32_t)a->group);
      const bool any = other < rows && k.x < k.y;
      low_all = max(low_all, wave_max_int(any ? k.x : 0));
      high_all = min(high_all, wave_min(any ? k.y : INT_MAX));
      low_any = min(low_any, wave_min(any ? k.x : INT_MAX));
      high_any = max(high_any, wave_max_int(any ? k.y : 0));
      if constexpr (KIND == kOptions) {
        const int row = row0 + x * 16 + col, node = (uint32_t)(row < rows ? row : 0) / (uint32_t)a->group;
        slope[x] = a->slopes ? a->slopes[head * a->group + (row < rows ? row : 0) - node * a->group] * 1.4426950408889634f : 0.0f;
        place[x] = (float)node - 16.0f * g;      // less the block's first key and the committed tokens' number
      }
    }
  }

  if constexpr (KIND != kMasks) {          // what no row of the workgroup sees is left out
    if (high_any < piece_end) piece_end = high_any;
    if (low_any / kBlock * kBlock > piece_from) piece_from = low_any / kBlock * kBlock;
  }

  bf16x8 qf[QT][kOps];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int row = row0 + t * 16 + col;
    const bool here = row < rows;
    const bf16_bits* p = a->q + (sq.first + (here ? row / a->group : 0)) * a->q_ts + (int64_t)(head * a->group + (here ? row % a->group : 0)) * a->q_hs;
#pragma unroll
    for (int i = 0; i < kOps; ++i) {
      const int base = (i * 4 + g) * 8;
      u32x4 x = {0, 0, 0, 0};
      if (here) {
        if (a->q_wide) {
          x = *reinterpret_cast<const u32x4*>(p + base);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] = p[base + 2 * j] | (uint32_t)p[base + 2 * j + 1] << 16;
        }
      }
      if (a->scale_log2 < 0.0f) x ^= 0x80008000u;          // the maxima below are taken before the scale
      qf[t][i] = __builtin_bit_cast(bf16x8, x);
    }
  }
  const float scale = fabsf(a->scale_log2), cap = KIND == kOptions ? a->cap_log2 : 0.0f, cap_in = KIND == kOptions ? a->cap_in : 0.0f;
  const bf16x8 ones = as_frag(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);      // a row of the sums of the weights as they are rounded

  // m is what scores are taken against: the running maximum, or up to kRise less, since every rise multiplies all results; -inf before the first
  // token is seen.
  f32x4 o[QT][kTiles], l_acc[kCodes ? 1 : QT];
  float m[QT], l_run[kCodes ? QT : 1];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
#pragma unroll
    for (int d = 0; d < kTiles; ++d) o[t][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (kCodes)
      l_run[t] = 0.0f;
    else
      l_acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    m[t] = -INFINITY;
  }

  const int page_tokens = (int)a->cache.page_tokens;
  const int page_shift = 31 - __builtin_clz(page_tokens);
  // (read by the scalar unit: a vector load would be waited for together with the keys that are under way)
  const Scalars table = (Scalars)(uintptr_t)(a->batch.table + (int64_t)b * a->batch.table_stride);
  const int64_t heads = a->cache.heads;
  const uint32_t pages = (uint32_t)a->cache.pages;
  const float* const k_scale = a->cache.k_scale;
  const float* const v_scale = a->cache.v_scale;
  const unsigned char* kp = static_cast<const unsigned char*>(a->cache.k);
  const unsigned char* vp = static_cast<const unsigned char*>(a->cache.v);

  int64_t end = piece_end;               // of the run that is worked on
  auto pages_of = [&](int64_t kb) {
    Pages p;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t pos = kb + 16 * u;
      int32_t x = -1;
      if (pos < end) x = table[pos >> page_shift];
      p.at[u] = x >= 0 && (uint32_t)x < pages ? x : -1;
    }
    return p;
  };

  const int64_t k_page = heads * page_tokens * F::kRow, v_page = heads * F::kVRows * page_tokens * F::kVSize;
  const int64_t k_head = (int64_t)head * page_tokens * F::kRow, v_head = (int64_t)head * F::kVRows * page_tokens * F::kVSize;
  const bool one_page = page_tokens >= kBlock;      // a block lies in one page: its address is the same for all threads but for an offset
  auto page_or_0 = [](int32_t p) { return (int64_t)(p < 0 ? 0 : p); };
  // Bytes at to at + 16 of key `key` of the block from kb on, and of tokens key to key + kVKeys - 1 of V row d.
  auto key_source = [&](int64_t kb, const Pages& p, int key, int at) {
    return kp + page_or_0(p.pick(key >> 4)) * k_page + k_head + ((kb + key) & (page_tokens - 1)) * F::kRow + at;
  };
  auto value_source = [&](int64_t kb, const Pages& p, int d, int key) {
    return vp + page_or_0(p.pick(key >> 4)) * v_page + v_head + ((kb + key) & (page_tokens - 1)) * F::kVSize + d * page_tokens * F::kVSize;
  };
  // Runs over the thread's units: keys(unit, u), values(unit, u).
  auto units = [&](auto keys, auto values) {
    const int first = wave * 64 + lane_anew();         // (what a unit's place gives is made here, not kept in registers)
    if constexpr (D::kApart) {
      if (wave < 2)
        keys(first, 0);
      else
        values(first - 128, 0);
    } else {
#pragma unroll
      for (int u = 0; u < D::kUnits; ++u) keys(first + 256 * u, u);
#pragma unroll
      for (int u = 0; u < D::kUnits; ++u) values(first + 256 * u, u);
    }
  };
  // Sends for a block: codes as they are; bf16 values to where they will be read, so that what lies in a lane's place decides which it fetches.
  auto send = [&](int64_t kb, int block, const Pages& p) {
    if constexpr (kCodes) {
      if (wave == 0) {       // the pairs, two tokens a lane: keys' to lanes 0 to 31, values' to the others
        const int me = lane_anew(), half = me & 31, token = half * 2;
        const int64_t at = (page_or_0(p.pick(token >> 4)) * heads + head) * page_tokens + ((kb + token) & (page_tokens - 1));
        to_lds(reinterpret_cast<const unsigned char*>((me < 32 ? k_scale : v_scale) + 2 * at), s_raw(block) + 2 * D::kKAll * 16);
      }
    }
    const int w64 = D::kApart ? (wave & 1) * 64 : wave * 64;
    unsigned char* const to_k = (kCodes ? s_raw(block) : s_k(block)) + w64 * 16;
    unsigned char* const to_v = (kCodes ? s_raw(block) + D::kKAll * 16 : s_v(block)) + w64 * 16;
    // Which key and bytes of it, and which V row and token, the lane whose place is `unit` fetches.
    auto key_of = [&](int unit, int* key, int* at) {
      const int row = unit / D::kKParts, c = unit % D::kKParts;
      if constexpr (kCodes) {
        *key = row;
        *at = c * 16;
      } else {
        const int i = row & 15, t = row >> 4;
        *key = (i >> 2) * 16 + t * 4 + (i & 3);
        *at = (W == 128 ? c ^ i : c ^ (i >> 1)) * 16;
      }
    };
    auto value_of = [&](int unit, int* d, int* key) {
      *d = unit / D::kVParts;
      const int c = unit % D::kVParts;
      *key = (kCodes ? c : c ^ ((*d >> 1) & 7)) * D::kVKeys;
    };
    if (one_page) {        // one address for all lanes, and a small offset
      const unsigned char* const k0 = kp + page_or_0(p.at[0]) * k_page + k_head + (kb & (page_tokens - 1)) * F::kRow;
      const unsigned char* const v0 = vp + page_or_0(p.at[0]) * v_page + v_head + (kb & (page_tokens - 1)) * F::kVSize;
      units([&](int unit, int u) {
              int key, at;
              key_of(unit, &key, &at);
              offset_to_lds(k0, key * F::kRow + at, to_k + u * 4096);
            },
            [&](int unit, int u) {
              int d, key;
              value_of(unit, &d, &key);
              offset_to_lds(v0, (d * page_tokens + key) * F::kVSize, to_v + u * 4096);
            });
    } else {
      units([&](int unit, int u) {
              int key, at;
              key_of(unit, &key, &at);
              to_lds(key_source(kb, p, key, at), to_k + u * 4096);
            },
            [&](int unit, int u) {
              int d, key;
              value_of(unit, &d, &key);
              to_lds(value_source(kb, p, d, key), to_v + u * 4096);
            });
    }
  };
  // Steps, zeros and rests of a block's tokens.  A pair that is not finite goes into the step alone, so that it meets the rows that see it and no
  // others.
  auto lay_pair = [&](int block, int which, float2 x) {
    float step = x.x, zero = rintf(fminf(fmaxf(-x.y / x.x, 0.0f), (float)((1 << (BITS == 16 ? 8 : BITS)) - 1)));
    float rest = fmaf(step, zero, x.y);
    if (fabsf(rest) <= 0x1p-20f * fabsf(x.y)) rest = 0.0f;        // the rounding of offset = -step * zero
    if (step == 0.0f) {
      zero = 0.0f;
      rest = x.y;
    }
    if (!(fabsf(x.x) < INFINITY) || !(fabsf(x.y) < INFINITY)) {
      step = NAN;
      zero = rest = 0.0f;
    }
    float* const to = s_pair(block) + 3 * kBlock * which + lane;
    to[0] = step;
    to[kBlock] = zero;
    to[2 * kBlock] = rest;
    const bool any = __any(rest != 0.0f || (which && fabsf(step) < kTiny));
    if (lane == 0) s_flag[2 * (block & (kDepth - 1)) + which] = any;
  };
  // From what was sent for, by the wavefront that did.
  auto lay_pairs = [&](int block) {
    if (wave) return;
    const u32x4 both = read_two(s_raw(block) + 2 * D::kKAll * 16 + lane * 8);
    lay_pair(block, 0, make_float2(__uint_as_float(both[0]), __uint_as_float(both[1])));
    lay_pair(block, 1, make_float2(__uint_as_float(both[2]), __uint_as_float(both[3])));
  };

  // A unit of keys or values as bf16 into its place.
  auto lay_key = [&](int block, int unit, u32x4 x) {
    unsigned char* const sk = s_k(block);
    const int key = unit / D::kKParts, part = unit % D::kKParts, i = (key >> 4) * 4 + (key & 3), t = (key & 15) >> 2;
    if constexpr (BITS == 16) {
      *reinterpret_cast<u32x4*>(sk + key_at<W>(t, i, part)) = x;
    } else {
      const float z = s_pair(block)[kBlock + key];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const uint32_t x0 = x[2 * c], x1 = x[2 * c + 1];
        if constexpr (BITS == 8) {
          *reinterpret_cast<u32x4*>(sk + key_at<W>(t, i, 2 * part + c)) = join(less_zero(x0, z), less_zero(x1, z));
        } else {
          *reinterpret_cast<u32x4*>(sk + key_at<W>(t, i, 2 * part + c)) = join(less_zero(x0 & 0x0f0f0f0fu, z), less_zero(x1 & 0x0f0f0f0fu, z));
          *reinterpret_cast<u32x4*>(sk + key_at<W>(t, i, D::kChunks / 2 + 2 * part + c)) =
              join(less_zero((x0 >> 4) & 0x0f0f0f0fu, z), less_zero((x1 >> 4) & 0x0f0f0f0fu, z));
        }
      }
    }
  };
  auto lay_value = [&](int block, int unit, u32x4 x) {
    unsigned char* const sv = s_v(block);
    const int d = unit / D::kVParts, part = unit % D::kVParts;
    if constexpr (BITS == 16) {
      *reinterpret_cast<u32x4*>(sv + value_at(d, part)) = x;
    } else {
      const float* const zeros = s_pair(block) + 4 * kBlock + part * 16;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const f32x4 z0 = *reinterpret_cast<const f32x4*>(zeros + 8 * c), z1 = *reinterpret_cast<const f32x4*>(zeros + 8 * c + 4);
        const uint32_t x0 = x[2 * c], x1 = x[2 * c + 1];
        if constexpr (BITS == 8) {
          *reinterpret_cast<u32x4*>(sv + value_at(d, 2 * part + c)) = join(less_zeros(x0, z0), less_zeros(x1, z1));
        } else {
          *reinterpret_cast<u32x4*>(sv + value_at(d, 2 * part + c)) = join(less_zeros(x0 & 0x0f0f0f0fu, z0), less_zeros(x1 & 0x0f0f0f0fu, z1));
          *reinterpret_cast<u32x4*>(sv + value_at(d + W / 2, 2 * part + c)) =
              join(less_zeros((x0 >> 4) & 0x0f0f0f0fu, z0), less_zeros((x1 >> 4) & 0x0f0f0f0fu, z1));
        }
      }
    }
  };

  for (int64_t begin = piece_from; begin < piece_end; begin += kRun) {
  end = begin + kRun < piece_end ? begin + kRun : piece_end;
  __syncthreads();
  // First the blocks of committed tokens, nearly all.  Codes: when turn n begins, block n's and n + 1's are on their way to LDS; the turn turns the
  // former into bf16, sends for block n + 2 in their place, and works.  bf16: block n is on its way, and n + 1 is sent for when it is there.
  // A block with rests or without a page is put off.
  const int64_t old_end = KIND == kMasks ? (sq.prefix < end ? sq.prefix : end) : (high_all < end ? high_all : end);
  const int blocks = old_end > begin ? (int)((old_end - begin) / kBlock) : 0;
  const int all_blocks = (int)((end - begin + kBlock - 1) / kBlock);
  constexpr int kAhead = kCodes ? 2 : 1;
  int later = 0;
  if (blocks > 0) {
    Pages ahead = pages_of(begin);       // of the block that is sent for next
    uint32_t holes = ahead.missing();     // bit j: block n + j has no page for some of its tokens
    send(begin, 0, ahead);
    if constexpr (kCodes) {
      ahead = pages_of(begin + kBlock);
      holes |= (uint32_t)ahead.missing() << 1;
      wait_loads<0>();
      lay_pairs(0);
      if (blocks > 1) send(begin + kBlock, 1, ahead);
    }
    ahead = pages_of(begin + kAhead * kBlock);
    pipeline_barrier();

    for (int n = 0; n < blocks; ++n) {
      const int64_t kb = begin + (int64_t)n * kBlock;
      const bool more = n + kAhead < blocks;
      holes |= (uint32_t)ahead.missing() << kAhead;
      if constexpr (kCodes) {
        // all but what was sent for last, the units of block n + 1: its pairs were sent for before them
        if (n + 1 < blocks) {
          wait_loads<D::kApart ? 1 : 2 * D::kUnits>();
          lay_pairs(n + 1);
        } else {
          wait_loads<0>();
        }
        const unsigned char* const raw = s_raw(n);
        units([&](int unit, int) { lay_key(n, unit, *reinterpret_cast<const u32x4*>(raw + unit * 16)); },
              [&](int unit, int) { lay_value(n, unit, *reinterpret_cast<const u32x4*>(raw + (D::kKAll + unit) * 16)); });
        pipeline_barrier();
        if (more) send(kb + kAhead * kBlock, n, ahead);
      } else {
        wait_loads<0>();
        pipeline_barrier();
        if (more) send(kb + kAhead * kBlock, n + 1, ahead);
      }
      ahead = pages_of(kb + (kAhead + 1) * kBlock);
      const unsigned char* const sk = s_k(n);
      const unsigned char* const sv = s_v(n);
      bool put_off = (holes & 1) || (KIND != kMasks && kb < low_all);
      holes >>= 1;
      if constexpr (kCodes) {
        const int* f = s_flag + 2 * (n & (kDepth - 1));
        put_off = put_off || __builtin_amdgcn_readfirstlane(f[0] | f[1]);
      }
      if (put_off) {
        if (tid == 0) s_later[later] = (uint16_t)n;
        ++later;
      }
      const bool work = !idle && !put_off;

      // The operands of a block in the order of their use: of each half those of the keys, then those of the values.  kRing of them are on their way
      // from LDS ahead of the products that take them.
      constexpr int kOfKeys = 2 * kOps, kOfHalf = kOfKeys + kTiles;
      bf16x8 ring[kRing];
      auto operand = [&](auto index) {
        constexpr int N = decltype(index)::value, H = N / kOfHalf, J = N % kOfHalf;
        if constexpr (H < 2) {
          if constexpr (J < kOfKeys)
            ring[N % kRing] = *reinterpret_cast<const bf16x8*>(sk + key_at<W>(2 * H + J / kOps, col, J % kOps * 4 + g));
          else
            ring[N % kRing] = *reinterpret_cast<const bf16x8*>(sv + value_at((J - kOfKeys) * 16 + col, g * 2 + H));
        }
      };

      // A half: the 32 keys 16 g + 8 H to 16 g + 8 H + 7 of the quarters.
      auto half = [&](auto h) {
        constexpr int H = decltype(h)::value;
        f32x4 s[QT][2];
#pragma unroll
        for (int x = 0; x < QT; ++x) s[x][0] = s[x][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        each<kOfKeys>([&](auto j) {
          constexpr int J = decltype(j)::value, N = H * kOfHalf + J;
#pragma unroll
          for (int x = 0; x < QT; ++x) s[x][J / kOps] = mfma(ring[N % kRing], qf[x][J % kOps], s[x][J / kOps]);
          operand(std::integral_constant<int, N + kRing>{});
          __builtin_amdgcn_sched_barrier(kArithmetic);
        });
        float ks[8];
        float v_step = 1.0f, v_inv = 1.0f;
        if constexpr (kCodes) {
          const float k_step = s_pair(n)[lane] * scale;
          v_step = s_pair(n)[3 * kBlock + lane];
          v_inv = __builtin_amdgcn_rcpf(v_step);
          each<8>([&](auto e) { ks[decltype(e)::value] = row_bcast<8 * H + decltype(e)::value>(k_step); });
        }
#pragma unroll
        for (int x = 0; x < QT; ++x) {
          const float base = m[x] == -INFINITY ? 0.0f : m[x];
#pragma unroll
          for (int e = 0; e < 8; ++e) s[x][e / 4][e % 4] = fmaf(s[x][e / 4][e % 4], kCodes ? ks[e] : scale, KIND == kOptions ? 0.0f : -base);
          if constexpr (KIND == kOptions) {
            if (cap != 0.0f) {
#pragma unroll
              for (int e = 0; e < 8; ++e) s[x][e / 4][e % 4] = capped(s[x][e / 4][e % 4], cap, cap_in);
            }
            const float near = (float)(sq.prefix - kb) - 8.0f * H;
#pragma unroll
            for (int e = 0; e < 8; ++e) s[x][e / 4][e % 4] = fmaf(-slope[x], fabsf(place[x] + (near - (float)e)), s[x][e / 4][e % 4]) - base;
          }
          const float top = fmaxf(fmaxf(fmaxf(s[x][0][0], s[x][0][1]), fmaxf(s[x][0][2], s[x][0][3])), fmaxf(fmaxf(s[x][1][0], s[x][1][1]), fmaxf(s[x][1][2], s[x][1][3])));
          if (__any(top > (m[x] == -INFINITY ? -INFINITY : kRise))) {
            const float by = raise(m[x], column_max(top));
            s[x][0] -= by;
            s[x][1] -= by;
            const float f = m_factor(by);
            if constexpr (kCodes)
              l_run[x] *= f;
            else
              l_acc[x] *= f;
#pragma unroll
            for (int d = 0; d < kTiles; ++d) o[x][d] *= f;
          }
        }
        bf16x8 pf[QT];
#pragma unroll
        for (int x = 0; x < QT; ++x) {
          float y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            y[e] = __builtin_amdgcn_exp2f(s[x][e / 4][e % 4]);
          }
          if constexpr (kCodes) each<8>([&](auto e) { y[decltype(e)::value] *= row_bcast<8 * H + decltype(e)::value>(v_step); });
          const uint32_t w[4] = {f32x2_to_bf16x2(y[0], y[1]), f32x2_to_bf16x2(y[2], y[3]), f32x2_to_bf16x2(y[4], y[5]), f32x2_to_bf16x2(y[6], y[7])};
          pf[x] = as_frag(w[0], w[1], w[2], w[3]);
          // The weights that the sum is divided by, as they are rounded.
          if constexpr (kCodes) each<8>([&](auto at) {
            constexpr int e = decltype(at)::value;
            l_run[x] += __uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16) * row_bcast<8 * H + e>(v_inv);
          });
        }
        each<kTiles>([&](auto d) {
          constexpr int D = decltype(d)::value, N = H * kOfHalf + kOfKeys + D;
#pragma unroll
          for (int x = 0; x < QT; ++x) o[x][D] = mfma(ring[N % kRing], pf[x], o[x][D]);
          operand(std::integral_constant<int, N + kRing>{});
          __builtin_amdgcn_sched_barrier(kArithmetic);
        });
        if constexpr (!kCodes) {
#pragma unroll
          for (int x = 0; x < QT; ++x) l_acc[x] = mfma(ones, pf[x], l_acc[x]);
        }
      };
      if (work) {
        each<kRing>(operand);
        half(std::integral_constant<int, 0>{});
        half(std::integral_constant<int, 1>{});
      }
      if constexpr (kCodes) pipeline_barrier();
    }
  }

  number();
  // Then what was put off, and the blocks of new tokens: one at a time, with every case.
  for (int k = 0; k < later + all_blocks - blocks; ++k) {
    __syncthreads();
    const int n = k < later ? (int)s_later[k] : blocks + k - later;
    const int64_t kb = begin + (int64_t)n * kBlock;
    const Pages p = pages_of(kb);
    u32x4 raw[D::kApart ? 1 : 2 * D::kUnits];          // keys, then values
    units([&](int unit, int u) { raw[u] = *reinterpret_cast<const u32x4*>(key_source(kb, p, unit / D::kKParts, unit % D::kKParts * 16)); },
          [&](int unit, int u) {
            raw[D::kApart ? 0 : D::kUnits + u] = *reinterpret_cast<const u32x4*>(value_source(kb, p, unit / D::kVParts, unit % D::kVParts * D::kVKeys));
          });
    if (tid == 0) s_flag[1] = 0;
    if constexpr (kCodes) {
      if (wave < 2) {
        const int32_t page = p.pick(g);
        const int64_t at = (page_or_0(page) * heads + head) * page_tokens + ((kb + lane) & (page_tokens - 1));
        float2 x = make_float2(0.0f, 0.0f);
        if (page >= 0 && kb + lane < end) x = reinterpret_cast<const float2*>(wave ? v_scale : k_scale)[at];
        lay_pair(0, wave, x);
      }
    }
    __syncthreads();
    units([&](int unit, int u) { lay_key(0, unit, raw[u]); },
          [&](int unit, int u) {
            u32x4 x = raw[D::kApart ? 0 : D::kUnits + u];
            if constexpr (BITS == 16) {
              // slots that hold no token hold anything; infinities and NaNs of new tokens are looked after below
              const int part = unit % D::kVParts;
              const int64_t left = p.pick(part >> 1) < 0 ? 0 : end - kb - part * 8;
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                x[j] &= (left > 2 * j ? 0xffffu : 0u) | (left > 2 * j + 1 ? 0xffff0000u : 0u);
                if (any_nonfinite(x[j])) s_flag[1] = 1;
              }
            }
            lay_value(0, unit, x);
          });
    __syncthreads();
    if (idle) continue;
    const unsigned char* const sk = s_k(0);
    const unsigned char* const sv = s_v(0);
    const bool odd = !kCodes && s_flag[1];
    float k_step = scale, v_step = 1.0f, k_rest = 0.0f, v_rest = 0.0f, v_inv = 1.0f, v_one = 0.0f;      // v_one: the weight goes in as it is
    if constexpr (kCodes) {
      const float* const pair = s_pair(0) + lane;
      k_step *= pair[0];
      k_rest = pair[2 * kBlock] * scale;
      v_step = pair[3 * kBlock];
      v_rest = pair[5 * kBlock];
      if (fabsf(v_step) < kTiny) {
        v_inv = 0.0f;
        v_one = 1.0f;
      } else {
        v_inv = __builtin_amdgcn_rcpf(v_step);
      }
    }
    const int64_t pos = kb + g * 16, j0 = pos - sq.prefix;
    uint32_t exists = 0;
    if (pos < end && p.pick(g) >= 0) exists = end - pos >= 16 ? 0xffffu : (1u << (int)(end - pos)) - 1;
#pragma unroll
    for (int x = 0; x < QT; ++x) {
      const int row = row0 + x * 16 + col;
      uint32_t vis;
      if constexpr (KIND == kMasks) {
        const int node = row / a->group;
        uint64_t seen = 0;
        if (row < rows) seen = a->mask ? a->mask[sq.first + node] : (2ull << node) - 1;
        if (sq.count < 64) seen &= (1ull << sq.count) - 1;
        if (j0 >= 0)
          vis = j0 < 64 ? (uint32_t)(seen >> j0) : 0;
        else
          vis = j0 > -16 ? (uint32_t)(seen << -j0) | ((1u << -j0) - 1) : 0xffffu;
      } else {
        vis = row < rows ? between(pos, chunk_keys(a, sq, (uint32_t)row / (uint32_t)a->group)) : 0;
      }
      vis &= exists;
      float q_sum = 0.0f;
      if constexpr (kCodes) {
#pragma unroll
        for (int i = 0; i < kOps; ++i) {
          const u32x4 q = __builtin_bit_cast(u32x4, qf[x][i]);
#pragma unroll
          for (int j = 0; j < 4; ++j) q_sum += __uint_as_float(q[j] << 16) + __uint_as_float(q[j] & 0xffff0000u);
        }
        q_sum = column_sum(q_sum);
      }
#pragma unroll 1
      for (int H = 0; H < 2; ++H) {
        f32x4 s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          s[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int i = 0; i < kOps; ++i) s[t] = mfma(*reinterpret_cast<const bf16x8*>(sk + key_at<W>(2 * H + t, col, i * 4 + g)), qf[x][i], s[t]);
        }
        const uint32_t see = vis >> (8 * H);
        float top = -INFINITY;
        const float base = m[x] == -INFINITY ? 0.0f : m[x];
        each<8>([&](auto at) {
          constexpr int e = decltype(at)::value;
          float v = s[e / 4][e % 4] * (kCodes ? row_bcast<e>(k_step) : k_step);
          if constexpr (kCodes) v += row_bcast<e>(k_rest) * q_sum;
          if constexpr (KIND == kOptions) {
            if (cap != 0.0f) v = capped(v, cap, cap_in);
            v = fmaf(-slope[x], fabsf(place[x] + ((float)(sq.prefix - kb) - (float)(8 * H + e))), v);
          }
          s[e / 4][e % 4] = (see >> e) & 1 ? v - base : -INFINITY;
          top = fmaxf(top, s[e / 4][e % 4]);
        });
        const float by = raise(m[x], column_max(top));
        const float f = m_factor(by);
        if constexpr (kCodes)
          l_run[x] *= f;
        else
          l_acc[x] *= f;
        // Each weight reaches the sum that divides and the rest of its value (c) as the product takes it: rounded, over the step.
        float y[8], c = 0.0f;
        each<8>([&](auto at) {
          constexpr int e = decltype(at)::value;
          y[e] = __builtin_amdgcn_exp2f(s[e / 4][e % 4] - by);
          if constexpr (kCodes) {
            const float one = y[e] * row_bcast<e>(v_one);
            const float add = one * row_bcast<e>(v_rest), w = y[e] * row_bcast<e>(v_step);      // (whatever pair the slot holds)
            l_run[x] += one;
            c += (see >> e) & 1 ? add : 0.0f;
            y[e] = (see >> e) & 1 ? w : 0.0f;
          }
        });
        const uint32_t w[4] = {f32x2_to_bf16x2(y[0], y[1]), f32x2_to_bf16x2(y[2], y[3]), f32x2_to_bf16x2(y[4], y[5]), f32x2_to_bf16x2(y[6], y[7])};
        const bf16x8 pf = as_frag(w[0], w[1], w[2], w[3]);
        if constexpr (kCodes) {
          each<8>([&](auto at) {
            constexpr int e = decltype(at)::value;
            const float weight = __uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16) * row_bcast<e>(v_inv);
            const float add = weight * row_bcast<e>(v_rest);
            l_run[x] += (see >> e) & 1 ? weight : 0.0f;
            c += (see >> e) & 1 ? add : 0.0f;
          });
          c = column_sum(c);
        }
#pragma unroll
        for (int d = 0; d < kTiles; ++d) o[x][d] = o[x][d] * f + c;
#pragma unroll
        for (int d = 0; d < kTiles; ++d) {
          u32x4 z = *reinterpret_cast<const u32x4*>(sv + value_at(d * 16 + col, g * 2 + H));
          if (odd) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if ((z[j] & 0x7f80u) == 0x7f80u) z[j] &= 0xffff0000u;
              if ((z[j] & 0x7f800000u) == 0x7f800000u) z[j] &= 0x0000ffffu;
            }
          }
          o[x][d] = mfma(__builtin_bit_cast(bf16x8, z), pf, o[x][d]);
        }
        if constexpr (!kCodes) l_acc[x] = mfma(ones, pf, l_acc[x]);
        if (odd) {
          // Infinities and NaNs among the values: each goes to the rows that see it, by itself.
          for (int e = 0; e < kBlock / 2; ++e) {
            const int eg = e >> 3, bit = e & 7, key = eg * 16 + 8 * H + bit;
            uint32_t word = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) word = (bit >> 1) == i ? w[i] : word;
            const float one = bf16_to_f32((bf16_bits)__shfl((int)(bit & 1 ? word >> 16 : word & 0xffffu), eg * 16 + col));
            const bool sees = (__shfl((int)see, eg * 16 + col) >> bit) & 1;
#pragma unroll
            for (int d = 0; d < kTiles; ++d)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const bf16_bits z = *reinterpret_cast<const bf16_bits*>(sv + value_at(d * 16 + g * 4 + r, key >> 3) + (key & 7) * 2);
                if (sees && (z & 0x7f80u) == 0x7f80u) o[x][d][r] += one * bf16_to_f32(z);
              }
          }
        }
        if constexpr (kCodes) {          // the other half's to where this half's were; after two turns all are back
          k_step = row_rotated<8>(k_step);
          k_rest = row_rotated<8>(k_rest);
          v_step = row_rotated<8>(v_step);
          v_rest = row_rotated<8>(v_rest);
          v_inv = row_rotated<8>(v_inv);
          v_one = row_rotated<8>(v_one);
        }
      }
    }
  }
  }
  if (idle) continue;

  number();
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    const int row = row0 + x * 16 + col;
    float l = kCodes ? column_sum(l_run[kCodes ? x : 0]) : l_acc[kCodes ? 0 : x][0];
    if constexpr (KIND != kMasks) {
      const int2 k = chunk_keys(a, sq, (uint32_t)(row < rows ? row : 0) / (uint32_t)a->group);
      if (k.x >= k.y) {
        m[x] = -INFINITY;
        l = 0.0f;
#pragma unroll
        for (int d = 0; d < kTiles; ++d) o[x][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      }
    }
    if (!piece.whole) {      // as the registers have it, 16 rows a tile: whole lines of memory
      float* const to = a->part + part_at(a, head, row_tile, piece.slot, row0 + x * 16 - row_tile * 64 * QT) * W + lane * 4;
#pragma unroll
      for (int d = 0; d < kTiles; ++d) *reinterpret_cast<f32x4*>(to + d * 256) = o[x][d];
    }
    if (row >= rows) continue;
    if (piece.whole) {
#pragma unroll
      for (int d = 0; d < kTiles; ++d) store_row4(a, sq, head, row, d * 16 + g * 4, o[x][d], l);
    } else {
      if (g == 0) a->part_ml[part_at(a, head, row_tile, piece.slot, row - row_tile * 64 * QT)] = make_float2(m[x], l);
    }
  }
  }
}

template <int BITS, int W, int QT, int KIND>
hipError_t launch_wide_as(const TreeArgs& a, dim3 grid, hipStream_t s) {
  constexpr int kShared = Wide<BITS, W>::kShared;        // above what a launch may ask for by itself
  static PerDeviceOnce once;
  const hipError_t e = once.run([] {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(k_tree_wide<BITS, W, QT, KIND>), hipFuncAttributeMaxDynamicSharedMemorySize, kShared);
  });
  if (e != hipSuccess) return e;
  k_tree_wide<BITS, W, QT, KIND><<<grid, 64 * kWaves, kShared, s>>>(a);
  return hipGetLastError();
}

}  // namespace

}  // namespace tree
}  // namespace conqur
