// The kernel of few rows (tree_attention.hip has the mathematics and what it measured).
#pragma once
#include "tree_attention.h"

namespace conqur {
namespace tree {

namespace {

template <int BITS, int W>
struct Keys {        // a lane's share of 64 keys: four tiles of 16
  uint32_t w[4][Format<BITS, W>::kWords];
};
template <int BITS, int W>
struct Values {      // a lane's 16 tokens of its V rows
  uint32_t w[Format<BITS, W>::kVTiles][Format<BITS, W>::kVWords];
};

// 16 bytes (8) from where `from` and a uniform offset, the same for all lanes, and a lane's offset point to.
__device__ __forceinline__ u32x4 load_b128(const unsigned char* from, int lane_offset, int offset) {
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(from), 0, 0x7fffffff, 0x00020000);
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, lane_offset, offset, 0));
}
__device__ __forceinline__ u32x2 load_b64(const unsigned char* from, int lane_offset, int offset) {
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(from), 0, 0x7fffffff, 0x00020000);
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, lane_offset, offset, 0));
}

// A lane's share of 64 keys: tile t's keys are 4 t further on.  at(bytes): 16 bytes (8) that far behind the lane's first key.
template <int BITS, int W, typename At16, typename At8>
__device__ __forceinline__ void load_keys(Keys<BITS, W>& k, At16 at16, At8 at8) {
  using F = Format<BITS, W>;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    if constexpr (F::kWords >= 4) {
#pragma unroll
      for (int i = 0; i < F::kWords / 4; ++i) {
        const u32x4 x = at16(t * 4 * F::kRow + i * 64);
#pragma unroll
        for (int j = 0; j < 4; ++j) k.w[t][4 * i + j] = x[j];
      }
    } else {
      const u32x2 x = at8(t * 4 * F::kRow);
      k.w[t][0] = x[0];
      k.w[t][1] = x[1];
    }
  }
}
template <int BITS, int W>
__device__ __forceinline__ bf16x8 key_operand(const Keys<BITS, W>& k, int t, int i) {
  if constexpr (BITS == 16) return as_frag(k.w[t][4 * i], k.w[t][4 * i + 1], k.w[t][4 * i + 2], k.w[t][4 * i + 3]);
  if constexpr (BITS == 8) {
    const uint32_t a = k.w[t][2 * i], b = k.w[t][2 * i + 1];
    return as_frag(bytes_to_bf16(a, 0), bytes_to_bf16(a, 1), bytes_to_bf16(b, 0), bytes_to_bf16(b, 1));
  }
  constexpr int kHalf = W / 64;                      // operands of the low halves
  const int s = i >= kHalf ? 4 : 0, o = (i % kHalf) * 2;
  const uint32_t a = k.w[t][o], b = k.w[t][o + 1];
  return as_frag(nibbles_to_bf16(a, s), nibbles_to_bf16(a, s + 8), nibbles_to_bf16(b, s), nibbles_to_bf16(b, s + 8));
}
// at(tile, bytes): 16 bytes that far behind the lane's first token, in its V row of that tile.
template <int BITS, int W, typename At>
__device__ __forceinline__ void load_values(Values<BITS, W>& v, At at) {
  using F = Format<BITS, W>;
#pragma unroll
  for (int t = 0; t < F::kVTiles; ++t)
#pragma unroll
    for (int i = 0; i < F::kVSize; ++i) {
      const u32x4 x = at(t, i * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) v.w[t][4 * i + j] = x[j];
    }
}
// Tile t of W / 16 output tiles, operand m of 2 (32 keys each).
template <int BITS, int W>
__device__ __forceinline__ bf16x8 value_operand(const Values<BITS, W>& v, int t, int m) {
  if constexpr (BITS == 16) return as_frag(v.w[t][4 * m], v.w[t][4 * m + 1], v.w[t][4 * m + 2], v.w[t][4 * m + 3]);
  if constexpr (BITS == 8) {
    const uint32_t a = v.w[t][2 * m], b = v.w[t][2 * m + 1];
    return as_frag(bytes_to_bf16(a, 0), bytes_to_bf16(a, 1), bytes_to_bf16(b, 0), bytes_to_bf16(b, 1));
  }
  constexpr int kHalf = W / 32;
  const int s = t >= kHalf ? 4 : 0;
  const uint32_t a = v.w[t % kHalf][2 * m], b = v.w[t % kHalf][2 * m + 1];
  return as_frag(nibbles_to_bf16(a, s), nibbles_to_bf16(a, s + 8), nibbles_to_bf16(b, s), nibbles_to_bf16(b, s + 8));
}
// Two neighbouring weights of a lane's four of a key tile, in the order in which value_operand has the tokens.
template <int BITS>
__device__ __forceinline__ void pack_weights(const float* w, uint32_t* out) {
  out[0] = f32x2_to_bf16x2(w[0], w[BITS == 4 ? 2 : 1]);
  out[1] = f32x2_to_bf16x2(w[BITS == 4 ? 1 : 2], w[3]);
}

// ONE_PAGE: pages of 64 tokens or more, so that a block lies in one and its address is the same for all lanes but for an offset.  (Both forms in one
// kernel take 60 registers more than either: 16-bit values 128 wide then spill, 215 -> 369 us for the batch of the figures below.)
template <int BITS, int W, int QT, bool ONE_PAGE, int KIND>
__global__ void __launch_bounds__(64 * kWaves, 2) k_tree(const TreeArgs) {
  Args a = kernel_args();
  using F = Format<BITS, W>;
  constexpr int kOps = W / 32;            // operands of the first product
  constexpr int kTiles = W / 16;          // tiles of the result
  constexpr bool kCodes = BITS != 16;
  constexpr int kStep = kBlock * kWaves;
  constexpr int kParts = QT > 1 || !kCodes ? 2 : 1, kT = 4 / kParts;      // parts of a block, key tiles of a part
  constexpr bool kThrough = QT == 1;      // the loop over committed tokens also fetches the first block behind them (with QT = 2 that takes registers which are not there)
  // The wavefronts' results meet here at the end: two wavefronts' at a time.
  __shared__ __attribute__((aligned(16))) float s_o[2][QT * kTiles][64][4];
  __shared__ float s_ml[2][QT][2][64];

  int head, row_tile;
  Pieces piece;
  place_of<KIND>(a, &head, &row_tile, &piece.b, &piece.run);
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int row0 = row_tile * 16 * QT;
  if constexpr (KIND != kMasks) {
    if (a->looks) zero_rows(a);
  }
  const bf16x8 ones = as_frag(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);      // a row of the sums of the weights as they are rounded
  for (bool first = true; piece.next(a, row0, first); first = false) {
    int lane, col, g;
    auto number = [&] {
      a = kernel_args();
      lane = lane_anew();
      col = lane & 15;
      g = lane >> 4;
    };
    number();
    const int b = piece.b;
    const Sequence sq = sequence_of(a, b);
    const int rows = sq.count * a->group;
    const int64_t base_key = KIND == kMasks ? 0 : (int64_t)first_block(a, sq, row0) * kBlock, limit = KIND == kMasks ? sq.length : tile_end(a, sq, row0);
    const int64_t piece_end = base_key + (int64_t)piece.last * kBlock;
    int64_t begin = base_key + (int64_t)piece.first * kBlock, end = piece_end < limit ? piece_end : limit;
    // A chunk: the keys of each row, and those that all rows see.  A row that sees nothing is taken to see all, and gets zeros at the end.
    int low_all = 0, high_all = 0, low_any = 0, high_any = 0;
    float slope[QT], place[QT];
    if constexpr (KIND != kMasks) {
      high_all = low_any = INT_MAX;
#pragma unroll
      for (int x = 0; x < QT; ++x) {
        const int row = row0 + x * 16 + col, node = (uint32_t)(row < rows ? row : 0) / (uint32_t)a->group;
        const int2 k = chunk_keys(a, sq, node);
        const bool any = row < rows && k.x < k.y;
        low_all = max(low_all, wave_max_int(any ? k.x : 0));
        high_all = min(high_all, wave_min(any ? k.y : INT_MAX));
        low_any = min(low_any, wave_min(any ? k.x : INT_MAX));
        high_any = max(high_any, wave_max_int(any ? k.y : 0));
        if constexpr (KIND == kOptions) {
          slope[x] = a->slopes ? a->slopes[head * a->group + (row < rows ? row : 0) - node * a->group] * 1.4426950408889634f : 0.0f;
          place[x] = (float)node - 16.0f * g;      // less the block's first key and the committed tokens' number
        }
      }
    }

    if constexpr (KIND != kMasks) {          // what no row sees is left out
      if (high_any < end) end = high_any;
      if (low_any / kBlock * kBlock > begin) begin = low_any / kBlock * kBlock;
    }

    // Queries: operand i of column `col`, in the order in which the keys' operands have the entries.
    bf16x8 qf[QT][kOps];
    float q_sum[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const int row = row0 + t * 16 + col;
      const bool here = row < rows;
      const bf16_bits* p = a->q + (sq.first + (here ? row / a->group : 0)) * a->q_ts + (int64_t)(head * a->group + (here ? row % a->group : 0)) * a->q_hs;
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < kOps; ++i) {
        bf16_bits e[8];
        const int base = entry_of<BITS, W>(i, g, 0);
        if (a->q_wide) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(p + base);
#pragma unroll
          for (int j = 0; j < 8; ++j) e[j] = (bf16_bits)(x[j / 2] >> (j % 2 * 16));
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) e[j] = p[base + j];
        }
        uint32_t u[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int x = entry_of<BITS, W>(i, g, 2 * j) - base, y = entry_of<BITS, W>(i, g, 2 * j + 1) - base;
          u[j] = here ? e[x] | (uint32_t)e[y] << 16 : 0;
          if (kCodes && here) sum += bf16_to_f32(e[x]) + bf16_to_f32(e[y]);
        }
        qf[t][i] = as_frag(u[0], u[1], u[2], u[3]);
      }
      q_sum[t] = kCodes ? column_sum(sum) : 0.0f;
    }

    f32x4 o[QT][kTiles], l_acc[kCodes ? 1 : QT];
    float m[QT], l_run[kCodes ? QT : 1], c_run[kCodes ? QT : 1];      // maxima as in raise(), sums of weights, what belongs to every entry of a row
#pragma unroll
    for (int t = 0; t < QT; ++t) {
#pragma unroll
      for (int d = 0; d < kTiles; ++d) o[t][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      if constexpr (kCodes)
        l_run[t] = c_run[t] = 0.0f;
      else
        l_acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      m[t] = -INFINITY;
    }

    const int page_tokens = (int)a->cache.page_tokens;
    const int page_shift = 31 - __builtin_clz(page_tokens);
    const Scalars table = (Scalars)(uintptr_t)(a->batch.table + (int64_t)b * a->batch.table_stride);
    const int64_t heads = a->cache.heads;
    const uint32_t pages = (uint32_t)a->cache.pages;
    const float* const k_scale = a->cache.k_scale;
    const float* const v_scale = a->cache.v_scale;
    const float scale = a->scale_log2, cap = KIND == kOptions ? a->cap_log2 : 0.0f, cap_in = KIND == kOptions ? a->cap_in : 0.0f;
    auto pages_of = [&](int64_t kb) {
      Pages p;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int64_t pos = kb + 16 * u;
        int32_t x = ONE_PAGE && u ? p.at[0] : -1;
        if (!(ONE_PAGE && u) && pos < end) x = table[pos >> page_shift];
        p.at[u] = x >= 0 && (uint32_t)x < pages ? x : -1;
      }
      return p;
    };
    const unsigned char* kp = static_cast<const unsigned char*>(a->cache.k);
    const unsigned char* vp = static_cast<const unsigned char*>(a->cache.v);
    const int v_pitch = page_tokens * F::kVSize;
    auto page_at = [&](int32_t p) { return (int64_t)(p < 0 ? 0 : p) * (ONE_PAGE ? heads : kernel_args()->cache.heads) + head; };      // where there is none, reads go to page 0 and are not used

    Keys<BITS, W> kf;
    Values<BITS, W> vf;
    float2 ks, vs;                      // the pair of key `lane` of the block
    auto fetch_keys = [&](int64_t kb, const Pages& p) {
      const int me = lane_anew(), c = me & 15, part = (me >> 4) * (F::kWords >= 4 ? 16 : 8);
      if constexpr (ONE_PAGE) {
        const int64_t at = page_at(p.at[0]) * page_tokens + (kb & (page_tokens - 1));
        const unsigned char* from = kp + at * F::kRow;
        const int offset = ((c >> 2) * 16 + (c & 3)) * F::kRow + part;
        load_keys<BITS, W>(kf, [&](int bytes) { return load_b128(from, offset + bytes, 0); }, [&](int bytes) { return load_b64(from, offset + bytes, 0); });
        if constexpr (kCodes) ks = __builtin_bit_cast(float2, load_b64(reinterpret_cast<const unsigned char*>(k_scale + 2 * at), me * 8, 0));
      } else {
        const unsigned char* from = static_cast<const unsigned char*>(kernel_args()->cache.k) + (page_at(p.pick(c >> 2)) * page_tokens + ((kb + (c >> 2) * 16) & (page_tokens - 1)) + (c & 3)) * F::kRow + part;
        load_keys<BITS, W>(kf, [&](int bytes) { return *reinterpret_cast<const u32x4*>(from + bytes); },
                           [&](int bytes) { return *reinterpret_cast<const u32x2*>(from + bytes); });
        if constexpr (kCodes) ks = reinterpret_cast<const float2*>(kernel_args()->cache.k_scale)[page_at(p.pick(me >> 4)) * page_tokens + ((kb + me) & (page_tokens - 1))];
      }
    };
    auto fetch_values = [&](int64_t kb, const Pages& p) {
      const int me = lane_anew(), c = me & 15, quarter = me >> 4;
      if constexpr (ONE_PAGE) {
        const int slot = (int)(kb & (page_tokens - 1));
        const unsigned char* from = vp + page_at(p.at[0]) * F::kVRows * v_pitch + slot * F::kVSize;
        const int offset = c * v_pitch + quarter * 16 * F::kVSize;
        load_values<BITS, W>(vf, [&](int t, int bytes) { return load_b128(from, offset + bytes, t * 16 * v_pitch); });
        if constexpr (kCodes) vs = __builtin_bit_cast(float2, load_b64(reinterpret_cast<const unsigned char*>(v_scale + 2 * (page_at(p.at[0]) * page_tokens + slot)), me * 8, 0));
      } else {
        const int64_t page = page_at(p.pick(quarter));
        const unsigned char* from = static_cast<const unsigned char*>(kernel_args()->cache.v) + (page * F::kVRows + c) * v_pitch + ((kb + quarter * 16) & (page_tokens - 1)) * F::kVSize;
        load_values<BITS, W>(vf, [&](int t, int bytes) {
          if (t > 0 && bytes == 0) from += 16 * v_pitch;      // (one pointer, not one a tile)
          return *reinterpret_cast<const u32x4*>(from + bytes);
        });
        if constexpr (kCodes) vs = reinterpret_cast<const float2*>(kernel_args()->cache.v_scale)[page * page_tokens + ((kb + me) & (page_tokens - 1))];
      }
    };
    // What the scores and the values have beside step times code, from a pair; see the top.  With a step of 0 (a constant row) or one so small that
    // weights times it leave the range, the offset is added by the weight itself.
    auto is_tiny = [&](float2 x) { return fabsf(x.x) < 1e-30f; };
    auto off_of = [&](float2 x) { return is_tiny(x) ? 0.0f : x.y / x.x - shifted<BITS>(); };
    auto inv_of = [&](float2 x) { return is_tiny(x) ? 0.0f : __builtin_amdgcn_rcpf(x.x); };
    auto place_of = [](int e) { return BITS == 4 ? (e % 4 == 1 ? 2 : e % 4 == 2 ? 1 : e % 4) : e % 4; };      // where pack_weights puts weight e of four

    // What is new falls to where the maximum was raised by `by`, and what was with it.
    auto lower = [&](int x, float by) {
      const float f = m_factor(by);
      if constexpr (kCodes) {
        l_run[x] *= f;
        c_run[x] *= f;
      } else {
        l_acc[x] *= f;
      }
#pragma unroll
      for (int d = 0; d < kTiles; ++d) o[x][d] *= f;
    };

    const int64_t old_end = KIND == kMasks ? (sq.prefix < end ? sq.prefix : end) : (high_all < end ? high_all : end);
    const int64_t plain_end = old_end > begin ? begin + (old_end - begin) / kBlock * kBlock : begin;
    for (int64_t run = begin; run < end; run += kRun) {
      const int64_t run_end = run + kRun < end ? run + kRun : end, plain = plain_end < run_end ? plain_end : run_end;
      uint64_t later = 0;               // blocks of the wavefront without a page for some of their tokens
      int64_t kb = run + wave * kBlock;
      const bool started = kb < plain;
      // First the blocks of committed tokens, nearly all.
      if (started) {
        Pages ahead = pages_of(kb);
        fetch_keys(kb, ahead);
        fetch_values(kb, ahead);
        bool hole = ahead.missing() || (KIND != kMasks && kb < low_all);
        ahead = pages_of(kb + kStep);
        uint64_t bit = 1;
        for (; kb < plain; kb += kStep, bit <<= 1) {
          const bool more = kb + kStep < (kThrough ? run_end : plain);
          const float k_step = kCodes ? ks.x * scale : scale, k_off = kCodes ? (ks.y - shifted<BITS>() * ks.x) * scale : 0.0f;
          // A block in parts: what of its scores is in registers at a time.
          each<kParts>([&](auto part) {
            constexpr int T = decltype(part)::value * kT, E0 = T * 4;          // first key tile, first of the lane's keys
            f32x4 s[QT][kT];
#pragma unroll
            for (int t = 0; t < kT; ++t) {
#pragma unroll
              for (int x = 0; x < QT; ++x) s[x][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
              for (int i = 0; i < kOps; ++i) {
                const bf16x8 kk = key_operand<BITS, W>(kf, T + t, i);
#pragma unroll
                for (int x = 0; x < QT; ++x) s[x][t] = mfma(kk, qf[x][i], s[x][t]);
              }
              __builtin_amdgcn_sched_barrier(0);      // (operands made ahead of their use fill the registers)
            }
            if (T + kT == 4 && more) fetch_keys(kb + kStep, ahead);
            if (hole) return;
            float base[QT], top[QT];
#pragma unroll
            for (int x = 0; x < QT; ++x) {
              base[x] = m[x] == -INFINITY ? 0.0f : m[x];
              top[x] = -INFINITY;
            }
            each<4 * kT>([&](auto e) {
              constexpr int E = decltype(e)::value;
              const float step = kCodes ? row_bcast<E0 + E>(k_step) : k_step, off = kCodes ? row_bcast<E0 + E>(k_off) : 0.0f;
#pragma unroll
              for (int x = 0; x < QT; ++x) {
                const float less = KIND == kOptions ? 0.0f : base[x];
                const float y = fmaf(s[x][E / 4][E % 4], step, kCodes ? fmaf(off, q_sum[x], -less) : -less);
                s[x][E / 4][E % 4] = y;
                if constexpr (KIND != kOptions) top[x] = fmaxf(top[x], y);
              }
            });
            if constexpr (KIND == kOptions) {
              if (cap != 0.0f) {
#pragma unroll
                for (int x = 0; x < QT; ++x)
#pragma unroll
                  for (int e = 0; e < 4 * kT; ++e) s[x][e / 4][e % 4] = capped(s[x][e / 4][e % 4], cap, cap_in);
              }
              const float near = (float)(sq.prefix - kb);
#pragma unroll
              for (int x = 0; x < QT; ++x)
#pragma unroll
                for (int e = 0; e < 4 * kT; ++e) {
                  const float y = fmaf(-slope[x], fabsf(place[x] + (near - (float)(E0 + e))), s[x][e / 4][e % 4]) - base[x];
                  s[x][e / 4][e % 4] = y;
                  top[x] = fmaxf(top[x], y);
                }
            }
#pragma unroll
            for (int x = 0; x < QT; ++x) {
              if (__any(top[x] > (m[x] == -INFINITY ? -INFINITY : kRise))) {
                const float by = raise(m[x], column_max(top[x]));
#pragma unroll
                for (int t = 0; t < kT; ++t) s[x][t] -= by;
                lower(x, by);
              }
            }
            uint32_t p[QT][kT][2];
            const float v_step = kCodes ? vs.x : 1.0f, v_off = kCodes ? off_of(vs) : 0.0f, v_inv = kCodes ? inv_of(vs) : 0.0f;
#pragma unroll
            for (int x = 0; x < QT; ++x) {
              float w[4 * kT];
#pragma unroll
              for (int e = 0; e < 4 * kT; ++e) {
                w[e] = __builtin_amdgcn_exp2f(s[x][e / 4][e % 4]);
              }
              if constexpr (kCodes) {
                if (__any(is_tiny(vs))) {
                  const float alone = is_tiny(vs) ? vs.y : 0.0f, one = is_tiny(vs) ? 1.0f : 0.0f;
                  each<4 * kT>([&](auto e) {
                    c_run[x] += w[decltype(e)::value] * row_bcast<E0 + decltype(e)::value>(alone);
                    l_run[x] += w[decltype(e)::value] * row_bcast<E0 + decltype(e)::value>(one);
                  });
                }
                each<4 * kT>([&](auto e) { w[decltype(e)::value] *= row_bcast<E0 + decltype(e)::value>(v_step); });
              }
#pragma unroll
              for (int t = 0; t < kT; ++t) pack_weights<BITS>(w + 4 * t, p[x][t]);
              if constexpr (kCodes) each<4 * kT>([&](auto e) {
                constexpr int E = decltype(e)::value;
                const uint32_t u = p[x][E / 4][place_of(E) / 2];
                const float rounded = __uint_as_float(place_of(E) % 2 ? u & 0xffff0000u : u << 16);
                c_run[x] += rounded * row_bcast<E0 + E>(v_off);
                l_run[x] += rounded * row_bcast<E0 + E>(v_inv);
              });
            }
#pragma unroll
            for (int h = 0; h < kT / 2; ++h) {
              bf16x8 pf[QT];
#pragma unroll
              for (int x = 0; x < QT; ++x) pf[x] = as_frag(p[x][2 * h][0], p[x][2 * h][1], p[x][2 * h + 1][0], p[x][2 * h + 1][1]);
#pragma unroll
              for (int d = 0; d < kTiles; ++d) {
                const bf16x8 vv = value_operand<BITS, W>(vf, d, T / 2 + h);
#pragma unroll
                for (int x = 0; x < QT; ++x) o[x][d] = mfma(vv, pf[x], o[x][d]);
                if (d % 2) __builtin_amdgcn_sched_barrier(0);
              }
              if constexpr (!kCodes) {
#pragma unroll
                for (int x = 0; x < QT; ++x) l_acc[x] = mfma(ones, pf[x], l_acc[x]);
              }
            }
          });
          if (hole) later |= bit;
          if (more) fetch_values(kb + kStep, ahead);
          hole = ahead.missing() || (KIND != kMasks && kb + kStep < low_all);
          ahead = pages_of(kb + 2 * kStep);
        }
      }

      // Then what was put off, and the blocks of new tokens: one at a time, with every case.
      number();
      for (bool fetched = kThrough && started && kb < run_end; later || kb < run_end; fetched = false) {
        int64_t at = kb;
        if (later && !fetched) {
          at = run + wave * kBlock + (int64_t)__builtin_ctzll(later) * kStep;
          later &= later - 1;
        } else {
          kb += kStep;
        }
        const Pages p = pages_of(at);
        if (!fetched) {
          fetch_keys(at, p);
          fetch_values(at, p);
        }
        const int64_t pos = at + g * 16, j0 = pos - sq.prefix;
        uint32_t exists = 0;
        if (pos < end && p.pick(g) >= 0) exists = end - pos >= 16 ? 0xffffu : (1u << (int)(end - pos)) - 1;
        bool odd = false;
        if constexpr (!kCodes) {
          // Slots that hold no token hold anything: zeros instead, for 0 * NaN is NaN.  Infinities and NaNs of new tokens are looked after below.
#pragma unroll
          for (int d = 0; d < F::kVTiles; ++d)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              vf.w[d][i] &= ((exists >> (2 * i)) & 1 ? 0xffffu : 0u) | ((exists >> (2 * i + 1)) & 1 ? 0xffff0000u : 0u);
              odd = odd || any_nonfinite(vf.w[d][i]);
            }
          odd = __any(odd);
        }
        const float k_step = kCodes ? ks.x * scale : scale, k_off = kCodes ? (ks.y - shifted<BITS>() * ks.x) * scale : 0.0f;
        const float v_step = kCodes ? vs.x : 1.0f, v_off = kCodes ? off_of(vs) : 0.0f, v_inv = kCodes ? inv_of(vs) : 0.0f;
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
          if (x) {                      // the operands made anew for the next 16 rows, not kept
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
              for (int i = 0; i < F::kWords; ++i) kf.w[t][i] = anew(kf.w[t][i]);
#pragma unroll
            for (int d = 0; d < F::kVTiles; ++d)
#pragma unroll
              for (int i = 0; i < F::kVWords; ++i) vf.w[d][i] = anew(vf.w[d][i]);
          }
          float w[16];
          float top = -INFINITY;
          const float base = m[x] == -INFINITY ? 0.0f : m[x];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < kOps; ++i) s = mfma(key_operand<BITS, W>(kf, t, i), qf[x][i], s);
#pragma unroll
            for (int r = 0; r < 4; ++r) w[4 * t + r] = s[r];
            __builtin_amdgcn_sched_barrier(0);
          }
          each<16>([&](auto e) {
            constexpr int E = decltype(e)::value;
            float y = w[E] * (kCodes ? row_bcast<E>(k_step) : k_step);
            if constexpr (kCodes) y += row_bcast<E>(k_off) * q_sum[x];
            if constexpr (KIND == kOptions) {
              if (cap != 0.0f) y = capped(y, cap, cap_in);
              y = fmaf(-slope[x], fabsf(place[x] + ((float)(sq.prefix - at) - (float)E)), y);
            }
            w[E] = (vis >> E) & 1 ? y - base : -INFINITY;
            top = fmaxf(top, w[E]);
          });
          const float by = raise(m[x], column_max(top));
          lower(x, by);
          uint32_t q[4][2];
#pragma unroll
          for (int e = 0; e < 16; ++e) w[e] = __builtin_amdgcn_exp2f(w[e] - by);
          if constexpr (kCodes) {        // (whatever pair the slot holds)
            if (__any(is_tiny(vs))) {
              const float alone = is_tiny(vs) ? vs.y : 0.0f, one = is_tiny(vs) ? 1.0f : 0.0f;
              each<16>([&](auto e) {
                constexpr int E = decltype(e)::value;
                const float add = w[E] * row_bcast<E>(alone);
                c_run[x] += (vis >> E) & 1 ? add : 0.0f;
                l_run[x] += w[E] * row_bcast<E>(one);
              });
            }
            each<16>([&](auto e) {
              constexpr int E = decltype(e)::value;
              const float y = w[E] * row_bcast<E>(v_step);
              w[E] = (vis >> E) & 1 ? y : 0.0f;
            });
          }
#pragma unroll
          for (int t = 0; t < 4; ++t) pack_weights<BITS>(w + 4 * t, q[t]);
          if constexpr (kCodes) each<16>([&](auto e) {
            constexpr int E = decltype(e)::value;
            const uint32_t u = q[E / 4][place_of(E) / 2];
            const float rounded = __uint_as_float(place_of(E) % 2 ? u & 0xffff0000u : u << 16);
            const float add = rounded * row_bcast<E>(v_off), weight = rounded * row_bcast<E>(v_inv);
            c_run[x] += (vis >> E) & 1 ? add : 0.0f;
            l_run[x] += (vis >> E) & 1 ? weight : 0.0f;
          });
          if (!kCodes && odd) {
            // One token at a time, its values to the rows that see it.
            for (int e = 0; e < kBlock; ++e) {
              const int eg = e >> 4, bit = e & 15;
              uint32_t pw = 0;
#pragma unroll
              for (int i = 0; i < 8; ++i) pw = (bit >> 1) == i ? q[i / 2][i % 2] : pw;
              const float one = bf16_to_f32((bf16_bits)__shfl((int)(bit & 1 ? pw >> 16 : pw & 0xffffu), eg * 16 + col));
              const bool sees = (__shfl((int)vis, eg * 16 + col) >> bit) & 1;
#pragma unroll
              for (int d = 0; d < kTiles; ++d) {
                // its values in the result's entries d * 16 + 4 g + r, which lane 4 g + r of quarter eg holds
                uint32_t word = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) word = (bit >> 1) == i ? vf.w[d % F::kVTiles][i % F::kVWords] : word;
                const uint32_t h = bit & 1 ? word >> 16 : word & 0xffffu;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                  const uint32_t y = (uint32_t)__shfl((int)h, eg * 16 + g * 4 + r);
                  if (sees && (y & 0x7f80u) == 0x7f80u) o[x][d][r] += one * bf16_to_f32((bf16_bits)y);
                }
              }
            }
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const bf16x8 pf = as_frag(q[2 * h][0], q[2 * h][1], q[2 * h + 1][0], q[2 * h + 1][1]);
#pragma unroll
            for (int d = 0; d < kTiles; ++d) {
              u32x4 z = __builtin_bit_cast(u32x4, value_operand<BITS, W>(vf, d, h));
              if (!kCodes && odd) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  if ((z[j] & 0x7f80u) == 0x7f80u) z[j] &= 0xffff0000u;
                  if ((z[j] & 0x7f800000u) == 0x7f800000u) z[j] &= 0x0000ffffu;
                }
              }
              o[x][d] = mfma(__builtin_bit_cast(bf16x8, z), pf, o[x][d]);
              if (d % 2) __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (!kCodes) l_acc[x] = mfma(ones, pf, l_acc[x]);
          }
        }
      }
    }

    // A row's sums over the lanes that shared its keys, and the constant that belongs to every entry of its result.
    number();
    float l[QT];
#pragma unroll
    for (int x = 0; x < QT; ++x) {
      l[x] = kCodes ? column_sum(l_run[kCodes ? x : 0]) : l_acc[kCodes ? 0 : x][0];
      if constexpr (kCodes) {
        const float c = column_sum(c_run[x]);
#pragma unroll
        for (int d = 0; d < kTiles; ++d) o[x][d] += c;
      }
    }
    if constexpr (KIND != kMasks) {
#pragma unroll
      for (int x = 0; x < QT; ++x) {
        const int row = row0 + x * 16 + col;
        const int2 k = chunk_keys(a, sq, (uint32_t)(row < rows ? row : 0) / (uint32_t)a->group);
        if (k.x < k.y) continue;
        m[x] = -INFINITY;
        l[x] = 0.0f;
#pragma unroll
        for (int d = 0; d < kTiles; ++d) o[x][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      }
    }
    // Wavefronts 2 and 3 into 0 and 1, then 1 into 0.
#pragma unroll
    for (int half = kWaves / 2; half > 0; half /= 2) {
      if (wave >= half && wave < 2 * half) {
#pragma unroll
        for (int x = 0; x < QT; ++x) {
#pragma unroll
          for (int d = 0; d < kTiles; ++d) *reinterpret_cast<f32x4*>(s_o[wave - half][x * kTiles + d][lane]) = o[x][d];
          s_ml[wave - half][x][0][lane] = m[x];
          s_ml[wave - half][x][1][lane] = l[x];
        }
      }
      __syncthreads();
      if (wave < half) {
#pragma unroll
        for (int x = 0; x < QT; ++x) {
          const float m2 = s_ml[wave][x][0][lane], l2 = s_ml[wave][x][1][lane];
          const float m_new = fmaxf(m[x], m2);
          const float f1 = m[x] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[x] - m_new);
          const float f2 = m2 == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m2 - m_new);
          m[x] = m_new;
          l[x] = l[x] * f1 + l2 * f2;
#pragma unroll
          for (int d = 0; d < kTiles; ++d) o[x][d] = o[x][d] * f1 + *reinterpret_cast<const f32x4*>(s_o[wave][x * kTiles + d][lane]) * f2;
        }
      }
      __syncthreads();
    }
    if (wave) continue;

#pragma unroll
    for (int x = 0; x < QT; ++x) {
      const int row = row0 + x * 16 + col;
      if (row >= rows) continue;
      if (piece.whole) {
#pragma unroll
        for (int d = 0; d < kTiles; ++d) store_row4(a, sq, head, row, d * 16 + g * 4, o[x][d], l[x]);
      } else {
        const int64_t at = part_at(a, head, row_tile, piece.slot, row - row0);
#pragma unroll
        for (int d = 0; d < kTiles; ++d) *reinterpret_cast<f32x4*>(a->part + at * W + d * 16 + g * 4) = o[x][d];
        if (g == 0) a->part_ml[at] = make_float2(m[x], l[x]);
      }
    }
  }
}

}  // namespace

}  // namespace tree
}  // namespace conqur
