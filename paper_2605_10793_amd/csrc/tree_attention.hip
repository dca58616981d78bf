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
#include "tree_attention.h"

using namespace conqur;
using namespace conqur::tree;

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
template <int BITS, int W, int QT, bool ONE_PAGE>
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

  const int head = blockIdx.x / a->row_tiles, row_tile = blockIdx.x % a->row_tiles;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int row0 = row_tile * 16 * QT;
  const bf16x8 ones = as_frag(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);      // a row of the sums of the weights as they are rounded
  Pieces piece;
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
    const int64_t begin = (int64_t)piece.first * kBlock, end = (int64_t)piece.last * kBlock < sq.length ? (int64_t)piece.last * kBlock : sq.length;

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
    const float scale = a->scale_log2;
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
    auto place = [](int e) { return BITS == 4 ? (e % 4 == 1 ? 2 : e % 4 == 2 ? 1 : e % 4) : e % 4; };      // where pack_weights puts weight e of four

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

    const int64_t old_end = sq.prefix < end ? sq.prefix : end;
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
        bool hole = ahead.missing();
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
                const float y = fmaf(s[x][E / 4][E % 4], step, kCodes ? fmaf(off, q_sum[x], -base[x]) : -base[x]);
                s[x][E / 4][E % 4] = y;
                top[x] = fmaxf(top[x], y);
              }
            });
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
                const uint32_t u = p[x][E / 4][place(E) / 2];
                const float rounded = __uint_as_float(place(E) % 2 ? u & 0xffff0000u : u << 16);
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
          hole = ahead.missing();
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
          const int row = row0 + x * 16 + col, node = row / a->group;
          uint64_t seen = 0;
          if (row < rows) seen = a->mask ? a->mask[sq.first + node] : (2ull << node) - 1;
          if (sq.count < 64) seen &= (1ull << sq.count) - 1;
          uint32_t vis;
          if (j0 >= 0)
            vis = j0 < 64 ? (uint32_t)(seen >> j0) : 0;
          else
            vis = j0 > -16 ? (uint32_t)(seen << -j0) | ((1u << -j0) - 1) : 0xffffu;
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
            const uint32_t u = q[E / 4][place(E) / 2];
            const float rounded = __uint_as_float(place(E) % 2 ? u & 0xffff0000u : u << 16);
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
      k_tree<BITS, W, 1, true><<<grid, 64 * kWaves, 0, s>>>(a);
    else if (p.qt == 1)
      k_tree<BITS, W, 1, false><<<grid, 64 * kWaves, 0, s>>>(a);
    else if (one_page)
      k_tree<BITS, W, kMostTiles, true><<<grid, 64 * kWaves, 0, s>>>(a);
    else
      k_tree<BITS, W, kMostTiles, false><<<grid, 64 * kWaves, 0, s>>>(a);
    e = hipGetLastError();
  }
  if (e != hipSuccess || p.splits <= 1) return e;
  const int64_t rows = (int64_t)a.max_query * a.group * a.cache.heads;
  if (p.wide)
    k_tree_join_tiles<W><<<dim3((a.max_query * a.group + 15) / 16, a.cache.heads, a.batch.sequences), W * 2, 0, s>>>(a);
  // A wavefront a row, or four where there are few rows and they have many pieces (one sequence of 30000 tokens: 33.3 us with four, 40.5 with one;
  // 16 of 2000 to 9000 tokens, 16 rows a head: 39.8 with one, 42.6 with four).
  else if (p.splits <= 64 && p.splits <= 8 * (int64_t)a.batch.sequences)
    k_tree_join<W, 1><<<dim3((uint32_t)((rows + 3) / 4), a.batch.sequences), 256, 0, s>>>(a);
  else
    k_tree_join<W, 4><<<dim3((uint32_t)rows, a.batch.sequences), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

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
  TreeArgs a;
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
