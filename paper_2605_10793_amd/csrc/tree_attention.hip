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

template <int BITS, int W>
__device__ __forceinline__ void load_keys(Keys<BITS, W>& k, const unsigned char* p) {    // p: row of the lane's first key
  using F = Format<BITS, W>;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const unsigned char* r = p + t * 4 * F::kRow;
    if constexpr (F::kWords >= 4) {
#pragma unroll
      for (int i = 0; i < F::kWords / 4; ++i) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(r + i * 64);
#pragma unroll
        for (int j = 0; j < 4; ++j) k.w[t][4 * i + j] = x[j];
      }
    } else {
      const u32x2 x = *reinterpret_cast<const u32x2*>(r);
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
template <int BITS, int W>
__device__ __forceinline__ void load_values(Values<BITS, W>& v, const unsigned char* p, int pitch) {   // p: the lane's row of the first tile
  using F = Format<BITS, W>;
#pragma unroll
  for (int t = 0; t < F::kVTiles; ++t)
#pragma unroll
    for (int i = 0; i < F::kVSize; ++i) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(p + (int64_t)t * 16 * pitch + i * 16);
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

template <int BITS, int W, int QT>
__global__ void __launch_bounds__(64 * kWaves, QT > 1 ? 1 : 2) k_tree(const TreeArgs a) {
  using F = Format<BITS, W>;
  constexpr int kOps = W / 32;            // operands of the first product
  constexpr int kTiles = W / 16;          // tiles of the result
  constexpr bool kCodes = BITS != 16;
  // The wavefronts' results meet here at the end: two wavefronts' at a time.
  __shared__ __attribute__((aligned(16))) float s_o[2][QT * kTiles][64][4];
  __shared__ float s_ml[2][QT][2][64];

  const int head = blockIdx.x / a.row_tiles, row_tile = blockIdx.x % a.row_tiles;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int row0 = row_tile * 16 * QT;
  Pieces piece;
  for (bool first = true; piece.next(a, row0, threadIdx.x & 63, first); first = false) {
  int lane, col, g;
  auto number = [&] {
    lane = anew(threadIdx.x & 63);
    col = lane & 15;
    g = lane >> 4;
  };
  number();
  const int b = piece.b;
  const Sequence sq = sequence_of(a, b);
  const int rows = sq.count * a.group;
  const int64_t begin = (int64_t)piece.first * kBlock, end = (int64_t)piece.last * kBlock < sq.length ? (int64_t)piece.last * kBlock : sq.length;

  // Queries: operand i of column `col`, and what the row sees among the new tokens.
  bf16x8 qf[QT][kOps];
  float q_sum[QT];
  uint64_t seen[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int row = row0 + t * 16 + col;
    const bool here = row < rows;
    const int node = here ? row / a.group : 0;
    const bf16_bits* p = a.q + (sq.first + node) * a.q_ts + (int64_t)(head * a.group + (here ? row % a.group : 0)) * a.q_hs;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kOps; ++i) {
      bf16_bits e[8];
      const int base = entry_of<BITS, W>(i, g, 0);
      if (a.q_wide) {
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
    uint64_t m = 0;
    if (here) m = a.mask ? a.mask[sq.first + node] : (2ull << node) - 1;
    if (sq.count < 64) m &= (1ull << sq.count) - 1;
    seen[t] = m;
  }

  f32x4 o[QT][kTiles];
  float m_run[QT], l_run[QT], c_run[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
#pragma unroll
    for (int d = 0; d < kTiles; ++d) o[t][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    m_run[t] = -INFINITY;
    l_run[t] = c_run[t] = 0.0f;
  }

  const int page_tokens = (int)a.cache.page_tokens;
  const int page_shift = 31 - __builtin_clz(page_tokens);
  const int32_t* table = a.batch.table + (int64_t)b * a.batch.table_stride;
  const int64_t heads = a.cache.heads;
  // Page of a group of 16 tokens from `pos` on, -1 where there is none; reads stay in the pool either way.
  auto page_of = [&](int64_t pos) {
    if (pos >= end) return -1;
    const int32_t p = table[pos >> page_shift];
    return p >= 0 && (uint64_t)p < a.cache.pages ? p : -1;
  };
  const unsigned char* kp = static_cast<const unsigned char*>(a.cache.k);
  const unsigned char* vp = static_cast<const unsigned char*>(a.cache.v);
  const int k_group = (col >> 2) * 16, v_group = g * 16;      // first of the 16 keys that the lane's A rows (its scores and V) come from
  const int v_pitch = page_tokens * F::kVSize;

  Keys<BITS, W> kf;
  Values<BITS, W> vf;
  float2 ks, vs;                      // the pair of key `lane` of the block
  int32_t page_k = 0, page_v = 0;     // of the block that the operands hold
  auto fetch_keys = [&](int64_t kb, int32_t pk, int32_t pv) {
    const int64_t slot = ((kb + k_group) & (page_tokens - 1)) + (col & 3);
    load_keys<BITS, W>(kf, kp + (((int64_t)(pk < 0 ? 0 : pk) * heads + head) * page_tokens + slot) * F::kRow + g * (F::kWords >= 4 ? 16 : 8));
    if constexpr (kCodes) {
      const int64_t at = ((int64_t)(pv < 0 ? 0 : pv) * heads + head) * page_tokens + ((kb + lane) & (page_tokens - 1));
      ks = reinterpret_cast<const float2*>(a.cache.k_scale)[at];
    }
  };
  auto fetch_values = [&](int64_t kb, int32_t pv) {
    const int64_t base = ((int64_t)(pv < 0 ? 0 : pv) * heads + head);
    load_values<BITS, W>(vf, vp + (base * F::kVRows + col) * v_pitch + ((kb + v_group) & (page_tokens - 1)) * F::kVSize, v_pitch);
    if constexpr (kCodes) vs = reinterpret_cast<const float2*>(a.cache.v_scale)[base * page_tokens + ((kb + lane) & (page_tokens - 1))];
  };

  int64_t kb = begin + wave * kBlock;
  int32_t next_k = -1, next_v = -1;
  if (kb < end) {
    page_k = page_of(kb + k_group);
    page_v = page_of(kb + v_group);
    fetch_keys(kb, page_k, page_v);
    fetch_values(kb, page_v);
    next_k = page_of(kb + kBlock * kWaves + k_group);
    next_v = page_of(kb + kBlock * kWaves + v_group);
  }
  for (; kb < end; kb += kBlock * kWaves) {
    const bool more = kb + kBlock * kWaves < end;
    const int32_t after_k = more ? page_of(kb + 2 * kBlock * kWaves + k_group) : -1, after_v = more ? page_of(kb + 2 * kBlock * kWaves + v_group) : -1;

    f32x4 s[QT][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int x = 0; x < QT; ++x) s[x][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < kOps; ++i) {
        const bf16x8 kk = key_operand<BITS, W>(kf, t, i);
#pragma unroll
        for (int x = 0; x < QT; ++x) s[x][t] = mfma(kk, qf[x][i], s[x][t]);
      }
    }
    // Keys that some row does not see: of the new tokens, behind the end, or of no page.
    const bool partial = kb + kBlock > sq.prefix || kb + kBlock > end || __any(page_v < 0);
    const float2 ks_now = ks;
    if (more) fetch_keys(kb + kBlock * kWaves, next_k, next_v);

    uint32_t vis[QT];
    if (partial) {
      const int64_t pos = kb + v_group;
      uint32_t exists = 0;
      if (page_v >= 0 && pos < end) exists = end - pos >= 16 ? 0xffffu : (1u << (int)(end - pos)) - 1;
      const int64_t j0 = pos - sq.prefix;
#pragma unroll
      for (int x = 0; x < QT; ++x) {
        uint32_t v;
        if (j0 >= 0)
          v = j0 < 64 ? (uint32_t)(seen[x] >> j0) : 0;
        else
          v = j0 > -16 ? (uint32_t)(seen[x] << -j0) | ((1u << -j0) - 1) : 0xffffu;
        vis[x] = v & exists;
      }
      if constexpr (!kCodes) {
        // Slots that hold no token yet hold anything: zeros instead, for 0 * NaN is NaN.
#pragma unroll
        for (int d = 0; d < F::kVTiles; ++d)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const uint32_t keep = ((exists >> (2 * i)) & 1 ? 0xffffu : 0u) | ((exists >> (2 * i + 1)) & 1 ? 0xffff0000u : 0u);
            vf.w[d][i] &= keep;
          }
      }
    }

    // A constant row has step 0 and code 0: its weight goes in as it is, and its offset with it.
    const float v_step = !kCodes || vs.x == 0.0f ? 1.0f : vs.x;
    // A step so small that weights times it leave the range: such a token's weight is added to the sum as it is.
    const bool tiny = kCodes && fabsf(v_step) < 1e-30f;
    const float v_inv = tiny ? 0.0f : 1.0f / v_step;
    const float v_off = kCodes ? vs.y / v_step - shifted<BITS>() : 0.0f;
    uint32_t p[QT][4][2];
#pragma unroll
    for (int x = 0; x < QT; ++x) {
      float v[16];
      float k_off = 0.0f;
      if constexpr (kCodes) k_off = (ks_now.y - shifted<BITS>() * ks_now.x) * a.scale_log2;
      const float k_step = kCodes ? ks_now.x * a.scale_log2 : 0.0f;
      each<16>([&](auto e) {
        constexpr int E = decltype(e)::value;
        const float acc = s[x][E / 4][E % 4];
        if constexpr (kCodes)
          v[E] = row_bcast<E>(k_step) * acc + row_bcast<E>(k_off) * q_sum[x];
        else
          v[E] = acc * a.scale_log2;
      });
      if (partial) {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = (vis[x] >> e) & 1 ? v[e] : -INFINITY;
      }
      float top = v[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top = fmaxf(top, v[e]);
      top = column_max(top);
      if (__any(top > m_run[x])) {
        const float m_new = fmaxf(m_run[x], top);
        const float f = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m_run[x] - m_new);
        m_run[x] = m_new;
        l_run[x] *= f;
        c_run[x] *= f;
#pragma unroll
        for (int d = 0; d < kTiles; ++d) o[x][d] *= f;
      }
      const float m = m_run[x] == -INFINITY ? 0.0f : m_run[x];
      if (__any(tiny)) each<16>([&](auto e) {
        constexpr int E = decltype(e)::value;
        l_run[x] += row_bcast<E>(tiny ? 1.0f : 0.0f) * __builtin_amdgcn_exp2f(v[E] - m);
      });
      each<16>([&](auto e) {
        constexpr int E = decltype(e)::value;
        const float w = __builtin_amdgcn_exp2f(v[E] - m);
        if constexpr (kCodes) {
          v[E] = w * row_bcast<E>(v_step);
          if (partial && !((vis[x] >> E) & 1)) v[E] = 0.0f;      // (whatever pair the slot holds)
        } else {
          l_run[x] += w;
          v[E] = w;
        }
      });
#pragma unroll
      for (int t = 0; t < 4; ++t) pack_weights<BITS>(v + 4 * t, p[x][t]);
      if constexpr (kCodes) {
        each<16>([&](auto e) {
          constexpr int E = decltype(e)::value;
          constexpr int kAt = BITS == 4 ? (E % 4 == 1 ? 2 : E % 4 == 2 ? 1 : E % 4) : E % 4;     // where pack_weights put it
          const uint32_t u = p[x][E / 4][kAt / 2];
          const float w = __uint_as_float(kAt % 2 ? u & 0xffff0000u : u << 16);
          const float c = w * row_bcast<E>(v_off), n = w * row_bcast<E>(v_inv);
          const bool out = partial && !((vis[x] >> E) & 1);
          c_run[x] += out ? 0.0f : c;
          l_run[x] += out ? 0.0f : n;
        });
      }
    }

    if constexpr (!kCodes) {
      // An infinity or a NaN among the values of new tokens is met by the rows that see it only.
      if (partial) {
        bool odd = false;
#pragma unroll
        for (int d = 0; d < F::kVTiles; ++d)
#pragma unroll
          for (int i = 0; i < 8; ++i) odd = odd || any_nonfinite(vf.w[d][i]);
        if (__any(odd)) {
          // One token at a time: its weight alone, then the product with its values alone, in the rows that see it.
          for (int e = 0; e < kBlock; ++e) {
            const int eg = e >> 4, bit = e & 15;
            bool bad = false;
#pragma unroll
            for (int d = 0; d < F::kVTiles; ++d)
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const uint32_t h = bit & 1 ? vf.w[d][i] >> 16 : vf.w[d][i] & 0xffffu;
                bad = bad || (g == eg && (bit >> 1) == i && (h & 0x7f80u) == 0x7f80u);
              }
            if (!__any(bad)) continue;
#pragma unroll
            for (int d = 0; d < kTiles; ++d) {
              // value of this token in the result's entries d * 16 + 4 g + r, which lane (4 g + r) of quarter eg holds
              uint32_t word = 0;
#pragma unroll
              for (int i = 0; i < 8; ++i) word = (bit >> 1) == i ? vf.w[d][i] : word;
              const uint32_t h = bit & 1 ? word >> 16 : word & 0xffffu;
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const uint32_t y = (uint32_t)__shfl((int)h, eg * 16 + g * 4 + r);
                const bool inf_or_nan = (y & 0x7f80u) == 0x7f80u;
#pragma unroll
                for (int x = 0; x < QT; ++x) {
                  uint32_t pw = 0;
#pragma unroll
                  for (int i = 0; i < 8; ++i) pw = (bit >> 1) == i ? p[x][i / 2][i % 2] : pw;
                  const uint32_t ph = (uint32_t)__shfl((int)(bit & 1 ? pw >> 16 : pw & 0xffffu), eg * 16 + col);
                  const uint32_t vb = (uint32_t)__shfl((int)vis[x], eg * 16 + col);
                  if (inf_or_nan && ((vb >> bit) & 1)) o[x][d][r] += bf16_to_f32((bf16_bits)ph) * bf16_to_f32((bf16_bits)y);
                }
              }
            }
          }
#pragma unroll
          for (int d = 0; d < F::kVTiles; ++d)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              uint32_t y = vf.w[d][i];
              if ((y & 0x7f80u) == 0x7f80u) y &= 0xffff0000u;
              if ((y & 0x7f800000u) == 0x7f800000u) y &= 0x0000ffffu;
              vf.w[d][i] = y;
            }
        }
      }
    }

#pragma unroll
    for (int m = 0; m < 2; ++m) {
#pragma unroll
      for (int d = 0; d < kTiles; ++d) {
        const bf16x8 vv = value_operand<BITS, W>(vf, d, m);
#pragma unroll
        for (int x = 0; x < QT; ++x) o[x][d] = mfma(vv, as_frag(p[x][2 * m][0], p[x][2 * m][1], p[x][2 * m + 1][0], p[x][2 * m + 1][1]), o[x][d]);
      }
    }
    if (more) fetch_values(kb + kBlock * kWaves, next_v);
    page_k = next_k;
    page_v = next_v;
    next_k = after_k;
    next_v = after_v;
  }

  number();
  // A row's sums over the lanes that shared its keys; the constant that belongs to every entry of the result.
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    l_run[x] = column_sum(l_run[x]);
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
        s_ml[wave - half][x][0][lane] = m_run[x];
        s_ml[wave - half][x][1][lane] = l_run[x];
      }
    }
    __syncthreads();
    if (wave < half) {
#pragma unroll
      for (int x = 0; x < QT; ++x) {
        const float m2 = s_ml[wave][x][0][lane], l2 = s_ml[wave][x][1][lane];
        const float m_new = fmaxf(m_run[x], m2);
        const float f1 = m_run[x] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_run[x] - m_new);
        const float f2 = m2 == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m2 - m_new);
        m_run[x] = m_new;
        l_run[x] = l_run[x] * f1 + l2 * f2;
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
      for (int d = 0; d < kTiles; ++d) store_row4(a, sq, head, row, d * 16 + g * 4, o[x][d], l_run[x]);
    } else {
      const int64_t at = part_at(a, head, row_tile, piece.slot, row - row0);
#pragma unroll
      for (int d = 0; d < kTiles; ++d) *reinterpret_cast<f32x4*>(a.part + at * W + d * 16 + g * 4) = o[x][d];
      if (g == 0) a.part_ml[at] = make_float2(m_run[x], l_run[x]);
    }
  }
  }
}

// Joins a row's pieces.  WAVES = 1: a wavefront a row, for up to 64 pieces; 4: a workgroup a row, for up to 256.  W / 4
// lanes read a piece's result as 16-byte vectors, 256 / W pieces at a time, and the first ones are under way before the maxima are.
template <int W, int WAVES>
__global__ void __launch_bounds__(256) k_tree_join(const TreeArgs a) {
  constexpr int kLanes = W / 4, kAt = 64 / kLanes;      // lanes of a piece, pieces of a wavefront at a time
  constexpr int kFirst = 4;                             // vectors a lane takes ahead
  __shared__ float s_f[256];
  __shared__ float s_red[2][4];
  __shared__ __attribute__((aligned(16))) float s_o[4][W];

  const int b = blockIdx.y;
  const Sequence sq = sequence_of(a, b);
  const int64_t heads = a.cache.heads;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t id = WAVES == 1 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x;
  const int row = (int)(id / heads), head = (int)(id % heads);
  if (row >= sq.count * a.group) return;
  const int row_tile = row / a.tile_rows;
  const Layout layout(a, row_tile * a.tile_rows, lane);
  int from = 0, to = 0;
  layout.range(b, &from, &to);
  const int p0 = from / layout.each, chunks = (to - 1) / layout.each - p0 + 1;
  if (chunks <= 1) return;
  // the first piece may be its workgroup's last, the others are their workgroups' first
  const int slot0 = 2 * p0 + (from > p0 * layout.each);
  auto at = [&](int c) { return part_at(a, head, row_tile, c ? 2 * (p0 + c) : slot0, row - row_tile * a.tile_rows); };
  const int first = (WAVES == 1 ? 0 : wave * kAt) + lane / kLanes;
  constexpr int kNext = WAVES * kAt;
  const int entry = lane % kLanes * 4;

  f32x4 v[kFirst];
#pragma unroll
  for (int i = 0; i < kFirst; ++i)
    if (first + i * kNext < chunks) v[i] = *reinterpret_cast<const f32x4*>(a.part + at(first + i * kNext) * W + entry);
  const int mine = WAVES == 1 ? lane : (int)threadIdx.x;
  const float2 ml = mine < chunks ? a.part_ml[at(mine)] : make_float2(-INFINITY, 0.0f);
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
    if (c < chunks) add(*reinterpret_cast<const f32x4*>(a.part + at(c) * W + entry), w);
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
__global__ void __launch_bounds__(W * 2) k_tree_join_tiles(const TreeArgs a) {
  const int b = blockIdx.z, head = blockIdx.y, row0 = blockIdx.x * 16;
  const Sequence sq = sequence_of(a, b);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
  if (row0 >= sq.count * a.group) return;
  const int row_tile = row0 / a.tile_rows, in_tile = row0 - row_tile * a.tile_rows;
  const Layout layout(a, row_tile * a.tile_rows, lane);
  int from = 0, to = 0;
  layout.range(b, &from, &to);
  const int p0 = from / layout.each, pieces = (to - 1) / layout.each - p0 + 1;
  if (pieces <= 1) return;
  auto at = [&](int c) { return part_at(a, head, row_tile, c ? 2 * (p0 + c) : 2 * p0 + (from > p0 * layout.each), in_tile); };

  float m = -INFINITY;
#pragma unroll 4
  for (int c = 0; c < pieces; ++c) m = fmaxf(m, a.part_ml[at(c) + col].x);
  f32x4 o[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
  float l = 0.0f;
#pragma unroll 4
  for (int c = 0; c < pieces; ++c) {
    const float2 ml = a.part_ml[at(c) + col];
    const float* const p = a.part + at(c) * W + wave * 512 + lane * 4;
    const f32x4 v0 = *reinterpret_cast<const f32x4*>(p), v1 = *reinterpret_cast<const f32x4*>(p + 256);
    const float f = ml.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml.x - m);
    l += ml.y * f;
    if (f != 0.0f) {
      o[0] += v0 * f;
      o[1] += v1 * f;
    }
  }
  if (row0 + col >= sq.count * a.group) return;
#pragma unroll
  for (int i = 0; i < 2; ++i) store_row4(a, sq, head, row0 + col, (wave * 2 + i) * 16 + g * 4, o[i], l);
}

constexpr int64_t kMaxStride = 1ll << 40;

struct Plan {
  bool wide;
  int qt, tile_rows, row_tiles, splits, min_blocks;
  int64_t context;
};

// How a call is cut: a cache head's rows into tiles, the sequences' blocks into runs.
Plan plan_of(const conqur_tree_call& c) {
  Plan p;
  const int64_t room = (int64_t)c.batch.table_columns * c.cache.page_tokens;
  p.context = (int64_t)(c.max_context < (uint64_t)room ? c.max_context : (uint64_t)room);
  const int rows = (int)(c.max_query * (c.q.heads / c.cache.heads));
  p.wide = rows > 32;
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
  p.splits = blocks <= kWaves || sequences > kMaxScan || sequences * groups >= 4096 ? 0 : (int)splits;
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
    if (p.qt == 1)
      k_tree<BITS, W, 1><<<grid, 64 * kWaves, 0, s>>>(a);
    else
      k_tree<BITS, W, 2><<<grid, 64 * kWaves, 0, s>>>(a);
    e = hipGetLastError();
  }
  if (e != hipSuccess || p.splits <= 1) return e;
  const int64_t rows = (int64_t)a.max_query * a.group * a.cache.heads;
  if (p.wide)
    k_tree_join_tiles<W><<<dim3((a.max_query * a.group + 15) / 16, a.cache.heads, a.batch.sequences), W * 2, 0, s>>>(a);
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
