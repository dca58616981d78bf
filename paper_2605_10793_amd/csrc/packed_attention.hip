// Attention of packed sequences over themselves.
//
//   u_ij = scale q_i k_j, s_ij = cap tanh(u_ij / cap) (cap 0: u_ij) - slope |i - j|, seen are max(0, first_i, i - window + 1) <= j < min(count, last_i)
//   o_i = sum_j e^(s_ij - m_i) v_j / sum_j e^(s_ij - m_i),  m_i = max_j s_ij,  lse_i = m_i + log sum_j e^(s_ij - m_i)
//
// in one pass over the keys, with running maxima and sums (in base 2).  The rows of a key head are its query heads times the tokens, token by token, so
// that a workgroup's 128 rows are few tokens whose keys nearly coincide.  Both products run transposed, S^T = K Q^T and O^T = V^T P^T (32x32x16 bf16 MFMA): a
// column is a row of the call, so that a lane holds scores of one row, the maximum needs one exchange, factors on O^T are the lane's own, and S^T leaves the
// first product as P^T has to enter the second: weights stay in registers.  64 keys and values at a time come to LDS without passing registers, a block
// (keys: two) ahead of the products; V is turned round as it is read from there.
//
// Bound by the matrix units' and the vector units' shares of a SIMD and by the clock that their load allows (the same calls over zeros take 0.85 of the time).
// So that a wavefront gives both work at once, a block's scores become weights between the products of the next block's scores, and those become scores between
// the products with V: 8 sequences of 2048 tokens, 32 and 8 heads of 128, 331 us for 348 (830 TFLOP/s over what is seen), one of 16384 at 1020 TFLOP/s.
// Eight wavefronts to a workgroup (348 us), more operands on their way from LDS (340 for 339) and a fourth wavefront to a SIMD where registers leave
// room for it (85.0 for 85.8) gave nothing.
#include "packed_attention.h"

namespace conqur {
namespace packed {

namespace {

template <int KS, int OPTIONS>
__global__ void __launch_bounds__(64 * kWaves, 2) k_packed(const PackedArgs) {
  using T = Tile<KS>;
  Args a = kernel_args();
  extern __shared__ __attribute__((aligned(1024))) unsigned char shared[];
  int* const s_bad = reinterpret_cast<int*>(shared + 4 * T::kBytes);          // of each buffer's values: whether they were not finite
  int* const s_odd = s_bad + 2 * kTile;                                       // whether any was
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5;
  const int head = blockIdx.x % a->heads;
  Item item;
  if (!item.find(a, blockIdx.x / a->heads, 7, a->group)) return;
  static_assert(kRows == 128, "");
  // The last rows, which see the most in a causal call, first.
  const int part = item.parts - 1 - item.part, group = a->group;
  const int rows = item.count * group;
  auto token_of = [&](int row) { return (int)((uint32_t)(row < rows ? row : rows - 1) / (uint32_t)group); };
  const int row = part * kRows + wave * 32 + (lane & 31), token = token_of(row);
  const int2 mine = keys_of(a, item, token);

  // Keys that any row of the workgroup sees, any of the wavefront, all of the wavefront, all of the workgroup.
  int begin, end, low, high, low_all, high_all, low_both, high_both;
  {
    auto none = [](int2 x) { return x.x >= x.y; };
    const bool empty = none(mine);
    low = wave_min(empty ? INT_MAX : mine.x);
    high = wave_max_int(mine.y);
    low_all = wave_max_int(empty ? INT_MAX : mine.x);
    high_all = wave_min(mine.y);
    const int2 x = keys_of(a, item, token_of(part * kRows + lane)), y = keys_of(a, item, token_of(part * kRows + 64 + lane));
    begin = wave_min(min(none(x) ? INT_MAX : x.x, none(y) ? INT_MAX : y.x));
    end = wave_max_int(max(x.y, y.y));
    low_both = wave_max_int(max(none(x) ? INT_MAX : x.x, none(y) ? INT_MAX : y.x));
    high_both = wave_min(min(x.y, y.y));
    if (part * kRows + wave * 32 >= rows) high = 0;
  }
  begin = begin / kTile * kTile;
  share_keys(&begin, &end, kTile);

  const int64_t row_token = item.first + token;
  const int q_head = head * group + (row < rows ? row : rows - 1) - token * group;
  bf16x8 qf[KS];
  load_rows<KS>(qf, a->q.data + row_token * a->q.ts + q_head * a->q.hs, h);

  const int k_stride = (int)(a->k.ts * 2), v_stride = (int)(a->v.ts * 2);
  const bf16_bits* const k0 = a->k.data + (int64_t)item.first * a->k.ts + head * a->k.hs;
  const bf16_bits* const v0 = a->v.data + (int64_t)item.first * a->v.ts + head * a->v.hs;
  const uint32_t lds = lds_of(shared);          // two tiles of keys, two of values
  auto send_keys = [&](int kb, int which) { send_tile<KS>(k0 + (int64_t)kb * a->k.ts, k_stride, item.count - kb, lds + which * T::kBytes, wave); };
  auto send_values = [&](int kb, int which) { send_tile<KS>(v0 + (int64_t)kb * a->v.ts, v_stride, item.count - kb, lds + (2 + which) * T::kBytes, wave); };

  f32x16 o[T::kTiles];
#pragma unroll
  for (int t = 0; t < T::kTiles; ++t) o[t] = f32x16{};
  float m = -INFINITY, l = 0.0f, top = -INFINITY;
  const float scale = a->scale_log2, cap = a->cap_log2, cap_in = a->cap_in, slope = OPTIONS & kBiased ? a->slopes[q_head] * kLog2e : 0.0f;
  const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
  float s[2][16];
  f32x16 next[2];          // scores of a block, less the maximum so far; products of the next
  // The wavefront's own blocks.
  const int from = max(begin, low / kTile * kTile), to_end = min(high, end);

  // A score of the block at kb from its product; the block's maximum, and what is not seen.
  auto score = [&](int kb, auto i) __attribute__((always_inline)) {
    constexpr int u = decltype(i)::value / 16, r = decltype(i)::value % 16;
    const float base = m == -INFINITY ? 0.0f : m;
    float x;
    if constexpr (OPTIONS & kCapped) {
      float none;
      x = capped(next[u][r], cap, cap_in, base, &none);
    } else {
      x = fmaf(next[u][r], scale, -base);
    }
    if constexpr (OPTIONS & kBiased) x = fmaf(-slope, fabsf((float)(token - kb - 4 * h) - (float)(32 * u + row_of(r, 0))), x);
    asm volatile("" : "+v"(x));
    s[u][r] = x;
  };
  auto finish = [&](int kb) __attribute__((always_inline)) {
    if (!(kb >= low_all && kb + kTile <= high_all)) {
      const int lo = mine.x - kb - 4 * h, hi = mine.y - kb - 4 * h;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[u][r] = 32 * u + row_of(r, 0) >= lo && 32 * u + row_of(r, 0) < hi ? s[u][r] : -INFINITY;
    }
    top = max17(s[1], max17(s[0], -INFINITY));
  };
  // A block's weights and results (NOW), and the next one's products (NEXT): the products of one run while the other's scores become weights, and the other way round.
  auto step = [&](int kb, int which, bool odd, auto now_, auto next_) __attribute__((always_inline)) {
    constexpr bool NOW = decltype(now_)::value, NEXT = decltype(next_)::value;
    if constexpr (NOW) {
      if (__any(top > (m == -INFINITY ? -INFINITY : kRise))) {
        top = halves(top, [](float x, float y) { return fmaxf(x, y); });
        const bool unset = m == -INFINITY;
        const float by = unset ? (top == -INFINITY ? 0.0f : top) : fmaxf(top, 0.0f);
        m = unset ? top : m + by;
        const float f = __builtin_amdgcn_exp2f(-fmaxf(by, 0.0f));          // (before the first score the sums are 0)
        l *= f;
#pragma unroll
        for (int t = 0; t < T::kTiles; ++t) o[t] *= f;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[u][r] -= by;
      }
    }
    const int here = lane_anew();
    // Weights rounded to bf16, as the second product takes them; the sum that divides takes them so, too.
    uint32_t p[2][8];
    auto weigh = [&](auto i) __attribute__((always_inline)) {
      constexpr int u = decltype(i)::value / 8, r = decltype(i)::value % 8;
      p[u][r] = f32x2_to_bf16x2(__builtin_amdgcn_exp2f(s[u][2 * r]), __builtin_amdgcn_exp2f(s[u][2 * r + 1]));
      l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, p[u][r]), ones, l, false);
    };
    if constexpr (NEXT) {
      const typename T::RowsAt keys(lds + (which ^ 1) * T::kBytes + T::row_at(here));
      next[0] = next[1] = f32x16{};
      in_turn<2 * KS>([&](auto i) { return keys.template get<decltype(i)::value % 2 * 32 * T::kPitch>(decltype(i)::value / 2); },
                         [&](auto i, bf16x8 f) {
                           constexpr int I = decltype(i)::value;
                           next[I % 2] = mfma32(f, qf[I / 2], next[I % 2]);
                           if constexpr (NOW) each_from<I * 16 / (2 * KS), (I + 1) * 16 / (2 * KS)>(weigh);
                         });
    } else {
      each<16>(weigh);
    }
    if constexpr (NOW) {
      const typename T::TurnedAt values(lds + (2 + which) * T::kBytes + T::turned_at(here));
      constexpr int N = 4 * T::kTiles;
      // Operand i of V: 16 keys, 32 entries.
      in_turn<N>(
          [&](auto i) {
            constexpr int I = decltype(i)::value, K = I / T::kTiles;
            return values.template get<K * 16 * T::kPitch>(I % T::kTiles);
          },
          [&](auto i, bf16x8 f) {
            constexpr int I = decltype(i)::value, K = I / T::kTiles;
            const uint32_t* w = &p[K / 2][K % 2 * 4];
            o[I % T::kTiles] = mfma32(f, frag_of(w[0], w[1], w[2], w[3]), o[I % T::kTiles]);
            if constexpr (NEXT) each_from<(I * 32 / N), ((I + 1) * 32 / N)>([&](auto j) __attribute__((always_inline)) { score(kb + kTile, j); });
          });
      if (odd) {
        for (int j = 0; j < kTile; ++j) {
          const int key = kb + j;
          if (!s_bad[which * kTile + j] || key >= item.count) continue;
          const bool see = key >= mine.x && key < mine.y;
          const bf16_bits* const from_v = v0 + (int64_t)key * a->v.ts + 4 * h;
#pragma unroll
          for (int t = 0; t < T::kTiles; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int entry = 32 * t + row_of(r, 0);
              const uint32_t x = entry < KS * 16 ? from_v[entry] : 0;
              o[t][r] += see && (x & 0x7f80u) == 0x7f80u ? __uint_as_float(x << 16) : 0.0f;
            }
        }
      }
    }
    if constexpr (NEXT) {
      if constexpr (!NOW) each<32>([&](auto j) __attribute__((always_inline)) { score(kb + kTile, j); });
      finish(kb + kTile);
    }
  };

  // What all wavefronts do at a block: wait for its values and the next keys, send for those behind.  Values that are not finite must not meet rows that do not see
  // them, for 0 * NaN is NaN: where some rows of the workgroup do not see all of the block they become zeros, and are added by themselves to the rows that do.
  auto arrive = [&](int kb, int which) __attribute__((always_inline)) {
    wait_loads<0>();
    pipeline_barrier();
    if (kb + kTile < end) send_values(kb + kTile, which ^ 1);
    if (kb + 2 * kTile < end) send_keys(kb + 2 * kTile, which);
    if (kb >= low_both && kb + kTile <= high_both) return false;
    const int me = lane_anew();
    const bool bad = clear_nonfinite<KS, kTile / kWaves>(lds + (2 + which) * T::kBytes, wave, me);
    if (bad) *s_odd = 1;
    if ((me & 3) == 0) s_bad[which * kTile + wave * 16 + (me >> 2)] = bad;
    pipeline_barrier();
    return *(volatile int*)s_odd != 0;
  };
  if (threadIdx.x == 0) *s_odd = 0;
  int which = 0, kb = begin;
  if (begin < end) {
    send_keys(begin, 0);
    send_values(begin, 0);
    if (begin + kTile < end) {
      send_keys(begin + kTile, 1);
      wait_loads<2 * T::kLoads>();
    } else {
      wait_loads<T::kLoads>();
    }
    pipeline_barrier();
  }
  if (from < to_end) {
    for (; kb < from; kb += kTile, which ^= 1) arrive(kb, which);
    step(kb - kTile, which ^ 1, false, std::false_type{}, std::true_type{});
    for (; kb + kTile < to_end; kb += kTile, which ^= 1) {
      const bool odd = arrive(kb, which);
      step(kb, which, odd, std::true_type{}, std::true_type{});
    }
    const bool odd = arrive(kb, which);
    step(kb, which, odd, std::true_type{}, std::false_type{});
    kb += kTile, which ^= 1;
  }
  for (; kb < end; kb += kTile, which ^= 1) arrive(kb, which);

  a = kernel_args();
  l = halves(l, [](float x, float y) { return x + y; });
  if (gridDim.y > 1) {
    f32x4* const to = shared_of<4 * T::kTiles>(a, (int)blockIdx.y, wave);
#pragma unroll
    for (int t = 0; t < T::kTiles; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) to[(t * 4 + r) * 64] = f32x4{o[t][4 * r], o[t][4 * r + 1], o[t][4 * r + 2], o[t][4 * r + 3]};
    if (h == 0) *shared_row_of(a, (int)blockIdx.y, wave * 32 + lane) = make_float4(m, l, 0.0f, 0.0f);
    return;
  }
  if (row >= rows) return;
  // Nothing seen, or every score -inf: zeros.
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  bf16_bits* const to = a->out.data + row_token * a->out.ts + q_head * a->out.hs + 4 * h;
  store_row<KS>(to, o, inv, wide8(a->out.data, a->out.ts, a->out.hs));
  if (a->lse && h == 0) a->lse[row_token * (a->heads * group) + q_head] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * (1.0f / kLog2e);
}

// What workgroups that share keys made, joined, for 32 entries of a row (blockIdx.y).
template <int KS>
__global__ void __launch_bounds__(64 * kWaves) k_packed_join(const PackedArgs) {
  using T = Tile<KS>;
  const Args a = kernel_args();
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5, t = blockIdx.y;
  const int head = blockIdx.x % a->heads, group = a->group;
  Item item;
  if (!item.find(a, blockIdx.x / a->heads, 7, group)) return;
  const int row = (item.parts - 1 - item.part) * kRows + wave * 32 + (lane & 31);
  if (row >= item.count * group) return;
  float top = -INFINITY, l = 0.0f;
  for (int i = 0; i < a->splits; ++i) top = fmaxf(top, shared_row_of(a, i, wave * 32 + (lane & 31))->x);
  f32x16 o = {};
  for (int i = 0; i < a->splits; ++i) {
    const float4 x = *shared_row_of(a, i, wave * 32 + (lane & 31));
    const float by = x.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(x.x - top);
    const f32x4* const from = shared_of<4 * T::kTiles>(a, i, wave) + t * 4 * 64;
    l = fmaf(x.y, by, l);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const f32x4 y = from[r * 64];
#pragma unroll
      for (int j = 0; j < 4; ++j) o[4 * r + j] = fmaf(y[j], by, o[4 * r + j]);
    }
  }
  const int token = (int)((uint32_t)row / (uint32_t)group), q_head = head * group + row - token * group;
  const int64_t row_token = item.first + token;
  store_tile<KS>(a->out.data + row_token * a->out.ts + q_head * a->out.hs + 4 * h, t, o, l == 0.0f ? 0.0f : 1.0f / l, wide8(a->out.data, a->out.ts, a->out.hs));
  if (a->lse && h == 0 && t == 0) a->lse[row_token * (a->heads * group) + q_head] = l == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * (1.0f / kLog2e);
}

template <int KS, int OPTIONS>
hipError_t launch(const PackedArgs& a, hipStream_t s) {
  constexpr int kShared = 4 * Tile<KS>::kBytes + 2 * kTile * 4 + 16;
  static PerDeviceOnce once;
  const hipError_t e = once.run([] { return hipFuncSetAttribute(reinterpret_cast<const void*>(k_packed<KS, OPTIONS>), hipFuncAttributeMaxDynamicSharedMemorySize, kShared); });
  if (e != hipSuccess) return e;
  const uint32_t workgroups = (uint32_t)(row_items(a) * a.heads);
  k_packed<KS, OPTIONS><<<dim3(workgroups, (uint32_t)a.splits), 64 * kWaves, kShared, s>>>(a);
  const hipError_t x = hipGetLastError();
  if (x != hipSuccess || a.splits == 1) return x;
  k_packed_join<KS><<<dim3(workgroups, Tile<KS>::kTiles), 64 * kWaves, 0, s>>>(a);
  return hipGetLastError();
}

template <int KS>
hipError_t launch(const PackedArgs& a, hipStream_t s) {
  if (a.cap_log2 != 0.0f) return a.slopes ? launch<KS, kBiased | kCapped>(a, s) : launch<KS, kCapped>(a, s);
  return a.slopes ? launch<KS, kBiased>(a, s) : launch<KS, 0>(a, s);
}

}  // namespace

hipError_t launch_forward(const PackedArgs& a, hipStream_t s) {
  switch (a.width) {
    case 32: return launch<2>(a, s);
    case 64: return launch<4>(a, s);
    case 80: return launch<5>(a, s);
    case 96: return launch<6>(a, s);
    default: return launch<8>(a, s);
  }
}

namespace {

// Rows that the kernels cannot read as they lie, laid out side by side.
__global__ void __launch_bounds__(256) k_lay(Rows from, bf16_bits* to, int64_t tokens, int heads, int width) {
  const int64_t n = tokens * heads * width;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int e = (int)(i % width);
    const int64_t row = i / width;
    to[i] = from.data[row / heads * from.ts + row % heads * from.hs + e];
  }
}

constexpr int64_t kMaxStride = 1ll << 40, kNear = 1ll << 22;      // elements; 128 rows kNear apart are addressed in 31 bits

bool heads_fine(const conqur_heads& h, uint64_t heads, uint32_t width, uint64_t tokens, bool output) {
  if (h.heads != heads || !h.data || reinterpret_cast<uintptr_t>(h.data) % 2) return false;
  if (h.token_stride < 0 || h.token_stride >= kMaxStride || h.head_stride < 0 || h.head_stride >= kMaxStride) return false;
  if (!output) return true;
  const __int128 w = width, ts = h.token_stride, hs = h.head_stride, heads_ = h.heads, n = tokens;
  if ((heads > 1 && hs < w) || (n > 1 && ts < w)) return false;
  return !(heads > 1 && n > 1 && ts < (heads_ - 1) * hs + w && hs < (n - 1) * ts + w);
}

// As the kernels read them: from multiples of 16 bytes, and (64 tokens' rows of a key head) within 31 bits.
bool plain(const conqur_heads& h) {
  return reinterpret_cast<uintptr_t>(h.data) % 16 == 0 && h.token_stride % 8 == 0 && h.head_stride % 8 == 0 && h.token_stride < kNear && h.head_stride < kNear;
}

bool call_fine(const conqur_attention_call* c) {
  if (!c || c->sequences < 1 || c->sequences > 65535 || !scores_fine(c->scale, c->cap) || c->window >= 1u << 31) return false;
  if (c->width != 32 && c->width != 64 && c->width != 80 && c->width != 96 && c->width != 128) return false;
  if (c->k.heads < 1 || c->k.heads > 65535 || c->q.heads < 1 || c->q.heads % c->k.heads || c->q.heads / c->k.heads > 64) return false;
  if (c->tokens >= 1ull << 31 || c->tokens * (c->q.heads / c->k.heads) >= (1ull << 31) - 256) return false;
  return ((c->tokens * (c->q.heads / c->k.heads)) / kRows + c->sequences + 2) * c->k.heads < 1ull << 24;          // workgroups of 256 threads, which 32 bits count
}
bool backward_fine(const conqur_attention_call* c) {
  return call_fine(c) && (c->tokens / kTile + c->sequences + 2) * c->k.heads < 1ull << 23;          // ... of 512
}

uint64_t lay_bytes(const conqur_attention_call& c, const conqur_heads& h) { return plain(h) ? 0 : (c.tokens * h.heads * c.width * 2 + 255) / 256 * 256; }
// How many workgroups share the keys of 128 rows, whose results a second launch joins.  A workgroup takes the keys that its rows see one block after the other;
// with fewer workgroups than the device takes at a time (two to a compute unit), the last rows' keys are what all wait for.  As many as make 512, of 256 keys or more
// each, if that saves the wait for 1024 keys or more: 4000 tokens, 4 heads, 1 key head, width 128: 80 us in one part, 46 in four, its gradients 376 and 236; one head of width
// 64: 62 and 26 in fifteen; 8 heads, 8 key heads: 80 and 72 in two.  1000 tokens, 32 heads, 8 key heads: 27, and 33 in two.
int key_splits(const conqur_attention_call& c) {
  if (!c.sequences || !c.k.heads) return 1;
  uint64_t seeing = c.tokens / c.sequences;
  if (c.window && c.window < seeing) seeing = c.window;
  const uint64_t rows = c.tokens * (c.q.heads / c.k.heads), workgroups = (rows / kRows + c.sequences) * c.k.heads;
  const uint64_t fill = workgroups ? 512 / workgroups : 1, most = fill < 16 ? fill : 16, n = seeing / 256 < most ? seeing / 256 : most;
  return n < 2 || seeing - seeing / n < 1024 ? 1 : (int)n;
}
struct ShareSizes {
  uint64_t rows, registers;
};
// each: entries that a row leaves.
ShareSizes share_sizes(const conqur_attention_call& c, int splits, int each) {
  if (splits == 1) return {0, 0};
  const uint64_t rows = (c.tokens * (c.q.heads / c.k.heads) / kRows + c.sequences + 2) * c.k.heads * kRows * splits, width = (c.width + 31) / 32 * 32;
  return {rows * sizeof(float4), rows * width * each * sizeof(float)};
}

struct BackwardSizes {
  uint64_t stat, seen, span, part;
  int parts, splits;
  ShareSizes share;
};
// In how many parts the rows of 64 keys are taken, by as many workgroups, whose sums a kernel of its own adds up.  A workgroup takes what sees its keys one step
// of 128 rows after the other; with fewer workgroups than the device takes at a time (one to a compute unit), the first keys' rows are what the others wait for.
// As many parts as make 512 workgroups (half the rows see a key, on average), of four steps or more: gradients of 2000 tokens, 8 heads, 1 key head, width 128:
// 344 us in one part, 200 in 15 (164 since keys are shared, too); 1000 tokens, 32 heads, 8 key heads: 125 and 115; 2 of 1500 tokens, 40 heads, 8 key heads (384 workgroups): 280, and 314 in two.
int key_parts(const conqur_attention_call& c, uint64_t workgroups) {
  if (!c.sequences) return 1;
  uint64_t seeing = c.tokens / c.sequences;
  if (c.window && c.window < seeing) seeing = c.window;
  const uint64_t steps = seeing * (c.q.heads / c.k.heads) / 128, fill = 512 / workgroups, most = fill < 16 ? fill : 16;
  return steps / 4 < 2 || most < 2 ? 1 : (int)(steps / 4 < most ? steps / 4 : most);
}
BackwardSizes backward_sizes(const conqur_attention_call& c) {
  auto up = [](uint64_t n) { return (n + 255) / 256 * 256; };
  const uint64_t rows = c.tokens * (c.q.heads / c.k.heads);      // (loads of 64 rows' may reach 128 rows behind the last)
  const uint64_t stat = c.cap != 0.0f || c.slopes ? sizeof(float4) : sizeof(float2);
  const uint64_t items = (c.tokens / kTile + c.sequences + 2) * c.k.heads, width = (c.width + 31) / 32 * 32;
  const int parts = key_parts(c, items);
  return {up((rows * c.k.heads + 128) * stat), up((rows + 128) * sizeof(int2)), up((rows / kRows + c.sequences + 2) * kWaves * sizeof(int4)),
          parts > 1 ? parts * items * kTile * width * 2 * sizeof(float) : 0, parts, key_splits(c), share_sizes(c, key_splits(c), 2)};
}

PackedArgs args_of(const conqur_attention_call& c) {
  PackedArgs a = {};
  auto rows = [](const conqur_heads& h) { return Rows{static_cast<bf16_bits*>(h.data), h.token_stride, h.head_stride}; };
  a.q = rows(c.q);
  a.k = rows(c.k);
  a.v = rows(c.v);
  a.out = rows(c.out);
  a.lse = c.lse;
  a.start = c.start;
  a.first = c.first;
  a.last = c.last;
  a.slopes = c.slopes;
  a.tokens = (int64_t)c.tokens;
  a.sequences = (int)c.sequences;
  a.heads = (int)c.k.heads;
  a.group = (int)(c.q.heads / c.k.heads);
  a.width = (int)c.width;
  a.window = (int)c.window;
  a.rest = c.zero_rest != 0;
  a.splits = key_splits(c);
  a.scale = c.scale;
  a.scale_log2 = c.scale * kLog2e;
  a.cap_log2 = c.cap * kLog2e;
  a.cap_in = c.cap == 0.0f ? 0.0f : 2.0f * kLog2e * c.scale / c.cap;
  return a;
}

// Takes rows that are not plain to `at`, which moves on.
hipError_t lay(const conqur_attention_call& c, const conqur_heads& h, Rows* r, unsigned char** at, hipStream_t s) {
  const uint64_t bytes = lay_bytes(c, h);
  if (!bytes) return hipSuccess;
  bf16_bits* const to = reinterpret_cast<bf16_bits*>(*at);
  const uint64_t blocks = (c.tokens * h.heads * c.width + 255) / 256;
  k_lay<<<dim3((uint32_t)(blocks < 65536 ? blocks : 65536)), 256, 0, s>>>(*r, to, (int64_t)c.tokens, (int)h.heads, (int)c.width);
  *r = Rows{to, (int64_t)h.heads * c.width, (int64_t)c.width};
  *at += bytes;
  return hipGetLastError();
}

bool room_fine(const conqur_attention_call& c, uint64_t need) {
  return need == 0 || (c.workspace && reinterpret_cast<uintptr_t>(c.workspace) % 16 == 0 && c.workspace_bytes >= need);
}
bool aligned4(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }
bool arrays_fine(const conqur_attention_call& c) {
  return c.start && aligned4(c.start) && aligned4(c.first) && aligned4(c.last) && aligned4(c.slopes) && aligned4(c.lse);
}

}  // namespace

}  // namespace packed
}  // namespace conqur

using namespace conqur;
using namespace conqur::packed;

extern "C" uint64_t conqur_attention_workspace(const conqur_attention_call* c) {
  if (!call_fine(c)) return 0;
  const ShareSizes share = share_sizes(*c, key_splits(*c), 1);
  return share.rows + share.registers + lay_bytes(*c, c->q) + lay_bytes(*c, c->k) + lay_bytes(*c, c->v);
}

extern "C" conqur_status conqur_attention(const conqur_attention_call* c, void* stream) {
  if (!call_fine(c)) return CONQUR_EINVAL;
  if (c->tokens == 0) return CONQUR_OK;
  if (!heads_fine(c->q, c->q.heads, c->width, c->tokens, false) || !heads_fine(c->k, c->k.heads, c->width, c->tokens, false) ||
      !heads_fine(c->v, c->k.heads, c->width, c->tokens, false) || !heads_fine(c->out, c->q.heads, c->width, c->tokens, true) || !arrays_fine(*c) ||
      !room_fine(*c, conqur_attention_workspace(c)))
    return CONQUR_EINVAL;
  PackedArgs a = args_of(*c);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  unsigned char* at = static_cast<unsigned char*>(c->workspace);
  const ShareSizes share = share_sizes(*c, a.splits, 1);
  a.shared_row = reinterpret_cast<float4*>(at);
  a.shared = reinterpret_cast<float*>(at + share.rows);
  at += share.rows + share.registers;
  hipError_t e = lay(*c, c->q, &a.q, &at, s);
  if (e == hipSuccess) e = lay(*c, c->k, &a.k, &at, s);
  if (e == hipSuccess) e = lay(*c, c->v, &a.v, &at, s);
  if (e == hipSuccess) e = launch_forward(a, s);
  return e == hipSuccess ? CONQUR_OK : CONQUR_EHIP;
}

extern "C" uint64_t conqur_attention_backward_workspace(const conqur_attention_call* c) {
  if (!backward_fine(c)) return 0;
  const BackwardSizes z = backward_sizes(*c);
  return z.stat + z.seen + z.span + z.part + z.share.rows + z.share.registers + lay_bytes(*c, c->q) + lay_bytes(*c, c->k) + lay_bytes(*c, c->v) + lay_bytes(*c, c->out) + lay_bytes(*c, c->out_grad);
}

extern "C" conqur_status conqur_attention_backward(const conqur_attention_call* c, void* stream) {
  if (!backward_fine(c)) return CONQUR_EINVAL;
  if (c->tokens == 0) return CONQUR_OK;
  const uint64_t q = c->q.heads, k = c->k.heads;
  if (!heads_fine(c->q, q, c->width, c->tokens, false) || !heads_fine(c->k, k, c->width, c->tokens, false) ||
      !heads_fine(c->v, k, c->width, c->tokens, false) || !heads_fine(c->out, q, c->width, c->tokens, false) ||
      !heads_fine(c->out_grad, q, c->width, c->tokens, false) || !heads_fine(c->q_grad, q, c->width, c->tokens, true) ||
      !heads_fine(c->k_grad, k, c->width, c->tokens, true) || !heads_fine(c->v_grad, k, c->width, c->tokens, true) || !c->lse || !arrays_fine(*c) ||
      !room_fine(*c, conqur_attention_backward_workspace(c)))
    return CONQUR_EINVAL;
  PackedArgs a = args_of(*c);
  a.out_grad = Rows{static_cast<bf16_bits*>(c->out_grad.data), c->out_grad.token_stride, c->out_grad.head_stride};
  a.q_grad = Rows{static_cast<bf16_bits*>(c->q_grad.data), c->q_grad.token_stride, c->q_grad.head_stride};
  a.k_grad = Rows{static_cast<bf16_bits*>(c->k_grad.data), c->k_grad.token_stride, c->k_grad.head_stride};
  a.v_grad = Rows{static_cast<bf16_bits*>(c->v_grad.data), c->v_grad.token_stride, c->v_grad.head_stride};
  const BackwardSizes z = backward_sizes(*c);
  unsigned char* at = static_cast<unsigned char*>(c->workspace);
  a.stat = reinterpret_cast<float2*>(at);
  a.seen = reinterpret_cast<int2*>(at + z.stat);
  a.span = reinterpret_cast<int4*>(at + z.stat + z.seen);
  a.part = reinterpret_cast<float*>(at + z.stat + z.seen + z.span);
  a.parts = z.parts;
  at += z.stat + z.seen + z.span + z.part;
  a.shared_row = reinterpret_cast<float4*>(at);
  a.shared = reinterpret_cast<float*>(at + z.share.rows);
  at += z.share.rows + z.share.registers;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  hipError_t e = lay(*c, c->q, &a.q, &at, s);
  if (e == hipSuccess) e = lay(*c, c->k, &a.k, &at, s);
  if (e == hipSuccess) e = lay(*c, c->v, &a.v, &at, s);
  if (e == hipSuccess) e = lay(*c, c->out, &a.out, &at, s);
  if (e == hipSuccess) e = lay(*c, c->out_grad, &a.out_grad, &at, s);
  if (e == hipSuccess) e = launch_backward(a, s);
  return e == hipSuccess ? CONQUR_OK : CONQUR_EHIP;
}
