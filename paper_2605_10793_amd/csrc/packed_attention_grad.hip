// Gradients of attention of packed sequences (packed_attention.hip has the formulas of the forward pass).
//
//   p_ij = e^(s_ij - lse_i), D_i = sum_d g_id o_id, ds_ij = p_ij (g_i v_j - D_i), du_ij = ds_ij (1 - tanh(u_ij / cap)^2)
//   dq_i = scale sum_j du_ij k_j,  dk_j = scale sum_i du_ij q_i,  dv_j = sum_i p_ij g_i      (g: the result's gradient)
//
// Two kernels, so that no sum's order depends on which workgroup comes first: one walks through the keys for some rows and leaves dq, the other walks through
// the rows for some keys, all query heads of the key head among them, and leaves dk and dv.  Scores are computed in both (7 products of the 5 that one pass
// would take).  The first also writes what the second needs of each row: lse, D, the keys it sees, and for 32 rows which keys any and all of them see.
#include "packed_attention.h"

namespace conqur {
namespace packed {

namespace {

// Registers 8 k to 8 k + 7 as an operand.
__device__ __forceinline__ bf16x8 pack8(const f32x16& x, int k) {
  return frag_of(f32x2_to_bf16x2(x[8 * k], x[8 * k + 1]), f32x2_to_bf16x2(x[8 * k + 2], x[8 * k + 3]), f32x2_to_bf16x2(x[8 * k + 4], x[8 * k + 5]),
                 f32x2_to_bf16x2(x[8 * k + 6], x[8 * k + 7]));
}

// What the other kernel needs of a row: `off` is D's error.
template <int OPTIONS>
__device__ __forceinline__ void leave_row(Args a, const Item& item, int head, int row, int token, int2 mine, float sum, float off, float lse, float dot, float slope) {
  const int64_t at = (int64_t)item.first * a->group + row, to = (int64_t)head * a->tokens * a->group + at;
  const float2 stat = make_float2(sum == 0.0f ? INFINITY : lse + __builtin_amdgcn_logf(sum), dot + off);
  if constexpr (OPTIONS)
    reinterpret_cast<float4*>(a->stat)[to] = make_float4(stat.x, stat.y, slope, __int_as_float(token));
  else
    a->stat[to] = stat;
  if (head == 0) a->seen[at] = mine;
}

constexpr int kKeys = 32;          // keys that lie in LDS at a time for k_packed_dq

// Operands that each lane keeps in LDS because its registers are full: what goes to scratch memory instead comes back behind all that is on its way to LDS.
constexpr int queries_in_lds(int steps) { return steps == 8 ? 3 : 0; }
constexpr int keys_in_lds(int steps) { return steps == 8 ? 4 : 0; }

template <int KS, int OPTIONS>
__global__ void __launch_bounds__(64 * kWaves, 2) k_packed_dq(const PackedArgs) {
  using T = Tile<KS>;
  constexpr int kBytes = kKeys * T::kPitch, kBuffer = 2 * kBytes, kQueriesInLds = queries_in_lds(KS), kOwn = (KS + kQueriesInLds) * 1024;
  Args a = kernel_args();
  extern __shared__ __attribute__((aligned(1024))) unsigned char shared[];
  unsigned char* const s_grad = shared + 2 * kBuffer;                                             // the wavefronts' operands of the gradient, and some of the queries
  float* const s_bad = reinterpret_cast<float*>(s_grad + kWaves * kOwn);                          // of each buffer's keys: NaN for those that were not finite, 0
  int* const s_odd = reinterpret_cast<int*>(s_bad + 2 * kKeys);                                   // whether any was
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5;
  const int head = blockIdx.x % a->heads;
  Item item;
  if (!item.find(a, blockIdx.x / a->heads, 7, a->group)) return;
  const int part = item.parts - 1 - item.part, group = a->group;
  const int rows = item.count * group;
  auto token_of = [&](int row) { return (int)((uint32_t)(row < rows ? row : rows - 1) / (uint32_t)group); };
  const int row = part * kRows + wave * 32 + (lane & 31), token = token_of(row);
  const int2 mine = keys_of(a, item, token);
  const bool empty = mine.x >= mine.y;

  int begin, end, low, high, low_all, high_all, low_both, high_both;      // (both: all rows of the workgroup)
  {
    auto none = [](int2 x) { return x.x >= x.y; };
    low = wave_min(empty ? INT_MAX : mine.x);
    high = wave_max_int(mine.y);
    low_all = wave_max_int(empty || row >= rows ? INT_MAX : mine.x);
    high_all = wave_min(mine.y);
    const int2 x = keys_of(a, item, token_of(part * kRows + lane)), y = keys_of(a, item, token_of(part * kRows + 64 + lane));
    begin = wave_min(min(none(x) ? INT_MAX : x.x, none(y) ? INT_MAX : y.x));
    end = wave_max_int(max(x.y, y.y));
    low_both = wave_max_int(max(none(x) ? INT_MAX : x.x, none(y) ? INT_MAX : y.x));
    high_both = wave_min(min(x.y, y.y));
    if (part * kRows + wave * 32 >= rows) high = 0;
  }
  begin = begin / kKeys * kKeys;
  share_keys(&begin, &end, kKeys);
  if (head == 0 && lane == 0 && blockIdx.y == 0) a->span[(int64_t)(item.base + part) * kWaves + wave] = make_int4(low, high, low_all, high_all);

  const int64_t row_token = item.first + token;
  const int q_head = head * group + (row < rows ? row : rows - 1) - token * group;
  float dot = 0.0f, lse = INFINITY;
  u32x4* const own_grad = reinterpret_cast<u32x4*>(s_grad + wave * kOwn) + lane;
  {
    bf16x8 gf[KS];
    load_rows<KS>(gf, a->out_grad.data + row_token * a->out_grad.ts + q_head * a->out_grad.hs, h);
#pragma unroll
    for (int s = 0; s < KS; ++s) own_grad[s * 64] = __builtin_bit_cast(u32x4, gf[s]);
    if (!empty) {
      bf16x8 of[KS];
      load_rows<KS>(of, a->out.data + row_token * a->out.ts + q_head * a->out.hs, h);
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int j = 0; j < 8; ++j) dot = fmaf((float)gf[s][j], (float)of[s][j], dot);
      lse = a->lse[row_token * (a->heads * group) + q_head] * kLog2e;
      if (lse == -INFINITY) lse = INFINITY;          // every score is -inf: no weights
    }
  }
  dot = halves(dot, [](float x, float y) { return x + y; });
  bf16x8 qf[KS - kQueriesInLds];
#pragma unroll
  for (int i = 0; i < KS; ++i) {
    const bf16x8 x = *reinterpret_cast<const bf16x8*>(a->q.data + row_token * a->q.ts + q_head * a->q.hs + 16 * i + 8 * h);
    if (i < kQueriesInLds)
      own_grad[(KS + i) * 64] = __builtin_bit_cast(u32x4, x);
    else
      qf[i - kQueriesInLds] = x;
  }

  const int k_stride = (int)(a->k.ts * 2), v_stride = (int)(a->v.ts * 2);
  const bf16_bits* const k0 = a->k.data + (int64_t)item.first * a->k.ts + head * a->k.hs;
  const bf16_bits* const v0 = a->v.data + (int64_t)item.first * a->v.ts + head * a->v.hs;
  const uint32_t lds = lds_of(shared), own_lds = lds_of(own_grad);
  auto own = [&](auto i) { return *(const __attribute__((address_space(3))) bf16x8*)(uintptr_t)(own_lds + decltype(i)::value * 1024); };
  auto send = [&](int kb, int which) {
    send_tile<KS, kKeys>(k0 + (int64_t)kb * a->k.ts, k_stride, item.count - kb, lds + which * kBuffer, wave);
    send_tile<KS, kKeys>(v0 + (int64_t)kb * a->v.ts, v_stride, item.count - kb, lds + which * kBuffer + kBytes, wave);
  };

  // The result, and the sum in lse, are of rounded weights: with D' and p' from them, l = sum p' and e = sum p' (g v - D') say by how much both are off: p = p' / l,
  // D = D' + e / l, and
  //   dq = scale / l (sum p' (g v - D') (..) k - e / l sum p' (..) k)
  // The factors of the first sum, which largely cancel, enter its product in two bf16 parts.  (Of dq's size, two sequences of 2048 tokens: 0.0036 off without
  // either, 0.0027 without the parts, 0.0023 with both, where the rounding of the result alone makes 0.0017.)
  f32x16 dq[T::kTiles], pk[T::kTiles];
#pragma unroll
  for (int t = 0; t < T::kTiles; ++t) dq[t] = pk[t] = f32x16{};
  float sum = 0.0f, off = 0.0f;
  const float scale = a->scale_log2, cap = a->cap_log2, cap_in = a->cap_in, slope = OPTIONS && a->slopes ? a->slopes[q_head] * kLog2e : 0.0f;

  if (threadIdx.x == 0) *s_odd = 0;
  if (begin < end) send(begin, 0);
  int which = 0;
  for (int kb = begin; kb < end; kb += kKeys, which ^= 1) {
    wait_loads<0>();
    pipeline_barrier();
    if (kb + kKeys < end) send(kb + kKeys, which ^ 1);
    const uint32_t sk = lds + which * kBuffer;           // the values lie behind the keys
    // Keys that are not finite must not meet rows that do not see them, for 0 * NaN is NaN: where some rows of the workgroup do not see all of the block they
    // become zeros, and what sees them NaN by itself.
    bool odd = false;
    if (kb < low_both || kb + kKeys > high_both) {
      const int me = lane_anew();
      const bool bad = clear_nonfinite<KS, kKeys / kWaves>(sk, wave, me);
      if (bad) *s_odd = 1;
      if ((me & 7) == 0) s_bad[which * kKeys + wave * 8 + (me >> 3)] = bad ? NAN : 0.0f;
      pipeline_barrier();
      odd = *(volatile int*)s_odd;
    }
    if (kb >= high || kb + kKeys <= low) continue;
    const bool all = kb >= low_all && kb + kKeys <= high_all;
    const int here = lane_anew();
    const typename T::RowsAt row_at(sk + T::row_at(here));
    struct Operands {
      bf16x8 rows, mine;
    };
    f32x16 s = f32x16{}, d = f32x16{};
    __builtin_amdgcn_s_setprio(1);           // before the other wavefront's arithmetic: 200 -> 190 us, two sequences of 2048 tokens
    in_turn<2 * KS, 3>(
        [&](auto i) {
          constexpr int I = decltype(i)::value / 2;
          if constexpr (decltype(i)::value % 2)
            return Operands{row_at.template get<kBytes>(I), own(std::integral_constant<int, I>{})};
          else if constexpr (I < kQueriesInLds)
            return Operands{row_at.template get<0>(I), own(std::integral_constant<int, KS + I>{})};
          else
            return Operands{row_at.template get<0>(I), qf[I - kQueriesInLds]};
        },
        [&](auto i, const Operands& f) {
          if constexpr (decltype(i)::value % 2)
            d = mfma32(f.rows, f.mine, d);
          else
            s = mfma32(f.rows, f.mine, s);
        });
    __builtin_amdgcn_s_setprio(0);
    if (odd) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] += s_bad[which * kKeys + row_of(r, h)];
    }
    const int lo = mine.x - kb - 4 * h, hi = mine.y - kb - 4 * h;
    const float at = (float)(token - kb - 4 * h);
    // The factors of an entry at a time, so that nothing but they stays in registers.
    auto factors = [&](auto all_seen, auto caps) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float x = 0.0f, y;
        if constexpr (decltype(caps)::value)
          y = capped(s[r], cap, cap_in, lse, &x);
        else
          y = fmaf(s[r], scale, -lse);
        if constexpr (OPTIONS) y = fmaf(-slope, fabsf(at - (float)row_of(r, 0)), y);
        float p = __builtin_amdgcn_exp2f(y), e = (d[r] - dot) * p;
        if constexpr (!decltype(all_seen)::value) {
          const uint32_t see = -(uint32_t)((row_of(r, 0) >= lo) & (row_of(r, 0) < hi));
          p = __uint_as_float(__float_as_uint(p) & see);
          e = __uint_as_float(__float_as_uint(e) & see);
          if constexpr (decltype(caps)::value) x = __uint_as_float(__float_as_uint(x) & see);
        }
        sum += p;
        off += e;
        if constexpr (decltype(caps)::value) {
          x = 4.0f * (x - x * x);
          p *= x;
          e *= x;
        }
        s[r] = p;
        d[r] = e;
      }
    };
    if constexpr (OPTIONS == kCapped)
      factors(std::false_type{}, std::true_type{});
    else if (all)
      factors(std::true_type{}, std::false_type{});
    else
      factors(std::false_type{}, std::false_type{});
    const bf16x8 pf[2] = {pack8(s, 0), pack8(s, 1)}, df[2] = {pack8(d, 0), pack8(d, 1)};
#pragma unroll
    for (int r = 0; r < 16; ++r) d[r] -= (float)df[r / 8][r % 8];
    const bf16x8 rest[2] = {pack8(d, 0), pack8(d, 1)};
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
    const typename T::TurnedAt turned_at(sk + T::turned_at(here));
    in_turn<2 * T::kTiles>([&](auto i) { return turned_at.template get<decltype(i)::value / T::kTiles * 16 * T::kPitch>(decltype(i)::value % T::kTiles); },
                           [&](auto i, bf16x8 f) {
                             constexpr int I = decltype(i)::value, t = I % T::kTiles;
                             dq[t] = mfma32(f, df[I / T::kTiles], dq[t]);
                             pk[t] = mfma32(f, pf[I / T::kTiles], pk[t]);
                             dq[t] = mfma32(f, rest[I / T::kTiles], dq[t]);
                           });
    __builtin_amdgcn_s_setprio(0);
  }

  sum = halves(sum, [](float x, float y) { return x + y; });
  off = halves(off, [](float x, float y) { return x + y; });
  a = kernel_args();
  if (gridDim.y > 1) {
    f32x4* const to = shared_of<8 * T::kTiles>(a, (int)blockIdx.y, wave);
#pragma unroll
    for (int t = 0; t < T::kTiles; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        to[(8 * t + r) * 64] = f32x4{dq[t][4 * r], dq[t][4 * r + 1], dq[t][4 * r + 2], dq[t][4 * r + 3]};
        to[(8 * t + 4 + r) * 64] = f32x4{pk[t][4 * r], pk[t][4 * r + 1], pk[t][4 * r + 2], pk[t][4 * r + 3]};
      }
    if (h == 0) *shared_row_of(a, (int)blockIdx.y, wave * 32 + lane) = make_float4(sum, off, lse, dot);
    return;
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  off *= inv;
  if (row >= rows) return;
  if (h == 0) leave_row<OPTIONS>(a, item, head, row, token, mine, sum, off, lse, dot, slope);
  bf16_bits* const to = a->q_grad.data + row_token * a->q_grad.ts + q_head * a->q_grad.hs + 4 * h;
#pragma unroll
  for (int t = 0; t < T::kTiles; ++t) dq[t] -= off * pk[t];
  store_row<KS>(to, dq, a->scale * inv, wide8(a->q_grad.data, a->q_grad.ts, a->q_grad.hs));
}

// What workgroups that share keys made, added up in their order, for 32 entries of a row (blockIdx.y).
template <int KS, int OPTIONS>
__global__ void __launch_bounds__(64 * kWaves) k_packed_dq_join(const PackedArgs) {
  using T = Tile<KS>;
  const Args a = kernel_args();
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5, t = blockIdx.y;
  const int head = blockIdx.x % a->heads, group = a->group;
  Item item;
  if (!item.find(a, blockIdx.x / a->heads, 7, group)) return;
  const int row = (item.parts - 1 - item.part) * kRows + wave * 32 + (lane & 31);
  if (row >= item.count * group) return;
  float4 all = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  f32x16 dq = {}, pk = {};
  for (int i = 0; i < a->splits; ++i) {
    const float4 x = *shared_row_of(a, i, wave * 32 + (lane & 31));
    all = make_float4(all.x + x.x, all.y + x.y, x.z, x.w);
    const f32x4* const from = shared_of<8 * T::kTiles>(a, i, wave) + 8 * t * 64;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const f32x4 y = from[r * 64], z = from[(4 + r) * 64];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        dq[4 * r + j] += y[j];
        pk[4 * r + j] += z[j];
      }
    }
  }
  const float inv = all.x == 0.0f ? 0.0f : 1.0f / all.x, off = all.y * inv;
  const int token = (int)((uint32_t)row / (uint32_t)group), q_head = head * group + row - token * group;
  if (h == 0 && t == 0)
    leave_row<OPTIONS>(a, item, head, row, token, keys_of(a, item, token), all.x, off, all.z, all.w, OPTIONS && a->slopes ? a->slopes[q_head] * kLog2e : 0.0f);
  dq -= off * pk;
  store_tile<KS>(a->q_grad.data + (item.first + (int64_t)token) * a->q_grad.ts + q_head * a->q_grad.hs + 4 * h, t, dq, a->scale * inv,
                 wide8(a->q_grad.data, a->q_grad.ts, a->q_grad.hs));
}

// Where the sums over part `p` of the rows are, of 32 keys of a workgroup.
template <int KS>
__device__ __forceinline__ f32x4* part_of(Args a, int p, int workgroup, int half) {
  return reinterpret_cast<f32x4*>(a->part) + (((int64_t)p * gridDim.x + workgroup) * 2 + half) * (2 * Tile<KS>::kTiles * 4 * 64);
}

// Eight wavefronts, which take 32 of the workgroup's 64 keys and 32 of 128 rows at a time each; their sums meet in LDS at the end.  (Four, two workgroups to a
// compute unit: 274 us for 193, two sequences of 2048 tokens.  A workgroup's time is what the rows of its keys take one after the other, and the first keys' rows
// are all there are.)  If there are few workgroups, several share the rows of 64 keys, step by step in turn.
constexpr int kKeyWaves = 8, kStep = 16 * kKeyWaves;                  // kStep: rows that lie in LDS at a time
template <int KS, int OPTIONS>
struct KeySide {
  static constexpr int kBytes = kStep * Tile<KS>::kPitch;             // of their queries, and of their gradients
  static constexpr int kStat = OPTIONS ? 16 : 8;                      // of a row: lse, D; slope, token
  static constexpr int kSeenAt = kStep * kStat;
  static constexpr int kBuffer = 2 * kBytes + kSeenAt + kStep * 8;
  static constexpr int kKeysAt = 2 * kBuffer;                         // operands of the keys
  static constexpr int kBadAt = kKeysAt + 2 * keys_in_lds(KS) * 1024;
  static constexpr int kShared = kBadAt + 2 * kStep * 4 + 16;
  static_assert(kKeyWaves / 2 * 64 * 8 * Tile<KS>::kTiles * 16 <= kShared, "sums meet where the tiles were");
};

template <int KS, int OPTIONS>
__global__ void __launch_bounds__(64 * kKeyWaves, 2) k_packed_dkv(const PackedArgs) {
  using T = Tile<KS>;
  using D = KeySide<KS, OPTIONS>;
  constexpr int kBytes = D::kBytes, kBuffer = D::kBuffer, kStat = D::kStat, kSeenAt = D::kSeenAt;
  Args a = kernel_args();
  extern __shared__ __attribute__((aligned(1024))) unsigned char shared[];
  float* const s_bad = reinterpret_cast<float*>(shared + D::kBadAt);              // of each buffer's rows: NaN for those that were not finite, 0
  int* const s_odd = reinterpret_cast<int*>(s_bad + 2 * kStep);                   // whether any was
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5;
  const int head = blockIdx.x % a->heads;
  Item item;
  if (!item.find(a, blockIdx.x / a->heads, 6, 1)) return;
  static_assert(kTile == 64, "");
  const int group = a->group, rows = item.count * group;
  const int k0 = item.part * kTile, key0 = k0 + 32 * (wave & 1), at_rows = wave >> 1;      // keys of the workgroup, of the wavefront; which 32 rows
  const int key = key0 + (lane & 31);
  const int64_t key_token = item.first + (key < item.count ? key : item.count - 1);
  if (threadIdx.x == 0) *s_odd = 0;
  constexpr int kKeysInLds = keys_in_lds(KS);
  bf16x8 kf[KS - kKeysInLds], vf[KS];
  u32x4* const own_keys = reinterpret_cast<u32x4*>(shared + D::kKeysAt + (wave & 1) * kKeysInLds * 1024) + lane;      // (all wavefronts of 32 keys write the same)
#pragma unroll
  for (int i = 0; i < KS; ++i) {
    const bf16x8 x = *reinterpret_cast<const bf16x8*>(a->k.data + key_token * a->k.ts + head * a->k.hs + 16 * i + 8 * h);
    if (i < kKeysInLds)
      own_keys[i * 64] = __builtin_bit_cast(u32x4, x);
    else
      kf[i - kKeysInLds] = x;
  }
  load_rows<KS>(vf, a->v.data + key_token * a->v.ts + head * a->v.hs, h);
  const uint32_t keys_lds = lds_of(own_keys);

  // Rows in thirty-twos, 64 of which (`chunk`) a wavefront looks at together; of those any of whose rows sees a key, four by four.
  const int4* const span = a->span + ((((int64_t)item.first * group) >> 7) + item.number) * kWaves;
  const int subs = item.rest ? 0 : (rows + 31) / 32;
  int next_chunk = a->last ? 0 : (int)((int64_t)k0 * group / kStep) * (kStep / 32), chunk = 0;
  uint64_t active = 0, some = 0, whole = 0, every = 0;
  struct Step {
    int sub;
    bool some, all, every;      // of the wavefront's keys and rows: any are seen, all are; all of the workgroup's
  };
  int turn = blockIdx.y;        // steps until the next that is this workgroup's
  auto next = [&](Step* x) {
    for (;;) {
      while (!active) {
        if (next_chunk >= subs) return false;
        chunk = next_chunk;
        next_chunk += 64;
        const int sub = chunk + lane;
        int4 s = make_int4(INT_MAX, 0, INT_MAX, 0);
        if (sub < subs) s = span[sub];
        const uint64_t near = __ballot(s.x < k0 + kTile && s.y > k0);
        some = __ballot(s.x < key0 + 32 && s.y > key0);
        whole = __ballot(s.z <= key0 && s.w >= key0 + 32);
        every = __ballot(s.z <= k0 && s.w >= k0 + kTile);
        active = (near | near >> 1 | near >> 2 | near >> 3) & 0x1111111111111111ull;
      }
      const int bit = __builtin_ctzll(active);
      active &= active - 1;
      if (turn-- > 0) continue;
      turn = (int)gridDim.y - 1;
      x->sub = chunk + bit;
      x->some = (some >> (bit + at_rows)) & 1;
      x->all = (whole >> (bit + at_rows)) & 1;
      x->every = ((every >> bit) & ((1 << kStep / 32) - 1)) == (1 << kStep / 32) - 1;
      return true;
    }
  };

  const bf16_bits* const q0 = a->q.data + (int64_t)item.first * a->q.ts + (int64_t)head * group * a->q.hs;
  const bf16_bits* const g0 = a->out_grad.data + (int64_t)item.first * a->out_grad.ts + (int64_t)head * group * a->out_grad.hs;
  const unsigned char* const stat0 = reinterpret_cast<const unsigned char*>(a->stat) + ((int64_t)head * a->tokens + item.first) * group * kStat;
  const int2* const seen0 = a->seen + (int64_t)item.first * group;
  const int q_ts = (int)(a->q.ts * 2), q_hs = (int)(a->q.hs * 2), g_ts = (int)(a->out_grad.ts * 2), g_hs = (int)(a->out_grad.hs * 2);
  const uint32_t over = (65536 + group - 1) / group;      // n * over >> 16 is n / group for n up to 192, group up to 64
  const uint32_t lds = lds_of(shared);
  auto send = [&](int sub, int which) {
    const int row0 = sub * 32, token0 = (int)((uint32_t)row0 / (uint32_t)group), lead = row0 - token0 * group;
    const u32x4 from_q = memory_at(q0 + token0 * a->q.ts), from_g = memory_at(g0 + token0 * a->out_grad.ts);
    const uint32_t to = lds + which * kBuffer;
    const int me = lane_anew();
    const int in = me / T::kChunks, c0 = (me % T::kChunks) ^ (T::kChunks == 16 ? in << 2 : ((in >> 1) & 1) << 2 | in >> 2);
    const int last = rows - 1 - row0;
#pragma unroll
    for (int i = 0; i < T::kLoads; ++i) {
      const int r0 = (wave * T::kLoads + i) * T::kRowsAt, n = lead + (r0 + in < last ? r0 + in : last);
      const int token = (int)(((uint32_t)n * over) >> 16), member = n - token * group;
      int c = c0 ^ (T::kChunks == 16 ? i & 3 : (i & 1) << 1);
      if (KS * 2 < T::kChunks) c = c < KS * 2 ? c : KS * 2 - 1;
      send16(from_q, to + r0 * T::kPitch, token * q_ts + member * q_hs + c * 16, 0);
      send16(from_g, to + kBytes + r0 * T::kPitch, token * g_ts + member * g_hs + c * 16, 0);
    }
    if (wave < kStat / 8) send16(memory_at(stat0 + (int64_t)row0 * kStat), to + 2 * kBytes + wave * 1024, wave * 1024 + me * 16, 0);
    if (wave == 2) send16(memory_at(seen0 + row0), to + 2 * kBytes + kSeenAt, me * 16, 0);
  };

  f32x16 dk[T::kTiles], dv[T::kTiles];
#pragma unroll
  for (int t = 0; t < T::kTiles; ++t) dk[t] = dv[t] = f32x16{};
  const float scale = a->scale_log2, cap = a->cap_log2, cap_in = a->cap_in;

  Step now, then;
  bool more = next(&now);
  if (more) send(now.sub, 0);
  if (wave >= 4) __builtin_amdgcn_s_setprio(1);          // of two wavefronts that share a SIMD, and begin a step together, one goes first: 376 -> 370 us, uneven prefixes
  for (int which = 0; more; which ^= 1, now = then) {
    more = next(&then);
    wait_loads<0>();
    pipeline_barrier();
    if (more) send(then.sub, which ^ 1);
    bool odd = false;          // (as in k_packed_dq: queries and gradients that are not finite)
    if (!now.every) {
      const int me = lane_anew();
      const bool bad_q = clear_nonfinite<KS, 16>(lds + which * kBuffer, wave, me), bad_g = clear_nonfinite<KS, 16>(lds + which * kBuffer + kBytes, wave, me);
      if (bad_q || bad_g) *s_odd = 1;
      if ((me & 3) == 0) s_bad[which * kStep + wave * 16 + (me >> 2)] = bad_q || bad_g ? NAN : 0.0f;
      pipeline_barrier();
      odd = *(volatile int*)s_odd;
    }
    if (!now.some) continue;
    const uint32_t sq = lds + which * kBuffer + at_rows * 32 * T::kPitch;           // the gradients lie behind the queries
    const unsigned char* const s_rows = shared + which * kBuffer + 2 * kBytes;
    const int here = lane_anew();
    const typename T::RowsAt row_at(sq + T::row_at(here));
    const int half = here >> 5;

    f32x16 s = f32x16{}, d = f32x16{};
    struct Operands {
      bf16x8 rows, keys;
    };
    in_turn<2 * KS>(
        [&](auto i) {
          constexpr int I = decltype(i)::value / 2;
          if constexpr (decltype(i)::value % 2)
            return Operands{row_at.template get<kBytes>(I), vf[I]};
          else if constexpr (I < kKeysInLds)
            return Operands{row_at.template get<0>(I), *(const __attribute__((address_space(3))) bf16x8*)(uintptr_t)(keys_lds + I * 1024)};
          else
            return Operands{row_at.template get<0>(I), kf[I - kKeysInLds]};
        },
        [&](auto i, const Operands& f) {
          if constexpr (decltype(i)::value % 2)
            d = mfma32(f.rows, f.keys, d);
          else
            s = mfma32(f.rows, f.keys, s);
        });
    if (odd) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] += s_bad[which * kStep + at_rows * 32 + row_of(r, half)];
    }
    {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float lse, dot, slope = 0.0f;
        int token = 0;
        if constexpr (OPTIONS) {
          const f32x4 x = *reinterpret_cast<const f32x4*>(s_rows + (at_rows * 32 + row_of(r, half)) * kStat);
          lse = x[0], dot = x[1], slope = x[2], token = __float_as_int(x[3]);
        } else {
          const f32x2 x = *reinterpret_cast<const f32x2*>(s_rows + (at_rows * 32 + row_of(r, half)) * kStat);
          lse = x[0], dot = x[1];
        }
        float x = 0.0f, y;
        if constexpr (OPTIONS == kCapped)
          y = capped(s[r], cap, cap_in, lse, &x);
        else
          y = fmaf(s[r], scale, -lse);
        if constexpr (OPTIONS) y = fmaf(-slope, fabsf((float)(token - key)), y);          // (24 bits do not hold every token)
        const float p = __builtin_amdgcn_exp2f(y);
        float e = (d[r] - dot) * p;
        if constexpr (OPTIONS == kCapped) e *= 4.0f * (x - x * x);
        s[r] = p;
        d[r] = e;
      }
    }
    if (!now.all) {
      const int left = rows - (now.sub + at_rows) * 32 - 4 * half;
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        typedef int i32x4 __attribute__((ext_vector_type(4)));
        const i32x4* const at = reinterpret_cast<const i32x4*>(s_rows + kSeenAt + (at_rows * 32 + 8 * r4 + 4 * half) * 8);
        const i32x4 x = at[0], y = at[1];
        const int lo[4] = {x[0], x[2], y[0], y[2]}, hi[4] = {x[1], x[3], y[1], y[3]};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t see = -(uint32_t)((key >= lo[j]) & (key < hi[j]) & (row_of(4 * r4 + j, 0) < left));
          s[4 * r4 + j] = __uint_as_float(__float_as_uint(s[4 * r4 + j]) & see);
          d[4 * r4 + j] = __uint_as_float(__float_as_uint(d[4 * r4 + j]) & see);
        }
      }
    }
    const bf16x8 pf[2] = {pack8(s, 0), pack8(s, 1)}, df[2] = {pack8(d, 0), pack8(d, 1)};
    __builtin_amdgcn_sched_barrier(0);
    const typename T::TurnedAt turned_at(sq + T::turned_at(here));
    // Operands of the queries and, odd ones, of the gradients: 16 rows, 32 entries.
    auto turned = [&](auto i) {
      constexpr int I = decltype(i)::value;
      return turned_at.template get<I % 2 * kBytes + I / 2 / T::kTiles * 16 * T::kPitch>(I / 2 % T::kTiles);
    };
    in_turn<4 * T::kTiles>(turned, [&](auto i, bf16x8 f) {
      constexpr int I = decltype(i)::value, t = I / 2 % T::kTiles, k = I / 2 / T::kTiles;
      if constexpr (I % 2)
        dv[t] = mfma32(f, pf[k], dv[t]);
      else
        dk[t] = mfma32(f, df[k], dk[t]);
    });
  }

  __syncthreads();
  // The sums of the last rows' wavefronts to the first ones'.
#pragma unroll
  for (int half = kKeyWaves / 4; half > 0; half /= 2) {
    f32x4* const s_sum = reinterpret_cast<f32x4*>(shared) + (wave & (2 * half - 1)) * 64 * 8 * T::kTiles + lane;
    if (at_rows >= half && at_rows < 2 * half) {
#pragma unroll
      for (int t = 0; t < T::kTiles; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s_sum[(t * 4 + r) * 64] = f32x4{dk[t][4 * r], dk[t][4 * r + 1], dk[t][4 * r + 2], dk[t][4 * r + 3]};
          s_sum[((T::kTiles + t) * 4 + r) * 64] = f32x4{dv[t][4 * r], dv[t][4 * r + 1], dv[t][4 * r + 2], dv[t][4 * r + 3]};
        }
    }
    __syncthreads();
    if (at_rows < half) {
#pragma unroll
      for (int t = 0; t < T::kTiles; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const f32x4 x = s_sum[(t * 4 + r) * 64], y = s_sum[((T::kTiles + t) * 4 + r) * 64];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            dk[t][4 * r + j] += x[j];
            dv[t][4 * r + j] += y[j];
          }
        }
    }
    __syncthreads();
  }
  a = kernel_args();
  if (wave >= 2) return;
  if (gridDim.y > 1) {
    f32x4* const to = part_of<KS>(a, (int)blockIdx.y, (int)blockIdx.x, wave) + lane;
#pragma unroll
    for (int t = 0; t < T::kTiles; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        to[(t * 4 + r) * 64] = f32x4{dk[t][4 * r], dk[t][4 * r + 1], dk[t][4 * r + 2], dk[t][4 * r + 3]};
        to[((T::kTiles + t) * 4 + r) * 64] = f32x4{dv[t][4 * r], dv[t][4 * r + 1], dv[t][4 * r + 2], dv[t][4 * r + 3]};
      }
    return;
  }
  if (key >= item.count) return;
  const bool k_wide = wide8(a->k_grad.data, a->k_grad.ts, a->k_grad.hs), v_wide = wide8(a->v_grad.data, a->v_grad.ts, a->v_grad.hs);
  bf16_bits* const to_k = a->k_grad.data + key_token * a->k_grad.ts + head * a->k_grad.hs + 4 * h;
  bf16_bits* const to_v = a->v_grad.data + key_token * a->v_grad.ts + head * a->v_grad.hs + 4 * h;
  store_row<KS>(to_k, dk, a->scale, k_wide);
  store_row<KS>(to_v, dv, 1.0f, v_wide);
}

// The sums of the rows' parts, in their order, for 32 entries of a key (blockIdx.y).
template <int KS>
__global__ void __launch_bounds__(128) k_packed_sum(const PackedArgs) {
  using T = Tile<KS>;
  const Args a = kernel_args();
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5, t = blockIdx.y;
  const int head = blockIdx.x % a->heads;
  Item item;
  if (!item.find(a, blockIdx.x / a->heads, 6, 1)) return;
  const int key = item.part * kTile + 32 * wave + (lane & 31);
  f32x16 dk = {}, dv = {};
  for (int p = 0; p < a->parts; ++p) {
    const f32x4* const from = part_of<KS>(a, p, (int)blockIdx.x, wave) + t * 4 * 64 + lane;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const f32x4 x = from[r * 64], y = from[(T::kTiles * 4 + r) * 64];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        dk[4 * r + j] += x[j];
        dv[4 * r + j] += y[j];
      }
    }
  }
  if (key >= item.count) return;
  const int64_t token = item.first + key;
  store_tile<KS>(a->k_grad.data + token * a->k_grad.ts + head * a->k_grad.hs + 4 * h, t, dk, a->scale, wide8(a->k_grad.data, a->k_grad.ts, a->k_grad.hs));
  store_tile<KS>(a->v_grad.data + token * a->v_grad.ts + head * a->v_grad.hs + 4 * h, t, dv, 1.0f, wide8(a->v_grad.data, a->v_grad.ts, a->v_grad.hs));
}

template <int KS, int OPTIONS>
hipError_t launch(const PackedArgs& a, hipStream_t s) {
  constexpr int kDq = 4 * kKeys * Tile<KS>::kPitch + kWaves * (KS + queries_in_lds(KS)) * 1024 + 2 * kKeys * 4 + 16, kDkv = KeySide<KS, OPTIONS>::kShared;
  static PerDeviceOnce once;
  hipError_t e = once.run([] {
    const hipError_t x = hipFuncSetAttribute(reinterpret_cast<const void*>(k_packed_dq<KS, OPTIONS>), hipFuncAttributeMaxDynamicSharedMemorySize, kDq);
    return x != hipSuccess ? x : hipFuncSetAttribute(reinterpret_cast<const void*>(k_packed_dkv<KS, OPTIONS>), hipFuncAttributeMaxDynamicSharedMemorySize, kDkv);
  });
  if (e != hipSuccess) return e;
  const uint32_t of_rows = (uint32_t)(row_items(a) * a.heads);
  k_packed_dq<KS, OPTIONS><<<dim3(of_rows, (uint32_t)a.splits), 64 * kWaves, kDq, s>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.splits > 1) {
    k_packed_dq_join<KS, OPTIONS><<<dim3(of_rows, Tile<KS>::kTiles), 64 * kWaves, 0, s>>>(a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const uint32_t workgroups = (uint32_t)(key_items(a) * a.heads);
  k_packed_dkv<KS, OPTIONS><<<dim3(workgroups, (uint32_t)a.parts), 64 * kKeyWaves, kDkv, s>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess || a.parts == 1) return e;
  k_packed_sum<KS><<<dim3(workgroups, Tile<KS>::kTiles), 128, 0, s>>>(a);
  return hipGetLastError();
}

template <int KS>
hipError_t launch(const PackedArgs& a, hipStream_t s) {
  return a.cap_log2 != 0.0f ? launch<KS, kCapped>(a, s) : a.slopes ? launch<KS, kBiased>(a, s) : launch<KS, 0>(a, s);
}

}  // namespace

hipError_t launch_backward(const PackedArgs& a, hipStream_t s) {
  switch (a.width) {
    case 32: return launch<2>(a, s);
    case 64: return launch<4>(a, s);
    case 80: return launch<5>(a, s);
    case 96: return launch<6>(a, s);
    default: return launch<8>(a, s);
  }
}

}  // namespace packed
}  // namespace conqur
