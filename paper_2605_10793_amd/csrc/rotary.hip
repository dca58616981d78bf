// Rotary positions of queries and keys, alone or in one pass with their per-head norms, and that pass's gradients.
//
//   rotary    y_a = m (x_a cos t - x_b sin t), y_b = m (x_b cos t + x_a sin t) over the pairs (a, b) of a head's first `part`
//             entries, t = position * frequency; the entries behind them are copied.  Transposed: sin -> -sin.
//   norm      x^ = x / sqrt(mean x^2 + eps), u = w x^, y = rotary(u)
//   gradient  h = rotary^T(g), dw = sum over tokens and heads of h x^, dx = (w h - x^ mean(w h x^)) / sqrt(mean x^2 + eps)
//
// All three are bound by HBM (3 to 14 operations an element) or, with few tokens, by launch latency.  So every row is read once
// and written once, and sums stay in registers:
//   * A row is cut into units of 2V entries, V of each half of a pair (half layout) or 2V neighbours (interleaved layout), so
//     that a lane holds both members of its pairs and reads and writes 16-byte vectors; 2^k lanes hold a row, a wavefront 64 / 2^k
//     rows at a time, and the row sums are VALU exchanges between those lanes.
//   * A wavefront works on one token at a time, so that its angles are taken once for all heads: every lane computes one pair's
//     sine and cosine (whole turns are dropped in 64 bits, so that positions of any size keep 32-bit angles) and passes it to
//     the lanes that need it through LDS.  A table of angles in memory would add 4 part bytes a token to the traffic and a bound on
//     the positions.
//   * Few tokens: the heads of a token are dealt to several wavefronts.
//   * The gradient keeps the next step's rows under way while it computes one (79 -> 59 us together with the next point), which the other
//     two, with more wavefronts a compute unit, do not need.  No barrier: a wavefront's angles are its own.
//   * The weights' gradients are summed per lane over the rows it meets, then over the lanes, the wavefronts and, by a second
//     launch, the workgroups, in a fixed order: no atomics, the same bits in every run.
//
// Measured, calls one behind the other: rotary of 4096 tokens of 32 + 8 heads of 128 in bf16 15.1 us (5.6 TB/s read and written), transposed of 1999
// tokens of 32 + 32 heads of 80 in fp32 16.2 us (5.1 TB/s); norms and rotary of 8192 tokens of 32 + 8 heads of 128 in bf16 36 us (4.7 TB/s), their
// gradients 59 us (4.3 TB/s; 50 and 4.6 in the two launches, and what lies between), in fp32 72 and 107 us (4.7 TB/s).  A token, or 64: 10 to
// 11 us a call, of which the kernel is 3.5 and 4.3; the rest is the caller's.
#include "../../include/conqur.h"

#include <math.h>

#include "kernels.h"

using namespace conqur;

namespace {

constexpr int kWaves = 4;            // wavefronts of a workgroup
constexpr int kMaxWidth = 512;
constexpr int kGradVector = 4;       // (8 bf16 entries a lane take 190 registers with the next rows under way, half the wavefronts: 60.8 us for the 58.9 below)
constexpr int kGradGroups = 1024;    // workgroups of the gradient's launch: four of 4 wavefronts on each of 256 compute units

struct View {                        // [token][head][width], entries next to each other
  const void* p;
  int64_t ts, hs;
};

struct RotaryArgs {
  View in[2], out[2], grad[2];       // queries, keys
  const void* w[2];
  int heads[2];
  int steps[2];                      // row groups of a token: ceil(heads / rows a wavefront holds)
  const int64_t* positions;
  const double* turns;
  float* part_sums;                  // gradient: [workgroup][2][width]
  int64_t tokens;
  int64_t tasks;                     // tokens * chunks
  int chunks, chunk_steps;           // a token's steps are dealt to `chunks` wavefronts
  int width, part;
  int lanes;                         // lanes of a row, a power of two
  float magnitude, eps, inv_width;
  int transposed;
};

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const bf16_bits* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(bf16_bits* p, float v) { *p = f32_to_bf16(v); }

template <int V>
__device__ __forceinline__ void load_vec(const float* p, float* v) {
  if constexpr (V % 4 == 0) {
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(p + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[i + j] = x[j];
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = p[i];
  }
}
template <int V>
__device__ __forceinline__ void load_vec(const bf16_bits* p, float* v) {
  if constexpr (V == 8) {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(u[i] << 16); v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
  } else if constexpr (V == 4) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    const uint32_t u[2] = {x.x, x.y};
#pragma unroll
    for (int i = 0; i < 2; ++i) { v[2 * i] = __uint_as_float(u[i] << 16); v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = bf16_to_f32(p[i]);
  }
}
template <int V>
__device__ __forceinline__ void store_vec(float* p, const float* v) {
  if constexpr (V % 4 == 0) {
#pragma unroll
    for (int i = 0; i < V; i += 4) *reinterpret_cast<f32x4*>(p + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] = v[i];
  }
}
template <int V>
__device__ __forceinline__ void store_vec(bf16_bits* p, const float* v) {
  if constexpr (V == 8) {
    *reinterpret_cast<uint4*>(p) = make_uint4(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]), f32x2_to_bf16x2(v[4], v[5]),
                                              f32x2_to_bf16x2(v[6], v[7]));
  } else if constexpr (V == 4) {
    *reinterpret_cast<uint2*>(p) = make_uint2(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]));
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] = f32_to_bf16(v[i]);
  }
}

// Sum over groups of `lanes` neighbouring lanes (a power of two), known to every lane of the group: exchanges by 1 and 2 within
// quads, then mirrored halves of 8 and rows of 16 (whose lanes hold the quads' sums already), then rows and halves of the wavefront.
template <int CTRL>
__device__ __forceinline__ float lane_perm(float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float group_sum(float v, int lanes) {
  if (lanes > 1) v += lane_perm<0xB1>(v);     // quad_perm 1,0,3,2
  if (lanes > 2) v += lane_perm<0x4E>(v);     // quad_perm 2,3,0,1
  if (lanes > 4) v += lane_perm<0x141>(v);    // row_half_mirror
  if (lanes > 8) v += lane_perm<0x140>(v);    // row_mirror
  if (lanes > 16) {
    const uint32_t u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
  if (lanes > 32) {
    const uint32_t u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
  return v;
}

enum Mode { kRotary, kNorm, kGrad };

// A lane's U units of a row (U > 1 only for V = 1): where their two vectors lie and the pair the first entry belongs to (-1: copied
// entries, behind the rotated part; -2: no unit).
template <int V, int U, bool INTERLEAVED>
struct Units {
  int a[U], b[U], pair[U];
  __device__ __forceinline__ Units(int first, int lanes, int width, int part) {
    const int rotated = part / (2 * V), all = width / (2 * V);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = first + i * lanes;
      if (u < rotated) {
        a[i] = INTERLEAVED ? 2 * u * V : u * V;
        b[i] = INTERLEAVED ? 2 * u * V + V : part / 2 + u * V;
        pair[i] = u * V;
      } else {
        a[i] = part + (u - rotated) * 2 * V;
        b[i] = a[i] + V;
        pair[i] = u < all ? -1 : -2;
      }
    }
  }
};

// The pairs of a unit: (x[i], x[V + i]) in the half layout, (x[2i], x[2i + 1]) in the interleaved one.
template <int V, bool INTERLEAVED>
__device__ __forceinline__ void rotate_unit(float* x, const float* cs, const float* sn) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int p = INTERLEAVED ? 2 * i : i, q = INTERLEAVED ? 2 * i + 1 : V + i;
    const float a = x[p], b = x[q];
    x[p] = a * cs[i] - b * sn[i];
    x[q] = b * cs[i] + a * sn[i];
  }
}

// The angles of a token's pairs, at `place`: whole turns are dropped in 64 bits.  The place is one wavefront's own, whose LDS accesses stay in order:
// no barrier (which would also wait for the rows that are being written), only that the compiler keeps that order.
__device__ __forceinline__ void put_angles(const RotaryArgs& a, int64_t position, double first_turns, int lane, float2* place) {
  const double pos = (double)position;
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  for (int p = lane; p < a.part / 2; p += 64) {
    const double t = pos * (p == lane ? first_turns : a.turns[p]);
    float sn, cs;
    sincospif(2.0f * (float)(t - floor(t)), &sn, &cs);
    place[p] = make_float2(cs * a.magnitude, (a.transposed ? -sn : sn) * a.magnitude);
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
template <int V, int U, bool INTERLEAVED>
__device__ __forceinline__ void take_angles(const Units<V, U, INTERLEAVED>& unit, const float2* place, float (*cs)[V], float (*sn)[V]) {
#pragma unroll
  for (int i = 0; i < U; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float2 x = unit.pair[i] >= 0 ? place[unit.pair[i] + j] : make_float2(1.0f, 0.0f);
      cs[i][j] = x.x;
      sn[i][j] = x.y;
    }
}

// A wavefront's task: steps [first, end) of a token.
struct Task {
  int64_t token;
  int first, end;
  __device__ __forceinline__ Task(const RotaryArgs& a, int64_t task) {
    token = task / a.chunks;
    first = (int)(task - token * a.chunks) * a.chunk_steps;
    end = min(first + a.chunk_steps, a.steps[0] + a.steps[1]);
  }
};

template <typename T, int V, int U, bool INTERLEAVED, Mode MODE>
__global__ void __launch_bounds__(64 * kWaves) k_rotary(const RotaryArgs a) {
  __shared__ float2 s_angle[kWaves][kMaxWidth / 2];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int lanes = a.lanes, rows = 64 / lanes, row = lane / lanes;
  const Units<V, U, INTERLEAVED> unit(lane % lanes, lanes, a.width, a.part);
  const double turns = lane < a.part / 2 ? a.turns[lane] : 0.0;
  const int64_t stride = (int64_t)gridDim.x * kWaves;
  for (int64_t at = (int64_t)blockIdx.x * kWaves + wave; at < a.tasks; at += stride) {
    const Task task(a, at);
    put_angles(a, a.positions[task.token], turns, lane, s_angle[wave]);
    float cs[U][V], sn[U][V];
    take_angles(unit, s_angle[wave], cs, sn);

#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const int lo = which ? max(task.first - a.steps[0], 0) : task.first;
      const int hi = which ? task.end - a.steps[0] : min(task.end, a.steps[0]);
      if (lo >= hi) continue;
      float w[U][2 * V];
      if constexpr (MODE == kNorm) {
        const T* pw = static_cast<const T*>(a.w[which]);
#pragma unroll
        for (int i = 0; i < U; ++i)
          if (unit.pair[i] > -2) {
            load_vec<V>(pw + unit.a[i], w[i]);
            load_vec<V>(pw + unit.b[i], w[i] + V);
          }
      }
      const T* pin = static_cast<const T*>(a.in[which].p) + task.token * a.in[which].ts;
      T* pout = const_cast<T*>(static_cast<const T*>(a.out[which].p)) + task.token * a.out[which].ts;
      for (int step = lo; step < hi; ++step) {
        const int head = step * rows + row;
        const bool here = head < a.heads[which];
        float x[U][2 * V];
#pragma unroll
        for (int i = 0; i < U; ++i)
          if (here && unit.pair[i] > -2) {
            const T* p = pin + head * a.in[which].hs;
            load_vec<V>(p + unit.a[i], x[i]);
            load_vec<V>(p + unit.b[i], x[i] + V);
          } else {
#pragma unroll
            for (int j = 0; j < 2 * V; ++j) x[i][j] = 0.0f;
          }

        if constexpr (MODE == kNorm) {
          float s = 0.0f;
#pragma unroll
          for (int i = 0; i < U; ++i)
#pragma unroll
            for (int j = 0; j < 2 * V; ++j) s += x[i][j] * x[i][j];
          const float rstd = 1.0f / sqrtf(group_sum(s, lanes) * a.inv_width + a.eps);
#pragma unroll
          for (int i = 0; i < U; ++i)
#pragma unroll
            for (int j = 0; j < 2 * V; ++j) x[i][j] = x[i][j] * rstd * w[i][j];
        }
#pragma unroll
        for (int i = 0; i < U; ++i)
          if (unit.pair[i] >= 0) rotate_unit<V, INTERLEAVED>(x[i], cs[i], sn[i]);
#pragma unroll
        for (int i = 0; i < U; ++i)
          if (here && unit.pair[i] > -2) {
            T* p = pout + head * a.out[which].hs;
            store_vec<V>(p + unit.a[i], x[i]);
            store_vec<V>(p + unit.b[i], x[i] + V);
          }
      }
    }
  }
}

// V entries as they are in memory.
template <typename T, int V>
struct alignas(V * sizeof(T)) Packed {
  T e[V];
  __device__ __forceinline__ void load(const T* p) { *this = *reinterpret_cast<const Packed*>(p); }
  __device__ __forceinline__ void unpack(float* v) const {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = load1(e + i);
  }
};

template <typename T>
struct Packed<T, 1> {
  float e;
  __device__ __forceinline__ void load(const T* p) { e = load1(p); }
  __device__ __forceinline__ void unpack(float* v) const { *v = e; }
};

// The gradients: as above, with the rows of the next step, of the next token after a token's last, under way while one is computed.  8 products and sums an
// element and three rows' traffic: bound by HBM.
template <typename T, int V, int U, bool INTERLEAVED>
__global__ void __launch_bounds__(64 * kWaves, V == 1 ? 2 : 4) k_norm_gradient(const RotaryArgs a) {
  __shared__ float2 s_angle[kWaves][kMaxWidth / 2];
  __shared__ float s_sum[kWaves][kMaxWidth];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int lanes = a.lanes, rows = 64 / lanes, row = lane / lanes;
  const Units<V, U, INTERLEAVED> unit(lane % lanes, lanes, a.width, a.part);
  const double turns = lane < a.part / 2 ? a.turns[lane] : 0.0;
  float dw[2][U][2 * V];
  Packed<T, V> w[2][U][2];
#pragma unroll
  for (int which = 0; which < 2; ++which)
#pragma unroll
    for (int i = 0; i < U; ++i) {
#pragma unroll
      for (int j = 0; j < 2 * V; ++j) dw[which][i][j] = 0.0f;
      if (a.heads[which] && unit.pair[i] > -2) {
        const T* p = static_cast<const T*>(a.w[which]);
        w[which][i][0].load(p + unit.a[i]);
        w[which][i][1].load(p + unit.b[i]);
      }
    }

  Packed<T, V> xs[U][2], gs[U][2];
  auto fetch = [&](int64_t token, int step) {
    const int which = step >= a.steps[0];
    const int head = (which ? step - a.steps[0] : step) * rows + row;
    if (head < (which ? a.heads[1] : a.heads[0])) {
      const View in = which ? a.in[1] : a.in[0], grad = which ? a.grad[1] : a.grad[0];
      const T* p = static_cast<const T*>(in.p) + token * in.ts + head * in.hs;
      const T* q = static_cast<const T*>(grad.p) + token * grad.ts + head * grad.hs;
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (unit.pair[i] > -2) {
          xs[i][0].load(p + unit.a[i]);
          xs[i][1].load(p + unit.b[i]);
          gs[i][0].load(q + unit.a[i]);
          gs[i][1].load(q + unit.b[i]);
        }
    }
  };

  const int64_t stride = (int64_t)gridDim.x * kWaves;
  int64_t at = (int64_t)blockIdx.x * kWaves + wave;
  int64_t position = 0;
  if (at < a.tasks) {
    const Task task(a, at);
    position = a.positions[task.token];
    fetch(task.token, task.first);
  }
  for (; at < a.tasks; at += stride) {
    const Task task(a, at), then(a, at + stride < a.tasks ? at + stride : at);
    put_angles(a, position, turns, lane, s_angle[wave]);
    position = a.positions[then.token];
    float cs[U][V], sn[U][V];
    take_angles(unit, s_angle[wave], cs, sn);

#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const int before = which ? a.steps[0] : 0;
      const int lo = max(task.first, before), hi = which ? task.end : min(task.end, a.steps[0]);
      T* pout = const_cast<T*>(static_cast<const T*>(a.out[which].p)) + task.token * a.out[which].ts;
      for (int step = lo; step < hi; ++step) {
        const int head = (step - before) * rows + row;
        const bool here = head < a.heads[which];
        float x[U][2 * V], g[U][2 * V];
#pragma unroll
        for (int i = 0; i < U; ++i) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            xs[i][h].unpack(x[i] + h * V);
            gs[i][h].unpack(g[i] + h * V);
          }
          if (!here || unit.pair[i] < -1) {      // (nothing to add, whatever its 1 / sqrt(eps))
#pragma unroll
            for (int j = 0; j < 2 * V; ++j) x[i][j] = g[i][j] = 0.0f;
          }
        }
        if (step + 1 < task.end)
          fetch(task.token, step + 1);
        else if (at + stride < a.tasks)
          fetch(then.token, then.first);

        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
          for (int j = 0; j < 2 * V; ++j) s += x[i][j] * x[i][j];
        const float rstd = 1.0f / sqrtf(group_sum(s, lanes) * a.inv_width + a.eps);
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < U; ++i) {
          if (unit.pair[i] >= 0) rotate_unit<V, INTERLEAVED>(g[i], cs[i], sn[i]);
          if (here && unit.pair[i] > -2) {
            float ws[2 * V];
            w[which][i][0].unpack(ws);
            w[which][i][1].unpack(ws + V);
#pragma unroll
            for (int j = 0; j < 2 * V; ++j) {
              x[i][j] *= rstd;                 // x^
              dw[which][i][j] += g[i][j] * x[i][j];
              g[i][j] *= ws[j];
              s += g[i][j] * x[i][j];
            }
          }
        }
        s = group_sum(s, lanes) * a.inv_width;
#pragma unroll
        for (int i = 0; i < U; ++i)
          if (here && unit.pair[i] > -2) {
#pragma unroll
            for (int j = 0; j < 2 * V; ++j) x[i][j] = rstd * (g[i][j] - x[i][j] * s);
            T* p = pout + head * a.out[which].hs;
            store_vec<V>(p + unit.a[i], x[i]);
            store_vec<V>(p + unit.b[i], x[i] + V);
          }
      }
    }
  }

#pragma unroll
  for (int which = 0; which < 2; ++which) {
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int j = 0; j < 2 * V; ++j) {
        float v = dw[which][i][j];
        for (int o = lanes; o < 64; o <<= 1) v += __shfl_xor(v, o);
        if (row == 0 && unit.pair[i] > -2) s_sum[wave][(j < V ? unit.a[i] : unit.b[i] - V) + j] = v;
      }
    __syncthreads();
    for (int c = threadIdx.x; c < a.width; c += 64 * kWaves) {
      float v = 0.0f;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) v += s_sum[i][c];
      a.part_sums[((int64_t)blockIdx.x * 2 + which) * a.width + c] = v;
    }
    __syncthreads();
  }
}

// dw[c] = sum over the workgroups of their sums, 16 columns and 64 interleaved shares a workgroup, in a fixed order.
__global__ void __launch_bounds__(1024) k_weight_sums(const float* __restrict__ part, int groups, int width, float* __restrict__ dq,
                                                      float* __restrict__ dk) {
  __shared__ float s[64][17];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15), share = threadIdx.x >> 4;
  float v = 0.0f;
  if (c < 2 * width) {
#pragma unroll 8
    for (int g = share; g < groups; g += 64) v += part[(int64_t)g * 2 * width + c];
  }
  s[share][threadIdx.x & 15] = v;
  __syncthreads();
  for (int o = 32; o > 0; o >>= 1) {
    if (share < o) s[share][threadIdx.x & 15] += s[share + o][threadIdx.x & 15];
    __syncthreads();
  }
  if (share == 0 && c < 2 * width) {
    float* out = c < width ? dq : dk;
    if (out) out[c < width ? c : c - width] = s[0][threadIdx.x];
  }
}

template <typename T, int V, int U, Mode MODE>
hipError_t launch_layout(const RotaryArgs& a, int layout, int groups, hipStream_t s) {
  if constexpr (MODE == kGrad) {
    if (layout)
      k_norm_gradient<T, V, U, true><<<groups, 64 * kWaves, 0, s>>>(a);
    else
      k_norm_gradient<T, V, U, false><<<groups, 64 * kWaves, 0, s>>>(a);
  } else if (layout) {
    k_rotary<T, V, U, true, MODE><<<groups, 64 * kWaves, 0, s>>>(a);
  } else {
    k_rotary<T, V, U, false, MODE><<<groups, 64 * kWaves, 0, s>>>(a);
  }
  return hipGetLastError();
}

bool aligned(const View& v, int64_t elems, int esz, int heads) {
  if (!heads) return true;
  return reinterpret_cast<uintptr_t>(v.p) % (uint64_t)(elems * esz) == 0 && v.ts % elems == 0 && v.hs % elems == 0;
}

// Vector length: the longest whose units cut both the rotated and the copied part, and at whose alignment every row starts.
int vector_length(const RotaryArgs& a, int esz, Mode mode) {
  for (int v = mode == kGrad ? kGradVector : 16 / esz; v > 1; v = v == 8 ? 4 : 1) {
    if (a.part % (2 * v) || (a.width - a.part) % (2 * v)) continue;
    bool ok = true;
    for (int i = 0; i < 2; ++i) {
      ok = ok && aligned(a.in[i], v, esz, a.heads[i]) && aligned(a.out[i], v, esz, a.heads[i]);
      if (mode == kGrad) ok = ok && aligned(a.grad[i], v, esz, a.heads[i]);
      if (mode != kRotary && a.heads[i]) ok = ok && reinterpret_cast<uintptr_t>(a.w[i]) % (uint64_t)(v * esz) == 0;
    }
    if (ok) return v;
  }
  return 1;
}

template <Mode MODE>
hipError_t launch(RotaryArgs& a, bool f32, int layout, int* groups_out, hipStream_t s) {
  const int v = vector_length(a, f32 ? 4 : 2, MODE);
  const int units = a.width / (2 * v);
  a.lanes = 1;
  while (a.lanes < units && a.lanes < 64) a.lanes *= 2;
  const int rows = 64 / a.lanes;
  for (int i = 0; i < 2; ++i) a.steps[i] = (a.heads[i] + rows - 1) / rows;
  const int steps = a.steps[0] + a.steps[1];
  // A token's heads go to one wavefront, which then takes the angles once for all of them; with fewer tokens than half the 4096
  // wavefronts that the gradient's launch holds at a time they are dealt out until there are as many.
  a.chunks = 1;
  while (a.chunks < steps && a.tokens * a.chunks < kGradGroups * kWaves / 2) ++a.chunks;
  a.chunk_steps = (steps + a.chunks - 1) / a.chunks;
  a.chunks = (steps + a.chunk_steps - 1) / a.chunk_steps;
  a.tasks = a.tokens * a.chunks;
  int64_t groups = (a.tasks + kWaves - 1) / kWaves;
  const int64_t most = MODE == kGrad ? kGradGroups : 1 << 20;
  if (groups > most) groups = most;
  *groups_out = (int)groups;
  if (f32) {
    if (v == 4) return launch_layout<float, 4, 1, MODE>(a, layout, (int)groups, s);
    return launch_layout<float, 1, 4, MODE>(a, layout, (int)groups, s);
  }
  if constexpr (MODE != kGrad) {
    if (v == 8) return launch_layout<bf16_bits, 8, 1, MODE>(a, layout, (int)groups, s);
  }
  if (v == 4) return launch_layout<bf16_bits, 4, 1, MODE>(a, layout, (int)groups, s);
  return launch_layout<bf16_bits, 1, 4, MODE>(a, layout, (int)groups, s);
}

constexpr int64_t kMaxStride = 1ll << 40;

// An input may have any strides, 0 among them (one row for all heads or tokens); an output's rows must not overlap.
bool view_of(const conqur_heads& h, uint32_t width, int64_t tokens, int esz, bool output, View* out) {
  if (!h.data || reinterpret_cast<uintptr_t>(h.data) % esz) return false;
  if (h.token_stride < 0 || h.token_stride >= kMaxStride || h.head_stride < 0 || h.head_stride >= kMaxStride) return false;
  if (output) {
    const __int128 w = width, ts = h.token_stride, hs = h.head_stride;
    if ((h.heads > 1 && hs < w) || (tokens > 1 && ts < w)) return false;
    if (h.heads > 1 && tokens > 1 && ts < (h.heads - 1) * hs + w && hs < (tokens - 1) * ts + w) return false;
  }
  *out = View{h.data, h.token_stride, h.head_stride};
  return true;
}

// Checks a call's arguments and fills the kernel's; false: CONQUR_EINVAL.
bool fill(const conqur_rotary_call* c, Mode mode, RotaryArgs* a) {
  if (!c || (c->dtype != CONQUR_F32 && c->dtype != CONQUR_BF16) || c->layout > CONQUR_INTERLEAVED || c->transposed > 1) return false;
  if (c->width < 2 || c->width > (uint32_t)kMaxWidth || c->width % 2 || c->part < 2 || c->part > c->width || c->part % 2) return false;
  if (c->tokens >= (1ull << 31)) return false;
  if (c->q.heads + (uint64_t)c->k.heads < 1 || c->q.heads > 65536 || c->k.heads > 65536) return false;
  if (!isfinite(c->magnitude)) return false;
  if (mode != kRotary && !(c->eps >= 0.0f && isfinite(c->eps))) return false;
  if (mode != kRotary && c->transposed) return false;
  *a = RotaryArgs{};
  a->tokens = (int64_t)c->tokens;
  if (a->tokens == 0) return true;
  if (!c->positions || !c->turns || reinterpret_cast<uintptr_t>(c->positions) % 8 || reinterpret_cast<uintptr_t>(c->turns) % 8) return false;
  const int esz = c->dtype == CONQUR_F32 ? 4 : 2;
  const conqur_heads* in[2] = {&c->q, &c->k};
  const conqur_heads* out[2] = {&c->q_out, &c->k_out};
  const conqur_heads* grad[2] = {&c->q_grad, &c->k_grad};
  const void* w[2] = {c->q_weight, c->k_weight};
  for (int i = 0; i < 2; ++i) {
    a->heads[i] = (int)in[i]->heads;
    if (!a->heads[i]) continue;
    if (out[i]->heads != in[i]->heads) return false;
    if (!view_of(*in[i], c->width, a->tokens, esz, false, &a->in[i]) || !view_of(*out[i], c->width, a->tokens, esz, true, &a->out[i])) return false;
    if (mode != kRotary && (!w[i] || reinterpret_cast<uintptr_t>(w[i]) % esz)) return false;
    a->w[i] = w[i];
    if (mode == kGrad && (grad[i]->heads != in[i]->heads || !view_of(*grad[i], c->width, a->tokens, esz, false, &a->grad[i]))) return false;
  }
  a->positions = c->positions;
  a->turns = c->turns;
  a->width = (int)c->width;
  a->part = (int)c->part;
  a->magnitude = c->magnitude;
  a->eps = c->eps;
  a->inv_width = 1.0f / (float)c->width;
  a->transposed = (int)c->transposed;
  return true;
}

}  // namespace

extern "C" conqur_status conqur_rotary_frequencies(uint32_t part, uint32_t scaling, double theta, double factor, double low, double high,
                                                   double context, double* turns_host, float* magnitude_host) {
  if (!turns_host || !magnitude_host || part < 2 || part > (uint32_t)kMaxWidth || part % 2 || scaling > CONQUR_SCALE_RAMP) return CONQUR_EINVAL;
  if (!(theta > 1.0) || !isfinite(theta)) return CONQUR_EINVAL;
  if (scaling != CONQUR_SCALE_NONE && (!(factor >= 1.0) || !isfinite(factor))) return CONQUR_EINVAL;
  if (scaling == CONQUR_SCALE_BASE && part < 4) return CONQUR_EINVAL;
  const bool bounded = scaling == CONQUR_SCALE_BANDS || scaling == CONQUR_SCALE_RAMP;
  if (bounded && (!(low > 0.0) || !(high > low) || !isfinite(high) || !(context > 0.0) || !isfinite(context))) return CONQUR_EINVAL;
  const double two_pi = 6.283185307179586476925;
  const double n = (double)part;
  const double base = scaling == CONQUR_SCALE_BASE ? theta * pow(factor, n / (n - 2.0)) : theta;
  // The pair that makes `r` turns within the context: theta^(-2j/n) context / (2 pi) = r.
  auto pair_of = [&](double r) { return n * log(context / (r * two_pi)) / (2.0 * log(theta)); };
  const double from = bounded ? fmax(floor(pair_of(high)), 0.0) : 0.0;
  const double to = bounded ? fmin(ceil(pair_of(low)), n - 1.0) : 0.0;
  for (uint32_t j = 0; j < part / 2; ++j) {
    const double t = pow(base, -2.0 * j / n) / two_pi;
    double keep = 1.0;                       // share of the unscaled frequency
    if (scaling == CONQUR_SCALE_LINEAR) keep = 0.0;
    if (scaling == CONQUR_SCALE_BANDS) keep = fmin(fmax((t * context - low) / (high - low), 0.0), 1.0);
    if (scaling == CONQUR_SCALE_RAMP) keep = 1.0 - fmin(fmax((j - from) / fmax(to - from, 1e-3), 0.0), 1.0);
    const bool scaled = scaling != CONQUR_SCALE_NONE && scaling != CONQUR_SCALE_BASE;
    turns_host[j] = scaled ? keep * t + (1.0 - keep) * t / factor : t;
  }
  *magnitude_host = scaling == CONQUR_SCALE_RAMP ? (float)(0.1 * log(factor) + 1.0) : 1.0f;
  return CONQUR_OK;
}

extern "C" conqur_status conqur_rotary(const conqur_rotary_call* call, void* stream) {
  RotaryArgs a;
  if (!fill(call, kRotary, &a)) return CONQUR_EINVAL;
  if (!a.tokens) return CONQUR_OK;
  int groups;
  return launch<kRotary>(a, call->dtype == CONQUR_F32, (int)call->layout, &groups, reinterpret_cast<hipStream_t>(stream)) == hipSuccess ? CONQUR_OK
                                                                                                                                       : CONQUR_EHIP;
}

extern "C" conqur_status conqur_qk_norm_rotary(const conqur_rotary_call* call, void* stream) {
  RotaryArgs a;
  if (!fill(call, kNorm, &a)) return CONQUR_EINVAL;
  if (!a.tokens) return CONQUR_OK;
  int groups;
  return launch<kNorm>(a, call->dtype == CONQUR_F32, (int)call->layout, &groups, reinterpret_cast<hipStream_t>(stream)) == hipSuccess ? CONQUR_OK
                                                                                                                                     : CONQUR_EHIP;
}

extern "C" uint64_t conqur_qk_norm_rotary_workspace(uint32_t width) {
  return (uint64_t)kGradGroups * 2 * (width < (uint32_t)kMaxWidth ? width : (uint32_t)kMaxWidth) * sizeof(float);
}

extern "C" conqur_status conqur_qk_norm_rotary_backward(const conqur_rotary_call* call, float* q_weight_grad, float* k_weight_grad, void* workspace,
                                                        uint64_t workspace_bytes, void* stream) {
  RotaryArgs a;
  if (!fill(call, kGrad, &a)) return CONQUR_EINVAL;
  if ((call->q.heads && !q_weight_grad) || (call->k.heads && !k_weight_grad) || !workspace) return CONQUR_EINVAL;
  if (reinterpret_cast<uintptr_t>(q_weight_grad) % 4 || reinterpret_cast<uintptr_t>(k_weight_grad) % 4) return CONQUR_EINVAL;
  if (reinterpret_cast<uintptr_t>(workspace) % 16 || workspace_bytes < conqur_qk_norm_rotary_workspace(call->width)) return CONQUR_EINVAL;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  a.part_sums = static_cast<float*>(workspace);
  a.transposed = 1;
  int groups = 0;
  if (a.tokens && launch<kGrad>(a, call->dtype == CONQUR_F32, (int)call->layout, &groups, s) != hipSuccess) return CONQUR_EHIP;
  const int width = (int)call->width;
  k_weight_sums<<<(2 * width + 15) / 16, 1024, 0, s>>>(a.part_sums, groups, width, call->q.heads ? q_weight_grad : nullptr,
                                                       call->k.heads ? k_weight_grad : nullptr);
  return hipGetLastError() == hipSuccess ? CONQUR_OK : CONQUR_EHIP;
}
