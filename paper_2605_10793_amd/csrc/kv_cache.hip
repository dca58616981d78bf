// Appending keys and values to a paged cache of bf16 rows or of zero-point codes of 8 or 4 bits.
//
//   per token and head: lo, hi over the row, step = (hi - lo) / (2^b - 1), zeta = -rint(lo / step), offset = -step zeta,
//   code = clamp(rint(y / step) + zeta, 0, 2^b - 1); value = step code + offset
//
// Bound by HBM: rows are read once, codes written once.  Keys lie as they come, but values lie with the tokens of a page side by
// side (attention contracts over tokens and reads them straight into matrix operands), so a workgroup takes the tokens of one head
// that fall into one block of 64 slots and turns them round in LDS; whole groups of 16 slots leave as 16-byte stores, the slots
// at a batch's ragged ends one by one.  W/16 lanes hold a row, both halves' entries of a code byte in the same lane, so that packing and
// the row's extremes stay in registers.
//
// Measured: 8 prompts of 517 to 2048 tokens (8 heads of 128) into 16-bit pages 17.7 to 18.9 us (4.4 to 4.7 TB/s read and written), into 4 or 8 bits with
// the values emitted 26 and 26.5 (3.7 and 4.0 TB/s); a token of each of 64 sequences into 4 bits, values emitted, 10.9 us a call, of which the
// kernel is 5.7: a chain of four reads (bounds, page, row, ...), then single bytes.
#include "../../include/conqur.h"

#include "kernels.h"

using namespace conqur;

namespace {

constexpr int kBlock = 64;        // slots of a workgroup
constexpr int kThreads = 256;
static_assert(kBlock == 64, "shifts by 6");
constexpr int kScan = 512;        // sequences among which a workgroup looks at each

struct AppendArgs {
  conqur_cache cache;
  conqur_batch batch;
  const bf16_bits* in[2];
  int64_t in_ts[2], in_hs[2];
  bf16_bits* val[2];              // null: not wanted
  int64_t val_ts[2], val_hs[2];
  int64_t tokens;
  int wide[2], val_wide[2];       // rows start at multiples of 16 bytes
  int first_block;                // number of the launch's first workgroup
};

__device__ __forceinline__ int clamp_to(int v, int64_t hi) { return v < 0 ? 0 : v > hi ? (int)hi : v; }

template <int CTRL>
__device__ __forceinline__ float lane_perm(float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// Over the 4 or 8 neighbouring lanes of a row.
template <int LANES, typename Op>
__device__ __forceinline__ float row_reduce(float v, Op op) {
  v = op(v, lane_perm<0xB1>(v));
  v = op(v, lane_perm<0x4E>(v));
  if constexpr (LANES > 4) v = op(v, lane_perm<0x141>(v));
  return v;
}

__device__ __forceinline__ void load16(const bf16_bits* p, int half, bool wide, uint32_t* u) {
  if (wide) {
    const uint4 a = *reinterpret_cast<const uint4*>(p), b = *reinterpret_cast<const uint4*>(p + half);
    u[0] = a.x; u[1] = a.y; u[2] = a.z; u[3] = a.w;
    u[4] = b.x; u[5] = b.y; u[6] = b.z; u[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u[i] = p[2 * i] | (uint32_t)p[2 * i + 1] << 16;
      u[4 + i] = p[half + 2 * i] | (uint32_t)p[half + 2 * i + 1] << 16;
    }
  }
}
__device__ __forceinline__ void store16(bf16_bits* p, int half, bool wide, const uint32_t* u) {
  if (wide) {
    *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
    *reinterpret_cast<uint4*>(p + half) = make_uint4(u[4], u[5], u[6], u[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      p[2 * i] = (bf16_bits)u[i];
      p[2 * i + 1] = (bf16_bits)(u[i] >> 16);
      p[half + 2 * i] = (bf16_bits)u[4 + i];
      p[half + 2 * i + 1] = (bf16_bits)(u[4 + i] >> 16);
    }
  }
}

// Codes of a lane's 16 entries (two runs of 8), four to a word, and the row's pair; every operation rounds on its own, as the
// definition has it.
template <int BITS, int LANES>
__device__ __forceinline__ void quantise(const uint32_t* u, uint32_t* code, float2* pair, uint32_t* values) {
#pragma clang fp contract(off)
  float y[16];
#pragma unroll
  for (int i = 0; i < 8; ++i) { y[2 * i] = __uint_as_float(u[i] << 16); y[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
  float lo = y[0], hi = y[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) { lo = fminf(lo, y[i]); hi = fmaxf(hi, y[i]); }
  lo = row_reduce<LANES>(lo, [](float a, float b) { return fminf(a, b); });
  hi = row_reduce<LANES>(hi, [](float a, float b) { return fmaxf(a, b); });
  constexpr float kTop = (float)((1 << BITS) - 1);
  const float step = (hi - lo) / kTop;
  const bool flat = step == 0.0f;
  const float safe = flat ? 1.0f : step;
  const float zeta = -rintf(lo / safe);
  const float offset = flat ? lo : -(step * zeta);
  *pair = make_float2(step, offset);
  float q[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float c = fminf(fmaxf(rintf(y[i] / safe) + zeta, 0.0f), kTop);
    q[i] = flat ? 0.0f : c;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    code[i] = (uint32_t)q[4 * i] | (uint32_t)q[4 * i + 1] << 8 | (uint32_t)q[4 * i + 2] << 16 | (uint32_t)q[4 * i + 3] << 24;
  if (values) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float a = step * q[2 * i], b = step * q[2 * i + 1];
      values[i] = f32x2_to_bf16x2(a + offset, b + offset);
    }
  }
}

// (69 registers, seven wavefronts a SIMD: left to itself the compiler takes 77 and six, a token of 2000 sequences in 4 bits 62.7 us for 59.1)
template <int BITS, int W>
__global__ void __launch_bounds__(kThreads, 7) k_append(const AppendArgs a) {
  constexpr int kLanes = W / 16;                                   // lanes of a row
  constexpr int kRows = kThreads / kLanes / 2;                     // tokens at a time
  constexpr int kBytes = BITS == 16 ? 2 * W : W * BITS / 8;        // bytes of a row in the cache
  constexpr int kPitch = kBytes + 4;                               // in LDS
  __shared__ __attribute__((aligned(16))) unsigned char s_v[kBlock * kPitch];

  // Sequence b's blocks are those from start[b] / 64 + 2b on, to start[b + 1] / 64 + 2b + 1: enough for every count and place (n tokens touch at
  // most n / 64 + 2 blocks of slots).  Where starts rise a block is one sequence's or no one's; where one falls, whose sequence has no tokens,
  // blocks of those before and behind it may have one number, and a workgroup does them all.
  const int id = a.first_block + (int)blockIdx.x;        // below 2^26
  const int head = blockIdx.y;
  const int sequences = (int)a.batch.sequences;
  auto bound = [&](int x) { return clamp_to(a.batch.start[x], a.tokens); };
  auto owns = [&](int x, int from, int to) { return from < to && (from >> 6) + 2 * x <= id && id <= (to >> 6) + 2 * x + 1; };
  // Each lane of a wavefront asks for one sequence: one read for up to 64 of them.  Of up to 512, first which 64 hold any; of more, the last 64 whose
  // first block is not behind this one, which are those that hold it if starts rise.  (A token of each of 512 sequences, 16 bits: 17.3 us, and 15.3
  // by the second way, which a fall leads astray.)
  const int me = threadIdx.x & 63;
  uint32_t some = 1;                 // bit c: the 64 sequences from 64 (group + c) on
  int group = 0;
  if (sequences > kScan) {
    for (int step = sequences <= 4096 ? 64 : 4096; step > 1; step /= 64) {
      const int x = group * 64 + me * step;
      const int first = x < sequences ? bound(x) : 0;
      group += (max(__popcll(__ballot(x < sequences && (first >> 6) + 2 * x <= id)), 1) - 1) * (step / 64);
    }
  } else if (sequences > 64) {
    // (each wavefront looks among 128 of them)
    __shared__ uint32_t s_some[kThreads / 64];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    some = 0;
#pragma unroll
    for (int c = 0; c < kScan / kThreads; ++c) {
      const int chunk = wave * (kScan / kThreads) + c, x = 64 * chunk + me;
      if (64 * chunk < sequences)
        some |= (uint32_t)(__any(x < sequences && owns(x, bound(min(x, sequences)), bound(min(x + 1, sequences)))) != 0) << chunk;
    }
    if (me == 0) s_some[wave] = some;
    __syncthreads();
    some = s_some[0] | s_some[1] | s_some[2] | s_some[3];
    some = (uint32_t)__builtin_amdgcn_readfirstlane((int)some);
  }
  bool again = false;
  for (; some; some &= some - 1) {
  const int base_x = 64 * (group + __builtin_ctz(some));
  int lane_from = 0, lane_to = 0, lane_before = 0;       // a sequence, its tokens, its prefix
  if (base_x + me < sequences) {
    lane_from = bound(base_x + me);
    lane_to = bound(base_x + me + 1);
    lane_before = a.batch.prefix[base_x + me];
  }
  for (uint64_t hits = __ballot(owns(base_x + me, lane_from, lane_to)); hits; hits &= hits - 1) {
  const int n = __builtin_ctzll(hits), b = base_x + n;
  const int from = __builtin_amdgcn_readlane(lane_from, n), to = __builtin_amdgcn_readlane(lane_to, n), before = __builtin_amdgcn_readlane(lane_before, n);
  const int64_t first = from, count = (int64_t)to - from, prefix = before < 0 ? 0 : before;
  const int page_tokens = (int)a.cache.page_tokens, page_shift = 31 - __builtin_clz(page_tokens);
  const int64_t room = (int64_t)a.batch.table_columns * page_tokens;
  const int64_t end = prefix + count < room ? prefix + count : room;
  const int64_t k = id - ((from >> 6) + 2 * b);
  const int64_t base = ((prefix >> 6) + k) * kBlock;             // first slot of the block, as a token number of the sequence
  if (base >= end || base + kBlock <= prefix) continue;
  if (again) __syncthreads();        // what the block before has in LDS has been read
  again = true;
  const int32_t* table = a.batch.table + (int64_t)b * a.batch.table_stride;
  const int64_t heads = a.cache.heads;

  // Neighbouring groups of lanes hold a token's key and its value: the same instructions for both (a few tokens wait for them to be read from
  // memory: 9.5 us for a token of 64 sequences with a copy of them for each, 6.2 us so), and both under way together.
  const int lane = threadIdx.x % kLanes, which = threadIdx.x / kLanes % 2;
  const bf16_bits* in = which ? a.in[1] : a.in[0];
  const int64_t in_ts = which ? a.in_ts[1] : a.in_ts[0], in_hs = which ? a.in_hs[1] : a.in_hs[0];
  const bool wide = which ? a.wide[1] : a.wide[0];
  for (int r = threadIdx.x / kLanes / 2; r < kBlock; r += kRows) {
    const int64_t pos = base + r;
    if (pos < prefix || pos >= end) continue;
    const int32_t page = table[pos >> page_shift];
    if (page < 0 || (uint64_t)page >= a.cache.pages) continue;
    const int64_t token = first + pos - prefix;
    const int64_t at = ((int64_t)page * heads + head) * page_tokens + (pos & (page_tokens - 1));
    uint32_t u[8];
    load16(in + token * in_ts + head * in_hs + 8 * lane, W / 2, wide, u);
    if constexpr (BITS == 16) {
      if (which == 0) {
        store16(static_cast<bf16_bits*>(a.cache.k) + at * W + 8 * lane, W / 2, true, u);
      } else {
        uint32_t* s = reinterpret_cast<uint32_t*>(s_v + r * kPitch);
#pragma unroll
        for (int i = 0; i < 4; ++i) { s[4 * lane + i] = u[i]; s[W / 4 + 4 * lane + i] = u[4 + i]; }
      }
    } else {
      uint32_t code[4], values[8];
      float2 pair;
      quantise<BITS, kLanes>(u, code, &pair, values);
      if (bf16_bits* val = which ? a.val[1] : a.val[0]) {
        const int64_t val_ts = which ? a.val_ts[1] : a.val_ts[0], val_hs = which ? a.val_hs[1] : a.val_hs[0];
        store16(val + token * val_ts + head * val_hs + 8 * lane, W / 2, which ? a.val_wide[1] : a.val_wide[0], values);
      }
      if (lane == 0) reinterpret_cast<float2*>(which ? a.cache.v_scale : a.cache.k_scale)[at] = pair;
      uint32_t* s = reinterpret_cast<uint32_t*>(s_v + r * kPitch);
      if constexpr (BITS == 4) {
        const uint32_t x = code[0] | code[2] << 4, y = code[1] | code[3] << 4;
        if (which == 0) {
          *reinterpret_cast<uint2*>(static_cast<unsigned char*>(a.cache.k) + at * (W / 2) + 8 * lane) = make_uint2(x, y);
        } else {
          s[2 * lane] = x;
          s[2 * lane + 1] = y;
        }
      } else {
        if (which == 0) {
          unsigned char* p = static_cast<unsigned char*>(a.cache.k) + at * W + 8 * lane;
          *reinterpret_cast<uint2*>(p) = make_uint2(code[0], code[1]);
          *reinterpret_cast<uint2*>(p + W / 2) = make_uint2(code[2], code[3]);
        } else {
          s[2 * lane] = code[0];
          s[2 * lane + 1] = code[1];
          s[W / 8 + 2 * lane] = code[2];
          s[W / 8 + 2 * lane + 1] = code[3];
        }
      }
    }
  }
  __syncthreads();

  // Values: row d of the page holds byte (bf16: entry) d of every token; a unit is 16 slots of one row.
  constexpr int kSize = BITS == 16 ? 2 : 1;
  constexpr int kOut = kBytes / kSize;
  for (int u = threadIdx.x; u < kOut * (kBlock / 16); u += kThreads) {
    const int d = u / (kBlock / 16), group = u % (kBlock / 16);
    const int64_t pos = base + group * 16;
    if (pos + 16 <= prefix || pos >= end) continue;
    const int32_t page = table[pos >> page_shift];
    if (page < 0 || (uint64_t)page >= a.cache.pages) continue;
    unsigned char* out = static_cast<unsigned char*>(a.cache.v) +
                         ((((int64_t)page * heads + head) * kOut + d) * page_tokens + (pos & (page_tokens - 1))) * kSize;
    const unsigned char* s = s_v + group * 16 * kPitch + d * kSize;
    if (pos >= prefix && pos + 16 <= end) {
      uint32_t w[4 * kSize];
      if constexpr (BITS == 16) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          w[i] = *reinterpret_cast<const bf16_bits*>(s + 2 * i * kPitch) | (uint32_t)*reinterpret_cast<const bf16_bits*>(s + (2 * i + 1) * kPitch) << 16;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          w[i] = s[4 * i * kPitch] | (uint32_t)s[(4 * i + 1) * kPitch] << 8 | (uint32_t)s[(4 * i + 2) * kPitch] << 16 |
                 (uint32_t)s[(4 * i + 3) * kPitch] << 24;
      }
#pragma unroll
      for (int i = 0; i < kSize; ++i) reinterpret_cast<uint4*>(out)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    } else {
      const int from_slot = pos < prefix ? (int)(prefix - pos) : 0, to_slot = end - pos < 16 ? (int)(end - pos) : 16;
#pragma unroll 1
      for (int i = from_slot; i < to_slot; ++i) {
        if constexpr (BITS == 16)
          reinterpret_cast<bf16_bits*>(out)[i] = *reinterpret_cast<const bf16_bits*>(s + i * kPitch);
        else
          out[i] = s[i * kPitch];
      }
    }
  }
  }
  }
}

constexpr int64_t kMaxStride = 1ll << 40;

bool strides_fine(const conqur_heads& h, uint32_t width, uint64_t tokens, bool output) {
  if (!h.data || reinterpret_cast<uintptr_t>(h.data) % 2) return false;
  if (h.token_stride < 0 || h.token_stride >= kMaxStride || h.head_stride < 0 || h.head_stride >= kMaxStride) return false;
  if (!output) return true;
  const __int128 w = width, ts = h.token_stride, hs = h.head_stride, heads = h.heads, n = tokens;
  if ((heads > 1 && hs < w) || (n > 1 && ts < w)) return false;
  return !(heads > 1 && n > 1 && ts < (heads - 1) * hs + w && hs < (n - 1) * ts + w);
}

bool is_wide(const conqur_heads& h) {
  return reinterpret_cast<uintptr_t>(h.data) % 16 == 0 && h.token_stride % 8 == 0 && h.head_stride % 8 == 0;
}

constexpr uint32_t kMostBlocks = 1u << 23;      // of a launch: a grid's threads are counted in 32 bits

template <int BITS>
void launch_width(AppendArgs a, uint32_t blocks, hipStream_t s) {
  for (uint32_t done = 0; done < blocks; done += kMostBlocks) {
    const dim3 grid(blocks - done < kMostBlocks ? blocks - done : kMostBlocks, a.cache.heads);
    a.first_block = (int)done;
    if (a.cache.width == 128)
      k_append<BITS, 128><<<grid, kThreads, 0, s>>>(a);
    else
      k_append<BITS, 64><<<grid, kThreads, 0, s>>>(a);
  }
}

}  // namespace

namespace conqur {

bool cache_fine(const conqur_cache& c) {
  if (c.bits != 16 && c.bits != 8 && c.bits != 4) return false;
  if (c.width != 64 && c.width != 128) return false;
  if (c.page_tokens < 16 || c.page_tokens > 256 || (c.page_tokens & (c.page_tokens - 1))) return false;
  if (c.heads < 1 || c.heads > 65535 || c.pages < 1 || c.pages >= (1ull << 31)) return false;
  if (!c.k || !c.v || reinterpret_cast<uintptr_t>(c.k) % 16 || reinterpret_cast<uintptr_t>(c.v) % 16) return false;
  if (c.bits != 16 && (!c.k_scale || !c.v_scale || reinterpret_cast<uintptr_t>(c.k_scale) % 16 || reinterpret_cast<uintptr_t>(c.v_scale) % 16)) return false;
  return true;
}

bool batch_fine(const conqur_batch& b) {
  if (!b.start || !b.prefix || !b.table) return false;
  if ((reinterpret_cast<uintptr_t>(b.start) | reinterpret_cast<uintptr_t>(b.prefix) | reinterpret_cast<uintptr_t>(b.table)) % 4) return false;
  if (b.sequences < 1 || b.sequences > 65535 || b.table_columns < 1 || b.table_columns >= (1u << 31)) return false;
  return b.table_stride >= (int64_t)b.table_columns && b.table_stride < kMaxStride;
}

}  // namespace conqur

extern "C" conqur_status conqur_cache_append(const conqur_append_call* c, void* stream) {
  if (!c || !cache_fine(c->cache) || !batch_fine(c->batch) || c->tokens >= (1ull << 31)) return CONQUR_EINVAL;
  if (c->tokens == 0) return CONQUR_OK;
  AppendArgs a;
  a.cache = c->cache;
  a.batch = c->batch;
  a.tokens = (int64_t)c->tokens;
  const conqur_heads* in[2] = {&c->k, &c->v};
  const conqur_heads* val[2] = {&c->k_values, &c->v_values};
  for (int i = 0; i < 2; ++i) {
    if (in[i]->heads != c->cache.heads || !strides_fine(*in[i], c->cache.width, c->tokens, false)) return CONQUR_EINVAL;
    a.in[i] = static_cast<const bf16_bits*>(in[i]->data);
    a.in_ts[i] = in[i]->token_stride;
    a.in_hs[i] = in[i]->head_stride;
    a.wide[i] = is_wide(*in[i]);
    a.val[i] = nullptr;
    a.val_ts[i] = a.val_hs[i] = 0;
    a.val_wide[i] = 0;
    if (!val[i]->heads) continue;
    if (c->cache.bits == 16 || val[i]->heads != c->cache.heads || !strides_fine(*val[i], c->cache.width, c->tokens, true)) return CONQUR_EINVAL;
    a.val[i] = static_cast<bf16_bits*>(val[i]->data);
    a.val_ts[i] = val[i]->token_stride;
    a.val_hs[i] = val[i]->head_stride;
    a.val_wide[i] = is_wide(*val[i]);
  }
  const uint32_t blocks = (uint32_t)(c->tokens / kBlock + 2 * (uint64_t)c->batch.sequences);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (c->cache.bits == 16)
    launch_width<16>(a, blocks, s);
  else if (c->cache.bits == 8)
    launch_width<8>(a, blocks, s);
  else
    launch_width<4>(a, blocks, s);
  return hipGetLastError() == hipSuccess ? CONQUR_OK : CONQUR_EHIP;
}
