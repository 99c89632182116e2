// Around an 8-bit K/V cache: rotary positions, quantising new K/V rows into the cache, reading tokens back as bf16.
//
// Format.  A row is one token's K or V of one KV head, x[0 .. D).  With a = max |x| it is stored as D one-byte codes
// round(x * (top * (1 / a))) and one fp32 scale a * (1 / top); top is the largest code, 448 (e4m3) or 127 (int8).  A row of a < 2^-110
// is stored as zeros with scale 0 (top / a would leave the range of fp32); a row that holds an infinity or a NaN has scale NaN and
// zero codes: codes are finite always, so a masked token of any content cannot reach a matrix product.  The codes lie as
// the bf16 caches do ([page, slot, KV head, dim], strides of the caller's), the scales as [page, KV head, K or V, slot], so that the
// attention kernels read a page's 2 x 16 scales of their head as one 128-byte line.
//
// Rotary positions.  Pair i of a head's first `rot` dims is turned by angle p f_i.  Angles are formed and reduced to a
// fraction of a turn in 64 bits (32 lose 0.01 rad at 10^5 positions), sine and cosine and the rotation are 32-bit.
//
// All three kernels are elementwise passes: what bounds a large call is memory, a small one its launch and two dependent
// round trips (the length or position, then the rows or page).  A lane has 16 elements of a row, 8 of each half of its pairs.
#pragma once
#include "select_blocks.hpp"
#include "vegas_common.hpp"

namespace vegas {

constexpr int kE4m3 = 0, kInt8 = 1;           // VEGAS_QUANT_*
constexpr int kRopeHalf = 0;                  // VEGAS_ROPE_HALF (1: interleaved)
constexpr int kUnit = 16;                     // elements of a row that one lane has

struct RopeParams {
  const double* inv_freq;   // [rot / 2] radians per position
  float magnitude;
  int32_t rot, layout;
};

struct RotateParams {
  RopeParams rope;
  const int32_t* positions; // [N]
  const uint16_t* x;        // bf16 [N, H, D]
  uint16_t* out;
  int64_t x_token, x_head, out_token, out_head;      // strides
  int32_t N, H;
  int32_t steps;            // steps of 64 / (D / 16) heads that one wave takes
};

struct QuantAppendParams {
  RopeParams rope;          // inv_freq == nullptr: no rotation
  const uint16_t* k_new;    // bf16 [B, T, Hkv, D]
  const uint16_t* v_new;
  const uint16_t* q;        // or nullptr; bf16 [B, T, Hq, D]
  uint16_t* q_out;
  const int32_t* new_lens;  // or nullptr
  int64_t kv_token, q_token, q_out_token;            // strides between tokens
  uint8_t* k_cache;
  uint8_t* v_cache;
  float* scales;
  const int32_t* block_table;
  const int32_t* seq_lens;
  int32_t* seq_lens_out;
  int32_t T, Hkv, Hq, max_blocks, max_tokens;
  int32_t steps;            // of a wave and token
  int64_t page_stride, token_stride, head_stride, num_pages;
  ExtendParams grow;        // sel_table != nullptr: the selection grows by the same tokens
};

struct QuantReadParams {
  const uint8_t* k_cache;
  const uint8_t* v_cache;
  const float* scales;
  const int32_t* table;     // [B, table_stride]
  const int32_t* lens;
  const int32_t* first;     // or nullptr
  uint16_t* k_out;          // bf16 [B, T, Hkv, D]
  uint16_t* v_out;
  int32_t T, Hkv, table_stride, max_tokens, page_shift;
  int64_t page_stride, token_stride, head_stride, num_pages;
};

// ---------------------------------------------------------------------------------------------------------- rotation

// (cos, sin) * magnitude of position pos: lane i works out pair i.
__device__ __forceinline__ f32x2 lane_angle(const RopeParams& rope, double freq, int pos) {
  const double turns = static_cast<double>(pos) * freq * 0.15915494309189533577;   // 1 / (2 pi)
  const float part = static_cast<float>(turns - __builtin_rint(turns));             // exact difference, in [-1/2, 1/2]
  float s, c;
  sincospif(2.0f * part, &s, &c);
  return f32x2{c * rope.magnitude, s * rope.magnitude};
}
// Those of pairs 8 u .. 8 u + 7 (u: this lane's unit), out of 64 in LDS.
__device__ __forceinline__ void read_angles(const f32x2* lds, int u, f32x2 (&cs)[8]) {
  const f32x4* at = reinterpret_cast<const f32x4*>(lds + 8 * min(u, 7));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x4 two = at[i];
    cs[2 * i] = f32x2{two[0], two[1]};
    cs[2 * i + 1] = f32x2{two[2], two[3]};
  }
}
__device__ __forceinline__ void unit_angles(const RopeParams& rope, double freq, int pos, f32x2* lds, int u, f32x2 (&cs)[8]) {
  const f32x2 mine = lane_angle(rope, freq, pos);
  wave_lds_fence();                           // (the last token's pairs have been read)
  lds[threadIdx.x & 63] = mine;
  wave_lds_fence();
  read_angles(lds, u, cs);
}
__device__ __forceinline__ double lane_frequency(const RopeParams& rope) {
  const int lane = threadIdx.x & 63;
  return lane < (rope.rot >> 1) ? rope.inv_freq[lane] : 0.0;
}

// Where the two eights of this lane's unit lie in the row.
struct UnitAt {
  int a, b;
  bool turned;
};
__device__ __forceinline__ UnitAt unit_at(const RopeParams& rope, bool rotates, int u) {
  UnitAt at;
  at.turned = rotates && u < (rope.rot >> 4);
  const bool apart = at.turned && rope.layout == kRopeHalf;
  at.a = apart ? 8 * u : 16 * u;
  at.b = apart ? (rope.rot >> 1) + 8 * u : 16 * u + 8;
  return at;
}
__device__ __forceinline__ void widen(const u32x4& raw, float* x) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(raw[e] << 16);
    x[2 * e + 1] = __uint_as_float(raw[e] & 0xffff0000u);
  }
}
__device__ __forceinline__ u32x4 narrow(const float* x) {     // to nearest even, NaN kept
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  u32x4 raw;
#pragma unroll
  for (int e = 0; e < 4; ++e) raw[e] = __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(x[2 * e]), static_cast<__bf16>(x[2 * e + 1])});
  return raw;
}
__device__ __forceinline__ void turn(float& a, float& b, const f32x2& cs) {
  const float x = a, y = b;
  a = x * cs[0] - y * cs[1];
  b = x * cs[1] + y * cs[0];
}
__device__ __forceinline__ void turn_unit(const RopeParams& rope, float (&x)[kUnit], const f32x2 (&cs)[8]) {
  if (rope.layout == kRopeHalf) {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn(x[i], x[8 + i], cs[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn(x[2 * i], x[2 * i + 1], cs[i]);
  }
}

// A wave per token and `steps` steps of heads; four steps' requests leave together.
template <int D>
__global__ __launch_bounds__(256) void rotate_kernel(const RotateParams p) {
  constexpr int LPR = D / kUnit, RPS = 64 / LPR, AHEAD = 4;     // lanes of a row, rows of a step
  __shared__ f32x2 pairs[4][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t tok = static_cast<int64_t>(blockIdx.x) * 4 + wave;
  if (tok >= p.N) return;
  const int u = lane % LPR, row = lane / LPR;
  const double freq = lane_frequency(p.rope);
  const int pos = p.positions[tok];
  const UnitAt at = unit_at(p.rope, true, u);
  const uint16_t* const x = p.x + tok * p.x_token;
  uint16_t* const out = p.out + tok * p.out_token;
  const int s1 = min((static_cast<int>(blockIdx.y) + 1) * p.steps, (p.H + RPS - 1) / RPS);
  f32x2 cs[8];
  bool known = false;
  for (int s0 = static_cast<int>(blockIdx.y) * p.steps; s0 < s1; s0 += AHEAD) {
    u32x4 raw[AHEAD][2];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int h = (s0 + i) * RPS + row;
      if (s0 + i < s1 && h < p.H) {
        raw[i][0] = *reinterpret_cast<const u32x4*>(x + h * p.x_head + at.a);
        raw[i][1] = *reinterpret_cast<const u32x4*>(x + h * p.x_head + at.b);
      }
    }
    if (!known) unit_angles(p.rope, freq, pos, pairs[wave], u, cs);
    known = true;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int h = (s0 + i) * RPS + row;
      if (s0 + i < s1 && h < p.H) {
        if (at.turned) {
          float v[kUnit];
          widen(raw[i][0], v);
          widen(raw[i][1], v + 8);
          turn_unit(p.rope, v, cs);
          raw[i][0] = narrow(v);
          raw[i][1] = narrow(v + 8);
        }
        *reinterpret_cast<u32x4*>(out + h * p.out_head + at.a) = raw[i][0];
        *reinterpret_cast<u32x4*>(out + h * p.out_head + at.b) = raw[i][1];
      }
    }
  }
}

// --------------------------------------------------------------------------------------------------------- quantising

// Largest of the LPR (8 or 4) lanes of a row.
template <int LPR>
__device__ __forceinline__ uint32_t row_lanes_max(uint32_t x) {
  auto with = [&](auto ctrl) {
    const uint32_t y = __builtin_amdgcn_update_dpp(0, static_cast<int>(x), decltype(ctrl)::value, 0xf, 0xf, true);
    x = x > y ? x : y;
  };
  with(std::integral_constant<int, 0xB1>{});                     // quad_perm: lanes 1 apart, 2 apart
  with(std::integral_constant<int, 0x4E>{});
  if constexpr (LPR == 8) with(std::integral_constant<int, 0x141>{});   // row_half_mirror: the other four
  return x;
}

// Codes (4 dwords) and scale of a row whose lanes have 16 elements each.
template <int FMT, int LPR>
__device__ __forceinline__ u32x4 quantise_unit(const float (&x)[kUnit], float& scale) {
  constexpr float kTop = FMT == kE4m3 ? 448.f : 127.f;
  constexpr float kTiny = 0x1p-110f;
  uint32_t top = 0u;                          // (bit patterns: a NaN is larger than every number)
#pragma unroll
  for (int i = 0; i < kUnit; ++i) {
    const uint32_t a = __float_as_uint(x[i]) & 0x7fffffffu;
    top = top > a ? top : a;
  }
  const float a = __uint_as_float(row_lanes_max<LPR>(top));
  const bool finite = __float_as_uint(a) < 0x7f800000u, live = finite && a >= kTiny;
  // (One correctly rounded reciprocal, products otherwise, each rounded by itself: whoever computes these gets the same codes.)
  const float inv = __fmul_rn(kTop, __frcp_rn(live ? a : 1.f));
  scale = !finite ? __builtin_nanf("") : live ? __fmul_rn(a, 1.f / kTop) : 0.f;
  u32x4 codes;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = x[4 * e + i] * inv;
    uint32_t c;
    if constexpr (FMT == kE4m3) {
      int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
      c = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true));
    } else {
      // (Over 1.5 * 2^23 the integers are a step apart: the sum rounds to the nearest even one, whose low byte is the code.)
#pragma clang fp contract(off)
      constexpr float kWhole = 12582912.f;
      const uint32_t r0 = __float_as_uint(y[0] + kWhole), r1 = __float_as_uint(y[1] + kWhole);
      const uint32_t r2 = __float_as_uint(y[2] + kWhole), r3 = __float_as_uint(y[3] + kWhole);
      c = __builtin_amdgcn_perm(r1, r0, 0x0c0c0400u) | __builtin_amdgcn_perm(r3, r2, 0x04000c0cu);
    }
    codes[e] = live ? c : 0u;
  }
  return codes;
}

// Writes a unit's codes (one 16-byte store where its eights are neighbours).
__device__ __forceinline__ void store_codes(uint8_t* dst, const UnitAt& at, const u32x4& codes) {
  if (at.b == at.a + 8) {
    *reinterpret_cast<u32x4*>(dst + at.a) = codes;
  } else {
    *reinterpret_cast<u32x2*>(dst + at.a) = u32x2{codes[0], codes[1]};
    *reinterpret_cast<u32x2*>(dst + at.b) = u32x2{codes[2], codes[3]};
  }
}
// How many tokens a sequence of n takes of this call.
__device__ __forceinline__ int taken_tokens(const QuantAppendParams& p, int b, int n) {
  int count = p.T;
  if (p.new_lens) count = min(max(p.new_lens[b], 0), p.T);
  const int64_t cap = min(static_cast<int64_t>(p.max_blocks) * kPage, static_cast<int64_t>(p.max_tokens));
  return n < 0 || static_cast<int64_t>(n) + count > cap ? 0 : count;   // no room: the sequence takes nothing
}
__device__ __forceinline__ void store_length(const QuantAppendParams& p, int b, int n, int count) {
  p.seq_lens_out[b] = n + count;
  if (p.grow.sel_table != nullptr && count > 0) {
    ExtendParams grow = p.grow;
    grow.num_new = count;
    extend_selection_row(grow, b, n + count);
  }
}

// Few new tokens of sequence blockIdx.z: a wave takes a token at a time, and of its steps (64 / (D / 16) heads of K, of V, of the
// queries) those of its grid row.  The length is read by every wave; who stores the new one has to be last:
//   IN_PLACE: one workgroup per sequence, a barrier between (few tokens); otherwise seq_lens_out is another array, or nullptr where
//   a second launch (advance_lengths_kernel) stores it.
template <int D, int FMT, bool IN_PLACE>
__global__ __launch_bounds__(IN_PLACE ? 1024 : 256) void append_quant_kernel(const QuantAppendParams p) {
  constexpr int LPR = D / kUnit, RPS = 64 / LPR, NW = IN_PLACE ? 16 : 4;
  __shared__ f32x2 pairs[NW][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int b = blockIdx.z;
  const int u = lane % LPR, row = lane / LPR;
  const bool rotates = p.rope.inv_freq != nullptr;
  const double freq = rotates ? lane_frequency(p.rope) : 0.0;
  const int n = p.seq_lens[b];
  const int count = taken_tokens(p, b, n);
  if constexpr (IN_PLACE) __syncthreads();
  const int sk = (p.Hkv + RPS - 1) / RPS, all = 2 * sk + (p.q ? (p.Hq + RPS - 1) / RPS : 0);
  const int32_t* const table = p.block_table + static_cast<int64_t>(b) * p.max_blocks;
  const UnitAt turned = unit_at(p.rope, rotates, u), plain = unit_at(p.rope, false, u);

  auto step = [&](int t, int s, int64_t page, const f32x2 (&cs)[8]) {
    const int64_t token = static_cast<int64_t>(b) * p.T + t;
    if (s >= 2 * sk) {                       // queries: rotated, bf16 again
      const int h = (s - 2 * sk) * RPS + row;
      if (h >= p.Hq) return;
      const uint16_t* src = p.q + token * p.q_token + h * D;
      uint16_t* dst = p.q_out + token * p.q_out_token + h * D;
      u32x4 lo = *reinterpret_cast<const u32x4*>(src + turned.a), hi = *reinterpret_cast<const u32x4*>(src + turned.b);
      if (turned.turned) {
        float x[kUnit];
        widen(lo, x);
        widen(hi, x + 8);
        turn_unit(p.rope, x, cs);
        lo = narrow(x);
        hi = narrow(x + 8);
      }
      *reinterpret_cast<u32x4*>(dst + turned.a) = lo;
      *reinterpret_cast<u32x4*>(dst + turned.b) = hi;
      return;
    }
    const bool is_v = s >= sk;
    const int h = (s - (is_v ? sk : 0)) * RPS + row;
    if (h >= p.Hkv) return;                  // (whole rows of lanes)
    const UnitAt at = is_v ? plain : turned;
    const uint16_t* src = (is_v ? p.v_new : p.k_new) + token * p.kv_token + h * D;
    float x[kUnit];
    widen(*reinterpret_cast<const u32x4*>(src + at.a), x);
    widen(*reinterpret_cast<const u32x4*>(src + at.b), x + 8);
    if (at.turned) turn_unit(p.rope, x, cs);
    // (The rotated key is quantised from fp32: a bf16 in between would be a second rounding and save nothing.)
    float scale;
    const u32x4 codes = quantise_unit<FMT, LPR>(x, scale);
    const int slot = (n + t) % kPage;
    uint8_t* dst = (is_v ? p.v_cache : p.k_cache) + page * p.page_stride + slot * p.token_stride + h * p.head_stride;
    store_codes(dst, at, codes);
    if (u == 0) p.scales[((page * p.Hkv + h) * 2 + (is_v ? 1 : 0)) * kPage + slot] = scale;
  };
  auto token = [&](int t, int s0, int s1) {
    int64_t page = table[(n + t) / kPage];
    page = page < 0 ? 0 : (page >= p.num_pages ? p.num_pages - 1 : page);   // a corrupt table cannot fault
    f32x2 cs[8];
    if (rotates) unit_angles(p.rope, freq, n + t, pairs[wave], u, cs);
    for (int s = s0; s < s1; ++s) step(t, s, page, cs);
  };
  if constexpr (IN_PLACE) {
    for (int i = wave; i < count * all; i += NW) token(i / all, i % all, i % all + 1);
  } else {
    const int s0 = static_cast<int>(blockIdx.y) * p.steps;
    const int t = static_cast<int>(blockIdx.x) * NW + wave;
    if (t < count) token(t, s0, min(s0 + p.steps, all));
  }
  if (threadIdx.x == 0 && (blockIdx.x | blockIdx.y) == 0 && p.seq_lens_out != nullptr) store_length(p, b, n, count);
}

// Many new tokens: a workgroup takes 16 of them and a wave four, a step's rows of all four asked for while the last step's are
// worked on.  (A wait for loads is one for the stores in front of them as well: what is asked for behind a step's stores comes a
// round trip late.)  Scales meet in LDS and leave as runs of the tokens of a page: stored one by one they are as many requests
// as the codes.  us a call (captured), with a token a wave at a time / so: 4 x 4096 tokens, 8 KV heads, 32 query heads 72.2 / 71.4
// (4.4 TB/s); 8 x 1011, head dimension 64, int8 12.1 / 10.8, 9.7 with the codes packed by byte permutes (a launch of next to nothing takes 3.3).
constexpr int kAppendTokens = 16, kAppendSteps = 8;
template <int D, int FMT>
__global__ __launch_bounds__(256) void append_pages_kernel(const QuantAppendParams p) {
  constexpr int LPR = D / kUnit, RPS = 64 / LPR, NW = 4, TW = kAppendTokens / NW;
  __shared__ __attribute__((aligned(16))) f32x2 pairs[NW][TW][64];
  __shared__ float scale_lds[kAppendSteps * RPS][kAppendTokens];
  __shared__ int32_t page_lds[kAppendTokens];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int b = blockIdx.z, t0 = static_cast<int>(blockIdx.x) * kAppendTokens, tw = t0 + TW * wave;
  const int u = lane % LPR, row = lane / LPR;
  const int sk = (p.Hkv + RPS - 1) / RPS, all = 2 * sk + (p.q ? (p.Hq + RPS - 1) / RPS : 0);
  const int s0 = static_cast<int>(blockIdx.y) * p.steps, s1 = min(s0 + p.steps, all);
  const bool rotates = p.rope.inv_freq != nullptr;
  const double freq = rotates ? lane_frequency(p.rope) : 0.0;
  const UnitAt turned = unit_at(p.rope, rotates, u), plain = unit_at(p.rope, false, u);
  struct Rows { u32x4 half[TW][2]; };
  auto fetch = [&](int s, Rows& r) {         // (the inputs have T tokens of every sequence, whatever it takes of them)
    const int part = s >= 2 * sk ? 2 : s >= sk ? 1 : 0;
    const int h = min((s - part * sk) * RPS + row, (part == 2 ? p.Hq : p.Hkv) - 1);
    const UnitAt at = part == 1 ? plain : turned;
    const uint16_t* const src = (part == 2 ? p.q : part == 1 ? p.v_new : p.k_new) + h * D;
    const int64_t stride = part == 2 ? p.q_token : p.kv_token;
#pragma unroll
    for (int i = 0; i < TW; ++i) {
      const uint16_t* const x = src + (static_cast<int64_t>(b) * p.T + min(tw + i, p.T - 1)) * stride;
      r.half[i][0] = *reinterpret_cast<const u32x4*>(x + at.a);
      r.half[i][1] = *reinterpret_cast<const u32x4*>(x + at.b);
    }
  };
  Rows now, next;
  fetch(s0, now);
  const int n = p.seq_lens[b];
  const int count = taken_tokens(p, b, n);
  const int32_t* const table = p.block_table + static_cast<int64_t>(b) * p.max_blocks;
  int64_t page[TW];
#pragma unroll
  for (int i = 0; i < TW; ++i) {
    page[i] = tw + i < count ? table[(n + tw + i) / kPage] : 0;
    page[i] = page[i] < 0 ? 0 : (page[i] >= p.num_pages ? p.num_pages - 1 : page[i]);   // a corrupt table cannot fault
    if (lane == 0) page_lds[TW * wave + i] = static_cast<int32_t>(page[i]);
    if (rotates) pairs[wave][i][lane] = lane_angle(p.rope, freq, n + tw + i);
  }
  wave_lds_fence();
  auto work = [&](int s, const Rows& r) {
    const int part = s >= 2 * sk ? 2 : s >= sk ? 1 : 0, h = (s - part * sk) * RPS + row;
    if (h >= (part == 2 ? p.Hq : p.Hkv)) return;         // (whole rows of lanes)
    const UnitAt at = part == 1 ? plain : turned;
#pragma unroll
    for (int i = 0; i < TW; ++i) {
      const int t = tw + i;
      if (t >= count) break;
      float x[kUnit];
      widen(r.half[i][0], x);
      widen(r.half[i][1], x + 8);
      if (at.turned) {
        f32x2 cs[8];
        read_angles(pairs[wave][i], u, cs);
        turn_unit(p.rope, x, cs);
      }
      if (part == 2) {
        uint16_t* const dst = p.q_out + (static_cast<int64_t>(b) * p.T + t) * p.q_out_token + h * D;
        *reinterpret_cast<u32x4*>(dst + at.a) = at.turned ? narrow(x) : r.half[i][0];
        *reinterpret_cast<u32x4*>(dst + at.b) = at.turned ? narrow(x + 8) : r.half[i][1];
      } else {
        float scale;
        const u32x4 codes = quantise_unit<FMT, LPR>(x, scale);
        store_codes((part == 1 ? p.v_cache : p.k_cache) + page[i] * p.page_stride + (n + t) % kPage * p.token_stride + h * p.head_stride, at, codes);
        if (u == 0) scale_lds[(s - s0) * RPS + row][TW * wave + i] = scale;
      }
    }
  };
  int s = s0;
  for (; s + 1 < s1; ++s) {
    fetch(s + 1, next);
    work(s, now);
    now = next;
  }
  work(s, now);
  __syncthreads();
  const int live = min(kAppendTokens, count - t0), kv_steps = min(s1, 2 * sk) - s0;
  for (int e = threadIdx.x; e < kv_steps * RPS * kAppendTokens; e += NW * 64) {
    const int r = e / kAppendTokens, i = e % kAppendTokens, step = s0 + r / RPS, part = step >= sk ? 1 : 0;
    const int h = (step - part * sk) * RPS + r % RPS;
    if (i < live && h < p.Hkv)
      p.scales[((static_cast<int64_t>(page_lds[i]) * p.Hkv + h) * 2 + part) * kPage + (n + t0 + i) % kPage] = scale_lds[r][i];
  }
  if (threadIdx.x == 0 && (blockIdx.x | blockIdx.y) == 0 && p.seq_lens_out != nullptr) store_length(p, b, n, count);
}

// The lengths (and selections) behind an append of many tokens in place, one thread per sequence.
__global__ void advance_lengths_kernel(const QuantAppendParams p, int32_t* seq_lens, int batch) {
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b >= batch) return;
  const int n = seq_lens[b];
  const int count = taken_tokens(p, b, n);
  if (count == 0) return;
  seq_lens[b] = n + count;
  if (p.grow.sel_table != nullptr) {
    ExtendParams grow = p.grow;
    grow.num_new = count;
    extend_selection_row(grow, b, n + count);
  }
}

// ------------------------------------------------------------------------------------------------------- reading back

// Eight codes as fp32.
template <int FMT>
__device__ __forceinline__ void widen_codes(const u32x2& w, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    if constexpr (FMT == kE4m3) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[e]), false);
      const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[e]), true);
      x[4 * e] = lo[0]; x[4 * e + 1] = lo[1]; x[4 * e + 2] = hi[0]; x[4 * e + 3] = hi[1];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * e + i] = static_cast<float>(static_cast<int8_t>(w[e] >> (8 * i)));
    }
  }
}

// A workgroup has 16 consecutive tokens of a sequence's list, a wave every fourth of them, a lane 8 elements of a row: it reads
// 8 bytes of a token's codes and writes 16 of its output row, both without gaps between lanes (NHD).
constexpr int kReadTokens = 16;
template <int D, int FMT>
__global__ __launch_bounds__(256) void read_quant_kernel(const QuantReadParams p) {
  constexpr int LPR = D / 8;                 // lanes of a row
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int b = blockIdx.z;
  int n = p.lens[b];
  n = n < 0 ? 0 : (n > p.max_tokens ? p.max_tokens : n);
  const int first = p.first ? max(p.first[b], 0) : 0;
  const int t0 = static_cast<int>(blockIdx.x) * kReadTokens;
  const int t1 = static_cast<int>(min(static_cast<int64_t>(min(t0 + kReadTokens, p.T)), static_cast<int64_t>(n) - first));
  const int32_t* const table = p.table + static_cast<int64_t>(b) * p.table_stride;
  for (int t = t0 + wave; t < t1; t += 4) {
    const int pos = first + t;
    int64_t page = table[pos >> p.page_shift];
    page = page < 0 ? 0 : (page >= p.num_pages ? p.num_pages - 1 : page);
    const int in_page = pos & ((1 << p.page_shift) - 1);
    const int64_t slot = (page << p.page_shift) + in_page;             // of the pool
    const int64_t at = page * p.page_stride + in_page * p.token_stride;
    const int64_t out = (static_cast<int64_t>(b) * p.T + t) * p.Hkv * D;
    const float* const scales = p.scales + (slot / kPage) * p.Hkv * 32 + slot % kPage;
    for (int e = lane; e < p.Hkv * LPR; e += 64) {
      const int h = e / LPR;
      const int64_t src = at + h * p.head_stride + (e % LPR) * 8;
      const u32x2 k = *reinterpret_cast<const u32x2*>(p.k_cache + src), v = *reinterpret_cast<const u32x2*>(p.v_cache + src);
      const float ks = scales[h * 32], vs = scales[h * 32 + kPage];
      float x[8];
      widen_codes<FMT>(k, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= ks;
      *reinterpret_cast<u32x4*>(p.k_out + out + e * 8) = narrow(x);
      widen_codes<FMT>(v, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= vs;
      *reinterpret_cast<u32x4*>(p.v_out + out + e * 8) = narrow(x);
    }
  }
}

}  // namespace vegas
