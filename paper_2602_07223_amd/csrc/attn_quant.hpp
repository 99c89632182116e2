// KV-streaming attention kernel over an 8-bit cache (quant_cache.hpp), gfx950: verification (several causal rows per head, page
// log-sum-exps beside the partial results) and draft or decode calls (one row per head over a page list) are the same kernel.
// Chunking, partial results, plans of ragged batches and merge kernels are those of the bf16 kernels.
//
//   logit(r, t) = c ks[t] sum_d q[r][d] kc[t][d],  w = 2^(logit - m),  O[r] += w vs[t] vc[t][:],  l += w     (c: softmax scale, log2 e)
//
// Codes become bf16 in registers (both formats' are exact in it) and the contractions are 16x16x32 bf16 MFMAs: a key's scale
// multiplies its column of logits behind the first contraction, a value's scale its weight in front of the second, so the
// matrix products see small exact numbers and a scale costs one multiplication per weight, not one per code.
//   * K: lane (token i, group kg) has the 16 codes kc[i][64 j + 16 kg ..], which are two A operands; any order of the contraction index
//     does, and the queries are laid out to match.
//   * V: lane (m, kg) loads D / 16 codes of the eight tokens 4 kg + e % 4 of page e / 4 -- the tokens whose weights it has
//     from the first contraction -- and pairs of tokens are brought together by byte permutes (e4m3) or byte-selecting
//     conversions (int8): the weights are the B operand as they stand, and nothing goes through LDS.
//   * Scales: a wave's 32 + 32 of a tile are one dword per lane, spread through LDS (four 16-byte reads) instead of being
//     loaded by all 16 lanes that use them.
//   * NT tiles of 16 query rows share a tile's loads and conversions.
//   * A row's reference m follows its maximum only when that has grown by more than 2^6: weights are then below 2^6 and the
//     usual rescaling of the outputs, and the reduction over the four lanes of a row, is seldom met.
// What bounds it: memory from 64 MB on.  A 32-token tile of a head is 8.25 KB (D = 128), half of the bf16 cache's, and costs 80
// conversions (e4m3; int8 192) and per 16 rows 16 MFMAs and about 90 vector instructions.  Loads run a whole tile ahead in a second set of
// registers.
// TOKENS: the page list has pages of fewer than 16 tokens (page_shift): every lane works out the address of one token
// of the tile, the wave shares them through LDS.
#pragma once
#include <type_traits>

#include "attn_draft.hpp"
#include "quant_cache.hpp"
#include "vegas_common.hpp"

namespace vegas {

struct QuantArgs {
  const float* scales;       // [page, KV head, 2, 16]
  int32_t page_shift;        // log2 of the page list's tokens per page
  int32_t park_bytes;        // dynamic LDS of the page log-sum-exps (COLLECT) or of the merge, whichever is larger
};

constexpr int kQuantVerifyNT = 3, kQuantDraftNT = 2;   // 16-row tiles of a workgroup, at most (what registers hold)
constexpr float kQuantSlack = 6.f;           // log2 of how far weights may pass 1

// Dynamic LDS: [parked page log-sum-exps | merge rows, NW x 16] [queries, 16 NT rows] [row maxima, sums][scales, addresses of a wave]
constexpr size_t quant_merge_bytes(int NW, int D) { return static_cast<size_t>(NW) * 16 * red_pitch(D) * sizeof(float); }
constexpr size_t quant_tail_bytes(int NW, int NT, int D) {
  return (NT > 1 ? static_cast<size_t>(16) * NT * row_pitch(D) : 0) + 2 * static_cast<size_t>(NW) * 16 * NT * sizeof(float) +
         static_cast<size_t>(NW) * (64 * sizeof(float) + 32 * sizeof(uint64_t));
}
inline size_t quant_park_bytes(int NW, int rows, int chunk_tokens, bool collect, int D) {
  const size_t merge = quant_merge_bytes(NW, D);
  const size_t park = collect ? (static_cast<size_t>(chunk_tokens) / kPage * rows * sizeof(float) + 15) / 16 * 16 : 0;
  return park > merge ? park : merge;
}

// Registers that the compiler takes for rewritten here: what is made of them stays behind this point.
template <typename T>
__device__ __forceinline__ void pin_one(T& r) {
  if constexpr (sizeof(T) == 4) {
    uint32_t x = r[0];
    asm volatile("" : "+v"(x));
    r[0] = x;
  } else {
    asm volatile("" : "+v"(r));
  }
}
template <typename... T>
__device__ __forceinline__ void pin(T&... regs) { (pin_one(regs), ...); }

// Two adjacent codes of a dword (its low or high half) as bf16.
template <bool HIGH>
__device__ __forceinline__ uint32_t e4m3_pair(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HIGH));
}
__device__ __forceinline__ uint32_t int8_pair(uint32_t a, uint32_t b, int byte_a, int byte_b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const float x = static_cast<float>(static_cast<int8_t>(a >> (8 * byte_a))), y = static_cast<float>(static_cast<int8_t>(b >> (8 * byte_b)));
  return __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(x), static_cast<__bf16>(y)});
}
// Eight consecutive codes as an MFMA operand.
template <int FMT>
__device__ __forceinline__ bf16x8 operand_of(uint32_t w0, uint32_t w1) {
  u32x4 r;
  if constexpr (FMT == kE4m3) {
    r = u32x4{e4m3_pair<false>(w0), e4m3_pair<true>(w0), e4m3_pair<false>(w1), e4m3_pair<true>(w1)};
  } else {
    r = u32x4{int8_pair(w0, w0, 0, 1), int8_pair(w0, w0, 2, 3), int8_pair(w1, w1, 0, 1), int8_pair(w1, w1, 2, 3)};
  }
  return __builtin_bit_cast(bf16x8, r);
}

template <int D, int FMT, int NT, int NW, bool TOKENS, int COLLECT, bool NT_LOADS>
__global__ __launch_bounds__(NW * 64, 2) void quant_stream_kernel(VEGAS_SPLIT_HOT_PARAMS, const SplitParams pfull, const QuantArgs qa) {
  SplitParams p = pfull;                     // (see attn_split_kernel: the preloaded arguments)
  VEGAS_SPLIT_HOT_ASSIGN(p);
  VEGAS_TL_DECL;
  VEGAS_TL(kTlEntry);
  static_assert(D == 128 || D == 64, "head dimension");
  static_assert(!TOKENS || COLLECT == 0, "page lists are not scored");
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr int KL = D / 64;                 // K loads of a page
  constexpr int KS = D / 32;                 // steps of the first contraction
  constexpr int NBLK = D / 16;               // 16-row blocks of the output, codes of a V load
  constexpr int kRed = red_pitch(D);
  constexpr bool TIGHT = NT * D > 128;       // conversions stay with the products that use them: hoisted, they take more registers than there are
  typedef unsigned int u32x1 __attribute__((ext_vector_type(1)));
  using VReg = typename std::conditional<NBLK == 8, u32x2, u32x1>::type;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, kg = lane >> 4;
  // Grid (chunk in a group of 8, KV head + Hkv * row block, group + groups * sequence).  Workgroups go round the 8 XCDs, so a chunk's heads and
  // row blocks meet on one of them, which then reads whole pages: 16 x 128 bytes of a token at a time.  (Heads first, an XCD reads every eighth
  // 128-byte line: @@)
  const int row_blocks = p.row_blocks & 255, groups = p.row_blocks >> 8;
  int h = blockIdx.y, rb = 0;
  if (row_blocks > 1) {
    rb = static_cast<int>(blockIdx.y) / p.Hkv;
    h -= rb * p.Hkv;
  }
  int b = blockIdx.z, split = blockIdx.x;
  if (groups > 1) {                          // (z < 2^16: the quotient is exact)
    b = static_cast<int>((static_cast<float>(blockIdx.z) + 0.5f) * __builtin_amdgcn_rcpf(static_cast<float>(groups)));
    split += 8 * (static_cast<int>(blockIdx.z) - b * groups);
  }
  int chunk_tokens = p.chunk_tokens;
  int c0 = split * chunk_tokens;
  int slot = split;
  int n = 0;
  if constexpr (!TOKENS) {
    if (p.plan) {                            // (groups is 1: no sequence in the grid) balanced chunking: workgroup `split` of this head -> (sequence, tokens)
      split = static_cast<int>(blockIdx.x + 8 * blockIdx.z);
      const BalancedSlot bs = balanced_slot(p.lens, p.batch, p.max_tokens, p.slots_target, p.slots_target2, p.share_group,
                                            p.slots_total, p.share_margin, 2, p.chunk_cap_units, kTile * NW, split,
                                            ((blockIdx.x | blockIdx.y | blockIdx.z) == 0 && wave == 0) ? p.plan : nullptr);
      b = __builtin_amdgcn_readfirstlane(bs.b);
      if (b < 0) return;
      c0 = __builtin_amdgcn_readfirstlane(bs.c0);
      chunk_tokens = __builtin_amdgcn_readfirstlane(bs.chunk);
      slot = __builtin_amdgcn_readfirstlane(bs.slot);
      n = bs.n;
    }
  }
  const int row0 = rb * 16 * NT;             // first row (of this KV head) handled here
  const int Rl = min(16 * NT, p.R - row0);

  // ---- one round trip for what the preloaded arguments can address: page ids, length, queries (see attn_split_kernel)
  const int32_t* table = p.table + static_cast<int64_t>(b) * p.table_stride;
  const int tile_first = c0 / kTile + wave;
  int last_page = 0;                         // (set below)
  // 16-token pages: ids of the wave's next 32 tiles, lane (k, half) <-> page `half` of tile tile_first + k NW.
  auto table_entry = [&](int kbase) -> int {
    int page = 2 * (tile_first + (kbase + (lane & 31)) * NW) + (lane >> 5);
    page = page < p.table_stride ? page : p.table_stride - 1;
    return table[page];
  };
  // Page lists: id of the page of token lane % 32 of tile k.
  auto ids_entry = [&](int k) -> int {
    const int64_t tok = static_cast<int64_t>(tile_first + k * NW) * kTile + (lane & 31);
    const int64_t page = tok >> qa.page_shift;
    return table[page < p.table_stride ? page : p.table_stride - 1];
  };
  auto into_pool = [&](int raw) -> int { return min(max(raw, 0), last_page); };
  int first_entry = TOKENS ? ids_entry(0) : table_entry(0);
  int zero = 0;
  asm("" : "+v"(zero));                      // (a vector load: a scalar one is waited for at once)
  if (!p.plan) n = p.lens[b + zero];

  // Queries: lane (row l16, kg) of tile nt, step 2 j + u: dims 64 j + 16 kg + 8 u .. + 7.  One tile's stay in registers, more go through LDS.
  const float rcp_g = __builtin_amdgcn_rcpf(static_cast<float>(p.g));
  const unsigned char* qbase = uniform_ptr(reinterpret_cast<const unsigned char*>(p.q + (static_cast<int64_t>(b) * p.G * p.Hq + h * p.g) * D));
  auto row_token = [&](int r) { return static_cast<int>((static_cast<float>(r) + 0.5f) * rcp_g); };   // (r < 128: exact)
  constexpr bool QREG = NT == 1;
  u32x4 qreg[QREG ? KS : 1];
  constexpr int QI = QREG ? 1 : (16 * NT * (D / 8) + NW * 64 - 1) / (NW * 64);
  u32x4 qraw[QI];
  int row_lim[NT];                           // token of the row, later the last position it sees
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) row_lim[nt] = row_token(row0 + min(16 * nt + l16, Rl - 1));
  if constexpr (QREG) {
    const int r = row0 + min(l16, Rl - 1);
    const uint32_t off = static_cast<uint32_t>(row_lim[0] * p.Hq + (r - row_lim[0] * p.g)) * (2u * D);
#pragma unroll
    for (int s = 0; s < KS; ++s) qreg[s] = gload<u32x4, false>(qbase, off + static_cast<uint32_t>(64 * (s >> 1) + 16 * kg + 8 * (s & 1)) * 2u);
  } else {
#pragma unroll
    for (int i = 0; i < QI; ++i) {
      const int idx = tid + i * NW * 64, r = row0 + min(idx / (D / 8), Rl - 1), t = row_token(r);
      qraw[i] = gload<u32x4, false>(qbase, static_cast<uint32_t>((t * p.Hq + (r - t * p.g)) * D + (idx % (D / 8)) * 8) * 2u);
    }
  }
  asm volatile("" : "+s"(p.k), "+s"(p.v), "+s"(p.page_stride), "+s"(p.token_stride), "+s"(p.head_stride), "+s"(p.num_pages),
               "+s"(p.out_direct), "+s"(p.max_tokens), "+s"(p.nsplit), "+s"(p.scale_log2e), "+s"(p.part_o), "+s"(p.part_ml));
  asm volatile("" : "+v"(first_entry), "+v"(n));
  n = __builtin_amdgcn_readfirstlane(n);
  n = n < 0 ? 0 : (n > p.max_tokens ? p.max_tokens : n);
  last_page = static_cast<int>(p.num_pages < INT32_MAX ? p.num_pages - 1 : INT32_MAX);
  const int64_t pbase = p.plan ? static_cast<int64_t>(h) * p.slots_total + slot : (static_cast<int64_t>(b) * p.Hkv + h) * p.nsplit + slot;

  unsigned char* qlds = smem + qa.park_bytes;
  float* sm_m = reinterpret_cast<float*>(qlds + (NT > 1 ? 16 * NT * row_pitch(D) : 0));      // [wave][16 NT]
  float* sm_l = sm_m + NW * 16 * NT;
  float* scale_lds = sm_l + NW * 16 * NT + wave * 64;                                        // [K: 32][V: 32] of a tile
  uint64_t* addr_lds = reinterpret_cast<uint64_t*>(sm_l + NW * 16 * NT + NW * 64) + wave * 32;
  float* lse_lds = reinterpret_cast<float*>(smem);                                           // [pages of the chunk][Rl]
  float* red = reinterpret_cast<float*>(smem);

  if (__builtin_expect(c0 >= n, 0)) {        // nothing to do, no partial is read
    if (p.out_direct != nullptr) {           // no merge kernel follows: the rows of an empty sequence are zeros
      for (int e = tid; e < Rl * D; e += NW * 64) {
        const int r = row0 + e / D, t = r / p.g;
        p.out_direct[((static_cast<int64_t>(b) * p.G + t) * p.Hq + h * p.g + (r - t * p.g)) * D + e % D] = 0;
      }
    }
    return;
  }
  VEGAS_TL(kTlLength);
  const int c1 = min(c0 + chunk_tokens, n);
  const int tile_end = (c1 + kTile - 1) / kTile;
  const int ntiles = tile_first < tile_end ? (tile_end - tile_first + NW - 1) / NW : 0;
  const int sees = n - p.G;                  // last position that row 0 sees
  const int64_t head_off = static_cast<int64_t>(h) * p.head_stride;
  const unsigned char* k_head = reinterpret_cast<const unsigned char*>(p.k) + head_off;
  const unsigned char* v_head = reinterpret_cast<const unsigned char*>(p.v) + head_off;
  const uint32_t ts = static_cast<uint32_t>(p.token_stride);
  // K load j of a page.  D = 128: tokens 8 j .. 8 j + 7 in whole 128-byte lines (exchange_k); half lines would be fetched twice.  D = 64: the
  // page's 16 rows of 64 bytes.
  const int k_tok = D == 128 ? l16 & 7 : l16;
  const uint32_t k_byte = 16u * kg + (D == 128 ? 64u * static_cast<uint32_t>(l16 >> 3) : 0u);
  const uint32_t k_lane_off = static_cast<uint32_t>(k_tok) * ts + k_byte;
  const uint32_t v_lane_off = static_cast<uint32_t>(4 * kg) * ts + static_cast<uint32_t>(NBLK * l16);
  typedef const __attribute__((address_space(1))) unsigned char* gbytes;

  struct Tile {
    u32x4 k[2][KL];
    VReg v[8];
    float scale;                             // lane < 32: K's of token `lane` of the tile; otherwise V's of token lane - 32
  };
  Tile ta, tb;
  int pagevec = TOKENS ? 0 : into_pool(first_entry);
  int ids_next = first_entry;                // page lists: raw ids of the tile whose loads go out next
  auto scale_at = [&](int64_t page16, int in_page) {
    return (gbytes)(reinterpret_cast<const unsigned char*>(qa.scales)) + ((page16 * p.Hkv + h) * 32 + (lane >> 5) * 16 + in_page) * 4;
  };
  auto issue = [&](int k, Tile& t) {
    if constexpr (TOKENS) {
      const int tok = lane & 31, in_page = ((tile_first + k * NW) * kTile + tok) & ((1 << qa.page_shift) - 1);
      const int64_t id = into_pool(ids_next);
      ids_next = ids_entry(k + 1);
      const int64_t pool_slot = (id << qa.page_shift) + in_page;
      wave_lds_fence();
      if (lane < 32) addr_lds[tok] = static_cast<uint64_t>(id * p.page_stride + in_page * p.token_stride);
      wave_lds_fence();
      t.scale = gload_at<float, NT_LOADS>(scale_at(pool_slot >> 4, static_cast<int>(pool_slot) & 15));
#pragma unroll
      for (int pg = 0; pg < 2; ++pg)
#pragma unroll
        for (int j = 0; j < KL; ++j) t.k[pg][j] = gload_at<u32x4, NT_LOADS>((gbytes)k_head + addr_lds[16 * pg + 8 * j + k_tok] + k_byte);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        t.v[e] = gload_at<VReg, NT_LOADS>((gbytes)v_head + addr_lds[16 * (e >> 2) + 4 * kg + (e & 3)] + NBLK * l16);
    } else {
      if ((k & 31) == 0 && k > 0) pagevec = into_pool(table_entry(k));
      const int ph0 = __builtin_amdgcn_readlane(pagevec, k & 31), ph1 = __builtin_amdgcn_readlane(pagevec, 32 + (k & 31));
      const uint64_t at0 = static_cast<uint64_t>(static_cast<uint32_t>(ph0)) * static_cast<uint64_t>(p.page_stride);
      const uint64_t at1 = static_cast<uint64_t>(static_cast<uint32_t>(ph1)) * static_cast<uint64_t>(p.page_stride);
      t.scale = gload_at<float, NT_LOADS>(scale_at((lane & 16) ? ph1 : ph0, l16));
#pragma unroll
      for (int pg = 0; pg < 2; ++pg)
#pragma unroll
        for (int j = 0; j < KL; ++j) t.k[pg][j] = gload<u32x4, NT_LOADS>(uniform_ptr(k_head + (pg ? at1 : at0)) + static_cast<uint32_t>(8 * j) * ts, k_lane_off);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        t.v[e] = gload<VReg, NT_LOADS>(uniform_ptr(v_head + (e < 4 ? at0 : at1)) + static_cast<uint32_t>(e & 3) * ts, v_lane_off);
    }
  };

  // Of the loads of a page, lanes l16 < 8 have codes 16 kg .. of tokens l16 and l16 + 8, the others codes 64 + 16 kg .. of tokens l16 - 8 and l16;
  // lanes 8 apart exchange them, and every lane has both pieces of token l16.
  auto exchange_k = [&](Tile& t) {
    if constexpr (D == 128) {
#pragma unroll
      for (int pg = 0; pg < 2; ++pg)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int a = static_cast<int>(t.k[pg][0][w]), c = static_cast<int>(t.k[pg][1][w]);
          t.k[pg][0][w] = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(a, c, 0x128, 0xf, 0xc, false));   // row_ror:8 into lanes 8 .. 15
          t.k[pg][1][w] = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(c, a, 0x128, 0xf, 0x3, false));   // into lanes 0 .. 7
        }
    }
  };

  f32x4 acc[NT][NBLK];
  float ref[NT], sum[NT];                    // a row's reference (the same in its four lanes) and this lane's share of its sum
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    row_lim[nt] += sees;
    ref[nt] = -INFINITY;
    sum[nt] = 0.f;
#pragma unroll
    for (int j = 0; j < NBLK; ++j) acc[nt][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // (COLLECT: pages of this chunk are parked as [page][row], all rows of the block)
  auto compute = [&](int k, Tile& t) {
    const int tok0 = (tile_first + k * NW) * kTile;
    scale_lds[lane] = lane < 32 ? t.scale * p.scale_log2e : t.scale;
    wave_lds_fence();
    exchange_k(t);
    f32x4 st[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) st[nt][0] = st[nt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      bf16x8 kop[2];
      if constexpr (TIGHT) pin(t.k[0][s >> 1], t.k[1][s >> 1]);
#pragma unroll
      for (int pg = 0; pg < 2; ++pg) kop[pg] = operand_of<FMT>(t.k[pg][s >> 1][2 * (s & 1)], t.k[pg][s >> 1][2 * (s & 1) + 1]);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        bf16x8 qop;
        if constexpr (QREG) qop = __builtin_bit_cast(bf16x8, qreg[s]);
        else qop = *reinterpret_cast<const bf16x8*>(qlds + (16 * nt + l16) * row_pitch(D) + (64 * (s >> 1) + 16 * kg + 8 * (s & 1)) * 2);
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) st[nt][pg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kop[pg], qop, st[nt][pg], 0, 0, 0);
      }
      if constexpr (TIGHT) __builtin_amdgcn_sched_barrier(0);
    }
    f32x4 ks[2], vs[2];
#pragma unroll
    for (int pg = 0; pg < 2; ++pg) {
      ks[pg] = *reinterpret_cast<const f32x4*>(scale_lds + 16 * pg + 4 * kg);
      vs[pg] = *reinterpret_cast<const f32x4*>(scale_lds + 32 + 16 * pg + 4 * kg);
    }
    const bool tail = tok0 + kTile - 1 > sees;         // some row does not see some token
    bf16x8 pb[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = st[nt][i >> 2][i & 3] * ks[i >> 2][i & 3];
      if (tail) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (tok0 + 16 * (i >> 2) + 4 * kg + (i & 3) > row_lim[nt]) x[i] = -INFINITY;
      }
      const float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
      if (__builtin_amdgcn_ballot_w64(top > ref[nt] + kQuantSlack) != 0) {
        const float now = fmaxf(ref[nt], quad_rows_max(top));
        const float alpha = now == -INFINITY ? 1.f : fast_exp2(ref[nt] - now);
        ref[nt] = now;
        sum[nt] *= alpha;
#pragma unroll
        for (int j = 0; j < NBLK; ++j) acc[nt][j] *= alpha;
      }
      const float use = ref[nt] == -INFINITY ? 0.f : ref[nt];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = fast_exp2(x[i] - use);
      const float s0 = (x[0] + x[1]) + (x[2] + x[3]), s1 = (x[4] + x[5]) + (x[6] + x[7]);
      sum[nt] += s0 + s1;
      if constexpr (COLLECT == 1) {
        // log2-sum-exp2 of the tile's two pages: lanes kg = 0 have page 0's, kg = 1 page 1's
        const float page0 = quad_rows_sum(s0), page1 = quad_rows_sum(s1);
        const float lse = use + fast_log2(kg == 0 ? page0 : page1);
        const int page = (tok0 - c0) / kPage + kg;
        if (kg < 2 && 16 * nt + l16 < Rl) lse_lds[page * Rl + 16 * nt + l16] = lse;
      }
      // The weights (below 2^6) times the values' scales are rounded to bf16, the second contraction's operand type: half a step of 2^-8 of
      // each weight, with random signs, beside the one of the bf16 output.  The sum has them unrounded.
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float w = x[i] * vs[i >> 2][i & 3];
        if (tail && x[i] == 0.f) w = 0.f;              // (a masked token's scale may be anything)
        pb[nt][i] = static_cast<__bf16>(w);
      }
      if constexpr (TIGHT) __builtin_amdgcn_sched_barrier(0);
    }
    if (FMT == kE4m3 && tok0 + kTile > n) {            // slots past the end may hold NaN codes: feed zeros
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (tok0 + 16 * (e >> 2) + 4 * kg + (e & 3) >= n) t.v[e] = VReg{};
    }
#pragma unroll
    for (int c = 0; c < NBLK / 4; ++c) {
      if constexpr (TIGHT) pin(t.v[0], t.v[1], t.v[2], t.v[3], t.v[4], t.v[5], t.v[6], t.v[7]);
      uint32_t lo[4], hi[4];                           // e4m3: codes 4 c, 4 c + 1 and 4 c + 2, 4 c + 3 of tokens 2 i, 2 i + 1
      if constexpr (FMT == kE4m3) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          lo[i] = __builtin_amdgcn_perm(t.v[2 * i + 1][c], t.v[2 * i][c], 0x05010400u);
          hi[i] = __builtin_amdgcn_perm(t.v[2 * i + 1][c], t.v[2 * i][c], 0x07030602u);
        }
      }
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        u32x4 raw;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (FMT == kE4m3) raw[i] = (d & 1) ? e4m3_pair<true>(d < 2 ? lo[i] : hi[i]) : e4m3_pair<false>(d < 2 ? lo[i] : hi[i]);
          else raw[i] = int8_pair(t.v[2 * i][c], t.v[2 * i + 1][c], d, d);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          acc[nt][4 * c + d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, raw), pb[nt], acc[nt][4 * c + d], 0, 0, 0);
        if constexpr (TIGHT) __builtin_amdgcn_sched_barrier(0);
      }
    }
#ifdef VEGAS_TIMELINE
    if (tl_stamps[kTlFirstTile] == 0) VEGAS_TL(kTlFirstTile);
#endif
  };

  if (ntiles > 0) issue(0, ta);
  VEGAS_TL(kTlLoadsIssued);
  if constexpr (!QREG) {                     // (every wave: the barrier)
#pragma unroll
    for (int i = 0; i < QI; ++i) {
      const int idx = tid + i * NW * 64;
      if (idx < 16 * NT * (D / 8)) *reinterpret_cast<u32x4*>(qlds + (idx / (D / 8)) * row_pitch(D) + (idx % (D / 8)) * 16) = qraw[i];
    }
    __syncthreads();
  }
  VEGAS_TL(kTlQueries);
  // ---- stream the chunk's tiles (prefetches are unconditional: the waits for a tile then count its successor's loads exactly)
  if (ntiles > 0) {
    int k = 0;
    for (; k + 2 < ntiles; k += 2) {
      issue(k + 1, tb);
      compute(k, ta);
      issue(k + 2, ta);
      compute(k + 1, tb);
    }
    if (k + 1 < ntiles) {
      issue(k + 1, tb);
      compute(k++, ta);
      ta = tb;
    }
    compute(k, ta);
  }
  VEGAS_TL(kTlStreamed);

  // ---- row references and sums of every wave
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const float l = quad_rows_sum(sum[nt]);
    if (kg == 0) {
      sm_m[wave * 16 * NT + 16 * nt + l16] = ref[nt];
      sm_l[wave * 16 * NT + 16 * nt + l16] = l;
    }
  }
  __syncthreads();
  if constexpr (COLLECT == 1) {              // the chunk's page log-sum-exps, collected rows of the block only, rows contiguous
    const int pages = (c1 - c0 + kPage - 1) / kPage;
    float* const dst = p.page_lse + ((static_cast<int64_t>(b) * p.Hkv + h) * p.lse_pages + c0 / kPage) * p.Rc;
    if (p.Rc == p.R && row_blocks == 1) {
      for (int e = tid; e < pages * Rl; e += NW * 64) dst[e] = lse_lds[e];
    } else {
      for (int e = tid; e < pages * Rl; e += NW * 64) {
        const int page = e / Rl, r = row0 + e - page * Rl;
        const int first = p.g, last = (p.G - 1) * p.g;           // Eq. 3: rows of the first and of the last token
        const int ci = p.Rc == p.R ? r : r < first ? r : r >= last ? r - last + first : -1;
        if (ci >= 0) dst[static_cast<int64_t>(page) * p.Rc + ci] = lse_lds[e];
      }
    }
    __syncthreads();
  }
  VEGAS_TL(kTlMerged);

  // ---- merge the waves, 16 rows at a time: every wave parks its rows, all threads scale and add the copies
  constexpr int V4 = D / 4;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int rows = min(16, Rl - 16 * nt);
    if (rows <= 0) break;
    if (nt > 0) __syncthreads();
    if (l16 < rows) {
      float* dst = red + (wave * 16 + l16) * kRed;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int d0 = NBLK * (4 * kg + i);
        *reinterpret_cast<f32x4*>(dst + d0) = f32x4{acc[nt][0][i], acc[nt][1][i], acc[nt][2][i], acc[nt][3][i]};
        if constexpr (NBLK == 8) *reinterpret_cast<f32x4*>(dst + d0 + 4) = f32x4{acc[nt][4 % NBLK][i], acc[nt][5 % NBLK][i], acc[nt][6 % NBLK][i], acc[nt][7 % NBLK][i]};
      }
    }
    __syncthreads();
    for (int e = tid; e < rows * V4; e += NW * 64) {
      const int row = e / V4, at = 16 * nt + row;
      float m = -INFINITY;
#pragma unroll
      for (int w = 0; w < NW; ++w) m = fmaxf(m, sm_m[w * 16 * NT + at]);
      const float use = m == -INFINITY ? 0.f : m;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
      float l = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float scale = fast_exp2(sm_m[w * 16 * NT + at] - use);
        o += *reinterpret_cast<const f32x4*>(red + (w * 16 + row) * kRed + 4 * (e % V4)) * scale;
        l += sm_l[w * 16 * NT + at] * scale;
      }
      const int r = row0 + at;
      if (p.out_direct != nullptr) {         // the only chunk: the bf16 rows (Eq. 1); a row with no visible key: zeros
        const float inv = l > 0.f ? 1.0f / l : 0.f;
        const int t = row_token(r);
        u32x2 packed;
        packed[0] = static_cast<uint32_t>(float_to_bf16_bits(o[0] * inv)) | (static_cast<uint32_t>(float_to_bf16_bits(o[1] * inv)) << 16);
        packed[1] = static_cast<uint32_t>(float_to_bf16_bits(o[2] * inv)) | (static_cast<uint32_t>(float_to_bf16_bits(o[3] * inv)) << 16);
        *reinterpret_cast<u32x2*>(p.out_direct + ((static_cast<int64_t>(b) * p.G + t) * p.Hq + h * p.g + (r - t * p.g)) * D + 4 * (e % V4)) = packed;
      } else {
        *reinterpret_cast<f32x4*>(p.part_o + (pbase * p.R + r) * D + 4 * (e % V4)) = o;
        if (e % V4 == 0) p.part_ml[pbase * p.R + r] = make_float2(m, l);
      }
    }
  }
  VEGAS_TL(kTlExit);
  VEGAS_TL_FLUSH(p.timeline, NW);
}

}  // namespace vegas
