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
//   * A row's base follows its maximum only when that has grown by more than 2^6: weights are then below 2^6 and the
//     usual rescaling of the outputs, and the reduction over the four lanes of a row, is seldom met.
// What bounds it: memory from 64 MB on, latencies below.  A 32-token tile of a head is 8.25 KB (D = 128), half of the bf16 cache's, and costs 80
// conversions (e4m3; int8 192) and per 16 rows 16 MFMAs and about 90 vector instructions; a copy that only loads its tiles takes 270 us
// where the kernel with 40 rows took 285.  Loads run a whole tile ahead in a second set of registers; three to five tiles ahead
// were no faster.  Captured calls with their merges: verification of 16 sequences of 8192..65536 tokens, 40 rows, 8 KV heads (1.26 GB)
// 266 us, without scores 229 (5.5 TB/s; the log-sum-exps, 47 MB written and read again, make the difference), 20 rows 245; one sequence of
// 32768, 20 rows 25.8 (first request to first tile 6 us, the stream at 6.8 TB/s, 2.5 to merge the waves, then the scores' launch);
// draft calls, 12 of 1000..48000 (642 MB, int8) 115 (5.6 TB/s), 16 of 8192 over single tokens 71 (3.9 TB/s: the scales of
// a token and head are two sectors of their line), one of 2080 6.6.
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
  int32_t park_tiles;        // COLLECT: tiles whose log-sum-exps a wave holds back (even)
};

constexpr int kQuantVerifyNT = 3, kQuantDraftNT = 2;  // 16-row tiles of a workgroup, at most: what registers hold
constexpr int kQuantVerifyWaves = 8, kQuantDraftWaves = 4;      // waves of a workgroup (wide ones, of long calls, and narrow ones)
constexpr int kQuantHeads = 4;                // KV heads of a workgroup, at most
constexpr float kQuantSlack = 6.f;           // log2 of how far weights may pass 1

// Dynamic LDS: [parked page log-sum-exps | merge rows, NW x 16] [queries, 16 NT rows a head] [row maxima, sums][scales, addresses of a wave]
constexpr size_t quant_merge_bytes(int NW, int D) { return static_cast<size_t>(NW) * 16 * red_pitch(D) * sizeof(float); }
constexpr size_t quant_tail_bytes(int NW, int NT, int D, int heads) {
  return (NT > 1 ? static_cast<size_t>(heads) * 16 * NT * row_pitch(D) : 0) + 2 * static_cast<size_t>(NW) * 16 * NT * sizeof(float) +
         static_cast<size_t>(NW) * (64 * sizeof(float) + 32 * sizeof(uint64_t));
}
// (A wave writes its log-sum-exps when park_tiles tiles have some, and up to two more may follow before it looks.)
constexpr size_t quant_park_bytes(int NW, int rows, int park_tiles, bool collect, int D) {
  const size_t merge = quant_merge_bytes(NW, D), park = collect ? static_cast<size_t>(NW) * (park_tiles + 2) * 2 * rows * sizeof(float) : 0;
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
  __shared__ int progress[NW];               // tiles that a wave has begun
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
  // Grid (chunk in a group of `across` <= 8, heads of a workgroup + Hkv / HP * row block, group + groups * sequence).  HP neighbouring KV heads share a
  // workgroup, wave w has head w % HP of them: their rows of a token are consecutive 128-byte lines, asked for at about the same time.
  // (A plain read of the lines alone, 16-token pages in random order, 1.2 GB: heads each by itself 5.7 TB/s, two together 6.4, four 6.8,
  // eight 6.9, head-major pages 6.9.)  Workgroups go round the 8 XCDs, so a chunk's heads and row blocks meet on one of them.
  constexpr bool WIDE = NW == kQuantVerifyWaves;       // (only such workgroups have several heads, or a plan)
  const int row_blocks = p.row_blocks & 15, hp_shift = WIDE ? (p.row_blocks >> 4) & 15 : 0;
  const int across = (p.row_blocks >> 8) & 15, groups = p.row_blocks >> 12;
  const int HP = 1 << hp_shift, sub = wave & (HP - 1), wv = wave >> hp_shift, NWH = NW >> hp_shift;   // NWH: waves of a head
  int hg = blockIdx.y, rb = 0;
  if (row_blocks > 1) {
    const int per_block = p.Hkv >> hp_shift;
    rb = static_cast<int>(blockIdx.y) / per_block;
    hg -= rb * per_block;
  }
  const int h0 = hg << hp_shift, h = h0 + sub;
  // (z < 2^16: the quotients are exact.  Chunks are turned by one from sequence to sequence: a ragged batch's last ones, which are short or
  // empty, would all be the same XCDs'.  96 sequences of 500..20000 tokens, 8 KV heads, chunks of 2048: 550 -> 402 us.)
  auto over = [](int a, int d) { return static_cast<int>((static_cast<float>(a) + 0.5f) * __builtin_amdgcn_rcpf(static_cast<float>(d))); };
  int b = blockIdx.z, group = 0;
  if (groups > 1) {
    b = over(blockIdx.z, groups);
    group = static_cast<int>(blockIdx.z) - b * groups;
  }
  int split = static_cast<int>(blockIdx.x) + b + group;
  split += 8 * group - across * over(split, across);
  int chunk_tokens = p.chunk_tokens;
  int c0 = split * chunk_tokens;
  int slot = split;
  int n = 0;
  if (WIDE && p.plan) {                      // (groups is 1: no sequence in the grid) balanced chunking: workgroup `split` of this head -> (sequence, tokens)
    split = static_cast<int>(blockIdx.x + 8 * blockIdx.z);
    const BalancedSlot bs = balanced_slot(p.lens, p.batch, p.max_tokens, p.slots_target, p.slots_target2, p.share_group,
                                          p.slots_total, p.share_margin, 2, p.chunk_cap_units, kTile * NWH, split,
                                          ((blockIdx.x | blockIdx.y | blockIdx.z) == 0 && wave == 0) ? p.plan : nullptr);
    b = __builtin_amdgcn_readfirstlane(bs.b);
    if (b < 0) return;
    c0 = __builtin_amdgcn_readfirstlane(bs.c0);
    chunk_tokens = __builtin_amdgcn_readfirstlane(bs.chunk);
    slot = __builtin_amdgcn_readfirstlane(bs.slot);
    n = bs.n;
  }
  const int row0 = rb * 16 * NT;             // first row (of this KV head) handled here
  const int Rl = min(16 * NT, p.R - row0);

  // ---- one round trip for what the preloaded arguments can address: page ids, length, queries (see attn_split_kernel)
  const int32_t* table = p.table + static_cast<int64_t>(b) * p.table_stride;
  const int tile_first = c0 / kTile + wv;
  int last_page = 0;                         // (set below)
  // 16-token pages: ids of the wave's next 32 tiles, lane (k, half) <-> page `half` of tile tile_first + k NWH.
  auto table_entry = [&](int kbase) -> int {
    int page = 2 * (tile_first + (kbase + (lane & 31)) * NWH) + (lane >> 5);
    page = page < p.table_stride ? page : p.table_stride - 1;
    return table[page];
  };
  // Page lists: id of the page of token lane % 32 of tile k.
  auto ids_entry = [&](int k) -> int {
    const int64_t tok = static_cast<int64_t>(tile_first + k * NWH) * kTile + (lane & 31);
    const int64_t page = tok >> qa.page_shift;
    return table[page < p.table_stride ? page : p.table_stride - 1];
  };
  auto into_pool = [&](int raw) -> int { return min(max(raw, 0), last_page); };
  int first_entry = TOKENS ? ids_entry(0) : table_entry(0);
  int zero = 0;
  asm("" : "+v"(zero));                      // (a vector load: a scalar one is waited for at once)
  if (!WIDE || !p.plan) n = p.lens[b + zero];

  // Queries: lane (row l16, kg) of tile nt, step 2 j + u: dims 64 j + 16 kg + 8 u .. + 7.  One tile's stay in registers, more go through LDS.
  const float rcp_g = __builtin_amdgcn_rcpf(static_cast<float>(p.g));
  const unsigned char* qbase = uniform_ptr(reinterpret_cast<const unsigned char*>(p.q + (static_cast<int64_t>(b) * p.G * p.Hq + (NT == 1 ? h : h0) * p.g) * D));
  auto row_token = [&](int r) { return static_cast<int>((static_cast<float>(r) + 0.5f) * rcp_g); };   // (r < 128: exact)
  constexpr bool QREG = NT == 1;
  u32x4 qreg[QREG ? NT : 1][KS];
  constexpr int QI = QREG ? 1 : (16 * NT * (D / 8) + NW * 64 - 1) / (NW * 64);
  constexpr int kHeads = QREG ? 1 : kQuantHeads;       // (of more tiles every head's rows are in LDS)
  u32x4 qraw[kHeads][QI];
  int row_lim[NT];                           // token of the row, later the last position it sees
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) row_lim[nt] = row_token(row0 + min(16 * nt + l16, Rl - 1));
  if constexpr (QREG) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = row0 + min(16 * nt + l16, Rl - 1);
      const uint32_t off = static_cast<uint32_t>(row_lim[nt] * p.Hq + (r - row_lim[nt] * p.g)) * (2u * D);
#pragma unroll
      for (int s = 0; s < KS; ++s) qreg[nt][s] = gload<u32x4, false>(qbase, off + static_cast<uint32_t>(64 * (s >> 1) + 16 * kg + 8 * (s & 1)) * 2u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < QI; ++i) {
      const int idx = tid + i * NW * 64, r = row0 + min(idx / (D / 8), Rl - 1), t = row_token(r);
      const uint32_t off = static_cast<uint32_t>((t * p.Hq + (r - t * p.g)) * D + (idx % (D / 8)) * 8) * 2u;
#pragma unroll
      for (int s = 0; s < kHeads; ++s)
        if (s < HP) qraw[s][i] = gload<u32x4, false>(qbase, off + static_cast<uint32_t>(s * p.g) * (2u * D));
    }
  }
  asm volatile("" : "+s"(p.k), "+s"(p.v), "+s"(p.page_stride), "+s"(p.token_stride), "+s"(p.head_stride), "+s"(p.num_pages),
               "+s"(p.out_direct), "+s"(p.max_tokens), "+s"(p.nsplit), "+s"(p.scale_log2e), "+s"(p.part_o), "+s"(p.part_ml));
  asm volatile("" : "+v"(first_entry), "+v"(n));
  n = __builtin_amdgcn_readfirstlane(n);
  n = n < 0 ? 0 : (n > p.max_tokens ? p.max_tokens : n);
  last_page = static_cast<int>(p.num_pages < INT32_MAX ? p.num_pages - 1 : INT32_MAX);
  // partial slot of head h0 + s: pbase + s * slots
  const bool planned = WIDE && p.plan;
  const int64_t slots = planned ? p.slots_total : p.nsplit;
  const int64_t pbase = (planned ? 0 : static_cast<int64_t>(b) * p.Hkv * p.nsplit) + h0 * slots + slot;

  unsigned char* qlds = smem + qa.park_bytes;
  float* sm_m = reinterpret_cast<float*>(qlds + (NT > 1 ? HP * 16 * NT * row_pitch(D) : 0));      // [wave][16 NT]
  const unsigned char* const my_q = qlds + sub * 16 * NT * row_pitch(D);
  float* sm_l = sm_m + NW * 16 * NT;
  float* scale_lds = sm_l + NW * 16 * NT + wave * 64;                                        // [K: 32][V: 32] of a tile
  uint64_t* addr_lds = reinterpret_cast<uint64_t*>(sm_l + NW * 16 * NT + NW * 64) + wave * 32;
  float* lse_lds = reinterpret_cast<float*>(smem) + wave * (qa.park_tiles + 2) * 2 * Rl;     // [tile][page][Rl] of this wave
  float* red = reinterpret_cast<float*>(smem);

  if (__builtin_expect(c0 >= n, 0)) {        // nothing to do, no partial is read
    if (p.out_direct != nullptr) {           // no merge kernel follows: the rows of an empty sequence are zeros
      for (int e = tid; e < HP * Rl * D; e += NW * 64) {
        const int s = e / (Rl * D), r = row0 + (e - s * Rl * D) / D, t = r / p.g;
        p.out_direct[((static_cast<int64_t>(b) * p.G + t) * p.Hq + (h0 + s) * p.g + (r - t * p.g)) * D + e % D] = 0;
      }
    }
    return;
  }
  VEGAS_TL(kTlLength);
  const int c1 = min(c0 + chunk_tokens, n);
  const int tile_end = (c1 + kTile - 1) / kTile;
  const int ntiles = tile_first < tile_end ? (tile_end - tile_first + NWH - 1) / NWH : 0;
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
    uint32_t k_off = k_lane_off, v_off = v_lane_off;
    asm volatile("" : "+v"(k_off), "+v"(v_off));                  // (32-bit offsets of scalar bases stay that)
    if constexpr (TOKENS) {
      const int tok = lane & 31, in_page = ((tile_first + k * NWH) * kTile + tok) & ((1 << qa.page_shift) - 1);
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
        for (int j = 0; j < KL; ++j) t.k[pg][j] = gload<u32x4, NT_LOADS>(uniform_ptr(k_head + (pg ? at1 : at0)) + static_cast<uint32_t>(8 * j) * ts, k_off);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        t.v[e] = gload<VReg, NT_LOADS>(uniform_ptr(v_head + (e < 4 ? at0 : at1)) + static_cast<uint32_t>(e & 3) * ts, v_off);
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
  // A row's weights are relative to its base (the same in its four lanes), which moves where a logit passes it by more than the limit; before the
  // row's first key the limit is -inf.  sum: this lane's share of the row's.
  float base[NT], limit[NT], sum[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    row_lim[nt] += sees;
    base[nt] = sum[nt] = 0.f;
    limit[nt] = -INFINITY;
#pragma unroll
    for (int j = 0; j < NBLK; ++j) acc[nt][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  int parked = 0;                            // COLLECT: the first tile whose log-sum-exps are still here
  auto compute = [&](int k, Tile& t) {
    const int tok0 = (tile_first + k * NWH) * kTile;
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
        if constexpr (QREG) qop = __builtin_bit_cast(bf16x8, qreg[nt][s]);
        else qop = *reinterpret_cast<const bf16x8*>(my_q + (16 * nt + l16) * row_pitch(D) + (64 * (s >> 1) + 16 * kg + 8 * (s & 1)) * 2);
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
      float x[8];                                      // logits over the row's base (log2 units), then weights
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __builtin_fmaf(st[nt][i >> 2][i & 3], ks[i >> 2][i & 3], -base[nt]);
      if (tail) {
        const int seen = row_lim[nt] - tok0 - 4 * kg;  // the last of this lane's tokens that the row sees
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (16 * (i >> 2) + (i & 3) > seen) x[i] = -INFINITY;
      }
      const float top = fmaxf(fmaxf(fmaxf(fmaxf(fmaxf(fmaxf(fmaxf(x[0], x[1]), x[2]), x[3]), x[4]), x[5]), x[6]), x[7]);
      if (__builtin_amdgcn_ballot_w64(top > limit[nt]) != 0) {
        const float over = quad_rows_max(top);         // (the four lanes of a row agree on all of this)
        const bool first = limit[nt] == -INFINITY, none = over == -INFINITY;
        const float up = none ? 0.f : first ? over : fmaxf(over, 0.f);
        const float alpha = first ? 1.f : fast_exp2(-up);
        base[nt] += up;
        limit[nt] = none ? limit[nt] : kQuantSlack;
        sum[nt] *= alpha;
#pragma unroll
        for (int j = 0; j < NBLK; ++j) acc[nt][j] *= alpha;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] -= up;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = fast_exp2(x[i]);
      const float s0 = (x[0] + x[1]) + (x[2] + x[3]), s1 = (x[4] + x[5]) + (x[6] + x[7]);
      sum[nt] += s0 + s1;
      if (COLLECT == 1 && p.page_lse != nullptr) {
        // log2-sum-exp2 of the tile's two pages: the lower half wave adds up page 0's, the upper one page 1's
        const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(s0), __float_as_uint(s1), false, false);
        const uint32_t half0 = halves[0], half1 = halves[1];
        const float two = __uint_as_float(half0) + __uint_as_float(half1);
        const auto rows = __builtin_amdgcn_permlane16_swap(__float_as_uint(two), __float_as_uint(two), false, false);
        const uint32_t quarter0 = rows[0], quarter1 = rows[1];
        const float lse = base[nt] + fast_log2(__uint_as_float(quarter0) + __uint_as_float(quarter1));
        if ((kg & 1) == 0 && 16 * nt + l16 < Rl) lse_lds[(2 * (k - parked) + (kg >> 1)) * Rl + 16 * nt + l16] = lse;
      }
      // The weights (below 2^6) times the values' scales are rounded to bf16, the second contraction's operand type: half a step of 2^-8 of
      // each weight, with random signs, beside the one of the bf16 output.  The sum has them unrounded.
      if (tail) {                                      // (a masked token's scale may be anything)
#pragma unroll
        for (int i = 0; i < 8; ++i) pb[nt][i] = static_cast<__bf16>(x[i] == 0.f ? 0.f : x[i] * vs[i >> 2][i & 3]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) pb[nt][i] = static_cast<__bf16>(x[i] * vs[i >> 2][i & 3]);
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

  // Writes the held-back log-sum-exps of the tiles before `end`: two pages a tile, the rows of a page contiguous.  (The stores are waited for:
  // as long as one may be under way the compiler waits for everything where it wants the oldest load.)
  auto write_parked = [&](int end) {
    wave_lds_fence();
    const int nblk = (n + kPage - 1) / kPage;
    const int first = p.g, last = (p.G - 1) * p.g;     // Eq. 3: rows of the first and of the last token
    float* const head = p.page_lse + (static_cast<int64_t>(b) * p.Hkv + h) * p.lse_pages * p.Rc;
    for (const int from = parked; parked < end; ++parked) {
      const int page0 = 2 * (tile_first + parked * NWH);
      float* const dst = head + static_cast<int64_t>(page0) * p.Rc;
      const int live = page0 + 1 < nblk ? 2 * Rl : Rl;
      for (int e = lane; e < live; e += 64) {
        const float lse = lse_lds[2 * (parked - from) * Rl + e];
        if (p.Rc == Rl) {
          dst[e] = lse;
        } else {
          const int page = e >= Rl ? 1 : 0, r = row0 + e - page * Rl;
          const int ci = p.Rc == p.R ? r : r < first ? r : r >= last ? r - last + first : -1;
          if (ci >= 0) dst[page * p.Rc + ci] = lse;
        }
      }
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);      // vmcnt(0)
    wave_lds_fence();
  };

  if (ntiles > 0) issue(0, ta);
  VEGAS_TL(kTlLoadsIssued);
  if constexpr (!QREG) {                     // (every wave: the barrier)
#pragma unroll
    for (int i = 0; i < QI; ++i) {
      const int idx = tid + i * NW * 64;
#pragma unroll
      for (int s = 0; s < kHeads; ++s)
        if (s < HP && idx < 16 * NT * (D / 8)) *reinterpret_cast<u32x4*>(qlds + (s * 16 * NT + idx / (D / 8)) * row_pitch(D) + (idx % (D / 8)) * 16) = qraw[s][i];
    }
    __syncthreads();
  }
  VEGAS_TL(kTlQueries);
  // ---- stream the chunk's tiles, a tile ahead (the last one peeled: prefetches are unconditional, so that the waits for a tile count its
  // successor's loads exactly.  Two or more tiles ahead change nothing, or lose what the registers cost.)
  // Of two waves on a SIMD the older one's requests go first: waves 4 .. 7 of eight were a tenth behind at the end.  Whoever is ahead gives way
  // (16 sequences of 8192..65536 tokens, 40 rows 282 -> 266 us, without scores 237 -> 228; 12 of 1000..48000 drafted 119.5 -> 115.3).
  if constexpr (WIDE) {
    if (lane == 0) progress[wave] = 0;
  }
  if (ntiles > 0) {
    int k = 0;
    for (; k + 2 < ntiles; k += 2) {
      if constexpr (WIDE) {
        volatile int* const at = progress;
        at[wave] = k;
        if (k > __builtin_amdgcn_readfirstlane(at[wave ^ (NW / 2)])) __builtin_amdgcn_s_setprio(0);
        else __builtin_amdgcn_s_setprio(1);
      }
      issue(k + 1, tb);
      compute(k, ta);
      issue(k + 2, ta);
      compute(k + 1, tb);
      if constexpr (COLLECT == 1) {
        if (k + 2 - parked >= qa.park_tiles && p.page_lse != nullptr) write_parked(k + 2);
      }
    }
    if (k + 1 < ntiles) {
      issue(k + 1, tb);
      compute(k++, ta);
      ta = tb;
    }
    compute(k, ta);
    if constexpr (COLLECT == 1)
      if (p.page_lse != nullptr) write_parked(ntiles);
  }
  VEGAS_TL(kTlStreamed);

  // ---- row references and sums of every wave
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const float l = quad_rows_sum(sum[nt]);
    if (kg == 0) {
      sm_m[wave * 16 * NT + 16 * nt + l16] = limit[nt] == -INFINITY ? -INFINITY : base[nt];
      sm_l[wave * 16 * NT + 16 * nt + l16] = l;
    }
  }
  __syncthreads();
  VEGAS_TL(kTlMerged);

  // ---- merge the waves, 16 rows at a time: every wave parks its rows, all threads scale and add the copies
  constexpr int V4 = D / 4;
  auto add_waves = [&](auto waves, int nt, int rows) {
    constexpr int N = decltype(waves)::value;
    for (int e = tid; e < (HP == 1 ? rows : 16 * HP) * V4; e += NW * 64) {
      const int s = e / (16 * V4), row = e / V4 & 15, at = 16 * nt + row;                    // (the head's waves: s, s + HP, ..)
      if (row >= rows) continue;
      float scale[N], m = -INFINITY, l = 0.f;
#pragma unroll
      for (int j = 0; j < N; ++j) scale[j] = sm_m[(s + (j << hp_shift)) * 16 * NT + at];
#pragma unroll
      for (int j = 0; j < N; ++j) m = fmaxf(m, scale[j]);
      const float use = m == -INFINITY ? 0.f : m;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int w = s + (j << hp_shift);
        scale[j] = fast_exp2(scale[j] - use);
        o += *reinterpret_cast<const f32x4*>(red + (w * 16 + row) * kRed + 4 * (e % V4)) * scale[j];
        l += sm_l[w * 16 * NT + at] * scale[j];
      }
      const int r = row0 + at;
      if (p.out_direct != nullptr) {         // the only chunk: the bf16 rows (Eq. 1); a row with no visible key: zeros
        const float inv = l > 0.f ? 1.0f / l : 0.f;
        const int t = row_token(r);
        u32x2 packed;
        packed[0] = static_cast<uint32_t>(float_to_bf16_bits(o[0] * inv)) | (static_cast<uint32_t>(float_to_bf16_bits(o[1] * inv)) << 16);
        packed[1] = static_cast<uint32_t>(float_to_bf16_bits(o[2] * inv)) | (static_cast<uint32_t>(float_to_bf16_bits(o[3] * inv)) << 16);
        *reinterpret_cast<u32x2*>(p.out_direct + ((static_cast<int64_t>(b) * p.G + t) * p.Hq + (h0 + s) * p.g + (r - t * p.g)) * D + 4 * (e % V4)) = packed;
      } else {
        const int64_t at_row = (pbase + s * slots) * p.R + r;
        *reinterpret_cast<f32x4*>(p.part_o + at_row * D + 4 * (e % V4)) = o;
        if (e % V4 == 0) p.part_ml[at_row] = make_float2(m, l);
      }
    }
  };
  auto add_copies = [&](int nt, int rows) {
    if constexpr (WIDE) {
      if (hp_shift == 2) return add_waves(std::integral_constant<int, NW / 4>{}, nt, rows);
      if (hp_shift == 1) return add_waves(std::integral_constant<int, NW / 2>{}, nt, rows);
    }
    add_waves(std::integral_constant<int, NW>{}, nt, rows);
  };
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
    add_copies(nt, rows);
  }
  VEGAS_TL(kTlExit);
  VEGAS_TL_FLUSH(p.timeline, NW);
}

}  // namespace vegas
