// Prefix-reuse prefill attention over a cache held in 8 or 4 bits (gfx950): items, columns, tiles and
// lazy softmax as in the bf16 prefill (prefill_impl.h), on tiles that arrive as codes.
//
// What bounds the bf16 kernel is vector work beside the products, and codes that every wave converts for itself
// are as much again (48 suffixes of 64-401 tokens over 500-3500, 4 bits, 32/8 heads of 128 dims: 483 us against
// 440 in bf16). So
//   - values become bf16 once a workgroup: a wave converts its block of a tile, two codes an instruction, from
//     where it arrived in LDS to where all waves read it, beside the products of a step (418 us);
//   - 4-bit keys are not converted: they and their groups' powers of two are operands of the matrix cores'
//     4-bit products as they lie in the slab, and the queries are taken in three parts of 6 bits (quant.h). The
//     three products take 3/4 of the bf16 ones' time, and come out as in 32 bits;
//   - 8-bit keys have no such partner (products of 8-bit codes are off by 2^-11 of the largest one), and a wave
//     converts its operands, exactly (460 us with 8 bits for the case above), a lane having dims
//     32 (2 (kk / 4) + hh) + 8 (kk % 4) .. of score product kk, which lie side by side and under one scale.
// A value's scale multiplies the weight of its token, before its rounding to bf16, which is one, as in the bf16 prefill:
// a second part of the weights, as the decode takes it, would be as many value products again, half as much matrix
// work more. A token whose scale is NaN makes NaN of all columns where all see it, however small its weight. In the
// last tiles, which some columns see only in part, the columns that see such a token are noted and its scale is cleared
// for the others, whose weight for it is 0; so are scales of slots past the sequence's end. (Noting in every tile,
// beside products where 0 times NaN is 0, took 0.5-2% longer.)
// Step kt: value products of tile kt - 1, the softmax of tile kt, score products of tile kt + 1 and the conversion
// of V(kt) are one block; K(kt + 2) and the codes of V(kt + 1) are loaded. Of the case above the step's vector
// work is 1.2 times the bf16 kernel's (32 products with scales), its time 415 us against 415-440, and 395 (980
// TFLOP/s) with the plan below; with 64 dims, where vector work weighs more, 1.16 times the bf16 kernel's.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "launch.h"
#include "prefill_impl.h"
#include "quant.h"

namespace pkv {
namespace {

constexpr int32_t kMostSplits = 64;  // (a lane each in the merge)
// Sequences up to which every wave ranks them for itself (seq_at_rank). With 64, 24 to 48 sequences take 2-6% longer.
constexpr int32_t kMostRanked = 16;

using pre::kCols;
using pre::kKeys;
using pre::kThreads;
using pre::kWaves;
using qnt::i32x8;
using qnt::kParts;

struct QuantPrefillArgs {
  const uint8_t* cache;
  const uint16_t* q;
  const int32_t* tables;
  const int32_t* cached_lens;
  const int32_t* cu_new_lens;
  uint16_t* out;
  float* lse;
  float* ws_o;
  float* ws_ml;
  const int32_t* order;
  int32_t max_blocks, num_seqs, hq, hkv, num_blocks, qtiles, split_keys, nsplit;
  bool by_rank;
  float scale_log2;
};

// What a column's weights are relative to is kept this many powers of two above the largest score seen when it was
// set, and moved when a score passes it: weights are at most 1, and sums of large finite values have as much room.
constexpr float kSlack = 8.f;

// (the outputs leave through the values' space, after the last product)
template <int D, int BITS>
struct CodeSmem {
  using S = qnt::Slab<D, BITS>;
  uint8_t k[2][4][S::kCodes + D / 2];             // a tile's four blocks: codes, then scales
  uint8_t vc[2][4][S::kCodes + 4 * kBlockSize];   // likewise
  uint16_t v[2][4][D * kBlockSize];  // values as bf16: [dim][16 slots], halves of odd eights of dims swapped
};

// The lane index afresh where it is used, so that nothing made of it is kept in registers through the steps.
__device__ __forceinline__ int lane_now() {
#if __HIP_DEVICE_COMPILE__
  int lane;
  asm volatile("v_and_b32 %0, 63, %1" : "=v"(lane) : "v"((int)threadIdx.x));
  return lane;
#else
  return 0;
#endif
}

// kBytes bytes, 16 a lane, from a slab of kSlab bytes to LDS (at: 16 lane from where they begin).
template <int kBytes, int kSlab>
__device__ __forceinline__ void load_codes(const uint8_t* slab, int at, uint8_t* to, int lane) {
  if constexpr (kBytes >= 1024) lds_load16(slab, kSlab, at, to);
  if constexpr (kBytes >= 2048) lds_load16<1024>(slab, kSlab, at, to);
  constexpr int kLeft = kBytes % 1024, kAt = kBytes - kLeft;
  if (lane < kLeft / 16) lds_load16<kAt>(slab, kSlab, at, to);
}

// The product of 4-bit codes (A) and a part of the queries (B, e2m3), 32x32x64. Lane l holds k 32 (l / 32) .. of A's
// row and of B's column l % 32, and their scales for these in byte kA of ka and byte kB of kb.
template <int kA, int kB>
__device__ __forceinline__ f32x16 mfma_codes(i32x8 x, i32x8 y, f32x16 c, uint32_t ka, uint32_t kb) {
#if __HIP_DEVICE_COMPILE__
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 2, kA, (int)ka, kB, (int)kb);
#else
  return c;
#endif
}

// The queries as the score products' operands, and the products' number for a tile.
template <int D, int BITS>
struct Queries {  // 4 bits: dims 32 (2 u + hh) .. in parts
  static constexpr int kProducts = D / 32 * kParts;
  i32x8 part[D / 64][kParts];
  uint32_t scale[D / 64];
  __device__ __forceinline__ void load(const uint16_t* row, int hh, bool ok) {
#pragma unroll
    for (int u = 0; u < D / 64; ++u) {
      qnt::u32x16 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const u32x4 y = ld16(row + u * 64 + hh * 32 + e * 8);
#pragma unroll
        for (int f = 0; f < 4; ++f) x[4 * e + f] = ok ? y[f] : 0u;
      }
      scale[u] = qnt::query_parts(x, part[u]);
    }
  }
};
template <int D>
struct Queries<D, 8> {  // dims 32 (2 (kk / 4) + hh) + 8 (kk % 4) ..
  static constexpr int kProducts = D / 8;
  bf16x8 x[D / 16];
  __device__ __forceinline__ void load(const uint16_t* row, int hh, bool ok) {
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      const u32x4 zero = {0u, 0u, 0u, 0u};
      const u32x4 y = ld16(row + kk / 4 * 64 + hh * 32 + kk % 4 * 8);
      x[kk] = as_bf16x8(ok ? y : zero);
    }
  }
};

template <int D, int BITS>
__device__ __forceinline__ void quant_prefill_item(const QuantPrefillArgs& a, const int i, const int kvh,
                                                   const int qt, const int p, const int row0, const int n,
                                                   const int split, CodeSmem<D, BITS>& sm) {
  using S = qnt::Slab<D, BITS>;
  constexpr int DB = D / 32;   // output blocks
  constexpr int kGroups = DB;  // groups that a tile's score products, and its value products, are issued in
  constexpr int kAhead = D == 64 ? 4 : 3;  // fragments of values read ahead of their products
  constexpr int kSums = D == 64 ? 4 : 2;  // partial sums of weights (as many as registers allow)
  constexpr int QOPS = Queries<D, BITS>::kProducts / kGroups, VOPS = 4;
  const int32_t* table = a.tables + (size_t)i * a.max_blocks;
  const int g = a.hq / a.hkv;
  const int ncols = n * g;
  const int col0 = qt * kCols;
  const int len = p + n;
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, lc = lane & 31, hh = lane >> 5;
  const int gcol = col0 + wave * 32 + lc;
  const bool col_ok = gcol < ncols;
  const int j = col_ok ? gcol / g : n - 1;
  const int lim_h = p + j - 8 * hh;  // last key this column sees, less the lane's offset within a block
  const int jmax = min(n - 1, (col0 + kCols - 1) / g);
  const int ntiles = (p + jmax + kKeys) / kKeys;
  const int kt0 = a.split_keys > 0 ? split * (a.split_keys / kKeys) : 0;
  const int kt_end = a.split_keys > 0 ? min(ntiles, kt0 + a.split_keys / kKeys) : ntiles;
  if (kt0 >= kt_end) return;  // (workgroup-uniform) an empty split
  const int nt = kt_end - kt0;
  const int wcol0 = col0 + wave * 32;
  const int j_lo = __builtin_amdgcn_readfirstlane(col0 / g);  // (a quotient stays in vector registers otherwise)
  const int wj_lo = __builtin_amdgcn_readfirstlane(min(wcol0 / g, n - 1));
  const bool wave_live = wcol0 < ncols;

  f32x16 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[db][r] = 0.f;
  float m = -INFINITY, lpart = 0.f;
  uint64_t hurt = 0;  // lanes whose column sees a value noted as NaN
  Queries<D, BITS> qf;

  // ---- the wave's blocks: lane l holds the one that the wave loads of tile kt0 + 64 c + l, where the sequence's
  // first block (or block 0) stands in past the sequence, the table and outside the pool ----
  auto checked = [&](int e, int other) { return e >= 0 && e < a.num_blocks ? e : other; };
  const int first = checked(table[0], 0);
  auto blocks_from = [&](int kt) {
    const int e = (kt + lane_now()) * 4 + wave;
    return e < a.max_blocks && e * kBlockSize < len ? checked(table[e], first) : first;
  };
  int blocks = blocks_from(kt0);
  const uint8_t* slab;  // of the newest tile whose keys are loaded or on their way
  auto next_slab = [&](int kt) {
    const int at = (kt - kt0) & 63;
    if (at == 0 && kt != kt0) blocks = blocks_from(kt);
    slab = a.cache + ((size_t)__builtin_amdgcn_readlane(blocks, at) * a.hkv + kvh) * S::kBytes;
  };
  auto issue_k = [&](auto buf) {
    const int ln = D == 64 ? lane : lane_now();  // (128 dims leave no register for it)
    load_codes<S::kCodes + D / 2, S::kBytes>(slab, ln * 16, sm.k[buf][wave], ln);
  };
  auto issue_v = [&](auto buf) {
    const int ln = D == 64 ? lane : lane_now();
    load_codes<S::kCodes + 4 * kBlockSize, S::kBytes>(slab, S::kValues + ln * 16, sm.vc[buf][wave], ln);
  };

  // ---- values: the wave's own block of a tile, from codes to bf16 ----
  const int col = lane & 15, quarter = lane >> 4;
  uint32_t vw[S::kWords];
  auto read_codes = [&](int kt, auto buf, auto last) {
    const uint8_t* at = &sm.vc[buf][wave][lane * (S::kLane < 16 ? S::kLane : 16)];
    if constexpr (S::kLane == 8) {
      const u32x2 x = ld8(at);
      vw[0] = x[0], vw[1] = x[1];
    } else {
#pragma unroll
      for (int u = 0; u < S::kLane / 16; ++u) {
        const u32x4 x = ld16(at + u * 1024);
#pragma unroll
        for (int e = 0; e < 4; ++e) vw[4 * u + e] = x[e];
      }
    }
    if constexpr (BITS == 8 && decltype(last)::value) {
      // (slots past the sequence's end may hold anything; codes of 4 bits are all finite)
      const int keep = min(max(len - kt * kKeys - wave * kBlockSize - 4 * quarter, 0), 4);
      const uint32_t mask = keep == 4 ? ~0u : (1u << 8 * keep) - 1u;
#pragma unroll
      for (int e = 0; e < S::kWords; ++e) vw[e] &= mask;
    }
  };
  const int v_to = (2 * col + ((quarter >> 1) ^ (col >> 3))) * 8 + (quarter & 1) * 4;
  auto land = [&](auto buf, auto part) {  // dims 16 part ..
    constexpr int kA = decltype(part)::value;
    st8(&sm.v[buf][wave][v_to + kA * 16 * kBlockSize], qnt::four_bf16<BITS, kA>(vw));
  };
  auto land_some = [&](auto buf, auto first, auto end) {
    constexpr int kA = decltype(first)::value, kEnd = decltype(end)::value;
    if constexpr (kA < kEnd) land(buf, std::integral_constant<int, kA>());
    if constexpr (kA + 1 < kEnd) land(buf, std::integral_constant<int, kA + 1>());
    if constexpr (kA + 2 < kEnd) land(buf, std::integral_constant<int, kA + 2>());
    if constexpr (kA + 3 < kEnd) land(buf, std::integral_constant<int, kA + 3>());
    static_assert(kEnd - kA <= 4, "dims of a call");
  };
  const int vread = (2 * lc + (hh ^ ((lc >> 3) & 1))) * 8;
  auto value_frag = [&](int buf, int f) {
    return ld16(&sm.v[buf][f / DB][vread + f % DB * 512]);
  };

  // ---- key operands: the lane's key of half-tile beta is block 2 beta + lc / 16, slot swap23(lc % 16)
  // (prefill_impl.h has why) ----
  const int slot = pre::swap23(lc & 15), blk = lc >> 4;
  uint32_t ks[2];  // the scale bytes of groups hh and 2 + hh, in bytes 0 and 2
  auto read_ks = [&](int buf) {
#pragma unroll
    for (int beta = 0; beta < 2; ++beta) {
      const uint8_t* at = &sm.k[buf][2 * beta + blk][S::kCodes + slot * (D / 32)];
      if constexpr (D == 128) ks[beta] = *reinterpret_cast<const uint32_t*>(at) >> (lane_now() >> 2 & 8);
      else ks[beta] = at[hh];
    }
  };
  // 16 bytes of codes: dims 32 (2 u + hh) .., 16 i further on with 8 bits
  auto key_codes = [&](int buf, int beta, int u, int i) {
    return ld16(&sm.k[buf][2 * beta + blk][((2 * u + hh) * (BITS / 4) + i) * 256 + slot * 16]);
  };
  // The score products of group kG of kGroups. 4 bits: product t takes dims 64 (t / 6) .., part t / 2 % 3 of the
  // queries, half-tile t % 2; 8 bits: dims 16 of kk = 2 kG + t / 2, half-tile t % 2. kc: codes, read ahead.
  u32x4 kc[2][2];
  auto read_first_codes = [&](int buf) {
    kc[0][0] = key_codes(buf, 0, 0, 0);
    kc[0][1] = key_codes(buf, 1, 0, 0);
  };
  auto scores = [&](auto index, int buf, f32x16 (&sc)[2]) {
    constexpr int kG = decltype(index)::value;
    if constexpr (BITS == 4) {
      if constexpr (D == 128 && kG == 1) {
        kc[1][0] = key_codes(buf, 0, 1, 0);
        kc[1][1] = key_codes(buf, 1, 1, 0);
      }
      auto product = [&](auto number) {  // dims 64 t / 6 .., part t / 2 % 3, half-tile t % 2
        constexpr int t = 3 * kG + decltype(number)::value, u = t / (2 * kParts), i = t / 2 % kParts, beta = t % 2;
        const u32x4 c = kc[u][beta];
        const i32x8 x = {(int)c[0], (int)c[1], (int)c[2], (int)c[3], 0, 0, 0, 0};
        sc[beta] = mfma_codes<2 * u, i>(x, qf.part[u][i], sc[beta], ks[beta], qf.scale[u]);
      };
      product(std::integral_constant<int, 0>());
      product(std::integral_constant<int, 1>());
      product(std::integral_constant<int, 2>());
    } else {
      if constexpr (kG + 1 < kGroups) {
        kc[(kG + 1) & 1][0] = key_codes(buf, 0, (kG + 1) / 2, (kG + 1) % 2);
        kc[(kG + 1) & 1][1] = key_codes(buf, 1, (kG + 1) / 2, (kG + 1) % 2);
      }
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int beta = t % 2, kk = 2 * kG + t / 2;
        const uint32_t byte = kG < 2 ? ks[beta] & 255u : ks[beta] >> 16 & 255u;
        const uint32_t w[2] = {kc[kG & 1][beta][t / 2 * 2], kc[kG & 1][beta][t / 2 * 2 + 1]};
        sc[beta] = mfma32(as_bf16x8(qnt::eight_bf16<BITS>(w, __uint_as_float(byte << 23))), qf.x[kk], sc[beta]);
      }
    }
  };

  // register r of half-tile beta: key key0 + 32 beta + 16 (r / 8) + 8 hh + r % 8
  auto mask_tile = [&](int key0, f32x16 (&sc)[2]) {
    const int d = lim_h - key0;
#pragma unroll
    for (int beta = 0; beta < 2; ++beta)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int c = 32 * beta + 16 * (r >> 3) + (r & 7);
        sc[beta][r] = c <= d ? sc[beta][r] : -INFINITY;
      }
  };
  // Value scales that are not finite, in a tile that not every column sees whole (lane t looks at token t; every
  // wave finds the same ones).
  auto drop_nan = [&](int key0, int buf) {
    const int ln = lane_now();
    uint32_t* scale = reinterpret_cast<uint32_t*>(&sm.vc[buf][ln >> 4][S::kCodes + 4 * (ln & 15)]);
    const bool mine = (*scale & qnt::kInfinite) == qnt::kInfinite;
    const uint64_t bad = __builtin_amdgcn_ballot_w64(mine);
    if (bad == 0) return;
    const int last = lim_h + (ln >> 2 & 8) - key0;  // the last token of the tile that the column sees
    const uint64_t seen = last < 0 ? 0 : last >= 63 ? ~uint64_t(0) : (uint64_t(2) << last) - 1;
    hurt |= __builtin_amdgcn_ballot_w64((bad & seen) != 0);
    __syncthreads();  // (all waves have looked)
    if (mine && wave == 0) *scale = 0u;
    __syncthreads();
  };
  // a slice's four tokens' value scales: half e2 of the eight of (beta, u)
  auto read_scales = [&](int buf, int b, int e2) {
    return ld16(&sm.vc[buf][b][S::kCodes + 4 * (8 * hh + 4 * e2)]);
  };
  auto weight_pair = [&](const f32x16 (&sc)[2], int b, int e, const u32x4& s, float neg_m, float (&sum)[kSums]) {
    const int beta = b >> 1, u = b & 1;
    const float x = fast_exp2(__builtin_fmaf(sc[beta][8 * u + 2 * e], a.scale_log2, neg_m));
    const float y = fast_exp2(__builtin_fmaf(sc[beta][8 * u + 2 * e + 1], a.scale_log2, neg_m));
    sum[2 * e % kSums] += x;
    sum[(2 * e + 1) % kSums] += y;
    return pack_bf16x2(x * __uint_as_float(s[2 * (e & 1)]), y * __uint_as_float(s[2 * (e & 1) + 1]));
  };
  auto total = [&](const float (&sum)[kSums]) {
    if constexpr (kSums == 2) return sum[0] + sum[1];
    else return (sum[0] + sum[1]) + (sum[2] + sum[3]);
  };
  auto weights = [&](int buf, f32x16 (&sc)[2], bf16x8 (&pw)[2][2]) {
    float sum[kSums] = {};
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const u32x4 s = read_scales(buf, b, e >> 1);
        w[e] = weight_pair(sc, b, e, s, -m, sum);
      }
      pw[b >> 1][b & 1] = as_bf16x8(w);
      __builtin_amdgcn_sched_barrier(0);  // (registers for one block's scales)
    }
    return total(sum);
  };

  // The matrix-core work of a step, in groups: value products of tile kt - 1 with the weights pw (PV), then score
  // products of the keys of tile kt + 1 (QK), which take the registers that pw leaves; beside them the sixteen
  // slices of the softmax of cur (SM) and the landing of the wave's block of V(kt) (LAND; last: kt is the item's
  // last tile).
  auto block = [&](auto qk, auto pv, auto smx, auto landing, auto last, int kt, auto buf, f32x16 (&sc)[2],
                   const bf16x8 (&pw)[2][2], const f32x16 (&cur)[2], bf16x8 (&pcur)[2][2], float (&sum)[kSums]) {
    constexpr bool QK = decltype(qk)::value, PV = decltype(pv)::value, SM = decltype(smx)::value;
    constexpr bool LAND = decltype(landing)::value;
    constexpr int GV = PV ? kGroups : 0, NG = GV + (QK ? kGroups : 0);
    constexpr int SLICES = SM ? 16 / NG : 0;
    constexpr int CHUNKS = LAND ? D / 16 : 0;
    constexpr int kbuf = 1 - decltype(buf)::value, vbuf = kbuf;
    const float neg_m = -m;
    uint32_t w[4][4];
    constexpr int QUADS = SLICES / 2;  // value scales of a group's slices, read a group ahead
    u32x4 s[2][QUADS > 0 ? QUADS : 1];
    u32x4 fr[8];
    auto scales_of = [&](int index, int group) {
#pragma unroll
      for (int h = 0; h < QUADS; ++h) {
        const int quad = QUADS * group + h;
        s[index][h] = read_scales(buf, quad >> 1, quad & 1);
      }
    };
    if constexpr (SM) scales_of(0, 0);
    if constexpr (PV) {
#pragma unroll
      for (int f = 0; f < kAhead; ++f) fr[f] = value_frag(vbuf, f);
    } else {
      read_ks(kbuf);
      read_first_codes(kbuf);
    }
    if constexpr (LAND) read_codes(kt, buf, last);
    using std::integral_constant;
    auto group = [&](auto index) {
      constexpr int G = decltype(index)::value;
      if constexpr (SM && G + 1 < NG) scales_of((G + 1) & 1, G + 1);
      if constexpr (G < GV) {
#pragma unroll
        for (int k = 0; k < VOPS; ++k) {
          const int f = G * VOPS + k, b = f / DB;
          if (f + kAhead < 4 * DB) fr[(f + kAhead) & 7] = value_frag(vbuf, f + kAhead);
          o[f % DB] = mfma32(as_bf16x8(fr[f & 7]), pw[b >> 1][b & 1], o[f % DB]);
        }
        if constexpr (QK && G == GV - 1) {
          read_ks(kbuf);
          read_first_codes(kbuf);
        }
      } else {
        scores(integral_constant<int, G - GV>(), kbuf, sc);
      }
#pragma unroll
      for (int h = 0; h < SLICES; ++h) {
        const int it = SLICES * G + h;  // slice (b, e)
        const int b = it >> 2, e = it & 3;
        w[b][e] = weight_pair(cur, b, e, s[G & 1][h / 2], neg_m, sum);
        asm volatile("" ::"v"(w[b][e]));  // the pack stays in this group
      }
      if constexpr (LAND)
        land_some(buf, std::integral_constant<int, G * CHUNKS / NG>(),
                  std::integral_constant<int, (G + 1) * CHUNKS / NG>());
      constexpr int kOps = G < GV ? VOPS : QOPS;
      constexpr int kVec = (SM ? 9 * SLICES : 0) + 2 * CHUNKS / NG + (BITS == 8 && G >= GV ? 16 : 1);
      if constexpr (G == 0) {  // the first operands are on their way
        __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, kVec / 2, 0);
      }
#pragma unroll
      for (int k = 0; k < kOps; ++k) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // 1 MFMA
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);  // LDS reads
        __builtin_amdgcn_sched_group_barrier(0x002, (kVec + kOps - 1) / kOps, 0);  // vector ops
        __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);  // an LDS write
      }
      // (the products stay in this group: the compiler takes them for pure, and would move them to their use)
      if constexpr (G >= GV) asm volatile("" ::"v"(sc[0]), "v"(sc[1]));
      __builtin_amdgcn_sched_barrier(0);
    };
    group(integral_constant<int, 0>());
    group(integral_constant<int, 1>());
    if constexpr (NG > 2) {
      group(integral_constant<int, 2>());
      group(integral_constant<int, 3>());
    }
    if constexpr (NG > 4) {
      group(integral_constant<int, 4>());
      group(integral_constant<int, 5>());
      group(integral_constant<int, 6>());
      group(integral_constant<int, 7>());
    }
    if constexpr (SM) {
#pragma unroll
      for (int b = 0; b < 4; ++b) pcur[b >> 1][b & 1] = as_bf16x8(u32x4{w[b][0], w[b][1], w[b][2], w[b][3]});
    }
  };
  auto zero_scores = [&](f32x16 (&sc)[2]) {
#pragma unroll
    for (int beta = 0; beta < 2; ++beta)
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[beta][r] = 0.f;
  };
  using yes_t = std::true_type;
  using no_t = std::false_type;

  auto land_all = [&](int kt, auto buf, auto last) {
    read_codes(kt, buf, last);
    land_some(buf, std::integral_constant<int, 0>(), std::integral_constant<int, 4>());
    if constexpr (D == 128)
      land_some(buf, std::integral_constant<int, 4>(), std::integral_constant<int, 8>());
  };
  auto step = [&](auto has_prev, auto has_next, int kt, auto buf, f32x16 (&cur)[2], f32x16 (&nxt)[2],
                  bf16x8 (&pprev)[2][2], bf16x8 (&pcur)[2][2]) {
    constexpr bool HN = decltype(has_next)::value, HP = decltype(has_prev)::value;
    using last_t = std::integral_constant<bool, !HN>;
    pre::wait_vmem();
    __syncthreads();  // K(kt + 1), V(kt)'s codes and V(kt - 1) have landed; all waves are done with step kt - 1
    if constexpr (HN) issue_v(std::integral_constant<int, 1 - decltype(buf)::value>());
    if (kt + 2 < kt_end) {
      next_slab(kt + 2);
      issue_k(buf);
    }
    const int key0 = kt * kKeys;
    if (key0 + kKeys - 1 > p + j_lo) drop_nan(key0, buf);
    if (!wave_live) {
      land_all(kt, buf, last_t());
      return;
    }
    if (key0 + kKeys - 1 > p + wj_lo) mask_tile(key0, cur);
    __builtin_amdgcn_s_setprio(2);
    float lnew = 0.f;
    float sum[kSums] = {};
    if constexpr (HN) zero_scores(nxt);
    if constexpr (HP) {
      block(has_next, yes_t(), yes_t(), yes_t(), last_t(), kt, buf, nxt, pprev, cur, pcur, sum);
      lnew = total(sum);
    } else {
      if constexpr (HN) block(yes_t(), no_t(), no_t(), yes_t(), last_t(), kt, buf, nxt, pprev, cur, pcur, sum);
      else land_all(kt, buf, last_t());
      const u32x4 zero = {0u, 0u, 0u, 0u};
#pragma unroll
      for (int b = 0; b < 4; ++b) pcur[b >> 1][b & 1] = as_bf16x8(zero);
    }
    asm volatile("" ::"v"(__builtin_bit_cast(u32x4, pcur[0][0])),
                 "v"(__builtin_bit_cast(u32x4, pcur[0][1])),
                 "v"(__builtin_bit_cast(u32x4, pcur[1][0])),
                 "v"(__builtin_bit_cast(u32x4, pcur[1][1])), "v"(lnew));
    __builtin_amdgcn_s_setprio(0);
    bool check = true;
    if constexpr (HP) check = __builtin_amdgcn_ballot_w64(!(lnew <= 1.f)) != 0;
    if (check) {
      float mx = -INFINITY;
#pragma unroll
      for (int beta = 0; beta < 2; ++beta)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, cur[beta][r]);
      mx = fmaxf(mx, pre::swap_halves(mx)) * a.scale_log2;
      const bool grow = mx > m;
      if (__builtin_amdgcn_ballot_w64(grow)) {
        const float m_new = grow ? mx + kSlack : m;
        const float alpha = fast_exp2(m - m_new);
        m = m_new;
        lpart *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[db][r] *= alpha;
        lnew = weights(buf, cur, pcur);
      }
    }
    lpart += lnew;
  };

  // prologue
  using even_t = std::integral_constant<int, 0>;  // (tile kt's buffers are those of kt - kt0's parity)
  using odd_t = std::integral_constant<int, 1>;
  next_slab(kt0);
  issue_k(even_t());
  issue_v(even_t());
  if (nt > 1) {
    next_slab(kt0 + 1);
    issue_k(odd_t());
  }
  {
    const int head = kvh * g + gcol % g;  // (a lane past the last column reads a valid row)
    qf.load(a.q + ((size_t)(row0 + j) * a.hq + (col_ok ? head : kvh * g)) * D, hh, col_ok);
  }
  pre::wait_vmem();
  __syncthreads();
  f32x16 sa[2], sb[2];
  bf16x8 pa[2][2], pb[2][2];
  if (wave_live) {
    float sum[kSums];
    zero_scores(sa);
    block(yes_t(), no_t(), no_t(), no_t(), no_t(), kt0 - 1, odd_t(), sa, pa, sb, pb, sum);
  }
  if (nt == 1) {
    step(no_t(), no_t(), kt0, even_t(), sa, sb, pb, pa);
  } else {
    step(no_t(), yes_t(), kt0, even_t(), sa, sb, pb, pa);
    int kt = kt0 + 1;
    for (; kt + 2 < kt_end; kt += 2) {
      step(yes_t(), yes_t(), kt, odd_t(), sb, sa, pa, pb);
      step(yes_t(), yes_t(), kt + 1, even_t(), sa, sb, pb, pa);
    }
    if (kt + 1 < kt_end) {
      step(yes_t(), yes_t(), kt, odd_t(), sb, sa, pa, pb);
      step(yes_t(), no_t(), kt + 1, even_t(), sa, sb, pb, pa);
    } else {
      step(yes_t(), no_t(), kt, odd_t(), sb, sa, pa, pb);
    }
  }
  // value products of the last tile
  __syncthreads();
  if (wave_live) {
    float sum[kSums];
    if (nt & 1) block(no_t(), yes_t(), no_t(), no_t(), no_t(), kt_end, odd_t(), sa, pa, sb, pb, sum);
    else block(no_t(), yes_t(), no_t(), no_t(), no_t(), kt_end, even_t(), sa, pb, sb, pa, sum);
  }
  __syncthreads();  // (the outputs take the values' space)

  const float l = lpart + pre::swap_halves(lpart);
  if (!wave_live) return;
  constexpr int CH = D / 8;     // 16-byte units per row
  constexpr int RPI = 64 / CH;  // rows per store
  uint16_t* tile = &sm.v[0][0][0] + wave * 32 * D;
  const int ln = lane_now();
  const int lcl = ln & 31, hhl = ln >> 5;
  if (hurt != 0) {
    const bool mine = (hurt >> ln & 1) != 0;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[db][r] = mine ? __uint_as_float(0x7FC00000u) : o[db][r];
  }
  // registers 4 r .. 4 r + 3 of output block db: dims 32 db + 8 r + 4 hhl ..
  auto unit = [&](int db, int r) { return 4 * db + r; };
  if (a.split_keys > 0) {
    const int gcp = wcol0 + lcl;
    const int jp = gcp / g;
    if (gcp < ncols && p + jp >= a.split_keys && p + jp >= kt0 * kKeys) {
      const size_t at =
          ((size_t)(row0 + jp) * a.hq + kvh * g + gcp % g) * (size_t)a.nsplit + (size_t)split;
      float* wo = a.ws_o + at * D + 4 * hhl;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          st16(wo + 8 * unit(db, r),
               u32x4{__float_as_uint(o[db][4 * r + 0]), __float_as_uint(o[db][4 * r + 1]),
                     __float_as_uint(o[db][4 * r + 2]), __float_as_uint(o[db][4 * r + 3])});
      if (hhl == 0) {
        a.ws_ml[at * 2 + 0] = m;
        a.ws_ml[at * 2 + 1] = l;
      }
    }
    if (split > 0) return;
  }
  auto row_ends_here = [&](int gc) { return a.split_keys == 0 || p + gc / g < a.split_keys; };
  const float inv = 1.f / l;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const u32x2 x = {pack_bf16x2(o[db][4 * r + 0] * inv, o[db][4 * r + 1] * inv),
                       pack_bf16x2(o[db][4 * r + 2] * inv, o[db][4 * r + 3] * inv)};
      st8(tile + lcl * D + (unit(db, r) ^ (lcl % CH)) * 8 + 4 * hhl, x);
    }
#pragma unroll
  for (int k = 0; k < 32 / RPI; ++k) {
    const int r = k * RPI + ln / CH;
    const int u = ln % CH;
    const u32x4 x = ld16(tile + r * D + ((u ^ (r % CH)) * 8));
    const int gc = wcol0 + r;
    if (gc < ncols && row_ends_here(gc))
      st16_nt(a.out + ((size_t)(row0 + gc / g) * a.hq + kvh * g + gc % g) * D + u * 8, x);
  }
  const int gcl = wcol0 + lcl;
  if (a.lse != nullptr && hhl == 0 && gcl < ncols && row_ends_here(gcl))
    a.lse[(size_t)(row0 + gcl / g) * a.hq + kvh * g + gcl % g] = (m + log2f(l)) * kLn2;
}

// One item per workgroup, in the order of the bf16 prefill (prefill_body has the reasons).
template <int D, int BITS>
__global__ __attribute__((amdgpu_flat_work_group_size(kThreads, kThreads), amdgpu_waves_per_eu(2, 2)))
void quant_prefill_kernel(const QuantPrefillArgs a) {
  __shared__ __align__(16) CodeSmem<D, BITS> sm;
  const int per = a.qtiles * a.nsplit;
  const int xcd = blockIdx.x & 7, pos = blockIdx.x >> 3;
  const int gpos = pos / per, group = gpos * 8 + xcd;
  const int idx = (pos % per + gpos) % per;
  const int qt = a.qtiles - 1 - idx / a.nsplit, split = idx % a.nsplit;
  if (group >= a.num_seqs * a.hkv) return;
  const int kvh = group % a.hkv;
  const int i = a.order != nullptr ? a.order[group / a.hkv]
                : a.by_rank ? seq_at_rank(a.cached_lens, a.cu_new_lens, a.num_seqs, group / a.hkv)
                            : group / a.hkv;
  const int p = a.cached_lens[i], row0 = a.cu_new_lens[i];
  const int n = a.cu_new_lens[i + 1] - row0;
  if (qt * kCols >= n * (a.hq / a.hkv)) return;
  quant_prefill_item<D, BITS>(a, i, kvh, qt, p, row0, n, split, sm);
}

// The splits' partial results of a row that reaches past split 0 (sequence blockIdx.y, one wave per query head)
// by their log-sum-exp weights.
template <int D>
__global__ __launch_bounds__(kThreads) void quant_prefill_merge_kernel(const QuantPrefillArgs a) {
  constexpr int PER = D / 64;
  const int i = blockIdx.y, lane = threadIdx.x & 63;
  const int r = (int)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row0 = a.cu_new_lens[i], n = a.cu_new_lens[i + 1] - row0;
  const int j = r / a.hq;
  if (j >= n) return;
  const int splits = (a.cached_lens[i] + j) / a.split_keys + 1;  // that the row reaches
  if (splits == 1) return;                                       // (written already)
  const size_t row = (size_t)(row0 + j) * a.hq + r % a.hq, at = row * a.nsplit;
  const float m = lane < splits ? a.ws_ml[(at + lane) * 2] : -INFINITY;
  const float l = lane < splits ? a.ws_ml[(at + lane) * 2 + 1] : 0.f;
  const float top = wave_all(m, Max());
  const float w = lane < splits ? fast_exp2(m - top) : 0.f;
  const float den = wave_all(w * l, Add());
  float o[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) o[e] = 0.f;
  const float* src = a.ws_o + at * D + lane * PER;
  for (int s = 0; s < splits; s += 8) add_partials<D>(src, w, s, splits, o);
  const float inv = 1.f / den;
  uint16_t* to = a.out + row * D + lane * PER;
  const uint32_t pair = pack_bf16x2(o[0] * inv, o[PER - 1] * inv);
  if constexpr (PER == 2) *reinterpret_cast<uint32_t*>(to) = pair;
  else *to = (uint16_t)pair;
  if (a.lse != nullptr && lane == 0) a.lse[row] = (top + log2f(den)) * kLn2;
}

// How a call is cut, by host arithmetic on its sizes: about `tiles` work items (kv head, 128 columns) on 512 places.
// Measured with 4 bits, lengths spread evenly, us, `none` and splits of that many keys:
//   - items that fill the chip are not split, but sequences taken longest first (a split costs 4 bytes per output dim
//     written and read: 24 suffixes of 50-300 tokens over 500-4000, 32/8 heads of 128, 201 without order, 185 with it,
//     211 with 3008; 128 single rows over 500-16000 316, and 388; but 450 items and more of one column tile each end
//     with the longest: 64 rows over 4000-60000 986, and 699);
//   - a few items are cut so that they fill it once (one of 400 over 16000, 32/8 heads of 128: 120 with 4096, 140 with
//     3328, 127 with 2048, 144 with 1024; one of 64 over 60000 77 with 2048, 91 with 1024), into 32 splits at most
//     and of 768 keys at least (one of 100 over 4000 27 with 768, 28 with 512, 30 with 1024);
//   - between these, splits of 3008 keys even out the lengths (40 of 30-100 over 2000-20000, 16/4 heads of 64: 209, 217
//     with 1536, 211 with 4096; 3 of 101-509 over 4096-16384, 32/8 of 128, 183, 193 and 208), or of 1536 for the
//     fewer of 64 dims (the same 3 101, 97 and 119; 32 of 1-8 over 4000-30000 96, 91.5 and 111).
PrefillSplit quant_prefill_plan(int32_t num_seqs, int32_t total_new, int32_t hq, int32_t hkv, int32_t head_dim,
                                int32_t max_new_len, int32_t max_total_len) {
  PrefillSplit sp{0, 1, false};
  if (num_seqs <= 0 || total_new <= 0 || hkv <= 0 || hq <= 0 || hq % hkv != 0 || max_new_len <= 0) return sp;
  const int64_t columns = (int64_t)total_new * (hq / hkv);
  const int64_t most = ((int64_t)max_new_len * (hq / hkv) + kCols - 1) / kCols;  // column tiles of a sequence
  const int64_t tiles = hkv * std::clamp<int64_t>((columns + num_seqs * (kCols / 2) + kCols - 1) / kCols, num_seqs,
                                                  num_seqs * most);
  // (the order is a launch of its own above kMostRanked sequences)
  sp.order = num_seqs > 1 && (num_seqs <= kMostRanked || (max_total_len >= 2048 && tiles >= 100));
  if (tiles >= 640 || (tiles >= 450 && columns >= (int64_t)num_seqs * 2 * kCols)) return sp;
  int64_t keys = head_dim == 64 && tiles < 250 ? 1536 : 3008;
  if (tiles <= 110) keys = std::max<int64_t>(768, max_total_len / std::min<int64_t>(32, 512 / tiles) + kKeys);
  else keys = std::max<int64_t>(keys, max_total_len / (4096 / tiles) + kKeys);
  keys = std::max<int64_t>(keys, max_total_len / kMostSplits + kKeys) / kKeys * kKeys;
  if (keys > 4096 && keys < 4500) keys = 4096;  // (the tiles whose blocks a wave holds: 120 against 128 with 4160)
  if (max_total_len <= keys) return sp;
  sp.split_keys = (int32_t)keys;
  sp.nsplit = (int32_t)((max_total_len + keys - 1) / keys);
  return sp;
}

}  // namespace

size_t quant_prefill_workspace_bytes(int32_t num_seqs, int32_t total_new, int32_t hq, int32_t hkv,
                                     int32_t head_dim, int32_t max_new_len, int32_t max_total_len) {
  const PrefillSplit sp = quant_prefill_plan(num_seqs, total_new, hq, hkv, head_dim, max_new_len, max_total_len);
  size_t bytes = sp.order ? order_bytes(num_seqs) : 0;
  if (sp.nsplit > 1) bytes += (size_t)total_new * hq * sp.nsplit * (head_dim + 2) * sizeof(float);
  return bytes;
}

hipError_t launch_quant_prefill(const uint8_t* cache, int32_t num_blocks, int32_t hkv, int32_t head_dim,
                                int32_t bits, const uint16_t* q, int32_t hq,
                                const int32_t* block_tables, int32_t max_blocks,
                                const int32_t* cached_lens, const int32_t* cu_new_lens,
                                int32_t num_seqs, int32_t total_new, int32_t max_new_len,
                                int32_t max_total_len, float scale, uint16_t* out, float* lse,
                                void* workspace, hipStream_t stream) {
  PrefillSplit sp{0, 1, false};
  if (workspace != nullptr)
    sp = quant_prefill_plan(num_seqs, total_new, hq, hkv, head_dim, max_new_len, max_total_len);
  QuantPrefillArgs a{};
  a.cache = cache;
  a.q = q;
  a.tables = block_tables;
  a.cached_lens = cached_lens;
  a.cu_new_lens = cu_new_lens;
  a.out = out;
  a.lse = lse;
  char* ws = static_cast<char*>(workspace);
  a.by_rank = sp.order && num_seqs <= kMostRanked;
  if (sp.order) {
    if (!a.by_rank) {
      int32_t* order = reinterpret_cast<int32_t*>(ws);
      const hipError_t err = launch_seq_order(cached_lens, cu_new_lens, num_seqs, order, stream);
      if (err != hipSuccess) return err;
      a.order = order;
    }
    ws += order_bytes(num_seqs);
  }
  if (sp.nsplit > 1) {
    a.ws_o = reinterpret_cast<float*>(ws);
    a.ws_ml = a.ws_o + (size_t)total_new * hq * sp.nsplit * head_dim;
  }
  const pre::PrefillGrid pg = pre::prefill_grid(hq, hkv, num_seqs, max_new_len, sp.nsplit);
  if (pg.items > INT32_MAX) return hipErrorInvalidValue;
  a.max_blocks = max_blocks;
  a.num_seqs = num_seqs;
  a.hq = hq;
  a.hkv = hkv;
  a.num_blocks = num_blocks;
  a.qtiles = (int32_t)pg.qtiles;
  a.split_keys = sp.split_keys;
  a.nsplit = sp.nsplit;
  a.scale_log2 = scale * kLog2e;
  auto* kern = head_dim == 128 ? (bits == 8 ? quant_prefill_kernel<128, 8> : quant_prefill_kernel<128, 4>)
                               : (bits == 8 ? quant_prefill_kernel<64, 8> : quant_prefill_kernel<64, 4>);
  hipLaunchKernelGGL(kern, dim3((unsigned)pg.items), dim3(kThreads), 0, stream, a);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess || sp.nsplit <= 1) return err;
  hipLaunchKernelGGL((head_dim == 128 ? quant_prefill_merge_kernel<128> : quant_prefill_merge_kernel<64>),
                     dim3((unsigned)(((int64_t)max_new_len * hq + kWaves - 1) / kWaves), (unsigned)num_seqs),
                     dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace pkv
