// Decode attention over a cache held in 8 or 4 bits (gfx950): sequence i's query heads of a kv head attend
// over its keys, out = sum_t softmax_t(scale <q, K[t]>) V[t], as pkv_decode_attention does over bf16.
//
// A wave takes four blocks (64 keys) at a time straight into the matrix-core operands, scores
// S^T = K Q^T and values O^T += V^T P^T, heads as columns. The slab is laid out as the operands are (quant.h),
// so a block's codes are one or two contiguous 16-byte loads of the wave, for keys and for values. Codes
// become bf16 two at a time by the conversion instruction, exactly: keys with their group's power of two,
// values as they are, since a token's value scale multiplies its weight.
//
// A product has 16 columns and a group often fewer heads, so the heads stand in the columns kWays = 2 or 4
// times over (g <= 8, g <= 4), and column (way w, head h) goes on with the scores of blocks w, w + kWays, ...
// alone: every lane's exponentials are of use. A weight goes to the value product in two bf16 parts, itself
// rounded and what that left over, within 2^-16 of itself together; the second stands in the next way's
// column, whose weights for the block would be zeros (kWays 1 takes a second product).
//
// What a weight is relative to is kept kSlack powers of two above the largest score seen when it was set, and
// moved when a score passes it. So weights are at most 1 and most steps need no lane exchange and no
// rescaling; the values of a cache are finite (or NaN), and zero weights are safe with them.
#include <math.h>

#include <algorithm>

#include "decode_impl.h"
#include "launch.h"
#include "quant.h"

namespace pkv {
namespace {

using dec::finite_max;
using qnt::Slab;

constexpr int kStep = 4;  // blocks per step
constexpr int kStepKeys = kStep * kBlockSize;
constexpr float kSlack = 8.f;  // (base 2)
constexpr int kMergeWaves = 4;
constexpr int kMaxSplits = 128;  // (two a lane in the merge)

// A lane's codes of a block: of the keys (slot col, dims D / 4 * grp ..), and of the values (slots
// 4 grp .., dims 16 a + col).
template <int D, int BITS>
struct BlockCodes {
  uint32_t w[Slab<D, BITS>::kWords];
  __device__ __forceinline__ void load(const uint8_t* slab, int first, int offset, int stride) {
    constexpr int kLane = Slab<D, BITS>::kLane;
    if constexpr (kLane == 8) {
      const u32x2 x = buf_ld8(slab, Slab<D, BITS>::kBytes, first + offset);
      w[0] = x[0], w[1] = x[1];
    } else {
#pragma unroll
      for (int u = 0; u < kLane / 16; ++u) {
        const u32x4 x = buf_ld16(slab, Slab<D, BITS>::kBytes, first + offset + u * stride);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[4 * u + e] = x[e];
      }
    }
  }
  __device__ __forceinline__ void read(const uint8_t* at, int stride) {
    constexpr int kLane = Slab<D, BITS>::kLane;
    if constexpr (kLane == 8) {
      const u32x2 x = ld8(at);
      w[0] = x[0], w[1] = x[1];
    } else {
#pragma unroll
      for (int u = 0; u < kLane / 16; ++u) {
        const u32x4 x = ld16(at + u * stride);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[4 * u + e] = x[e];
      }
    }
  }
};
__device__ __forceinline__ uint32_t buf_ld1(const void* base, int bytes, int voffset) {
#if __HIP_DEVICE_COMPILE__
  const __amdgpu_buffer_rsrc_t rsrc =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, bytes, kBufferFlags);
  return __builtin_amdgcn_raw_buffer_load_b8(rsrc, voffset, 0, 0);
#else
  return 0u;
#endif
}

template <int D, int BITS, int kA>
__device__ __forceinline__ void value_products(const BlockCodes<D, BITS>& even,
                                               const BlockCodes<D, BITS>& odd, const bf16x8 p,
                                               f32x4 (&acc)[D / 16]) {
  const u32x2 x = qnt::four_bf16<BITS, kA>(even.w), y = qnt::four_bf16<BITS, kA>(odd.w);
  acc[kA] = mfma16(as_bf16x8(u32x4{x[0], x[1], y[0], y[1]}), p, acc[kA]);
  if constexpr (kA + 1 < D / 16) value_products<D, BITS, kA + 1>(even, odd, p, acc);
}

// Where slabs are small (all but 8 bits and 128 dims) a wave's slabs come through LDS, loaded straight there, keys'
// and values' halves apart: the next step's are on their way from when this step's have been read. The registers
// that codes in flight would take are free for more waves: 128 sequences of 4000-32000 keys, 16/4 heads of 64 dims,
// 4 bits 129 us against 137 with registers (8 bits 225 both), 256 of 512-4096 41.5 and 46.7 (8 bits 69 and 75), 512 of
// 1-300 keys, 32/8 heads of 128, 4 bits 23.6 and 24.9. (Two steps ahead, which leaves two waves a SIMD unit with 128
// dims: 26.1 there, elsewhere within 2%.)
template <int D, int BITS>
struct Ring {
  using S = Slab<D, BITS>;
  static constexpr bool kUsed = S::kBytes <= 2304;
  static constexpr int kKeyBytes = S::kCodes + D / 2, kValueBytes = S::kCodes + 4 * kBlockSize;
  static constexpr int kLoads = kStep * ((kKeyBytes + 1023) / 1024);  // of the keys, or the values, of a step
  static_assert((kKeyBytes + 1023) / 1024 == (kValueBytes + 1023) / 1024 && kLoads < 64, "counted loads");
  uint8_t k[kUsed ? kStep : 1][kKeyBytes];
  uint8_t v[kUsed ? kStep : 1][kValueBytes];
};
template <int kBytes, int kPart = 0>
__device__ __forceinline__ void load_codes(const uint8_t* from, uint8_t* to, int lane) {
  if ((kPart + 1) * 1024 <= kBytes || lane < (kBytes - kPart * 1024) / 16)
    lds_load16(from, kBytes, kPart * 1024 + lane * 16, to + kPart * 1024);
  if constexpr ((kPart + 1) * 1024 < kBytes) load_codes<kBytes, kPart + 1>(from, to, lane);
}
// Wait until at most kLeft of the wave's loads are outstanding (they end in order).
template <int kLeft>
__device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt(0x0F70 | (kLeft & 15) | (kLeft >> 4) << 14);
  asm volatile("" ::: "memory");
}

// Wait until the wave's LDS reads have ended: what they read may be loaded over.
__device__ __forceinline__ void wait_reads() {
  __builtin_amdgcn_s_waitcnt(0xC07F);
  asm volatile("" ::: "memory");
}

// One wave's share: keys [k0, k1) of a sequence, k0 a multiple of 16, not empty. Leaves, summed over the
// ways, the unnormalised output (lane (col, grp) holds dims 16 a + 4 grp + 0..3 of head col % (16 / kWays)),
// what the weights are relative to (base 2) and their sum.
template <int D, int BITS, int kWays>
__device__ __forceinline__ void quant_range(const QuantDecodeArgs& a, const bf16x8 (&qf)[D / 32],
                                            const int32_t* __restrict__ table, const int kvh,
                                            const int k0, const int k1, f32x4 (&acc_out)[D / 16],
                                            float& m_out, float& l_out, Ring<D, BITS>& ring) {
  constexpr bool kRing = Ring<D, BITS>::kUsed;
  constexpr int kRingLoads = Ring<D, BITS>::kLoads;
  using S = Slab<D, BITS>;
  constexpr int KK = D / 32, DB = D / 16;
  constexpr int kMine = kStep / kWays;  // blocks per step whose scores a column goes on with
  const int lane = threadIdx.x & 63;
  const int col = lane & 15, grp = lane >> 4;
  const int way = col / (16 / kWays);
  // offsets of the lane's codes and scales within a slab
  const int key_at = S::kLane == 8 ? (grp / 2) * 256 + col * 16 + (grp & 1) * 8
                                   : grp * (S::kLane / 16) * 256 + col * 16;
  const int key_scale_at = S::kKeyScales + col * (D / 32) + grp * D / 128;
  const int value_at = S::kValues + lane * (S::kLane < 16 ? S::kLane : 16);

  // The range's blocks, 64 at a time: lane l holds the address of slab 64 c + l, where pool block 0 stands in past
  // the range and for entries outside the pool. The next 64 entries are on their way.
  const int b_first = k0 / kBlockSize;
  const int nblk = (k1 - k0 + kBlockSize - 1) / kBlockSize;
  const uint8_t* head = a.cache + (size_t)kvh * S::kBytes;
  const size_t stride = (size_t)a.hkv * S::kBytes;
  auto entries = [&](int c) {
    const int r = 64 * c + lane;
    return r < nblk && b_first + r < a.max_blocks ? table[b_first + r] : 0;
  };
  int slab_lo, slab_hi;
  auto set_slabs = [&](int e) {
    const size_t at = (size_t)head + (size_t)(e < 0 || e >= a.num_blocks ? 0 : e) * stride;
    slab_lo = (int)(uint32_t)at;
    slab_hi = (int)(uint32_t)(at >> 32);
  };
  const int raw0 = entries(0);
  int raw_next = entries(1), chunk = 0, next = 0;  // next: the first block of the step to load, in its 64
  set_slabs(raw0);
  auto next_step = [&] {
    next += kStep;
    if (next == 64) {
      next = 0;
      set_slabs(raw_next);
      raw_next = entries(++chunk + 1);
    }
  };
  auto slab = [&](int i) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane(slab_lo, next + i);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane(slab_hi, next + i);
    return reinterpret_cast<const uint8_t*>((size_t)hi << 32 | lo);
  };

  f32x4 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, lpart = 0.f;

  BlockCodes<D, BITS> k[kStep], v[kStep];
  uint32_t ks[kStep];
  u32x4 vs[kMine];
  auto load_k = [&] {
#pragma unroll
    for (int i = 0; i < kStep; ++i) {
      const uint8_t* s = slab(i);
      if constexpr (kRing) {
        load_codes<Ring<D, BITS>::kKeyBytes>(s, ring.k[i], lane);
      } else {
        k[i].load(s, 0, key_at, 256);
        ks[i] = buf_ld1(s, S::kBytes, key_scale_at);
      }
    }
  };
  auto load_v = [&] {
    if constexpr (kRing) {
#pragma unroll
      for (int i = 0; i < kStep; ++i)
        load_codes<Ring<D, BITS>::kValueBytes>(slab(i) + S::kValues, ring.v[i], lane);
    } else {
#pragma unroll
      for (int i = 0; i < kStep; ++i) v[i].load(slab(i), 0, value_at, 1024);
#pragma unroll
      for (int j = 0; j < kMine; ++j) {
        const uint8_t* s = slab(j * kWays);
#pragma unroll
        for (int w = 1; w < kWays; ++w) {
          const uint8_t* x = slab(j * kWays + w);
          s = way == w ? x : s;
        }
        vs[j] = ld16(s + S::kValueScales + 16 * grp);
      }
    }
  };
  load_k();
  load_v();
  for (int t0 = k0;; t0 += kStepKeys) {
    const bool more = t0 + kStepKeys < k1;
    if constexpr (kRing) {
      wait_loads<kRingLoads>();  // (the values' may still be on their way)
#pragma unroll
      for (int i = 0; i < kStep; ++i) {
        k[i].read(ring.k[i] + key_at, 256);
        ks[i] = ring.k[i][key_scale_at];
      }
    }
    f32x4 st[kStep];
#pragma unroll
    for (int i = 0; i < kStep; ++i) {
      const float scale = __uint_as_float(ks[i] << 23);
      st[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
        st[i] = mfma16(as_bf16x8(qnt::eight_bf16<BITS>(k[i].w + kk * BITS / 4, scale)), qf[kk], st[i]);
    }
    if constexpr (kRing) wait_reads();
    if (more) {
      next_step();
      load_k();  // (in flight through the rest of this step)
    }
    if constexpr (kRing) {
      if (more) wait_loads<kRingLoads>();
      else wait_loads<0>();
#pragma unroll
      for (int i = 0; i < kStep; ++i) v[i].read(ring.v[i] + value_at - S::kValues, 1024);
#pragma unroll
      for (int j = 0; j < kMine; ++j) vs[j] = ld16(ring.v[j * kWays + way] + S::kCodes + 16 * grp);
    }
    // lane holds keys 4 grp + r of its way's blocks
    float sv[kMine][4], weigh[kMine][4];
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float x = st[j * kWays][r];
#pragma unroll
        for (int w = 1; w < kWays; ++w) x = way == w ? st[j * kWays + w][r] : x;
        sv[j][r] = x;
        weigh[j][r] = __uint_as_float(vs[j][r]);
      }
    }
    if (t0 + kStepKeys > k1) {  // slots past the end, which may hold anything
#pragma unroll
      for (int j = 0; j < kMine; ++j) {
        const int left = k1 - t0 - (j * kWays + way) * kBlockSize - 4 * grp;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          sv[j][r] = r < left ? sv[j][r] : -INFINITY;
          weigh[j][r] = r < left ? weigh[j][r] : 0.f;
        }
      }
      if constexpr (BITS == 8) {  // (codes of 4 bits are all finite)
#pragma unroll
        for (int i = 0; i < kStep; ++i) {
          const int left = min(max(k1 - t0 - i * kBlockSize - 4 * grp, 0), 4);
          const uint32_t mask = left == 4 ? ~0u : (1u << 8 * left) - 1u;
#pragma unroll
          for (int e = 0; e < S::kWords; ++e) v[i].w[e] &= mask;
        }
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, sv[j][r]);
    }
    mx *= a.scale_log2;
    if (__builtin_amdgcn_ballot_w64(mx > m) != 0) {
      const float top = ways_max<kWays>(dec::wave_max16(mx));
      const float m_new = top > m ? top + kSlack : m;
      const float alpha = fast_exp2(m - finite_max(m_new));
      m = m_new;
      lpart *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) {
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[db][r] *= alpha;
      }
    }
    const float m_sub = finite_max(m);
    constexpr int kProducts = kWays == 1 ? 2 : 1;
    uint32_t p[kProducts][kStep][2];
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
      float x[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[r] = fast_exp2(fmaf(sv[j][r], a.scale_log2, -m_sub));
        lpart += x[r];
        x[r] *= weigh[j][r];
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        uint32_t first, second;
        two_parts(x[2 * e], x[2 * e + 1], first, second);
        if constexpr (kWays == 1) {
          p[0][j][e] = first;
          p[1][j][e] = second;
        } else {
          // (the second part of the way before, from its columns)
          second = dpp<kWays == 4 ? kRor4 : kRor8>(second);
#pragma unroll
          for (int w = 0; w < kWays; ++w)
            p[0][j * kWays + w][e] = way == w ? first : way == (w + 1) % kWays ? second : 0u;
        }
      }
    }
#pragma unroll
    for (int n = 0; n < kProducts; ++n) {
#pragma unroll
      for (int i = 0; i < kStep; i += 2)
        value_products<D, BITS, 0>(
            v[i], v[i + 1],
            as_bf16x8(u32x4{p[n][i][0], p[n][i][1], p[n][i + 1][0], p[n][i + 1][1]}), acc);
    }
    if (!more) break;
    if constexpr (kRing) wait_reads();
    load_v();
  }
  l_out = ways_sum<kWays>(dec::wave_sum16(lpart));
  m_out = m;
#pragma unroll
  for (int db = 0; db < DB; ++db) {
#pragma unroll
    for (int r = 0; r < 4; ++r) acc_out[db][r] = ways_sum<kWays>(acc[db][r]);
  }
}

// The sequence and split of item seq (wave-uniform) of a kv head: first every split but its sequence's last, then
// the last ones, which may be short; what lies behind is no item. So the grid, which is made for the longest
// sequence, holds what it has to at its start, and short work at its end. Past kListSeqs sequences item s is
// split s % splits of its sequence.
constexpr int kListSeqs = 512;
__device__ __forceinline__ bool find_item(const QuantDecodeArgs& a, int& seq, int& split) {
  const int item = seq, lane = threadIdx.x & 63;
  auto splits_of = [&](int len) { return max((min(len, a.max_len) + a.split_keys - 1) / a.split_keys, 1); };
  if (a.num_seqs > kListSeqs) {
    seq = item / a.splits;
    split = item % a.splits;
    return split < splits_of(a.seq_lens[seq]);
  }
  int before = 0;
  for (int base = 0; base < a.num_seqs; base += 64) {
    const int mine = base + lane < a.num_seqs ? splits_of(a.seq_lens[base + lane]) - 1 : 0;
    const int upto = wave_scan(mine);
    const int all = __builtin_amdgcn_readlane(upto, 63), at = item - before;
    if (at < all) {
      const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > at));
      seq = base + l;
      split = at - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(mine, l));
      return true;
    }
    before += all;
  }
  seq = item - before;
  if (seq >= a.num_seqs) return false;
  split = splits_of(a.seq_lens[seq]) - 1;
  return true;
}

// kParts waves per (sequence, kv head, split): each takes an equal share of the split's keys, and the shares
// meet in LDS. With several splits, the results are partial ones for the merge below.
template <int D, int BITS, int kWays, int kParts>
__global__ __launch_bounds__(64 * kParts) __attribute__((amdgpu_waves_per_eu(BITS == 4 && kWays > 1 ? 3 : 2)))
void quant_decode_kernel(const QuantDecodeArgs a) {
  constexpr int DB = D / 16;
  union Smem {
    dec::DecodeSmem<D, kParts> merge;
    Ring<D, BITS> ring[kParts];
  };
  __shared__ __align__(16) Smem smem;
  auto& sm = smem.merge;
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // (heads side by side, which share their blocks' neighbourhood in memory: with a head's splits side by side 64
  // sequences of 8192-32768 keys, 4 bits, 64/8 heads of 128 dims take 13% longer)
  const int kvh = (int)(blockIdx.x % a.hkv);
  int seq = (int)(blockIdx.x / a.hkv), split = 0;
  if (a.splits > 1 && !find_item(a, seq, split)) return;
  const int g = a.hq / a.hkv;
  const int len = min(a.seq_lens[seq], a.max_len);
  const int k0 = split * a.split_keys;
  const size_t row0 = (size_t)seq * a.hq + kvh * g;
  if (k0 >= len) {  // (workgroup-uniform) nothing here; a sequence without keys gives zeros
    if (len <= 0 && split == 0) {
      for (int u = threadIdx.x; u < g * (D / 8); u += 64 * kParts)
        st16(a.out + row0 * D + u * 8, u32x4{0u, 0u, 0u, 0u});
      if (a.lse != nullptr && (int)threadIdx.x < g) a.lse[row0 + threadIdx.x] = -INFINITY;
    }
    return;
  }
  const int k1 = min(len, k0 + a.split_keys);
  const int share = ((k1 - k0 + kParts - 1) / kParts + kStepKeys - 1) / kStepKeys * kStepKeys;
  const int s0 = min(k0 + wave * share, k1), s1 = min(s0 + share, k1);
  const int h = col % (16 / kWays), way = col / (16 / kWays);
  if (s0 < s1) {
    bf16x8 qf[D / 32];  // the heads kWays times over (zeros past the group's): dims D / 4 * grp ..
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) {
      u32x4 x = {0u, 0u, 0u, 0u};
      if (h < g) x = ld16(a.q + (row0 + h) * D + grp * (D / 4) + kk * 8);
      qf[kk] = as_bf16x8(x);
    }
    f32x4 acc[DB];
    float m, l;
    quant_range<D, BITS, kWays>(a, qf, a.tables + (size_t)seq * a.max_blocks, kvh, s0, s1, acc, m, l, smem.ring[wave]);
    if constexpr (Ring<D, BITS>::kUsed) __syncthreads();  // (the results take the ring's space)
    if (h < g) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
        if (db % kWays == way)
          st16(&sm.o[wave][h][db * 16 + 4 * grp], __builtin_bit_cast(u32x4, acc[db]));
      if (lane < 16 / kWays) {
        sm.m[wave][h] = m;
        sm.l[wave][h] = l;
      }
    }
  } else if constexpr (Ring<D, BITS>::kUsed) {
    __syncthreads();
  }
  if (s0 >= s1 && lane < g) {
    sm.m[wave][lane] = -INFINITY;
    sm.l[wave][lane] = 0.f;
  }
  __syncthreads();
  const int used = (k1 - k0 + share - 1) / share;  // shares that have keys
  for (int u = threadIdx.x; u < g * (D / 4); u += 64 * kParts) {  // one thread per (head, 4 dims)
    const int hh = u / (D / 4), d = (u % (D / 4)) * 4;
    float mx = -INFINITY;
#pragma unroll
    for (int s = 0; s < kParts; ++s) mx = fmaxf(mx, sm.m[s][hh]);
    float den = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < kParts; ++s) {
      if (s >= used) break;
      const float w = fast_exp2(sm.m[s][hh] - finite_max(mx));
      den += w * sm.l[s][hh];
      const f32x4 x = __builtin_bit_cast(f32x4, ld16(&sm.o[s][hh][d]));
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += w * x[e];
    }
    const size_t row = row0 + hh;
    if (a.splits == 1 || len <= a.split_keys) {
      const float inv = 1.f / den;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = den == 0.f ? 0.f : o[e] * inv;
      st8(a.out + row * D + d, u32x2{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])});
      if (a.lse != nullptr && d == 0) a.lse[row] = (mx + log2f(den)) * kLn2;
    } else {
      const size_t slot = row * a.splits + split;
      st16(a.ws_o + slot * D + d, __builtin_bit_cast(u32x4, o));
      if (d == 0) {
        a.ws_ml[slot * 2] = mx;
        a.ws_ml[slot * 2 + 1] = den;
      }
    }
  }
}

// The splits' partial results of a (sequence, query head) by their log-sum-exp weights, on one wave, or on
// kMergeWaves that take the splits in runs and meet in LDS.
template <int D, bool kWide>
__global__ __launch_bounds__(64 * kMergeWaves) void quant_merge_kernel(const QuantDecodeArgs a) {
  constexpr int PER = D / 64, kRounds = kMaxSplits / 64;
  __shared__ float sum[kMergeWaves][D];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int64_t item = kWide ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * kMergeWaves + wave;
  if (item >= (int64_t)a.num_seqs * a.hq) return;
  const int len = min(a.seq_lens[item / a.hq], a.max_len);
  const int n = (len + a.split_keys - 1) / a.split_keys;
  if (n <= 1) return;  // (written already)
  const float* ml = a.ws_ml + (size_t)item * a.splits * 2;
  const float* src = a.ws_o + (size_t)item * a.splits * D + lane * PER;
  float m[kRounds], w[kRounds], top = -INFINITY, den = 0.f;  // lane l: splits l, 64 + l, ..
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int s = 64 * r + lane;
    m[r] = s < n ? ml[s * 2] : -INFINITY;
    w[r] = s < n ? ml[s * 2 + 1] : 0.f;
    top = fmaxf(top, m[r]);
  }
  top = wave_all(top, Max());
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const float x = fast_exp2(m[r] - finite_max(top));
    den += x * w[r];
    w[r] = x;
  }
  den = wave_all(den, Add());
  float o[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) o[e] = 0.f;
  const int run = kWide ? ((n + kMergeWaves - 1) / kMergeWaves + 7) / 8 * 8 : kMaxSplits;
  const int s0 = kWide ? wave * run : 0, s1 = min(n, s0 + run);
#pragma unroll
  for (int r = 0; r < kRounds; ++r)
    for (int s = max(s0, 64 * r); s < min(s1, 64 * (r + 1)); s += 8)
      add_partials<D>(src + (size_t)64 * r * D, w[r], s - 64 * r, min(s1, 64 * (r + 1)) - 64 * r, o);
  if constexpr (kWide) {
#pragma unroll
    for (int e = 0; e < PER; ++e) sum[wave][lane * PER + e] = o[e];
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      o[e] = 0.f;
#pragma unroll
      for (int k = 0; k < kMergeWaves; ++k) o[e] += sum[k][lane * PER + e];
    }
  }
  const float inv = 1.f / den;
#pragma unroll
  for (int e = 0; e < PER; ++e) o[e] = den == 0.f ? 0.f : o[e] * inv;
  uint16_t* dst = a.out + (size_t)item * D + lane * PER;
  if constexpr (PER == 2) {
    *reinterpret_cast<uint32_t*>(dst) = pack_bf16x2(o[0], o[1]);
  } else {
    dst[0] = (uint16_t)(pack_bf16x2(o[0], 0.f) & 0xFFFFu);
  }
  if (a.lse != nullptr && lane == 0) a.lse[item] = (top + log2f(den)) * kLn2;
}

// How a call is cut: host arithmetic on its sizes alone. Measured with 128 dims and 4 bits (8 bits alike), groups
// = sequences x kv heads, lengths spread evenly, us:
struct QuantCut {
  int parts;       // waves per (sequence, kv head, split)
  int splits;      // of the longest sequence
  int split_keys;  // (a multiple of 64)
};
QuantCut quant_cut(int32_t num_seqs, int32_t hkv, int32_t max_len) {
  const int64_t groups = (int64_t)num_seqs * hkv;
  QuantCut c{4, 1, max_len};
  int64_t keys = max_len;
  if (max_len <= 2048) {
    // One launch. Four waves share an item; one wave takes it where short items fill the chip
    // (4096 groups of 10-100 keys 15.6 against 23.2, of 1-300 26.9 and 33.2, of 100-600 51.2 and 51.3), and
    // eight where there are few and each is worth it (128 of 300-1000 keys 8.8 against 10.4, 256 of 700-2000
    // 14.3 and 17.0; but 512 of 50-300 10.7 and 8.7, 512 of 700-2000 27.8 and 24.7).
    if (groups >= 2048 && max_len <= 512) c.parts = 1;
    else if (groups <= 384 && max_len > 512) c.parts = 8;
  } else if (max_len > 8192) {
    // Splits even out long sequences and fill the chip, and each costs a partial result: with 2^23 keys and more
    // of 4096 (512 groups of 8192-32768 270 against 277 with 2048 and 289 with 1024, 160 of 8000-64000 150, 151
    // and 155), below that of 2048 (64 of 8192-65536 67 against 72 with 4096, 384 of 500-16000 89, 91 and 91.5
    // with 1024), of 512 and more where items are fewer than two a compute unit (8 of 8000-32000 13.6 against
    // 19.3 with 2048, 8 of 131072 31.1 with 2048 against 36.4).
    keys = std::min<int64_t>(std::max<int64_t>(groups * max_len / 512, 512), groups * max_len >= 1 << 23 ? 4096 : 2048);
  } else if (groups < 1024) {
    // (8 groups of 2000-8000 keys 10.8 with 512 against 17.4 with 2048 and 31 unsplit, 64 16.7 with 1024
    // against 20.1 and 51.7, 192 of 500-8000 35.2, 36.0 and 67.7, 512 84.6, 87.0 and 83.4; 2048 unsplit 267
    // against 276)
    keys = std::min<int64_t>(std::max<int64_t>(groups * max_len / 512, 512), 1024);
  }
  keys = std::max<int64_t>(keys, ((int64_t)max_len + kMaxSplits - 1) / kMaxSplits);
  if (groups >= (1 << 16)) keys = max_len;  // (items enough, and a grid holds no more)
  c.split_keys = (int)std::min<int64_t>((keys + 255) / 256 * 256, INT32_MAX - 255);
  c.splits = (int)(((int64_t)max_len + c.split_keys - 1) / c.split_keys);
  return c;
}

template <int D, int BITS, int kWays>
hipError_t launch_cut(const QuantDecodeArgs& a, const QuantCut& c, hipStream_t stream) {
  const int64_t items = (int64_t)a.num_seqs * a.hkv * c.splits;
  if (items * 64 * c.parts > UINT32_MAX) return hipErrorInvalidValue;
  auto* kern = c.parts == 1   ? quant_decode_kernel<D, BITS, kWays, 1>
               : c.parts == 4 ? quant_decode_kernel<D, BITS, kWays, 4>
                              : quant_decode_kernel<D, BITS, kWays, 8>;
  hipLaunchKernelGGL(kern, dim3((unsigned)items), dim3(64 * c.parts), 0, stream, a);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess || c.splits == 1) return err;
  const int64_t rows = (int64_t)a.num_seqs * a.hq;
  const bool wide = c.splits > 16;
  hipLaunchKernelGGL((wide ? quant_merge_kernel<D, true> : quant_merge_kernel<D, false>),
                     dim3((unsigned)(wide ? rows : (rows + kMergeWaves - 1) / kMergeWaves)),
                     dim3(64 * kMergeWaves), 0, stream, a);
  return hipGetLastError();
}

template <int D, int BITS>
hipError_t launch_ways(const QuantDecodeArgs& a, const QuantCut& c, hipStream_t stream) {
  const int g = a.hq / a.hkv;
  return g <= 4   ? launch_cut<D, BITS, 4>(a, c, stream)
         : g <= 8 ? launch_cut<D, BITS, 2>(a, c, stream)
                  : launch_cut<D, BITS, 1>(a, c, stream);
}

}  // namespace

size_t quant_decode_workspace_bytes(int32_t num_seqs, int32_t hq, int32_t hkv, int32_t head_dim,
                                    int32_t bits, int32_t max_len) {
  const QuantCut c = quant_cut(num_seqs, hkv, max_len);
  if (c.splits == 1) return 0;
  return (size_t)num_seqs * hq * c.splits * (head_dim + 2) * sizeof(float);
}

hipError_t launch_quant_decode(QuantDecodeArgs a, int head_dim, int bits, void* workspace,
                               hipStream_t stream) {
  const QuantCut c = quant_cut(a.num_seqs, a.hkv, a.max_len);
  a.split_keys = c.split_keys;
  a.splits = c.splits;
  a.ws_o = static_cast<float*>(workspace);
  a.ws_ml = a.ws_o + (size_t)a.num_seqs * a.hq * c.splits * head_dim;
  if (head_dim == 128)
    return bits == 8 ? launch_ways<128, 8>(a, c, stream) : launch_ways<128, 4>(a, c, stream);
  return bits == 8 ? launch_ways<64, 8>(a, c, stream) : launch_ways<64, 4>(a, c, stream);
}

}  // namespace pkv
