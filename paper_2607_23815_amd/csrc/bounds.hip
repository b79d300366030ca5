// Key bounds per block (gfx950): for every block that holds new tokens, and every kv head, the
// largest and the smallest value of each dim over the block's keys,
//   bounds[block][h][0][d] = max_s K[s][d],   bounds[block][h][1][d] = min_s K[s][d],
// s over the block's filled slots (older tokens included; the tail slots may hold any bits). A
// NaN among them makes both NaN. A max picks a key's own bits, so nothing is rounded.
//
// Bound by reading the keys (a slab, one block of one head, is 256 D bits read and 32 D written),
// if the arithmetic stays small beside it: two dims at a time as 16-bit integers in the values'
// order, and the 16 slots, which lie in 16 lanes, meet in four steps that halve what a lane holds
// (a lane keeps one half of its dims, its partner the other), 22 lane exchanges for a slab of 128
// dims where reducing every word in every lane takes 128. A workgroup takes a block with all its
// heads (with fewer than four heads, blocks enough for four waves), and a wave has its next slab's
// loads in flight while it reduces one. 64 documents of 1024-16384 tokens, 8 heads of 128 dims: 234 us,
// 5.5 TB/s (with ordinary loads 266, then with 4 blocks per workgroup 269, with 16 292; 2 documents 8.3, 10.7 and 26.0; but 64 with
// one head 32.5 a block at a time, 25.5 by four).
#include "device_utils.h"
#include "launch.h"
#include "wave_utils.h"

namespace pkv {
namespace {

constexpr int kWaves = 4;

typedef __attribute__((ext_vector_type(2))) int16_t s16x2;

// bf16 bits to integers in the values' order, and back (its own inverse): -NaN below -inf below ..
// -0 below +0 .. below +inf below NaN.
__device__ __forceinline__ uint32_t ordered(uint32_t w) {
  const s16x2 v = __builtin_bit_cast(s16x2, w);
  return w ^ (__builtin_bit_cast(uint32_t, (s16x2)(v >> 15)) & 0x7FFF7FFFu);
}
__device__ __forceinline__ uint32_t pk_max(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(s16x2, a),
                                                                __builtin_bit_cast(s16x2, b)));
}
__device__ __forceinline__ uint32_t pk_min(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(s16x2, a),
                                                                __builtin_bit_cast(s16x2, b)));
}
// Lanes pair up (kCtrl); the one with `upper` set goes on with the upper half of the n words, the
// other with the lower half, each of both lanes' values.
template <int kCtrl, int n>
__device__ __forceinline__ void halve(bool upper, uint32_t* hi, uint32_t* lo) {
#pragma unroll
  for (int k = 0; k < n / 2; ++k) {
    const uint32_t keep_hi = upper ? hi[k + n / 2] : hi[k], give_hi = upper ? hi[k] : hi[k + n / 2];
    const uint32_t keep_lo = upper ? lo[k + n / 2] : lo[k], give_lo = upper ? lo[k] : lo[k + n / 2];
    hi[k] = pk_max(keep_hi, dpp<kCtrl>(give_hi));
    lo[k] = pk_min(keep_lo, dpp<kCtrl>(give_lo));
  }
}
constexpr int kMirror16 = 0x140, kMirror8 = 0x141, kMirror4 = 0x1B, kSwap2 = 0xB1;

template <int D>
struct Slab {
  u32x4 v[D / 32];  // chunk 4 kk + grp of the lane's slot
};

template <int D>
__device__ __forceinline__ void reduce_slab(const Slab<D>& s, uint16_t* out) {
  constexpr int N = D / 8;  // words of the lane: D / 32 chunks of 4
  const int lane = threadIdx.x & 63, slot = lane & 15, grp = lane >> 4;
  uint32_t hi[N], lo[N];
#pragma unroll
  for (int k = 0; k < N; ++k) hi[k] = lo[k] = ordered(s.v[k / 4][k % 4]);
  halve<kMirror16, N>((slot & 8) != 0, hi, lo);
  halve<kMirror8, N / 2>((slot & 4) != 0, hi, lo);
  halve<kMirror4, N / 4>((slot & 2) != 0, hi, lo);
  int word;  // the word of the lane's first N that it ends with
  if constexpr (N == 16) {
    halve<kSwap2, 2>((slot & 1) != 0, hi, lo);
    word = slot;
  } else {  // one word left before the last step: both lanes keep it
    hi[0] = pk_max(hi[0], dpp<kSwap2>(hi[0]));
    lo[0] = pk_min(lo[0], dpp<kSwap2>(lo[0]));
    word = slot >> 1;
  }
  // a NaN of either sign lies past its infinity: it makes both NaN
  const s16x2 h = __builtin_bit_cast(s16x2, hi[0]), l = __builtin_bit_cast(s16x2, lo[0]);
  uint32_t top = ordered(hi[0]), low = ordered(lo[0]);
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    if (h[e] > 0x7F80 || l[e] < -0x7F81) {
      top |= 0x7FC0u << (16 * e);
      low |= 0x7FC0u << (16 * e);
    }
  }
  uint32_t* dst = reinterpret_cast<uint32_t*>(out) + ((word / 4) * 4 + grp) * 4 + word % 4;
  if (N == 16 || (slot & 1) == 0) {
    dst[0] = top;
    dst[D / 2] = low;
  }
}

template <int D, bool kOnce>
__global__ __launch_bounds__(64 * kWaves) void block_bounds_kernel(
    const uint16_t* __restrict__ k_cache, uint16_t* __restrict__ bounds,
    const int32_t* __restrict__ block_tables, int32_t max_blocks,
    const int32_t* __restrict__ cached_lens, const int32_t* __restrict__ cu_new_lens,
    int32_t hkv, int32_t num_blocks, int32_t run) {
  constexpr int SLAB = D * kBlockSize;
  const int i = blockIdx.y;
  const int p = cached_lens[i];
  const int n = cu_new_lens[i + 1] - cu_new_lens[i];
  if (n <= 0 || p < 0) return;
  const int64_t len = (int64_t)p + n;
  const int64_t first = p / kBlockSize + (int64_t)blockIdx.x * run;
  const int64_t end = min(min((len + kBlockSize - 1) / kBlockSize, (int64_t)max_blocks), first + run);
  const int lane = threadIdx.x & 63, slot = lane & 15, grp = lane >> 4;
  const int32_t* table = block_tables + (size_t)i * max_blocks;
  // the wave's slabs: (block, head) pairs wave, wave + kWaves, ..
  int64_t b = first;
  int h = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  auto settle = [&]() {
    while (h >= hkv) {
      h -= hkv;
      ++b;
    }
  };
  auto load = [&](Slab<D>& s, int64_t& at) {  // the slab (b, h); at: its bounds, or -1
    at = -1;
    if (b >= end) return;
    const int id = table[b];
    if (id < 0 || id >= num_blocks) return;
    at = ((int64_t)id * hkv + h) * 2 * D;
    const int filled = (int)min(len - b * kBlockSize, (int64_t)kBlockSize);
    const uint16_t* base = k_cache + ((size_t)id * hkv + h) * SLAB;
    const int off = (grp * kBlockSize + min(slot, filled - 1)) * 16;
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) {
      const int o = off + kk * 4 * kBlockSize * 16;
      const char* from = reinterpret_cast<const char*>(base) + o;
      s.v[kk] = kOnce ? __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(from))
                      : buf_ld16(base, SLAB * 2, o);
    }
  };
  Slab<D> s[2];
  int64_t at[2];
  settle();
  load(s[0], at[0]);
  while (b < end) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      h += kWaves;
      settle();
      load(s[1 - k], at[1 - k]);
      if (at[k] >= 0) reduce_slab<D>(s[k], bounds + at[k]);
      if (b >= end) break;
    }
  }
}

}  // namespace

hipError_t launch_block_bounds(const KvView& kv, uint16_t* bounds, const int32_t* block_tables,
                               int32_t max_blocks, const int32_t* cached_lens,
                               const int32_t* cu_new_lens, int32_t num_seqs, int32_t max_new_len,
                               hipStream_t stream) {
  // blocks that max_new_len tokens can touch, wherever the first one falls in the table
  const int64_t blocks = std::min<int64_t>(((int64_t)max_new_len + kBlockSize - 2) / kBlockSize + 1,
                                           max_blocks);
  const int run = (kWaves + kv.hkv - 1) / kv.hkv;  // (at least a slab for every wave)
  const dim3 grid((unsigned)((blocks + run - 1) / run), (unsigned)num_seqs);
  // Keys beyond what the last-level cache (256 MB) can still hold of their append are read past the
  // caches: 64 documents (1.1 GB of keys) 234 us against 266, of 64 dims 125 and 137; 8 documents (140
  // MB) the other way, 29.7 and 27.4.
  const bool once = (int64_t)num_seqs * max_new_len * kv.hkv * kv.head_dim * 2 > int64_t(256) << 20;
  auto* kern = kv.head_dim == 128
                   ? (once ? block_bounds_kernel<128, true> : block_bounds_kernel<128, false>)
                   : (once ? block_bounds_kernel<64, true> : block_bounds_kernel<64, false>);
  hipLaunchKernelGGL(kern, grid, dim3(64 * kWaves), 0, stream, kv.k, bounds, block_tables,
                     max_blocks, cached_lens, cu_new_lens, kv.hkv, kv.num_blocks, run);
  return hipGetLastError();
}

}  // namespace pkv
