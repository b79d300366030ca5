// A cache held in 8 or 4 bits (gfx950): new tokens quantised as they are appended, blocks of the bf16 pool
// quantised, and quantised blocks read back. quant.h has the slab and its scales.
//
// All three are bound by memory: 4 D bytes of bf16 and D bits / 4 + D / 32 + 4 of codes and scales per
// token and kv head, each once. A wave takes one block of a kv head (two heads of 64 dims in the append).
// Codes of values stand for four slots side by side in a lane, so a wave's lanes are laid out as the slab
// is: in the pool's blocks a lane's loads are those of its own codes' values; rows of new tokens come
// in as rows, four tokens of the same dims a lane, and the value codes cross the lanes in LDS.
#include <algorithm>

#include "launch.h"
#include "quant.h"

namespace pkv {
namespace {

using qnt::Slab;

constexpr int kWaves = 4;  // per workgroup

// The largest of the lanes' numbers: over quads, 8, 16 lanes (all get it).
template <int kLanes>
__device__ __forceinline__ uint32_t top_lanes(uint32_t v) {
  v = max(v, dpp<0xB1>(v));
  v = max(v, dpp<0x4E>(v));
  if constexpr (kLanes >= 8) v = max(v, dpp<0x141>(v));
  if constexpr (kLanes >= 16) v = max(v, dpp<0x140>(v));
  return v;
}

__device__ __forceinline__ float low(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float high(uint32_t pair) { return __uint_as_float(pair & 0xFFFF0000u); }

// Eight bf16 of a key group as codes (one or two words).
template <int BITS>
__device__ __forceinline__ void key_codes(u32x4 x, uint32_t top, float inverse, uint32_t* w) {
  constexpr float kMost = Slab<128, BITS>::kMost;
  float y[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    y[2 * e] = qnt::clamp_code(low(x[e]) * inverse, kMost);
    y[2 * e + 1] = qnt::clamp_code(high(x[e]) * inverse, kMost);
  }
  if constexpr (BITS == 4) {
    w[0] = qnt::two_codes<4, 0>(0u, y[0], y[1]);
    w[0] = qnt::two_codes<4, 1>(w[0], y[2], y[3]);
    w[0] = qnt::two_codes<4, 2>(w[0], y[4], y[5]);
    w[0] = qnt::two_codes<4, 3>(w[0], y[6], y[7]);
  } else {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      w[e] = qnt::two_codes<8, 0>(0u, y[4 * e], y[4 * e + 1]);
      w[e] = qnt::two_codes<8, 1>(w[e], y[4 * e + 2], y[4 * e + 3]);
    }
  }
  if (!qnt::stored(top)) {
    w[0] = 0u;
    if constexpr (BITS == 8) w[1] = 0u;
  }
}

// One value of four slots as codes: 16 bits of `into` from 16 kHalf on, or a whole word.
template <int BITS, int kHalf>
__device__ __forceinline__ uint32_t value_codes(uint32_t into, const float (&x)[4],
                                                const float (&inverse)[4]) {
  float y[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) y[j] = qnt::over_scale(x[j], inverse[j]);
  if constexpr (BITS == 4) {
    into = qnt::two_codes<4, 2 * kHalf>(into, y[0], y[1]);
    return qnt::two_codes<4, 2 * kHalf + 1>(into, y[2], y[3]);
  } else {
    into = qnt::two_codes<8, 0>(into, y[0], y[1]);
    return qnt::two_codes<8, 1>(into, y[2], y[3]);
  }
}

// The bits of four slots' codes in a word (4 bits: of two dims) whose slots are in `slots`.
template <int BITS>
__device__ __forceinline__ uint32_t slot_mask(uint32_t slots) {
  uint32_t m = 0u;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (slots >> j & 1) m |= BITS == 4 ? 0x000F000Fu << 4 * j : 0xFFu << 8 * j;
  return m;
}

// ---- append ----
// Lane (q, head, c) holds chunk c (8 dims) of slots 4 q + j. Rows: 16 bytes a lane, a row's lanes side by
// side. The value codes go through LDS into the slab's order, and a quarter that the new tokens fill only
// partly is read and merged; a block belongs to one sequence and its kv head's slab to one wave, so
// nobody else writes there.
template <int D, int BITS>
__global__ __launch_bounds__(64 * kWaves) void quant_append_kernel(const QuantAppendArgs a) {
  using S = Slab<D, BITS>;
  constexpr int kChunks = D / 8, kHeads = 128 / D;
  constexpr int kRegion = S::kCodes * kHeads;  // value codes of a wave, in LDS
  __shared__ __align__(16) uint8_t lds[kWaves][kRegion];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int seq = blockIdx.y;
  const int per = (a.hkv + kWaves * kHeads - 1) / (kWaves * kHeads);  // workgroups per block
  const int head0 = ((int)(blockIdx.x % per) * kWaves + wave) * kHeads;
  if (head0 >= a.hkv) return;
  const int c = lane % kChunks, sub = lane / kChunks % kHeads, q = lane >> 4;
  const int p = a.cached_lens[seq], row0 = a.cu_new_lens[seq];
  const int64_t end = (int64_t)p + (a.cu_new_lens[seq + 1] - row0);
  const int64_t b = p / kBlockSize + (int64_t)(blockIdx.x / per);
  if (p < 0 || b * kBlockSize >= end || b >= a.max_blocks) return;
  const int id = a.tables[(size_t)seq * a.max_blocks + b];
  if (id < 0 || id >= a.num_blocks) return;
  const int head = head0 + sub;
  const bool mine = head < a.hkv;
  const int first = max((int)(p - b * kBlockSize), 0);                      // the block's new slots
  const int last = (int)min(end - b * kBlockSize, (int64_t)kBlockSize);
  uint8_t* slab = a.cache + ((size_t)id * a.hkv + head0) * S::kBytes;       // of the wave's first head
  const int64_t t0 = row0 + b * kBlockSize - p;                             // the row of slot 0

  // value codes of the quarters that are filled partly, as they are
  constexpr int kPieces = kRegion / 1024 > 0 ? (kRegion + 1023) / 1024 : 1;  // 16 bytes a lane each
  constexpr int kQuarter = 16 * (S::kLane < 16 ? S::kLane : 16);             // bytes, within a plane
  u32x4 old[kPieces];
  uint32_t slots[kPieces];
  uint8_t* piece[kPieces];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int at = i * 1024 + lane * 16;
    const int h = at / S::kCodes, off = at % S::kCodes;
    const int quarter = off / kQuarter % 4;
    uint32_t s = 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int slot = 4 * quarter + j;
      if (slot >= first && slot < last) s |= 1u << j;
    }
    slots[i] = at < kRegion && head0 + h < a.hkv ? s : 0u;
    piece[i] = slab + (size_t)h * S::kBytes + S::kValues + off;
    old[i] = u32x4{0u, 0u, 0u, 0u};
    if (slots[i] != 0u && slots[i] != 15u) old[i] = ld16(piece[i]);
  }

  // (rows that are there: wave-uniform slots, and one address a lane that steps by the rows' stride: 158 us against
  // 168 with an address a row, 32 prompts of 1024-8192 tokens, 4 bits, 8 heads of 128)
  const int row_first = (int)max((int64_t)first, min(-t0, (int64_t)kBlockSize));
  const int row_last = (int)min((int64_t)last, max(a.rows - t0, (int64_t)0));
  const uint16_t* k_row = a.k + (t0 + 4 * q) * a.k_stride + head * D + c * 8;
  const uint16_t* v_row = a.v + (t0 + 4 * q) * a.v_stride + head * D + c * 8;
  u32x4 k[4], v[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int slot = 4 * q + j;
    k[j] = v[j] = u32x4{0u, 0u, 0u, 0u};
    if (mine && slot >= row_first && slot < row_last) {
      k[j] = ld16(k_row + j * a.k_stride);
      v[j] = ld16(v_row + j * a.v_stride);
    }
  }
  uint8_t* my_slab = slab + (size_t)sub * S::kBytes;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int slot = 4 * q + j;
    uint32_t top = 0u;
#pragma unroll
    for (int e = 0; e < 4; ++e) top = qnt::top_of(k[j][e], top);
    top = top_lanes<4>(top);
    uint32_t byte;
    float inverse;
    qnt::key_scale<BITS>(top, byte, inverse);
    uint32_t w[2];
    key_codes<BITS>(k[j], top, inverse, w);
    if (mine && slot >= first && slot < last) {
      uint8_t* to = my_slab + (c * BITS / 16) * 256 + slot * 16 + c * BITS % 16;
      if constexpr (BITS == 4) *reinterpret_cast<uint32_t*>(to) = w[0];
      else st8(to, u32x2{w[0], w[1]});
      if (c % 4 == 0) my_slab[S::kKeyScales + slot * (D / 32) + c / 4] = (uint8_t)byte;
    }
  }
  float inverse[4];
  uint32_t live = 0u;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int slot = 4 * q + j;
    uint32_t top = 0u;
#pragma unroll
    for (int e = 0; e < 4; ++e) top = qnt::top_of(v[j][e], top);
    top = top_lanes<kChunks>(top);
    const float scale = qnt::value_scale<BITS>(top);
    inverse[j] = __builtin_amdgcn_rcpf(scale);
    if (qnt::stored(top)) live |= 1u << j;
    if (mine && c == 0 && slot >= first && slot < last)
      *reinterpret_cast<float*>(my_slab + S::kValueScales + 4 * slot) = scale;
  }
  const uint32_t live_mask = slot_mask<BITS>(live);
  // dim 8 c + e is dim 16 (c / 2) + (8 (c % 2) + e)
  uint8_t* region = lds[wave] + sub * S::kCodes;
  constexpr int kRun = 16 / (BITS / 2);  // entries of 16 bytes (of a lane's share of a plane)
  const int entry = c / 2;
  const int lane_bytes = S::kLane < 16 ? S::kLane : 16;
  uint8_t* to = region + entry / kRun * 1024 + (16 * q + 8 * (c & 1)) * lane_bytes +
                entry % kRun * (BITS / 2);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = e & 1 ? high(v[j][e / 2]) : low(v[j][e / 2]);
    const uint32_t w = value_codes<BITS, 0>(0u, x, inverse) & live_mask;
    if constexpr (BITS == 4) *reinterpret_cast<uint16_t*>(to + e * lane_bytes) = (uint16_t)w;
    else *reinterpret_cast<uint32_t*>(to + e * lane_bytes) = w;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    if (slots[i] == 0u) continue;
    u32x4 w = ld16(lds[wave] + i * 1024 + lane * 16);
    if (slots[i] != 15u) {
      const uint32_t m = slot_mask<BITS>(slots[i]);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = (w[e] & m) | (old[i][e] & ~m);
    }
    st16(piece[i], w);
  }
}

// ---- blocks of the bf16 pool, to and from ----
// One wave per (pair, kv head).
__device__ __forceinline__ bool block_pair(const QuantBlocksArgs& a, int src_blocks, int dst_blocks,
                                           int& src, int& dst, int& head) {
  const int64_t item = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t pair = item / a.hkv;
  if (pair >= a.num_pairs) return false;
  head = (int)(item % a.hkv);
  src = a.pairs[2 * pair];
  dst = a.pairs[2 * pair + 1];
  return src >= 0 && src < src_blocks && dst >= 0 && dst < dst_blocks;
}

template <int D, int BITS>
__global__ __launch_bounds__(64 * kWaves) void quant_blocks_kernel(const QuantBlocksArgs a) {
  using S = Slab<D, BITS>;
  int src, dst, head;
  if (!block_pair(a, a.pool_blocks, a.num_blocks, src, dst, head)) return;
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const size_t from = ((size_t)src * a.hkv + head) * (D * kBlockSize);
  uint8_t* slab = a.cache + ((size_t)dst * a.hkv + head) * S::kBytes;
  u32x4 k[D / 32];  // dims D / 4 * grp .. of slot col
  u32x2 v[D / 16];  // slots 4 grp .. of dims 16 a + col
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
    k[i] = ld16(a.k_cache + from + ((grp * (D / 32) + i) * kBlockSize + col) * 8);
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
    v[i] = ld8(a.v_cache + from + (i * 16 + col) * kBlockSize + 4 * grp);

  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
#pragma unroll
    for (int e = 0; e < 4; ++e) top = qnt::top_of(k[i][e], top);
  }
  if constexpr (D == 64) {  // a group of 32 dims is two lanes'
    const u32x2 both = with_row(top);
    top = max(both[0], both[1]);
  }
  uint32_t byte;
  float inverse;
  qnt::key_scale<BITS>(top, byte, inverse);
  uint32_t w[S::kWords];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) key_codes<BITS>(k[i], top, inverse, w + i * BITS / 4);
  constexpr int kUnits = S::kLane >= 16 ? S::kLane / 16 : 1;
  if constexpr (S::kLane == 8) {
    st8(slab + (grp / 2) * 256 + col * 16 + (grp & 1) * 8, u32x2{w[0], w[1]});
  } else {
#pragma unroll
    for (int u = 0; u < kUnits; ++u)
      st16(slab + (grp * kUnits + u) * 256 + col * 16,
           u32x4{w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]});
  }
  if (D == 128 || (grp & 1) == 0)
    slab[S::kKeyScales + col * (D / 32) + grp * D / 128] = (uint8_t)byte;

  uint32_t tops[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      tops[2 * e] = max(tops[2 * e], v[i][e] << 16 & 0x7FFF0000u);
      tops[2 * e + 1] = max(tops[2 * e + 1], v[i][e] & 0x7FFF0000u);
    }
  }
  float scale[4], over[4];
  uint32_t live = 0u;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    tops[j] = top_lanes<16>(tops[j]);
    scale[j] = qnt::value_scale<BITS>(tops[j]);
    over[j] = __builtin_amdgcn_rcpf(scale[j]);
    if (qnt::stored(tops[j])) live |= 1u << j;
  }
  if (col == 0)
    st16(slab + S::kValueScales + 16 * grp,
         u32x4{__float_as_uint(scale[0]), __float_as_uint(scale[1]), __float_as_uint(scale[2]),
               __float_as_uint(scale[3])});
  const uint32_t mask = slot_mask<BITS>(live);
#pragma unroll
  for (int i = 0; i < D / 16; i += BITS == 4 ? 2 : 1) {
    const float x[4] = {low(v[i][0]), high(v[i][0]), low(v[i][1]), high(v[i][1])};
    uint32_t c = value_codes<BITS, 0>(0u, x, over);
    if constexpr (BITS == 4) {
      const float y[4] = {low(v[i + 1][0]), high(v[i + 1][0]), low(v[i + 1][1]), high(v[i + 1][1])};
      c = value_codes<BITS, 1>(c, y, over);
    }
    w[i * BITS / 8] = c & mask;
  }
  if constexpr (S::kLane == 8) {
    st8(slab + S::kValues + lane * 8, u32x2{w[0], w[1]});
  } else {
#pragma unroll
    for (int u = 0; u < kUnits; ++u)
      st16(slab + S::kValues + u * 1024 + lane * 16,
           u32x4{w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]});
  }
}

template <int D, int BITS, int kA>
__device__ __forceinline__ void restore_values(const uint32_t* w, const u32x4 scale, uint16_t* to) {
  st8(to + kA * 16 * kBlockSize, qnt::four_scaled<BITS, kA>(w, scale));
  if constexpr (kA + 1 < D / 16) restore_values<D, BITS, kA + 1>(w, scale, to);
}

template <int D, int BITS>
__global__ __launch_bounds__(64 * kWaves) void dequant_blocks_kernel(const QuantBlocksArgs a) {
  using S = Slab<D, BITS>;
  int src, dst, head;
  if (!block_pair(a, a.num_blocks, a.pool_blocks, src, dst, head)) return;
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const uint8_t* slab = a.cache + ((size_t)src * a.hkv + head) * S::kBytes;
  const size_t to = ((size_t)dst * a.hkv + head) * (D * kBlockSize);
  uint32_t k[S::kWords], v[S::kWords];
  if constexpr (S::kLane == 8) {
    const u32x2 x = ld8(slab + (grp / 2) * 256 + col * 16 + (grp & 1) * 8);
    const u32x2 y = ld8(slab + S::kValues + lane * 8);
    k[0] = x[0], k[1] = x[1], v[0] = y[0], v[1] = y[1];
  } else {
#pragma unroll
    for (int u = 0; u < S::kLane / 16; ++u) {
      const u32x4 x = ld16(slab + (grp * (S::kLane / 16) + u) * 256 + col * 16);
      const u32x4 y = ld16(slab + S::kValues + u * 1024 + lane * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) k[4 * u + e] = x[e], v[4 * u + e] = y[e];
    }
  }
  const uint32_t byte = slab[S::kKeyScales + col * (D / 32) + grp * D / 128];
  const u32x4 scale = ld16(slab + S::kValueScales + 16 * grp);
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
    st16(a.k_cache + to + ((grp * (D / 32) + i) * kBlockSize + col) * 8,
         qnt::eight_bf16<BITS>(k + i * BITS / 4, __uint_as_float(byte << 23)));
  restore_values<D, BITS, 0>(v, scale, a.v_cache + to + col * kBlockSize + 4 * grp);
}


}  // namespace

size_t quant_slab_bytes(int32_t head_dim, int32_t bits) {
  return (size_t)4 * head_dim * bits + head_dim / 2 + 4 * kBlockSize;
}

hipError_t launch_quant_append(const QuantAppendArgs& a, int32_t num_seqs, int32_t max_new_len,
                               int head_dim, int bits, hipStream_t stream) {
  const int heads = kWaves * (128 / head_dim);
  const int64_t blocks = ((int64_t)max_new_len + 2 * kBlockSize - 2) / kBlockSize;
  const int64_t per = (a.hkv + heads - 1) / heads;
  const int64_t wgs = std::min<int64_t>(blocks, a.max_blocks) * per;
  if (wgs * 64 * kWaves > UINT32_MAX) return hipErrorInvalidValue;
  auto* kern = head_dim == 128
                   ? (bits == 8 ? quant_append_kernel<128, 8> : quant_append_kernel<128, 4>)
                   : (bits == 8 ? quant_append_kernel<64, 8> : quant_append_kernel<64, 4>);
  hipLaunchKernelGGL(kern, dim3((unsigned)wgs, (unsigned)num_seqs), dim3(64 * kWaves), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_quant_blocks(const QuantBlocksArgs& a, bool back, int head_dim, int bits,
                               hipStream_t stream) {
  const int64_t wgs = ((int64_t)a.num_pairs * a.hkv + kWaves - 1) / kWaves;
  if (wgs * 64 * kWaves > UINT32_MAX) return hipErrorInvalidValue;
  auto* kern = head_dim == 128
                   ? (bits == 8 ? (back ? dequant_blocks_kernel<128, 8> : quant_blocks_kernel<128, 8>)
                                : (back ? dequant_blocks_kernel<128, 4> : quant_blocks_kernel<128, 4>))
                   : (bits == 8 ? (back ? dequant_blocks_kernel<64, 8> : quant_blocks_kernel<64, 8>)
                                : (back ? dequant_blocks_kernel<64, 4> : quant_blocks_kernel<64, 4>));
  hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(64 * kWaves), 0, stream, a);
  return hipGetLastError();
}

}  // namespace pkv
