// Key bounds per block (gfx950): for every block that holds new tokens, and every kv head, the
// largest and the smallest value of each dim over the block's keys,
//   bounds[block][h][0][d] = max_s K[s][d],   bounds[block][h][1][d] = min_s K[s][d],
// s over the block's filled slots (older tokens included; the tail slots may hold any bits). A
// NaN among them makes both NaN. A max picks a key's own bits, so nothing is rounded.
//
// Bound by reading the keys (a block's slab for one head is 256 D bits read, 32 D written): a
// wave takes one slab, lane (slot, chunk group) loads 16 bytes of a slot, and the 16 slots meet
// in lane shuffles.
#include "device_utils.h"
#include "launch.h"

namespace pkv {
namespace {

constexpr int kWaves = 4;

template <int D>
__global__ __launch_bounds__(64 * kWaves) void block_bounds_kernel(
    const uint16_t* __restrict__ k_cache, uint16_t* __restrict__ bounds,
    const int32_t* __restrict__ block_tables, int32_t max_blocks,
    const int32_t* __restrict__ cached_lens, const int32_t* __restrict__ cu_new_lens,
    int32_t hkv, int32_t num_blocks) {
  constexpr int SLAB = D * kBlockSize;
  const int i = blockIdx.z;
  const int h = blockIdx.y * kWaves + (threadIdx.x >> 6);
  if (h >= hkv) return;
  const int lane = threadIdx.x & 63, slot = lane & 15, grp = lane >> 4;
  const int p = cached_lens[i];
  const int n = cu_new_lens[i + 1] - cu_new_lens[i];
  if (n <= 0 || p < 0) return;
  const int64_t len = (int64_t)p + n;
  const int64_t b = p / kBlockSize + (int64_t)blockIdx.x;
  if (b * kBlockSize >= len || b >= max_blocks) return;
  const int blk = block_tables[(size_t)i * max_blocks + b];
  if (blk < 0 || blk >= num_blocks) return;
  const int filled = (int)min(len - b * kBlockSize, (int64_t)kBlockSize);
  const uint16_t* slab = k_cache + ((size_t)blk * hkv + h) * SLAB;
  uint16_t* out = bounds + ((size_t)blk * hkv + h) * 2 * D;
#pragma unroll
  for (int kk = 0; kk < D / 32; ++kk) {
    const int c = kk * 4 + grp;
    u32x4 v = ld16(slab + (size_t)(c * kBlockSize + min(slot, filled - 1)) * 8);
    float hi[8], lo[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = __uint_as_float(e & 1 ? v[e / 2] & 0xFFFF0000u : v[e / 2] << 16);
      hi[e] = lo[e] = x;
    }
#pragma unroll
    for (int o = 8; o >= 1; o >>= 1) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = __shfl_xor(hi[e], o), y = __shfl_xor(lo[e], o);
        hi[e] = x > hi[e] || x != x ? x : hi[e];  // (a NaN wins and stays)
        lo[e] = y < lo[e] || y != y ? y : lo[e];
      }
    }
    if (slot < 2) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = slot == 0 ? hi[2 * e] : lo[2 * e];
        const float y = slot == 0 ? hi[2 * e + 1] : lo[2 * e + 1];
        w[e] = (__float_as_uint(x) >> 16) | (__float_as_uint(y) & 0xFFFF0000u);
      }
      st16(out + slot * D + c * 8, w);
    }
  }
}

}  // namespace

hipError_t launch_block_bounds(const KvView& kv, uint16_t* bounds, const int32_t* block_tables,
                               int32_t max_blocks, const int32_t* cached_lens,
                               const int32_t* cu_new_lens, int32_t num_seqs, int32_t max_new_len,
                               hipStream_t stream) {
  const dim3 grid((unsigned)((max_new_len + kBlockSize - 1) / kBlockSize + 1),
                  (unsigned)((kv.hkv + kWaves - 1) / kWaves), (unsigned)num_seqs);
  auto* kern = kv.head_dim == 128 ? block_bounds_kernel<128> : block_bounds_kernel<64>;
  hipLaunchKernelGGL(kern, grid, dim3(64 * kWaves), 0, stream, kv.k, bounds, block_tables,
                     max_blocks, cached_lens, cu_new_lens, kv.hkv, kv.num_blocks);
  return hipGetLastError();
}

}  // namespace pkv
