// Attention over chosen blocks (gfx950): row t's g query heads of a kv head attend over the keys of
// the blocks that the row's list names for that kv head,
//   out[t][h] = sum_p softmax_p(scale <q[t][h], K[p]>) V[p],  p in the listed blocks, p < row_lens[t].
// The running maximum and weight sum of the softmax make it one pass over the keys. A wave streams
// two blocks at a time into the matrix-core operands as the decode does (scores S^T = K Q^T, values
// O^T += V^T P^T; the g heads are columns); the list takes the table's place: a wave turns 64
// entries at a time into pool offsets, those that name no visible block dropped.
#include <math.h>

#include "decode_impl.h"
#include "launch.h"

namespace pkv {
namespace {

using dec::DecodeFrag;
using dec::decode_load;
using dec::finite_max;

// One wave's share: entries [e0, e1) of a list. Leaves the unnormalised output (lane (col, grp)
// holds dims 16 db + 4 grp + 0..3 of column col), the running maximum (base 2) and the lane's part
// of the weight sum.
template <int D>
__device__ __forceinline__ void sparse_range(const SparseArgs& a, const bf16x8 (&qf)[D / 32],
                                             const int32_t* __restrict__ list,
                                             const int32_t* __restrict__ table, int kvh, int len,
                                             int e0, int e1, f32x4 (&acc)[D / 16], float& m,
                                             float& lpart) {
  constexpr int KK = D / 32, DB = D / 16, SLAB = D * kBlockSize;
  const int lane = threadIdx.x & 63;
  const int col = lane & 15, grp = lane >> 4;
  const int n = len > 0 ? min((len - 1) / kBlockSize + 1, a.max_blocks) : 0;  // the row's blocks
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  m = -INFINITY;
  lpart = 0.f;
  const size_t head_off = (size_t)kvh * SLAB;
  for (int e = e0; e < e1; e += 64) {
    // 64 entries: pool block and filled slots, the visible ones moved to the front lanes
    int b = e + lane < e1 ? list[e + lane] : -1;
    int id = b >= 0 && b < n ? table[b] : -1;
    const bool live = id >= 0 && id < a.num_blocks;
    int keys = live ? min(len - b * kBlockSize, kBlockSize) : 0;
    if (!live) id = 0;  // (a stand-in, read and masked)
    const uint64_t mask = __builtin_amdgcn_ballot_w64(live);
    const int count = __builtin_popcountll(mask);
    const uint64_t below = (1ull << lane) - 1;
    const int to = live ? __builtin_popcountll(mask & below)
                        : count + __builtin_popcountll(~mask & below);
    id = __builtin_amdgcn_ds_permute(to * 4, id);
    keys = __builtin_amdgcn_ds_permute(to * 4, keys);
    for (int s = 0; s < count; s += 2) {
      const int s1 = min(s + 1, 63);
      const int n0 = __builtin_amdgcn_readlane(keys, s);
      const int n1 = s + 1 < count ? __builtin_amdgcn_readlane(keys, s1) : 0;
      DecodeFrag<D> f;
      decode_load<D>(f, a.k_cache, a.v_cache,
                     (size_t)__builtin_amdgcn_readlane(id, s) * a.hkv * SLAB + head_off,
                     (size_t)__builtin_amdgcn_readlane(id, s1) * a.hkv * SLAB + head_off, col, grp);
      f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        s0 = mfma16(as_bf16x8(f.k[0][kk]), qf[kk], s0);
        s1v = mfma16(as_bf16x8(f.k[1][kk]), qf[kk], s1v);
      }
      float sv[8];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        sv[r] = 4 * grp + r < n0 ? s0[r] * a.scale_log2 : -INFINITY;
        sv[4 + r] = 4 * grp + r < n1 ? s1v[r] * a.scale_log2 : -INFINITY;
      }
      float mx = sv[0];
#pragma unroll
      for (int r = 1; r < 8; ++r) mx = fmaxf(mx, sv[r]);
      mx = dec::wave_max16(mx);
      const float m_new = fmaxf(m, mx);
      const float m_sub = finite_max(m_new);
      const float alpha = fast_exp2(m - m_sub);
      float pv[8], ps = 0.f;
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        pv[r] = fast_exp2(sv[r] - m_sub);
        ps += pv[r];
      }
      lpart = lpart * alpha + ps;
      m = m_new;
      const u32x4 pb = {pack_bf16x2(pv[0], pv[1]), pack_bf16x2(pv[2], pv[3]),
                        pack_bf16x2(pv[4], pv[5]), pack_bf16x2(pv[6], pv[7])};
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        u32x2 va = f.v[0][db], vb = f.v[1][db];
        if (n0 < kBlockSize) va = dec::mask_v4(va, 4 * grp, n0);
        if (n1 < kBlockSize) vb = dec::mask_v4(vb, 4 * grp, n1);
        const u32x4 vv = {va[0], va[1], vb[0], vb[1]};
        f32x4 c = acc[db];
#pragma unroll
        for (int r = 0; r < 4; ++r) c[r] *= alpha;
        acc[db] = mfma16(as_bf16x8(vv), as_bf16x8(pb), c);
      }
    }
  }
}

// One wave per (row, kv head).
template <int D>
__global__ __launch_bounds__(64) void sparse_wave_kernel(const SparseArgs a) {
  constexpr int DB = D / 16;
  const int64_t item = blockIdx.x;
  const int64_t row = item / a.hkv;
  const int kvh = (int)(item % a.hkv);
  const int seq = a.row_seq != nullptr ? a.row_seq[row] : (int)row;
  if (seq < 0 || seq >= a.num_seqs) return;  // a padding row
  const int len = max(a.row_lens[row], 0);
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const int g = a.hq / a.hkv;
  bf16x8 qf[D / 32];
  dec::decode_load_q<D>(a.q, (int)row, a.hq, g, kvh, qf);
  f32x4 acc[DB];
  float m, lpart;
  sparse_range<D>(a, qf, a.sel + item * a.blocks, a.tables + (size_t)seq * a.max_blocks, kvh, len,
                  0, a.blocks, acc, m, lpart);
  const float l = dec::wave_sum16(lpart);
  if (col >= g) return;
  const size_t o = (size_t)row * a.hq + kvh * g + col;
  // no weight (no visible key, or scores of -infinity alone): zeros, whatever the sums hold
  const float inv = 1.f / l;
  uint16_t* dst = a.out + o * D;
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    float v[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = l == 0.f ? 0.f : acc[db][r] * inv;
    st8(dst + db * 16 + 4 * grp, u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])});
  }
  if (a.lse != nullptr && grp == 0) a.lse[o] = (m + log2f(l)) * kLn2;
}

}  // namespace

size_t sparse_workspace_bytes(int64_t items, int32_t g, int32_t head_dim, int32_t blocks) {
  (void)items, (void)g, (void)head_dim, (void)blocks;
  return 0;
}

hipError_t launch_sparse_attention(SparseArgs a, int head_dim, void* workspace,
                                   hipStream_t stream) {
  (void)workspace;
  const int64_t items = a.rows * a.hkv;
  hipLaunchKernelGGL(head_dim == 128 ? sparse_wave_kernel<128> : sparse_wave_kernel<64>,
                     dim3((unsigned)items), dim3(64), 0, stream, a);
  return hipGetLastError();
}

}  // namespace pkv
