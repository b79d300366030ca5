// Rotary positions with several axes, fused with the append to the paged cache (gfx950).
//
// Pair j of a head's first rot_dim dims, (x_a, x_b), is turned by the angle
//   phi_j = positions[axis_of[j]][t] * inv_freq[j]:
//   y_a = x_a cos phi_j - x_b sin phi_j,   y_b = x_b cos phi_j + x_a sin phi_j,
// with (a, b) = (j, j + rot_dim / 2), or (2j, 2j + 1) where interleaved. Queries go to q_out, keys
// to their slot of the pool's chunk-major slab, values unturned to the dim-major slab.
//
// Angles are counted in turns: positions * (inv_freq / 2 pi) in 64 bits, less its nearest whole
// number, so a far position loses nothing (in 32 bits position 10^6 is off by 0.03 rad). Sine and
// cosine are then taken in 32 bits, the products and sums too, and each output is rounded once.
// They are found once per (row, pair) of a workgroup and serve all its heads.
//
// Bound by memory (every row read once and written once); a workgroup takes a window of
// consecutive rows and some of the heads. V's slab holds 8 tokens of one dim in 16 bytes, so a
// run of rows that fills a half-slab is written whole by the workgroup in whose window it begins
// (it looks up to 7 rows past the window's end); rows of a half-slab only partly covered are
// written in 2-byte pieces, which need no read and cannot race with another workgroup's.
#include "device_utils.h"
#include "launch.h"

namespace pkv {
namespace {

constexpr int kThreads = 256;
constexpr int kWindow = 16;  // most rows of a window
constexpr int kAhead = 7;    // rows past it that a run begun in it can reach

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Eight pairs whose first dims are in x and second dims in y: cs points at pair 0's (cos, sin).
__device__ __forceinline__ void turn_halves(u32x4& x, u32x4& y, const float2* cs) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 c0 = cs[2 * e], c1 = cs[2 * e + 1];
    const float a0 = lo_f(x[e]), a1 = hi_f(x[e]), b0 = lo_f(y[e]), b1 = hi_f(y[e]);
    x[e] = pack_bf16x2(a0 * c0.x - b0 * c0.y, a1 * c1.x - b1 * c1.y);
    y[e] = pack_bf16x2(b0 * c0.x + a0 * c0.y, b1 * c1.x + a1 * c1.y);
  }
}
// Four pairs of neighbours.
__device__ __forceinline__ void turn_neighbours(u32x4& x, const float2* cs) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 c = cs[e];
    const float a = lo_f(x[e]), b = hi_f(x[e]);
    x[e] = pack_bf16x2(a * c.x - b * c.y, b * c.x + a * c.y);
  }
}

template <int D>
__global__ __launch_bounds__(kThreads) void rope_append_kernel(const RopeArgs a) {
  constexpr int NCH = D / 8;
  constexpr int SLAB = D * kBlockSize;
  constexpr int ROW = D + 8;
  __shared__ float2 cs[kWindow][D / 2];
  __shared__ int64_t slots[kWindow + kAhead + 1];  // of rows t0 - 1 ..
  __shared__ __align__(16) uint16_t tile[(kWindow + kAhead) * ROW];
  __shared__ int runs[kWindow][2];  // first row within the window, length
  __shared__ int num_runs;

  const int t = threadIdx.x;
  const int64_t t0 = (int64_t)blockIdx.x * a.window;
  const int n = (int)min((int64_t)a.window, a.rows - t0);        // the window's rows
  const int staged = (int)min((int64_t)n + kAhead, a.rows - t0);  // with those a run can reach
  const int64_t num_slots = (int64_t)a.num_blocks * kBlockSize;
  if (t <= staged) {
    const int64_t r = t0 + t - 1;
    const int64_t s = r >= 0 ? a.slot_map[r] : -1;
    slots[t] = s >= 0 && s < num_slots ? s : -1;
  }
  const int half = a.rot_dim / 2;
  for (int u = t; u < n * half; u += kThreads) {
    const int r = u / half, j = u % half;
    const double turns = (double)a.positions[(int64_t)a.axis_of[j] * a.pos_stride + t0 + r] *
                         a.turns[j];
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    cs[r][j] = make_float2(c * a.scale, s * a.scale);
  }
  __syncthreads();
  if (t < 64) {  // the runs that begin in the window
    bool starts = false;
    int len = 1;
    if (t < n) {
      const int64_t s = slots[t + 1];
      starts = s >= 0 && !((s & 7) != 0 && slots[t] == s - 1);
      while (len < 8 && t + len < staged && ((s + len) & 7) != 0 && slots[t + 1 + len] == s + len)
        ++len;
    }
    const uint64_t m = __builtin_amdgcn_ballot_w64(starts);
    if (starts) {
      const int k = __builtin_popcountll(m & ((1ull << t) - 1));
      runs[k][0] = t;
      runs[k][1] = len;
    }
    if (t == 0) num_runs = __builtin_popcountll(m);
  }
  // Units of a head's row: the turned ones (two chunks of 8 dims, or one where neighbours pair),
  // then the chunks past rot_dim.
  const int turned = a.interleaved ? a.rot_dim / 8 : a.rot_dim / 16;
  const int units = turned + (D - a.rot_dim) / 8;
  // loads one unit's one or two chunks, turns them, and tells which chunks they are
  auto unit = [&](const uint16_t* row, int r, int u, u32x4& x, u32x4& y, int& cx, int& cy) {
    cy = -1;
    if (u >= turned) {
      cx = a.rot_dim / 8 + (u - turned);
      x = ld16(row + cx * 8);
    } else if (a.interleaved) {
      cx = u;
      x = ld16(row + cx * 8);
      turn_neighbours(x, &cs[r][cx * 4]);
    } else {
      cx = u;
      cy = u + turned;
      x = ld16(row + cx * 8);
      y = ld16(row + cy * 8);
      turn_halves(x, y, &cs[r][cx * 8]);
    }
  };

  const int g = a.hq / a.hkv;
  for (int h = blockIdx.y; h < a.hkv; h += gridDim.y) {
    // queries of the group: consecutive threads take consecutive chunks of a row
    for (int w = t; w < n * g * units; w += kThreads) {
      const int u = w % units, rest = w / units;
      const int qh = h * g + rest % g, r = rest / g;
      if (slots[r + 1] < 0) continue;
      u32x4 x, y;
      int cx, cy;
      unit(a.q + (t0 + r) * a.q_stride + (int64_t)qh * D, r, u, x, y, cx, cy);
      uint16_t* dst = a.q_out + (t0 + r) * a.q_out_stride + (int64_t)qh * D;
      st16(dst + cx * 8, x);
      if (cy >= 0) st16(dst + cy * 8, y);
    }
    // keys: consecutive threads take the same chunk of consecutive rows (16 bytes of
    // consecutive slots are contiguous)
    for (int w = t; w < n * units; w += kThreads) {
      const int r = w % n, u = w / n;
      const int64_t s = slots[r + 1];
      if (s < 0) continue;
      u32x4 x, y;
      int cx, cy;
      unit(a.k + (t0 + r) * a.k_stride + (int64_t)h * D, r, u, x, y, cx, cy);
      uint16_t* slab = a.k_cache + ((s >> 4) * a.hkv + h) * SLAB + (s & 15) * 8;
      st16(slab + (size_t)cx * kBlockSize * 8, x);
      if (cy >= 0) st16(slab + (size_t)cy * kBlockSize * 8, y);
    }
    // values: the rows staged, then column by column
    __syncthreads();  // (the tile's readers of the previous head, and the runs)
    for (int w = t; w < staged * NCH; w += kThreads) {
      const int r = w / NCH, c = w % NCH;
      if (slots[r + 1] >= 0)
        st16(&tile[r * ROW + c * 8], ld16(a.v + (t0 + r) * a.v_stride + (int64_t)h * D + c * 8));
    }
    __syncthreads();
    for (int w = t; w < num_runs * D; w += kThreads) {
      const int k = w % num_runs, d = w / num_runs;
      const int r = runs[k][0], len = runs[k][1];
      const int64_t s = slots[r + 1];
      uint16_t* dst = a.v_cache + ((s >> 4) * a.hkv + h) * SLAB + (size_t)d * kBlockSize + (s & 15);
      if (len == 8) {
        uint16_t vals[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) vals[e] = tile[(r + e) * ROW + d];
        u32x4 packed;
        __builtin_memcpy(&packed, vals, 16);
        st16(dst, packed);
      } else {
        for (int e = 0; e < len; ++e) dst[e] = tile[(r + e) * ROW + d];
      }
    }
  }
}

}  // namespace

hipError_t launch_rope_append(RopeArgs a, int head_dim, hipStream_t stream) {
  a.window = kWindow;
  const int64_t windows = (a.rows + a.window - 1) / a.window;
  if (windows > (1 << 24)) return hipErrorInvalidValue;  // (2^32 threads of a grid)
  const dim3 grid((unsigned)windows, (unsigned)std::min(a.hkv, 8));
  if (head_dim == 128)
    hipLaunchKernelGGL(rope_append_kernel<128>, grid, dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(rope_append_kernel<64>, grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace pkv
