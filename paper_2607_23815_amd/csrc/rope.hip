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
// Bound by memory (every row read once and written once). A workgroup takes a window of consecutive rows
// and a kv head with its query heads at a time; its first kBatch * kThreads units' loads go out at once,
// before the angles are found. These are all of a window's with halves of 128 dims and up to 5 query heads
// a kv head, which then waits once and not once per part; more heads, and neighbours and partial rotation
// from 3 on (twice the units), load the others behind the first ones' stores. V's slab holds 8
// tokens of one dim in 16 bytes, so a run of rows that fills a half-slab is written whole by the
// workgroup in whose window it begins (it looks up to 7 rows past the window's end); rows of a
// half-slab only partly covered are written in 2-byte pieces, which need no read and cannot race
// with another workgroup's. 16-byte stores go past the caches, and a window's heads are neighbouring
// workgroups, so that its rows are read whole at about the same time. 16k rows of 32/8 heads of 128 dims:
// 86.8 us, 4.5 TB/s; 64/8 heads 133.0 us, 5.0 TB/s, the rate of a large copy (windows side by side instead
// of heads 104.6 and 173.6, then with ordinary stores 108.9 and 175.3). Neighbours 97.4 and 149.6; the
// first 64 dims turned 103.8 and 164.6.
#include "device_utils.h"
#include "launch.h"

namespace pkv {
namespace {

constexpr int kThreads = 256;
constexpr int kWindow = 16;  // rows of a window at most
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

// How a head's dims pair up: all of them with the one half a head away; neighbours; the first
// rot_dim with the one half of rot_dim away.
enum : int { kHalves = 0, kNeighbours = 1, kPartial = 2 };

template <int D, int kStyle>
__global__ __launch_bounds__(kThreads) void rope_append_kernel(const RopeArgs a) {
  constexpr int NCH = D / 8;
  constexpr int SLAB = D * kBlockSize;
  constexpr int ROW = D + 8;
  // A unit is one thread's part of a head's row: two chunks of 8 dims that pair up, or one chunk.
  constexpr int kUnits = kStyle == kHalves ? D / 16 : D / 8;
  constexpr int kBatch = 3;  // units of a thread at a time (4 query heads and the key head of 16 rows)
  constexpr int kStage = ((kWindow + kAhead) * NCH + kThreads - 1) / kThreads;
  __shared__ __align__(16) float2 cs[kWindow][D / 2 + 2];
  __shared__ int64_t slots[kWindow + kAhead];
  __shared__ __align__(16) uint16_t tile[(kWindow + kAhead) * ROW];
  __shared__ int runs[kWindow][2];  // first row within the window, length
  __shared__ int num_runs;

  const int t = threadIdx.x;
  const int64_t t0 = (int64_t)(blockIdx.x / a.hkv) << a.window;
  const int n = (int)min((int64_t)1 << a.window, a.rows - t0);    // the window's rows
  const int staged = (int)min((int64_t)n + kAhead, a.rows - t0);  // with those a run can reach
  const int g = a.hq / a.hkv;
  const int half = a.rot_dim / 2;
  const int turned = kStyle == kHalves ? kUnits : kStyle == kNeighbours ? a.rot_dim / 8 : a.rot_dim / 16;
  const int units = kStyle == kPartial ? turned + (D - a.rot_dim) / 8 : kUnits;

  // unit w of a kv head's units: of query head g' < g of the group, or of the key head (g' == g)
  struct Unit {
    int u, r, head;
    bool live;
  };
  auto unit_at = [&](int w) {
    Unit x;
    x.u = w % kUnits;
    x.r = w / kUnits & ((1 << a.window) - 1);
    x.head = w / kUnits >> a.window;
    x.live = x.r < n && x.head <= g && (kStyle != kPartial || x.u < units);
    return x;
  };
  // a unit's chunks (the second, or -1)
  auto first_chunk = [&](int u) { return kStyle == kPartial && u >= turned ? a.rot_dim / 8 + (u - turned) : u; };
  auto second_chunk = [&](int u) {
    return kStyle == kHalves ? u + D / 16 : kStyle == kPartial && u < turned ? u + turned : -1;
  };
  u32x4 x[kBatch], y[kBatch], v[kStage];
  auto load_units = [&](int h, int w0) {
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const Unit q = unit_at(w0 + k * kThreads + t);
      if (!q.live) continue;
      const uint16_t* row = q.head < g ? a.q + (t0 + q.r) * a.q_stride + (int64_t)(h * g + q.head) * D
                                       : a.k + (t0 + q.r) * a.k_stride + (int64_t)h * D;
      x[k] = ld16(row + first_chunk(q.u) * 8);
      const int c = second_chunk(q.u);
      if (c >= 0) y[k] = ld16(row + c * 8);
    }
  };
  auto store_units = [&](int h, int w0) {
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const Unit q = unit_at(w0 + k * kThreads + t);
      if (!q.live) continue;
      const int64_t s = slots[q.r];
      if (s < 0) continue;
      const int c0 = first_chunk(q.u), c1 = second_chunk(q.u);
      if (kStyle == kNeighbours) {
        if (q.u < turned) turn_neighbours(x[k], &cs[q.r][q.u * 4]);
      } else if (q.u < turned) {
        turn_halves(x[k], y[k], &cs[q.r][q.u * 8]);
      }
      if (q.head < g) {
        uint16_t* row = a.q_out + (t0 + q.r) * a.q_out_stride + (int64_t)(h * g + q.head) * D;
        st16_nt(row + c0 * 8, x[k]);
        if (c1 >= 0) st16_nt(row + c1 * 8, y[k]);
      } else {  // (16 bytes of consecutive slots are contiguous)
        uint16_t* slab = a.k_cache + ((s >> 4) * a.hkv + h) * SLAB + (s & 15) * 8;
        st16_nt(slab + c0 * kBlockSize * 8, x[k]);
        if (c1 >= 0) st16_nt(slab + c1 * kBlockSize * 8, y[k]);
      }
    }
  };
  auto load_v = [&](int h) {
#pragma unroll
    for (int k = 0; k < kStage; ++k) {
      const int w = k * kThreads + t;
      if (w < staged * NCH)
        v[k] = ld16(a.v + (t0 + w / NCH) * a.v_stride + (int64_t)h * D + w % NCH * 8);
    }
  };

  const int h = blockIdx.x % a.hkv;  // (the heads of a window side by side: its rows are read whole)
  load_units(h, 0);
  load_v(h);
  if (t < 64) {  // the slots, and the runs that begin in the window
    const int64_t num_slots = (int64_t)a.num_blocks * kBlockSize;
    auto slot_at = [&](int64_t r) {
      const int64_t s = a.slot_map[r];
      return s < num_slots ? s : -1;
    };
    const int64_t s = t < staged ? slot_at(t0 + t) : -1;
    int64_t prev = __shfl_up(s, 1);
    if (t == 0) prev = t0 > 0 ? slot_at(t0 - 1) : -1;
    if (t < staged) slots[t] = s;
    // a row goes on with the run before it within a half-slab
    const bool on = s >= 0 && (s & 7) != 0 && prev == s - 1;
    const uint64_t ons = __builtin_amdgcn_ballot_w64(on);
    const bool starts = t < n && s >= 0 && !on;
    const uint64_t m = __builtin_amdgcn_ballot_w64(starts);
    if (starts) {
      const int k = __builtin_popcountll(m & ((1ull << t) - 1));
      runs[k][0] = t;
      runs[k][1] = 1 + __builtin_ctzll(~(ons >> (t + 1)));
    }
    if (t == 0) num_runs = __builtin_popcountll(m);
  }
  for (int w = t; w < n * half; w += kThreads) {
    const int r = w / half, j = w - r * half;
    const double turns = (double)a.positions[(int64_t)a.axis_of[j] * a.pos_stride + t0 + r] *
                         a.turns[j];
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    cs[r][j] = make_float2(c * a.scale, s * a.scale);
  }
  const int all = (g + 1) * kUnits << a.window;
#pragma unroll
  for (int k = 0; k < kStage; ++k) {
    const int w = k * kThreads + t;
    if (w < staged * NCH) st16(&tile[w / NCH * ROW + w % NCH * 8], v[k]);
  }
  __syncthreads();
  store_units(h, 0);
  for (int w0 = kBatch * kThreads; w0 < all; w0 += kBatch * kThreads) {
    load_units(h, w0);
    store_units(h, w0);
  }
  // values column by column, neighbouring threads at the runs of one dim
  for (int w = t; w < num_runs * D; w += kThreads) {
    const int d = w / num_runs, k = w - d * num_runs;
    const int r = runs[k][0], len = runs[k][1];
    const int64_t s = slots[r];
    uint16_t* dst = a.v_cache + ((s >> 4) * a.hkv + h) * SLAB + d * kBlockSize + (s & 15);
    if (len == 8) {
      uint16_t vals[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) vals[e] = tile[(r + e) * ROW + d];
      u32x4 packed;
      __builtin_memcpy(&packed, vals, 16);
      st16_nt(dst, packed);
    } else {
      for (int e = 0; e < len; ++e) dst[e] = tile[(r + e) * ROW + d];
    }
  }
}

template <int D>
hipError_t launch_style(const RopeArgs& a, dim3 grid, hipStream_t stream) {
  auto* kern = a.interleaved    ? rope_append_kernel<D, kNeighbours>
               : a.rot_dim == D ? rope_append_kernel<D, kHalves>
                                : rope_append_kernel<D, kPartial>;
  hipLaunchKernelGGL(kern, grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope_append(RopeArgs a, int head_dim, hipStream_t stream) {
  // Windows of 16 rows where there are rows enough, smaller ones where a launch would have fewer than 384
  // workgroups (8 kv heads, us at 1, 2, 4, 8, 16 rows: 48 rows of a decode step 5.3, 5.5, 5.5, 6.6, 9.1; 256
  // 10.3, 7.6, 7.5, 8.4, 10.8; 100 rows of a prompt 5.2, 4.8, 4.6, 5.1, 6.1; 1344 32.1, 19.3, 13.0, 11.4, 9.4).
  a.window = 4;
  while (a.window > 0 && (((a.rows - 1) >> a.window) + 1) * a.hkv < 384) --a.window;
  const dim3 grid((unsigned)((((a.rows - 1) >> a.window) + 1) * a.hkv));
  return head_dim == 128 ? launch_style<128>(a, grid, stream) : launch_style<64>(a, grid, stream);
}

}  // namespace pkv
