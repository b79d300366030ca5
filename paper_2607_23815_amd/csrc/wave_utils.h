// Exchanges between the lanes of a wave without LDS: data-parallel moves within rows of 16 lanes, and
// swaps of rows and halves. And a load of 4 bytes.
#pragma once

#include "device_utils.h"

namespace pkv {

// The value of another lane of the row of 16 (kCtrl: a DPP control).
template <int kCtrl>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, kCtrl, 0xF, 0xF, true);
}
// x and its value in the lane 16 (or 32) away, in some order.
__device__ __forceinline__ u32x2 with_row(uint32_t x) {
#if __HIP_DEVICE_COMPILE__
  const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  return u32x2{r[0], r[1]};
#else
  return u32x2{x, x};
#endif
}
__device__ __forceinline__ u32x2 with_half(uint32_t x) {
#if __HIP_DEVICE_COMPILE__
  const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return u32x2{r[0], r[1]};
#else
  return u32x2{x, x};
#endif
}
// Every lane's value combined, in every lane (32-bit types); over 16 lanes, and over the wave.
template <typename T, typename F>
__device__ __forceinline__ T row_all(T v, F op) {
  auto step = [&](uint32_t other) { v = op(v, __builtin_bit_cast(T, other)); };
  step(dpp<0x128>(__builtin_bit_cast(uint32_t, v)));  // rotations within 16 lanes
  step(dpp<0x124>(__builtin_bit_cast(uint32_t, v)));
  step(dpp<0x122>(__builtin_bit_cast(uint32_t, v)));
  step(dpp<0x121>(__builtin_bit_cast(uint32_t, v)));
  return v;
}
template <typename T, typename F>
__device__ __forceinline__ T wave_all(T v, F op) {
  v = row_all(v, op);
  auto pair = [&](u32x2 r) {  // (elements copied: a bit cast takes whole objects)
    const uint32_t x = r[0], y = r[1];
    v = op(__builtin_bit_cast(T, x), __builtin_bit_cast(T, y));
  };
  pair(with_row(__builtin_bit_cast(uint32_t, v)));
  pair(with_half(__builtin_bit_cast(uint32_t, v)));
  return v;
}
struct Max {
  __device__ float operator()(float x, float y) const { return fmaxf(x, y); }
  __device__ uint32_t operator()(uint32_t x, uint32_t y) const { return max(x, y); }
  __device__ int operator()(int x, int y) const { return max(x, y); }
};
struct Or {
  __device__ int operator()(int x, int y) const { return x | y; }
};
struct Add {
  __device__ int operator()(int x, int y) const { return x + y; }
  __device__ float operator()(float x, float y) const { return x + y; }
};

// A 4-byte load through a buffer resource (as buf_ld16): zero at or past `bytes`.
__device__ __forceinline__ uint32_t buf_ld4(const void* base, int bytes, int voffset) {
#if __HIP_DEVICE_COMPILE__
  const __amdgpu_buffer_rsrc_t rsrc =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, bytes, kBufferFlags);
  return __builtin_amdgcn_raw_buffer_load_b32(rsrc, voffset, 0, 0);
#else
  return 0u;
#endif
}

// The sum over the lanes up to this one: within 16 lanes, then over the rows before.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);
  return v;
}
}  // namespace pkv
