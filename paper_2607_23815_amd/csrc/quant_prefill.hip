// Prefix-reuse prefill attention over a cache held in 8 or 4 bits (gfx950): the items, products, softmax and
// plan of the bf16 prefill (prefill_impl.h), on tiles that come from codes.
//
// A code times its scale is exact in bf16 (quant.h), so a tile in LDS is what the block's restored copy in the
// bf16 pool would be, and the results are pkv_prefill_attention's on that copy, bit for bit. A wave loads the
// codes of its block of a tile straight into the place of the tile in LDS, a quarter or half of it, and when
// they have landed takes them out, and puts the block there as bf16: no registers are held through a
// step's products, of which the softmax and the accumulators leave none.
#include "launch.h"
#include "prefill_impl.h"
#include "quant.h"

namespace pkv {
namespace {

template <int D, int BITS>
struct CodeTiles {
  using S = qnt::Slab<D, BITS>;
  static constexpr bool kDirect = false;
  const uint8_t* cache;

  // The codes of one side of a block, then its scales (64 bytes of values', D / 2 of keys'), to lds.
  template <int kScales>
  __device__ __forceinline__ static void issue(const uint8_t* from, uint16_t* lds, int lane) {
    uint8_t* to = reinterpret_cast<uint8_t*>(lds);
    constexpr int kBytes = S::kCodes + kScales;
    issue_loads<0, kBytes>(from, to, lane);
  }
  template <int kPart, int kBytes>
  __device__ __forceinline__ static void issue_loads(const uint8_t* from, uint8_t* to, int lane) {
    if constexpr ((kPart + 1) * 1024 <= kBytes)
      lds_load16(from, kBytes, kPart * 1024 + lane * 16, to + kPart * 1024);
    else if (lane < (kBytes - kPart * 1024) / 16)
      lds_load16(from, kBytes, kPart * 1024 + lane * 16, to + kPart * 1024);
    if constexpr ((kPart + 1) * 1024 < kBytes) issue_loads<kPart + 1, kBytes>(from, to, lane);
  }
  __device__ __forceinline__ const uint8_t* slab(int blk, int hkv, int kvh) const {
    return cache + ((size_t)blk * hkv + kvh) * S::kBytes;
  }
  __device__ __forceinline__ void issue_k(uint16_t* lds, int blk, int hkv, int kvh) const {
    issue<D / 2>(slab(blk, hkv, kvh), lds, lane_now());
  }
  __device__ __forceinline__ void issue_v(uint16_t* lds, int blk, int hkv, int kvh) const {
    issue<4 * kBlockSize>(slab(blk, hkv, kvh) + S::kValues, lds, lane_now());
  }

  // (the lane index afresh where it is used, so that no address made of it is kept through the steps)
  __device__ __forceinline__ static int lane_now() {
    int lane;
    asm volatile("v_and_b32 %0, 63, %1" : "=v"(lane) : "v"((int)threadIdx.x));
    return lane;
  }
  // This lane's codes, from a block's in LDS. (What follows writes where other lanes read here: the fence
  // keeps the wave's reads ahead.)
  __device__ __forceinline__ static void take(const uint8_t* lds, int at, int stride, uint32_t* w) {
    if constexpr (S::kLane == 8) {
      const u32x2 x = ld8(lds + at);
      w[0] = x[0], w[1] = x[1];
    } else {
#pragma unroll
      for (int u = 0; u < S::kLane / 16; ++u) {
        const u32x4 x = ld16(lds + at + u * stride);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[4 * u + e] = x[e];
      }
    }
  }
  __device__ __forceinline__ static void taken() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  // Chunk c of slot s goes to the unit that the score product reads it from.
  __device__ __forceinline__ void land_k(uint16_t* lds) const {
    const int lane = lane_now();
    const int col = lane & 15, grp = lane >> 4;
    const uint8_t* raw = reinterpret_cast<const uint8_t*>(lds);
    uint32_t k[S::kWords];
    take(raw, S::kLane == 8 ? (grp / 2) * 256 + col * 16 + (grp & 1) * 8
                            : grp * (S::kLane / 16) * 256 + col * 16, 256, k);
    const float scale =
        __uint_as_float((uint32_t)raw[S::kKeyScales + col * (D / 32) + grp * D / 128] << 23);
    taken();
    uint16_t* to = lds + (grp * (D / 32) * kBlockSize + pre::swap23(col)) * 8;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
      st16(to + i * kBlockSize * 8, qnt::eight_bf16<BITS>(k + i * BITS / 4, scale));
  }
  template <int kA>
  __device__ __forceinline__ static void put_values(const uint32_t* v, const u32x4 scale, uint16_t* to) {
    st8(to + kA * 16 * kBlockSize, qnt::four_scaled<BITS, kA>(v, scale));
    if constexpr (kA + 1 < D / 16) put_values<kA + 1>(v, scale, to);
  }
  // (the half that holds slots 8 h .. of dim d is unit 2 d + (h ^ (d / 8 % 2)))
  __device__ __forceinline__ void land_v(uint16_t* lds) const {
    const int lane = lane_now();
    const int col = lane & 15, grp = lane >> 4;
    const uint8_t* raw = reinterpret_cast<const uint8_t*>(lds);
    uint32_t v[S::kWords];
    take(raw, lane * (S::kLane < 16 ? S::kLane : 16), 1024, v);
    const u32x4 scale = ld16(raw + S::kCodes + 16 * grp);
    taken();
    put_values<0>(v, scale, lds + (2 * col + ((grp >> 1) ^ (col >> 3))) * 8 + (grp & 1) * 4);
  }
};

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

// (kPlan as in prefill.hip)
template <int D, int BITS, bool kPlan>
__global__ __attribute__((amdgpu_flat_work_group_size(pre::kThreads, pre::kThreads),
                          amdgpu_waves_per_eu(2, 2)))
void quant_prefill_kernel(const QuantPrefillArgs a) {
  __shared__ __align__(16) pre::PrefillSmem<D> sm;
  const CodeTiles<D, BITS> tiles{a.cache};
  if constexpr (kPlan)
    pre::prefill_body<D>(a.q, tiles, a.tables, a.max_blocks, a.cached_lens, a.cu_new_lens, a.num_seqs,
                         a.hq, a.hkv, a.num_blocks, a.qtiles, a.scale_log2, a.out, a.lse, blockIdx.x,
                         sm, a.split_keys, a.nsplit, a.ws_o, a.ws_ml, a.order, a.by_rank);
  else
    pre::prefill_body<D>(a.q, tiles, a.tables, a.max_blocks, a.cached_lens, a.cu_new_lens, a.num_seqs,
                         a.hq, a.hkv, a.num_blocks, a.qtiles, a.scale_log2, a.out, a.lse, blockIdx.x,
                         sm);
}

}  // namespace

hipError_t launch_quant_prefill(const uint8_t* cache, int32_t num_blocks, int32_t hkv, int32_t head_dim,
                                int32_t bits, const uint16_t* q, int32_t hq,
                                const int32_t* block_tables, int32_t max_blocks,
                                const int32_t* cached_lens, const int32_t* cu_new_lens,
                                int32_t num_seqs, int32_t total_new, int32_t max_new_len,
                                int32_t max_total_len, float scale, uint16_t* out, float* lse,
                                void* workspace, hipStream_t stream) {
  PrefillSplit sp{0, 1, false};
  if (workspace != nullptr)
    sp = prefill_split_plan(num_seqs, hq, hkv, max_new_len, max_total_len);
  QuantPrefillArgs a{};
  a.cache = cache;
  a.q = q;
  a.tables = block_tables;
  a.cached_lens = cached_lens;
  a.cu_new_lens = cu_new_lens;
  a.out = out;
  a.lse = lse;
  char* ws = static_cast<char*>(workspace);
  a.by_rank = sp.order && num_seqs <= kPrefillRankSeqs;
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
  const bool plan = sp.order || sp.nsplit > 1;
  auto* kern = head_dim == 128
                   ? (bits == 8 ? (plan ? quant_prefill_kernel<128, 8, true> : quant_prefill_kernel<128, 8, false>)
                                : (plan ? quant_prefill_kernel<128, 4, true> : quant_prefill_kernel<128, 4, false>))
                   : (bits == 8 ? (plan ? quant_prefill_kernel<64, 8, true> : quant_prefill_kernel<64, 8, false>)
                                : (plan ? quant_prefill_kernel<64, 4, true> : quant_prefill_kernel<64, 4, false>));
  hipLaunchKernelGGL(kern, dim3((unsigned)pg.items), dim3(pre::kThreads), 0, stream, a);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess || sp.nsplit <= 1) return err;
  return launch_prefill_merge(head_dim, cached_lens, cu_new_lens, num_seqs, hq, max_new_len, sp, a.ws_o,
                              a.ws_ml, out, lse, stream);
}

}  // namespace pkv
