// The C ABI's device calls: host-side argument validation, then the gfx950 kernel launches.
// Every check happens before any launch, so a refused call has enqueued nothing.
#include <hip/hip_runtime.h>

#include <atomic>
#include <cmath>
#include <cstdlib>
#include <cstring>
#include <string>

#include "internal.h"
#include "launch.h"

namespace pkv {

namespace {
thread_local std::string g_last_error;
}

pkv_status fail(pkv_status status, const std::string& message) {
  g_last_error = message;
  return status;
}

pkv_status ok() {
  g_last_error.clear();
  return PKV_OK;
}

namespace {

constexpr int kMaxGridZ = 65535;
constexpr int kMaxGridX = 1 << 30;

pkv_status check_kv(const pkv_paged_kv* kv, const char* fn, KvView* view) {
  const std::string f(fn);
  if (kv == nullptr) return fail(PKV_ERR_INVALID_ARG, f + ": kv is NULL");
  if (kv->k_cache == nullptr || kv->v_cache == nullptr)
    return fail(PKV_ERR_INVALID_ARG, f + ": k_cache / v_cache is NULL");
  if (kv->num_blocks <= 0 || kv->num_kv_heads <= 0)
    return fail(PKV_ERR_INVALID_ARG, f + ": num_blocks and num_kv_heads must be positive");
  if (kv->block_size != kSupportedBlockSize)
    return fail(PKV_ERR_UNSUPPORTED_SHAPE, f + ": block_size must be 16");
  if (kv->head_dim != 64 && kv->head_dim != 128)
    return fail(PKV_ERR_UNSUPPORTED_SHAPE, f + ": head_dim must be 64 or 128");
  if ((reinterpret_cast<uintptr_t>(kv->k_cache) | reinterpret_cast<uintptr_t>(kv->v_cache)) & 15)
    return fail(PKV_ERR_INVALID_ARG, f + ": k_cache / v_cache must be 16-byte aligned");
  view->k = static_cast<uint16_t*>(kv->k_cache);
  view->v = static_cast<uint16_t*>(kv->v_cache);
  view->num_blocks = kv->num_blocks;
  view->hkv = kv->num_kv_heads;
  view->head_dim = kv->head_dim;
  return PKV_OK;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

pkv_status launched(hipError_t err, const char* fn) {
  if (err != hipSuccess)
    return fail(PKV_ERR_HIP, std::string(fn) + ": " + hipGetErrorString(err));
  return ok();
}

// Opt-in validation of device metadata: off unless PKV_DEBUG_VALIDATE is set (and not "0")
// in the environment when the library first needs the setting, or pkv_set_debug_validate
// turns it on.
std::atomic<int> g_debug_validate{-1};

bool debug_validate() {
  int v = g_debug_validate.load(std::memory_order_relaxed);
  if (v < 0) {
    const char* e = std::getenv("PKV_DEBUG_VALIDATE");
    v = (e != nullptr && e[0] != '\0' && std::strcmp(e, "0") != 0) ? 1 : 0;
    int expected = -1;
    g_debug_validate.compare_exchange_strong(expected, v);
    v = g_debug_validate.load(std::memory_order_relaxed);
  }
  return v == 1;
}

// With validation on: run the checks (waiting for the stream) and refuse the call if any
// fails; with it off: nothing.
pkv_status check_metadata(const char* fn, const MetaCheck* checks, int n, hipStream_t stream) {
  if (!debug_validate()) return PKV_OK;
  uint32_t bad = 0u;
  int32_t seq = -1, which = -1;
  const hipError_t err = validate_metadata(checks, n, stream, &bad, &seq, &which);
  if (err != hipSuccess) return fail(PKV_ERR_HIP, std::string(fn) + ": " + hipGetErrorString(err));
  if (bad == 0u) return PKV_OK;
  std::string what;
  if (bad & kMetaBadBlockId) what += " a block id outside the pool;";
  if (bad & kMetaBadLength) what += " a length outside its host maximum or the table;";
  if (bad & kMetaBadSlot) what += " a slot outside the pool;";
  if (bad & kMetaBadOffsets) what += " token offsets not starting at 0, decreasing or not ending at the total;";
  std::string batch;
  if (n > 1) batch = which == 0 ? " of the prefill batch" : " of the decode batch";
  return fail(PKV_ERR_BAD_METADATA, std::string(fn) + ": PKV_DEBUG_VALIDATE refused the call:" +
                                        what + " first offending " +
                                        (checks[0].mode >= kMetaSlots ? "row " : "sequence ") +
                                        std::to_string(seq) + batch);
}

MetaCheck meta(int32_t mode, const KvView& view, const int32_t* tables, int32_t max_blocks,
               const int32_t* lens, const int32_t* cu, int32_t num_seqs, int64_t total,
               int64_t max_len, int64_t max_total) {
  MetaCheck c{};
  c.mode = mode;
  c.tables = tables;
  c.max_blocks = max_blocks;
  c.num_blocks = view.num_blocks;
  c.lens = lens;
  c.cu = cu;
  c.num_seqs = num_seqs;
  c.total = total;
  c.max_len = max_len;
  c.max_total = max_total;
  return c;
}

// Argument checks of a prefill batch (prefill and mixed calls); *empty when there is nothing
// to compute.
pkv_status check_prefill(const KvView& view, const char* fn, const void* q, int32_t num_q_heads,
                         const int32_t* block_tables, int32_t max_blocks,
                         const int32_t* cached_lens, const int32_t* cu_new_lens,
                         int32_t num_seqs, int32_t total_new, int32_t max_new_len,
                         int32_t max_total_len, float scale, const void* out,
                         const void* workspace, size_t workspace_bytes, bool* empty) {
  const std::string f(fn);
  *empty = false;
  if (num_q_heads <= 0 || num_q_heads % view.hkv != 0)
    return fail(PKV_ERR_UNSUPPORTED_SHAPE,
                f + ": num_q_heads must be a positive multiple of num_kv_heads");
  if (num_seqs < 0 || total_new < 0 || max_new_len < 0 || max_total_len < 0 || max_blocks < 0)
    return fail(PKV_ERR_INVALID_ARG, f + ": negative size");
  if (num_seqs == 0 || total_new == 0) {
    *empty = true;
    return ok();
  }
  if (q == nullptr || out == nullptr || block_tables == nullptr || cached_lens == nullptr ||
      cu_new_lens == nullptr)
    return fail(PKV_ERR_INVALID_ARG, f + ": NULL pointer");
  if (!aligned16(q) || !aligned16(out))
    return fail(PKV_ERR_INVALID_ARG, f + ": q / out must be 16-byte aligned");
  if (max_new_len == 0 || max_total_len < max_new_len || max_blocks == 0)
    return fail(PKV_ERR_INVALID_ARG,
                f + ": need 0 < max_new_len <= max_total_len, max_blocks > 0");
  if ((int64_t)max_blocks * kSupportedBlockSize < max_total_len)
    return fail(PKV_ERR_INVALID_ARG, f + ": max_total_len exceeds max_blocks * block_size");
  if (!(scale > 0.f)) return fail(PKV_ERR_INVALID_ARG, f + ": scale <= 0");
  if (num_seqs > kMaxGridZ)
    return fail(PKV_ERR_INVALID_ARG, f + ": more than 65535 sequences");
  // A workspace enables the key split of batches too small to fill the chip; without one
  // (NULL) the launch does not split. One that is given must hold what the split needs.
  const size_t need = prefill_workspace_bytes(num_seqs, total_new, num_q_heads, view.hkv,
                                              view.head_dim, max_new_len, max_total_len);
  if (need > 0 && workspace != nullptr && (workspace_bytes < need || !aligned16(workspace)))
    return fail(PKV_ERR_INVALID_ARG,
                f + ": workspace too small or not 16-byte aligned (see "
                    "pkv_prefill_workspace_bytes; NULL runs without the key split)");
  return ok();
}

// Argument checks of a decode batch (decode and mixed calls). With scratch set the call
// brings no workspace: the fixed scratch array must hold what it needs.
pkv_status check_decode(const KvView& view, const char* fn, const void* q, int32_t num_q_heads,
                        const int32_t* block_tables, int32_t max_blocks,
                        const int32_t* seq_lens, int32_t num_seqs, int32_t max_seq_len,
                        float scale, const void* out, const void* workspace,
                        size_t workspace_bytes, bool* empty, bool scratch = false) {
  const std::string f(fn);
  *empty = false;
  if (num_q_heads <= 0 || num_q_heads % view.hkv != 0 || num_q_heads / view.hkv > 16)
    return fail(PKV_ERR_UNSUPPORTED_SHAPE,
                f + ": num_q_heads must be a multiple of num_kv_heads, with at most 16 query "
                    "heads per kv head");
  if (num_seqs < 0 || max_seq_len < 0 || max_blocks < 0)
    return fail(PKV_ERR_INVALID_ARG, f + ": negative size");
  if (num_seqs == 0) {
    *empty = true;
    return ok();
  }
  if (q == nullptr || out == nullptr || block_tables == nullptr || seq_lens == nullptr)
    return fail(PKV_ERR_INVALID_ARG, f + ": NULL pointer");
  if (!aligned16(q) || !aligned16(out))
    return fail(PKV_ERR_INVALID_ARG, f + ": q / out must be 16-byte aligned");
  if (max_seq_len == 0 || max_blocks == 0)
    return fail(PKV_ERR_INVALID_ARG, f + ": max_seq_len, max_blocks must be > 0");
  if ((int64_t)max_blocks * kSupportedBlockSize < max_seq_len)
    return fail(PKV_ERR_INVALID_ARG, f + ": max_seq_len exceeds max_blocks * block_size");
  if (!(scale > 0.f)) return fail(PKV_ERR_INVALID_ARG, f + ": scale <= 0");
  const size_t need = decode_workspace_bytes(num_seqs, num_q_heads, view.hkv, view.head_dim,
                                             max_seq_len);
  if (scratch) {
    if (need > kDecodeScratchBytes)
      return fail(PKV_ERR_INVALID_ARG,
                  f + ": the call needs " + std::to_string(need) +
                      " bytes of workspace, above the fixed scratch of " +
                      std::to_string(kDecodeScratchBytes) +
                      " bytes (pkv_decode_attention takes a caller-owned workspace)");
    return ok();
  }
  if (need > 0 && (workspace == nullptr || workspace_bytes < need || !aligned16(workspace)))
    return fail(PKV_ERR_INVALID_ARG,
                f + ": workspace missing, too small or not 16-byte aligned "
                    "(see pkv_decode_workspace_bytes)");
  return ok();
}

constexpr int64_t kMaxRowItems = (int64_t(1) << 22) - 1;  // (row, kv head) pairs of a sparse read

// Argument checks that both sparse calls make of their rows.
pkv_status check_rows(const std::string& f, int32_t num_q_heads, int32_t hkv, const void* q,
                      const int32_t* block_tables, int32_t max_blocks, int32_t num_seqs,
                      const int32_t* row_seq, const int32_t* row_lens, int32_t rows,
                      int32_t blocks, const void* sel, bool* empty) {
  *empty = false;
  if (num_q_heads <= 0 || num_q_heads % hkv != 0 || num_q_heads / hkv > 16)
    return fail(PKV_ERR_UNSUPPORTED_SHAPE,
                f + ": num_q_heads must be a multiple of num_kv_heads, with at most 16 query "
                    "heads per kv head");
  if (rows < 0 || num_seqs < 0 || max_blocks < 0 || blocks < 0)
    return fail(PKV_ERR_INVALID_ARG, f + ": negative size");
  if (rows == 0) {
    *empty = true;
    return ok();
  }
  if (row_seq == nullptr && rows != num_seqs)
    return fail(PKV_ERR_INVALID_ARG, f + ": without row_seq, rows must equal num_seqs");
  if (blocks == 0) return fail(PKV_ERR_INVALID_ARG, f + ": blocks must be > 0");
  if (q == nullptr || row_lens == nullptr || sel == nullptr ||
      (block_tables == nullptr && num_seqs > 0 && max_blocks > 0))
    return fail(PKV_ERR_INVALID_ARG, f + ": NULL pointer");
  if (!aligned16(q)) return fail(PKV_ERR_INVALID_ARG, f + ": q must be 16-byte aligned");
  if ((int64_t)rows * hkv > kMaxRowItems)
    return fail(PKV_ERR_INVALID_ARG, f + ": 2^22 rows x kv heads or more");
  return PKV_OK;
}

struct QuantView {
  uint8_t* cache;
  int32_t num_blocks, hkv, head_dim, bits;
};

pkv_status check_quant(const pkv_quant_kv* kv, const std::string& f, QuantView* view) {
  if (kv == nullptr) return fail(PKV_ERR_INVALID_ARG, f + ": the quantised cache is NULL");
  if (kv->cache == nullptr) return fail(PKV_ERR_INVALID_ARG, f + ": cache is NULL");
  if (kv->num_blocks <= 0 || kv->num_kv_heads <= 0)
    return fail(PKV_ERR_INVALID_ARG, f + ": num_blocks and num_kv_heads must be positive");
  if (kv->block_size != kSupportedBlockSize)
    return fail(PKV_ERR_UNSUPPORTED_SHAPE, f + ": block_size must be 16");
  if (kv->head_dim != 64 && kv->head_dim != 128)
    return fail(PKV_ERR_UNSUPPORTED_SHAPE, f + ": head_dim must be 64 or 128");
  if (kv->bits != 4 && kv->bits != 8)
    return fail(PKV_ERR_UNSUPPORTED_SHAPE, f + ": bits must be 4 or 8");
  if (!aligned16(kv->cache))
    return fail(PKV_ERR_INVALID_ARG, f + ": cache must be 16-byte aligned");
  view->cache = static_cast<uint8_t*>(kv->cache);
  view->num_blocks = kv->num_blocks;
  view->hkv = kv->num_kv_heads;
  view->head_dim = kv->head_dim;
  view->bits = kv->bits;
  return PKV_OK;
}
// The view that metadata is checked and a bf16 call's arguments are looked at with.
KvView shape_of(const QuantView& v) { return KvView{nullptr, nullptr, v.num_blocks, v.hkv, v.head_dim}; }

pkv_status convert_blocks(const char* fn, const pkv_paged_kv* kv, const pkv_quant_kv* quant, bool back,
                          const int32_t* pairs, int32_t num_pairs, void* stream) {
  const std::string f(fn);
  KvView pool;
  pkv_status st = check_kv(kv, fn, &pool);
  if (st != PKV_OK) return st;
  QuantView view;
  st = check_quant(quant, f, &view);
  if (st != PKV_OK) return st;
  if (pool.hkv != view.hkv || pool.head_dim != view.head_dim)
    return fail(PKV_ERR_INVALID_ARG, f + ": the pools' num_kv_heads or head_dim differ");
  if (num_pairs < 0) return fail(PKV_ERR_INVALID_ARG, f + ": negative size");
  if (num_pairs == 0) return ok();
  if (pairs == nullptr) return fail(PKV_ERR_INVALID_ARG, f + ": NULL pointer");
  if ((int64_t)num_pairs * view.hkv > (1 << 26) - 4)  // (waves of a launch, four a workgroup, below 2^32 threads)
    return fail(PKV_ERR_INVALID_ARG, f + ": more than 2^26 - 4 pairs x kv heads");
  const QuantBlocksArgs a{view.cache, pool.k, pool.v, pairs, num_pairs, view.hkv, view.num_blocks,
                          pool.num_blocks};
  return launched(launch_quant_blocks(a, back, view.head_dim, view.bits,
                                      static_cast<hipStream_t>(stream)),
                  fn);
}

}  // namespace
}  // namespace pkv

using namespace pkv;

extern "C" {

const char* pkv_last_error(void) { return pkv::g_last_error.c_str(); }

int32_t pkv_abi_version(void) { return 2; }

pkv_status pkv_set_debug_validate(int32_t on) {
  g_debug_validate.store(on != 0 ? 1 : 0, std::memory_order_relaxed);
  return ok();
}

int32_t pkv_get_debug_validate(void) { return debug_validate() ? 1 : 0; }

pkv_status pkv_kv_append(const pkv_paged_kv* kv, const void* k_new, const void* v_new,
                         const int32_t* block_tables, int32_t max_blocks,
                         const int32_t* cached_lens, const int32_t* cu_new_lens,
                         int32_t num_seqs, int32_t total_new, int32_t max_new_len,
                         void* stream) {
  const char* fn = "pkv_kv_append";
  KvView view;
  pkv_status st = check_kv(kv, fn, &view);
  if (st != PKV_OK) return st;
  if (num_seqs < 0 || total_new < 0 || max_new_len < 0 || max_blocks < 0)
    return fail(PKV_ERR_INVALID_ARG, "pkv_kv_append: negative size");
  if (num_seqs == 0 || total_new == 0) return ok();
  if (k_new == nullptr || v_new == nullptr || block_tables == nullptr ||
      cached_lens == nullptr || cu_new_lens == nullptr)
    return fail(PKV_ERR_INVALID_ARG, "pkv_kv_append: NULL pointer");
  if (!aligned16(k_new) || !aligned16(v_new))
    return fail(PKV_ERR_INVALID_ARG, "pkv_kv_append: k_new / v_new must be 16-byte aligned");
  if (max_new_len == 0 || max_blocks == 0)
    return fail(PKV_ERR_INVALID_ARG, "pkv_kv_append: max_new_len and max_blocks must be > 0");
  if (num_seqs > kMaxGridZ)
    return fail(PKV_ERR_INVALID_ARG, "pkv_kv_append: more than 65535 sequences per call");
  {
    const MetaCheck c = meta(kMetaAppend, view, block_tables, max_blocks, cached_lens,
                             cu_new_lens, num_seqs, total_new, max_new_len,
                             (int64_t)max_blocks * kSupportedBlockSize);
    if ((st = check_metadata(fn, &c, 1, static_cast<hipStream_t>(stream))) != PKV_OK) return st;
  }
  return launched(launch_kv_append(view, static_cast<const uint16_t*>(k_new),
                                   static_cast<const uint16_t*>(v_new), block_tables,
                                   max_blocks, cached_lens, cu_new_lens, num_seqs, max_new_len,
                                   static_cast<hipStream_t>(stream)),
                  fn);
}

size_t pkv_prefill_workspace_bytes(int32_t num_seqs, int32_t total_new, int32_t num_q_heads,
                                   int32_t num_kv_heads, int32_t head_dim, int32_t max_new_len,
                                   int32_t max_total_len) {
  if (num_seqs <= 0 || total_new <= 0 || num_q_heads <= 0 || num_kv_heads <= 0 ||
      head_dim <= 0 || max_new_len <= 0 || max_total_len <= 0 ||
      num_q_heads % num_kv_heads != 0)
    return 0;
  return prefill_workspace_bytes(num_seqs, total_new, num_q_heads, num_kv_heads, head_dim,
                                 max_new_len, max_total_len);
}

pkv_status pkv_prefill_attention(const pkv_paged_kv* kv, const void* q, int32_t num_q_heads,
                                 const int32_t* block_tables, int32_t max_blocks,
                                 const int32_t* cached_lens, const int32_t* cu_new_lens,
                                 int32_t num_seqs, int32_t total_new, int32_t max_new_len,
                                 int32_t max_total_len, float scale, void* out, float* lse,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  const char* fn = "pkv_prefill_attention";
  KvView view;
  pkv_status st = check_kv(kv, fn, &view);
  if (st != PKV_OK) return st;
  bool empty = false;
  st = check_prefill(view, fn, q, num_q_heads, block_tables, max_blocks, cached_lens,
                     cu_new_lens, num_seqs, total_new, max_new_len, max_total_len, scale, out,
                     workspace, workspace_bytes, &empty);
  if (st != PKV_OK || empty) return st;
  {
    const MetaCheck c = meta(kMetaPrefill, view, block_tables, max_blocks, cached_lens,
                             cu_new_lens, num_seqs, total_new, max_new_len, max_total_len);
    if ((st = check_metadata(fn, &c, 1, static_cast<hipStream_t>(stream))) != PKV_OK) return st;
  }
  const bool split = workspace != nullptr &&
                     prefill_workspace_bytes(num_seqs, total_new, num_q_heads, view.hkv,
                                             view.head_dim, max_new_len, max_total_len) > 0;
  return launched(launch_prefill(view, static_cast<const uint16_t*>(q), num_q_heads,
                                 block_tables, max_blocks, cached_lens, cu_new_lens, num_seqs,
                                 total_new, max_new_len, max_total_len, scale,
                                 static_cast<uint16_t*>(out), lse, split ? workspace : nullptr,
                                 static_cast<hipStream_t>(stream)),
                  fn);
}

size_t pkv_decode_workspace_bytes(int32_t num_seqs, int32_t num_q_heads, int32_t num_kv_heads,
                                  int32_t head_dim, int32_t max_seq_len) {
  if (num_seqs <= 0 || num_q_heads <= 0 || num_kv_heads <= 0 || head_dim <= 0 ||
      max_seq_len <= 0)
    return 0;
  return decode_workspace_bytes(num_seqs, num_q_heads, num_kv_heads, head_dim, max_seq_len);
}

pkv_status pkv_decode_attention(const pkv_paged_kv* kv, const void* q, int32_t num_q_heads,
                                const int32_t* block_tables, int32_t max_blocks,
                                const int32_t* seq_lens, int32_t num_seqs, int32_t max_seq_len,
                                float scale, void* out, float* lse, void* workspace,
                                size_t workspace_bytes, void* stream) {
  const char* fn = "pkv_decode_attention";
  KvView view;
  pkv_status st = check_kv(kv, fn, &view);
  if (st != PKV_OK) return st;
  bool empty = false;
  st = check_decode(view, fn, q, num_q_heads, block_tables, max_blocks, seq_lens, num_seqs,
                    max_seq_len, scale, out, workspace, workspace_bytes, &empty);
  if (st != PKV_OK || empty) return st;
  {
    const MetaCheck c = meta(kMetaDecode, view, block_tables, max_blocks, seq_lens, nullptr,
                             num_seqs, -1, max_seq_len, 0);
    if ((st = check_metadata(fn, &c, 1, static_cast<hipStream_t>(stream))) != PKV_OK) return st;
  }
  return launched(launch_decode(view, static_cast<const uint16_t*>(q), num_q_heads,
                                block_tables, max_blocks, seq_lens, num_seqs, max_seq_len, scale,
                                static_cast<uint16_t*>(out), lse, workspace,
                                static_cast<hipStream_t>(stream)),
                  fn);
}

pkv_status pkv_decode_attention_noalloc(const pkv_paged_kv* kv, const void* q,
                                        int32_t num_q_heads, const int32_t* block_tables,
                                        int32_t max_blocks, const int32_t* seq_lens,
                                        int32_t num_seqs, int32_t max_seq_len, float scale,
                                        void* out, float* lse, void* stream) {
  const char* fn = "pkv_decode_attention_noalloc";
  static_assert(PKV_DECODE_NOALLOC_MAX_BYTES == kDecodeScratchBytes,
                "the header's limit is the scratch array's size");
  KvView view;
  pkv_status st = check_kv(kv, fn, &view);
  if (st != PKV_OK) return st;
  bool empty = false;
  st = check_decode(view, fn, q, num_q_heads, block_tables, max_blocks, seq_lens, num_seqs,
                    max_seq_len, scale, out, nullptr, 0, &empty, /*scratch=*/true);
  if (st != PKV_OK || empty) return st;
  {
    const MetaCheck c = meta(kMetaDecode, view, block_tables, max_blocks, seq_lens, nullptr,
                             num_seqs, -1, max_seq_len, 0);
    if ((st = check_metadata(fn, &c, 1, static_cast<hipStream_t>(stream))) != PKV_OK) return st;
  }
  void* ws = nullptr;
  const hipError_t err = decode_scratch(&ws);
  if (err != hipSuccess) return launched(err, fn);
  return launched(launch_decode(view, static_cast<const uint16_t*>(q), num_q_heads,
                                block_tables, max_blocks, seq_lens, num_seqs, max_seq_len, scale,
                                static_cast<uint16_t*>(out), lse, ws,
                                static_cast<hipStream_t>(stream)),
                  fn);
}

pkv_status pkv_mixed_attention(const pkv_paged_kv* kv, int32_t num_q_heads, float scale,
                               const void* q, const int32_t* block_tables, int32_t max_blocks,
                               const int32_t* cached_lens, const int32_t* cu_new_lens,
                               int32_t num_seqs, int32_t total_new, int32_t max_new_len,
                               int32_t max_total_len, void* out, float* lse, const void* dq,
                               const int32_t* d_block_tables, int32_t d_max_blocks,
                               const int32_t* seq_lens, int32_t d_num_seqs,
                               int32_t max_seq_len, void* d_out, float* d_lse,
                               void* workspace, size_t workspace_bytes, void* stream) {
  const char* fn = "pkv_mixed_attention";
  KvView view;
  pkv_status st = check_kv(kv, fn, &view);
  if (st != PKV_OK) return st;
  bool no_prefill = false, no_decode = false;
  st = check_prefill(view, fn, q, num_q_heads, block_tables, max_blocks, cached_lens,
                     cu_new_lens, num_seqs, total_new, max_new_len, max_total_len, scale, out,
                     nullptr, 0, &no_prefill);
  if (st != PKV_OK) return st;
  st = check_decode(view, fn, dq, num_q_heads, d_block_tables, d_max_blocks, seq_lens,
                    d_num_seqs, max_seq_len, scale, d_out, workspace, workspace_bytes,
                    &no_decode);
  if (st != PKV_OK) return st;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (no_prefill && no_decode) return ok();
  {
    MetaCheck c[2];
    c[0] = meta(kMetaPrefill, view, block_tables, max_blocks, cached_lens, cu_new_lens,
                no_prefill ? 0 : num_seqs, total_new, max_new_len, max_total_len);
    c[1] = meta(kMetaDecode, view, d_block_tables, d_max_blocks, seq_lens, nullptr,
                no_decode ? 0 : d_num_seqs, -1, max_seq_len, 0);
    if ((st = check_metadata(fn, c, 2, s)) != PKV_OK) return st;
  }
  if (no_decode)
    return launched(launch_prefill(view, static_cast<const uint16_t*>(q), num_q_heads,
                                   block_tables, max_blocks, cached_lens, cu_new_lens, num_seqs,
                                   total_new, max_new_len, max_total_len, scale,
                                   static_cast<uint16_t*>(out), lse, nullptr, s),
                    fn);
  if (no_prefill)
    return launched(launch_decode(view, static_cast<const uint16_t*>(dq), num_q_heads,
                                  d_block_tables, d_max_blocks, seq_lens, d_num_seqs,
                                  max_seq_len, scale, static_cast<uint16_t*>(d_out), d_lse,
                                  workspace, s),
                    fn);
  return launched(launch_mixed(view, num_q_heads, scale, static_cast<const uint16_t*>(q),
                               block_tables, max_blocks, cached_lens, cu_new_lens, num_seqs,
                               max_new_len, static_cast<uint16_t*>(out), lse,
                               static_cast<const uint16_t*>(dq), d_block_tables, d_max_blocks,
                               seq_lens, d_num_seqs, max_seq_len, static_cast<uint16_t*>(d_out),
                               d_lse, workspace, s),
                  fn);
}

pkv_status pkv_gather_kv(const pkv_paged_kv* kv, const int32_t* block_tables,
                         int32_t max_blocks, const int32_t* lens, const int32_t* cu_lens,
                         int32_t num_seqs, int32_t max_len, void* k_out, void* v_out,
                         void* stream) {
  const char* fn = "pkv_gather_kv";
  KvView view;
  pkv_status st = check_kv(kv, fn, &view);
  if (st != PKV_OK) return st;
  if (num_seqs < 0 || max_len < 0 || max_blocks < 0)
    return fail(PKV_ERR_INVALID_ARG, "pkv_gather_kv: negative size");
  if (num_seqs == 0 || max_len == 0) return ok();
  if (block_tables == nullptr || lens == nullptr || cu_lens == nullptr || k_out == nullptr ||
      v_out == nullptr)
    return fail(PKV_ERR_INVALID_ARG, "pkv_gather_kv: NULL pointer");
  if (!aligned16(k_out) || !aligned16(v_out))
    return fail(PKV_ERR_INVALID_ARG, "pkv_gather_kv: outputs must be 16-byte aligned");
  if (num_seqs > kMaxGridZ)
    return fail(PKV_ERR_INVALID_ARG, "pkv_gather_kv: more than 65535 sequences per call");
  {
    const MetaCheck c = meta(kMetaGather, view, block_tables, max_blocks, lens, cu_lens,
                             num_seqs, -1, max_len, 0);
    if ((st = check_metadata(fn, &c, 1, static_cast<hipStream_t>(stream))) != PKV_OK) return st;
  }
  return launched(launch_gather_kv(view, block_tables, max_blocks, lens, cu_lens, num_seqs,
                                   max_len, static_cast<uint16_t*>(k_out),
                                   static_cast<uint16_t*>(v_out),
                                   static_cast<hipStream_t>(stream)),
                  fn);
}

pkv_status pkv_copy_blocks(const pkv_paged_kv* kv, const int32_t* pairs, int32_t num_pairs,
                           void* stream) {
  const char* fn = "pkv_copy_blocks";
  KvView view;
  pkv_status st = check_kv(kv, fn, &view);
  if (st != PKV_OK) return st;
  if (num_pairs < 0) return fail(PKV_ERR_INVALID_ARG, "pkv_copy_blocks: negative size");
  if (num_pairs == 0) return ok();
  if (pairs == nullptr) return fail(PKV_ERR_INVALID_ARG, "pkv_copy_blocks: NULL pointer");
  if (num_pairs > kMaxGridX)
    return fail(PKV_ERR_INVALID_ARG, "pkv_copy_blocks: too many pairs per call");
  return launched(launch_copy_blocks(view, pairs, num_pairs, static_cast<hipStream_t>(stream)),
                  fn);
}

pkv_status pkv_extend_tables(int32_t* block_tables, int32_t max_blocks,
                             const int32_t* cached_lens, const int32_t* new_lens,
                             int32_t num_seqs, const int32_t* free_blocks, int32_t num_free,
                             const int32_t* free_used, int32_t* free_used_out,
                             int32_t* cu_new_lens, int32_t* seq_lens, int32_t* status,
                             int32_t max_rows, int64_t* slot_map, int32_t* row_seq,
                             int32_t* positions, int32_t* row_lens, void* stream) {
  const char* fn = "pkv_extend_tables";
  if (max_blocks < 0 || num_seqs < 0 || num_free < 0 || max_rows < 0)
    return fail(PKV_ERR_INVALID_ARG, "pkv_extend_tables: negative size");
  if (max_rows > kMaxGridX)
    return fail(PKV_ERR_INVALID_ARG, "pkv_extend_tables: more than 2^30 rows");
  if (free_used == nullptr || free_used_out == nullptr || cu_new_lens == nullptr ||
      status == nullptr)
    return fail(PKV_ERR_INVALID_ARG, "pkv_extend_tables: NULL pointer");
  if (num_seqs > 0 && (cached_lens == nullptr || new_lens == nullptr || seq_lens == nullptr ||
                       (block_tables == nullptr && max_blocks > 0)))
    return fail(PKV_ERR_INVALID_ARG, "pkv_extend_tables: NULL pointer");
  if (num_free > 0 && free_blocks == nullptr)
    return fail(PKV_ERR_INVALID_ARG, "pkv_extend_tables: free_blocks is NULL");
  const ExtendArgs a{block_tables, max_blocks,    cached_lens, new_lens, num_seqs,  free_blocks,
                     num_free,     free_used,     free_used_out, cu_new_lens, seq_lens, status,
                     max_rows,     slot_map,      row_seq,     positions, row_lens};
  return launched(launch_extend_tables(a, static_cast<hipStream_t>(stream)), fn);
}

pkv_status pkv_rope_append(const pkv_paged_kv* kv, const pkv_rope* rope, const void* q,
                           int64_t q_stride, int32_t num_q_heads, const void* k_new,
                           int64_t k_stride, const void* v_new, int64_t v_stride,
                           const int64_t* slot_map, const int32_t* positions,
                           int64_t pos_stride, int32_t rows, void* q_out, int64_t q_out_stride,
                           void* stream) {
  const char* fn = "pkv_rope_append";
  const std::string f(fn);
  KvView view;
  pkv_status st = check_kv(kv, fn, &view);
  if (st != PKV_OK) return st;
  if (num_q_heads <= 0 || num_q_heads % view.hkv != 0)
    return fail(PKV_ERR_UNSUPPORTED_SHAPE,
                f + ": num_q_heads must be a positive multiple of num_kv_heads");
  if (rope == nullptr) return fail(PKV_ERR_INVALID_ARG, f + ": rope is NULL");
  if (rope->rot_dim < 0 || rope->rot_dim > view.head_dim || rope->rot_dim % 16 != 0)
    return fail(PKV_ERR_UNSUPPORTED_SHAPE,
                f + ": rot_dim must be a multiple of 16, at most head_dim");
  if (rope->num_axes < 1 || rope->num_axes > PKV_ROPE_MAX_AXES)
    return fail(PKV_ERR_INVALID_ARG, f + ": num_axes must be 1 to 4");
  if (!std::isfinite(rope->scale)) return fail(PKV_ERR_INVALID_ARG, f + ": scale is not finite");
  for (int j = 0; j < rope->rot_dim / 2; ++j) {
    if (rope->axis_of[j] >= rope->num_axes)
      return fail(PKV_ERR_INVALID_ARG, f + ": axis_of names an axis past num_axes");
    if (!(std::fabs(rope->inv_freq[j]) <= 0x1p20))  // (an angle of 2^51 has no fraction left)
      return fail(PKV_ERR_INVALID_ARG, f + ": inv_freq is not finite, or above 2^20");
  }
  if (rows < 0) return fail(PKV_ERR_INVALID_ARG, f + ": negative size");
  if (rows == 0) return ok();
  if (((int64_t)rows + 15) / 16 * view.hkv >= (1 << 24))  // (workgroups of a launch)
    return fail(PKV_ERR_INVALID_ARG, f + ": 2^28 rows x kv heads or more");
  if (q == nullptr || k_new == nullptr || v_new == nullptr || slot_map == nullptr ||
      q_out == nullptr || (positions == nullptr && rope->rot_dim > 0))
    return fail(PKV_ERR_INVALID_ARG, f + ": NULL pointer");
  if (!aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(q_out))
    return fail(PKV_ERR_INVALID_ARG, f + ": q / k_new / v_new / q_out must be 16-byte aligned");
  const int64_t q_row = (int64_t)num_q_heads * view.head_dim;
  const int64_t kv_row = (int64_t)view.hkv * view.head_dim;
  if (q_stride < q_row || q_out_stride < q_row || k_stride < kv_row || v_stride < kv_row ||
      (q_stride | q_out_stride | k_stride | v_stride) & 7)
    return fail(PKV_ERR_INVALID_ARG,
                f + ": row strides must be multiples of 8 elements that hold a row");
  if (rope->num_axes > 1 && pos_stride < rows)
    return fail(PKV_ERR_INVALID_ARG, f + ": pos_stride is below rows");
  {
    MetaCheck c = meta(kMetaSlots, view, nullptr, 0, nullptr, nullptr, rows, -1, 0, 0);
    c.slots = slot_map;
    if ((st = check_metadata(fn, &c, 1, static_cast<hipStream_t>(stream))) != PKV_OK) return st;
  }
  RopeArgs a{};
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k_new);
  a.v = static_cast<const uint16_t*>(v_new);
  a.q_out = static_cast<uint16_t*>(q_out);
  a.k_cache = view.k;
  a.v_cache = view.v;
  a.slot_map = slot_map;
  a.positions = positions;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.q_out_stride = q_out_stride;
  a.pos_stride = pos_stride;
  a.rows = rows;
  a.hq = num_q_heads;
  a.hkv = view.hkv;
  a.num_blocks = view.num_blocks;
  a.rot_dim = rope->rot_dim;
  a.interleaved = rope->interleaved != 0;
  a.scale = rope->scale;
  for (int j = 0; j < rope->rot_dim / 2; ++j) {
    a.axis_of[j] = rope->axis_of[j];
    a.turns[j] = rope->inv_freq[j] / 6.283185307179586476925;
  }
  return launched(launch_rope_append(a, view.head_dim, static_cast<hipStream_t>(stream)), fn);
}

pkv_status pkv_block_bounds(const pkv_paged_kv* kv, void* bounds, const int32_t* block_tables,
                            int32_t max_blocks, const int32_t* cached_lens,
                            const int32_t* cu_new_lens, int32_t num_seqs, int32_t max_new_len,
                            void* stream) {
  const char* fn = "pkv_block_bounds";
  KvView view;
  pkv_status st = check_kv(kv, fn, &view);
  if (st != PKV_OK) return st;
  if (num_seqs < 0 || max_new_len < 0 || max_blocks < 0)
    return fail(PKV_ERR_INVALID_ARG, "pkv_block_bounds: negative size");
  if (num_seqs == 0 || max_new_len == 0 || max_blocks == 0) return ok();
  if (bounds == nullptr || block_tables == nullptr || cached_lens == nullptr ||
      cu_new_lens == nullptr)
    return fail(PKV_ERR_INVALID_ARG, "pkv_block_bounds: NULL pointer");
  if (!aligned16(bounds))
    return fail(PKV_ERR_INVALID_ARG, "pkv_block_bounds: bounds must be 16-byte aligned");
  if (num_seqs > kMaxGridZ)
    return fail(PKV_ERR_INVALID_ARG, "pkv_block_bounds: more than 65535 sequences per call");
  if (max_blocks >= (1 << 24))  // (workgroups of a launch)
    return fail(PKV_ERR_INVALID_ARG, "pkv_block_bounds: 2^24 blocks of a sequence or more");
  {
    const MetaCheck c = meta(kMetaAppend, view, block_tables, max_blocks, cached_lens,
                             cu_new_lens, num_seqs, -1, max_new_len,
                             (int64_t)max_blocks * kSupportedBlockSize);
    if ((st = check_metadata(fn, &c, 1, static_cast<hipStream_t>(stream))) != PKV_OK) return st;
  }
  return launched(launch_block_bounds(view, static_cast<uint16_t*>(bounds), block_tables,
                                      max_blocks, cached_lens, cu_new_lens, num_seqs,
                                      max_new_len, static_cast<hipStream_t>(stream)),
                  fn);
}

size_t pkv_select_workspace_bytes(int32_t rows, int32_t num_q_heads, int32_t num_kv_heads,
                                  int32_t head_dim, int32_t max_len, int32_t blocks) {
  if (rows <= 0 || num_q_heads <= 0 || num_kv_heads <= 0 || head_dim <= 0 || max_len <= 0 ||
      blocks <= 0 || (int64_t)rows * num_kv_heads > kMaxRowItems ||
      max_len > kSelectMaxBlocks * kSupportedBlockSize)
    return 0;
  return select_workspace_bytes((int64_t)rows * num_kv_heads, max_len, blocks);
}

pkv_status pkv_select_blocks(const void* bounds, int32_t num_blocks, int32_t num_kv_heads,
                             int32_t head_dim, const void* q, int32_t num_q_heads,
                             const int32_t* block_tables, int32_t max_blocks, int32_t num_seqs,
                             const int32_t* row_seq, const int32_t* row_lens, int32_t rows,
                             int32_t max_len, int32_t sink_blocks, int32_t recent_blocks,
                             int32_t blocks, int32_t* sel, void* workspace,
                             size_t workspace_bytes, void* stream) {
  const char* fn = "pkv_select_blocks";
  const std::string f(fn);
  if (num_blocks <= 0 || num_kv_heads <= 0)
    return fail(PKV_ERR_INVALID_ARG, f + ": num_blocks and num_kv_heads must be positive");
  if (head_dim != 64 && head_dim != 128)
    return fail(PKV_ERR_UNSUPPORTED_SHAPE, f + ": head_dim must be 64 or 128");
  bool empty = false;
  pkv_status st = check_rows(f, num_q_heads, num_kv_heads, q, block_tables, max_blocks, num_seqs,
                             row_seq, row_lens, rows, blocks, sel, &empty);
  if (st != PKV_OK || empty) return st;
  if (bounds == nullptr || !aligned16(bounds))
    return fail(PKV_ERR_INVALID_ARG, f + ": bounds is NULL or not 16-byte aligned");
  if (max_len < 0) return fail(PKV_ERR_INVALID_ARG, f + ": negative size");
  if (max_len > kSelectMaxBlocks * kSupportedBlockSize)
    return fail(PKV_ERR_INVALID_ARG, f + ": max_len is above 2^20");
  if ((int64_t)max_blocks * kSupportedBlockSize < max_len)
    return fail(PKV_ERR_INVALID_ARG, f + ": max_len exceeds max_blocks * block_size");
  if (sink_blocks < 0 || recent_blocks < 1 || (int64_t)sink_blocks + recent_blocks > blocks)
    return fail(PKV_ERR_INVALID_ARG,
                f + ": need sink_blocks >= 0, recent_blocks >= 1 and their sum <= blocks");
  const size_t need = select_workspace_bytes((int64_t)rows * num_kv_heads, max_len, blocks);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need || !aligned16(workspace)))
    return fail(PKV_ERR_INVALID_ARG,
                f + ": workspace missing, too small or not 16-byte aligned "
                    "(see pkv_select_workspace_bytes)");
  const hipStream_t s = static_cast<hipStream_t>(stream);
  {
    KvView view{nullptr, nullptr, num_blocks, num_kv_heads, head_dim};
    MetaCheck c = meta(kMetaRows, view, block_tables, max_blocks, row_lens, nullptr, rows, -1,
                       max_len, 0);
    c.row_seq = row_seq;
    c.table_rows = num_seqs;
    if ((st = check_metadata(fn, &c, 1, s)) != PKV_OK) return st;
  }
  SelectArgs a{};
  a.bounds = static_cast<const uint16_t*>(bounds);
  a.q = static_cast<const uint16_t*>(q);
  a.tables = block_tables;
  a.row_seq = row_seq;
  a.row_lens = row_lens;
  a.sel = sel;
  a.rows = rows;
  a.max_blocks = max_blocks;
  a.num_seqs = num_seqs;
  a.max_len = max_len;
  a.hq = num_q_heads;
  a.hkv = num_kv_heads;
  a.num_blocks = num_blocks;
  a.blocks = blocks;
  a.sink = sink_blocks;
  a.recent = recent_blocks;
  return launched(launch_select_blocks(a, head_dim, workspace, s), fn);
}

size_t pkv_sparse_workspace_bytes(int32_t rows, int32_t num_q_heads, int32_t num_kv_heads,
                                  int32_t head_dim, int32_t blocks) {
  if (rows <= 0 || num_q_heads <= 0 || num_kv_heads <= 0 || num_q_heads % num_kv_heads != 0 ||
      head_dim <= 0 || blocks <= 0 || blocks > kSelectMaxBlocks ||
      (int64_t)rows * num_kv_heads > kMaxRowItems)
    return 0;
  return sparse_workspace_bytes((int64_t)rows * num_kv_heads, num_q_heads / num_kv_heads,
                                head_dim, blocks);
}

pkv_status pkv_sparse_attention(const pkv_paged_kv* kv, const void* q, int32_t num_q_heads,
                                const int32_t* block_tables, int32_t max_blocks,
                                int32_t num_seqs, const int32_t* row_seq,
                                const int32_t* row_lens, int32_t rows, const int32_t* sel,
                                int32_t blocks, float scale, void* out, float* lse,
                                void* workspace, size_t workspace_bytes, void* stream) {
  const char* fn = "pkv_sparse_attention";
  const std::string f(fn);
  KvView view;
  pkv_status st = check_kv(kv, fn, &view);
  if (st != PKV_OK) return st;
  bool empty = false;
  st = check_rows(f, num_q_heads, view.hkv, q, block_tables, max_blocks, num_seqs, row_seq,
                  row_lens, rows, blocks, sel, &empty);
  if (st != PKV_OK || empty) return st;
  if (blocks > kSelectMaxBlocks)
    return fail(PKV_ERR_INVALID_ARG, f + ": more than 65536 blocks of a row");
  if (out == nullptr || !aligned16(out))
    return fail(PKV_ERR_INVALID_ARG, f + ": out is NULL or not 16-byte aligned");
  if (!(scale > 0.f)) return fail(PKV_ERR_INVALID_ARG, f + ": scale <= 0");
  const size_t need = sparse_workspace_bytes((int64_t)rows * view.hkv, num_q_heads / view.hkv,
                                             view.head_dim, blocks);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need || !aligned16(workspace)))
    return fail(PKV_ERR_INVALID_ARG,
                f + ": workspace missing, too small or not 16-byte aligned "
                    "(see pkv_sparse_workspace_bytes)");
  const hipStream_t s = static_cast<hipStream_t>(stream);
  {
    // (lengths past the table and entries outside the pool are in order here)
    MetaCheck c = meta(kMetaRows, view, nullptr, 0, row_lens, nullptr, rows, -1, INT32_MAX, 0);
    c.row_seq = row_seq;
    c.table_rows = num_seqs;
    if ((st = check_metadata(fn, &c, 1, s)) != PKV_OK) return st;
  }
  SparseArgs a{};
  a.k_cache = view.k;
  a.v_cache = view.v;
  a.q = static_cast<const uint16_t*>(q);
  a.tables = block_tables;
  a.row_seq = row_seq;
  a.row_lens = row_lens;
  a.sel = sel;
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.rows = rows;
  a.max_blocks = max_blocks;
  a.num_seqs = num_seqs;
  a.hq = num_q_heads;
  a.hkv = view.hkv;
  a.num_blocks = view.num_blocks;
  a.blocks = blocks;
  a.scale_log2 = scale * 1.44269504088896340736f;
  return launched(launch_sparse_attention(a, view.head_dim, workspace, s), fn);
}

size_t pkv_quant_block_bytes(int32_t num_kv_heads, int32_t head_dim, int32_t bits) {
  if (num_kv_heads <= 0 || (head_dim != 64 && head_dim != 128) || (bits != 4 && bits != 8)) return 0;
  return (size_t)num_kv_heads * quant_slab_bytes(head_dim, bits);
}

pkv_status pkv_quant_append(const pkv_quant_kv* kv, const void* k_new, int64_t k_stride,
                            const void* v_new, int64_t v_stride, const int32_t* block_tables,
                            int32_t max_blocks, const int32_t* cached_lens,
                            const int32_t* cu_new_lens, int32_t num_seqs, int32_t total_new,
                            int32_t max_new_len, void* stream) {
  const char* fn = "pkv_quant_append";
  const std::string f(fn);
  QuantView view;
  pkv_status st = check_quant(kv, f, &view);
  if (st != PKV_OK) return st;
  if (num_seqs < 0 || total_new < 0 || max_new_len < 0 || max_blocks < 0)
    return fail(PKV_ERR_INVALID_ARG, f + ": negative size");
  if (num_seqs == 0 || total_new == 0) return ok();
  if (k_new == nullptr || v_new == nullptr || block_tables == nullptr || cached_lens == nullptr ||
      cu_new_lens == nullptr)
    return fail(PKV_ERR_INVALID_ARG, f + ": NULL pointer");
  if (!aligned16(k_new) || !aligned16(v_new))
    return fail(PKV_ERR_INVALID_ARG, f + ": k_new / v_new must be 16-byte aligned");
  const int64_t row = (int64_t)view.hkv * view.head_dim;
  if (k_stride < row || v_stride < row || (k_stride | v_stride) & 7)
    return fail(PKV_ERR_INVALID_ARG,
                f + ": row strides must be multiples of 8 elements that hold a row");
  if (max_new_len == 0 || max_blocks == 0)
    return fail(PKV_ERR_INVALID_ARG, f + ": max_new_len and max_blocks must be > 0");
  if (num_seqs > kMaxGridZ)
    return fail(PKV_ERR_INVALID_ARG, f + ": more than 65535 sequences per call");
  if (((int64_t)max_new_len / kSupportedBlockSize + 2) * view.hkv >= (1 << 24))
    return fail(PKV_ERR_INVALID_ARG, f + ": 2^24 blocks x kv heads of a sequence or more");
  const hipStream_t s = static_cast<hipStream_t>(stream);
  {
    const MetaCheck c = meta(kMetaAppend, shape_of(view), block_tables, max_blocks, cached_lens,
                             cu_new_lens, num_seqs, total_new, max_new_len,
                             (int64_t)max_blocks * kSupportedBlockSize);
    if ((st = check_metadata(fn, &c, 1, s)) != PKV_OK) return st;
  }
  QuantAppendArgs a{};
  a.cache = view.cache;
  a.k = static_cast<const uint16_t*>(k_new);
  a.v = static_cast<const uint16_t*>(v_new);
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.rows = total_new;
  a.tables = block_tables;
  a.cached_lens = cached_lens;
  a.cu_new_lens = cu_new_lens;
  a.max_blocks = max_blocks;
  a.hkv = view.hkv;
  a.num_blocks = view.num_blocks;
  return launched(launch_quant_append(a, num_seqs, max_new_len, view.head_dim, view.bits, s), fn);
}

pkv_status pkv_quant_blocks(const pkv_paged_kv* from, const pkv_quant_kv* to, const int32_t* pairs,
                            int32_t num_pairs, void* stream) {
  return convert_blocks("pkv_quant_blocks", from, to, false, pairs, num_pairs, stream);
}

pkv_status pkv_dequant_blocks(const pkv_quant_kv* from, const pkv_paged_kv* to, const int32_t* pairs,
                              int32_t num_pairs, void* stream) {
  return convert_blocks("pkv_dequant_blocks", to, from, true, pairs, num_pairs, stream);
}

size_t pkv_quant_decode_workspace_bytes(int32_t num_seqs, int32_t num_q_heads, int32_t num_kv_heads,
                                        int32_t head_dim, int32_t bits, int32_t max_seq_len) {
  if (num_seqs <= 0 || num_q_heads <= 0 || num_kv_heads <= 0 || num_q_heads % num_kv_heads != 0 ||
      head_dim <= 0 || max_seq_len <= 0 || (int64_t)num_seqs * num_kv_heads > kMaxRowItems)
    return 0;
  return quant_decode_workspace_bytes(num_seqs, num_q_heads, num_kv_heads, head_dim, bits,
                                      max_seq_len);
}

pkv_status pkv_quant_decode_attention(const pkv_quant_kv* kv, const void* q, int32_t num_q_heads,
                                      const int32_t* block_tables, int32_t max_blocks,
                                      const int32_t* seq_lens, int32_t num_seqs,
                                      int32_t max_seq_len, float scale, void* out, float* lse,
                                      void* workspace, size_t workspace_bytes, void* stream) {
  const char* fn = "pkv_quant_decode_attention";
  const std::string f(fn);
  QuantView view;
  pkv_status st = check_quant(kv, f, &view);
  if (st != PKV_OK) return st;
  if (num_q_heads <= 0 || num_q_heads % view.hkv != 0 || num_q_heads / view.hkv > 16)
    return fail(PKV_ERR_UNSUPPORTED_SHAPE,
                f + ": num_q_heads must be a multiple of num_kv_heads, with at most 16 query "
                    "heads per kv head");
  if (num_seqs < 0 || max_seq_len < 0 || max_blocks < 0)
    return fail(PKV_ERR_INVALID_ARG, f + ": negative size");
  if (num_seqs == 0) return ok();
  if (q == nullptr || out == nullptr || block_tables == nullptr || seq_lens == nullptr)
    return fail(PKV_ERR_INVALID_ARG, f + ": NULL pointer");
  if (!aligned16(q) || !aligned16(out))
    return fail(PKV_ERR_INVALID_ARG, f + ": q / out must be 16-byte aligned");
  if (max_seq_len == 0 || max_blocks == 0)
    return fail(PKV_ERR_INVALID_ARG, f + ": max_seq_len, max_blocks must be > 0");
  if ((int64_t)max_blocks * kSupportedBlockSize < max_seq_len)
    return fail(PKV_ERR_INVALID_ARG, f + ": max_seq_len exceeds max_blocks * block_size");
  if (max_seq_len > (1 << 30)) return fail(PKV_ERR_INVALID_ARG, f + ": max_seq_len above 2^30");
  if (!(scale > 0.f)) return fail(PKV_ERR_INVALID_ARG, f + ": scale <= 0");
  if ((int64_t)num_seqs * view.hkv > kMaxRowItems)
    return fail(PKV_ERR_INVALID_ARG, f + ": 2^22 sequences x kv heads or more");
  const size_t need = quant_decode_workspace_bytes(num_seqs, num_q_heads, view.hkv, view.head_dim,
                                                   view.bits, max_seq_len);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need || !aligned16(workspace)))
    return fail(PKV_ERR_INVALID_ARG,
                f + ": workspace missing, too small or not 16-byte aligned "
                    "(see pkv_quant_decode_workspace_bytes)");
  const hipStream_t s = static_cast<hipStream_t>(stream);
  {
    // (a length of 0 is in order here)
    MetaCheck c = meta(kMetaRows, shape_of(view), block_tables, max_blocks, seq_lens, nullptr,
                       num_seqs, -1, max_seq_len, 0);
    c.table_rows = num_seqs;
    if ((st = check_metadata(fn, &c, 1, s)) != PKV_OK) return st;
  }
  QuantDecodeArgs a{};
  a.cache = view.cache;
  a.q = static_cast<const uint16_t*>(q);
  a.tables = block_tables;
  a.seq_lens = seq_lens;
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.max_blocks = max_blocks;
  a.num_seqs = num_seqs;
  a.max_len = max_seq_len;
  a.hq = num_q_heads;
  a.hkv = view.hkv;
  a.num_blocks = view.num_blocks;
  a.scale_log2 = scale * 1.44269504088896340736f;
  return launched(launch_quant_decode(a, view.head_dim, view.bits, workspace, s), fn);
}

size_t pkv_quant_prefill_workspace_bytes(int32_t num_seqs, int32_t total_new, int32_t num_q_heads,
                                         int32_t num_kv_heads, int32_t head_dim, int32_t bits,
                                         int32_t max_new_len, int32_t max_total_len) {
  if ((bits != 4 && bits != 8) || (head_dim != 64 && head_dim != 128) || max_total_len <= 0) return 0;
  return quant_prefill_workspace_bytes(num_seqs, total_new, num_q_heads, num_kv_heads, head_dim,
                                       max_new_len, max_total_len);
}

pkv_status pkv_quant_prefill_attention(const pkv_quant_kv* kv, const void* q, int32_t num_q_heads,
                                       const int32_t* block_tables, int32_t max_blocks,
                                       const int32_t* cached_lens, const int32_t* cu_new_lens,
                                       int32_t num_seqs, int32_t total_new, int32_t max_new_len,
                                       int32_t max_total_len, float scale, void* out, float* lse,
                                       void* workspace, size_t workspace_bytes, void* stream) {
  const char* fn = "pkv_quant_prefill_attention";
  QuantView view;
  pkv_status st = check_quant(kv, fn, &view);
  if (st != PKV_OK) return st;
  const KvView shape = shape_of(view);
  bool empty = false;
  st = check_prefill(shape, fn, q, num_q_heads, block_tables, max_blocks, cached_lens, cu_new_lens,
                     num_seqs, total_new, max_new_len, max_total_len, scale, out, nullptr, 0, &empty);
  if (st != PKV_OK || empty) return st;
  const size_t need = quant_prefill_workspace_bytes(num_seqs, total_new, num_q_heads, view.hkv,
                                                    view.head_dim, max_new_len, max_total_len);
  if (need > 0 && workspace != nullptr && (workspace_bytes < need || !aligned16(workspace)))
    return fail(PKV_ERR_INVALID_ARG,
                std::string(fn) + ": workspace too small or not 16-byte aligned (see "
                                  "pkv_quant_prefill_workspace_bytes; NULL runs without the plan)");
  if (max_total_len > (1 << 30))
    return fail(PKV_ERR_INVALID_ARG, std::string(fn) + ": max_total_len above 2^30");
  const hipStream_t s = static_cast<hipStream_t>(stream);
  {
    const MetaCheck c = meta(kMetaPrefill, shape, block_tables, max_blocks, cached_lens, cu_new_lens,
                             num_seqs, total_new, max_new_len, max_total_len);
    if ((st = check_metadata(fn, &c, 1, s)) != PKV_OK) return st;
  }
  const bool plan = workspace != nullptr && need > 0;
  return launched(launch_quant_prefill(view.cache, view.num_blocks, view.hkv, view.head_dim,
                                       view.bits, static_cast<const uint16_t*>(q), num_q_heads,
                                       block_tables, max_blocks, cached_lens, cu_new_lens, num_seqs,
                                       total_new, max_new_len, max_total_len, scale,
                                       static_cast<uint16_t*>(out), lse, plan ? workspace : nullptr,
                                       s),
                  fn);
}

}  // extern "C"
