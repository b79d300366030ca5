// Internal launch entry points of the gfx950 kernels (called by api.cpp after argument
// validation). Every pointer is device memory; every size was checked on the host.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "decode_cut.h"

namespace pkv {

struct KvView {
  uint16_t* k;  // bf16 [num_blocks][hkv][D/8][16][8]
  uint16_t* v;  // bf16 [num_blocks][hkv][D][16]
  int32_t num_blocks;
  int32_t hkv;
  int32_t head_dim;
};

hipError_t launch_kv_append(const KvView& kv, const uint16_t* k_new, const uint16_t* v_new,
                            const int32_t* block_tables, int32_t max_blocks,
                            const int32_t* cached_lens, const int32_t* cu_new_lens,
                            int32_t num_seqs, int32_t max_new_len, hipStream_t stream);

hipError_t launch_gather_kv(const KvView& kv, const int32_t* block_tables, int32_t max_blocks,
                            const int32_t* lens, const int32_t* cu_lens, int32_t num_seqs,
                            int32_t max_len, uint16_t* k_out, uint16_t* v_out,
                            hipStream_t stream);

// A step's block tables and row metadata (pkv_extend_tables). seq_lens may be cached_lens and
// free_used_out free_used: each is read before it is written.
struct ExtendArgs {
  int32_t* tables;
  int32_t max_blocks;
  const int32_t* cached_lens;
  const int32_t* new_lens;
  int32_t num_seqs;
  const int32_t* free_blocks;
  int32_t num_free;
  const int32_t* free_used;
  int32_t* free_used_out;
  int32_t* cu_new_lens;
  int32_t* seq_lens;
  int32_t* status;
  int32_t max_rows;
  int64_t* slot_map;   // these four: [max_rows], or null
  int32_t* row_seq;
  int32_t* positions;
  int32_t* row_lens;
};
hipError_t launch_extend_tables(const ExtendArgs& a, hipStream_t stream);

// Rotary positions and append (pkv_rope_append). Strides are in elements (rows of q, k, v and
// q_out, axes of positions); turns[j] = inv_freq[j] / (2 pi).
struct RopeArgs {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* q_out;
  uint16_t* k_cache;
  uint16_t* v_cache;
  const int64_t* slot_map;
  const int32_t* positions;
  int64_t q_stride, k_stride, v_stride, q_out_stride, pos_stride;
  int64_t rows;
  int32_t hq, hkv, num_blocks, rot_dim, interleaved;
  int32_t window;  // log2 of a workgroup's rows (set by the launch)
  float scale;
  uint8_t axis_of[64];
  double turns[64];
};
hipError_t launch_rope_append(RopeArgs a, int head_dim, hipStream_t stream);

// Key bounds of the blocks that hold new tokens (pkv_block_bounds).
hipError_t launch_block_bounds(const KvView& kv, uint16_t* bounds, const int32_t* block_tables,
                               int32_t max_blocks, const int32_t* cached_lens,
                               const int32_t* cu_new_lens, int32_t num_seqs, int32_t max_new_len,
                               hipStream_t stream);

// The choice of blocks (pkv_select_blocks). Workspace, in floats: two halves of a 64-bit key per
// (row, kv head, block) (the first is the 32-bit score before), then the largest |bound| per
// most_step * 16 blocks.
constexpr int32_t kSelectMaxBlocks = 65536;  // blocks of a row
struct SelectArgs {
  const uint16_t* bounds;
  const uint16_t* q;
  const int32_t* tables;
  const int32_t* row_seq;  // null: row i is sequence i
  const int32_t* row_lens;
  int32_t* sel;
  int64_t rows;
  int32_t max_blocks, num_seqs, max_len, hq, hkv, num_blocks, blocks, sink, recent;
  int64_t stride;  // of a (row, kv head), in blocks (set by the launch, like the rest)
  int32_t most_step;  // tiles of 16 blocks that an entry of tile_most speaks for
  float* scores;
  float* low;
  float* tile_most;
};
size_t select_workspace_bytes(int64_t items, int32_t max_len, int32_t blocks);
hipError_t launch_select_blocks(SelectArgs a, int head_dim, void* workspace, hipStream_t stream);

// Attention over chosen blocks (pkv_sparse_attention).
struct SparseArgs {
  const uint16_t* k_cache;
  const uint16_t* v_cache;
  const uint16_t* q;
  const int32_t* tables;
  const int32_t* row_seq;  // null: row i is sequence i
  const int32_t* row_lens;
  const int32_t* sel;
  uint16_t* out;
  float* lse;  // or null
  int64_t rows;
  int32_t max_blocks, num_seqs, hq, hkv, num_blocks, blocks;
  float scale_log2;
  // set by the launch: a list's cut across workgroups, and the splits' partial results
  int64_t xcd_items;  // items of each XCD's part, or 0: items in order
  int32_t splits, split_entries;
  float* ws_o;
  float* ws_ml;
};
size_t sparse_workspace_bytes(int64_t items, int32_t g, int32_t head_dim, int32_t blocks);
hipError_t launch_sparse_attention(SparseArgs a, int head_dim, void* workspace,
                                   hipStream_t stream);

// A cache held in 8 or 4 bits: uint8 [num_blocks][hkv][quant_slab_bytes]; quant.h has the slab.
size_t quant_slab_bytes(int32_t head_dim, int32_t bits);
struct QuantAppendArgs {
  uint8_t* cache;
  const uint16_t* k;  // rows, k_stride and v_stride elements apart
  const uint16_t* v;
  int64_t k_stride, v_stride, rows;
  const int32_t* tables;
  const int32_t* cached_lens;
  const int32_t* cu_new_lens;
  int32_t max_blocks, hkv, num_blocks;
};
hipError_t launch_quant_append(const QuantAppendArgs& a, int32_t num_seqs, int32_t max_new_len,
                               int head_dim, int bits, hipStream_t stream);
// Pairs (block of the bf16 pool, block of the cache); back: (block of the cache, block of the pool).
struct QuantBlocksArgs {
  uint8_t* cache;
  uint16_t* k_cache;
  uint16_t* v_cache;
  const int32_t* pairs;
  int32_t num_pairs, hkv, num_blocks, pool_blocks;
};
hipError_t launch_quant_blocks(const QuantBlocksArgs& a, bool back, int head_dim, int bits,
                               hipStream_t stream);
struct QuantDecodeArgs {
  const uint8_t* cache;
  const uint16_t* q;
  const int32_t* tables;
  const int32_t* seq_lens;
  uint16_t* out;
  float* lse;  // or null
  int32_t max_blocks, num_seqs, max_len, hq, hkv, num_blocks;
  float scale_log2;
  // set by the launch: keys per split, splits of the longest sequence, the splits' partial results
  int32_t split_keys, splits;
  float* ws_o;
  float* ws_ml;
};
size_t quant_decode_workspace_bytes(int32_t num_seqs, int32_t hq, int32_t hkv, int32_t head_dim,
                                    int32_t bits, int32_t max_len);
hipError_t launch_quant_decode(QuantDecodeArgs a, int head_dim, int bits, void* workspace,
                               hipStream_t stream);
// As launch_prefill, over the cache, with a plan of its own.
size_t quant_prefill_workspace_bytes(int32_t num_seqs, int32_t total_new, int32_t hq, int32_t hkv,
                                     int32_t head_dim, int32_t max_new_len, int32_t max_total_len);
hipError_t launch_quant_prefill(const uint8_t* cache, int32_t num_blocks, int32_t hkv, int32_t head_dim,
                                int32_t bits, const uint16_t* q, int32_t hq,
                                const int32_t* block_tables, int32_t max_blocks,
                                const int32_t* cached_lens, const int32_t* cu_new_lens,
                                int32_t num_seqs, int32_t total_new, int32_t max_new_len,
                                int32_t max_total_len, float scale, uint16_t* out, float* lse,
                                void* workspace, hipStream_t stream);

hipError_t launch_copy_blocks(const KvView& kv, const int32_t* pairs, int32_t num_pairs,
                              hipStream_t stream);

// Prefill plan, from the host arguments only. Key split: a batch whose work items cannot
// fill the chip (few sequences, few new tokens) and whose keys are long has each item's keys
// cut at multiples of split_keys (a multiple of 1024) into nsplit parts, run as separate work
// items and merged; otherwise split_keys = 0 and nsplit = 1. Order: a batch with long keys
// (up to at least 8192) takes its sequences longest first.
struct PrefillSplit {
  int32_t split_keys;
  int32_t nsplit;
  bool order;
};
PrefillSplit prefill_split_plan(int32_t num_seqs, int32_t hq, int32_t hkv, int32_t max_new_len,
                                int32_t max_total_len);
// Workspace of the plan (0 when it needs none): the sequence order when ordered, then when
// split the fp32 partial outputs [total_new][hq][nsplit][head_dim] and their (maximum, weight
// sum) pairs.
size_t prefill_workspace_bytes(int32_t num_seqs, int32_t total_new, int32_t hq, int32_t hkv,
                               int32_t head_dim, int32_t max_new_len, int32_t max_total_len);
// With workspace == nullptr the launch does not split.
hipError_t launch_prefill(const KvView& kv, const uint16_t* q, int32_t hq,
                          const int32_t* block_tables, int32_t max_blocks,
                          const int32_t* cached_lens, const int32_t* cu_new_lens,
                          int32_t num_seqs, int32_t total_new, int32_t max_new_len,
                          int32_t max_total_len, float scale, uint16_t* out, float* lse,
                          void* workspace, hipStream_t stream);

size_t decode_workspace_bytes(int32_t num_seqs, int32_t hq, int32_t hkv, int32_t head_dim,
                              int32_t max_seq_len);
// The pieces of a decode launch, shared with the mixed launch: the cut into work items and the
// workspace layout (the sequence order, then the splits' partial results), the ordering
// kernel, and the merge of partial results (nothing when no sequence splits).
struct DecodePlan : DecodeCut {
  // The launch takes its sequences longest first, by an order written before it (ordered) or
  // by each wave's ranking of the lengths (by_rank; at most 64 sequences).
  bool ordered, by_rank;
  int32_t* order;
  float* ws_o;
  float* ws_ml;
};
DecodePlan decode_plan(const KvView& kv, int32_t hq, int32_t num_seqs, int32_t max_seq_len,
                       int32_t max_blocks, void* workspace);
// (nothing when the plan does not order)
hipError_t launch_decode_order(const DecodePlan& p, const int32_t* seq_lens, int32_t num_seqs,
                               hipStream_t stream);
// Longest-first order of sequences by lens[i] (+ cu[i + 1] - cu[i] when cu is given), and the
// bytes it takes in a workspace (256-byte rounded).
hipError_t launch_seq_order(const int32_t* lens, const int32_t* cu, int32_t num_seqs,
                            int32_t* order, hipStream_t stream);
size_t order_bytes(int32_t num_seqs);
hipError_t launch_decode_merge(const KvView& kv, const DecodePlan& p, int32_t hq,
                               const int32_t* seq_lens, int32_t num_seqs, uint16_t* out,
                               float* lse, hipStream_t stream);
hipError_t launch_decode(const KvView& kv, const uint16_t* q, int32_t hq,
                         const int32_t* block_tables, int32_t max_blocks,
                         const int32_t* seq_lens, int32_t num_seqs, int32_t max_seq_len,
                         float scale, uint16_t* out, float* lse, void* workspace,
                         hipStream_t stream);

// The allocation-free decode's workspace (a file-scope device array of kDecodeScratchBytes):
// its address on the current device, looked up on the first call per device.
constexpr size_t kDecodeScratchBytes = size_t(32) << 20;
hipError_t decode_scratch(void** ptr);

// Opt-in metadata validation (PKV_DEBUG_VALIDATE). One check per batch of a call: for
// append / prefill, `lens` are the cached lengths and `cu` the new-token offsets (ending at
// `total`), each sequence's new tokens at most `max_len` and cached + new at most
// `max_total`; for decode, `lens` are the sequence lengths (1 .. max_len); for gather, `lens`
// the gathered lengths (at most max_len, equal to the cu steps). Every table entry the call
// reads or writes must name a pool block. For slots and
// rows, a row stands where a sequence does.
enum : int32_t { kMetaAppend = 0, kMetaPrefill = 1, kMetaDecode = 2, kMetaGather = 3,
                 kMetaSlots = 4, kMetaRows = 5 };
enum : uint32_t { kMetaBadBlockId = 1u, kMetaBadLength = 2u, kMetaBadOffsets = 4u,
                  kMetaBadSlot = 8u };
struct MetaCheck {
  int32_t mode;
  const int32_t* tables;
  int32_t max_blocks;
  int32_t num_blocks;
  const int32_t* lens;
  const int32_t* cu;  // null for decode
  int32_t num_seqs;
  int64_t total;      // cu[num_seqs] must equal it (< 0: not checked)
  int64_t max_len;
  int64_t max_total;
  const int64_t* slots;  // kMetaSlots: [num_seqs] rows' slots, each -1 or within the pool
  const int32_t* row_seq;  // kMetaRows: [num_seqs] rows' sequences, each -1 or below table_rows
  int32_t table_rows;      // (null: row i is sequence i), lens their visible keys (0 .. max_len);
                           // tables null: their entries are not looked at
};
// Runs the checks in order on `stream` and waits for each; *bad = the failed check's bits
// (0 if all pass), *first_seq its lowest offending sequence, *which its index.
hipError_t validate_metadata(const MetaCheck* checks, int n_checks, hipStream_t stream,
                             uint32_t* bad, int32_t* first_seq, int32_t* which);

// Mixed launch: a prefill batch (arguments as launch_prefill) and a decode batch (d_*, as
// launch_decode, with its workspace) in one fused kernel between the decode's ordering
// kernel and its merge. Both batches must be non-empty.
hipError_t launch_mixed(const KvView& kv, int32_t hq, float scale, const uint16_t* q,
                        const int32_t* block_tables, int32_t max_blocks,
                        const int32_t* cached_lens, const int32_t* cu_new_lens, int32_t num_seqs,
                        int32_t max_new_len, uint16_t* out, float* lse, const uint16_t* dq,
                        const int32_t* d_block_tables, int32_t d_max_blocks,
                        const int32_t* seq_lens, int32_t d_num_seqs, int32_t max_seq_len,
                        uint16_t* d_out, float* d_lse, void* workspace, hipStream_t stream);

}  // namespace pkv
