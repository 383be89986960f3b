// Types shared by the host side (gift_kv_host.cpp) and the kernels
// (gift_kv.hip) of include/gift_kv.h.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gift_kv.h"

namespace gift {

// Error reporting and the geometry rules of gift_host.cpp.
void clear_error() noexcept;
gift_status report(gift_status s, const char* message) noexcept;
gift_status report_hip(hipError_t e, const char* what) noexcept;
gift_status paged_geometry(const gift_paged_kv* kv) noexcept;

// Where K and V of a layer's (block, token, head) lie.
struct KvView {
  uint8_t* base;  // of K of block 0, token 0, head 0 (append: of layer 0)
  int64_t v_off;  // from K to V
  uint64_t layer_stride, block_stride, token_stride, head_stride;
  uint64_t n_blocks;
  uint32_t n_layers, heads, head_dim, block_shift;
};

struct TablesArgs {
  gift_kv_step s;
  uint32_t block_shift;
};
hipError_t launch_kv_tables(const TablesArgs& a, hipStream_t s);

struct AppendArgs {
  KvView kv;
  gift_kv_rows src;
  const int64_t* slots;
  const uint32_t* index;
  uint32_t n_slots;
};
hipError_t launch_kv_append(const AppendArgs& a, hipStream_t s);

struct AttnArgs {
  KvView kv;
  gift_tree_attention_args a;
  uint32_t group;  // query heads of a KV head
};
// The same over a quantised cache: kv is of its elements, of one byte each, and the drafted rows of `a` are NULL.
struct QuantAttnArgs : AttnArgs {
  KvView scales;
  uint32_t most_wg;  // workgroups that columns are divided among; there may be more where they stay whole
};
// The attention's workspace: counters of the columns that are joined and of
// runs of their parts (zero between calls: the workgroup that counts a last
// part clears the counter), a quarter and a half of them, then two places per
// workgroup for a column's part.  The largest ones are those of a workgroup per
// CU with 8 waves of 32 columns of 128 elements and their maxima and sums.
constexpr uint32_t kAttnCounters = 16384;
constexpr size_t kAttnPlace = 8 * (128 * 32 * 4 + 1024);
struct AttnWork {
  uint8_t* mem;
  uint32_t cus;
  size_t partial_bytes;  // past the counters
};
hipError_t launch_tree_attention(const AttnArgs& a, uint32_t dtype, const AttnWork& w, hipStream_t s);
hipError_t launch_quant_attention(const QuantAttnArgs& a, uint32_t dtype, const AttnWork& w, hipStream_t s);

// How a call is cut by rows: those of a workgroup of 256 threads, workgroups that share them (their heads,
// or layers), and rows of a launch.
struct RowsPlan {
  uint32_t rows, parts, launch;
};
RowsPlan qk_norm_rope_plan(const gift_qk_rows& a);
hipError_t launch_qk_norm_rope(const gift_qk_rows& a, hipStream_t s);

struct QuantAppendArgs {
  KvView kv, scales;  // bases: of layer 0
  gift_kv_rows src;
  const int64_t* slots;
  const uint32_t* index;
  uint32_t n_slots, layer, n_layers;
};
hipError_t launch_kv_append_quant(const QuantAppendArgs& a, uint32_t dtype, hipStream_t s);

struct QuantReadArgs {
  KvView kv, scales;
  gift_kv_read_args a;
  uint64_t row0;  // the first row of a launch
};
RowsPlan kv_read_quant_plan(const gift_kv_read_args& a);
hipError_t launch_kv_read_quant(const QuantReadArgs& a, hipStream_t s);

}  // namespace gift
