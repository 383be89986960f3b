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

}  // namespace gift
