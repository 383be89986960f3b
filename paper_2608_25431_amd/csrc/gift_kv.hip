// Kernels of include/gift_kv.h: block tables and slot maps, rows into the
// paged cache, attention of drafted tokens over it.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gift_kv_attention.hpp"
#include "gift_kv_internal.hpp"

namespace gift {
namespace {

// ---------------------------------------------------------------------------
// Block tables and slot maps
// ---------------------------------------------------------------------------

// What request b asks for: blocks that hold its cached tokens, blocks with its
// new ones, and blocks to take (none where its table row is too short).
struct Ask {
  uint32_t len, add, have, want, need;
  bool fits;
};

__device__ inline Ask ask_of(const TablesArgs& a, uint32_t b) {
  Ask k;
  k.len = a.s.lens[b];
  k.add = a.s.new_lens[b];
  const uint64_t round = a.s.block_tokens - 1;
  const uint64_t have = ((uint64_t)k.len + round) >> a.block_shift,
                 want = ((uint64_t)k.len + k.add + round) >> a.block_shift;
  k.fits = want <= a.s.table_width;
  k.have = (uint32_t)have;
  k.want = (uint32_t)want;
  k.need = k.fits ? (uint32_t)(want - have) : 0u;
  return k;
}

// The label that block id had.
__device__ inline uint32_t claim(const TablesArgs& a, uint32_t id, uint32_t user) {
  uint32_t label = GIFT_LABEL_UNOWNED;
  __hip_atomic_compare_exchange_strong(a.s.block_labels + id, &label, user, __ATOMIC_RELAXED, __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT);
  return label;
}

__device__ inline void disown(const TablesArgs& a, uint32_t id) {
  __hip_atomic_store(a.s.block_labels + id, GIFT_LABEL_UNOWNED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

struct Sums {
  uint64_t blocks, rows;
};

__device__ inline Sums operator+(Sums x, Sums y) { return Sums{x.blocks + y.blocks, x.rows + y.rows}; }

__device__ inline Sums shfl_up(Sums v, int d) {
  return Sums{__shfl_up((unsigned long long)v.blocks, d), __shfl_up((unsigned long long)v.rows, d)};
}

// Inclusive running sums over the workgroup's threads; *all gets the total.
template <int T>
__device__ Sums scan(Sums v, Sums* lds, Sums* all) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const Sums u = shfl_up(v, d);
    if (lane >= d) v = v + u;
  }
  if (lane == kWave - 1) lds[wave] = v;
  __syncthreads();
  Sums before{0, 0}, total{0, 0};
#pragma unroll
  for (int w = 0; w < T / kWave; w++) {
    const Sums x = lds[w];
    if (w < wave) before = before + x;
    total = total + x;
  }
  __syncthreads();
  *all = total;
  return before + v;
}

// TPR threads serve a request, T make a workgroup.  Which blocks a request
// takes and where its rows start are running sums over the requests before
// it; every workgroup sums those itself (8 B of L2-resident lengths per
// request), so that one launch suffices.  Bound by latency: lengths, ids, labels
// and slots wait for each other (1024 requests of 128-2048 tokens 6.1 us, 32 of
// up to 131072 tokens 9.7 us, of which a launch that does nothing is about 4;
// about 0.6 us of it is the claim of new blocks).
// Workgroup 0 writes what belongs to no single request: the row ranges, the
// count of taken blocks and the slots past the last row.
template <int TPR, int T>
__global__ __launch_bounds__(T) void k_kv_tables(TablesArgs a) {
  __shared__ Sums lds[T / kWave];
  __shared__ uint32_t flags[T / TPR];
  const uint32_t n = a.s.n_reqs, tid = threadIdx.x;
  if (blockIdx.x == 0) {
    Sums carry{0, 0}, all;
    uint64_t taken = 0;
    if (tid == 0) a.s.row_begin[0] = 0;
    for (uint32_t base = 0; base < n; base += T) {
      const uint32_t b = base + tid;
      Sums own{0, 0};
      uint32_t need = 0;
      if (b < n) {
        const Ask k = ask_of(a, b);
        need = k.need;
        own = Sums{k.need, k.add};
      }
      const Sums upto = carry + scan<T>(own, lds, &all);
      if (b < n) {
        a.s.row_begin[b + 1] = (uint32_t)(upto.rows < a.s.n_slots ? upto.rows : a.s.n_slots);
        if (need && upto.blocks <= a.s.n_free && upto.rows <= a.s.n_slots) taken = upto.blocks;
      }
      carry = carry + all;
    }
    // a thread's last granted request is its furthest; the largest of all of them counts
#pragma unroll
    for (int d = kWave / 2; d; d /= 2) {
      const uint64_t o = __shfl_xor((unsigned long long)taken, d);
      taken = o > taken ? o : taken;
    }
    if (tid % kWave == 0) lds[tid / kWave].blocks = taken;
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < T / kWave; w++) taken = lds[w].blocks > taken ? lds[w].blocks : taken;
      a.s.taken[0] = (uint32_t)taken;
    }
    for (uint64_t r = carry.rows + tid; r < a.s.n_slots; r += T) a.s.slots[r] = -1;
    return;
  }
  constexpr uint32_t kPer = T / TPR;
  const uint32_t first = (blockIdx.x - 1) * kPer, group = tid / TPR, lane = tid % TPR, b = first + group;
  // lengths of the requests before these, on their way while the tables are read
  Sums mine{0, 0}, before;
#pragma unroll 4
  for (uint32_t p = tid; p < first; p += T) {
    const Ask k = ask_of(a, p);
    mine = mine + Sums{k.need, k.add};
  }
  if (lane == 0) flags[group] = 0;
  Ask k{};
  uint32_t user = 0, bad = 0;
  uint32_t* row = nullptr;
  if (b < n) {
    k = ask_of(a, b);
    user = a.s.users[b];
    if (user >= GIFT_LABEL_PARAM) bad = 1;  // no user: what these labels stand for is nobody's
    row = a.s.tables + (uint64_t)b * a.s.table_stride;
    // owner check of the blocks that hold tokens, eight in flight per thread
    const uint32_t have = k.have < a.s.table_width ? k.have : a.s.table_width;
    for (uint32_t j = lane; j < have; j += 8 * TPR) {
      uint32_t id[8], label[8];
#pragma unroll
      for (int u = 0; u < 8; u++) {
        const uint32_t at = j + u * TPR;
        id[u] = row[at < have ? at : j];
      }
#pragma unroll
      for (int u = 0; u < 8; u++) label[u] = id[u] < a.s.n_blocks ? a.s.block_labels[id[u]] : GIFT_LABEL_UNOWNED;
#pragma unroll
      for (int u = 0; u < 8; u++) bad |= (id[u] >= a.s.n_blocks || label[u] != user) ? 1u : 0u;
    }
  }
  scan<T>(mine, lds, &before);
  bool granted = false;
  uint32_t claimed = lane;  // this thread has claimed blocks lane, lane + TPR, ... below this one
  const uint32_t* from = nullptr;
  if (b < n) {
    for (uint32_t p = first; p < b; p++) {
      const Ask o = ask_of(a, p);
      before = before + Sums{o.need, o.add};
    }
    granted = user < GIFT_LABEL_PARAM && k.fits && (k.add == 0 || before.rows + k.add <= a.s.n_slots) &&
              (k.need == 0 || before.blocks + k.need <= a.s.n_free);
    from = a.s.free_blocks + before.blocks;  // read only where granted
    // A block is claimed by swapping its label from unowned to the user, so that no two users get it and none gets what
    // another owns, whatever the free list holds; four in flight per thread.  One that has the user's label already may
    // be taken (a step may be run again) but is not given back with the others if the request is refused: the slots of
    // the request's rows, at least one a block and each written by one thread, hold which is which until they are known.
    if (granted)
      for (; claimed < k.need; claimed += 4 * TPR) {
        uint32_t id[4], label[4];
        bool all = true;
#pragma unroll
        for (int u = 0; u < 4; u++) id[u] = claimed + u * TPR < k.need ? from[claimed + u * TPR] : 0;
#pragma unroll
        for (int u = 0; u < 4; u++) {
          label[u] = user;  // as it was found
          if (claimed + u * TPR < k.need) label[u] = id[u] < a.s.n_blocks ? claim(a, id[u], user) : GIFT_LABEL_PARAM;
        }
#pragma unroll
        for (int u = 0; u < 4; u++) all = all && (label[u] == GIFT_LABEL_UNOWNED || label[u] == user);
        if (!all) {
#pragma unroll
          for (int u = 0; u < 4; u++)
            if (label[u] == GIFT_LABEL_UNOWNED) disown(a, id[u]);
          bad |= 2u;
          break;
        }
#pragma unroll
        for (int u = 0; u < 4; u++)
          if (claimed + u * TPR < k.need) a.s.slots[before.rows + claimed + u * TPR] = label[u] == GIFT_LABEL_UNOWNED;
      }
    if (bad) atomicOr(&flags[group], bad);
  }
  __syncthreads();
  if (b >= n) return;
  bad = flags[group];
  if (granted && (bad & 2u)) {
    granted = false;
    for (uint32_t j = lane; j < k.need && j < claimed; j += TPR)
      if (a.s.slots[before.rows + j]) disown(a, from[j]);
  }
  const int32_t verdict = (bad & 1u) ? GIFT_SEG_OWNER_MIXED : granted ? GIFT_SEG_OK : GIFT_SEG_NO_SPACE;
  if (granted)
    for (uint32_t j = lane; j < k.need; j += TPR) row[k.have + j] = from[j];
  if (lane == 0) {
    a.s.verdicts[b] = verdict;
    a.s.lens_out[b] = verdict == GIFT_SEG_OK ? k.len + k.add : k.len;
  }
  for (uint32_t i = lane; i < k.add; i += TPR) {
    const uint64_t r = before.rows + i;
    if (r >= a.s.n_slots) break;
    int64_t slot = -1;
    if (verdict == GIFT_SEG_OK) {
      const uint32_t pos = k.len + i, at = pos >> a.block_shift;
      const uint32_t id = at < k.have ? row[at] : from[at - k.have];
      slot = ((int64_t)id << a.block_shift) + (pos & (a.s.block_tokens - 1));
    }
    a.s.slots[r] = slot;
  }
}

// ---------------------------------------------------------------------------
// Rows into the cache
// ---------------------------------------------------------------------------

// A thread copies 16 bytes of K and of V of one row; rows, heads and pieces in
// the order in which the sources have them, layers along the grid's second
// dimension.  Bound by memory: 2.2 GB of prompts (16 requests, 32 layers of 8
// heads of 128 elements) take 0.79 ms, 5.5 TB/s read and written together.
__global__ __launch_bounds__(256) void k_kv_append(AppendArgs a) {
  const uint32_t units = a.kv.head_dim / 8, per_row = units * a.kv.heads;  // 16 B each
  const uint64_t total = (uint64_t)a.n_slots * per_row;
  for (uint32_t layer = blockIdx.y; layer < a.kv.n_layers; layer += gridDim.y)
    for (uint64_t u = (uint64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += (uint64_t)gridDim.x * 256) {
      const uint32_t i = (uint32_t)(u / per_row), w = (uint32_t)(u - (uint64_t)i * per_row), h = w / units, c = w - h * units;
      const int64_t slot = a.slots[i];
      const uint64_t src = a.index ? a.index[i] : i;
      if (slot < 0 || (uint64_t)slot >> a.kv.block_shift >= a.kv.n_blocks || src >= a.src.n_rows) continue;
      const uint4 k = *(const uint4*)((const uint8_t*)a.src.k + layer * a.src.k_layer_stride + src * a.src.k_row_stride +
                                      h * a.src.k_head_stride + c * 16);
      const uint4 v = *(const uint4*)((const uint8_t*)a.src.v + layer * a.src.v_layer_stride + src * a.src.v_row_stride +
                                      h * a.src.v_head_stride + c * 16);
      uint8_t* to = a.kv.base + layer * a.kv.layer_stride + ((uint64_t)slot >> a.kv.block_shift) * a.kv.block_stride +
                    ((uint64_t)slot & ((1ull << a.kv.block_shift) - 1)) * a.kv.token_stride + h * a.kv.head_stride + c * 16;
      *(uint4*)to = k;
      *(uint4*)(to + a.kv.v_off) = v;
    }
}

}  // namespace

hipError_t launch_kv_tables(const TablesArgs& a, hipStream_t s) {
  const uint32_t n = a.s.n_reqs;
  // threads per request, by the entries and slots that one may have
  const uint64_t per = n ? a.s.table_width + a.s.n_slots / n : 0;
  if (per <= 256)
    k_kv_tables<64, 256><<<1 + (n + 3) / 4, 256, 0, s>>>(a);
  else if (per <= 2048)
    k_kv_tables<256, 256><<<1 + n, 256, 0, s>>>(a);
  else
    k_kv_tables<1024, 1024><<<1 + n, 1024, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_kv_append(const AppendArgs& a, hipStream_t s) {
  const uint64_t units = (uint64_t)a.n_slots * a.kv.heads * (a.kv.head_dim / 8);
  const uint64_t blocks = (units + 255) / 256;
  k_kv_append<<<dim3((uint32_t)(blocks < 65536 ? blocks : 65536), a.kv.n_layers < 65535 ? a.kv.n_layers : 65535), 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_tree_attention(const AttnArgs& a, uint32_t dtype, const AttnWork& w, hipStream_t s) {
  return dtype == GIFT_BF16 ? attend_by_dim<Bf16>(a, w, s) : attend_by_dim<F16>(a, w, s);
}

}  // namespace gift
