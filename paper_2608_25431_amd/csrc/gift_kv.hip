// Kernels of include/gift_kv.h: block tables and slot maps, rows into the
// paged cache, attention of drafted tokens over it.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gift_kv_internal.hpp"

namespace gift {
namespace {

constexpr int kWave = 64;

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
// it; every workgroup sums those itself (12 B of L2-resident lengths per
// request), so that one launch suffices.  Workgroup 0 writes what belongs to
// no single request: the row ranges, the count of taken blocks and the slots
// past the last row.
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
        if (need && upto.blocks <= a.s.n_free) taken = upto.blocks;
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
  const uint32_t first = (blockIdx.x - 1) * kPer, group = tid / TPR, lane = tid % TPR;
  Sums mine{0, 0}, before;
  for (uint32_t b = tid; b < first; b += T) {
    const Ask k = ask_of(a, b);
    mine = mine + Sums{k.need, k.add};
  }
  scan<T>(mine, lds, &before);
  const uint32_t b = first + group;
  if (lane == 0) flags[group] = 0;
  __syncthreads();
  Ask k{};
  uint32_t user = 0, bad = 0;
  bool granted = false;
  uint32_t* row = nullptr;
  const uint32_t* from = nullptr;
  if (b < n) {
    for (uint32_t p = first; p < b; p++) {
      const Ask o = ask_of(a, p);
      before = before + Sums{o.need, o.add};
    }
    k = ask_of(a, b);
    user = a.s.users[b];
    row = a.s.tables + (uint64_t)b * a.s.table_stride;
    granted = k.fits && (k.need == 0 || before.blocks + k.need <= a.s.n_free);
    from = a.s.free_blocks + before.blocks;  // read only where granted
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
    if (granted)
      for (uint32_t j = lane; j < k.need; j += TPR) bad |= from[j] >= a.s.n_blocks ? 2u : 0u;
    if (bad) atomicOr(&flags[group], bad);
  }
  __syncthreads();
  if (b >= n) return;
  bad = flags[group];
  granted = granted && !(bad & 2u);
  const bool room = before.rows + k.add <= a.s.n_slots;
  const int32_t verdict = (bad & 1u) ? GIFT_SEG_OWNER_MIXED : (granted && room) ? GIFT_SEG_OK : GIFT_SEG_NO_SPACE;
  if (granted)
    for (uint32_t j = lane; j < k.need; j += TPR) {
      const uint32_t id = from[j];
      row[k.have + j] = id;
      a.s.block_labels[id] = user;
    }
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

__global__ __launch_bounds__(256) void k_kv_append(AppendArgs a) {
  const uint32_t units = a.kv.head_dim / 8, per_row = units * a.kv.heads;  // 16 B each
  const uint32_t layer = blockIdx.y;
  const uint64_t total = (uint64_t)a.n_slots * per_row;
  for (uint64_t u = (uint64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += (uint64_t)gridDim.x * 256) {
    const uint32_t i = (uint32_t)(u / per_row), w = (uint32_t)(u % per_row), h = w / units, c = w % units;
    const int64_t slot = a.slots[i];
    const uint64_t src = a.index ? a.index[i] : i;
    if (slot < 0 || (uint64_t)slot >> a.kv.block_shift >= a.kv.n_blocks || src >= a.src.n_rows) continue;
    const uint4 k = *(const uint4*)((const uint8_t*)a.src.k + layer * a.src.k_layer_stride + src * a.src.k_row_stride +
                                    h * a.src.k_head_stride + c * 16);
    const uint4 v = *(const uint4*)((const uint8_t*)a.src.v + layer * a.src.v_layer_stride + src * a.src.v_row_stride +
                                    h * a.src.v_head_stride + c * 16);
    uint8_t* to = a.kv.base + layer * a.kv.layer_stride + ((uint64_t)slot >> a.kv.block_shift) * a.kv.block_stride +
                  ((uint64_t)slot & ((1ull << a.kv.block_shift) - 1)) * a.kv.token_stride + h * a.kv.head_stride +
                  c * 16;
    *(uint4*)to = k;
    *(uint4*)(to + a.kv.v_off) = v;
  }
}

// ---------------------------------------------------------------------------
// Attention
// ---------------------------------------------------------------------------

struct Bf16 {
  __device__ static float up(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
  __device__ static uint16_t down(float f) {
    const __bf16 b = (__bf16)f;
    return __builtin_bit_cast(uint16_t, b);
  }
};
struct F16 {
  __device__ static float up(uint16_t x) { return (float)__builtin_bit_cast(_Float16, x); }
  __device__ static uint16_t down(float f) { return __builtin_bit_cast(uint16_t, (_Float16)f); }
};

template <class E>
__device__ float dot8(uint4 x, uint4 y) {
  const uint32_t* p = (const uint32_t*)&x;
  const uint32_t* q = (const uint32_t*)&y;
  float s = 0;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    s += E::up((uint16_t)p[i]) * E::up((uint16_t)q[i]);
    s += E::up((uint16_t)(p[i] >> 16)) * E::up((uint16_t)(q[i] >> 16));
  }
  return s;
}

// One wave per (row, query head).  A lane scores one key of 64 at a time, then
// the wave adds the keys' V rows, each lane head_dim / 64 elements.
template <class E>
__global__ __launch_bounds__(256) void k_attention_plain(AttnArgs p) {
  const gift_tree_attention_args& a = p.a;
  const uint64_t unit = (uint64_t)blockIdx.x * 4 + threadIdx.x / kWave;
  const uint32_t lane = threadIdx.x % kWave;
  if (unit >= a.n_rows * a.n_heads) return;
  const uint32_t r = (uint32_t)(unit / a.n_heads), h = (uint32_t)(unit % a.n_heads), g = h / p.group;
  const uint32_t D = p.kv.head_dim;
  uint32_t b = a.n_reqs, r0 = 0, r1 = 0;
  for (uint32_t i = 0; i < a.n_reqs; i++)
    if (r >= a.row_begin[i] && r < a.row_begin[i + 1]) {
      b = i;
      break;
    }
  float m = -INFINITY, l = 0, acc[4] = {0, 0, 0, 0};
  if (b < a.n_reqs && (!a.verdicts || a.verdicts[b] == GIFT_SEG_OK)) {
    r0 = a.row_begin[b];
    r1 = a.row_begin[b + 1] < a.n_rows ? a.row_begin[b + 1] : (uint32_t)a.n_rows;
    const uint32_t most = a.table_width << p.kv.block_shift, len = a.lens[b] < most ? a.lens[b] : most;
    const uint32_t n = a.k ? r1 - r0 : 0;
    const uint8_t* q = (const uint8_t*)a.q + r * a.q_row_stride + h * a.q_head_stride;
    for (uint32_t j0 = 0; j0 < len + n; j0 += kWave) {
      const uint32_t j = j0 + lane;
      const uint8_t *kp = nullptr, *vp = nullptr;
      if (j < len) {
        const uint32_t id = a.tables[b * a.table_stride + (j >> p.kv.block_shift)];
        if (id < p.kv.n_blocks) {
          kp = p.kv.base + a.layer * p.kv.layer_stride + id * p.kv.block_stride +
               (j & ((1u << p.kv.block_shift) - 1)) * p.kv.token_stride + g * p.kv.head_stride;
          vp = kp + p.kv.v_off;
        }
      } else if (j < len + n) {
        const uint32_t t = j - len;
        const bool see = a.mask ? t < 32ull * a.mask_words && ((a.mask[(uint64_t)r * a.mask_words + t / 32] >> (t % 32)) & 1)
                                : t <= r - r0;
        if (see) {
          kp = (const uint8_t*)a.k + (r0 + t) * a.k_row_stride + g * a.k_head_stride;
          vp = (const uint8_t*)a.v + (r0 + t) * a.v_row_stride + g * a.v_head_stride;
        }
      }
      float s = -INFINITY;
      if (kp) {
        s = 0;
        for (uint32_t c = 0; c < D / 8; c++) s += dot8<E>(*(const uint4*)(q + 16 * c), *(const uint4*)(kp + 16 * c));
        s *= a.scale;
      }
      float top = s;
      for (int d = 32; d; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
      const float m2 = fmaxf(m, top), safe = m2 == -INFINITY ? 0.f : m2, fix = expf(m - safe);
      const float w = kp ? expf(s - safe) : 0.f;
      float sum = w;
      for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d);
      l = l * fix + sum;
      m = m2;
      for (int i = 0; i < 4; i++) acc[i] *= fix;
      for (int j2 = 0; j2 < kWave; j2++) {
        const uint8_t* row = (const uint8_t*)__shfl((unsigned long long)vp, j2);
        if (!row) continue;
        const float wj = __shfl(w, j2);
#pragma unroll
        for (int i = 0; i < 4; i++)
          if (lane + 64 * i < D) acc[i] += wj * E::up(*(const uint16_t*)(row + 2 * (lane + 64 * i)));
      }
    }
  }
  uint8_t* o = (uint8_t*)a.out + r * a.out_row_stride + h * a.out_head_stride;
#pragma unroll
  for (int i = 0; i < 4; i++)
    if (lane + 64 * i < D)
      *(uint16_t*)(o + 2 * (lane + 64 * i)) = E::down(m == -INFINITY ? 0.f : acc[i] / l);
  if (a.lse && lane == 0) a.lse[(uint64_t)r * a.n_heads + h] = m == -INFINITY ? -INFINITY : m + logf(l);
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
  k_kv_append<<<dim3((uint32_t)(blocks < 65536 ? blocks : 65536), a.kv.n_layers), 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_tree_attention(const AttnArgs& a, uint32_t dtype, hipStream_t s) {
  const uint64_t blocks = (a.a.n_rows * a.a.n_heads + 3) / 4;
  if (blocks > 0x7FFFFFFF) return hipErrorInvalidValue;
  if (dtype == GIFT_BF16)
    k_attention_plain<Bf16><<<(uint32_t)blocks, 256, 0, s>>>(a);
  else
    k_attention_plain<F16><<<(uint32_t)blocks, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace gift
