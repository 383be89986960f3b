// Kernels of include/gift_kv.h: block tables and slot maps, rows into the
// paged cache, attention of drafted tokens over it.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gift_kv_internal.hpp"
#include "gift_kv_units.hpp"

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

// ---------------------------------------------------------------------------
// Attention
// ---------------------------------------------------------------------------

// The rows of a request that read one KV head (its tokens times the query
// heads of the head) form the columns of 32-wide tiles, keys the rows:
//     S^T = K Q^T,   P = exp2(c (S - max)),   O^T += V^T P^T
// on the 32x32x16 matrix instruction.  With keys as rows, a lane holds scores
// of one query only, so the maximum and the sum of a softmax row stay in the
// lane (and its partner 32 lanes on), rescaling O is one factor per lane, and
// the registers that hold P^T are the second product's operand as they are:
// the order of keys in a contraction is free, so V^T is read in the same
// order, four keys at a time, by the transposing LDS read.
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct Bf16 {
  typedef bf16x8 vec;
  typedef __bf16 elem;
  static constexpr uint16_t kExp = 0x7F80;  // exponent bits: all set in NaN and infinities
  // Weights are 8 bits of bfloat16 in two operands, the upper half of the float and what is left of it: with one
  // operand their rounding would add as much error again as the output's own.
  static constexpr int kParts = 2;
  static constexpr float kSlack = 8.f;  // octaves that a score may pass what the weights refer to
  static constexpr float kTop = 0.f;    // octaves by which all weights are raised
  __device__ static void parts(const f32x16& p, int k, vec* w) {
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const uint32_t x = __float_as_uint(p[8 * k + i]);
      w[0][i] = __builtin_bit_cast(elem, (uint16_t)(x >> 16));
      w[1][i] = (elem)(p[8 * k + i] - __uint_as_float(x & 0xFFFF0000u));
    }
  }
  __device__ static f32x16 mfma(vec a, vec b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
struct F16 {
  typedef f16x8 vec;
  typedef _Float16 elem;
  static constexpr uint16_t kExp = 0x7C00;
  // One operand: 11 bits of weights against 11 of the output.  They refer to the maximum itself, whose own weight is then
  // not rounded (8 octaves of slack: errors of 131072 tokens 17% larger, and no faster).  That weight is 2^15, so that the
  // type's range below it is used: 11 bits down to 2^-29 of the maximum's, steps of 2^-39 of it below.  With the maximum's
  // at 1 there would be steps of 2^-24 from 2^-14 on and nothing below 2^-25, while the sum holds weights in 32 bits: beside
  // a key of large score whose V is near 0, the others would lose their part in the output.
  static constexpr int kParts = 1;
  static constexpr float kSlack = 0.f, kTop = 15.f;
  __device__ static void parts(const f32x16& p, int k, vec* w) {
#pragma unroll
    for (int i = 0; i < 8; i++) w[0][i] = (elem)p[8 * k + i];
  }
  __device__ static f32x16 mfma(vec a, vec b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

constexpr int kTileKeys = 32;

// Weights are exp2(c s - c m) by one multiplication and addition, with c m rounded once: off by up to half its last place,
// the same factor for every key until the reference m moves.  From 4096 on (a factor of 1 +- 2^-13) what the rounding left
// out is subtracted; without it, weights of scores past 2^31 would all be 0 or infinite.
constexpr float kFarShift = 4096.f;

// WQ waves share a tile of keys, each with 32 columns of its own; WK groups of
// them take different keys, TK tiles a group in a round.
template <int D_, int WQ_, int WK_, int TK_>
struct Shape {
  static constexpr int D = D_, WQ = WQ_, WK = WK_, TK = TK_;
  static constexpr int kWaves = WQ * WK, kThreads = kWave * kWaves, kTiles = WK * TK;  // per round
  // a wave that shares its tiles with no other needs no second buffer: its LDS accesses are in order
  static constexpr int kBufs = WQ == 1 ? 1 : 2;
  // LDS rows are padded so that the 16-byte reads of K down a column and the transposing reads of V over four rows
  // fall into different banks
  static constexpr int kKRow = 2 * D + 16, kVRow = 2 * D + 32, kTileBytes = kTileKeys * (kKRow + kVRow);
  // a row's 16-byte pieces go to a power of two of lanes (D = 96: 12 of 16 lanes load)
  static constexpr int kPieces = D / 8, kLanes = D <= 64 ? 8 : D <= 128 ? 16 : 32, kRowsAtOnce = kWave / kLanes;
  static constexpr int kLoads = kTileKeys * TK / (kRowsAtOnce * WQ);  // 16-byte loads of K (and of V) per lane and round
  static constexpr int kRows = kRowsAtOnce * kLoads;                  // rows that a wave loads in a round
  static constexpr int kAcc = D / 32;
  static constexpr int kStepTiles = TK >= 2 ? 2 : 1;
  static constexpr bool kQueriesInLds = WQ == 1;
  // 64 requests stay in registers, four a lane; otherwise the next one is loaded when its turn comes, which shows less
  // where a column takes longer
  static constexpr bool kKeepsRequests = WQ == 1 && D <= 128;
  static constexpr int kTileArea = kBufs * kTiles * kTileBytes, kMergeArea = kWaves * (kAcc * 4096 + 512);
  static constexpr int kArea = kTileArea > kMergeArea ? kTileArea : kMergeArea;
  static constexpr size_t kPartial = (size_t)WQ * (kAcc * 4096 + 1024);
  static_assert(kLoads >= 1 && kRows <= kWave, "rows of a round");
};

// What a request's arrays say, cut to the buffers.
struct Said {
  uint32_t row0, rows, len;
  uint32_t dead;  // rejected: zeros
};

__device__ inline Said said_of(const AttnArgs& p, uint32_t b) {
  const gift_tree_attention_args& a = p.a;
  // loads without a branch between them, so that they are on their way together
  const uint32_t at = b < a.n_reqs ? b : a.n_reqs - 1;
  const uint32_t r0 = a.row_begin[at], r1 = a.row_begin[at + 1], len = a.lens[at];
  const uint32_t verdict = (a.verdicts ? (const uint32_t*)a.verdicts : a.lens)[at];
  const uint32_t total = (uint32_t)a.n_rows, most = a.table_width << p.kv.block_shift;
  Said s;
  s.row0 = r0 < total ? r0 : total;
  const uint32_t end = r1 < total ? r1 : total;
  s.rows = b < a.n_reqs && end > s.row0 ? end - s.row0 : 0;
  s.len = len < most ? len : most;
  s.dead = a.verdicts && verdict != GIFT_SEG_OK;
  return s;
}

// A request as the kernel works on it.
struct Req {
  uint32_t row0, rows, len, ctx_tiles, tiles, rounds, cols, col_tiles;
  bool dead;
};

template <class S>
__device__ inline Req req_of(const AttnArgs& p, const Said& s) {
  Req r;
  r.row0 = s.row0;
  r.rows = s.rows;
  r.len = s.len;
  r.dead = s.dead;
  r.ctx_tiles = (r.len + kTileKeys - 1) / kTileKeys;
  r.tiles = r.ctx_tiles + (p.a.k ? (r.rows + kTileKeys - 1) / kTileKeys : 0);
  const uint32_t rounds = (r.tiles + S::kTiles - 1) / S::kTiles;
  r.rounds = r.dead || rounds == 0 ? 1 : rounds;
  r.col_tiles = (uint32_t)(((uint64_t)r.rows * p.group + 32 * S::WQ - 1) / (32 * S::WQ));
  r.cols = r.col_tiles * p.kv.heads;
  return r;
}

template <class S>
__device__ inline uint64_t units_of(const AttnArgs& p, const Said& s) {
  const Req r = req_of<S>(p, s);
  return (uint64_t)r.cols * r.rounds;
}

// Request b0 + i in scalar registers, of the 64 that a wave's lanes hold.
template <class S>
__device__ inline Req req_at(const AttnArgs& p, const Said& s, uint32_t i) {
  Said u;
  u.row0 = __builtin_amdgcn_readlane(s.row0, i);
  u.rows = __builtin_amdgcn_readlane(s.rows, i);
  u.len = __builtin_amdgcn_readlane(s.len, i);
  u.dead = __builtin_amdgcn_readlane(s.dead, i);
  Req r = req_of<S>(p, u);
  r.rounds = __builtin_amdgcn_readfirstlane(r.rounds);
  r.col_tiles = __builtin_amdgcn_readfirstlane(r.col_tiles);
  r.cols = __builtin_amdgcn_readfirstlane(r.cols);
  return r;
}

// Running state of one wave's 32 columns: lane l holds column l % 32; of O^T
// the elements d = 32 t + 8 (i / 4) + 4 (l / 32) + i % 4.
template <class S>
struct State {
  float m, l;  // what the weights refer to (an unscaled score), this lane's part of the sum of weights
  f32x16 o[S::kAcc];
  __device__ void clear() {
    m = -INFINITY;
    l = 0;
#pragma unroll
    for (int t = 0; t < S::kAcc; t++) o[t] = f32x16{};
  }
  // dst: [kAcc * 4][64] f32x4, then [64] (m, l)
  __device__ void put(f32x4* dst, uint32_t lane) const {
#pragma unroll
    for (int t = 0; t < S::kAcc; t++)
#pragma unroll
      for (int q = 0; q < 4; q++)
        dst[(t * 4 + q) * kWave + lane] = f32x4{o[t][4 * q], o[t][4 * q + 1], o[t][4 * q + 2], o[t][4 * q + 3]};
    ((f32x2*)(dst + S::kAcc * 4 * kWave))[lane] = f32x2{m, l};
  }
};

__device__ inline f32x2 published(const uint64_t* at) {
  return __builtin_bit_cast(f32x2, __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

__device__ inline uint64_t uniform(uint64_t x) {
  return (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(x >> 32)) << 32 | __builtin_amdgcn_readfirstlane((uint32_t)x);
}

// x, worked out here: without it the compiler keeps what it can derive from a lane's number in a register for each use
// across the loop over the keys, and spills the operands.
__device__ inline uint32_t fresh(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Global memory by name: a pointer put together from integers would load by flat instructions, which count among the LDS
// accesses too, so that every wait for LDS would wait for the rows on their way.
typedef const __attribute__((address_space(1))) uint8_t* global_bytes;
typedef const __attribute__((address_space(1))) u32x4* global_pieces;

__device__ inline global_bytes pointer_of(const uint8_t* p, uint32_t lane) {
  const uint32_t lo = __builtin_amdgcn_ds_bpermute(4 * lane, (uint32_t)(uintptr_t)p),
                 hi = __builtin_amdgcn_ds_bpermute(4 * lane, (uint32_t)((uintptr_t)p >> 32));
  return (global_bytes)((uint64_t)hi << 32 | lo);
}

__device__ inline float other_half(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(threadIdx.x & 32 ? r[0] : r[1]);
}
__device__ inline float max_of_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Work is cut evenly: a round (kTiles tiles of 32 keys) of a column tile (32 WQ
// rows of one request and KV head) is a unit, and of all units in a row every
// workgroup takes the same number, whichever requests they belong to.  A column
// whose units lie in several workgroups is joined by the one that finishes last,
// in the order of the parts, so that the result does not depend on who that is.
// Bound by memory where rows are few: K and V of 131072 tokens (8 heads of 128
// elements, 537 MB) take 111 us, 4.8 TB/s, which is what a large copy reaches.
// With many rows by what a wave does one after the other: 32 requests of
// 2048-8192 tokens with trees of 16-32 tokens and 64 heads (729 MB, 142 GFLOP)
// take 290 us.  Without products and exponentials the loads and stores alone take
// 183 us of it; scores add about 70, exponentials 50, the product with V 100, and
// two waves a SIMD that meet once a round hide a third of that.
template <class E, class S, int MINW>
__global__ __launch_bounds__(S::kThreads, MINW) void k_tree_attention(AttnArgs p, uint8_t* work) {
  typedef typename E::vec vec;
  const gift_tree_attention_args& a = p.a;
  __shared__ __align__(16) uint8_t area[S::kArea];
  __shared__ __align__(16) uint8_t queries[S::kQueriesInLds ? 32 * S::kKRow : 16];
  __shared__ uint8_t row_flags[S::kBufs][S::kTiles][kTileKeys];  // bit 0: the key exists, bit 1: its V is not finite
  __shared__ uint64_t sums[S::kWaves];
  __shared__ uint64_t found[2];
  __shared__ uint32_t last_one;
  const uint32_t tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave),
                 wq = wave % S::WQ, wk = wave / S::WQ, half = lane / 32, col = lane % 32;
  uint32_t n_wg = gridDim.x, wg = blockIdx.x;

  // This workgroup's units, and the request that holds the first of them.  Every workgroup sums the requests' units
  // itself: up to 64 of them each wave for itself, a request a lane, without waiting for another; more of them the
  // workgroup together.
  const uint32_t row_first = a.n_reqs ? a.row_begin[0] : 0, row_last = a.n_reqs ? a.row_begin[a.n_reqs] : 0;
  Said said{0, 0, 0, 0};  // of requests b0 + lane
  if (a.n_reqs) said = said_of(p, lane);
  // rows of no request
  {
    const uint32_t total = (uint32_t)a.n_rows;
    uint32_t lo = row_first, hi = row_last;
    lo = lo < total ? lo : total;
    hi = hi < lo ? lo : hi < total ? hi : total;
    const uint32_t loose = lo + (total - hi);
    for (uint32_t i = wg; i < loose; i += n_wg) {
      const uint32_t r = i < lo ? i : hi + (i - lo);
      for (uint32_t u = tid; u < a.n_heads * S::kPieces; u += S::kThreads)
        *(u32x4*)((uint8_t*)a.out + r * a.out_row_stride + u / S::kPieces * a.out_head_stride + u % S::kPieces * 16) =
            u32x4{0, 0, 0, 0};
      if (a.lse)
        for (uint32_t h = tid; h < a.n_heads; h += S::kThreads) a.lse[(uint64_t)r * a.n_heads + h] = -INFINITY;
    }
  }
  if (a.n_reqs == 0) return;
  uint32_t b0 = 0, bi = 0;       // bi: the current request among them
  uint64_t total, unit, unit_end, base;  // base: first unit of the current request
  auto share = [&]() -> bool {
    if (total < n_wg) {
      if (wg >= total) return false;
      n_wg = (uint32_t)total;  // a unit each
    } else if (n_wg % 8 == 0) {
      // neighbours in the order of work share an XCD (and its L2), where column tiles of one KV head read the same keys
      wg = wg % 8 * (n_wg / 8) + wg / 8;
    }
    return true;
  };
  auto running = [&](uint64_t v) -> uint64_t {
    if (!__any(v >> 25)) {  // 32 bits hold the sum: additions across lanes without LDS
      uint32_t x = (uint32_t)v;
      x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xF, 0xF, true);   // the lane before, in a row of 16
      x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xF, 0xF, true);   // two before
      x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xF, 0xF, true);   // four
      x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xF, 0xF, true);   // eight
      x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xA, 0xF, false);  // a row's last to the next row
      x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xC, 0xF, false);  // the first half's last to the second
      return x;
    }
#pragma unroll 1
    for (int d = 1; d < kWave; d *= 2) {
      const uint64_t u = __shfl_up((unsigned long long)v, d);
      if (lane >= (uint32_t)d) v += u;
    }
    return v;
  };
  auto first_of = [&](uint32_t w) -> uint64_t {
    return n_wg == total ? w : quotient(w * total, n_wg, 1.0 / (double)n_wg);
  };
  if (a.n_reqs <= kWave) {
    const uint64_t mine = units_of<S>(p, said), upto = running(mine);
    total = uniform(__shfl((unsigned long long)upto, kWave - 1));
    if (!share()) return;
    unit = first_of(wg);
    bi = __builtin_ctzll(__ballot(unit < upto));
    base = uniform(__shfl((unsigned long long)(upto - mine), bi));
  } else {
    const uint32_t per = (a.n_reqs + S::kThreads - 1) / S::kThreads;
    uint64_t mine = 0;
#pragma unroll 4
    for (uint32_t i = 0; i < per; i++) mine += units_of<S>(p, said_of(p, tid * per + i));
    uint64_t upto = running(mine);
    if (lane == kWave - 1) sums[wave] = upto;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < S::kWaves; w++) {
      if ((uint32_t)w < wave) upto += sums[w];
      total += sums[w];
    }
    total = uniform(total);
    if (!share()) return;
    unit = first_of(wg);
    if (upto - mine <= unit && unit < upto) {
      uint64_t at = upto - mine;
      uint32_t b = tid * per;
      for (;; b++) {
        const uint64_t n = units_of<S>(p, said_of(p, b));
        if (unit < at + n) break;
        at += n;
      }
      found[0] = b;
      found[1] = at;
    }
    __syncthreads();
    b0 = __builtin_amdgcn_readfirstlane((uint32_t)found[0]);
    base = uniform(found[1]);
    said = said_of(p, b0 + lane);
  }
  // scalar from here on: divisions leave vector registers
  unit = uniform(unit);
  unit_end = uniform(first_of(wg + 1));
  const uint64_t first = unit;

  const float c = fmaxf(fabsf(a.scale) * 1.44269504f, 1.17549435e-38f);
  const uint32_t neg = a.scale < 0 ? 0x80008000u : 0u;
  const uint32_t row_lane = lane % S::kRows;  // the row whose address this lane works out
  // of the group's TK * 32 rows
  const uint32_t my_row = wq * S::kRowsAtOnce + row_lane % S::kRowsAtOnce + row_lane / S::kRowsAtOnce * (S::kRowsAtOnce * S::WQ);
  const uint32_t piece = lane % S::kLanes, at_once = lane / S::kLanes;
  const uint32_t read_at = 16 * (S::kPieces == S::kLanes || piece < (uint32_t)S::kPieces ? piece : 0);
  // where this lane's first piece of K and of V goes in LDS
  const uint32_t to_row = wq * S::kRowsAtOnce + at_once,
                 to_tile = (wk * S::TK + to_row / kTileKeys) * S::kTileBytes + piece * 16,
                 k_to = to_tile + to_row % kTileKeys * S::kKRow,
                 v_to = to_tile + kTileKeys * S::kKRow + to_row % kTileKeys * S::kVRow;
  uint32_t* counters = (uint32_t*)work;
  uint8_t* partials = work + 4 * kAttnCounters;

  Req r = req_at<S>(p, said, bi);
  while (unit < unit_end) {
    while (unit >= base + (uint64_t)r.cols * r.rounds) {
      base += (uint64_t)r.cols * r.rounds;
      if (++bi == kWave || !S::kKeepsRequests) {
        b0 += bi;
        bi = 0;
        said = said_of(p, b0 + lane);
      }
      r = req_at<S>(p, said, bi);
    }
    const Unit at = unit_of(unit - base, r.rounds);
    const uint32_t column = __builtin_amdgcn_readfirstlane(at.column), it0 = __builtin_amdgcn_readfirstlane(at.round);
    const uint64_t col_first = unit - it0, col_last = col_first + r.rounds - 1;
    const uint32_t it1 = (uint32_t)(unit_end - unit < r.rounds - it0 ? it0 + (unit_end - unit) : r.rounds);
    const uint32_t g = __builtin_amdgcn_readfirstlane(quotient(column, r.col_tiles)), ct = column - g * r.col_tiles;
    // this lane's query row
    const uint32_t rows = r.rows * p.group, qrow = (ct * S::WQ + wq) * 32 + col;
    const bool qlive = qrow < rows;
    const bool wave_live = (ct * S::WQ + wq) * 32 < rows;
    const uint32_t token = quotient(qlive ? qrow : 0, p.group), head = g * p.group + (qlive ? qrow - token * p.group : 0);
    const uint64_t qtok = r.row0 + token;
    State<S> st;
    st.clear();
    if (!r.dead && r.tiles) {
      // Queries: in registers, or in LDS where all waves have the same ones and need the registers for keys on their way.
      vec q[S::kQueriesInLds ? 1 : S::D / 16];
      if constexpr (!S::kQueriesInLds) {
        const uint8_t* qp = (const uint8_t*)a.q + qtok * a.q_row_stride + head * a.q_head_stride + half * 16;
#pragma unroll
        for (int s = 0; s < S::D / 16; s++) q[s] = __builtin_bit_cast(vec, *(const u32x4*)(qp + 32 * s) ^ neg);
      }
      const uint32_t* tab = a.tables + (uint64_t)(b0 + bi) * a.table_stride;
      const uint8_t* kbase = p.kv.base + a.layer * p.kv.layer_stride + g * p.kv.head_stride;
      const uint8_t *dk = (const uint8_t*)a.k + r.row0 * a.k_row_stride + g * a.k_head_stride,
                    *dv = (const uint8_t*)a.v + r.row0 * a.v_row_stride + g * a.v_head_stride;
      const uint32_t ctx_keys = r.ctx_tiles * kTileKeys;

      // Loads of a round, first step: the block id of this lane's row.  It is asked for two rounds ahead and before the
      // rows of the round between, since loads come back in order and the addresses wait for it.
      auto block_of = [&](uint32_t it) -> uint32_t {
        const uint32_t j = (it * S::kTiles + wk * S::TK) * kTileKeys + my_row;
        return *(it < it1 && j < r.len ? tab + (j >> p.kv.block_shift) : a.row_begin);  // no branch around the load
      };
      // Second step: this lane's row.
      struct Row {
        const uint8_t *k, *v;
        bool ok;       // it exists
        bool drafted;  // it is past the cached keys
        bool any;      // the round's rows of this wave may hold drafted keys
      };
      auto row_of = [&](uint32_t it, uint32_t id) -> Row {
        const uint32_t j = (it * S::kTiles + wk * S::TK) * kTileKeys + my_row;
        Row x;
        x.any = (it * S::kTiles + wk * S::TK + S::TK) * kTileKeys > ctx_keys;
        x.drafted = x.any && j >= ctx_keys;
        x.k = kbase + id * p.kv.block_stride + (j & ((1u << p.kv.block_shift) - 1)) * p.kv.token_stride;
        x.v = x.k + p.kv.v_off;
        x.ok = it < it1 && j < r.len && id < p.kv.n_blocks;
        if (x.drafted) {
          const uint32_t t = j - ctx_keys;
          x.ok = it < it1 && a.k && t < r.rows;
          x.k = dk + t * a.k_row_stride;
          x.v = dv + t * a.v_row_stride;
        }
        if (!x.ok) x.k = x.v = (const uint8_t*)a.q;  // a row that may be read, of which nothing is used
        return x;
      };
      // Third step: the rows' pieces, each lane from the address that another lane worked out.
      auto fetch = [&](u32x4 (&x)[S::kLoads], const uint8_t* rows) {
        const uint32_t first = fresh(at_once);
#pragma unroll
        for (int i = 0; i < S::kLoads; i++) {
          const global_bytes from = pointer_of(rows, i * S::kRowsAtOnce + first);
          x[i] = *(global_pieces)(from + read_at);
        }
      };
      // Fourth step: into LDS.
      constexpr int kStep = S::kRowsAtOnce * S::WQ;  // rows from one load to the next: a multiple or a divisor of a tile's
      auto store_k = [&](const u32x4 (&x)[S::kLoads], uint32_t buf) {
        uint8_t* at = area + buf * (S::kTiles * S::kTileBytes) + fresh(k_to);
#pragma unroll
        for (int i = 0; i < S::kLoads; i++)
          if (S::kPieces == S::kLanes || piece < (uint32_t)S::kPieces)
            *(u32x4*)(at + i * kStep / kTileKeys * S::kTileBytes + i * kStep % kTileKeys * S::kKRow) = x[i];
      };
      // V rows of keys that do not exist, and drafted ones that are not finite, are stored as zeros: a weight of zero
      // times NaN would reach every row.  Cached ones stay as they are, since every row of the request sees them.
      auto store_v = [&](u32x4 (&x)[S::kLoads], const Row& row, uint32_t buf) {
        uint32_t flag = row.ok ? 1u : 0u;
        const uint64_t oks = __ballot(row.ok);
        if (oks != ~0ull) {
          const uint32_t mine = (uint32_t)(oks >> fresh(at_once));  // bit i * kRowsAtOnce: the row of load i
#pragma unroll
          for (int i = 0; i < S::kLoads; i++)
            if (!(mine >> (i * S::kRowsAtOnce) & 1)) x[i] = u32x4{0, 0, 0, 0};
        }
        if (row.any) {
          const uint32_t mine = (uint32_t)(__ballot(row.drafted) >> fresh(at_once));
          u16x2 top[S::kLoads], all{0, 0};  // largest exponents of a piece's elements
#pragma unroll
          for (int i = 0; i < S::kLoads; i++) {
            top[i] = u16x2{0, 0};
#pragma unroll
            for (int e = 0; e < 4; e++)
              top[i] = __builtin_elementwise_max(top[i], __builtin_bit_cast(u16x2, x[i][e] & (E::kExp * 0x10001u)));
            if (!(mine >> (i * S::kRowsAtOnce) & 1)) top[i] = u16x2{0, 0};
            all = __builtin_elementwise_max(all, top[i]);
          }
          if (__any(all[0] == E::kExp || all[1] == E::kExp)) {
            const uint32_t first = fresh(at_once), own = fresh(row_lane);
            constexpr uint64_t kOneRow = (1ull << S::kLanes) - 1;
#pragma unroll
            for (int i = 0; i < S::kLoads; i++) {
              const uint64_t odds = __ballot((top[i][0] == E::kExp || top[i][1] == E::kExp) && piece < (uint32_t)S::kPieces);
              if (odds >> (first * S::kLanes) & kOneRow) x[i] = u32x4{0, 0, 0, 0};
              if (own / S::kRowsAtOnce == (uint32_t)i && (odds >> (own % S::kRowsAtOnce * S::kLanes) & kOneRow)) flag |= 2u;
            }
          }
        }
        uint8_t* at = area + buf * (S::kTiles * S::kTileBytes) + fresh(v_to);
#pragma unroll
        for (int i = 0; i < S::kLoads; i++)
          if (S::kPieces == S::kLanes || piece < (uint32_t)S::kPieces)
            *(u32x4*)(at + i * kStep / kTileKeys * S::kTileBytes + i * kStep % kTileKeys * S::kVRow) = x[i];
        if (lane < (uint32_t)S::kRows) row_flags[buf][wk * S::TK + my_row / kTileKeys][my_row % kTileKeys] = (uint8_t)flag;
      };
      auto meet = [&]() {
        if constexpr (S::WQ == 1) {
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          __builtin_amdgcn_wave_barrier();
        } else {
          __syncthreads();
        }
      };
      // A step takes kStepTiles tiles: two where a wave has them, whose independent products and exponentials fill each
      // other's latencies and share one maximum.
      constexpr int kN = S::kStepTiles;
      auto scores = [&](const uint8_t* tile, f32x16 (&sc)[kN]) {
#pragma unroll
        for (int n = 0; n < kN; n++) sc[n] = f32x16{};
        const uint8_t* krow = tile + col * S::kKRow + half * 16;
        constexpr int kSteps = S::D / 16, kAheadK = 2;  // operands on their way while products are made
        vec kd[kAheadK + 1][kN], qd[kAheadK + 1];
        auto keys = [&](int d) {
#pragma unroll
          for (int n = 0; n < kN; n++) kd[d % (kAheadK + 1)][n] = *(const vec*)(krow + n * S::kTileBytes + 32 * d);
          qd[d % (kAheadK + 1)] = S::kQueriesInLds ? *(const vec*)(queries + col * S::kKRow + half * 16 + 32 * d)
                                                   : q[S::kQueriesInLds ? 0 : d];
        };
#pragma unroll
        for (int d = 0; d < kAheadK; d++) keys(d);
#pragma unroll
        for (int d = 0; d < kSteps; d++) {
          if (d + kAheadK < kSteps) keys(d + kAheadK);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int n = 0; n < kN; n++) sc[n] = E::mfma(kd[d % (kAheadK + 1)][n], qd[d % (kAheadK + 1)], sc[n]);
        }
      };
      auto seen = [&](uint32_t see, int i) -> bool { return see >> (8 * (i / 4) + i % 4) & 1; };  // of see >> 4 half
      // scores of tiles t, t + 1, ... to weights; flag: their row_flags of row `col`
      auto weigh = [&](f32x16 (&sc)[kN], uint32_t t, const uint32_t (&flag)[kN]) {
        uint32_t see[kN];
        bool part = false;
#pragma unroll
        for (int n = 0; n < kN; n++) {
          see[n] = (uint32_t)__ballot(flag[n] & 1);
          part |= see[n] != ~0u;
        }
        const bool draft = t + kN > r.ctx_tiles;
        part |= draft;
        if (part) {
#pragma unroll
          for (int n = 0; n < kN; n++) {
            if (t + n >= r.ctx_tiles) {
              const uint32_t word = t + n - r.ctx_tiles;
              if (a.mask)
                see[n] &= word < a.mask_words ? a.mask[qtok * a.mask_words + word] : 0u;
              else
                see[n] &= token >= 32 * word + 31 ? ~0u : token < 32 * word ? 0u : (2u << (token - 32 * word)) - 1;
            }
            const uint32_t mine = see[n] >> (4 * half);
#pragma unroll
            for (int i = 0; i < 16; i++)
              if (!seen(mine, i)) sc[n][i] = -INFINITY;
          }
        }
        float top = sc[0][0];
#pragma unroll
        for (int n = 0; n < kN; n++)
#pragma unroll
          for (int i = 0; i < 16; i++) top = fmaxf(top, sc[n][i]);
        top = max_of_halves(top);
        // What weights refer to need not be the maximum itself: while no score passes it by kSlack octaves it stays, and
        // the sums with it (random scores raise the maximum of some column in most steps).  A column's own scores decide,
        // so that a row's bits do not depend on the rows beside it.
        const bool grow = (top - st.m) * c > E::kSlack;
        const float mn = grow ? top : st.m, safe = mn == -INFINITY ? 0.f : mn;
        if (__any(grow)) {
          const float f = exp2f((st.m - safe) * c);
          st.l *= f;
#pragma unroll
          for (int d = 0; d < S::kAcc; d++) st.o[d] *= f;
          st.m = mn;
        }
        float shift = -safe * c;
        const bool far = fabsf(shift) > kFarShift;
        if (E::kTop != 0.f && !far) shift += E::kTop;
        if (__any(far)) {
          // what the product's rounding left out, for the columns whose own scores need it
          const float left = far ? __builtin_fmaf(safe, c, shift) - E::kTop : 0.f;
#pragma unroll
          for (int n = 0; n < kN; n++)
#pragma unroll
            for (int i = 0; i < 16; i++) sc[n][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[n][i], c, shift) - left);
        } else {
#pragma unroll
          for (int n = 0; n < kN; n++)
#pragma unroll
            for (int i = 0; i < 16; i++) sc[n][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[n][i], c, shift));
        }
        float sum[4] = {0, 0, 0, 0};
#pragma unroll
        for (int n = 0; n < kN; n++)
#pragma unroll
          for (int i = 0; i < 16; i++) sum[i % 4] += sc[n][i];
        st.l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        if (draft) {
#pragma unroll 1
          for (int n = 0; n < kN; n++) {
            uint32_t odd = t + n >= r.ctx_tiles ? (uint32_t)__ballot(flag[n] & 2) : 0u;
            while (odd) {  // drafted keys whose V is not finite: only for the rows that see them
              const uint32_t key = __builtin_ctz(odd);
              odd &= odd - 1;
              float own = 0;
#pragma unroll
              for (int i = 0; i < 16; i++)
                if ((uint32_t)(8 * (i / 4) + i % 4) == (key & ~4u)) own = n ? sc[kN - 1][i] : sc[0][i];
              const float theirs = other_half(own), weight = (key >> 2 & 1) == half ? own : theirs;
              const typename E::elem* vp =
                  (const typename E::elem*)(dv + (uint64_t)((t + n - r.ctx_tiles) * kTileKeys + key) * a.v_row_stride);
              if ((n ? see[kN - 1] : see[0]) >> key & 1) {
#pragma unroll
                for (int d = 0; d < S::kAcc; d++)
#pragma unroll
                  for (int i = 0; i < 16; i++) st.o[d][i] += weight * (float)vp[32 * d + 8 * (i / 4) + 4 * half + i % 4];
              }
            }
          }
        }
      };
      auto add_values = [&](const uint8_t* tile, const f32x16 (&p)[kN]) {
        const uint8_t* vrow = tile + kTileKeys * S::kKRow + (4 * half + lane % 16 / 4) * S::kVRow +
                              (lane / 16 % 2 * 16 + lane % 4 * 4) * 2;
        typedef __attribute__((address_space(3))) s16x4 lds4;
        union Frag {
          s16x4 x[2];
          vec v;
        };
        // step i: V^T of 16 keys for elements 32 d .. 32 d + 31
        constexpr int kSteps = 2 * kN * S::kAcc;
        auto values = [&](int i, Frag& u) {
          const uint8_t* at = vrow + i / (2 * S::kAcc) * S::kTileBytes + i / S::kAcc % 2 * (16 * S::kVRow) + i % S::kAcc * 64;
          u.x[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)at);
          u.x[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(at + 8 * S::kVRow));
        };
        constexpr int kAheadV = 2;  // operands on their way while products are made
        Frag u[kAheadV + 1];
#pragma unroll
        for (int i = 0; i < kAheadV; i++) values(i, u[i]);
        vec w[E::kParts];
#pragma unroll
        for (int i = 0; i < kSteps; i++) {
          if (i % S::kAcc == 0) E::parts(p[i / (2 * S::kAcc)], i / S::kAcc % 2, w);
          if (i + kAheadV < kSteps) values(i + kAheadV, u[(i + kAheadV) % (kAheadV + 1)]);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int e = 0; e < E::kParts; e++) st.o[i % S::kAcc] = E::mfma(u[i % (kAheadV + 1)].v, w[e], st.o[i % S::kAcc]);
        }
      };

      if constexpr (S::WQ == 1) {
        // A tile of the wave's own a round.  One set of registers brings K of the next tile while V of this one is in
        // use, and V while K is.
        static_assert(S::TK == 1, "a tile a round");
        u32x4 x[S::kLoads];
        const uint8_t* tile = area + wk * S::kTileBytes;
        uint32_t id = block_of(it0), next = block_of(it0 + 1);
        constexpr int kQ = (32 * S::kPieces + S::kThreads - 1) / S::kThreads;
        u32x4 qx[kQ];
#pragma unroll
        for (int i = 0; i < kQ; i++) {
          const uint32_t u = tid + i * S::kThreads, line = u / S::kPieces,
                         row = line < 32 && ct * 32 + line < rows ? ct * 32 + line : 0, tok = quotient(row, p.group);
          qx[i] = *(const u32x4*)((const uint8_t*)a.q + (uint64_t)(r.row0 + tok) * a.q_row_stride +
                                  (uint64_t)(g * p.group + (row - tok * p.group)) * a.q_head_stride + u % S::kPieces * 16);
        }
        Row row = row_of(it0, id);
        fetch(x, row.k);
#pragma unroll
        for (int i = 0; i < kQ; i++) {
          const uint32_t u = tid + i * S::kThreads;
          if (u < 32 * S::kPieces) *(u32x4*)(queries + u / S::kPieces * S::kKRow + u % S::kPieces * 16) = qx[i] ^ neg;
        }
        store_k(x, 0);
        fetch(x, row.v);
        __syncthreads();
        for (uint32_t it = it0;; it++) {
          const uint32_t t = it * S::kTiles + wk;
          const bool more = it + 1 < it1;
          f32x16 sc[1];
          meet();
          scores(tile, sc);
          store_v(x, row, 0);
          if (more) {
            id = next;
            next = block_of(it + 2);
            row = row_of(it + 1, id);
            fetch(x, row.k);
          }
          meet();
          const uint32_t flag[1] = {row_flags[0][wk][col]};
          weigh(sc, t, flag);
          add_values(tile, sc);
          if (!more) break;
          meet();
          store_k(x, 0);
          fetch(x, row.v);
        }
      } else {
        // A round is in one buffer while the next one goes to the other; the one after it is on its way.  A wave that is
        // done with its products stores and asks ahead while others still compute.
        u32x4 xk[S::kLoads], xv[S::kLoads];
        uint32_t id = block_of(it0), next = block_of(it0 + 1);
        Row row = row_of(it0, id);
        fetch(xk, row.k);
        fetch(xv, row.v);
        for (uint32_t it = it0;; it++) {
          const uint32_t buf = (it - it0) & 1;
          store_k(xk, buf);
          store_v(xv, row, buf);
          if (it + 1 < it1) {
            id = next;
            next = block_of(it + 2);
            row = row_of(it + 1, id);
            fetch(xk, row.k);
            fetch(xv, row.v);
          }
          meet();
          if (wave_live) {
#pragma unroll 1
            for (int s = 0; s < S::TK; s += kN) {
              const uint32_t t = it * S::kTiles + wk * S::TK + s;
              if (t >= r.tiles) break;
              const uint8_t* tile = area + (buf * S::kTiles + wk * S::TK + s) * S::kTileBytes;
              f32x16 sc[kN];
              uint32_t flag[kN];
#pragma unroll
              for (int n = 0; n < kN; n++) flag[n] = row_flags[buf][wk * S::TK + s + n][col];
              // a wave's products go before another's exponentials on the SIMD (32 requests of 2048-8192 tokens: 306 -> 302)
              __builtin_amdgcn_s_setprio(1);
              scores(tile, sc);
              __builtin_amdgcn_s_setprio(0);
              weigh(sc, t, flag);
              __builtin_amdgcn_s_setprio(1);
              add_values(tile, sc);
              __builtin_amdgcn_s_setprio(0);
            }
          }
          if (it + 1 == it1) break;
        }
      }
      st.l += other_half(st.l);
    }

    // The column's states go to LDS, and from there each wave of a query group takes every WK-th 32 elements of D: the
    // key groups' states are added on the way.  (What follows runs once a column, so it is kept short instead of
    // unrolled: code that is not in the instruction cache yet costs more than what it does.)
    constexpr size_t kPer = S::kAcc * 4096 + 512;  // bytes of a wave's state
    __syncthreads();
    st.put((f32x4*)(area + wave * kPer), lane);
    __syncthreads();
    auto state = [&](int k) { return (const f32x4*)(area + (k * S::WQ + wq) * kPer); };
    float m = -INFINITY, l = 0;
    f32x2 ml[S::WK];
#pragma unroll
    for (int k = 0; k < S::WK; k++) {
      ml[k] = ((const f32x2*)(state(k) + S::kAcc * 4 * kWave))[lane];
      m = fmaxf(m, ml[k][0]);
    }
    {
      const float safe = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int k = 0; k < S::WK; k++) {
        ml[k][0] = exp2f((ml[k][0] - safe) * c);  // the state's factor
        l += ml[k][1] * ml[k][0];
      }
    }
    auto chunk = [&](int t) -> f32x16 {
      f32x16 o = f32x16{};
#pragma unroll
      for (int k = 0; k < S::WK; k++)
#pragma unroll
        for (int q = 0; q < 4; q++) {
          const f32x4 v = state(k)[(t * 4 + q) * kWave + lane];
#pragma unroll
          for (int e = 0; e < 4; e++) o[4 * q + e] += v[e] * ml[k][0];
        }
      return o;
    };
    auto write = [&](int t, const f32x16& o, float m, float l) {
      const float inv = l == 0.f ? 0.f : 1.f / l;
      constexpr float kUnit = 1.f / (float)(1u << (int)E::kTop);
      uint8_t* op = (uint8_t*)a.out + qtok * a.out_row_stride + head * a.out_head_stride + half * 8 + 64 * t;
#pragma unroll
      for (int k = 0; k < 4; k++) {
        typedef typename E::elem elem4 __attribute__((ext_vector_type(4)));
        elem4 x;
#pragma unroll
        for (int e = 0; e < 4; e++) x[e] = (typename E::elem)(o[4 * k + e] * inv);
        *(elem4*)(op + 16 * k) = x;
      }
      if (a.lse && t == 0 && half == 0)
        a.lse[qtok * a.n_heads + head] = l == 0.f ? -INFINITY : (m * c + __builtin_amdgcn_logf(l * kUnit)) * 0.693147181f;
    };
    // the workgroup that has a unit: most often this one
    auto owner = [&](uint64_t u) -> uint32_t {
      if (u >= first && u < unit_end) return wg;
      return n_wg == total ? (uint32_t)u : (uint32_t)quotient((u + 1) * n_wg - 1, total, 1.0 / (double)total);
    };
    const uint32_t w0 = owner(col_first), parts = owner(col_last) - w0 + 1;
    if (parts == 1) {
      if (qlive)
#pragma unroll 1
        for (int t = wk; t < S::kAcc; t += S::WK) write(t, chunk(t), m, l);
    } else {
      // A column's parts are joined by the workgroup that finishes last; many of them in two steps, by the last of each
      // run of parts and then by the last of the runs, so that no workgroup has more than about the root of them to read
      // (64 parts in one step: 25 us longer).
      const uint32_t run = parts <= 8 ? parts : parts <= 64 ? 8 : parts <= 256 ? 16 : 64;
      // Of a workgroup's parts at most the first joins a column begun before it, and at most the last one begins a
      // column that others end: two places each.
      auto place = [&](uint32_t w) -> uint64_t* {
        return (uint64_t*)(partials + (2 * w + (w == w0 ? 1 : 0)) * S::kPartial + wq * (S::kPartial / S::WQ));
      };
      // Words that workgroups of other XCDs read: stores and loads at the device's scope, past the XCDs' own L2s.  A
      // fence would write back and drop the whole L2 instead (64 requests of 128-2048 tokens: 185 us longer).
      // Elements of O, then [2][64] maxima and sums: those of a part, and those of the run that begins with it.
      auto publish = [&](uint64_t* to, int t, const f32x16& o, float m, float l, int joined) {
#pragma unroll
        for (int q = 0; q < 8; q++)
          __hip_atomic_store(to + ((t * 4 + q / 2) * kWave + lane) * 2 + q % 2,
                             __builtin_bit_cast(uint64_t, f32x2{o[2 * q], o[2 * q + 1]}), __ATOMIC_RELAXED,
                             __HIP_MEMORY_SCOPE_AGENT);
        if (t == 0)
          __hip_atomic_store(to + (S::kAcc * 8 + joined) * kWave + lane, __builtin_bit_cast(uint64_t, f32x2{m, l}),
                             __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      };
      auto last_of = [&](uint32_t* counter, uint32_t n) -> bool {
        __builtin_amdgcn_s_waitcnt(0);  // the stores have arrived before the count goes up
        __syncthreads();
        if (tid == 0) {
          last_one = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == n - 1;
          if (last_one) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // for the next call
        }
        __syncthreads();
        return __builtin_amdgcn_readfirstlane(last_one);
      };
      if (qlive)
#pragma unroll 1
        for (int t = wk; t < S::kAcc; t += S::WK) publish(place(wg), t, chunk(t), m, l, 0);
      // n published states, of every step-th workgroup from w on, in that order
      uint32_t w = w0 + (wg - w0) / run * run, n = w0 + parts - w < run ? w0 + parts - w : run, step = 1;
      uint32_t* counter = run == parts ? counters + w0 : counters + kAttnCounters / 4 + 2 * w + (w == w0 ? 1 : 0);
      while (last_of(counter, n)) {
        const bool whole = run == parts || step == run;
        if (qlive)
#pragma unroll 1
          for (int t = wk; t < S::kAcc; t += S::WK) {
            constexpr uint32_t kAhead = S::WQ == 1 && S::D <= 128 ? 8 : 4;  // states on their way at a time
            float m = -INFINITY, l = 0;
            f32x16 o = f32x16{};
#pragma unroll 1
            for (uint32_t j = 0; j < n; j += kAhead) {
              f32x2 x[kAhead][8], ml[kAhead];
#pragma unroll
              for (uint32_t u = 0; u < kAhead; u++) {
                const uint64_t* from = place(w + (j + u < n ? j + u : n - 1) * step);
                ml[u] = published(from + (S::kAcc * 8 + (step > 1)) * kWave + lane);
#pragma unroll
                for (int q = 0; q < 8; q++) x[u][q] = published(from + ((t * 4 + q / 2) * kWave + lane) * 2 + q % 2);
              }
              float mn = m;
#pragma unroll
              for (uint32_t u = 0; u < kAhead; u++) mn = fmaxf(mn, ml[u][0]);
              const float safe = mn == -INFINITY ? 0.f : mn, f0 = exp2f((m - safe) * c);
              l *= f0;
              o *= f0;
              m = mn;
#pragma unroll
              for (uint32_t u = 0; u < kAhead; u++)
                if (j + u < n) {
                  const float f = exp2f((ml[u][0] - safe) * c);
                  l += ml[u][1] * f;
#pragma unroll
                  for (int e = 0; e < 16; e++) o[e] += x[u][e / 2][e % 2] * f;
                }
            }
            // a run's elements take the place of its first part's, which no other wave reads
            if (whole)
              write(t, o, m, l);
            else
              publish(place(w), t, o, m, l, 1);
          }
        if (whole) break;
        w = w0;
        n = (parts + run - 1) / run;
        step = run;
        counter = counters + w0;
      }
    }
    __syncthreads();
    unit += it1 - it0;
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

namespace {

template <class E, class S, int MINW>
hipError_t attend(const AttnArgs& a, const AttnWork& w, hipStream_t s) {
  // as many workgroups as run at once: MINW waves on each SIMD, four SIMDs
  uint32_t grid = w.cus * (4 * MINW / S::kWaves);
  static_assert(4 * MINW % S::kWaves == 0, "whole workgroups");
  if (2 * grid * S::kPartial > w.partial_bytes || grid > kAttnCounters / 4) return hipErrorInvalidValue;
  // and no more than the lengths can give work to, as far as the host knows them
  const uint64_t tiles = (((uint64_t)a.a.table_width << a.kv.block_shift) + a.a.n_rows) / kTileKeys + 2,
                 cols = (uint64_t)a.kv.heads * (a.a.n_rows * a.group / (32 * S::WQ) + a.a.n_reqs),
                 rounds = tiles / S::kTiles + 1;
  if (cols < grid && cols * rounds < grid) grid = cols * rounds ? (uint32_t)(cols * rounds) : 1;
  k_tree_attention<E, S, MINW><<<grid, S::kThreads, 0, s>>>(a, w.mem);
  return hipGetLastError();
}

// Waves that share a tile of keys, by the rows that a request has on average at
// a KV head.  Two workgroups of four waves a CU run out of step with each
// other, one's products under the other's barrier; from 129 rows on eight waves
// share a tile, so that keys are not read twice.  In us, the same inputs call
// after call, 64 requests of 128-2048 tokens with 1 / 8 / 16 / 24 / 32 drafted
// tokens at a group of 4 (4, 32, 64, 96, 128 rows): a wave each 58 / 68 / 99 /
// 147 / 206; two 66 / 74 / 79 / 119 / 158; four 76 / 83 / 84 / 107 / 133; eight
// 111 / 107 / 116 / 111 / 154.  32 requests of 2048-8192 tokens, 192 rows on
// average: one 783, two 443, four 347, eight 286.
// With 256 elements a wave takes all registers of its SIMD, and four waves are
// as many as there are.
template <class E, int D>
hipError_t attend_by_rows(const AttnArgs& a, const AttnWork& w, hipStream_t s) {
  const uint64_t rows = a.a.n_reqs ? (a.a.n_rows * a.group + a.a.n_reqs - 1) / a.a.n_reqs : 1;
  constexpr int kPerSimd = D <= 128 ? 2 : 1;
  if (rows <= 32) return attend<E, Shape<D, 1, 4, 1>, kPerSimd>(a, w, s);
  if (rows <= 64) return attend<E, Shape<D, 2, 2, 1>, kPerSimd>(a, w, s);
  if constexpr (D <= 128)
    if (rows > 128) return attend<E, Shape<D, 8, 1, 4>, kPerSimd>(a, w, s);
  return attend<E, Shape<D, 4, 1, 2>, kPerSimd>(a, w, s);
}

template <class E>
hipError_t attend_by_dim(const AttnArgs& a, const AttnWork& w, hipStream_t s) {
  switch (a.kv.head_dim) {
    case 64: return attend_by_rows<E, 64>(a, w, s);
    case 96: return attend_by_rows<E, 96>(a, w, s);
    case 128: return attend_by_rows<E, 128>(a, w, s);
    default: return attend_by_rows<E, 256>(a, w, s);
  }
}

}  // namespace

hipError_t launch_tree_attention(const AttnArgs& a, uint32_t dtype, const AttnWork& w, hipStream_t s) {
  return dtype == GIFT_BF16 ? attend_by_dim<Bf16>(a, w, s) : attend_by_dim<F16>(a, w, s);
}

}  // namespace gift
