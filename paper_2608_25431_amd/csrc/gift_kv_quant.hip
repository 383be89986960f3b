// Kernels of include/gift_kv.h around a quantised cache: norm and rotation of queries and keys, rows into the cache, cached
// tokens back in 16 bits, and attention over it (gift_kv_attention.hpp).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gift_kv_attention.hpp"
#include "gift_kv_internal.hpp"
#include "gift_kv_narrow.hpp"

namespace gift {
namespace {

constexpr int kThreads = 256;
// Workgroups of a launch.  One of 2^32 threads along a dimension or more runs nothing, without an error, so that more rows
// take another launch.
constexpr uint32_t kMostGroups = 1u << 18;

template <class E>
__device__ inline float upper_of(uint32_t x) {
  return (float)__builtin_bit_cast(typename E::elem, (uint16_t)(x >> 16));
}
template <class E>
__device__ inline float lower_of(uint32_t x) {
  return (float)__builtin_bit_cast(typename E::elem, (uint16_t)x);
}
template <class E>
__device__ inline uint32_t packed(float lower, float upper) {
  return (uint32_t)__builtin_bit_cast(uint16_t, (typename E::elem)lower) |
         (uint32_t)__builtin_bit_cast(uint16_t, (typename E::elem)upper) << 16;
}
template <class E>
__device__ inline void floats_of(const u32x4& x, float* y) {
#pragma unroll
  for (int i = 0; i < 4; i++) y[2 * i] = lower_of<E>(x[i]), y[2 * i + 1] = upper_of<E>(x[i]);
}
template <class E>
__device__ inline u32x4 pieces_of(const float* y) {
  u32x4 x;
#pragma unroll
  for (int i = 0; i < 4; i++) x[i] = packed<E>(y[2 * i], y[2 * i + 1]);
  return x;
}

// ---------------------------------------------------------------------------
// Norm and rotation
// ---------------------------------------------------------------------------

constexpr int kMostRows = 8;    // rows of a workgroup
constexpr int kMostPairs = 128;

// A lane holds 16 elements of a head, in two pieces of 8 that pair with each
// other (or each within itself, where pairs are adjacent), so that a rotation
// needs no other lane; a head's sum of squares is joined over its 4 to 16
// lanes.  The rows' sines and cosines are worked out once a workgroup, of
// angles whose whole turns are taken off in 64 bits.  Bound by memory: 17203
// rows of 40 heads of 128 elements (352 MB read and written) take 72 us, 4.9
// TB/s, which is what a large copy reaches; one row 2.9, a launch about 2.
template <class E, int D>
__global__ __launch_bounds__(kThreads) void k_qk_norm_rope(gift_qk_rows a, uint32_t rows_each) {
  constexpr int kUsed = D / 16, kGroup = kUsed <= 4 ? 4 : kUsed <= 8 ? 8 : 16;  // lanes of a head
  __shared__ __align__(16) float cosines[kMostRows][kMostPairs], sines[kMostRows][kMostPairs];
  const uint32_t tid = threadIdx.x, lane = tid % kGroup, heads = a.q_heads + a.k_heads, pairs = a.rotary_dim / 2;
  const uint64_t row0 = (uint64_t)blockIdx.x * rows_each;
  const uint32_t rows = (uint32_t)(a.n_rows - row0 < rows_each ? a.n_rows - row0 : rows_each);
  for (uint32_t u = tid; u < rows * pairs; u += kThreads) {
    const uint32_t r = quotient(u, pairs), i = u - r * pairs;
    uint32_t axis = 0, upto = a.sections[0];
#pragma unroll
    for (uint32_t x = 1; x < 4; x++)
      if (x < a.n_axes && i >= upto) axis = x, upto += a.sections[x];
    const double turns = (double)a.positions[axis * a.position_stride + row0 + r] * (double)a.inv_freq[i] * 0.15915494309189535;
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    cosines[r][i] = c;
    sines[r][i] = s;
  }
  __syncthreads();
  const bool on = lane < (uint32_t)kUsed, turned = lane < a.rotary_dim / 16;
  // this lane's pieces
  uint32_t c0 = 2 * lane, c1 = 2 * lane + 1;
  if (!a.interleaved && turned) c0 = lane, c1 = lane + a.rotary_dim / 16;
  for (uint32_t u = blockIdx.y * (kThreads / kGroup) + tid / kGroup; u < rows * heads; u += gridDim.y * (kThreads / kGroup)) {
    const uint32_t r = quotient(u, heads), h = u - r * heads, kh = h - a.q_heads;
    const uint64_t row = row0 + r;
    const bool is_q = h < a.q_heads;
    const uint8_t* from = is_q ? (const uint8_t*)a.q + row * a.q_row_stride + h * a.q_head_stride
                               : (const uint8_t*)a.k + row * a.k_row_stride + kh * a.k_head_stride;
    uint8_t* to = is_q ? (uint8_t*)a.q_out + row * a.q_out_row_stride + h * a.q_out_head_stride
                       : (uint8_t*)a.k_out + row * a.k_out_row_stride + kh * a.k_out_head_stride;
    const uint8_t* weight = (const uint8_t*)(is_q ? a.q_weight : a.k_weight);
    float x[16], w[16];
    if (on) {
      floats_of<E>(*(const u32x4*)(from + 16 * c0), x);
      floats_of<E>(*(const u32x4*)(from + 16 * c1), x + 8);
    } else {
#pragma unroll
      for (int i = 0; i < 16; i++) x[i] = 0;
    }
    if (weight) {
      if (on) {
        floats_of<E>(*(const u32x4*)(weight + 16 * c0), w);
        floats_of<E>(*(const u32x4*)(weight + 16 * c1), w + 8);
      }
      float sum = 0;
#pragma unroll
      for (int i = 0; i < 16; i++) sum += x[i] * x[i];
#pragma unroll
      for (int d = 1; d < kGroup; d *= 2) sum += __shfl_xor(sum, d);
      const float by = 1.f / sqrtf(sum * (1.f / D) + a.eps);
#pragma unroll
      for (int i = 0; i < 16; i++) x[i] = x[i] * by * w[i];
    }
    if (turned) {
      const float *cs = &cosines[r][8 * lane], *sn = &sines[r][8 * lane];
      if (a.interleaved) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
          const float p = x[2 * i], q = x[2 * i + 1];
          x[2 * i] = p * cs[i] - q * sn[i];
          x[2 * i + 1] = q * cs[i] + p * sn[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; i++) {
          const float p = x[i], q = x[8 + i];
          x[i] = p * cs[i] - q * sn[i];
          x[8 + i] = q * cs[i] + p * sn[i];
        }
      }
    }
    if (on) {
      *(u32x4*)(to + 16 * c0) = pieces_of<E>(x);
      *(u32x4*)(to + 16 * c1) = pieces_of<E>(x + 8);
    }
  }
}

// ---------------------------------------------------------------------------
// Rows into the cache
// ---------------------------------------------------------------------------

__device__ inline float as_float(Bf16, uint32_t bits) { return __uint_as_float(bits << 16); }
__device__ inline float as_float(F16, uint32_t bits) { return (float)__builtin_bit_cast(_Float16, (uint16_t)bits); }

// 16 elements of a row, whose other half of a group of 32 the neighbouring lane has: the group's factor byte, and the
// elements divided by it.  Magnitudes of 16-bit floats order as their bits do.
template <class E>
__device__ inline uint32_t quantise(const u32x4 (&x)[2], u32x4& y) {
  u16x2 top{0, 0};
#pragma unroll
  for (int i = 0; i < 8; i++)
    top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, x[i / 4][i % 4] & 0x7FFF7FFFu));
  uint32_t most = top[0] > top[1] ? top[0] : top[1];
  uint32_t other = __shfl_xor(most, 1);
  most = most > other ? most : other;
  const bool odd = most >= E::kExp;  // NaN or infinities: the largest of the others counts
  if (__any(odd)) {
    if (odd) {
      most = 0;
#pragma unroll
      for (int i = 0; i < 16; i++) {
        const uint32_t m = x[i / 8][i / 2 % 4] >> 16 * (i % 2) & 0x7FFF;
        if (m < E::kExp && m > most) most = m;
      }
    }
    other = __shfl_xor(most, 1);
    most = most > other ? most : other;
  }
  const uint32_t bits = __float_as_uint(as_float(E(), most));
  const int32_t wanted = (int32_t)(bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000);  // 1.75 * 2^8 = 448
  const uint32_t byte = wanted < 27 ? 27 : wanted;
  const float by = __uint_as_float((254 - byte) << 23);
  float f[16];
  floats_of<E>(x[0], f);
  floats_of<E>(x[1], f + 8);
#pragma unroll
  for (int i = 0; i < 16; i++) f[i] *= by;
  // the type's largest numbers would round to one past its range: 256 times the largest factor
  const bool highest = byte >= (E::kExp == F16::kExp ? 135 : 247);
  if (__any(highest)) {
    if (highest)
#pragma unroll
      for (int i = 0; i < 16; i++) f[i] = f[i] > 240.f ? 240.f : f[i] < -240.f ? -240.f : f[i];
  }
#pragma unroll
  for (int i = 0; i < 4; i++) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i], f[4 * i + 1], 0, false);
    y[i] = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2], f[4 * i + 3], w, true);
  }
  if (__any(odd)) {
#pragma unroll
    for (int i = 0; i < 16; i++) {
      const uint32_t e = x[i / 8][i / 2 % 4] >> 16 * (i % 2) & 0xFFFF;
      if ((e & 0x7FFF) >= E::kExp) y[i / 4] = (y[i / 4] & ~(255u << 8 * (i % 4))) | (0x7Fu | (e >> 8 & 0x80)) << 8 * (i % 4);
    }
  }
  return byte;
}

// A thread quantises 16 elements of K and of V of one row; rows, heads and
// pieces in the order in which the sources have them, layers along the grid's
// second dimension.  A group of 32 elements is two neighbouring lanes'.  Bound
// by memory: 2.2 GB of prompts (16 requests, 32 layers of 8 heads of 128
// elements) take 0.61 ms, 5.4 TB/s read and written together.
template <class E>
__global__ __launch_bounds__(kThreads) void k_kv_append_quant(QuantAppendArgs a) {
  const uint32_t units = a.kv.head_dim / 16, per_row = units * a.kv.heads, groups = units / 2,
                 space = a.kv.head_dim == 256 ? 8 : 4;
  const uint64_t total = (uint64_t)a.n_slots * per_row;
  for (uint32_t l = blockIdx.y; l < a.n_layers; l += gridDim.y)
    for (uint64_t u = (uint64_t)blockIdx.x * kThreads + threadIdx.x; u < total; u += (uint64_t)gridDim.x * kThreads) {
      const uint32_t i = (uint32_t)(u / per_row), w = (uint32_t)(u - (uint64_t)i * per_row), h = w / units, c = w - h * units;
      const int64_t slot = a.slots[i];
      const uint64_t src = a.index ? a.index[i] : i;
      if (slot < 0 || (uint64_t)slot >> a.kv.block_shift >= a.kv.n_blocks || src >= a.src.n_rows) continue;
      const u32x4* k = (const u32x4*)((const uint8_t*)a.src.k + l * a.src.k_layer_stride + src * a.src.k_row_stride +
                                      h * a.src.k_head_stride + c * 32);
      const u32x4* v = (const u32x4*)((const uint8_t*)a.src.v + l * a.src.v_layer_stride + src * a.src.v_row_stride +
                                      h * a.src.v_head_stride + c * 32);
      const u32x4 kx[2] = {k[0], k[1]}, vx[2] = {v[0], v[1]};
      u32x4 ky, vy;
      const uint32_t kb = quantise<E>(kx, ky), vb = quantise<E>(vx, vy);
      const uint64_t layer = a.layer + l, block = (uint64_t)slot >> a.kv.block_shift,
                     token = (uint64_t)slot & ((1ull << a.kv.block_shift) - 1);
      uint8_t* to = a.kv.base + layer * a.kv.layer_stride + block * a.kv.block_stride + token * a.kv.token_stride +
                    h * a.kv.head_stride + c * 16;
      *(u32x4*)to = ky;
      *(u32x4*)(to + a.kv.v_off) = vy;
      if (c % 2 == 0) {
        uint8_t* f = a.scales.base + layer * a.scales.layer_stride + block * a.scales.block_stride +
                     token * a.scales.token_stride + h * a.scales.head_stride + c / 2;
        f[0] = (uint8_t)kb;
        f[a.scales.v_off] = (uint8_t)vb;
        if (c / 2 + groups < space) f[groups] = f[a.scales.v_off + groups] = 0;
      }
    }
}

// ---------------------------------------------------------------------------
// Cached tokens back in 16 bits
// ---------------------------------------------------------------------------

constexpr int kReadRows = 16;  // rows of a workgroup

// A workgroup finds out where its rows' tokens lie, then reads them, 16 elements of K and of V a thread.  Bound by memory: 16
// requests of 128-2048 tokens out of 16 layers of 8 heads of 128 elements (1.4 GB read and written) take 0.29 ms, 4.9 TB/s.
template <class E>
__global__ __launch_bounds__(kThreads) void k_kv_read_quant(QuantReadArgs p) {
  const gift_kv_read_args& a = p.a;
  __shared__ int64_t slots[kReadRows];  // -1: zeros, -2: left as it is
  const uint32_t tid = threadIdx.x, units = p.kv.head_dim / 16, per_row = units * p.kv.heads;
  const uint64_t row0 = p.row0 + (uint64_t)blockIdx.x * kReadRows;
  if (tid < kReadRows) {
    const uint64_t r = row0 + tid;
    int64_t slot = -2;
    if (r < a.n_rows) {
      uint32_t lo = 0, hi = a.n_reqs;  // the last request that begins at r or before it
      while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        if (a.row_begin[mid] <= r) lo = mid;
        else hi = mid;
      }
      const uint32_t begin = a.row_begin[lo];
      if (begin <= r && r < a.row_begin[lo + 1]) {
        slot = -1;
        const uint64_t token = (a.first ? a.first[lo] : 0) + (r - begin), most = (uint64_t)a.table_width << p.kv.block_shift;
        if ((!a.verdicts || a.verdicts[lo] == GIFT_SEG_OK) && token < a.lens[lo] && token < most) {
          const uint32_t id = a.tables[lo * a.table_stride + (token >> p.kv.block_shift)];
          if (id < p.kv.n_blocks)
            slot = ((int64_t)id << p.kv.block_shift) + (int64_t)(token & ((1ull << p.kv.block_shift) - 1));
        }
      }
    }
    slots[tid] = slot;
  }
  __syncthreads();
  for (uint32_t l = blockIdx.y; l < a.n_layers; l += gridDim.y) {
    const uint64_t layer = a.layer + l;
    for (uint64_t u = tid; u < (uint64_t)kReadRows * per_row; u += kThreads) {
      const uint32_t i = (uint32_t)(u / per_row), w = (uint32_t)(u - (uint64_t)i * per_row), h = w / units, c = w - h * units;
      const int64_t slot = slots[i];
      if (slot == -2) continue;
      u32x4 ky[2] = {}, vy[2] = {};
      if (slot >= 0) {
        const uint64_t block = (uint64_t)slot >> p.kv.block_shift, token = (uint64_t)slot & ((1ull << p.kv.block_shift) - 1);
        const uint8_t* from = p.kv.base + layer * p.kv.layer_stride + block * p.kv.block_stride + token * p.kv.token_stride +
                              h * p.kv.head_stride + c * 16;
        const uint8_t* f = p.scales.base + layer * p.scales.layer_stride + block * p.scales.block_stride +
                           token * p.scales.token_stride + h * p.scales.head_stride + c / 2;
        const u32x4 k = *(const u32x4*)from, v = *(const u32x4*)(from + p.kv.v_off);
        values_of<E>(k, factor(f[0], 0), ky);
        values_of<E>(v, factor(f[p.scales.v_off], 0), vy);
      }
      u32x4* k = (u32x4*)((uint8_t*)a.k + l * a.k_layer_stride + (row0 + i) * a.k_row_stride + h * a.k_head_stride + c * 32);
      u32x4* v = (u32x4*)((uint8_t*)a.v + l * a.v_layer_stride + (row0 + i) * a.v_row_stride + h * a.v_head_stride + c * 32);
      k[0] = ky[0];
      k[1] = ky[1];
      v[0] = vy[0];
      v[1] = vy[1];
    }
  }
}

template <class E>
hipError_t norm_rope(const gift_qk_rows& a, const RowsPlan& plan, hipStream_t s) {
  const uint32_t rows = plan.rows;
  const dim3 grid((uint32_t)((a.n_rows + rows - 1) / rows), plan.parts);
  switch (a.head_dim) {
    case 64: k_qk_norm_rope<E, 64><<<grid, kThreads, 0, s>>>(a, rows); break;
    case 96: k_qk_norm_rope<E, 96><<<grid, kThreads, 0, s>>>(a, rows); break;
    case 128: k_qk_norm_rope<E, 128><<<grid, kThreads, 0, s>>>(a, rows); break;
    default: k_qk_norm_rope<E, 256><<<grid, kThreads, 0, s>>>(a, rows);
  }
  return hipGetLastError();
}

// With 256 elements a wave takes all registers of its SIMD.
template <class E, int W>
hipError_t attend_rows_by_dim(const QuantAttnArgs& a, const AttnWork& w, hipStream_t s) {
  switch (a.kv.head_dim) {
    case 64: return attend_rows<E, Narrow<64, W>, 2>(a, w, s);
    case 96: return attend_rows<E, Narrow<96, W>, 2>(a, w, s);
    case 128: return attend_rows<E, Narrow<128, W>, 2>(a, w, s);
    default: return attend_rows<E, Narrow<256, 4>, 1>(a, w, s);
  }
}

// Up to 16 rows at a KV head on average the tiles are 16 columns wide (64 single tokens over 128-2048: 62 us with 32, 49
// with 16).  Two workgroups of four waves a CU, so that one's loads fill the other's changes of columns (49 us, with one of
// eight 64); where there are no more columns than CUs, one of eight, whose columns have fewer parts to join (one request of
// 8192 tokens: 20.7 with four, 17.8; of 131072 the same).
template <class E>
hipError_t attend_quantised(const QuantAttnArgs& a, const AttnWork& w, hipStream_t s) {
  const uint64_t rows = a.a.n_reqs ? (a.a.n_rows * a.group + a.a.n_reqs - 1) / a.a.n_reqs : 1;
  if (rows <= 16)
    return (uint64_t)a.a.n_reqs * a.kv.heads <= w.cus ? attend_rows_by_dim<E, 8>(a, w, s) : attend_rows_by_dim<E, 4>(a, w, s);
  return attend_by_dim<E>(a, w, s);
}

}  // namespace

RowsPlan qk_norm_rope_plan(const gift_qk_rows& a) {
  // Rows of a workgroup: about 100 heads, so that sines are made few times over and workgroups stay short, as long as there
  // are enough of them (17203 rows of 40 heads of 128: one row 86 us, two 72, three 73, eight 79; of 3 heads 20, 13, 13, 10).
  const uint64_t heads = (uint64_t)a.q_heads + a.k_heads, want = heads > 50 ? 2 : heads > 12 ? 100 / heads : kMostRows,
                 most = a.n_rows / 1024;
  const uint32_t rows = most < 1 ? 1 : (uint32_t)(most < want ? most : want);
  const uint32_t at_once = kThreads / (a.head_dim <= 64 ? 4 : a.head_dim <= 128 ? 8 : 16);
  const uint64_t items = rows * heads, parts = rows > 1 ? 1 : (items + at_once - 1) / at_once;
  return RowsPlan{rows, (uint32_t)(parts < 1024 ? parts : 1024), kMostGroups * rows};
}

hipError_t launch_qk_norm_rope(const gift_qk_rows& a, hipStream_t s) {
  const RowsPlan plan = qk_norm_rope_plan(a);
  for (uint64_t row = 0; row < a.n_rows; row += plan.launch) {
    auto from = [&](const void* p, uint64_t stride) -> void* { return p ? (uint8_t*)p + row * stride : nullptr; };
    gift_qk_rows b = a;
    b.n_rows = a.n_rows - row < plan.launch ? a.n_rows - row : plan.launch;
    b.q = from(a.q, a.q_row_stride);
    b.k = from(a.k, a.k_row_stride);
    b.q_out = from(a.q_out, a.q_out_row_stride);
    b.k_out = from(a.k_out, a.k_out_row_stride);
    b.positions = (const int32_t*)from(a.positions, 4);
    const hipError_t e = a.dtype == GIFT_BF16 ? norm_rope<Bf16>(b, plan, s) : norm_rope<F16>(b, plan, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_kv_append_quant(const QuantAppendArgs& a, uint32_t dtype, hipStream_t s) {
  const uint64_t units = (uint64_t)a.n_slots * a.kv.heads * (a.kv.head_dim / 16), blocks = (units + kThreads - 1) / kThreads;
  const dim3 grid((uint32_t)(blocks < 65536 ? blocks : 65536), a.n_layers < 65535 ? a.n_layers : 65535);
  if (dtype == GIFT_BF16)
    k_kv_append_quant<Bf16><<<grid, kThreads, 0, s>>>(a);
  else
    k_kv_append_quant<F16><<<grid, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

RowsPlan kv_read_quant_plan(const gift_kv_read_args& a) {
  return RowsPlan{(uint32_t)kReadRows, a.n_layers < 65535 ? a.n_layers : 65535, kMostGroups * kReadRows};
}

hipError_t launch_kv_read_quant(const QuantReadArgs& a, hipStream_t s) {
  const RowsPlan plan = kv_read_quant_plan(a.a);
  for (uint64_t row = 0; row < a.a.n_rows; row += plan.launch) {
    QuantReadArgs b = a;
    b.row0 = row;
    const uint64_t rows = a.a.n_rows - row < plan.launch ? a.a.n_rows - row : plan.launch;
    const dim3 grid((uint32_t)((rows + plan.rows - 1) / plan.rows), plan.parts);
    if (a.a.dtype == GIFT_BF16)
      k_kv_read_quant<Bf16><<<grid, kThreads, 0, s>>>(b);
    else
      k_kv_read_quant<F16><<<grid, kThreads, 0, s>>>(b);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_quant_attention(const QuantAttnArgs& a, uint32_t dtype, const AttnWork& w, hipStream_t s) {
  return dtype == GIFT_BF16 ? attend_quantised<Bf16>(a, w, s) : attend_quantised<F16>(a, w, s);
}

}  // namespace gift
