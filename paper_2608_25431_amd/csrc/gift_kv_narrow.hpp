// Attention of few rows over a quantised cache: up to 16 of a request at a KV head, which a single token with up to 16 query
// heads a KV head is.
#pragma once

#include "gift_kv_attention.hpp"

namespace gift {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef const __attribute__((address_space(1))) u32x2* global_halves;

__device__ inline f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mfma16(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// Over the four lanes that hold parts of one column: 16, 32 and 48 lanes on.
__device__ inline float max_of_quarters(float x) {
  x = max_of_halves(x);
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float sum_of_quarters(float x) {
  x += other_half(x);
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Waves that take a tile of 32 keys each in a round, all with the same 16 columns.
template <int D_, int W_>
struct Narrow {
  typedef QuantAttnArgs Args;
  static constexpr int D = D_, kCols = 16, kWaves = W_, kThreads = kWave * kWaves, kTiles = kWaves, kPieces = D / 8;
  // in token order, back to back: 64 single tokens over 128-2048 take 56 us with neighbours on one XCD and 50 without, one
  // over 131072 74 and 73
  static constexpr bool kNeighbours = false;
  static constexpr uint32_t kWhole = 20;
  static constexpr int kSteps = D / 32;                       // of 32 elements of a score's product
  static constexpr int kFull = D / 64, kHalf = D / 32 % 2;    // loads of 16 bytes and of 8 that a lane makes of a row
  static constexpr int kWords = D == 256 ? 2 : 1;             // of a row's factors
  static constexpr int kVRow = 2 * D + 32, kTileBytes = kTileKeys * kVRow;
  static constexpr int kAcc = D / 16;
  static constexpr int kState = kAcc * 1024 + 512;            // bytes of a wave's state in LDS
  static constexpr int kArea = kWaves * (kTileBytes > kState ? kTileBytes : kState);
  static constexpr size_t kPartial = kAcc * 1024 + 1024;
};

// As k_tree_attention, on tiles of 32 keys by 16 columns and the 16x16x32 matrix instructions.  A lane holds a
// quarter of the elements of two keys, whose addresses it works out itself: keys go from memory to the products in
// registers, since the order of elements in a product is free (the queries are read in the same order), and only V
// goes through LDS, to be transposed.
// Bound by memory: K and V of 131072 tokens (8 heads of 128 elements, 277 MB) take 62 us where a head's tokens follow each
// other and 73 where heads lie between them, call after call: 4.5 and 3.8 TB/s, 5.6 and 4.7 while keys are read (from 65536
// tokens to 131072), and about 13 us for the launch, the first loads and the joining of parts.  Of 64 single tokens over
// 128-2048 in token order (50 us) 194 MB come from memory where 155 are needed: 32 bytes hold a token's factors of all heads,
// and heads run on different XCDs, each of which fetches the line (head by head 164 MB and 47 us).
// In a kernel trace, where 131072 tokens with heads between take 82 us and 64 single ones 49: three workgroups a CU 104, loads
// that pass the caches 92; the next column's first loads ahead of this one's joining 51 to 54, cuts moved to columns' ends 51,
// no products and exponentials 47.
template <class E, class S, int MINW>
__global__ __launch_bounds__(S::kThreads, MINW) void k_quant_rows(QuantAttnArgs p, uint8_t* work) {
  typedef typename E::vec vec;
  const gift_tree_attention_args& a = p.a;
  __shared__ __align__(16) uint8_t area[S::kArea];
  __shared__ uint64_t sums[S::kWaves];
  __shared__ uint64_t found[2];
  __shared__ uint32_t last_one;
  const uint32_t tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave), col = lane % 16,
                 part = lane / 16;
  Cut cut;
  cut.n_wg = gridDim.x;
  cut.wg = blockIdx.x;
  if (!cut_work<S>(p, tid, wave, lane, sums, found, cut)) return;
  const uint32_t n_wg = cut.n_wg, wg = cut.wg;
  const uint64_t total = cut.total, first = cut.first, unit_end = cut.end;

  const float c = fmaxf(fabsf(a.scale) * 1.44269504f, 1.17549435e-38f);
  const uint32_t neg = a.scale < 0 ? 0x80008000u : 0u;
  uint32_t* counters = (uint32_t*)work;
  uint8_t* partials = work + 4 * kAttnCounters;
  // elements 8 of a step that this lane has of a row: of its piece of 16, or of 8 where half a piece is left
  auto element = [&](int s) -> uint32_t {
    return s / 2 < S::kFull ? s / 2 * 64 + part * 16 + s % 2 * 8 : S::kFull * 64 + part * 8;
  };

  // A column, and the rounds of it that this workgroup has.  (No member is smaller than a register: copies of padding end up
  // in memory, with all that goes with it.)
  struct Column {
    Req r;
    uint32_t b, g, ct, it0, it1;
    uint32_t live;  // there are keys to look at
  };
  uint32_t b0 = cut.b0, bi = cut.bi;  // bi: a request among those of said
  Said said = cut.said;               // of requests b0 + lane
  uint64_t base = cut.base;           // first unit of that request
  auto describe = [&](uint64_t unit) -> Column {
    Column x;
    x.r = req_at<S>(p, said, bi);
    while (unit >= base + (uint64_t)x.r.cols * cut.units(x.r)) {
      base += (uint64_t)x.r.cols * cut.units(x.r);
      if (++bi == kWave) {
        b0 += bi;
        bi = 0;
        said = said_of(p, b0 + lane);
      }
      x.r = req_at<S>(p, said, bi);
    }
    const Unit at = unit_of(unit - base, cut.units(x.r));
    const uint32_t column = __builtin_amdgcn_readfirstlane(at.column);
    x.b = b0 + bi;
    x.it0 = __builtin_amdgcn_readfirstlane(at.round);
    x.it1 = !cut.whole && unit_end - unit < x.r.rounds - x.it0 ? (uint32_t)(x.it0 + (unit_end - unit)) : x.r.rounds;
    x.g = __builtin_amdgcn_readfirstlane(quotient(column, x.r.col_tiles));
    x.ct = column - x.g * x.r.col_tiles;
    x.live = !x.r.dead && x.r.tiles;
    return x;
  };
  // this lane's query row of a column
  struct Query {
    bool live;
    uint32_t token, head;
    uint64_t row;
  };
  auto query_of = [&](const Column& y) -> Query {
    const uint32_t all = y.r.rows * p.group, at = y.ct * 16 + col;
    Query x;
    x.live = at < all;
    x.token = quotient(x.live ? at : 0, p.group);
    x.head = y.g * p.group + (x.live ? at - x.token * p.group : 0);
    x.row = y.r.row0 + x.token;
    return x;
  };
  // the workgroup that has a unit: most often this one
  auto owner = [&](uint64_t u) -> uint32_t {
    if (u >= first && u < unit_end) return wg;
    return n_wg == total ? (uint32_t)u : (uint32_t)quotient((u + 1) * n_wg - 1, total, 1.0 / (double)total);
  };
  auto place = [&](uint32_t w, uint32_t w0) -> uint64_t* {
    return (uint64_t*)(partials + (2 * w + (w == w0 ? 1 : 0)) * S::kPartial);
  };
  auto publish = [&](uint64_t* to, int t, const f32x4& x, float m, float l, int joined) {
#pragma unroll
    for (int h = 0; h < 2; h++)
      __hip_atomic_store(to + (t * 2 + h) * kWave + lane, __builtin_bit_cast(uint64_t, f32x2{x[2 * h], x[2 * h + 1]}),
                         __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (t == 0)
      __hip_atomic_store(to + (S::kAcc * 2 + joined) * kWave + lane, __builtin_bit_cast(uint64_t, f32x2{m, l}),
                         __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  };
  auto write = [&](const Query& q, int t, const f32x4& x, float m, float l) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    constexpr float kUnit = 1.f / (float)(1u << (int)E::kTop);
    typedef typename E::elem elem4 __attribute__((ext_vector_type(4)));
    elem4 y;
#pragma unroll
    for (int e = 0; e < 4; e++) y[e] = (typename E::elem)(x[e] * inv);
    *(elem4*)((uint8_t*)a.out + q.row * a.out_row_stride + q.head * a.out_head_stride + 32 * t + 8 * part) = y;
    if (a.lse && t == 0 && part == 0)
      a.lse[q.row * a.n_heads + q.head] = l == 0.f ? -INFINITY : (m * c + __builtin_amdgcn_logf(l * kUnit)) * 0.693147181f;
  };

  struct Keys {
    u32x4 full[2][S::kFull];
    u32x2 half[2];
  };
  Keys k, v;
  vec q[S::kSteps];
  const uint8_t* row[2];
  bool ok[2];
  uint32_t kf[2][S::kWords], vf[2][S::kWords], next[2];
  const uint32_t in_block = (1u << p.kv.block_shift) - 1;
  uint8_t* tile = area + wave * S::kTileBytes;
  for (uint64_t unit = first; unit < unit_end;) {
    const Column now = describe(unit);
    const Req& r = now.r;
    const Query qu = query_of(now);
    const uint32_t token = qu.token;
    const uint64_t qtok = qu.row;
    f32x4 o[S::kAcc];
    float m = -INFINITY, l = 0;  // what the weights refer to (an unscaled score), this lane's part of the sum of weights
#pragma unroll
    for (int t = 0; t < S::kAcc; t++) o[t] = f32x4{};
    if (now.live) {
      const uint32_t* tab = a.tables + (uint64_t)now.b * a.table_stride;
      const uint8_t *kbase = p.kv.base + a.layer * p.kv.layer_stride + now.g * p.kv.head_stride,
                    *fbase = p.scales.base + a.layer * p.scales.layer_stride + now.g * p.scales.head_stride;
      const int32_t own = (int32_t)(r.len - r.rows);  // the first of the rows' own tokens in the cache
      const uint32_t it0 = now.it0, it1 = now.it1;

      // the block ids of this lane's two keys of a round, asked for two rounds ahead
      auto ask = [&](uint32_t it, uint32_t (&id)[2]) {
#pragma unroll
        for (int b = 0; b < 2; b++) {
          const uint32_t j = (it * S::kTiles + wave) * kTileKeys + 16 * b + col;
          id[b] = *(it < it1 && j < r.len ? tab + (j >> p.kv.block_shift) : a.row_begin);  // no branch around the load
        }
      };
      auto locate = [&](uint32_t it, const uint32_t (&id)[2]) {
#pragma unroll
        for (int b = 0; b < 2; b++) {
          const uint32_t j = (it * S::kTiles + wave) * kTileKeys + 16 * b + col;
          ok[b] = it < it1 && j < r.len && id[b] < p.kv.n_blocks;
          row[b] = kbase + id[b] * p.kv.block_stride + (j & in_block) * p.kv.token_stride;
          const uint8_t* f = fbase + id[b] * p.scales.block_stride + (j & in_block) * p.scales.token_stride;
          const global_words kw = (global_words)(ok[b] ? f : (const uint8_t*)a.q),  // what may be read, of which nothing is used
              vw = (global_words)(ok[b] ? f + p.scales.v_off : (const uint8_t*)a.q);
#pragma unroll
          for (int i = 0; i < S::kWords; i++) kf[b][i] = kw[i], vf[b][i] = vw[i];
        }
      };
      auto fetch = [&](Keys& x, int64_t off) {
#pragma unroll
        for (int b = 0; b < 2; b++) {
          const global_bytes from = (global_bytes)(ok[b] ? row[b] + off : (const uint8_t*)a.q);
#pragma unroll
          for (int i = 0; i < S::kFull; i++) x.full[b][i] = *(global_pieces)(from + (ok[b] ? 64 * i + 16 * part : 0));
          if constexpr (S::kHalf) x.half[b] = *(global_halves)(from + (ok[b] ? 64 * S::kFull + 8 * part : 0));
        }
      };
      // elements of step s of key b in 16 bits
      auto operand = [&](const Keys& x, const uint32_t (&f)[2][S::kWords], int b, int s) -> u32x4 {
        u32x2 e;
        float by;
        if (s / 2 < S::kFull) {
          const u32x4 w = x.full[b][s / 2];
          e = s % 2 ? u32x2{w[2], w[3]} : u32x2{w[0], w[1]};
          by = factor(f[b][s / 4], s / 2 % 2 * 2 + part / 2);
        } else {
          e = x.half[b];
          by = factor(f[b][0], 2 * S::kFull);
        }
        return u32x4{E::template two<false>(e[0], by), E::template two<true>(e[0], by), E::template two<false>(e[1], by),
                     E::template two<true>(e[1], by)};
      };

      uint32_t id[2];
      ask(it0, id);
      ask(it0 + 1, next);
      {
        const uint8_t* from = (const uint8_t*)a.q + qtok * a.q_row_stride + qu.head * a.q_head_stride;
#pragma unroll
        for (int s = 0; s < S::kSteps; s++) q[s] = __builtin_bit_cast(vec, *(const u32x4*)(from + 2 * element(s)) ^ neg);
      }
      locate(it0, id);
      fetch(k, 0);
      fetch(v, p.kv.v_off);
      for (uint32_t it = it0;; it++) {
        const uint32_t t = it * S::kTiles + wave;
        const bool more = it + 1 < it1;
        const uint32_t exist = ((uint32_t)__ballot(ok[0]) & 0xFFFFu) | (uint32_t)__ballot(ok[1]) << 16;
        const bool was[2] = {ok[0], ok[1]};
        uint32_t factors[2][S::kWords];
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
          for (int i = 0; i < S::kWords; i++) factors[b][i] = vf[b][i];
        f32x4 sc[2] = {f32x4{}, f32x4{}};
#pragma unroll
        for (int s = 0; s < S::kSteps; s++)
#pragma unroll
          for (int b = 0; b < 2; b++) sc[b] = mfma16(__builtin_bit_cast(vec, operand(k, kf, b, s)), q[s], sc[b]);
        if (more) {
          id[0] = next[0], id[1] = next[1];
          ask(it + 2, next);
          locate(it + 1, id);
          fetch(k, 0);
        }

        // V to LDS, in 16 bits
        const bool draft = (a.mask || r.rows > 1) && (own < 0 || t * kTileKeys + kTileKeys > (uint32_t)own);
        uint32_t odd = 0;  // keys of the rows' own tokens whose V is not finite: only for the rows that see them
        {
          u32x4 wide[2][2 * S::kFull + S::kHalf];
#pragma unroll
          for (int b = 0; b < 2; b++)
#pragma unroll
            for (int s = 0; s < S::kSteps; s++) wide[b][s] = operand(v, factors, b, s);
          if (exist != ~0u) {  // weights of zero times NaN would reach every row
#pragma unroll
            for (int b = 0; b < 2; b++)
#pragma unroll
              for (int s = 0; s < S::kSteps; s++)
                if (!was[b]) wide[b][s] = u32x4{0, 0, 0, 0};
          }
          if (draft) {
#pragma unroll
            for (int b = 0; b < 2; b++) {
              u16x2 top{0, 0};
#pragma unroll
              for (int s = 0; s < S::kSteps; s++)
#pragma unroll
                for (int e = 0; e < 4; e++)
                  top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, wide[b][s][e] & (E::kExp * 0x10001u)));
              const uint32_t j = t * kTileKeys + 16 * b + col;
              uint64_t x = __ballot((top[0] == E::kExp || top[1] == E::kExp) && (own < 0 || j >= (uint32_t)own));
              x |= x >> 32;
              x |= x >> 16;
              odd |= ((uint32_t)x & 0xFFFFu) << 16 * b;
            }
            if (odd) {
#pragma unroll
              for (int b = 0; b < 2; b++)
#pragma unroll
                for (int s = 0; s < S::kSteps; s++)
                  if (odd >> (16 * b + col) & 1) wide[b][s] = u32x4{0, 0, 0, 0};
            }
          }
#pragma unroll
          for (int b = 0; b < 2; b++)
#pragma unroll
            for (int s = 0; s < S::kSteps; s++) *(u32x4*)(tile + (16 * b + col) * S::kVRow + 2 * element(s)) = wide[b][s];
        }
        if (more) fetch(v, p.kv.v_off);

        // scores to weights
        uint32_t see = exist;
        const int32_t from = (int32_t)(t * kTileKeys) - own;  // the tile's first key among the rows' own
        if (from > -kTileKeys) {
          if (a.mask) {
            const uint32_t *words = a.mask + qtok * a.mask_words, by = from & 31;
            const int32_t w = from >> 5;  // -1: the tile begins before the rows' own
            const uint32_t lower = w < 0 ? ~0u : (uint32_t)w < a.mask_words ? words[w] : 0u,
                           upper = (uint32_t)(w + 1) < a.mask_words ? words[w + 1] : 0u;
            see &= by ? lower >> by | upper << (32 - by) : lower;
          } else {
            const int32_t ahead = (int32_t)token - from;  // keys behind the tile's first that the row sees
            see &= ahead >= kTileKeys - 1 ? ~0u : ahead < 0 ? 0u : (2u << ahead) - 1;
          }
        }
        if (__any(see != ~0u)) {
          const uint32_t mine = see >> 4 * part;
#pragma unroll
          for (int b = 0; b < 2; b++)
#pragma unroll
            for (int i = 0; i < 4; i++)
              if (!(mine >> (16 * b + i) & 1)) sc[b][i] = -INFINITY;
        }
        float top = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])),
                          fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
        top = max_of_quarters(top);
        // What weights refer to stays while no score passes it by kSlack octaves.  A column's own scores decide, so that a
        // row's bits do not depend on the rows beside it.
        const bool grow = (top - m) * c > E::kSlack;
        const float mn = grow ? top : m, safe = mn == -INFINITY ? 0.f : mn;
        if (__any(grow)) {
          const float f = exp2f((m - safe) * c);
          l *= f;
#pragma unroll
          for (int d = 0; d < S::kAcc; d++) o[d] *= f;
          m = mn;
        }
        float shift = -safe * c;
        const bool far = fabsf(shift) > kFarShift;
        if (E::kTop != 0.f && !far) shift += E::kTop;
        float left = 0;
        if (__any(far)) left = far ? __builtin_fmaf(safe, c, shift) - E::kTop : 0.f;  // what the product's rounding left out
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
          for (int i = 0; i < 4; i++) sc[b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][i], c, shift) - left);
        l += ((sc[0][0] + sc[0][1]) + (sc[0][2] + sc[0][3])) + ((sc[1][0] + sc[1][1]) + (sc[1][2] + sc[1][3]));
        while (odd) {
          const uint32_t key = __builtin_ctz(odd);
          odd &= odd - 1;
          float mine = 0;
#pragma unroll
          for (int b = 0; b < 2; b++)
#pragma unroll
            for (int i = 0; i < 4; i++)
              if ((uint32_t)(16 * b + i) == (key & ~12u)) mine = sc[b][i];
          const float weight = __shfl(mine, (key / 4 % 4) * 16 + col);
          const uint32_t pos = t * kTileKeys + key, block = tab[pos >> p.kv.block_shift], slot = pos & in_block;
          const uint8_t *vp = kbase + p.kv.v_off + block * p.kv.block_stride + slot * p.kv.token_stride,
                        *f = fbase + p.scales.v_off + block * p.scales.block_stride + slot * p.scales.token_stride;
          if (see >> key & 1) {
#pragma unroll
            for (int d = 0; d < S::kAcc; d++) {
              typedef typename E::elem elem2 __attribute__((ext_vector_type(2)));
              const uint32_t x = *(const uint32_t*)(vp + 16 * d + 4 * part);
              const float by = factor(f[d / 2], 0);
              const elem2 lower = __builtin_bit_cast(elem2, E::template two<false>(x, by)),
                          upper = __builtin_bit_cast(elem2, E::template two<true>(x, by));
              o[d] += weight * f32x4{(float)lower[0], (float)lower[1], (float)upper[0], (float)upper[1]};
            }
          }
        }

        // V^T P^T: a lane's weights are those of keys 4 part .. 4 part + 3 and of the same behind 16
        f32x16 weights;  // of which the first half is in use
#pragma unroll
        for (int i = 0; i < 8; i++) weights[i] = sc[i / 4][i % 4];
        vec w[E::kParts];
        E::parts(weights, 0, w);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        typedef __attribute__((address_space(3))) s16x4 lds4;
        union Frag {
          s16x4 x[2];
          vec v;
        };
        const uint8_t* vrow = tile + (4 * part + col / 4) * S::kVRow + col % 4 * 8;
#pragma unroll
        for (int d = 0; d < S::kAcc; d++) {
          Frag u;
          u.x[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(vrow + 32 * d));
          u.x[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(vrow + 32 * d + 16 * S::kVRow));
#pragma unroll
          for (int e = 0; e < E::kParts; e++) o[d] = mfma16(u.v, w[e], o[d]);
        }
        if (!more) break;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
      l = sum_of_quarters(l);
    }

    // The column's states go to LDS, and from there each wave takes every kWaves-th 16 elements of D.
    __syncthreads();
    {
      f32x4* to = (f32x4*)(area + wave * S::kState);
#pragma unroll
      for (int t = 0; t < S::kAcc; t++) to[t * kWave + lane] = o[t];
      ((f32x2*)(to + S::kAcc * kWave))[lane] = f32x2{m, l};
    }
    __syncthreads();
    auto state = [&](int k) { return (const f32x4*)(area + k * S::kState); };
    m = -INFINITY, l = 0;
    f32x2 ml[S::kWaves];
#pragma unroll
    for (int k = 0; k < S::kWaves; k++) {
      ml[k] = ((const f32x2*)(state(k) + S::kAcc * kWave))[lane];
      m = fmaxf(m, ml[k][0]);
    }
    {
      const float safe = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int k = 0; k < S::kWaves; k++) {
        ml[k][0] = exp2f((ml[k][0] - safe) * c);  // the state's factor
        l += ml[k][1] * ml[k][0];
      }
    }
    auto chunk = [&](int t) -> f32x4 {
      f32x4 x = f32x4{};
#pragma unroll
      for (int k = 0; k < S::kWaves; k++) x += state(k)[t * kWave + lane] * ml[k][0];
      return x;
    };
    const uint64_t col_first = unit - now.it0;
    const uint32_t w0 = owner(col_first), parts = owner(col_first + cut.units(r) - 1) - w0 + 1;
    if (qu.live)
#pragma unroll 1
      for (int t = wave; t < S::kAcc; t += S::kWaves)
        if (parts == 1)
          write(qu, t, chunk(t), m, l);
        else
          publish(place(wg, w0), t, chunk(t), m, l, 0);
    if (parts > 1) {
      // Parts are joined as in k_tree_attention, by the workgroup that finishes last, many of them in two steps.
      const uint32_t run = parts <= 8 ? parts : parts <= 64 ? 8 : parts <= 256 ? 16 : 64;
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
      // n published states, of every step-th workgroup from w on, in that order
      uint32_t w = w0 + (wg - w0) / run * run, n = w0 + parts - w < run ? w0 + parts - w : run, step = 1;
      uint32_t* counter = run == parts ? counters + w0 : counters + kAttnCounters / 4 + 2 * w + (w == w0 ? 1 : 0);
      while (last_of(counter, n)) {
        const bool whole = run == parts || step == run;
        if (qu.live)
#pragma unroll 1
          for (int t = wave; t < S::kAcc; t += S::kWaves) {
            constexpr uint32_t kAhead = 8;  // states on their way at a time
            float m = -INFINITY, l = 0;
            f32x4 z = f32x4{};
#pragma unroll 1
            for (uint32_t j = 0; j < n; j += kAhead) {
              f32x2 y[kAhead][2], ml[kAhead];
#pragma unroll
              for (uint32_t u = 0; u < kAhead; u++) {
                const uint64_t* from = place(w + (j + u < n ? j + u : n - 1) * step, w0);
                ml[u] = published(from + (S::kAcc * 2 + (step > 1)) * kWave + lane);
#pragma unroll
                for (int h = 0; h < 2; h++) y[u][h] = published(from + (t * 2 + h) * kWave + lane);
              }
              float mn = m;
#pragma unroll
              for (uint32_t u = 0; u < kAhead; u++) mn = fmaxf(mn, ml[u][0]);
              const float safe = mn == -INFINITY ? 0.f : mn, f0 = exp2f((m - safe) * c);
              l *= f0;
              z *= f0;
              m = mn;
#pragma unroll
              for (uint32_t u = 0; u < kAhead; u++)
                if (j + u < n) {
                  const float f = exp2f((ml[u][0] - safe) * c);
                  l += ml[u][1] * f;
                  z += f32x4{y[u][0][0], y[u][0][1], y[u][1][0], y[u][1][1]} * f;
                }
            }
            // a run's elements take the place of its first part's, which no other wave reads
            if (whole)
              write(qu, t, z, m, l);
            else
              publish(place(w, w0), t, z, m, l, 1);
          }
        if (whole) break;
        w = w0;
        n = (parts + run - 1) / run;
        step = run;
        counter = counters + w0;
      }
    }
    __syncthreads();
    unit += cut.whole ? 1 : now.it1 - now.it0;
  }
}

template <class E, class S, int MINW>
hipError_t attend_rows(const QuantAttnArgs& a, const AttnWork& w, hipStream_t s) {
  uint32_t grid = w.cus * (4 * MINW / S::kWaves);  // as many workgroups as run at once: MINW waves on each SIMD, four SIMDs
  if (2 * grid * S::kPartial > w.partial_bytes || grid > kAttnCounters / 4) return hipErrorInvalidValue;
  // and no more than the lengths can give work to, as far as the host knows them
  const uint64_t tiles = ((uint64_t)a.a.table_width << a.kv.block_shift) / kTileKeys + 2,
                 cols = (uint64_t)a.kv.heads * (a.a.n_rows * a.group / S::kCols + a.a.n_reqs), rounds = tiles / S::kTiles + 1;
  if (cols < grid && cols * rounds < grid) grid = cols * rounds ? (uint32_t)(cols * rounds) : 1;
  QuantAttnArgs b = a;
  b.most_wg = grid;
  k_quant_rows<E, S, MINW><<<grid_of_columns<S>(a, grid, cols), S::kThreads, 0, s>>>(b, w.mem);
  return hipGetLastError();
}

}  // namespace
}  // namespace gift
