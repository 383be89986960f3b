// Host side of include/gift_kv.h: argument checks and launches.  Everything
// that depends on lengths, tables, slots or masks happens in the kernels of
// gift_kv.hip; nothing is allocated, staged or waited for in a call, so a
// call costs one kernel launch and may be captured.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdio.h>

#include <algorithm>
#include <new>

#include "gift.h"
#include "gift_kv.h"
#include "gift_kv_internal.hpp"

using namespace gift;

struct gift_attention_work_s {
  int device;
  AttnWork w;
};

namespace {

bool mul_ok(uint64_t a, uint64_t b, uint64_t* r) { return !__builtin_mul_overflow(a, b, r); }
bool add_ok(uint64_t a, uint64_t b, uint64_t* r) { return !__builtin_add_overflow(a, b, r); }

bool pow2(uint64_t x) { return x != 0 && (x & (x - 1)) == 0; }

bool unaligned(const void* p, uint32_t to = 16) { return ((uintptr_t)p & (to - 1)) != 0; }

// A strided array in memory: count[d] steps of stride[d] bytes around rows of
// row bytes.  False where the last byte's offset does not fit 64 bits.
struct Strided {
  const void* p;
  uint64_t row;
  uint64_t count[3], stride[3];
  bool extent(uint64_t* bytes) const {
    *bytes = row;
    for (int d = 0; d < 3; d++) {
      uint64_t span;
      if (count[d] == 0) {
        *bytes = 0;
        return true;
      }
      if (!mul_ok(stride[d], count[d] - 1, &span) || !add_ok(*bytes, span, bytes)) return false;
    }
    return (uintptr_t)p <= UINT64_MAX - *bytes;
  }
};

bool overlap(const void* a, uint64_t na, const void* b, uint64_t nb) {
  return na && nb && (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}

struct Range {
  const void* p;
  uint64_t n;  // bytes
};

bool overlap(const Range& a, const Range& b) { return overlap(a.p, a.n, b.p, b.n); }

// Rules of gift_kv_format within a gift_paged_kv; fills the kernels' view.
gift_status check_format(const gift_paged_kv* kv, const gift_kv_format* f, KvView* view) {
  if (!kv || !f) return report(GIFT_E_INVALID, "null cache description or format");
  gift_status s = paged_geometry(kv);
  if (s != GIFT_OK) return s;
  if (f->dtype != GIFT_BF16 && f->dtype != GIFT_F16) return report(GIFT_E_INVALID, "format: unknown dtype");
  if (f->n_heads == 0) return report(GIFT_E_INVALID, "format: n_heads must be >= 1");
  if (f->head_dim != 64 && f->head_dim != 96 && f->head_dim != 128 && f->head_dim != 256)
    return report(GIFT_E_INVALID, "format: head_dim must be 64, 96, 128 or 256");
  if (!pow2(f->block_tokens)) return report(GIFT_E_INVALID, "format: block_tokens must be a power of two");
  if ((f->k_offset | f->v_offset | f->token_stride | f->head_stride) & 15u)
    return report(GIFT_E_INVALID, "format: offsets and strides must be multiples of 16");
  const uint64_t row = 2ull * f->head_dim;
  Strided rows{nullptr, row, {f->block_tokens, f->n_heads, 1}, {f->token_stride, f->head_stride, 0}};
  uint64_t extent;
  if (!rows.extent(&extent)) return report(GIFT_E_INVALID, "format: rows exceed the chunk");
  for (uint64_t off : {f->k_offset, f->v_offset}) {
    uint64_t part = 0, end;
    if (kv->n_parts > 1) part = std::min<uint64_t>(off / kv->part_stride, kv->n_parts - 1);
    if (!add_ok(off - part * kv->part_stride, extent, &end) || end > kv->chunk_bytes)
      return report(GIFT_E_INVALID, "format: rows exceed the chunk");
  }
  struct Dim {
    uint64_t stride, count;
  } d[3] = {{f->token_stride, f->block_tokens},
            {f->head_stride, f->n_heads},
            {f->k_offset < f->v_offset ? f->v_offset - f->k_offset : f->k_offset - f->v_offset, 2}};
  std::sort(d, d + 3, [](const Dim& x, const Dim& y) { return x.stride < y.stride; });
  uint64_t inner = row;
  for (const Dim& x : d) {
    if (x.count <= 1) continue;
    if (x.stride < inner) return report(GIFT_E_INVALID, "format: rows of a block overlap");
    inner += x.stride * (x.count - 1);  // within a chunk or two: fits
  }
  uint64_t end = kv->chunk_bytes, span;
  if (!mul_ok(kv->layer_stride, kv->n_layers - 1, &span) || !add_ok(end, span, &end) ||
      !mul_ok(kv->block_stride, kv->n_blocks - 1, &span) || !add_ok(end, span, &end) ||
      !mul_ok(kv->part_stride, kv->n_parts - 1, &span) || !add_ok(end, span, &end) || end > kv->cache_bytes)
    return report(GIFT_E_RANGE, "paged: chunks exceed cache_bytes");
  view->base = (uint8_t*)kv->base + f->k_offset;
  view->v_off = (int64_t)f->v_offset - (int64_t)f->k_offset;
  view->layer_stride = kv->layer_stride;
  view->block_stride = kv->block_stride;
  view->token_stride = f->token_stride;
  view->head_stride = f->head_stride;
  view->n_blocks = kv->n_blocks;
  view->n_layers = kv->n_layers;
  view->heads = f->n_heads;
  view->head_dim = f->head_dim;
  view->block_shift = (uint32_t)__builtin_ctz(f->block_tokens);
  return GIFT_OK;
}

constexpr uint64_t kMost = 0x7FFFFFFFull;  // rows, slots and cached tokens of a request

}  // namespace

extern "C" {

gift_status gift_kv_tables(const gift_kv_step* step, hipStream_t stream) {
  clear_error();
  if (!step) return report(GIFT_E_INVALID, "null step");
  const gift_kv_step& s = *step;
  if (!pow2(s.block_tokens)) return report(GIFT_E_INVALID, "block_tokens must be a power of two");
  if (!s.row_begin || !s.taken) return report(GIFT_E_INVALID, "null row_begin or taken");
  if (s.n_reqs && (!s.users || !s.lens || !s.new_lens || !s.lens_out || !s.verdicts))
    return report(GIFT_E_INVALID, "null users, lens, new_lens, lens_out or verdicts");
  if (s.n_reqs && (s.table_width == 0 || !s.tables || !s.block_labels || s.n_blocks == 0))
    return report(GIFT_E_INVALID, "null or empty tables or block_labels");
  if (s.n_reqs && s.table_stride < s.table_width) return report(GIFT_E_INVALID, "table_stride below table_width");
  if ((s.n_free && !s.free_blocks) || (s.n_slots && !s.slots))
    return report(GIFT_E_INVALID, "null free_blocks or slots");
  uint64_t tokens, entries = 0;
  if (!mul_ok(s.table_width, s.block_tokens, &tokens) || tokens > kMost)
    return report(GIFT_E_TOO_LARGE, "table_width * block_tokens exceeds 2^31 - 1");
  if (s.n_slots > kMost) return report(GIFT_E_TOO_LARGE, "n_slots exceeds 2^31 - 1");
  if (s.n_reqs > kMost) return report(GIFT_E_TOO_LARGE, "n_reqs exceeds 2^31 - 1");
  if (s.n_reqs && (!mul_ok(s.table_stride, s.n_reqs - 1, &entries) || !add_ok(entries, s.table_width, &entries) ||
                   entries > UINT64_MAX / 4 || s.n_blocks > UINT64_MAX / 4))
    return report(GIFT_E_INVALID, "table sizes overflow");
  const uint64_t per = 4ull * s.n_reqs;
  const Range in[] = {{s.users, per}, {s.lens, per}, {s.new_lens, per}, {s.free_blocks, 4ull * s.n_free}},
              out[] = {{s.tables, 4 * entries}, {s.block_labels, 4 * s.n_blocks}, {s.slots, 8 * s.n_slots},
                       {s.row_begin, per + 4},  {s.lens_out, per},                {s.taken, 4},
                       {s.verdicts, per}};
  const int n_out = (int)(sizeof out / sizeof out[0]);
  for (const Range& r : in)
    if (r.n && unaligned(r.p, 4)) return report(GIFT_E_INVALID, "an array is not aligned to its elements");
  for (const Range& r : out)
    if (r.n && unaligned(r.p, r.p == s.slots ? 8 : 4))
      return report(GIFT_E_INVALID, "an array is not aligned to its elements");
  for (int i = 0; i < n_out; i++) {
    for (const Range& r : in)
      if (overlap(out[i], r)) return report(GIFT_E_INVALID, "an output overlaps an input");
    for (int j = 0; j < i; j++)
      if (overlap(out[i], out[j])) return report(GIFT_E_INVALID, "outputs overlap");
  }
  hipError_t e = launch_kv_tables(TablesArgs{s, (uint32_t)__builtin_ctz(s.block_tokens)}, stream);
  return e == hipSuccess ? GIFT_OK : report_hip(e, "kv_tables");
}

gift_status gift_kv_append(const gift_paged_kv* kv, const gift_kv_format* format, const int64_t* slots,
                           uint64_t n_slots, const uint32_t* index, const gift_kv_rows* rows, hipStream_t stream) {
  clear_error();
  AppendArgs a;
  gift_status st = check_format(kv, format, &a.kv);
  if (st != GIFT_OK) return st;
  if (!rows) return report(GIFT_E_INVALID, "null rows");
  if (n_slots > kMost || rows->n_rows > kMost) return report(GIFT_E_TOO_LARGE, "more than 2^31 - 1 slots or rows");
  if (n_slots && !slots) return report(GIFT_E_INVALID, "null slots");
  if (n_slots && (unaligned(slots, 8) || unaligned(index, 4)))
    return report(GIFT_E_INVALID, "slots or index not aligned to its elements");
  if (overlap(slots, 8 * n_slots, kv->base, kv->cache_bytes) ||
      (index && overlap(index, 4 * n_slots, kv->base, kv->cache_bytes)))
    return report(GIFT_E_INVALID, "slots or index overlaps the cache");
  if (n_slots && rows->n_rows) {
    if (!rows->k || !rows->v || unaligned(rows->k) || unaligned(rows->v))
      return report(GIFT_E_INVALID, "k or v null or not 16-byte aligned");
    if ((rows->k_layer_stride | rows->k_row_stride | rows->k_head_stride | rows->v_layer_stride | rows->v_row_stride |
         rows->v_head_stride) & 15u)
      return report(GIFT_E_INVALID, "strides of k and v must be multiples of 16");
    const uint64_t row = 2ull * a.kv.head_dim;
    const Strided src[2] = {
        {rows->k, row, {a.kv.n_layers, rows->n_rows, a.kv.heads}, {rows->k_layer_stride, rows->k_row_stride, rows->k_head_stride}},
        {rows->v, row, {a.kv.n_layers, rows->n_rows, a.kv.heads}, {rows->v_layer_stride, rows->v_row_stride, rows->v_head_stride}}};
    for (const Strided& x : src) {
      uint64_t n;
      if (!x.extent(&n)) return report(GIFT_E_INVALID, "sizes of k and v overflow");
      if (overlap(x.p, n, kv->base, kv->cache_bytes)) return report(GIFT_E_INVALID, "k or v overlaps the cache");
    }
  }
  if (n_slots == 0 || rows->n_rows == 0) return GIFT_OK;
  a.src = *rows;
  a.slots = slots;
  a.index = index;
  a.n_slots = (uint32_t)n_slots;
  hipError_t e = launch_kv_append(a, stream);
  return e == hipSuccess ? GIFT_OK : report_hip(e, "kv_append");
}

gift_status gift_attention_work_create(hipStream_t stream, gift_attention_work* out) {
  clear_error();
  if (!out) return report(GIFT_E_INVALID, "null out");
  *out = nullptr;
  int dev;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return report_hip(e, "hipGetDevice");
  hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
  e = hipStreamIsCapturing(stream, &capture);
  if (e != hipSuccess) return report_hip(e, "hipStreamIsCapturing");
  // an allocation and a synchronisation would end the capture
  if (capture != hipStreamCaptureStatusNone) return report(GIFT_E_INVALID, "the stream is being captured");
  int cus = 0;
  e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
  if (e != hipSuccess) return report_hip(e, "hipDeviceGetAttribute");
  if (cus < 1) cus = 1;
  if (cus > (int)kAttnCounters / 8) cus = kAttnCounters / 8;  // two workgroups a CU at most
  gift_attention_work w = new (std::nothrow) gift_attention_work_s{dev, {nullptr, (uint32_t)cus, 2 * kAttnPlace * cus}};
  if (!w) return report(GIFT_E_NOMEM, "host memory");
  const size_t counters = 4ull * kAttnCounters;
  e = hipMalloc((void**)&w->w.mem, counters + w->w.partial_bytes);
  if (e != hipSuccess) {
    delete w;
    return report_hip(e, "attention workspace");
  }
  e = hipMemsetAsync(w->w.mem, 0, counters, stream);
  if (e == hipSuccess) e = hipStreamSynchronize(stream);
  if (e != hipSuccess) {
    (void)hipFree(w->w.mem);
    delete w;
    return report_hip(e, "attention workspace");
  }
  *out = w;
  return GIFT_OK;
}

gift_status gift_attention_work_destroy(gift_attention_work w) {
  clear_error();
  if (!w) return GIFT_OK;
  int dev;
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess && dev != w->device) e = hipSetDevice(w->device);
  if (e == hipSuccess) e = hipDeviceSynchronize();
  hipError_t f = hipFree(w->w.mem);
  if (e == hipSuccess && dev != w->device) e = hipSetDevice(dev);
  delete w;
  if (e == hipSuccess) e = f;
  return e == hipSuccess ? GIFT_OK : report_hip(e, "attention workspace");
}

gift_status gift_tree_attention(gift_attention_work work, const gift_paged_kv* kv, const gift_kv_format* format,
                                const gift_tree_attention_args* args, hipStream_t stream) {
  clear_error();
  if (!work || !args) return report(GIFT_E_INVALID, "null workspace or arguments");
  AttnArgs a;
  gift_status st = check_format(kv, format, &a.kv);
  if (st != GIFT_OK) return st;
  const gift_tree_attention_args& g = *args;
  if (g.n_heads == 0 || g.n_heads % a.kv.heads)
    return report(GIFT_E_INVALID, "n_heads must be a multiple of the format's n_heads");
  if (g.layer >= a.kv.n_layers) return report(GIFT_E_INVALID, "layer past the cache's layers");
  if (!isfinite(g.scale)) return report(GIFT_E_INVALID, "scale must be finite");
  if (g.n_rows > kMost) return report(GIFT_E_TOO_LARGE, "more than 2^31 - 1 rows");
  uint64_t tokens, heads_rows;
  if (!mul_ok(g.table_width, format->block_tokens, &tokens) || tokens > kMost)
    return report(GIFT_E_TOO_LARGE, "table_width * block_tokens exceeds 2^31 - 1");
  if (!mul_ok(g.n_rows, g.n_heads, &heads_rows) || heads_rows > UINT32_MAX)
    return report(GIFT_E_TOO_LARGE, "n_rows * n_heads exceeds 2^32 - 1");
  if (g.n_reqs > kMost) return report(GIFT_E_TOO_LARGE, "n_reqs exceeds 2^31 - 1");
  if (g.n_reqs && (!g.row_begin || !g.lens)) return report(GIFT_E_INVALID, "null row_begin or lens");
  if (g.n_reqs && g.table_width && !g.tables) return report(GIFT_E_INVALID, "null tables");
  if (g.n_reqs && g.table_stride < g.table_width) return report(GIFT_E_INVALID, "table_stride below table_width");
  if (!g.k != !g.v) return report(GIFT_E_INVALID, "k and v must both be given or both be NULL");
  if (g.mask && g.mask_words == 0) return report(GIFT_E_INVALID, "mask_words must be >= 1 with a mask");
  for (const void* p : {(const void*)g.lse, (const void*)g.row_begin, (const void*)g.lens, (const void*)g.tables,
                        (const void*)g.mask, (const void*)g.verdicts})
    if (unaligned(p, 4)) return report(GIFT_E_INVALID, "an array is not aligned to its elements");
  if (g.n_rows) {
    if (!g.q || !g.out || unaligned(g.q) || unaligned(g.k) || unaligned(g.v) || unaligned(g.out))
      return report(GIFT_E_INVALID, "q, k, v or out null or not 16-byte aligned");
    if ((g.q_row_stride | g.q_head_stride | g.out_row_stride | g.out_head_stride) & 15u)
      return report(GIFT_E_INVALID, "strides of q and out must be multiples of 16");
    if (g.k && ((g.k_row_stride | g.k_head_stride | g.v_row_stride | g.v_head_stride) & 15u))
      return report(GIFT_E_INVALID, "strides of k and v must be multiples of 16");
    const uint64_t row = 2ull * a.kv.head_dim, rows = g.n_rows, kvh = g.k ? a.kv.heads : 0;
    uint64_t n_out, n;
    const Strided out{g.out, row, {rows, g.n_heads, 1}, {g.out_row_stride, g.out_head_stride, 0}};
    if (!out.extent(&n_out)) return report(GIFT_E_INVALID, "size of out overflows");
    uint64_t lo = std::min(g.out_row_stride, g.out_head_stride), lo_n = rows, hi = g.out_head_stride, hi_n = g.n_heads;
    if (g.out_head_stride < g.out_row_stride) lo_n = g.n_heads, hi = g.out_row_stride, hi_n = rows;
    if ((lo_n > 1 && lo < row) || (hi_n > 1 && hi < row + (lo_n > 1 ? lo * (lo_n - 1) : 0)))
      return report(GIFT_E_INVALID, "rows of out overlap");
    if (overlap(out.p, n_out, kv->base, kv->cache_bytes)) return report(GIFT_E_INVALID, "out overlaps the cache");
    const Range lse{g.lse, g.lse ? 4 * heads_rows : 0};
    if (overlap(lse, Range{kv->base, kv->cache_bytes}) || overlap(lse, Range{g.out, n_out}))
      return report(GIFT_E_INVALID, "lse overlaps out or the cache");
    const Strided in[3] = {{g.q, row, {rows, g.n_heads, 1}, {g.q_row_stride, g.q_head_stride, 0}},
                           {g.k, row, {rows, kvh, 1}, {g.k_row_stride, g.k_head_stride, 0}},
                           {g.v, row, {rows, kvh, 1}, {g.v_row_stride, g.v_head_stride, 0}}};
    for (const Strided& x : in) {
      if (!x.extent(&n)) return report(GIFT_E_INVALID, "sizes of q, k or v overflow");
      if (overlap(out.p, n_out, x.p, n)) return report(GIFT_E_INVALID, "out overlaps q, k or v");
      if (overlap(lse, Range{x.p, n})) return report(GIFT_E_INVALID, "lse overlaps q, k or v");
    }
    uint64_t entries = 0, words = 0;
    if (g.n_reqs && g.table_width &&
        (!mul_ok(g.table_stride, g.n_reqs - 1, &entries) || !add_ok(entries, g.table_width, &entries)))
      return report(GIFT_E_INVALID, "sizes overflow");
    if (g.mask && !mul_ok(rows, g.mask_words, &words)) return report(GIFT_E_INVALID, "sizes overflow");
    if (entries > UINT64_MAX / 4 || words > UINT64_MAX / 4) return report(GIFT_E_INVALID, "sizes overflow");
    const uint64_t per = 4ull * g.n_reqs;
    for (const Range& r : {Range{g.row_begin, g.n_reqs ? per + 4 : 0}, Range{g.lens, per}, Range{g.tables, 4 * entries},
                           Range{g.mask, 4 * words}, Range{g.verdicts, g.verdicts ? per : 0}})
      if (overlap(lse, r) || overlap(Range{g.out, n_out}, r))
        return report(GIFT_E_INVALID, "out or lse overlaps row_begin, lens, tables, mask or verdicts");
  }
  int dev;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return report_hip(e, "hipGetDevice");
  if (dev != work->device) return report(GIFT_E_INVALID, "the workspace belongs to another device");
  if (g.n_rows == 0) return GIFT_OK;
  a.a = g;
  a.group = g.n_heads / a.kv.heads;
  e = launch_tree_attention(a, format->dtype, work->w, stream);
  return e == hipSuccess ? GIFT_OK : report_hip(e, "tree_attention");
}

}  // extern "C"
