/*
 * gift_kv.h -- the paged KV cache of gift.h in use on the device: block
 * tables and slot maps from request lengths, rows of K and V written into the
 * cache, and attention of drafted tokens over it.  A decode worker that has
 * opened a sealed handoff into its cache (gift_open_paged) steps with these
 * three calls, and seals the cache's blocks again with gift_seal_paged.
 *
 * The conventions are those of gift.h: argument errors are found on the host
 * before anything is enqueued, all work goes to `stream`, outputs are valid
 * once the stream reaches the end of the call, and the caller owns every
 * buffer.  Lengths, tables, labels, slots and masks are device arrays that
 * the kernels read when the stream gets there, so that one step's outputs are
 * the next one's inputs without a host copy.  What they hold is checked on the
 * device: no value in them makes a kernel read or write outside the buffers
 * that the call was given.  The calls allocate nothing, create no event and
 * read no result back, so they may be captured into a HIP graph.
 *
 * Ownership (GIFT Sec. 4.2: per KV block) is kept as in gift.h: a request
 * whose table names a block that is labelled with anyone else, or a block id
 * outside the cache, gets the verdict OWNER_MIXED, its new rows get no slots,
 * and attention given that verdict returns zeros for it.  A manipulated block
 * table thus shows only as this request's failure.
 */
#ifndef GIFT_KV_H
#define GIFT_KV_H

#include <stdint.h>

#include "gift.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A verdict beside those of gift.h: the request's tokens do not fit (its row
 * of the table, the free list or the slot array is too short for them). */
enum { GIFT_SEG_NO_SPACE = 3 };

/* Element types of K, V, queries and outputs. */
enum { GIFT_BF16 = 1, GIFT_F16 = 2 };

/*
 * How the tokens lie within a (layer, block) of a gift_paged_kv: K of token t
 * and head h is the head_dim elements at
 *     base + layer*layer_stride + block*block_stride
 *          + k_offset + t*token_stride + h*head_stride
 * and V likewise from v_offset.  Requirements (else GIFT_E_INVALID): a known
 * dtype; n_heads >= 1; head_dim 64, 96, 128 or 256; block_tokens a power of
 * two; offsets and strides multiples of 16; every row inside one chunk of one
 * part; no two rows overlap (sorted by stride, each of token, head and the
 * distance of K and V is at least the extent of everything inside it).
 */
typedef struct {
  uint32_t dtype;        /* GIFT_BF16 or GIFT_F16 */
  uint32_t n_heads;      /* KV heads */
  uint32_t head_dim;     /* elements */
  uint32_t block_tokens; /* tokens of a block */
  uint64_t k_offset, v_offset;        /* bytes */
  uint64_t token_stride, head_stride; /* bytes */
} gift_kv_format;

/* One step of the block tables.  Request b has lens[b] cached tokens in the
 * first ceil(lens[b] / block_tokens) blocks of its table row and adds
 * new_lens[b] (0 is allowed). */
typedef struct {
  uint32_t n_reqs;
  uint32_t block_tokens;         /* a power of two */
  uint64_t n_blocks;             /* blocks of the cache: ids and labels */
  const uint32_t* users;         /* device, n_reqs: each request's owner */
  const uint32_t* lens;          /* device, n_reqs */
  const uint32_t* new_lens;      /* device, n_reqs */
  const uint32_t* free_blocks;   /* device, n_free ids, taken from the front */
  uint32_t n_free;
  uint32_t table_width;          /* entries of a row that may be used */
  uint64_t table_stride;         /* entries from row to row */
  uint32_t* tables;              /* device, in and out */
  uint32_t* block_labels;        /* device, n_blocks, in and out */
  int64_t* slots;                /* device, n_slots, out */
  uint64_t n_slots;              /* < 2^31 */
  uint32_t* row_begin;           /* device, n_reqs + 1, out */
  uint32_t* lens_out;            /* device, n_reqs, out */
  uint32_t* taken;               /* device, 1, out */
  int32_t* verdicts;             /* device, n_reqs, out */
} gift_kv_step;

/*
 * Block tables and slot maps from request lengths.
 *   Rows: request b's new tokens are rows row_begin[b] .. row_begin[b+1] - 1 of
 *     the step (the running sum of new_lens, at most n_slots).
 *   Blocks: requests take blocks from the front of the free list in request
 *     order, as many as their new tokens need beyond their last block.  The
 *     blocks are entered in the request's table row and labelled with its
 *     user.  A request whose tokens would pass table_width takes none, nor do
 *     requests with rows that pass n_slots; from the first request on that the
 *     free list cannot serve whole, no request that needs a block gets one.
 *     taken[0] is the number of blocks that left the list.
 *   Slots: slots[row] = block * block_tokens + place of the token, where the
 *     row's K and V belong in the cache; -1 for rows of a request whose
 *     verdict is not OK and for rows of no request.
 *   Verdicts: OWNER_MIXED if one of the blocks that already held tokens is
 *     labelled otherwise than the request's user or lies outside the cache,
 *     or if its user is one of the labels that no user has
 *     (GIFT_LABEL_PARAM, GIFT_LABEL_UNOWNED; it takes no blocks then);
 *     else NO_SPACE if the request's tokens do not fit or the free list gives
 *     it an id outside the cache or a block with another owner's label (a
 *     released block's label is set back to GIFT_LABEL_UNOWNED before its id
 *     is listed again); else OK.  Which blocks a request takes goes
 *     by the lengths alone: the blocks of a request that turns out mixed are
 *     entered and labelled all the same, so that they are released with it.
 *     Of a request that the list gives a wrong id no block is entered or
 *     labelled.
 *   Release: where entries past a request's blocks hold an id outside the
 *     cache, its row names, whatever the verdict, the blocks that it holds,
 *     those taken in this step among them.  A mixed request keeps its length,
 *     so that a further step with new tokens would take blocks again and enter
 *     them over these: it is released first, or adds nothing.  Ids among the
 *     first taken[0] whose label is GIFT_LABEL_UNOWNED afterwards came to
 *     nobody and may be listed again.
 *   lens_out[b] = lens[b] + new_lens[b] for OK requests, else lens[b].
 * The ids of the free list are distinct and no table names them.  If they are
 * not, still no block comes to two users and none changes its owner: of the
 * users that the list gives the same id one at most gets it (which one, if
 * any, may differ from call to call), and a request whose table names a block
 * that another user's request takes is OWNER_MIXED.  Requests of one user may
 * then share a block, and the verdict of one whose table names it may be
 * either.
 * Outputs must not overlap inputs or each other (GIFT_E_INVALID), except that
 * tables and block_labels are both.  All arrays are aligned to their elements
 * (GIFT_E_INVALID), here and in the calls below.
 * Errors: GIFT_E_INVALID (null arrays, block_tokens no power of two, n_reqs
 * or table_width 0 where the other is not, table_stride below table_width),
 * GIFT_E_TOO_LARGE (table_width * block_tokens or n_slots past 2^31 - 1).
 */
gift_status gift_kv_tables(const gift_kv_step* step, hipStream_t stream);

/* Rows of K and V: element 0 of layer l, row r, head h is at
 * k + l*k_layer_stride + r*k_row_stride + h*k_head_stride (bytes), its
 * head_dim elements follow; V likewise. */
typedef struct {
  const void *k, *v; /* device, 16-byte aligned */
  uint64_t n_rows;
  uint64_t k_layer_stride, k_row_stride, k_head_stride; /* bytes, multiples of 16 */
  uint64_t v_layer_stride, v_row_stride, v_head_stride;
} gift_kv_rows;

/*
 * Writes rows of K and V of all layers of a cache into their slots: for each
 * i < n_slots with slots[i] >= 0, row index[i] of the sources (row i if index
 * is NULL) goes to token slots[i] % block_tokens of block
 * slots[i] / block_tokens, in every layer and head.  Slots below 0 or past
 * the cache and rows past n_rows are left out.  The elements are copied as
 * they are.  No slot may appear twice (which row it gets is not defined
 * then).  With the rows of a speculative step as sources and the accepted
 * rows' numbers in index, only what was accepted reaches the cache.
 *   slots  device, n_slots; index  device, n_slots u32, or NULL.
 * Errors: GIFT_E_INVALID (null or unaligned arrays, strides no multiple of
 * 16, arrays that overlap the cache, the format), GIFT_E_RANGE (chunks exceed cache_bytes), GIFT_E_TOO_LARGE
 * (more than 2^31 - 1 slots or rows).
 */
gift_status gift_kv_append(const gift_paged_kv* kv, const gift_kv_format* format, const int64_t* slots,
                           uint64_t n_slots, const uint32_t* index, const gift_kv_rows* rows, hipStream_t stream);

/* Device workspace of gift_tree_attention (about 72 MB): calls that are
 * ordered on one stream, and graphs replayed there, may share one; calls that
 * may overlap need one each. */
typedef struct gift_attention_work_s* gift_attention_work;

/* Allocates a workspace on the current device and clears what must start
 * clear, on `stream`, which is synchronised before return.
 * Errors: GIFT_E_INVALID (null out, a stream that is being captured),
 * GIFT_E_NOMEM, GIFT_E_HIP. */
gift_status gift_attention_work_create(hipStream_t stream, gift_attention_work* out);

/* Frees it; synchronises the device first.  NULL is a no-op. */
gift_status gift_attention_work_destroy(gift_attention_work w);

typedef struct {
  uint64_t n_rows;        /* rows of q, k, v and out, < 2^31 */
  uint32_t n_reqs;
  uint32_t n_heads;       /* query heads, a multiple of the format's n_heads */
  uint32_t layer;         /* of the cache */
  float scale;            /* of the scores, finite; usually 1 / sqrt(head_dim) */
  const void* q;          /* device; [n_rows][n_heads][head_dim] */
  const void *k, *v;      /* device; [n_rows][format n_heads][head_dim], or both NULL: no drafted keys */
  void* out;              /* device; as q */
  float* lse;             /* device, [n_rows][n_heads] contiguous, or NULL */
  uint64_t q_row_stride, q_head_stride;     /* bytes, multiples of 16, as all that follow */
  uint64_t k_row_stride, k_head_stride;
  uint64_t v_row_stride, v_head_stride;
  uint64_t out_row_stride, out_head_stride;
  const uint32_t* row_begin; /* device, n_reqs + 1: request b has rows row_begin[b] .. row_begin[b+1] - 1 */
  const uint32_t* lens;      /* device, n_reqs: cached tokens */
  const uint32_t* tables;    /* device, [n_reqs][table_stride] */
  uint32_t table_width;      /* entries of a row that may be used */
  uint64_t table_stride;
  const uint32_t* mask;      /* device, [n_rows][mask_words], or NULL */
  uint32_t mask_words;
  const int32_t* verdicts;   /* device, n_reqs, or NULL: all OK */
} gift_tree_attention_args;

/*
 * Attention of the rows of every request (the tokens of a draft tree, or a
 * single token, or a chunk of a prompt) over the request's cached tokens and
 * over the drafted rows themselves, in one call.  Query head h reads KV head
 * h / (n_heads / format n_heads).  Row i of a request sees
 *   - all lens[b] cached tokens, K and V through its table row, and
 *   - drafted row j of the same request if bit j % 32 of word j / 32 of its
 *     row of the mask is set (a tree: the bits of its ancestors and its own);
 *     rows past 32 * mask_words are not seen; without a mask, j <= i.
 * With s_j = scale * q_i . k_j over what the row sees,
 *   out = sum_j exp(s_j) v_j / sum_j exp(s_j),  lse = log sum_j exp(s_j);
 * a row that sees nothing gets out = 0 and lse = -inf.  So do the rows of a
 * request whose verdict is not OK and rows that belong to no request.  What a
 * row does not see has no part in it, whatever it holds (NaN and infinities
 * included); an element of V that it sees and that is not finite makes that
 * element of out not finite.  A table entry outside the cache is not followed:
 * its tokens are not seen.  lens past table_width * block_tokens are cut to
 * it; row_begin is taken as rising and cut to n_rows (where it falls, rows
 * that two requests claim, or one and nobody, hold what either writes).
 * Scores, maxima, sums and the running output are 32-bit floats; for the
 * product with V the weights exp(s_j - m) are rounded to 16 significant bits
 * (bfloat16, in two parts; m at most 5.6 below the largest score) or to 11
 * (float16; m the largest score so far; weights under 2^-29 of the largest to
 * steps of 2^-39 of it), and the output is rounded once at the end.
 * The same inputs give the same bits.
 *   out and lse must not overlap each other, the cache or any other array of
 *   the call.
 * Errors: GIFT_E_INVALID (null or unaligned arrays, strides, head counts,
 * layer, scale, the format), GIFT_E_RANGE (chunks exceed cache_bytes),
 * GIFT_E_TOO_LARGE (rows, or table_width * block_tokens, past 2^31 - 1, or
 * n_rows * n_heads past 2^32 - 1).
 */
gift_status gift_tree_attention(gift_attention_work work, const gift_paged_kv* kv, const gift_kv_format* format,
                                const gift_tree_attention_args* args, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* GIFT_KV_H */
