/*
 * moa_cache.h -- C ABI of the paged K/V cache for NVIDIA B200 (sm_100a): tokens are appended with their positions applied on
 * the way, and attended to by one new query per head.
 *
 * A cache is a pool of pages, each of `page` keys and values of every K/V head; which pages a sequence has, and in which order, is a table that
 * the caller keeps.  So sequences grow without moving and a pool serves any mixture of lengths.
 *
 * Conventions as in moa_attn.h (device pointers, caller-owned memory, asynchronous on `stream`, errors by moa_status, found before
 * anything is enqueued).  What lives in device memory (positions, slots, tables, lengths) is not seen by the host: the kernels check
 * it and read or write nothing outside the pool.
 */
#ifndef MOA_CACHE_H
#define MOA_CACHE_H

#include "moa_block.h"

#ifdef __cplusplus
extern "C" {
#endif

/* What a page holds.
 * MOA_CACHE_BF16: [H_kv][K, V][page][d] bfloat16.
 * MOA_CACHE_INT4: 4.5 bits per element.  A group is 32 neighbouring elements of a key (value) of one head; its scale is
 *     s = bf16(amax / 7), and the code c of an element x is 8 + rint(x / s) (halves to even), 1 .. 15: it stands for (c - 8) s.
 *     A group with amax < 2^-100 has s = 0 and codes of 8, one with an infinity or a NaN has s = NaN and codes of 8.
 *     For each K/V head, a page is page/16 blocks of 18 d bytes, 16 keys each: K codes (8 d bytes), K scales (d), V codes (8 d), V scales
 *     (d).  Inside a block, with g = d/32 groups, key r = 0 .. 15, element x = 32 y + z (group y):
 *       K code   nibble 4 (z % 2) + z % 8 / 2 (the lowest first) of the 32-bit word at byte  r d/2 + 4 (z/8 g + y)
 *       K scale  bf16 at byte 8 d + 2 ((2 (r % 8) + r/8) g + y)
 *       V code   nibble 4 (y % 2) + z % 4 of the 32-bit word at byte  9 d + 128 g (r/8) + 4 g (4 (z/4) + r % 8 / 2) + 2 g (r % 2) + 4 (y/2)
 *       V scale  bf16 at byte 17 d + 8 g (r % 8 / 2) + 8 y + 4 (r/8) + 2 (r % 2)
 *     (the places in which the warp-level products of the attention take them from wide loads). */
typedef enum { MOA_CACHE_BF16 = 0, MOA_CACHE_INT4 = 1 } moa_cache_format;

/* The pool: `pages` pages of `page` keys (a multiple of 16, 16 .. 1024), page p at p * page_stride bytes from its start (0: pages one after the
 * other; else a multiple of 16 and at least moa_cache_page_bytes).  H_kv >= 1; d in {64, 128}; pages >= 1; pool 16-byte aligned. */
typedef struct {
    int32_t pages, page, H_kv, d;
    int32_t format;          /* moa_cache_format */
    int32_t reserved;        /* 0 */
    int64_t page_stride;
} moa_cache_desc;
/* Bytes of a page; 0 for an invalid desc. */
size_t moa_cache_page_bytes(const moa_cache_desc *desc);

/* Appends T tokens: k is turned by its position (as moa_rope_fwd) and rounded to bf16, and k and v go to the key `slot` of the
 * pool, slot = page * (keys per page) + place in the page.  q, where there is one (H > 0), is turned into q_out in the same launch.
 * q, q_out: T x H x d; k, v: T x H_kv x d, strides {token, head} in elements as in moa_rope_desc: the parts of a packed projection need
 * no copy; q_out may be q, with its strides; what is written must overlap nothing else.  pos [T] int32, slot [T] int64.  A slot outside the pool (-1 for the padding of a batch) writes nothing
 * (q_out is written all the same).  The slots of one call must differ from each other; where two are the same, that key holds
 * a mixture of the two tokens.  d_rot: a multiple of 16 up to d; 0 (with H = 0; pos, inv_freq NULL): nothing is turned.
 * K's rounding is the nearest bf16 of the rotation in 64 bits, so a 4-bit page holds what quantising the bf16 page's keys would give.
 * dtype of q, k, v, q_out: MOA_BF16. */
typedef struct {
    moa_cache_desc cache;
    int32_t T, H, d_rot;
    int32_t layout;          /* moa_rope_layout */
    float   factor;
    int32_t dtype;
    int64_t q_stride[2], k_stride[2], v_stride[2], q_out_stride[2];
} moa_append_desc;
moa_status moa_kv_append(const moa_append_desc *desc, const void *q, const void *k, const void *v, const int32_t *pos,
                         const int64_t *slot, const float *inv_freq, void *q_out, void *pool, void *stream);

/* Reads T keys and values back: k[t], v[t] (T x H_kv x d, strides as above) = what the pool holds at slot[t]; zeros for a slot outside the
 * pool.  dtype of k, v: MOA_BF16 (4-bit values rounded once) or MOA_F32 (exact). */
typedef struct {
    moa_cache_desc cache;
    int32_t T;
    int32_t dtype;
    int64_t k_stride[2], v_stride[2];
} moa_gather_desc;
moa_status moa_kv_gather(const moa_gather_desc *desc, const void *pool, const int64_t *slot, void *k, void *v, void *stream);

/* Decode attention over the pages: sequence b has lens[b] keys, key j in page table[b][j / page] at j % page:
 *     out[b,h,:] = softmax_j(scale q[b,h,:] . K_j) V_j,   j < lens[b],   K/V head h / (H / H_kv)
 * Every key and value that a sequence has is read once, whatever the group H / H_kv (1 .. 16).  A sequence without keys gives zeros (and lse = -inf);
 * lengths are cut to 0 .. max_pages * page; the keys of a page number outside the pool are left out (as masked), whatever memory holds past
 * the end of a sequence does not count.
 * q: B x H x d, strides {sequence, head} as above; out [B,H,d]; lse [B,H] fp32 natural-log logsumexp of the scaled scores, may be NULL;
 * table int32, rows of max_pages entries, table_stride entries apart (0: max_pages); lens [B] int32.  dtype of q, out:
 * MOA_BF16.  Scores, statistics and sums are fp32.  Weights: bf16 pages and groups of 1 to 8, 16 bits (two bf16 pieces, a product each);
 * groups of 9 to 16, rounded once to bf16; pages of 4 bits, the weight's product with V's scale is rounded once to bf16.  |scale| <= 2^60.  A page of 4 bits
 * wants |q| < 2^59 and |v| < 2^55.  Its codes are used as numbers at the low end of bf16, against operands raised by up to 2^68, so fp32's last place lies higher
 * there: a query's product with the codes of a group is kept to 2^-84 (times the group's scale), a result's sum over 16 keys to 2^-80; results below 2^-72 have fewer
 * bits than bf16, those below 2^-80 may be 0.  A score that is NaN makes its row NaN.  Lengths are read on the device only: a captured call serves growing sequences.
 * Workspace: moa_paged_decode_workspace_bytes (partial results of sequences that several CTAs share); two calls that may
 * overlap need two. */
typedef struct {
    moa_cache_desc cache;
    int32_t B, H, max_pages;
    int32_t dtype;
    float   scale;
    int32_t reserved;        /* 0 */
    int64_t table_stride;
    int64_t q_stride[2];
} moa_paged_decode_desc;
size_t moa_paged_decode_workspace_bytes(const moa_paged_decode_desc *desc);
moa_status moa_paged_decode(const moa_paged_decode_desc *desc, const void *q, const void *pool, const int32_t *table,
                            const int32_t *lens, void *out, float *lse, void *ws, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MOA_CACHE_H */
