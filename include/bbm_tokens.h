/*
 * bbm_tokens.h -- operators on packed tokens: slots of a paged cache, rotary positions, causal attention over packed prompts
 * with grouped heads (forward and backward), and a cache in 4 bits with the attention that reads it.  Part of libbbm; the
 * conventions of bbm.h hold: device pointers owned by the caller, work enqueued on `stream`, nothing allocated, retained or
 * synchronised, arguments checked on the host before any GPU call, BBM_OK or a negative code with bbm_last_error().  No entry
 * point keeps state between calls; a workspace holds nothing before a call and is free when the call's work is done, so calls
 * that may run at the same time each need one of their own.
 *
 * Packed tokens.  The tokens of R requests (or sequences) lie one behind the other in T rows; request r has rows
 * cu[r] .. cu[r+1] - 1, with cu int32 [R+1] on the device, not decreasing.  Rows before cu[0] or from cu[R] on belong to nobody: no
 * operator writes them (bbm_build_slots and bbm_kv4_read, which write all T rows, say what they write there).  Offsets outside
 * 0 .. T are cut to that range.
 *
 * Unless a function says otherwise, outputs and workspaces overlap neither inputs nor each other (the same pointer is refused).  What rows
 * of nobody hold does not matter (it may be an infinity or a NaN); the rows of requests are taken to be finite, as are the cache's groups: an
 * infinity or a NaN among them may reach any row of its own request.
 *
 * Scores, their sums and the log-sum-exp are fp32 numbers: a softmax_scale lies within 2^-100 .. 2^100, sums of products of q and k stay below
 * 2^126 before and after it, as do 2^16 times the sums of |v| over a request's keys.  Within that, attention is as exact for large scores as fp32
 * scores allow: equal ones share a row, however large.  The gradients form their probabilities again from the fp32 log-sum-exp, half a step of which is a relative error of
 * 2^-24 times its size in all of a row's: they are meant for scores (times softmax_scale) up to 2^12, and from 2^20 on say nothing.
 *
 * A packed tensor is bf16 [T][heads][d] with any row and head strides (in elements, multiples of 8; the d elements of a head
 * are contiguous and 16-byte aligned), so the q, k and v parts of one projection's output, or [heads][T][d], need no copy.
 */
#ifndef BBM_TOKENS_H
#define BBM_TOKENS_H

#include "bbm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A packed tensor: element (t, h, i) lies at ptr + t * row_stride + h * head_stride + i. */
typedef struct bbm_packed {
  void* ptr;
  int64_t row_stride;
  int64_t head_stride;
} bbm_packed;

/*
 * Slots of a step.  Request r has ctx_lens[r] tokens in the cache and gets new_lens[r] more (negative counts stand for 0); the
 * page that holds its position p is block_table[r * table_stride + p / page], its slot that page * page + p % page.  A request
 * that needs pages it does not have takes the next ones of free_pages [n_free], from index *free_at on, in the order of
 * requests and positions.  Written:
 *   block_table  the entries of pages taken; -1 where the list has ended.  Positions behind max_pages * page get no page.
 *   cu_new [R+1], lens [R]   packed offsets of the new tokens; tokens in the cache after the step
 *   positions [T], slots [T] of every new token; slot -1 where it has no page.  Rows from cu_new[R] on: position 0, slot -1.
 *                            Of more than T new tokens the first T are written.
 *   free_next [1]            *free_at + the pages asked for; beyond n_free, the list was too short
 * block_table is read and written, but only entries behind a request's last page are written, so that a call may be repeated.
 * 1 <= R <= BBM_SLOTS_MAX_REQUESTS; page 16, 32, 64 or 128; totals fit 31 bits.
 */
#define BBM_SLOTS_MAX_REQUESTS 16384
int bbm_build_slots(const int32_t* ctx_lens, const int32_t* new_lens, int64_t R, int32_t* block_table, int64_t table_stride,
                    int64_t max_pages, int page, const int32_t* free_pages, int64_t n_free, const int32_t* free_at, int64_t T,
                    int32_t* cu_new, int32_t* lens, int32_t* positions, int32_t* slots, int32_t* free_next, void* stream);

/*
 * Rotary positions.  For token t and pair j < rot / 2, with a = positions[t] * freqs[j] (freqs fp32 [rot/2]; the product and
 * its reduction are taken in 64 bits, so that far positions lose nothing):
 *   y1 = mscale * (x1 cos a - x2 sin a),   y2 = mscale * (x2 cos a + x1 sin a)
 * Pair j is elements (j, j + rot/2) of a head, or (2j, 2j + 1) if `interleaved`; the elements from rot on are copied.  `inverse`
 * turns by -a: the gradient of the operator.  k may have Hk = 0 (and is not looked at then).  out == in (same pointer and strides) is
 * allowed, any other overlap is not.  d a multiple of 16, at most 512; rot even, 2 <= rot <= d.
 */
int bbm_rope(const bbm_packed* q, const bbm_packed* q_out, int64_t H, const bbm_packed* k, const bbm_packed* k_out, int64_t Hk,
             int64_t T, int d, int rot, int interleaved, int inverse, const int32_t* positions, const float* freqs, float mscale,
             void* stream);

/*
 * Causal attention over packed prompts: query i of a sequence sees its keys 0 .. i; query head h reads key head h / (H / Hk), H a
 * multiple of Hk.  O bf16 packed, lse fp32 [H][T] (natural logarithm; may be NULL) are written for the rows of the sequences.
 * d 64 or 128.  Scores are formed from the bf16 inputs without a further rounding; probabilities are rounded to bf16 for the
 * second product, their sum is taken before that.  Rows must not lie upon each other (of more than one token, row strides of at least d), here and in
 * the backward pass, inputs included; a head stride of 0, heads that share their values, is fine.
 */
int bbm_prompt_attn_fwd(const bbm_packed* q, const bbm_packed* k, const bbm_packed* v, const bbm_packed* o, float* lse, int64_t T,
                        int64_t R, const int32_t* cu, int64_t H, int64_t Hk, int d, float softmax_scale, void* stream);

/* Its gradients: dQ, dK, dV (packed; dK and dV summed over the query heads of a group) from dO, O and lse of the forward.
 * Deterministic.  The workspace needs bbm_prompt_attn_bwd_workspace_bytes(T, R, H, Hk, d) bytes, 16-byte aligned, contents of no matter. */
size_t bbm_prompt_attn_bwd_workspace_bytes(int64_t T, int64_t R, int64_t H, int64_t Hk, int d);
int bbm_prompt_attn_bwd(const bbm_packed* q, const bbm_packed* k, const bbm_packed* v, const bbm_packed* o, const bbm_packed* d_o,
                        const float* lse, const bbm_packed* dq, const bbm_packed* dk, const bbm_packed* dv, int64_t T, int64_t R,
                        const int32_t* cu, int64_t H, int64_t Hk, int d, float softmax_scale, void* workspace, size_t workspace_bytes,
                        void* stream);

/*
 * A paged cache of keys and values in 4 bits.  The d elements of a token and head are d / 32 groups; a group holds a scale byte
 * s = e + 127, e the smallest integer with max|x| <= 7 * 2^e, between -120 and 125, and for every element a code of x / 2^e rounded
 * to the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 (codes 0 .. 7, ties to the even code, 8 added for a negative x): no value within the
 * scales' range is off by more than half of its interval, the largest by more than 1/7.  A group with an infinity or a NaN gets s = 255, and all its
 * values are NaN when they are read.  Element 2i is in the low half of byte i.  d 64 or 128; page 16, 32, 64 or 128 tokens.
 *   k, v     uint8 [pages][Hk][page][d/2]
 *   k_scale  uint8 [pages][Hk][page][d/32]
 *   v_scale  uint8 [pages][Hk][d/32][page]
 * all contiguous and 16-byte aligned.  Slot s is token s % page of page s / page; pages * page < 2^31.
 */
typedef struct bbm_kv4_cache {
  uint8_t* k;
  uint8_t* k_scale;
  uint8_t* v;
  uint8_t* v_scale;
  int64_t pages;
  int64_t Hk;
  int32_t page;
  int32_t d;
} bbm_kv4_cache;

/* k, v packed [T][Hk][d] into the slots [T] int32.  Rows with a slot outside the cache (-1) are left out.  Two rows with the same slot
 * leave that slot's contents unspecified. */
int bbm_kv4_append(const bbm_packed* k, const bbm_packed* v, int64_t T, const int32_t* slots, const bbm_kv4_cache* cache, void* stream);

/* The values that the cache holds for the slots [T]: k_out, v_out packed [T][Hk][d] (exact in bf16); rows with a slot outside the cache
 * are zeros. */
int bbm_kv4_read(const int32_t* slots, int64_t T, const bbm_kv4_cache* cache, const bbm_packed* k_out, const bbm_packed* v_out,
                 void* stream);

/*
 * Attention of new tokens over the cache.  Request r has lens[r] keys in it, the n = cu[r+1] - cu[r] new tokens' (rows outside 0 .. T counted) the last of
 * them; key p lies on page block_table[r * table_stride + p / page].  Query i of the request sees the keys 0 .. lens[r] - n + i,
 * or, with `mask`, keys 0 .. lens[r] - n - 1 and new key j where bit j % 64 of mask[t * mask_words + j / 64] is set (t the query's
 * row; bits from n or 64 * mask_words on count as not set).  Keys on a page outside the cache (-1) or behind max_pages * page are not seen.  A query that sees no
 * key gets O = 0 and lse = -inf.  Query head h reads key head h / (H / Hk).  O and lse fp32 [H][T] (may be NULL) as in
 * bbm_prompt_attn_fwd.  max_len is a hint for the work split (the longest of lens, or an upper bound); any positive number gives
 * correct results.  The workspace needs bbm_kv4_attn_workspace_bytes bytes for the same T, R, H, Hk, d and max_len, 16-byte aligned,
 * contents of no matter.
 * max_pages * page and T * H / Hk at most 2^30.
 */
size_t bbm_kv4_attn_workspace_bytes(int64_t T, int64_t R, int64_t H, int64_t Hk, int d, int64_t max_len);
int bbm_kv4_attn(const bbm_packed* q, const bbm_packed* o, float* lse, int64_t T, int64_t R, const int32_t* cu, const int32_t* lens,
                 const int32_t* block_table, int64_t table_stride, int64_t max_pages, const uint64_t* mask, int64_t mask_words,
                 const bbm_kv4_cache* cache, int64_t H, float softmax_scale, int64_t max_len, void* workspace,
                 size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif
