/*
 * bbm_cache.h -- operators on the 4-bit cache of many and long answers: attention behind prefixes that requests share, the attention
 * weight that each key has gathered, and the eviction of the keys that gathered least.  Part of libbbm; the conventions of bbm_tokens.h hold.
 *
 * Groups.  Requests group_cu[g] .. group_cu[g+1] - 1 (int32 [S+1], not decreasing, on the device like all below; cut to 0 .. R) are group g: their first
 * shared_lens[g] (int32 [S]; negative ones stand for 0) keys are the same, and lie in front of the new tokens of each of them that has any.  The rows of the block table are complete: the
 * row of each request holds the pages of its shared keys too.  Pages whose keys are all shared are the same in all rows; of one that is shared in part (shared_lens is no multiple of the page) each
 * request has a copy of its own, since it goes on there.  Requests in front of
 * group_cu[0] or from group_cu[S] on share nothing.  S may be 0 (group_cu and shared_lens are not looked at then).  Where a group's keys are not the same, or a shared key does not
 * lie in front of a request's new tokens, the results of that group's requests are unspecified.
 */
#ifndef BBM_CACHE_H
#define BBM_CACHE_H

#include "bbm_tokens.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Attention of new tokens over the cache: what bbm_kv4_attn gives for the same arguments (its sums in another order), but the keys that a group shares are read
 * once for all of its requests.  max_shared and max_own are hints for the work split (the longest of shared_lens, and of what requests have
 * behind their shared keys, or upper bounds); any positive numbers give correct results.  The workspace needs bbm_kv4_shared_attn_workspace_bytes
 * bytes for the same sizes, 16-byte aligned, contents of no matter.  Sizes as in bbm_kv4_attn; S at most R.
 */
size_t bbm_kv4_shared_attn_workspace_bytes(int64_t T, int64_t R, int64_t S, int64_t H, int64_t Hk, int d, int64_t max_shared, int64_t max_own);
int bbm_kv4_shared_attn(const bbm_packed* q, const bbm_packed* o, float* lse, int64_t T, int64_t R, const int32_t* cu, const int32_t* lens,
                        const int32_t* block_table, int64_t table_stride, int64_t max_pages, int64_t S, const int32_t* group_cu,
                        const int32_t* shared_lens, const uint64_t* mask, int64_t mask_words, const bbm_kv4_cache* cache, int64_t H,
                        float softmax_scale, int64_t max_shared, int64_t max_own, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Weights of the keys.  `weights` and `out` are fp32 [pages][Hk][page], contiguous, 16-byte aligned, a number for each token and key head of the cache; they may be
 * the same, and overlap in no other way.  For each request with a new token that has a row, each of its keys j and each key head,
 *   out[j] = decay * weights[j] + the sum over its new tokens i that see j (as in bbm_kv4_attn) and the heads h of the group of exp(softmax_scale <q_i, k_j> - lse[h][i]),
 * with 0 for weights[j] of the new tokens' own keys, whose slots may hold anything.  With lse of the attention of the same step that is the probability which
 * the keys got (a row of lse = -infinity gives nothing, whatever its query holds).  The keys that a group shares get the sum over all its requests, and one decay; those on a page
 * that is shared in part what the requests gave to their copies, each for itself.  Written are the slots of the keys that there
 * are (a key without a page is left out), others stay as they are.  A page that lies in two requests' rows
 * other than as a wholly shared one of the same group gets unspecified numbers.  Deterministic.  Meant for scores (times softmax_scale) up to 2^12, like the gradients.
 * 0 <= decay <= 1; R * Hk below 2^19, other sizes as in bbm_kv4_attn.  max_shared and max_own are hints for the work split, as above.
 * The kernel and its work split go by averages over the requests.  Requests of few and of many new tokens, or a very long one among short ones, are better given in calls of their own: parts of cu,
 * lens and block_table, and q and lse as they are, since rows outside the offsets are nobody's (255 requests of one token and one of 1500: 8.1 ms in one call, 0.29 in two).
 */
int bbm_kv4_weights(const bbm_packed* q, const float* lse, int64_t T, int64_t R, const int32_t* cu, const int32_t* lens, const int32_t* block_table,
                    int64_t table_stride, int64_t max_pages, int64_t S, const int32_t* group_cu, const int32_t* shared_lens, const uint64_t* mask,
                    int64_t mask_words, const bbm_kv4_cache* cache, int64_t H, float softmax_scale, float decay, const float* weights, float* out,
                    int64_t max_shared, int64_t max_own, void* stream);

/*
 * Eviction.  Request r has n = lens[r] keys (negative: 0; cut to max_pages * page) and keeps b = max(budget, f + recent) of them, f = max(0, first[r]) (0 if first is NULL); if n <= b, all
 * of them, and nothing of it changes.  Otherwise, for each key head, keys 0 .. f - 1 and the last `recent` stay, and of those between the b - f - recent with the largest weights
 * (equal ones: the lowest positions; a NaN counts as less than any number).  The kept ones move together to positions 0 .. b - 1, codes, scales and weights alike:
 *   those in front of position b - recent stay where they are; those between it and the last `recent` go to the places of evicted ones, the first to the
 *   first and so on; the last `recent`, in their order, go to b - recent .. b - 1.
 * Heads choose for themselves: a position then holds other tokens in other heads.  Their rotary positions are in the keys; those of later tokens run on, which is bbm_build_slots' positions plus
 * what the request has lost so far (the sums of lens - new_lens).  Positions from b on keep what they held.
 * Written besides:
 *   new_lens [R]    min(n, b) (n as cut)
 *   free_pages      the pages behind position b, back in front of *free_at: with e = min(*free_at, n_free) entries e - m .. e - 1 of free_pages [n_free] get the m pages given back, in
 *                   the order of requests and positions (entries of the table that name no page are not given back, nor is a page whose place would lie in front of the list)
 *   free_next [1]   e - m
 * The block table is not written: entries behind a request's last page may hold anything, as for bbm_build_slots, which takes from *free_at = free_next on what came back.
 * free_pages, free_at and free_next may all be NULL (pages are not given back then), free_pages alone if n_free is 0.  Keys on a page outside the cache count as less than a NaN, and what would move from or to one does not.
 * A page that another request reads too (a shared prefix) has to lie within first[r], which protects it.  new_lens may be lens.  weights as above.
 * The workspace needs bbm_kv4_evict_workspace_bytes bytes for the same R, Hk and max_pages * page, 16-byte aligned, contents of no matter.  1 <= R <= BBM_SLOTS_MAX_REQUESTS, R * Hk at most 2^21, budget >= 1 (of
 * what a table holds at most 2^19), recent >= 0.  max_len is a hint (the longest of lens, or an upper bound); any positive number gives the same results.
 */
size_t bbm_kv4_evict_workspace_bytes(int64_t R, int64_t Hk, int64_t max_keys);
int bbm_kv4_evict(const bbm_kv4_cache* cache, float* weights, int64_t R, const int32_t* lens, const int32_t* block_table, int64_t table_stride, int64_t max_pages,
                  int64_t budget, int64_t recent, const int32_t* first, int32_t* new_lens, int32_t* free_pages, int64_t n_free, const int32_t* free_at, int32_t* free_next,
                  int64_t max_len, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif
