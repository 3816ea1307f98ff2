/*
 * bbm_cache.h -- operators on the 4-bit cache of many and long answers: attention behind prefixes that requests share, and the attention
 * weight that each key has gathered.  Part of libbbm; the conventions of bbm_tokens.h hold.
 *
 * Groups.  Requests group_cu[g] .. group_cu[g+1] - 1 (int32 [S+1], not decreasing, on the device like all below; cut to 0 .. R) are group g: their first
 * shared_lens[g] (int32 [S]; negative ones stand for 0) keys are the same, and lie in front of the new tokens of each of them that has any.  The rows of the block table are complete: the
 * row of each request holds the pages of its shared keys too, of which those in the row of the group's first request are read.  Requests in front of
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
 * the keys got (a row of lse = -infinity gives nothing).  The keys that a group shares get the sum over all its requests, and one decay.  Written are the slots of the keys that there
 * are (a key without a page is left out), others stay as they are.  A page that lies in two requests' rows
 * other than as a shared one of the same group gets unspecified numbers.  Deterministic.  Meant for scores (times softmax_scale) up to 2^12, like the gradients.
 * 0 <= decay <= 1.  max_shared and max_own are hints for the work split, as above.
 */
int bbm_kv4_weights(const bbm_packed* q, const float* lse, int64_t T, int64_t R, const int32_t* cu, const int32_t* lens, const int32_t* block_table,
                    int64_t table_stride, int64_t max_pages, int64_t S, const int32_t* group_cu, const int32_t* shared_lens, const uint64_t* mask,
                    int64_t mask_words, const bbm_kv4_cache* cache, int64_t H, float softmax_scale, float decay, const float* weights, float* out,
                    int64_t max_shared, int64_t max_own, void* stream);

#ifdef __cplusplus
}
#endif
#endif
