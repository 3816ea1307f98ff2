// The 4-bit cache's format (include/bbm_tokens.h) in device code.
#pragma once
#include "bbm_packed.h"
#include "bbm_tile.h"

namespace bbm {

struct Kv4 {
  uint8_t *k, *k_scale, *v, *v_scale;
  int32_t pages, Hk, page_shift, page;
};

inline int check_kv4(const char* fn, const bbm_kv4_cache* c) {
  if (!c) return fail(BBM_EINVAL, "%s: cache must not be NULL", fn);
  if (!c->k || !c->k_scale || !c->v || !c->v_scale) return fail(BBM_EINVAL, "%s: the cache's pointers must not be NULL", fn);
  if (!aligned(c->k, 16) || !aligned(c->k_scale, 16) || !aligned(c->v, 16) || !aligned(c->v_scale, 16))
    return fail(BBM_EINVAL, "%s: the cache's pointers must be 16-byte aligned", fn);
  if (c->pages < 1 || c->Hk < 1) return fail(BBM_EINVAL, "%s: pages=%lld, Hk=%lld must be >= 1", fn, (long long)c->pages, (long long)c->Hk);
  if (c->d != 64 && c->d != 128) return fail(BBM_EUNSUPPORTED, "%s: d=%d has no kernel instance (64, 128)", fn, c->d);
  if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return fail(BBM_EUNSUPPORTED, "%s: page=%d is none of 16, 32, 64, 128", fn, c->page);
  if (c->pages > 0x7fffffffll / c->page || c->Hk > 65535)  // (by division: a product of the caller's may wrap)
    return fail(BBM_EUNSUPPORTED, "%s: cache too large (%lld pages of %d, %lld heads)", fn, (long long)c->pages, c->page, (long long)c->Hk);
  return BBM_OK;
}
inline Kv4 kv4_of(const bbm_kv4_cache* c) {
  return Kv4{c->k, c->k_scale, c->v, c->v_scale, (int32_t)c->pages, (int32_t)c->Hk, c->page == 16 ? 4 : c->page == 32 ? 5 : c->page == 64 ? 6 : 7, c->page};
}

// Lengths and block table of requests, the mask over their new tokens, and the groups that share prefixes.
inline int check_table(const char* fn, const int32_t* lens, const int32_t* table, int64_t stride, int64_t max_pages, int page) {
  if (!lens || !aligned(lens, 4) || !table || !aligned(table, 4)) return fail(BBM_EINVAL, "%s: lens and block_table must be non-NULL 4-byte aligned pointers", fn);
  if (max_pages < 1 || stride < max_pages) return fail(BBM_EINVAL, "%s: max_pages=%lld must be >= 1, table_stride=%lld no less than it", fn, (long long)max_pages, (long long)stride);
  if (max_pages > kMaxTokens / page) return fail(BBM_EUNSUPPORTED, "%s: max_pages=%lld is too large", fn, (long long)max_pages);
  return BBM_OK;
}
inline int check_mask(const char* fn, const uint64_t* mask, int64_t mask_words) {
  if (!aligned(mask, 8)) return fail(BBM_EINVAL, "%s: mask must be 8-byte aligned", fn);
  if (mask ? mask_words < 1 : mask_words != 0) return fail(BBM_EINVAL, "%s: mask_words=%lld does not fit the mask", fn, (long long)mask_words);
  if (mask_words > (1 << 20)) return fail(BBM_EUNSUPPORTED, "%s: mask_words=%lld is too large", fn, (long long)mask_words);
  return BBM_OK;
}
inline int check_groups(const char* fn, int64_t R, int64_t S, const int32_t* group_cu, const int32_t* shared_lens, int64_t max_shared, int64_t max_own) {
  if (S < 0 || S > R) return fail(BBM_EINVAL, "%s: S=%lld is outside 0 .. R=%lld", fn, (long long)S, (long long)R);
  if (S > 0 && (!group_cu || !shared_lens || !aligned(group_cu, 4) || !aligned(shared_lens, 4)))
    return fail(BBM_EINVAL, "%s: group_cu and shared_lens must be non-NULL 4-byte aligned pointers", fn);
  if (max_shared < 1 || max_own < 1) return fail(BBM_EINVAL, "%s: max_shared=%lld and max_own=%lld must be >= 1", fn, (long long)max_shared, (long long)max_own);
  return BBM_OK;
}

// A scale byte as the conversion takes it: in the exponent's place of a float.  It looks at nothing else (sign and fraction may be anything), 255
// gives NaNs, 0 gives 2^-127.
__device__ __forceinline__ float scale_of(uint32_t s) { return __uint_as_float(s << 23); }

// The eight values of 32 bits of codes.
__device__ __forceinline__ bf16x8 values_of(uint32_t codes, float scale) {
  union {
    bf16x2 p[4];
    bf16x8 all;
  } x;
  x.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
  x.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
  x.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
  x.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
  return x.all;
}

// The group of request r and its shared keys, -1 and 0 if it has none; 64 groups in one trip to memory.
struct Group {
  int g, keys;
};
__device__ __forceinline__ Group group_of(const int32_t* group_cu, const int32_t* shared_lens, int S, int r) {
  const int lane = threadIdx.x & 63;
  for (int g0 = 0; g0 < S; g0 += 64) {
    const int g = min(g0 + lane, S - 1), c0 = group_cu[g], c1 = group_cu[g + 1], keys = shared_lens[g];
    const uint64_t has = __ballot(c0 <= r && r < c1);
    if (has) {
      const int l = __ffsll((unsigned long long)has) - 1;
      return {min(g0 + l, S - 1), __builtin_amdgcn_readlane(keys, l)};
    }
  }
  return {-1, 0};
}

// Which of 64 keys new token i of a request may see, as far as its order or its words of the mask (NULL: causal) go; w0: the first key, counted from the new tokens on.
__device__ __forceinline__ uint64_t seen_from(const uint64_t* words, int mask_words, int i, int w0) {
  if (!words) return bits_up_to(i - w0);
  auto word = [&](int n) { return n < mask_words ? words[n] : 0ull; };
  if (w0 <= -64) return ~0ull;
  if (w0 < 0) return word(0) << -w0 | ((1ull << -w0) - 1ull);
  const int sh = w0 & 63;
  return sh ? word(w0 >> 6) >> sh | word((w0 >> 6) + 1) << (64 - sh) : word(w0 >> 6);
}

// A request's row of the block table, read by scalar loads (through the constant address space: no kernel that reads it writes it).  As a vector load a page's
// number would be waited for together with the keys and values asked for before it.
typedef const int32_t __attribute__((address_space(4)))* Table;

}  // namespace bbm
