// The 4-bit cache's format (include/bbm_tokens.h) in device code.
#pragma once
#include "bbm_mfma.h"
#include "bbm_packed.h"

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

}  // namespace bbm
