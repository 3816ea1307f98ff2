// Packed tensors (include/bbm_tokens.h): their host checks, and the way from a work-group's number to its piece of a request.
#pragma once
#include "bbm_internal.h"
#include "bbm_tokens.h"

#include <initializer_list>

namespace bbm {

constexpr int64_t kMaxTokens = 1ll << 30;
constexpr int64_t kMaxWgs = 1ll << 24;  // work-groups of 256 threads that a launch may have, less one: it counts threads in 32 bits
constexpr int64_t kMaxRowStride = 1ll << 22;  // a tile of 128 rows stays within the 2^31 bytes of a buffer resource

// `rows` x `heads` x d elements; an output's must not lie upon each other.
inline int check_packed(const char* fn, const char* name, const bbm_packed* x, int64_t rows, int64_t heads, int64_t d, bool output) {
  if (!x || (!x->ptr && rows > 0)) return fail(BBM_EINVAL, "%s: %s must not be NULL", fn, name);
  if (!aligned(x->ptr, 16)) return fail(BBM_EINVAL, "%s: %s must be 16-byte aligned", fn, name);
  if (x->row_stride < 0 || x->head_stride < 0 || x->row_stride % 8 || x->head_stride % 8)
    return fail(BBM_EINVAL, "%s: strides of %s (%lld, %lld) must be multiples of 8 elements, not negative", fn, name, (long long)x->row_stride, (long long)x->head_stride);
  if (rows > 1 && x->row_stride > kMaxRowStride) return fail(BBM_EUNSUPPORTED, "%s: row stride %lld of %s is beyond %lld elements", fn, (long long)x->row_stride, name, (long long)kMaxRowStride);
  if (heads > 1 && x->head_stride > (1ll << 40)) return fail(BBM_EUNSUPPORTED, "%s: head stride %lld of %s is too large", fn, (long long)x->head_stride, name);
  if (output) {
    const bool rows_first = x->row_stride >= x->head_stride;  // (the longer stride; one that is never taken does not count)
    const int64_t inner = rows_first ? x->head_stride : x->row_stride, n_inner = rows_first ? heads : rows;
    const int64_t outer = rows_first ? x->row_stride : x->head_stride, n_outer = rows_first ? rows : heads;
    if ((n_inner > 1 && inner < d) || (n_outer > 1 && outer < (n_inner > 1 ? (n_inner - 1) * inner : 0) + d))
      return fail(BBM_EINVAL, "%s: rows or heads of %s overlap (strides %lld, %lld)", fn, name, (long long)x->row_stride, (long long)x->head_stride);
  }
  return BBM_OK;
}

// The overlap that a caller is most likely to ask for: an output (or a workspace) in the place of an input or of another output.  NULL: not there.
inline int check_apart(const char* fn, std::initializer_list<const void*> outputs, std::initializer_list<const void*> inputs) {
  for (auto a = outputs.begin(); a != outputs.end(); ++a) {
    if (!*a) continue;
    for (const void* x : inputs)
      if (x == *a) return fail(BBM_EINVAL, "%s: an output must not be an input", fn);
    for (auto b = outputs.begin(); b != a; ++b)
      if (*b == *a) return fail(BBM_EINVAL, "%s: two outputs must not be the same", fn);
  }
  return BBM_OK;
}

// T rows, R requests, H query heads over Hk key heads.
inline int check_tokens(const char* fn, int64_t T, int64_t R, const int32_t* cu, int64_t H, int64_t Hk) {
  if (T < 0 || R < 1 || H < 1 || Hk < 1) return fail(BBM_EINVAL, "%s: T=%lld must be >= 0, R=%lld, H=%lld, Hk=%lld >= 1", fn, (long long)T, (long long)R, (long long)H, (long long)Hk);
  if (H % Hk) return fail(BBM_EINVAL, "%s: H=%lld is no multiple of Hk=%lld", fn, (long long)H, (long long)Hk);
  if (!cu || !aligned(cu, 4)) return fail(BBM_EINVAL, "%s: cu must be a non-NULL 4-byte aligned pointer", fn);
  if (T > kMaxTokens || R > kMaxTokens || H > 65535 || T * H > (1ll << 36)) return fail(BBM_EUNSUPPORTED, "%s: problem too large (T=%lld, R=%lld, H=%lld)", fn, (long long)T, (long long)R, (long long)H);
  return BBM_OK;
}

// (Beyond these the factors that the kernels make of it are no finite numbers in fp32.)
inline int check_scale(const char* fn, float softmax_scale) {
  if (!(softmax_scale > 0.0f) || !(softmax_scale < INFINITY)) return fail(BBM_EINVAL, "%s: softmax_scale must be finite and > 0", fn);
  if (softmax_scale < 0x1p-100f || softmax_scale > 0x1p100f) return fail(BBM_EUNSUPPORTED, "%s: softmax_scale=%g is outside 2^-100 .. 2^100", fn, (double)softmax_scale);
  return BBM_OK;
}

struct Span {
  int r, begin, end;  // request, its first row and the one behind its last
  int piece;          // which piece of it
};

// The sum of x over this lane and those in front of it: within rows of 16 lanes, then the last lanes of the rows in front.
__device__ __forceinline__ int wave_prefix_sum(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // from 1, 2, 4, 8 lanes in front
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // the last lane of rows 0 and 2 to rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // the last lane of row 1 to rows 2 and 3
  return x;
}

// Which piece of which request is number `at`?  Requests are cut into pieces of `unit` columns, `mul` columns a row; the host, which does not know the
// offsets, launches for T * mul / unit + R of them, and no batch has more (floor((a + n) / u) + 1 >= floor(a / u) + ceil(n / u)).
// Up to kCounted requests, all lanes of a wave count the pieces, 64 requests at a time: numbers follow each other without holes, and those that
// belong to nobody (begin = end) are the last ones.  With the numbers below, requests of one piece each had every other number: work-groups go to
// the shader engines of an XCD in turn, and half of them got nothing (16 requests of 128 columns over 4096 keys of the 4-bit cache: 104 us instead of 81).
// Beyond, request r's pieces have the numbers from cu[r] * mul / unit + r on, found by a search that takes a trip to memory for every
// factor of 64 in R, and there are holes.  Counted / searched, us: one token each of 200 requests of up to 300 keys 19.5 / 20.7; forward over 100, 300, 500 sequences of
// up to 100 tokens 11.9 / 12.6, 27.6 / 27.8, 44.3 / 43.3, over 600 and 1000 54.6 / 50.2, 93 / 79.
constexpr int kCounted = 512;
// `cu` gives offset r of R + 1, by cu(r).
template <typename Offsets>
__device__ __forceinline__ Span find_piece_of(Offsets cu, int R, int T, int mul, int unit, int at) {
  const int lane = threadIdx.x & 63;
  auto cut = [&](int c) { return min(max(c, 0), T); };
  Span s;
  s.r = s.begin = s.end = s.piece = 0;
  if (R <= kCounted) {
    int before = 0;  // pieces of the requests in front of these
    // 64 requests from r0 on, of which the lane holds one; true if the piece was among them
    auto among = [&](int r0, int c0, int c1) __attribute__((always_inline)) {
      const int begin = cut(c0), end = max(begin, cut(c1));
      const int mine = r0 + lane < R ? (int)(((uint32_t)(end - begin) * (uint32_t)mul + (uint32_t)(unit - 1)) / (uint32_t)unit) : 0;
      const int sum = wave_prefix_sum(mine), all = __builtin_amdgcn_readlane(sum, 63);
      if (at >= before + all) {
        before += all;
        return false;
      }
      const int l = __ffsll((unsigned long long)__ballot(before + sum > at)) - 1;
      s.r = r0 + l;
      s.begin = __builtin_amdgcn_readlane(begin, l);
      s.end = __builtin_amdgcn_readlane(end, l);
      s.piece = at - before - __builtin_amdgcn_readlane(sum - mine, l);
      return true;
    };
    if (R <= 64) {
      const int r = min(lane, R - 1);
      among(0, cu(r), cu(r + 1));
      return s;
    }
    for (int r0 = 0; r0 < R; r0 += 256) {  // (four times 64 in one trip to memory)
      int c0[4], c1[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = min(r0 + 64 * i + lane, R - 1);
        c0[i] = cu(r), c1[i] = cu(r + 1);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (among(r0 + 64 * i, c0[i], c1[i])) return s;
    }
    return s;
  }
  auto first = [&](int c, int r) { return (int64_t)cut(c) * mul / unit + r; };
  int lo = 0, n = R;  // the last r in lo .. lo + n - 1 with first(r) <= at (r = lo if there is none)
  while (n > 1) {
    const int step = (n + 63) / 64;
    const int r = lo + lane * step;
    const bool ok = lane * step < n && first(cu(min(r, R)), r) <= at;
    const int hits = __popcll(__ballot(ok));
    const int k = max(0, hits - 1) * step;
    lo += k;
    n = min(step, n - k);
  }
  const int c0 = cu(lo), c1 = cu(lo + 1);
  s.r = __builtin_amdgcn_readfirstlane(lo);
  s.begin = __builtin_amdgcn_readfirstlane(cut(c0));
  s.end = __builtin_amdgcn_readfirstlane(max(cut(c0), cut(c1)));
  const int64_t piece = at - first(c0, lo);
  const bool real = piece >= 0 && piece * unit < (int64_t)(s.end - s.begin) * mul;
  s.piece = __builtin_amdgcn_readfirstlane(real ? (int)piece : 0);
  if (__builtin_amdgcn_readfirstlane(real) == 0) s.end = s.begin;
  return s;
}
__device__ __forceinline__ Span find_piece(const int32_t* __restrict__ cu, int R, int T, int mul, int unit, int at) {
  return find_piece_of([=](int r) __attribute__((always_inline)) { return cu[r]; }, R, T, mul, unit, at);
}
inline int64_t count_pieces(int64_t T, int64_t R, int64_t mul, int64_t unit) { return T * mul / unit + R; }

}  // namespace bbm
