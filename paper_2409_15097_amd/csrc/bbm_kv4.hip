// Writing to and reading from the 4-bit cache (include/bbm_tokens.h).  Bound by memory: 2 bytes an element on the one side, 17/32 on the
// other.  Four lanes share a group of 32 elements, 8 each: 16 bytes of bf16 and 4 bytes of codes a lane, the largest magnitude of
// the group over two exchanges between neighbouring lanes.
#include "bbm_kv4.h"

namespace {

using bbm::bf16x8, bbm::Kv4;

struct Kv4Params {
  Kv4 c;
  __bf16 *k, *v;
  int64_t k_row, k_head, v_row, v_head;
  const int32_t* slots;
  int32_t T, items;  // 8 elements of one tensor each
};

template <int CTRL>
__device__ __forceinline__ uint32_t max_with(uint32_t x) {
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true));
}

// Where an item's bytes lie in the cache.
template <int D>
struct Place {
  bool values;        // v, not k
  int t, h, c;        // token, head, 8-element chunk
  int64_t code, scale;
  bool inside;
  __device__ __forceinline__ Place(const Kv4Params& P, int n) {
    const int per_token = P.c.Hk * (D / 8);
    t = n / (2 * per_token);
    int m = n - t * 2 * per_token;
    values = m >= per_token;
    m -= values ? per_token : 0;
    h = m / (D / 8);
    c = m % (D / 8);
    const int slot = P.slots[t];
    const int page = slot >> P.c.page_shift, at = slot & (P.c.page - 1);
    inside = slot >= 0 && page < P.c.pages;
    const int64_t head = (int64_t)page * P.c.Hk + h;
    code = (head * P.c.page + at) * (D / 2) + c * 4;
    scale = values ? (head * (D / 32) + c / 4) * P.c.page + at : (head * P.c.page + at) * (D / 32) + c / 4;
  }
};

template <int D>
__global__ __launch_bounds__(256) void kv4_append_kernel(const Kv4Params P) {
  const int n = blockIdx.x * 256 + threadIdx.x;
  if (n >= P.items) return;  // (whole groups: the items of a group are in or out together)
  const Place<D> at(P, n);
  if (!at.inside) return;
  const __bf16* const src = at.values ? P.v + (int64_t)at.t * P.v_row + at.h * P.v_head : P.k + (int64_t)at.t * P.k_row + at.h * P.k_head;
  const uint4 raw = *reinterpret_cast<const uint4*>(src + at.c * 8);
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
  // magnitudes are compared as integers: the order of finite numbers, with infinities and NaNs above them
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = max(top, max(w[i] & 0x7fffu, w[i] >> 16 & 0x7fffu));
  top = max_with<0xB1>(top);  // lane ^ 1
  top = max_with<0x4E>(top);  // lane ^ 2
  // top = m * 2^E with 7 bits of m behind the point: top <= 7 * 2^e = 1.75 * 2^(e + 2) holds from e = E - 2 on if m <= 1.75, else from
  // E - 1 on.  (A subnormal top is far below the smallest scale.)
  const int E = (int)(top >> 7) - 127;
  const int e = min(max((top & 127) <= 96 ? E - 2 : E - 1, -120), 125);
  const bool finite = top < 0x7f80u;
  const uint32_t s = finite ? (uint32_t)(e + 127) : 255u;
  const float scale = __uint_as_float(s << 23);
  uint32_t codes = 0;
  auto lo = [&](int i) { return __uint_as_float(w[i] << 16); };
  auto hi = [&](int i) { return __uint_as_float(w[i] & 0xffff0000u); };
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, lo(0), hi(0), scale, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, lo(1), hi(1), scale, 1);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, lo(2), hi(2), scale, 2);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, lo(3), hi(3), scale, 3);
  *reinterpret_cast<uint32_t*>((at.values ? P.c.v : P.c.k) + at.code) = codes;
  if ((at.c & 3) == 0) (at.values ? P.c.v_scale : P.c.k_scale)[at.scale] = (uint8_t)s;
}

template <int D>
__global__ __launch_bounds__(256) void kv4_read_kernel(const Kv4Params P) {
  const int n = blockIdx.x * 256 + threadIdx.x;
  if (n >= P.items) return;
  const Place<D> at(P, n);
  bf16x8 x = {};
  if (at.inside) {
    const uint32_t codes = *reinterpret_cast<const uint32_t*>((at.values ? P.c.v : P.c.k) + at.code);
    const uint32_t s = (at.values ? P.c.v_scale : P.c.k_scale)[at.scale];
    x = bbm::values_of(codes, bbm::scale_of(s));
  }
  __bf16* const dst = at.values ? P.v + (int64_t)at.t * P.v_row + at.h * P.v_head : P.k + (int64_t)at.t * P.k_row + at.h * P.k_head;
  *reinterpret_cast<bf16x8*>(dst + at.c * 8) = x;
}

int kv4_move(const char* fn, const bbm_packed* k, const bbm_packed* v, int64_t T, const int32_t* slots, const bbm_kv4_cache* cache, bool write, void* stream) {
  using namespace bbm;
  clear_error();
  if (int rc = check_kv4(fn, cache)) return rc;
  if (T < 0) return fail(BBM_EINVAL, "%s: T=%lld must be >= 0", fn, (long long)T);
  if (int rc = check_packed(fn, "k", k, T, cache->Hk, cache->d, !write)) return rc;
  if (int rc = check_packed(fn, "v", v, T, cache->Hk, cache->d, !write)) return rc;
  if ((T > 0 && !slots) || !aligned(slots, 4)) return fail(BBM_EINVAL, "%s: slots must be a non-NULL 4-byte aligned pointer", fn);
  const int64_t items = T > kMaxTokens ? 1ll << 40 : T * cache->Hk * (cache->d / 8) * 2;
  if (items > 0x7fffff00ll) return fail(BBM_EUNSUPPORTED, "%s: problem too large (T=%lld, Hk=%lld)", fn, (long long)T, (long long)cache->Hk);
  if (T == 0) return BBM_OK;
  Kv4Params P;
  P.c = kv4_of(cache);
  P.k = static_cast<__bf16*>(k->ptr), P.v = static_cast<__bf16*>(v->ptr);
  P.k_row = k->row_stride, P.k_head = k->head_stride, P.v_row = v->row_stride, P.v_head = v->head_stride;
  P.slots = slots, P.T = (int32_t)T, P.items = (int32_t)items;
  const unsigned wgs = (unsigned)ceil_div(items, 256);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (write) {
    if (cache->d == 64) kv4_append_kernel<64><<<wgs, 256, 0, s>>>(P);
    else kv4_append_kernel<128><<<wgs, 256, 0, s>>>(P);
  } else {
    if (cache->d == 64) kv4_read_kernel<64><<<wgs, 256, 0, s>>>(P);
    else kv4_read_kernel<128><<<wgs, 256, 0, s>>>(P);
  }
  return launch_status(fn);
}

}  // namespace

extern "C" __attribute__((visibility("default"))) int bbm_kv4_append(const bbm_packed* k, const bbm_packed* v, int64_t T, const int32_t* slots, const bbm_kv4_cache* cache,
                                                                     void* stream) {
  return kv4_move("bbm_kv4_append", k, v, T, slots, cache, true, stream);
}

extern "C" __attribute__((visibility("default"))) int bbm_kv4_read(const int32_t* slots, int64_t T, const bbm_kv4_cache* cache, const bbm_packed* k_out, const bbm_packed* v_out,
                                                                   void* stream) {
  return kv4_move("bbm_kv4_read", k_out, v_out, T, slots, cache, false, stream);
}
