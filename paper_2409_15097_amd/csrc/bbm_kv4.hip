// Writing to and reading from the 4-bit cache (include/bbm_tokens.h).  Bound by memory: 2 bytes an element on the one side, 17/32 on the
// other.  Four lanes share a group of 32 elements, 8 each: 16 bytes of bf16 and 4 bytes of codes a lane, the largest magnitude of
// the group over two exchanges between neighbouring lanes.  A thread takes the same place of K and of V, so that finding it is paid once.
// 16384 tokens of 8 heads of 128: 21 us either way, 85 MB at 4.1 TB/s (25 and 26 with the threads of a launch shared out between K and V); 64 tokens 2.8 us.
#include "bbm_kv4.h"

namespace {

using bbm::bf16x8, bbm::Kv4;

struct Kv4Params {
  Kv4 c;
  __bf16 *k, *v;
  int64_t k_row, k_head, v_row, v_head;
  const int32_t* slots;
  uint32_t items, per_token, inverse;  // 8 elements of both tensors each; of a token; 2^32 / per_token, rounded down
};

template <int CTRL>
__device__ __forceinline__ uint32_t max_with(uint32_t x) {
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true));
}

// Where an item's bytes lie in the cache.
template <int D>
struct Place {
  uint32_t t, h, c;  // token, head, 8-element chunk
  int64_t code, k_scale, v_scale;
  bool inside;
  __device__ __forceinline__ Place(const Kv4Params& P, uint32_t n) {
    t = __umulhi(n, P.inverse);  // n / per_token, or one less
    uint32_t m = n - t * P.per_token;
    if (m >= P.per_token) ++t, m -= P.per_token;
    h = m / (D / 8);
    c = m % (D / 8);
    const int slot = P.slots[t];
    const int page = slot >> P.c.page_shift, at = slot & (P.c.page - 1);
    inside = slot >= 0 && page < P.c.pages;
    const int64_t head = (int64_t)page * P.c.Hk + h, key = (head << P.c.page_shift) + at;
    code = key * (D / 2) + c * 4;
    k_scale = key * (D / 32) + c / 4;
    v_scale = ((head * (D / 32) + c / 4) << P.c.page_shift) + at;
  }
};

// Eight elements of a group as codes, and the group's scale byte.
__device__ __forceinline__ uint32_t encode(const uint4& raw, uint32_t& s) {
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
  s = top < 0x7f80u ? (uint32_t)(e + 127) : 255u;
  const float scale = __uint_as_float(s << 23);
  auto lo = [&](int i) { return __uint_as_float(w[i] << 16); };
  auto hi = [&](int i) { return __uint_as_float(w[i] & 0xffff0000u); };
  uint32_t codes = 0;
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, lo(0), hi(0), scale, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, lo(1), hi(1), scale, 1);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, lo(2), hi(2), scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, lo(3), hi(3), scale, 3);
}

template <int D>
__global__ __launch_bounds__(256) void kv4_append_kernel(const Kv4Params P) {
  const uint32_t n = blockIdx.x * 256 + threadIdx.x;
  if (n >= P.items) return;  // (whole groups: the items of a group are in or out together)
  const Place<D> at(P, n);
  if (!at.inside) return;
  const uint4 k = *reinterpret_cast<const uint4*>(P.k + (int64_t)at.t * P.k_row + at.h * P.k_head + at.c * 8);
  const uint4 v = *reinterpret_cast<const uint4*>(P.v + (int64_t)at.t * P.v_row + at.h * P.v_head + at.c * 8);
  uint32_t ks, vs;
  const uint32_t kc = encode(k, ks), vc = encode(v, vs);
  *reinterpret_cast<uint32_t*>(P.c.k + at.code) = kc;
  *reinterpret_cast<uint32_t*>(P.c.v + at.code) = vc;
  if ((at.c & 3) == 0) {
    P.c.k_scale[at.k_scale] = (uint8_t)ks;
    P.c.v_scale[at.v_scale] = (uint8_t)vs;
  }
}

template <int D>
__global__ __launch_bounds__(256) void kv4_read_kernel(const Kv4Params P) {
  const uint32_t n = blockIdx.x * 256 + threadIdx.x;
  if (n >= P.items) return;
  const Place<D> at(P, n);
  bf16x8 k = {}, v = {};
  if (at.inside) {
    const uint32_t kc = *reinterpret_cast<const uint32_t*>(P.c.k + at.code), vc = *reinterpret_cast<const uint32_t*>(P.c.v + at.code);
    const uint32_t ks = P.c.k_scale[at.k_scale], vs = P.c.v_scale[at.v_scale];
    k = bbm::values_of(kc, bbm::scale_of(ks));
    v = bbm::values_of(vc, bbm::scale_of(vs));
  }
  *reinterpret_cast<bf16x8*>(P.k + (int64_t)at.t * P.k_row + at.h * P.k_head + at.c * 8) = k;
  *reinterpret_cast<bf16x8*>(P.v + (int64_t)at.t * P.v_row + at.h * P.v_head + at.c * 8) = v;
}

int kv4_move(const char* fn, const bbm_packed* k, const bbm_packed* v, int64_t T, const int32_t* slots, const bbm_kv4_cache* cache, bool write, void* stream) {
  using namespace bbm;
  clear_error();
  if (int rc = check_kv4(fn, cache)) return rc;
  if (T < 0) return fail(BBM_EINVAL, "%s: T=%lld must be >= 0", fn, (long long)T);
  const int64_t per_token = cache->Hk * (cache->d / 8);
  if (T > 0x7fffff00ll / per_token) return fail(BBM_EUNSUPPORTED, "%s: problem too large (T=%lld, Hk=%lld)", fn, (long long)T, (long long)cache->Hk);
  if (int rc = check_packed(fn, "k", k, T, cache->Hk, cache->d, !write)) return rc;
  if (int rc = check_packed(fn, "v", v, T, cache->Hk, cache->d, !write)) return rc;
  if ((T > 0 && !slots) || !aligned(slots, 4)) return fail(BBM_EINVAL, "%s: slots must be a non-NULL 4-byte aligned pointer", fn);
  const int64_t items = T * per_token;
  if (T == 0) return BBM_OK;
  const bbm_kv4_cache& c = *cache;
  if (int rc = write ? check_apart(fn, {c.k, c.k_scale, c.v, c.v_scale}, {k->ptr, v->ptr, slots}) : check_apart(fn, {k->ptr, v->ptr}, {slots, c.k, c.k_scale, c.v, c.v_scale}))
    return rc;
  Kv4Params P;
  P.c = kv4_of(cache);
  P.k = static_cast<__bf16*>(k->ptr), P.v = static_cast<__bf16*>(v->ptr);
  P.k_row = k->row_stride, P.k_head = k->head_stride, P.v_row = v->row_stride, P.v_head = v->head_stride;
  P.slots = slots, P.items = (uint32_t)items, P.per_token = (uint32_t)per_token, P.inverse = (uint32_t)((1ll << 32) / per_token);
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
