// Slots of a step (include/bbm_tokens.h): two prefix sums over the requests (new tokens, pages asked for), then every token and
// every page of the step finds its request in them.
//
// A step needs the whole sums before anything else, and R requests are few against the tokens of a long step: every
// work-group forms both sums for itself in LDS (8 R bytes read from the cache, no second launch, no exchange between work-groups) and
// then takes its share of the tokens and of the new pages, each of which is found by bisection in LDS.
// Bound by latency: 64 requests of a token each 3.3 us, of which a launch is 2; 1000 requests of up to 256 tokens (128 thousand, 63 work-groups) 8.0.
#include "bbm_packed.h"

namespace {

constexpr int NT = 1024;
constexpr int kTokensPerWg = 2048;

struct SlotParams {
  const int32_t *ctx, *add;
  int32_t* table;
  const int32_t *free_pages, *free_at;
  int32_t *cu, *lens, *positions, *slots, *free_next;
  int64_t table_stride;
  int64_t n_free;
  int32_t R, T, max_pages, page_shift;
};

__device__ __forceinline__ int clamped(int x) { return max(x, 0); }
// tokens in the cache behind the step, within 31 bits
__device__ __forceinline__ int total(int ctx, int add) { return (int)min((int64_t)ctx + add, (int64_t)0x7fffffff); }

__global__ __launch_bounds__(NT) void slots_kernel(const SlotParams P) {
  extern __shared__ int32_t sums[];  // cu [R + 1], pages taken before request r [R + 1]
  __shared__ int32_t wave_s[2][NT / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int32_t* const cu_s = sums;
  int32_t* const pg_s = sums + P.R + 1;
  const int round = (1 << P.page_shift) - 1;
  auto pages = [&](int n) { return (int)min(((int64_t)n + round) >> P.page_shift, (int64_t)P.max_pages); };

  // a thread's `per` requests lie one behind the other
  const int per = (P.R + NT - 1) / NT, r0 = tid * per, r1 = min(P.R, r0 + per);
  int n = 0, g = 0;
  for (int r = r0; r < r1; ++r) {
    const int c = clamped(P.ctx[r]), a = clamped(P.add[r]);
    n += a;
    g += pages(total(c, a)) - pages(c);
  }
  int in = n, ig = g;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int x = __shfl_up(in, d), y = __shfl_up(ig, d);
    if (lane >= d) in += x, ig += y;
  }
  if (lane == 63) wave_s[0][wave] = in, wave_s[1][wave] = ig;
  __syncthreads();
  int bn = in - n, bg = ig - g;
  for (int w = 0; w < wave; ++w) bn += wave_s[0][w], bg += wave_s[1][w];
  for (int r = r0; r < r1; ++r) {
    const int c = clamped(P.ctx[r]), a = clamped(P.add[r]), t = total(c, a);
    cu_s[r] = bn;
    pg_s[r] = bg;
    if (blockIdx.x == 0) {
      P.cu[r] = bn;
      P.lens[r] = t;
    }
    bn += a;
    bg += pages(t) - pages(c);
    if (r == P.R - 1) {
      cu_s[P.R] = bn;
      pg_s[P.R] = bg;
    }
  }
  __syncthreads();
  const int n_new = cu_s[P.R], n_pages = pg_s[P.R], from = *P.free_at;
  if (blockIdx.x == 0 && tid == 0) {
    P.cu[P.R] = n_new;
    *P.free_next = from + n_pages;
  }
  // the last request whose sum is at most x
  auto find = [&](const int32_t* s, int x) {
    int lo = 0, hi = P.R;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s[mid] <= x) lo = mid;
      else hi = mid;
    }
    return lo;
  };
  auto free_page = [&](int f) {  // page number f of those that the step takes
    const int64_t at = (int64_t)from + f;
    return at >= 0 && at < P.n_free ? P.free_pages[at] : -1;
  };
  for (int f = blockIdx.x * NT + tid; f < n_pages; f += gridDim.x * NT) {
    const int r = find(pg_s, f);
    const int col = pages(clamped(P.ctx[r])) + (f - pg_s[r]);
    if (col < P.max_pages) P.table[(int64_t)r * P.table_stride + col] = free_page(f);
  }
  for (int t = blockIdx.x * NT + tid; t < P.T; t += gridDim.x * NT) {
    int pos = 0, slot = -1;
    if (t < n_new) {
      const int r = find(cu_s, t), c = clamped(P.ctx[r]);
      pos = total(c, clamped(t - cu_s[r]));  // (not negative, whatever the sums were)
      const int col = pos >> P.page_shift, held = pages(c);
      // (a page that the step takes comes from the list: the table's entry may not have been written yet)
      const int page = col >= P.max_pages ? -1 : col < held ? P.table[(int64_t)r * P.table_stride + col] : free_page(pg_s[r] + col - held);
      const int64_t s = ((int64_t)page << P.page_shift) + (pos & round);
      if (page >= 0 && s <= 0x7fffffff) slot = (int)s;
    }
    P.positions[t] = pos;
    P.slots[t] = slot;
  }
}

}  // namespace

extern "C" __attribute__((visibility("default"))) int bbm_build_slots(const int32_t* ctx_lens, const int32_t* new_lens, int64_t R, int32_t* block_table,
                                                                      int64_t table_stride, int64_t max_pages, int page, const int32_t* free_pages,
                                                                      int64_t n_free, const int32_t* free_at, int64_t T, int32_t* cu_new, int32_t* lens,
                                                                      int32_t* positions, int32_t* slots, int32_t* free_next, void* stream) {
  using namespace bbm;
  const char* fn = "bbm_build_slots";
  clear_error();
  if (R < 1 || T < 0 || max_pages < 1 || n_free < 0)
    return fail(BBM_EINVAL, "%s: R=%lld, max_pages=%lld must be >= 1, T=%lld, n_free=%lld >= 0", fn, (long long)R, (long long)max_pages, (long long)T, (long long)n_free);
  if (!ctx_lens || !new_lens || !block_table || !free_at || !cu_new || !lens || !free_next || (T > 0 && (!positions || !slots)) || (n_free > 0 && !free_pages))
    return fail(BBM_EINVAL, "%s: no pointer may be NULL", fn);
  for (const void* p : {(const void*)ctx_lens, (const void*)new_lens, (const void*)block_table, (const void*)free_pages, (const void*)free_at, (const void*)cu_new,
                        (const void*)lens, (const void*)positions, (const void*)slots, (const void*)free_next})
    if (!aligned(p, 4)) return fail(BBM_EINVAL, "%s: pointers must be 4-byte aligned", fn);
  if (table_stride < max_pages) return fail(BBM_EINVAL, "%s: table_stride=%lld is less than max_pages=%lld", fn, (long long)table_stride, (long long)max_pages);
  if (page != 16 && page != 32 && page != 64 && page != 128) return fail(BBM_EUNSUPPORTED, "%s: page=%d is none of 16, 32, 64, 128", fn, page);
  if (R > BBM_SLOTS_MAX_REQUESTS) return fail(BBM_EUNSUPPORTED, "%s: R=%lld requests, more than %d", fn, (long long)R, BBM_SLOTS_MAX_REQUESTS);
  if (T > kMaxTokens || max_pages > 0x7fffffffll / R)  // (by division: a product of the caller's may wrap)
    return fail(BBM_EUNSUPPORTED, "%s: T=%lld or R=%lld times max_pages=%lld is too large", fn, (long long)T, (long long)R, (long long)max_pages);
  // (Every work-group reads the inputs while others write.  The pointers of no tokens or no pages may be anything.)
  if (int rc = check_apart(fn, {cu_new, lens, T > 0 ? positions : nullptr, T > 0 ? slots : nullptr, free_next, block_table}, {ctx_lens, new_lens, n_free > 0 ? free_pages : nullptr, free_at}))
    return rc;
  SlotParams P;
  P.ctx = ctx_lens, P.add = new_lens, P.table = block_table, P.free_pages = free_pages, P.free_at = free_at;
  P.cu = cu_new, P.lens = lens, P.positions = positions, P.slots = slots, P.free_next = free_next;
  P.table_stride = table_stride, P.n_free = n_free;
  P.R = (int32_t)R, P.T = (int32_t)T, P.max_pages = (int32_t)max_pages;
  P.page_shift = page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : 7;
  const size_t lds = (size_t)(2 * (R + 1)) * sizeof(int32_t);
  int64_t wgs = ceil_div(T, kTokensPerWg);
  wgs = wgs < 1 ? 1 : wgs > 256 ? 256 : wgs;
  if (lds > (64u << 10)) {
    // (of the function on the current device; a repeated call changes nothing)
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(slots_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, 8 * (BBM_SLOTS_MAX_REQUESTS + 1));
    if (e != hipSuccess) return fail(BBM_EHIP, "%s: %s", fn, hipGetErrorString(e));
  }
  slots_kernel<<<(unsigned)wgs, NT, lds, static_cast<hipStream_t>(stream)>>>(P);
  return launch_status(fn);
}
