// Weights that the keys of the 4-bit cache gather (include/bbm_cache.h): out = decay * weights + the sum of exp(scale <q, k> - lse) over the queries that see a key.
//
// One kernel, no exchange between work-groups: a wave owns 64 keys of one key head at a time and walks the columns (query token, head of the group) of its request, or of
// its group for shared keys, 16 at a time:
//   S = K Q^T (16 keys x 16 columns x 32 elements an instruction): lane (n, q) = (l % 16, l / 16) loads D / 4 elements of key n from q * D / 4 on, and of column n likewise, and has
//   the scores of keys 4 q .. 4 q + 3 with column n; their exponentials are added up in the lane, and over 16 lanes at the end.
// With up to 16 columns the cache's bytes are the bound (half of the attention's, values are not read: 17/32 byte an element, and 8 a key), so the next keys are under
// way while these are used; with more, the codes are converted once for all columns, and the products and exponentials are the bound.
#include "bbm_cache.h"
#include "bbm_kv4.h"

#include <algorithm>

namespace {

using bbm::bf16x8, bbm::Kv4, bbm::scalar;
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr int NW = 4;
constexpr int NB = 4;                // blocks of 16 keys that a wave has
constexpr int kStep = 16 * NB * NW;  // keys of a work-group's step

struct WeightParams {
  Kv4 c;
  const __bf16* q;
  const float* lse;
  const float* weights;
  float* out;
  int64_t q_row, q_head, table_stride;
  const int32_t *cu, *lens, *table, *group_cu, *shared_lens;
  const uint64_t* mask;
  int32_t T, R, S, G, max_pages, mask_words;
  int32_t group_parts, own_parts;  // work-groups of a group and key head, of a request and key head
  int32_t group_wgs, own_wgs;      // of all of them
  float rc, decay;                 // softmax_scale * log2(e)
};

// Whose keys a work-group has, and who looks at them.
struct Owner {
  int r;            // row of the block table
  int begin, end;   // rows of the queries
  int from, len;    // its keys
  int prefix;       // keys in front of the new tokens (causal: of the first one that has a row here)
  int fresh;        // from this key on, new tokens
};
__device__ __forceinline__ int max_keys(const WeightParams& P) { return (int)min((int64_t)P.max_pages << P.c.page_shift, (int64_t)0x7fffffff); }
__device__ __forceinline__ int shared_of(const WeightParams& P, int g) { return (int)scalar(max(0, min(P.shared_lens[g], max_keys(P))) & ~15); }
__device__ __forceinline__ int row_cut(const WeightParams& P, int c) { return min(max(c, 0), P.T); }
__device__ __forceinline__ int request_cut(const WeightParams& P, int g) { return min(max(P.group_cu[g], 0), P.R); }
__device__ __forceinline__ Owner owner_of_group(const WeightParams& P, int g) {
  const int r0 = request_cut(P, g), r1 = request_cut(P, g + 1);
  Owner x;
  x.begin = (int)scalar(row_cut(P, P.cu[r0])), x.end = (int)scalar(row_cut(P, P.cu[r1]));
  x.r = min((int)scalar(r0), P.R - 1);
  x.from = 0;
  x.len = x.prefix = x.fresh = shared_of(P, g);
  return x;
}
__device__ __forceinline__ Owner owner_of_request(const WeightParams& P, int r) {
  const int c0 = (int)scalar(P.cu[r]), c1 = (int)scalar(P.cu[r + 1]), len = (int)scalar(P.lens[r]);
  Owner x;
  x.r = r;
  x.begin = row_cut(P, c0), x.end = row_cut(P, c1);
  x.fresh = (int)((uint32_t)len - (uint32_t)max(0, c1 - c0));
  x.prefix = P.mask ? x.fresh : (int)((uint32_t)x.fresh + (uint32_t)x.begin - (uint32_t)c0);
  x.len = max(0, min(len, max_keys(P)));
  const int g = bbm::group_of(P.group_cu, P.S, r);
  x.from = g >= 0 ? min(shared_of(P, g), x.len) : 0;
  return x;
}

template <int D>
__global__ __launch_bounds__(64 * NW, 3) void kv4_weights_kernel(const WeightParams P) {
  constexpr int KS = D / 32;  // steps of a product, and words of codes that a lane loads of a key
  const int lane = threadIdx.x & 63, n = lane & 15, kq = lane >> 4;
  const int wave = (int)scalar(threadIdx.x >> 6);
  const int ahead = (P.group_wgs + 7) & ~7;  // (a multiple of 8, so that both kinds spread over the XCDs alike)
  const bool group = (int)blockIdx.x < ahead;
  const int wg = (int)blockIdx.x - (group ? 0 : ahead), total = group ? P.group_wgs : P.own_wgs, parts = group ? P.group_parts : P.own_parts;
  if (wg >= total) return;
  const int at = bbm::logical_wg(wg, total), part = at % parts, hk = at / parts % P.c.Hk, unit = at / parts / P.c.Hk;
  const Owner x = group ? owner_of_group(P, unit) : owner_of_request(P, unit);
  const int cols = (x.end - x.begin) * P.G;
  if (x.end <= x.begin) return;

  struct Raw {
    uint32_t k[NB][KS], ks[NB];
    f32x4 old;       // of the four keys that this lane writes: 4 kq .. of block n (n < NB)
    int64_t place;   // where they lie
    int have;        // how many of them are there
  };
  const bbm::Table table = (bbm::Table)(uintptr_t)(P.table + x.r * P.table_stride);
  struct Pages {
    int p[NB];
  };
  auto pages_at = [&](int j) __attribute__((always_inline)) {
    Pages y;
#pragma unroll
    for (int b = 0; b < NB; ++b) y.p[b] = table[scalar(min(j + 16 * b, x.len - 1) >> P.c.page_shift)];
    return y;
  };
  // the wave's 64 keys from j on; of those that are not there zeros, and of the weights the cache's first
  auto load = [&](Raw& z, int j, const Pages& pages) __attribute__((always_inline)) {
    z.have = 0;
    z.place = 0;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int jb = j + 16 * b, page = pages.p[b];
      const bool there = jb < x.len && page >= 0 && page < P.c.pages;
      const int64_t key = ((int64_t)page * P.c.Hk + hk) * P.c.page + (jb & (P.c.page - 1));
      const __amdgpu_buffer_rsrc_t k_r = bbm::buffer_of(P.c.k + key * (D / 2), there ? 16 * (D / 2) : 0), ks_r = bbm::buffer_of(P.c.k_scale + key * (D / 32), there ? D / 2 : 0);
      if constexpr (D == 128) {
        const bbm::u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(k_r, n * (D / 2) + kq * 16, 0, 0);
        for (int i = 0; i < 4; ++i) z.k[b][i] = w[i];
      } else {
        const bbm::u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(k_r, n * (D / 2) + kq * 8, 0, 0);
        for (int i = 0; i < 2; ++i) z.k[b][i] = w[i];
      }
      z.ks[b] = __builtin_amdgcn_raw_buffer_load_b8(ks_r, n * (D / 32) + kq * D / 128, 0, 0);
      if (n == b && there) z.have = max(0, min(4, x.len - jb - 4 * kq)), z.place = key + 4 * kq;
    }
    z.old = *reinterpret_cast<const f32x4*>(P.weights + z.place);
  };
  auto store = [&](const Raw& z, int j, f32x4 (&sum)[NB]) __attribute__((always_inline)) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) sum[b][r] = bbm::row_sum<16>(sum[b][r]);
    f32x4 y = n == 0 ? sum[0] : n == 1 ? sum[1] : n == 2 ? sum[2] : sum[3];
    const int fresh = x.fresh - (j + 16 * n + 4 * kq);  // how many of the four were there before
#pragma unroll
    for (int r = 0; r < 4; ++r) y[r] += r < fresh ? P.decay * z.old[r] : 0.0f;
    if (z.have == 4) {
      *reinterpret_cast<f32x4*>(P.out + z.place) = y;
    } else {
#pragma unroll
      for (int r = 0; r < 3; ++r)
        if (r < z.have) P.out[z.place + r] = y[r];
    }
  };

  // The lane's column, 16 further with every tile: its token and head, and where its query and its log-sum-exp lie.
  struct Column {
    int col, i, g;
    const __bf16* q;
    const float* lse;
  };
  const int di = 16 / P.G, dg = 16 % P.G;
  const __bf16* const q0 = P.q + (int64_t)x.begin * P.q_row + (int64_t)hk * P.G * P.q_head + kq * (D / 4);
  const float* const lse0 = P.lse + (int64_t)hk * P.G * P.T + x.begin;
  auto column = [&](int c) __attribute__((always_inline)) {
    Column y;
    y.col = c, y.i = c / P.G, y.g = c - y.i * P.G;
    y.q = q0 + y.i * P.q_row + y.g * P.q_head;
    y.lse = lse0 + (int64_t)y.g * P.T + y.i;
    return y;
  };
  auto advance = [&](Column& y) __attribute__((always_inline)) {
    y.col += 16, y.i += di, y.g += dg;
    y.q += di * P.q_row + dg * P.q_head;
    y.lse += (int64_t)dg * P.T + di;
    if (y.g >= P.G) {
      y.g -= P.G, y.i += 1;
      y.q += P.q_row - P.G * P.q_head;
      y.lse += 1 - (int64_t)P.G * P.T;
    }
  };
  struct Query {
    bf16x8 q[KS];
    float nl;  // what is added to its exponents
  };
  // (columns behind the last read the first one's query, and add nothing)
  auto fetch = [&](const Column& y) __attribute__((always_inline)) {
    Query z;
    const bool there = y.col < cols;
    const __bf16* const p = there ? y.q : q0;
    const float l = *(there ? y.lse : lse0);
#pragma unroll
    for (int s = 0; s < KS; ++s) z.q[s] = *reinterpret_cast<const bf16x8*>(p + 8 * s);
    z.nl = there && l != -INFINITY ? l * -kLog2e : -INFINITY;
    return z;
  };
  // the exponentials of 16 keys from j on with the lane's column; all_see: the last key that all 16 columns see
  auto add = [&](f32x4& sum, f32x4 s, const Query& z, const Column& y, int j, int all_see) __attribute__((always_inline)) {
    f32x4 p;
#pragma unroll
    for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], P.rc, z.nl));
    if (j + 15 > all_see) {
      const int i = min(y.i, x.end - x.begin - 1);
      const uint32_t seen = (uint32_t)bbm::seen_from(P.mask ? P.mask + (int64_t)(x.begin + i) * P.mask_words : nullptr, P.mask_words, i, j + 4 * kq - x.prefix);
#pragma unroll
      for (int r = 0; r < 4; ++r) p[r] = seen >> r & 1 ? p[r] : 0.0f;
    }
    sum += p;
  };

  int j = x.from + part * kStep + wave * (16 * NB);
  if (j >= x.len) return;
  const int next = parts * kStep;
  if (cols <= 16) {
    const Column y = column(n);
    const Query z = fetch(y);
    const int all_see = P.mask ? x.prefix - 1 : x.prefix;
    auto use = [&](Raw& a, int j) __attribute__((always_inline)) {
      f32x4 sum[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        f32x4 s = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        sum[b] = s;
#pragma unroll
        for (int i = 0; i < KS; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bbm::values_of(a.k[b][i], bbm::scale_of(a.ks[b])), z.q[i], s, 0, 0, 0);
        add(sum[b], s, z, y, j + 16 * b, all_see);
      }
      store(a, j, sum);
    };
    // the next keys are asked for before these are used, their pages a step before that
    Raw a, b;
    load(a, j, pages_at(j));
    Pages pages = pages_at(j + next);
#pragma unroll 1
    for (;;) {
      load(b, j + next, pages);
      pages = pages_at(j + 2 * next);
      use(a, j);
      j += next;
      if (j >= x.len) return;
      load(a, j + next, pages);
      pages = pages_at(j + 2 * next);
      use(b, j);
      j += next;
      if (j >= x.len) return;
    }
  }
#pragma unroll 1
  for (; j < x.len; j += next) {
    Raw a;
    load(a, j, pages_at(j));
    // (a causal key is seen by no column in front of its own token's)
    const int start = P.mask ? 0 : min(max(0, j - x.prefix), x.end - x.begin - 1) * P.G & ~15;
    Column y = column(start + n);
    Query z = fetch(y);
    bf16x8 k[NB][KS];
    f32x4 sum[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      sum[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < KS; ++i) k[b][i] = bbm::values_of(a.k[b][i], bbm::scale_of(a.ks[b]));
    }
    int i0 = start / P.G, g0 = start - i0 * P.G;  // the tile's first column
#pragma unroll 1
    for (int c = start; c < cols; c += 16) {
      const int all_see = P.mask ? x.prefix - 1 : x.prefix + i0;
      Column yn = y;
      advance(yn);
      const Query zn = fetch(yn);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        f32x4 s = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < KS; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[b][i], z.q[i], s, 0, 0, 0);
        add(sum[b], s, z, y, j + 16 * b, all_see);
      }
      y = yn, z = zn;
      i0 += di, g0 += dg;
      if (g0 >= P.G) g0 -= P.G, i0 += 1;
    }
    store(a, j, sum);
  }
}

// Work-groups of an owner: enough to fill the chip, no more than it has steps for.
constexpr int64_t kFill = 2048, kMaxParts = 1 << 17;  // (two steps behind a key are still a 32-bit number)
inline int64_t parts_of(int64_t owners, int64_t Hk, int64_t keys, bool many_columns) {
  const int64_t steps = bbm::ceil_div(std::min<int64_t>(keys, bbm::kMaxTokens), kStep);
  return std::min(many_columns ? steps : std::min(steps, bbm::ceil_div(kFill, owners * Hk)), kMaxParts);
}

}  // namespace

extern "C" __attribute__((visibility("default"))) int bbm_kv4_weights(const bbm_packed* q, const float* lse, int64_t T, int64_t R, const int32_t* cu, const int32_t* lens,
                                                                      const int32_t* block_table, int64_t table_stride, int64_t max_pages, int64_t S, const int32_t* group_cu,
                                                                      const int32_t* shared_lens, const uint64_t* mask, int64_t mask_words, const bbm_kv4_cache* cache, int64_t H,
                                                                      float softmax_scale, float decay, const float* weights, float* out, int64_t max_shared, int64_t max_own,
                                                                      void* stream) {
  using namespace bbm;
  const char* fn = "bbm_kv4_weights";
  clear_error();
  if (int rc = check_kv4(fn, cache)) return rc;
  if (int rc = check_tokens(fn, T, R, cu, H, cache->Hk)) return rc;
  if (int rc = check_packed(fn, "q", q, T, H, cache->d, false)) return rc;
  if ((T > 0 && !lse) || !aligned(lse, 4)) return fail(BBM_EINVAL, "%s: lse must be a non-NULL 4-byte aligned pointer", fn);
  if (int rc = check_table(fn, lens, block_table, table_stride, max_pages, cache->page)) return rc;
  if (int rc = check_groups(fn, R, S, group_cu, shared_lens, max_shared, max_own)) return rc;
  if (int rc = check_mask(fn, mask, mask_words)) return rc;
  if (int rc = check_scale(fn, softmax_scale)) return rc;
  if (!(decay >= 0.0f && decay <= 1.0f)) return fail(BBM_EINVAL, "%s: decay=%g is outside 0 .. 1", fn, (double)decay);
  if (!weights || !out || !aligned(weights, 16) || !aligned(out, 16)) return fail(BBM_EINVAL, "%s: weights and out must be non-NULL 16-byte aligned pointers", fn);
  const int64_t G = H / cache->Hk;
  if (T * G > kMaxTokens) return fail(BBM_EUNSUPPORTED, "%s: problem too large (T=%lld, H=%lld)", fn, (long long)T, (long long)H);
  if (T == 0) return BBM_OK;
  if (int rc = check_apart(fn, {out}, {q->ptr, lse, cu, lens, block_table, mask, cache->k, cache->k_scale, S > 0 ? group_cu : nullptr, S > 0 ? shared_lens : nullptr})) return rc;
  WeightParams P = {};
  P.c = kv4_of(cache);
  P.q = static_cast<const __bf16*>(q->ptr), P.lse = lse, P.weights = weights, P.out = out;
  P.q_row = q->row_stride, P.q_head = q->head_stride, P.table_stride = table_stride;
  P.cu = cu, P.lens = lens, P.table = block_table, P.group_cu = group_cu, P.shared_lens = shared_lens, P.mask = mask;
  P.T = (int32_t)T, P.R = (int32_t)R, P.S = (int32_t)S, P.G = (int32_t)G, P.max_pages = (int32_t)max_pages, P.mask_words = (int32_t)mask_words;
  P.rc = softmax_scale * kLog2e, P.decay = decay;
  const int64_t group_parts = S > 0 ? parts_of(S, cache->Hk, max_shared, T * G > 16 * S) : 1, own_parts = parts_of(R, cache->Hk, max_own, T * G > 16 * R);
  const int64_t group_wgs = S * cache->Hk * group_parts, own_wgs = R * cache->Hk * own_parts;
  if (R * cache->Hk >= kMaxWgs || group_wgs >= kMaxWgs / 2 || own_wgs >= kMaxWgs / 2)
    return fail(BBM_EUNSUPPORTED, "%s: problem too large (R=%lld, Hk=%lld, keys %lld and %lld)", fn, (long long)R, (long long)cache->Hk, (long long)max_shared, (long long)max_own);
  P.group_parts = (int32_t)group_parts, P.own_parts = (int32_t)own_parts, P.group_wgs = (int32_t)group_wgs, P.own_wgs = (int32_t)own_wgs;
  const unsigned wgs = (unsigned)(((group_wgs + 7) & ~7ll) + own_wgs);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (cache->d == 64) kv4_weights_kernel<64><<<wgs, 64 * NW, 0, s>>>(P);
  else kv4_weights_kernel<128><<<wgs, 64 * NW, 0, s>>>(P);
  return launch_status(fn);
}
