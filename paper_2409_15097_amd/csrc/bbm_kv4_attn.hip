// Attention of new tokens over the 4-bit cache (include/bbm_tokens.h).
// A wave takes a query row of one head, 64 keys at a time, a key a lane.
#include "bbm_kv4.h"

namespace {

using bbm::bf16x8, bbm::Kv4;

struct Kv4AttnParams {
  Kv4 c;
  const __bf16* q;
  __bf16* o;
  float* lse;
  int64_t q_row, q_head, o_row, o_head, table_stride;
  const int32_t *cu, *lens, *table;
  const uint64_t* mask;
  int32_t T, R, G, max_pages, mask_words;
  float scale;
};

constexpr int kRows = 4;

template <int D>
__global__ __launch_bounds__(64 * kRows) void kv4_attn_kernel(const Kv4AttnParams P) {
  __shared__ float q_s[kRows][D];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = blockIdx.y, hk = h / P.G;
  const bbm::Span s = bbm::find_piece(P.cu, P.R, P.T, 1, kRows, blockIdx.x);
  const int i = s.piece * kRows + wave, t = s.begin + i;
  const bool live = t < s.end;
  if (live)
    for (int e = lane; e < D; e += 64) q_s[wave][e] = (float)P.q[(int64_t)t * P.q_row + h * P.q_head + e];
  __syncthreads();
  if (!live) return;
  const int len = min((int64_t)P.lens[s.r], (int64_t)P.max_pages << P.c.page_shift), prefix = P.lens[s.r] - (s.end - s.begin);
  auto page_of = [&](int j) { return P.table[s.r * P.table_stride + (j >> P.c.page_shift)]; };
  auto sees = [&](int j) {
    if (j >= len) return false;
    const int page = page_of(j);
    if (page < 0 || page >= P.c.pages) return false;
    if (!P.mask) return j <= prefix + i;
    const int n = j - prefix;
    return n < 0 || (n / 64 < P.mask_words && (P.mask[(int64_t)t * P.mask_words + n / 64] >> (n % 64) & 1) != 0);
  };
  float m = -INFINITY, l = 0.0f, o[D / 64] = {};
  for (int j0 = 0; j0 < len; j0 += 64) {
    const int j = j0 + lane;
    float x = -INFINITY;
    if (sees(j)) {
      x = 0.0f;
      const int64_t at = ((int64_t)page_of(j) * P.c.Hk + hk) * P.c.page + (j & (P.c.page - 1));
      for (int c = 0; c < D; c += 8) {
        const bf16x8 kk = bbm::values_of(*reinterpret_cast<const uint32_t*>(P.c.k + at * (D / 2) + c / 2), bbm::scale_of(P.c.k_scale[at * (D / 32) + c / 32]));
        for (int e = 0; e < 8; ++e) x += q_s[wave][c + e] * (float)kk[e];
      }
      x *= P.scale;
    }
    float top = x;
    for (int b = 32; b; b >>= 1) top = fmaxf(top, __shfl_xor(top, b));
    const float m_new = fmaxf(m, top), m_fin = m_new == -INFINITY ? 0.0f : m_new;
    const float alpha = __expf(m - m_fin), p = __expf(x - m_fin);
    float sum = p;
    for (int b = 32; b; b >>= 1) sum += __shfl_xor(sum, b);
    l = l * alpha + sum;
    m = m_new;
    for (int e = 0; e < D / 64; ++e) o[e] *= alpha;
    for (uint64_t todo = __ballot(x > -INFINITY); todo; todo &= todo - 1) {
      const int jj = __ffsll((unsigned long long)todo) - 1;
      const float pj = __shfl(p, jj);
      const int64_t head = (int64_t)page_of(j0 + jj) * P.c.Hk + hk;
      const int at = (j0 + jj) & (P.c.page - 1);
      for (int e = 0; e < D / 64; ++e) {
        const int c = e * 64 + lane;
        const bf16x8 vv = bbm::values_of(P.c.v[(head * P.c.page + at) * (D / 2) + c / 2], bbm::scale_of(P.c.v_scale[(head * (D / 32) + c / 32) * P.c.page + at]));
        o[e] += pj * (float)(c & 1 ? vv[1] : vv[0]);
      }
    }
  }
  for (int e = 0; e < D / 64; ++e) P.o[(int64_t)t * P.o_row + h * P.o_head + e * 64 + lane] = (__bf16)(l > 0.0f ? o[e] / l : 0.0f);
  if (P.lse && lane == 0) P.lse[(int64_t)h * P.T + t] = l > 0.0f ? m + __logf(l) : -INFINITY;
}

}  // namespace

extern "C" __attribute__((visibility("default"))) size_t bbm_kv4_attn_workspace_bytes(int64_t T, int64_t R, int64_t H, int64_t Hk, int d, int64_t max_len) {
  (void)T, (void)R, (void)H, (void)Hk, (void)d, (void)max_len;
  return 0;
}

extern "C" __attribute__((visibility("default"))) int bbm_kv4_attn(const bbm_packed* q, const bbm_packed* o, float* lse, int64_t T, int64_t R, const int32_t* cu,
                                                                   const int32_t* lens, const int32_t* block_table, int64_t table_stride, int64_t max_pages,
                                                                   const uint64_t* mask, int64_t mask_words, const bbm_kv4_cache* cache, int64_t H,
                                                                   float softmax_scale, int64_t max_len, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace bbm;
  const char* fn = "bbm_kv4_attn";
  clear_error();
  if (int rc = check_kv4(fn, cache)) return rc;
  if (int rc = check_tokens(fn, T, R, cu, H, cache->Hk)) return rc;
  if (int rc = check_packed(fn, "q", q, T, H, cache->d, false)) return rc;
  if (int rc = check_packed(fn, "o", o, T, H, cache->d, true)) return rc;
  if (!lens || !aligned(lens, 4) || !block_table || !aligned(block_table, 4)) return fail(BBM_EINVAL, "%s: lens and block_table must be non-NULL 4-byte aligned pointers", fn);
  if (!aligned(lse, 4) || !aligned(mask, 8)) return fail(BBM_EINVAL, "%s: lse must be 4-byte aligned, mask 8-byte aligned", fn);
  if (max_pages < 1 || table_stride < max_pages || max_len < 1)
    return fail(BBM_EINVAL, "%s: max_pages=%lld, max_len=%lld must be >= 1, table_stride=%lld no less than max_pages", fn, (long long)max_pages, (long long)max_len, (long long)table_stride);
  if (mask ? mask_words < 1 : mask_words != 0) return fail(BBM_EINVAL, "%s: mask_words=%lld does not fit the mask", fn, (long long)mask_words);
  if (max_pages * cache->page >= (1ll << 31) || mask_words > (1 << 20)) return fail(BBM_EUNSUPPORTED, "%s: max_pages=%lld or mask_words=%lld is too large", fn, (long long)max_pages, (long long)mask_words);
  if (!(softmax_scale > 0.0f) || !(softmax_scale < INFINITY)) return fail(BBM_EINVAL, "%s: softmax_scale must be finite and > 0", fn);
  const size_t need = bbm_kv4_attn_workspace_bytes(T, R, H, cache->Hk, cache->d, max_len);
  if (need > 0 && (!workspace || workspace_bytes < need))
    return fail(BBM_EWORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need, workspace ? workspace_bytes : (size_t)0);
  if (!aligned(workspace, 16)) return fail(BBM_EINVAL, "%s: workspace must be 16-byte aligned", fn);
  if (T == 0) return BBM_OK;
  Kv4AttnParams P;
  P.c = kv4_of(cache);
  P.q = static_cast<const __bf16*>(q->ptr), P.o = static_cast<__bf16*>(o->ptr), P.lse = lse;
  P.q_row = q->row_stride, P.q_head = q->head_stride, P.o_row = o->row_stride, P.o_head = o->head_stride, P.table_stride = table_stride;
  P.cu = cu, P.lens = lens, P.table = block_table, P.mask = mask;
  P.T = (int32_t)T, P.R = (int32_t)R, P.G = (int32_t)(H / cache->Hk), P.max_pages = (int32_t)max_pages, P.mask_words = (int32_t)mask_words, P.scale = softmax_scale;
  const dim3 grid((unsigned)count_pieces(T, R, 1, kRows), (unsigned)H);
  if (cache->d == 64) kv4_attn_kernel<64><<<grid, 64 * kRows, 0, static_cast<hipStream_t>(stream)>>>(P);
  else kv4_attn_kernel<128><<<grid, 64 * kRows, 0, static_cast<hipStream_t>(stream)>>>(P);
  return launch_status(fn);
}
