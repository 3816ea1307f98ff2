// Causal attention over packed prompts with grouped heads (include/bbm_tokens.h): forward.
// A wave takes a query row of one head, 64 keys at a time, a key a lane.
#include "bbm_mfma.h"
#include "bbm_packed.h"

namespace {

using bbm::bf16x8;

struct PromptParams {
  const __bf16 *q, *k, *v;
  __bf16* o;
  float* lse;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;
  const int32_t* cu;
  int32_t T, R, G;
  float scale;
};

constexpr int kRows = 4;  // rows of a work-group, one a wave

template <int D>
__global__ __launch_bounds__(64 * kRows) void prompt_fwd_kernel(const PromptParams P) {
  __shared__ float q_s[kRows][D];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = blockIdx.y, hk = h / P.G;
  const bbm::Span s = bbm::find_piece(P.cu, P.R, P.T, 1, kRows, blockIdx.x);
  const int i = s.piece * kRows + wave, t = s.begin + i;
  const bool live = t < s.end;
  if (live)
    for (int e = lane; e < D; e += 64) q_s[wave][e] = (float)P.q[(int64_t)t * P.q_row + h * P.q_head + e];
  __syncthreads();
  if (!live) return;
  float m = -INFINITY, l = 0.0f, o[D / 64] = {};
  for (int j0 = 0; j0 <= i; j0 += 64) {
    const int j = j0 + lane;
    float x = -INFINITY;
    if (j <= i) {
      x = 0.0f;
      const __bf16* const row = P.k + (int64_t)(s.begin + j) * P.k_row + hk * P.k_head;
      for (int c = 0; c < D; c += 8) {
        const bf16x8 kk = *reinterpret_cast<const bf16x8*>(row + c);
        for (int e = 0; e < 8; ++e) x += q_s[wave][c + e] * (float)kk[e];
      }
      x *= P.scale;
    }
    float top = x;
    for (int b = 32; b; b >>= 1) top = fmaxf(top, __shfl_xor(top, b));
    const float m_new = fmaxf(m, top), alpha = __expf(m - m_new), p = __expf(x - m_new);
    float sum = p;
    for (int b = 32; b; b >>= 1) sum += __shfl_xor(sum, b);
    l = l * alpha + sum;
    m = m_new;
    for (int e = 0; e < D / 64; ++e) o[e] *= alpha;
    for (int jj = 0; jj < min(64, i + 1 - j0); ++jj) {
      const float pj = __shfl(p, jj);
      const __bf16* const row = P.v + (int64_t)(s.begin + j0 + jj) * P.v_row + hk * P.v_head;
      for (int e = 0; e < D / 64; ++e) o[e] += pj * (float)row[e * 64 + lane];
    }
  }
  for (int e = 0; e < D / 64; ++e) P.o[(int64_t)t * P.o_row + h * P.o_head + e * 64 + lane] = (__bf16)(o[e] / l);
  if (P.lse && lane == 0) P.lse[(int64_t)h * P.T + t] = m + __logf(l);
}

}  // namespace

extern "C" __attribute__((visibility("default"))) int bbm_prompt_attn_fwd(const bbm_packed* q, const bbm_packed* k, const bbm_packed* v, const bbm_packed* o, float* lse,
                                                                          int64_t T, int64_t R, const int32_t* cu, int64_t H, int64_t Hk, int d, float softmax_scale,
                                                                          void* stream) {
  using namespace bbm;
  const char* fn = "bbm_prompt_attn_fwd";
  clear_error();
  if (int rc = check_tokens(fn, T, R, cu, H, Hk)) return rc;
  if (d != 64 && d != 128) return fail(BBM_EUNSUPPORTED, "%s: d=%d has no kernel instance (64, 128)", fn, d);
  if (int rc = check_packed(fn, "q", q, T, H, d, false)) return rc;
  if (int rc = check_packed(fn, "k", k, T, Hk, d, false)) return rc;
  if (int rc = check_packed(fn, "v", v, T, Hk, d, false)) return rc;
  if (int rc = check_packed(fn, "o", o, T, H, d, true)) return rc;
  if (!aligned(lse, 4)) return fail(BBM_EINVAL, "%s: lse must be 4-byte aligned", fn);
  if (!(softmax_scale > 0.0f) || !(softmax_scale < INFINITY)) return fail(BBM_EINVAL, "%s: softmax_scale must be finite and > 0", fn);
  if (T == 0) return BBM_OK;
  PromptParams P;
  P.q = static_cast<const __bf16*>(q->ptr), P.k = static_cast<const __bf16*>(k->ptr), P.v = static_cast<const __bf16*>(v->ptr), P.o = static_cast<__bf16*>(o->ptr);
  P.q_row = q->row_stride, P.q_head = q->head_stride, P.k_row = k->row_stride, P.k_head = k->head_stride;
  P.v_row = v->row_stride, P.v_head = v->head_stride, P.o_row = o->row_stride, P.o_head = o->head_stride;
  P.lse = lse, P.cu = cu, P.T = (int32_t)T, P.R = (int32_t)R, P.G = (int32_t)(H / Hk), P.scale = softmax_scale;
  const dim3 grid((unsigned)count_pieces(T, R, 1, kRows), (unsigned)H);
  if (d == 64) prompt_fwd_kernel<64><<<grid, 64 * kRows, 0, static_cast<hipStream_t>(stream)>>>(P);
  else prompt_fwd_kernel<128><<<grid, 64 * kRows, 0, static_cast<hipStream_t>(stream)>>>(P);
  return launch_status(fn);
}
