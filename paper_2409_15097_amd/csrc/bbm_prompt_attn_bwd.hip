// Causal attention over packed prompts with grouped heads (include/bbm_tokens.h): gradients.
// A wave takes a query row (dQ) or a key row (dK, dV), 64 keys or queries at a time, one a lane.
#include "bbm_mfma.h"
#include "bbm_packed.h"

namespace {

using bbm::bf16x8;

struct Tensor {
  __bf16* p;
  int64_t row, head;
  __device__ __forceinline__ __bf16* at(int64_t t, int h) const { return p + t * row + h * head; }
};

struct PromptBwdParams {
  Tensor q, k, v, o, d_o, dq, dk, dv;
  const float* lse;
  float* delta;  // [H][T]
  const int32_t* cu;
  int32_t T, R, G;
  float scale;
};

constexpr int kRows = 4;

template <int D>
__device__ __forceinline__ float dot(const float* a, const __bf16* row) {
  float x = 0.0f;
  for (int c = 0; c < D; c += 8) {
    const bf16x8 b = *reinterpret_cast<const bf16x8*>(row + c);
    for (int e = 0; e < 8; ++e) x += a[c + e] * (float)b[e];
  }
  return x;
}

template <int D>
__global__ __launch_bounds__(64 * kRows) void prompt_dq_kernel(const PromptBwdParams P) {
  __shared__ float q_s[kRows][D], g_s[kRows][D];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = blockIdx.y, hk = h / P.G;
  const bbm::Span s = bbm::find_piece(P.cu, P.R, P.T, 1, kRows, blockIdx.x);
  const int i = s.piece * kRows + wave, t = s.begin + i;
  const bool live = t < s.end;
  float delta = 0.0f;
  if (live)
    for (int e = lane; e < D; e += 64) {
      q_s[wave][e] = (float)P.q.at(t, h)[e];
      g_s[wave][e] = (float)P.d_o.at(t, h)[e];
      delta += g_s[wave][e] * (float)P.o.at(t, h)[e];
    }
  __syncthreads();
  if (!live) return;
  for (int b = 32; b; b >>= 1) delta += __shfl_xor(delta, b);
  if (lane == 0) P.delta[(int64_t)h * P.T + t] = delta;
  const float lse = P.lse[(int64_t)h * P.T + t];
  float dq[D / 64] = {};
  for (int j0 = 0; j0 <= i; j0 += 64) {
    const int j = j0 + lane;
    float ds = 0.0f;
    if (j <= i) {
      const float p = __expf(dot<D>(q_s[wave], P.k.at(s.begin + j, hk)) * P.scale - lse);
      ds = p * (dot<D>(g_s[wave], P.v.at(s.begin + j, hk)) - delta);
    }
    for (int jj = 0; jj < min(64, i + 1 - j0); ++jj) {
      const float x = __shfl(ds, jj);
      const __bf16* const row = P.k.at(s.begin + j0 + jj, hk);
      for (int e = 0; e < D / 64; ++e) dq[e] += x * (float)row[e * 64 + lane];
    }
  }
  for (int e = 0; e < D / 64; ++e) P.dq.at(t, h)[e * 64 + lane] = (__bf16)(dq[e] * P.scale);
}

template <int D>
__global__ __launch_bounds__(64 * kRows) void prompt_dkv_kernel(const PromptBwdParams P) {
  __shared__ float k_s[kRows][D], v_s[kRows][D];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, hk = blockIdx.y;
  const bbm::Span s = bbm::find_piece(P.cu, P.R, P.T, 1, kRows, blockIdx.x);
  const int j = s.piece * kRows + wave, t = s.begin + j, n = s.end - s.begin;
  const bool live = t < s.end;
  if (live)
    for (int e = lane; e < D; e += 64) {
      k_s[wave][e] = (float)P.k.at(t, hk)[e];
      v_s[wave][e] = (float)P.v.at(t, hk)[e];
    }
  __syncthreads();
  if (!live) return;
  float dk[D / 64] = {}, dv[D / 64] = {};
  for (int h = hk * P.G; h < (hk + 1) * P.G; ++h)
    for (int i0 = j; i0 < n; i0 += 64) {
      const int i = i0 + lane;
      float p = 0.0f, ds = 0.0f;
      if (i < n) {
        const int64_t at = (int64_t)h * P.T + s.begin + i;
        p = __expf(dot<D>(k_s[wave], P.q.at(s.begin + i, h)) * P.scale - P.lse[at]);
        ds = p * (dot<D>(v_s[wave], P.d_o.at(s.begin + i, h)) - P.delta[at]);
      }
      for (int ii = 0; ii < min(64, n - i0); ++ii) {
        const float pi = __shfl(p, ii), di = __shfl(ds, ii);
        const __bf16* const g = P.d_o.at(s.begin + i0 + ii, h);
        const __bf16* const q = P.q.at(s.begin + i0 + ii, h);
        for (int e = 0; e < D / 64; ++e) {
          dv[e] += pi * (float)g[e * 64 + lane];
          dk[e] += di * (float)q[e * 64 + lane];
        }
      }
    }
  for (int e = 0; e < D / 64; ++e) {
    P.dk.at(t, hk)[e * 64 + lane] = (__bf16)(dk[e] * P.scale);
    P.dv.at(t, hk)[e * 64 + lane] = (__bf16)dv[e];
  }
}

}  // namespace

extern "C" __attribute__((visibility("default"))) size_t bbm_prompt_attn_bwd_workspace_bytes(int64_t T, int64_t H) {
  if (T < 0 || H < 1 || T > bbm::kMaxTokens || H > 65535) return 0;
  return (size_t)(T * H) * sizeof(float);
}

extern "C" __attribute__((visibility("default"))) int bbm_prompt_attn_bwd(const bbm_packed* q, const bbm_packed* k, const bbm_packed* v, const bbm_packed* o,
                                                                          const bbm_packed* d_o, const float* lse, const bbm_packed* dq, const bbm_packed* dk,
                                                                          const bbm_packed* dv, int64_t T, int64_t R, const int32_t* cu, int64_t H, int64_t Hk, int d,
                                                                          float softmax_scale, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace bbm;
  const char* fn = "bbm_prompt_attn_bwd";
  clear_error();
  if (int rc = check_tokens(fn, T, R, cu, H, Hk)) return rc;
  if (d != 64 && d != 128) return fail(BBM_EUNSUPPORTED, "%s: d=%d has no kernel instance (64, 128)", fn, d);
  const struct {
    const char* name;
    const bbm_packed* x;
    int64_t heads;
    bool output;
  } all[] = {{"q", q, H, false}, {"k", k, Hk, false}, {"v", v, Hk, false}, {"o", o, H, false}, {"d_o", d_o, H, false}, {"dq", dq, H, true}, {"dk", dk, Hk, true}, {"dv", dv, Hk, true}};
  for (const auto& a : all)
    if (int rc = check_packed(fn, a.name, a.x, T, a.heads, d, a.output)) return rc;
  if ((T > 0 && !lse) || !aligned(lse, 4)) return fail(BBM_EINVAL, "%s: lse must be a non-NULL 4-byte aligned pointer", fn);
  if (!(softmax_scale > 0.0f) || !(softmax_scale < INFINITY)) return fail(BBM_EINVAL, "%s: softmax_scale must be finite and > 0", fn);
  const size_t need = bbm_prompt_attn_bwd_workspace_bytes(T, H);
  if (need > 0 && (!workspace || workspace_bytes < need))
    return fail(BBM_EWORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need, workspace ? workspace_bytes : (size_t)0);
  if (!aligned(workspace, 16)) return fail(BBM_EINVAL, "%s: workspace must be 16-byte aligned", fn);
  if (T == 0) return BBM_OK;
  PromptBwdParams P;
  Tensor* const to[] = {&P.q, &P.k, &P.v, &P.o, &P.d_o, &P.dq, &P.dk, &P.dv};
  for (int i = 0; i < 8; ++i) *to[i] = Tensor{static_cast<__bf16*>(all[i].x->ptr), all[i].x->row_stride, all[i].x->head_stride};
  P.lse = lse, P.delta = static_cast<float*>(workspace), P.cu = cu;
  P.T = (int32_t)T, P.R = (int32_t)R, P.G = (int32_t)(H / Hk), P.scale = softmax_scale;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const unsigned pieces = (unsigned)count_pieces(T, R, 1, kRows);
  const dim3 rows(pieces, (unsigned)H), keys(pieces, (unsigned)Hk);
  if (d == 64) prompt_dq_kernel<64><<<rows, 64 * kRows, 0, s>>>(P), prompt_dkv_kernel<64><<<keys, 64 * kRows, 0, s>>>(P);
  else prompt_dq_kernel<128><<<rows, 64 * kRows, 0, s>>>(P), prompt_dkv_kernel<128><<<keys, 64 * kRows, 0, s>>>(P);
  return launch_status(fn);
}
