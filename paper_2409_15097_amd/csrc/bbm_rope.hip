// Rotary positions of queries and keys (include/bbm_tokens.h), and with the angles negated their gradient.
//
// Bound by memory: every element is read and written once.  A work-group takes a few tokens with all their heads: it forms
// the sines and cosines of its tokens' angles once, in LDS, and turns all heads of both tensors with them.  An item is two chunks of
// VEC elements: the two halves of VEC pairs, or two chunks that are copied.
// The angle is a product in 64 bits, reduced to a part of a turn there: in 32 bits an angle of 10^5 is off by 4e-3.
#include "bbm_packed.h"

namespace {

constexpr int NT = 256;

struct RopeTensor {
  const __bf16* in;
  __bf16* out;
  int64_t in_row, in_head, out_row, out_head;
};

struct RopeParams {
  RopeTensor x[2];
  const int32_t* positions;
  const float* freqs;
  float mscale, sign;
  int32_t T, H0, H, d, rot, tokens;  // H0 heads of x[0], H of both; tokens of a work-group
};

template <int VEC>
struct Chunk {
  typedef __bf16 type __attribute__((ext_vector_type(VEC)));
};
template <>
struct Chunk<1> {
  typedef __bf16 type __attribute__((ext_vector_type(1)));
};

template <int VEC, bool EVEN>
__global__ __launch_bounds__(NT) void rope_kernel(const RopeParams P) {
  typedef typename Chunk<VEC>::type V;
  extern __shared__ float2 turn_s[];  // (cos, sin) of [token][pair]
  const int tid = threadIdx.x, pairs = P.rot >> 1;
  const int t0 = blockIdx.x * P.tokens, nt = min(P.tokens, P.T - t0);
  for (int n = tid; n < nt * pairs; n += NT) {
    const int t = n / pairs, j = n - t * pairs;
    const double turns = (double)P.positions[t0 + t] * ((double)P.freqs[j] * 0.15915494309189533577);
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    turn_s[n] = make_float2(c * P.mscale, s * P.mscale * P.sign);
  }
  __syncthreads();
  const int per_head = P.d / (2 * VEC), per_token = per_head * P.H;
  for (int n = tid; n < nt * per_token; n += NT) {
    const int t = n / per_token, m = n - t * per_token, h = m / per_head, c = m - h * per_head;
    const RopeTensor& x = P.x[h < P.H0 ? 0 : 1];
    const int hx = h < P.H0 ? h : h - P.H0;
    const __bf16* const in = x.in + (int64_t)(t0 + t) * x.in_row + hx * x.in_head;
    __bf16* const out = x.out + (int64_t)(t0 + t) * x.out_row + hx * x.out_head;
    // neighbouring pairs: chunks 2c and 2c + 1; halves: chunk c of either half, behind them two chunks that are copied
    const bool turned = EVEN || c * VEC < pairs;
    const int a_at = turned && !EVEN ? c * VEC : 2 * c * VEC, b_at = a_at + (turned && !EVEN ? pairs : VEC);
    const V a = *reinterpret_cast<const V*>(in + a_at), b = *reinterpret_cast<const V*>(in + b_at);
    V ya = a, yb = b;
    const float2* const turn = turn_s + t * pairs + c * VEC;
    if constexpr (EVEN) {
#pragma unroll
      for (int e = 0; e < 2 * VEC; e += 2) {
        if (c * VEC + e / 2 < pairs) {
          const float2 w = turn[e / 2];
          const float p = e < VEC ? (float)a[e % VEC] : (float)b[e % VEC], q = e < VEC ? (float)a[e % VEC + 1] : (float)b[e % VEC + 1];
          const __bf16 y1 = (__bf16)(p * w.x - q * w.y), y2 = (__bf16)(q * w.x + p * w.y);
          if (e < VEC) ya[e % VEC] = y1, ya[e % VEC + 1] = y2;
          else yb[e % VEC] = y1, yb[e % VEC + 1] = y2;
        }
      }
    } else if (turned) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float2 w = turn[e];
        ya[e] = (__bf16)((float)a[e] * w.x - (float)b[e] * w.y);
        yb[e] = (__bf16)((float)b[e] * w.x + (float)a[e] * w.y);
      }
    }
    *reinterpret_cast<V*>(out + a_at) = ya;
    *reinterpret_cast<V*>(out + b_at) = yb;
  }
}

}  // namespace

extern "C" __attribute__((visibility("default"))) int bbm_rope(const bbm_packed* q, const bbm_packed* q_out, int64_t H, const bbm_packed* k, const bbm_packed* k_out,
                                                               int64_t Hk, int64_t T, int d, int rot, int interleaved, int inverse, const int32_t* positions,
                                                               const float* freqs, float mscale, void* stream) {
  using namespace bbm;
  const char* fn = "bbm_rope";
  clear_error();
  if (T < 0 || H < 1 || Hk < 0) return fail(BBM_EINVAL, "%s: T=%lld, Hk=%lld must be >= 0, H=%lld >= 1", fn, (long long)T, (long long)Hk, (long long)H);
  if (d < 16 || d > 512 || d % 16) return fail(BBM_EUNSUPPORTED, "%s: d=%d is no multiple of 16 up to 512", fn, d);
  if (rot < 2 || rot > d || rot % 2) return fail(BBM_EINVAL, "%s: rot=%d must be even, 2 .. d=%d", fn, rot, d);
  if (T > kMaxTokens || H + Hk > 65535) return fail(BBM_EUNSUPPORTED, "%s: problem too large (T=%lld, H=%lld, Hk=%lld)", fn, (long long)T, (long long)H, (long long)Hk);
  if (T > 0 && (!positions || !freqs)) return fail(BBM_EINVAL, "%s: positions and freqs must not be NULL", fn);
  if (!aligned(positions, 4) || !aligned(freqs, 4)) return fail(BBM_EINVAL, "%s: positions and freqs must be 4-byte aligned", fn);
  if (!(mscale > -INFINITY && mscale < INFINITY)) return fail(BBM_EINVAL, "%s: mscale must be finite", fn);
  if (int rc = check_packed(fn, "q", q, T, H, d, false)) return rc;
  if (int rc = check_packed(fn, "q_out", q_out, T, H, d, true)) return rc;
  if (Hk > 0) {
    if (int rc = check_packed(fn, "k", k, T, Hk, d, false)) return rc;
    if (int rc = check_packed(fn, "k_out", k_out, T, Hk, d, true)) return rc;
  }
  auto same_or_apart = [&](const bbm_packed* a, const bbm_packed* b) { return a->ptr != b->ptr || (a->row_stride == b->row_stride && a->head_stride == b->head_stride); };
  if (!same_or_apart(q, q_out) || (Hk > 0 && !same_or_apart(k, k_out))) return fail(BBM_EINVAL, "%s: in place, input and output need the same strides", fn);
  if (T == 0) return BBM_OK;
  RopeParams P;
  auto tensor = [](const bbm_packed* a, const bbm_packed* b) {
    return RopeTensor{static_cast<const __bf16*>(a->ptr), static_cast<__bf16*>(b->ptr), a->row_stride, a->head_stride, b->row_stride, b->head_stride};
  };
  P.x[0] = tensor(q, q_out);
  P.x[1] = Hk > 0 ? tensor(k, k_out) : P.x[0];
  P.positions = positions, P.freqs = freqs, P.mscale = mscale, P.sign = inverse ? -1.0f : 1.0f;
  P.T = (int32_t)T, P.H0 = (int32_t)H, P.H = (int32_t)(H + Hk), P.d = d, P.rot = rot;
  // Tokens of a work-group: a few items for every thread, as long as there are four work-groups a CU
  const int64_t items = (H + Hk) * d / 16;
  int64_t tokens = 1;
  while (tokens < 8 && tokens * items < 4 * NT && ceil_div(T, 2 * tokens) >= 1024) tokens *= 2;
  P.tokens = (int32_t)tokens;
  const unsigned wgs = (unsigned)ceil_div(T, tokens);
  const size_t lds = (size_t)(tokens * (rot / 2)) * sizeof(float2);
  hipStream_t s = static_cast<hipStream_t>(stream);
  // halves: chunks must not straddle the middle and the end of the part that is turned
  if (interleaved) rope_kernel<8, true><<<wgs, NT, lds, s>>>(P);
  else if (rot % 16 == 0) rope_kernel<8, false><<<wgs, NT, lds, s>>>(P);
  else if (rot % 8 == 0) rope_kernel<4, false><<<wgs, NT, lds, s>>>(P);
  else if (rot % 4 == 0) rope_kernel<2, false><<<wgs, NT, lds, s>>>(P);
  else rope_kernel<1, false><<<wgs, NT, lds, s>>>(P);
  return launch_status(fn);
}
