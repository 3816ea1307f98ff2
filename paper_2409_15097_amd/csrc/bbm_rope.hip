// Rotary positions of queries and keys (include/bbm_tokens.h), and with the angles negated their gradient.
//
// Bound by memory: every element is read and written once.  A work-group takes a few tokens with all their heads: it forms
// the sines and cosines of its tokens' angles once, in LDS, and turns all heads of both tensors with them.
// 16381 tokens of 40 heads of 128 elements: 66 us with rot = 128, 69 with 64 or neighbouring pairs, 4.9 - 5.1 TB/s (a large copy reaches
// 4.8); 33 tokens: 3.8 us, a launch and three trips to memory.  Streaming stores: 84 us, 89 with streaming loads too.
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

typedef __bf16 Chunk __attribute__((ext_vector_type(8)));

// (cos, sin) of the angles of tokens t0 .. t0 + nt - 1, [token][pair]; a barrier has to follow.
__device__ __forceinline__ void turns_of(const RopeParams& P, float2* turn_s, int t0, int nt, int pairs) {
  for (int n = threadIdx.x; n < nt * pairs; n += NT) {
    const int t = n / pairs, j = n - t * pairs;
    const double turns = (double)P.positions[t0 + t] * ((double)P.freqs[j] * 0.15915494309189533577);
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    turn_s[n] = make_float2(c * P.mscale, s * P.mscale * P.sign);
  }
}

// An item is two chunks of 8 elements: the two halves of 8 pairs, or (EVEN: always) two chunks side by side, turned or copied.
template <bool EVEN>
__global__ __launch_bounds__(NT) void rope_kernel(const RopeParams P) {
  extern __shared__ __align__(16) float2 turn_s[];
  const int tid = threadIdx.x, pairs = P.rot >> 1;
  const int t0 = blockIdx.x * P.tokens, nt = min(P.tokens, P.T - t0);
  turns_of(P, turn_s, t0, nt, pairs);
  __syncthreads();
  const int per_head = P.d / 16, per_token = per_head * P.H;
  for (int n = tid; n < nt * per_token; n += NT) {
    const int t = n / per_token, m = n - t * per_token, h = m / per_head, c = m - h * per_head;
    const RopeTensor& x = P.x[h < P.H0 ? 0 : 1];
    const int hx = h < P.H0 ? h : h - P.H0;
    const __bf16* const in = x.in + (int64_t)(t0 + t) * x.in_row + hx * x.in_head;
    __bf16* const out = x.out + (int64_t)(t0 + t) * x.out_row + hx * x.out_head;
    // neighbouring pairs: chunks 2c and 2c + 1; halves: chunk c of either half, behind them two chunks that are copied
    const bool turned = EVEN || c * 8 < pairs;
    const int a_at = turned && !EVEN ? c * 8 : 16 * c, b_at = a_at + (turned && !EVEN ? pairs : 8);
    const Chunk a = *reinterpret_cast<const Chunk*>(in + a_at), b = *reinterpret_cast<const Chunk*>(in + b_at);
    Chunk ya = a, yb = b;
    const float2* const turn = turn_s + t * pairs + c * 8;
    if constexpr (EVEN) {
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        if (c * 8 + e / 2 < pairs) {
          const float2 w = turn[e / 2];
          const float p = e < 8 ? (float)a[e % 8] : (float)b[e % 8], q = e < 8 ? (float)a[e % 8 + 1] : (float)b[e % 8 + 1];
          const __bf16 y1 = (__bf16)(p * w.x - q * w.y), y2 = (__bf16)(q * w.x + p * w.y);
          if (e < 8) ya[e % 8] = y1, ya[e % 8 + 1] = y2;
          else yb[e % 8] = y1, yb[e % 8 + 1] = y2;
        }
      }
    } else if (turned) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 w = turn[e];
        ya[e] = (__bf16)((float)a[e] * w.x - (float)b[e] * w.y);
        yb[e] = (__bf16)((float)b[e] * w.x + (float)a[e] * w.y);
      }
    }
    *reinterpret_cast<Chunk*>(out + a_at) = ya;
    *reinterpret_cast<Chunk*>(out + b_at) = yb;
  }
}

// Halves whose middle or end lies inside a chunk: whole heads go through LDS, STEP chunks a thread at a time, and an element finds the other
// one of its pair there.  (All of a head is read before any of it is written, also in place.)  16381 tokens of 40 heads of 128, rot = 126, 100, 44:
// 75, 75, 73 us; with items of one, two and two pairs in rope_kernel 158, 101, 114 us (33 tokens: 5.1 us against 6.1, 4.6 and 4.7).
constexpr int STEP = 2;
__global__ __launch_bounds__(NT) void rope_staged_kernel(const RopeParams P) {
  extern __shared__ __align__(16) float2 turn_s[];
  const int tid = threadIdx.x, pairs = P.rot >> 1;
  const int t0 = blockIdx.x * P.tokens, nt = min(P.tokens, P.T - t0);
  __bf16* const x_s = reinterpret_cast<__bf16*>(turn_s + (P.tokens * pairs + 1) / 2 * 2);
  turns_of(P, turn_s, t0, nt, pairs);
  const int per_head = P.d / 8, step_heads = STEP * NT / per_head, heads = nt * P.H;
  for (int h0 = 0; h0 < heads; h0 += step_heads) {
    Chunk a[STEP];
    __bf16* out[STEP];
    int at[STEP], turn[STEP];
    if (h0 > 0) __syncthreads();  // (the last step's readers of x_s)
#pragma unroll
    for (int u = 0; u < STEP; ++u) {
      const int n = tid + u * NT, hl = n / per_head, g = h0 + hl;
      out[u] = nullptr;
      if (hl >= step_heads || g >= heads) continue;
      const int t = g / P.H, h = g - t * P.H;
      const RopeTensor& x = P.x[h < P.H0 ? 0 : 1];
      const int hx = h < P.H0 ? h : h - P.H0;
      at[u] = (n - hl * per_head) * 8, turn[u] = t * pairs;
      a[u] = *reinterpret_cast<const Chunk*>(x.in + (int64_t)(t0 + t) * x.in_row + hx * x.in_head + at[u]);
      out[u] = x.out + (int64_t)(t0 + t) * x.out_row + hx * x.out_head + at[u];
      *reinterpret_cast<Chunk*>(x_s + n * 8) = a[u];
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < STEP; ++u) {
      if (!out[u]) continue;
      Chunk y = a[u];
      if (at[u] < P.rot) {
        const __bf16* const row = x_s + (tid + u * NT) * 8;  // this chunk
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int i = at[u] + e;
          const bool first = i < pairs, turned = i < P.rot;
          const int other = first ? pairs : -pairs;
          const float2 w = turn_s[turn[u] + (turned ? (first ? i : i - pairs) : 0)];
          const float p = (float)a[u][e], q = (float)row[turned ? e + other : e];
          // as the kernel above rounds it: the first of a pair p c - q s, the second p c + q s
          const float r = first ? p * w.x - q * w.y : p * w.x + q * w.y;
          y[e] = turned ? (__bf16)r : a[u][e];
        }
      }
      *reinterpret_cast<Chunk*>(out[u]) = y;
    }
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
  if (T > kMaxTokens || H > 65535 || Hk > 65535 - H) return fail(BBM_EUNSUPPORTED, "%s: problem too large (T=%lld, H=%lld, Hk=%lld)", fn, (long long)T, (long long)H, (long long)Hk);
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
  // Tokens of a work-group: a few items for every thread, as long as there are four work-groups a CU and 16 KiB hold their angles
  const int64_t items = (H + Hk) * d / 16;
  int64_t tokens = 1;
  while (tokens * items < 4 * NT && 2 * tokens * (rot / 2) <= 2048 && ceil_div(T, 2 * tokens) >= 1024) tokens *= 2;
  P.tokens = (int32_t)tokens;
  if (ceil_div(T, tokens) >= kMaxWgs) return fail(BBM_EUNSUPPORTED, "%s: problem too large (T=%lld, H=%lld)", fn, (long long)T, (long long)H);
  // (a tensor is turned in place, or into a place that is no input)
  if (int rc = check_apart(fn, {q_out->ptr, Hk > 0 ? k_out->ptr : nullptr}, {positions, freqs})) return rc;
  if (Hk > 0 && (q_out->ptr == k->ptr || k_out->ptr == q->ptr)) return fail(BBM_EINVAL, "%s: an output must not be the other tensor's input", fn);
  const unsigned wgs = (unsigned)ceil_div(T, tokens);
  const size_t lds = (size_t)(tokens * (rot / 2) + 1) / 2 * 2 * sizeof(float2);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (interleaved) rope_kernel<true><<<wgs, NT, lds, s>>>(P);
  else if (rot % 16 == 0) rope_kernel<false><<<wgs, NT, lds, s>>>(P);
  else rope_staged_kernel<<<wgs, NT, lds + STEP * NT * 16, s>>>(P);
  return launch_status(fn);
}
