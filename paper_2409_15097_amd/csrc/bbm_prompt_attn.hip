// Causal attention over packed prompts with grouped heads (include/bbm_tokens.h): forward.
//
// One pass over the keys with the running maximum and sum of a softmax.  A work-group takes 32 * NW query rows of one head of one sequence, a
// wave 32 of them, one lane a row (with its partner l ^ 32): the transposed products S^T = K Q^T and O^T += V^T P^T, as in the forward under
// masks.  Keys come in tiles of 64 through LDS, copied while the tile before is multiplied.  No mask is in memory: the tiles in front of
// the work-group's first row are seen whole; of those from there on a lane's row gives the keys that it sees.
// Scores are not rounded between the products: the scale multiplies them inside the exponential, in fp32, one fused multiply-add an
// element.  P is rounded to bf16 for the second product, half a step each, and summed before that.
// Bound by the matrix instructions with the exponentials between them: two prompts of 8192 and 6554 tokens, 32 heads of 128, 0.90 TFLOP counted as
// the pairs that are seen, 800 - 850 us a call, 1.06 - 1.13 PFLOP/s (a large bf16 product reaches 1.14 on this card; the matrix pipe is busy for 60 % of the cycles of a
// clock that falls to 1.5 GHz); 4096 tokens, 32 / 8 heads of 64, 87 us, 0.79 PFLOP/s; short prompts by one chain of tiles: 37 of 1 to 300 tokens, 16 heads of 64, 9.5 us.
#include "bbm_mfma.h"
#include "bbm_prompt.h"
#include "bbm_softmax.h"

namespace {

using bbm::bf16x8, bbm::f32x16, bbm::global, bbm::IntC, bbm::mfma_ring, bbm::partner_sum, bbm::scalar, bbm::TileAddr, bbm::TL;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLazy = 8.0f;  // the running maximum moves when a row exceeds it by a factor of 2^8: P and its sum keep their relative precision

struct PromptParams {
  bbm::Rows q, k, v, o;
  float* lse;
  const int32_t* cu;
  int32_t T, R, G, H, pieces;
  float rc;    // softmax_scale * log2(e)
  float lazy;  // kLazy as a difference of scores
};
typedef bbm::InPlace<PromptParams> Args;

__device__ __forceinline__ float partner_max(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// HALVES = 2 (short launches): a work-group takes 64 rows, and two waves share 32 of them, each with 32 keys of every tile; their results meet behind the
// last one.
template <int D, int HALVES>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void prompt_fwd_kernel(const PromptParams) {
  Args P = bbm::kernel_args<PromptParams>();
  using L = TL<D>;
  constexpr int NW = 4, BR = 32 * NW / HALVES, KS = D / 16, DB = D / 32;
  constexpr int KB = 2 / HALVES;  // halves of a tile's keys that a wave takes
  static_assert(2 * 32 * D <= L::ELEMS, "two 32 x D slabs must fit in a tile buffer");
  __shared__ __attribute__((aligned(16))) __bf16 k_s0[L::ELEMS];
  __shared__ __attribute__((aligned(16))) __bf16 k_s1[L::ELEMS];
  __shared__ __attribute__((aligned(16))) __bf16 v_s0[L::ELEMS];
  __shared__ __attribute__((aligned(16))) __bf16 v_s1[L::ELEMS];

  const int lane = threadIdx.x & 63, lq = lane & 31, hh = lane >> 5;
  const int wave = (int)scalar(threadIdx.x >> 6);
  const int half = HALVES == 2 ? wave & 1 : 0;  // of the keys
  const bbm::Work work = bbm::work_of(blockIdx.x, P->H);
  const int h = work.plane;
  if (work.number >= P->pieces) return;
  const bbm::Span s = bbm::find_piece(global(P->cu), P->R, P->T, 1, BR, P->pieces - 1 - work.number);  // (long rows first)
  const int n = s.end - s.begin, row0 = s.piece * BR;
  if (n <= 0) return;
  const int wrow = row0 + 32 * (wave / HALVES), wrows = max(0, min(32, n - wrow));  // this wave's rows
  const int n_tiles = (min(n, row0 + BR) + 63) / 64, n_full = row0 / 64 & ~1;
  const float rc = P->rc, lazy = P->lazy;

  const int k_row = P->k.row, v_row = P->v.row;
  const __bf16* const kg = global(P->k.p) + h / P->G * P->k.head + (int64_t)s.begin * k_row;
  const __bf16* const vg = global(P->v.p) + h / P->G * P->v.head + (int64_t)s.begin * v_row;
  bbm::TileCopy<D, NW> kc, vc;
  kc.init(wave, lane, k_row);
  vc.init(wave, lane, v_row);
  constexpr int LPW = bbm::TileCopy<D, NW>::PIECES;
  auto copy_piece = [&](int jt, int rows, __bf16* kd, __bf16* vd, int i) {
    if (i < LPW)
      kc.piece(kg + (int64_t)jt * 64 * k_row, rows, k_row, kd, i, wave);
    else
      vc.piece(vg + (int64_t)jt * 64 * v_row, rows, v_row, vd, i - LPW, wave);
  };
  auto rows_at = [&](int jt) { return jt < n_tiles ? bbm::rows_of_tile(jt * 64, n) : 0; };

  // Q by way of the buffers of parity 1, the first tile into those of parity 0
  __bf16* const q_stage = (wave / 2 == 0 ? k_s1 : v_s1) + wave % 2 * 32 * D;
  bbm::copy_slab<D>(global(P->q.p) + h * P->q.head + (int64_t)(s.begin + wrow) * P->q.row, wrows, P->q.row, q_stage, lane);
#pragma unroll
  for (int i = 0; i < 2 * LPW; ++i) copy_piece(0, rows_at(0), k_s0, v_s0, i);
  TileAddr<D> A;
  A.init(lane);
  for (int i = 0; i < 2; ++i) {  // this wave's keys of a tile
    A.ra[i] += half * (32 / L::NBLK) * D;
    A.ta[i] += 2 * half * (D == 64 ? 2 * D : D);
  }
  bf16x8 qf[KS];
  f32x16 oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
    for (int e = 0; e < 16; ++e) oacc[db][e] = 0.0f;
  bbm::RunningMax top;
  float l_run = 0.0f;
  __builtin_amdgcn_s_waitcnt(0);
#pragma unroll
  for (int t = 0; t < KS; ++t) qf[t] = bbm::slab_frag<D>(q_stage, t, lane);

  auto step = [&](auto pb, auto part, int jt) __attribute__((always_inline)) {
    constexpr int PB = decltype(pb)::value;
    constexpr bool PART = decltype(part)::value != 0;
    __builtin_amdgcn_s_waitcnt(0);  // this wave's copies of the tile have landed
    __syncthreads();                // ... and everyone's; every wave is done with the buffers refilled below
    __bf16* const k_cur = PB ? k_s1 : k_s0;
    __bf16* const v_cur = PB ? v_s1 : v_s0;
    __bf16* const k_oth = PB ? k_s0 : k_s1;
    __bf16* const v_oth = PB ? v_s0 : v_s1;
    // the next tile's copies go out between the matrix instructions of the first product; behind the last tile they copy zero rows
    const int rows1 = rows_at(jt + 1);
    const bool live = wrows > 0 && (!PART || jt * 64 + 32 * half < wrow + wrows);
    if (!live) {
#pragma unroll
      for (int i = 0; i < 2 * LPW; ++i) copy_piece(jt + 1, rows1, k_oth, v_oth, i);
      return;
    }
    f32x16 sc[KB];
    __builtin_amdgcn_s_setprio(2);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
      for (int e = 0; e < 16; ++e) sc[kb][e] = 0.0f;
    mfma_ring<KB * KS, 4>([&](auto i) { return A.row_frag(k_cur, decltype(i)::value % KB, decltype(i)::value / KB); },
                          [&](auto i, bf16x8 f) {
                            constexpr int x = decltype(i)::value;
                            sc[x % KB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, qf[x / KB], sc[x % KB], 0, 0, 0);
                          },
                          [&](auto i) {
                            constexpr int x = decltype(i)::value, GAP = KB * KS / (2 * LPW);  // matrix instructions per copy
                            static_assert(GAP * 2 * LPW == KB * KS, "the copies must find room");
                            if constexpr (x % GAP == 0) copy_piece(jt + 1, rows1, k_oth, v_oth, x / GAP);
                          });
    __builtin_amdgcn_s_setprio(0);
    if constexpr (PART) {
      const uint64_t seen = bbm::bits_up_to(wrow + lq - jt * 64 - 32 * half);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const uint32_t w = (uint32_t)(seen >> (32 * kb)) >> (4 * hh);
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[kb][e] = bbm::keep_if(w, e, sc[kb][e]);
      }
    }
    float mx = sc[0][0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sc[kb][e]);
    top.update(partner_max(mx), lazy, rc, [&](float alpha) __attribute__((always_inline)) {
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db)
        for (int e = 0; e < 16; ++e) oacc[db][e] *= alpha;
    });
    if (top.far) {
      const float off = top.offset(rc);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
        for (int e = 0; e < 16; ++e) sc[kb][e] -= off;
    }
    __builtin_amdgcn_s_setprio(1);
    // the exponentials of 16 keys behind the matrix instructions of the 16 before
    bf16x8 pf[2];
    auto exps = [&](int u, int e0, int e1) {
#pragma unroll
      for (int e = e0; e < e1; ++e) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[u / 2][8 * (u % 2) + e], rc, top.nm));
        l_run += p;  // (before it is rounded: the log-sum-exp is an fp32 result)
        pf[u & 1][e] = (__bf16)p;
      }
    };
    exps(0, 0, 8);
    mfma_ring<2 * KB * DB, 3>([&](auto i) { return A.tr_frag(v_cur, decltype(i)::value / DB, decltype(i)::value % DB); },
                         [&](auto i, bf16x8 f) {
                           constexpr int x = decltype(i)::value;
                           oacc[x % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, pf[x / DB & 1], oacc[x % DB], 0, 0, 0);
                         },
                         [&](auto i) {
                           constexpr int x = decltype(i)::value, PER = 8 / DB;
                           if constexpr (x / DB < 2 * KB - 1) exps(x / DB + 1, x % DB * PER, (x % DB + 1) * PER);
                         });
    __builtin_amdgcn_s_setprio(0);
  };

  // tiles seen whole, two at a time (the buffers change places with every tile), then one or two that are not, or of which one is
#pragma unroll 1
  for (int jt = 0; jt < n_full; jt += 2) {
    step(IntC<0>{}, IntC<0>{}, jt);
    step(IntC<1>{}, IntC<0>{}, jt + 1);
  }
  step(IntC<0>{}, IntC<1>{}, n_full);
  if (n_full + 1 < n_tiles) step(IntC<1>{}, IntC<1>{}, n_full + 1);
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();  // the output is staged in the tile buffers
  if constexpr (HALVES == 2) {
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    static_assert((32 * D + 2 * 64) * sizeof(float) <= L::ELEMS * sizeof(__bf16), "a wave's sums and statistics must fit in a tile buffer");
    f32x4* const sums = reinterpret_cast<f32x4*>(wave / 2 == 0 ? k_s1 : v_s1) + lane;
    float2* const stats = reinterpret_cast<float2*>((wave / 2 == 0 ? k_s1 : v_s1) + 32 * D * 2) + lane;
    if (half == 1) {
#pragma unroll
      for (int i = 0; i < 4 * DB; ++i) sums[i * 64] = f32x4{oacc[i / 4][i % 4 * 4], oacc[i / 4][i % 4 * 4 + 1], oacc[i / 4][i % 4 * 4 + 2], oacc[i / 4][i % 4 * 4 + 3]};
      *stats = make_float2(top.m, l_run);
    }
    __syncthreads();
    if (half == 1) return;
    const float2 other = *stats;
    const float m_new = fmaxf(top.m, other.x), m_fin = m_new == -INFINITY ? 0.0f : m_new;
    const float w0 = bbm::weight(top.m, m_fin, rc), w1 = bbm::weight(other.x, m_fin, rc);
    l_run = w0 * l_run + w1 * other.y;
    top.m = m_new;
#pragma unroll
    for (int i = 0; i < 4 * DB; ++i) {
      const f32x4 y = sums[i * 64];
      for (int e = 0; e < 4; ++e) oacc[i / 4][i % 4 * 4 + e] = w0 * oacc[i / 4][i % 4 * 4 + e] + w1 * y[e];
    }
  }
  if (wrows == 0) return;
  const float l_tot = partner_sum(l_run);
  __bf16* const stage = (wave / 2 == 0 ? k_s0 : v_s0) + wave % 2 * 32 * D;
  bbm::store_strided<D>(oacc, 1.0f / l_tot, stage, global(P->o.p) + h * P->o.head + (int64_t)(s.begin + wrow) * P->o.row, wrows, P->o.row, lane);
  if (global(P->lse) && hh == 0 && lq < wrows) global(P->lse)[(int64_t)h * P->T + s.begin + wrow + lq] = bbm::log_sum(top.m, l_tot, rc);
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
  if (int rc = check_rows(fn, "q", q, T, H, d, false)) return rc;
  if (int rc = check_rows(fn, "k", k, T, Hk, d, false)) return rc;
  if (int rc = check_rows(fn, "v", v, T, Hk, d, false)) return rc;
  if (int rc = check_rows(fn, "o", o, T, H, d, true)) return rc;
  if (!aligned(lse, 4)) return fail(BBM_EINVAL, "%s: lse must be 4-byte aligned", fn);
  if (int rc = check_scale(fn, softmax_scale)) return rc;
  if (T == 0) return BBM_OK;
  if (int rc = check_apart(fn, {o->ptr, lse}, {q->ptr, k->ptr, v->ptr, cu})) return rc;
  PromptParams P;
  P.q = rows_of(q, T, d), P.k = rows_of(k, T, d), P.v = rows_of(v, T, d), P.o = rows_of(o, T, d);
  P.lse = lse, P.cu = cu, P.T = (int32_t)T, P.R = (int32_t)R, P.G = (int32_t)(H / Hk), P.H = (int32_t)H, P.rc = softmax_scale * kLog2e, P.lazy = kLazy / P.rc;
  const bool halves = split_keys(T, R, H);
  const int64_t pieces = count_pieces(T, R, 1, halves ? 64 : 128), wgs = work_groups(H, pieces);
  if (wgs >= kMaxWgs) return fail(BBM_EUNSUPPORTED, "%s: problem too large (T=%lld, H=%lld)", fn, (long long)T, (long long)H);
  P.pieces = (int32_t)pieces;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (halves) {
    if (d == 64) prompt_fwd_kernel<64, 2><<<(unsigned)wgs, 256, 0, s>>>(P);
    else prompt_fwd_kernel<128, 2><<<(unsigned)wgs, 256, 0, s>>>(P);
  } else {
    if (d == 64) prompt_fwd_kernel<64, 1><<<(unsigned)wgs, 256, 0, s>>>(P);
    else prompt_fwd_kernel<128, 1><<<(unsigned)wgs, 256, 0, s>>>(P);
  }
  return launch_status(fn);
}
