// Causal attention over packed prompts with grouped heads (include/bbm_tokens.h): gradients.
//
// With P = exp(scale Q K^T - lse) on the pairs that are seen, dP = dO V^T, D_i = <dO_i, O_i>, dS = P o (dP - D):
//   dV = P^T dO,   dK = scale * dS^T Q,   dQ = scale * dS K,   dK and dV summed over the heads of a group.
// Without atomics, so that results do not depend on an order.  One kernel leaves -D and -lse / scale in the workspace, one launch takes both gradients:
//   dQ          a work-group takes 128 query rows of one head, a lane a row (HALVES: 64, two lanes a row, each with half the keys), and walks its tiles of
//               64 keys: S^T = K Q^T, dP^T = V dO^T, dQ^T += K^T dS^T;
//   dK and dV   a work-group takes 64 keys of one key head and walks the tiles of 64 queries of every head of the group, a wave 32 keys and
//               32 queries of a tile: S = Q K^T, dP = dO V^T, dV^T += dO^T P, dK^T += Q^T dS, all in its registers.
// Each step is one chain of matrix instructions with the copies of the next tile, the exponentials and the roundings behind them.  As in the forward
// the scale multiplies the scores inside the exponential in fp32; P and dS are rounded to bf16 for the products that they enter, dS once, from the
// fp32 P (from the rounded one the gradients are no faster, 570 against 568 us for 1 x 4096 tokens, 32 / 8 heads of 128, and dK off by 0.0030 instead of 0.0025), and D is formed from the
// O that the forward rounded, which is the O that was used: <dO, O> as a program would form it.
// Bound by the matrix instructions: sequences of 4096 and 3277 tokens, 32 / 8 heads of 128, forward and backward, 0.79 TFLOP (pairs that are seen) in 920 - 985 us;
// with the scores and dP that dQ and dK, dV both form, 9 products are multiplied where 7 are counted, 1.03 - 1.10 PFLOP/s.  Short sequences by a chain of steps of
// 0.5 to 1 us: 13 of 1 to 1024, 16 heads of 64, 34 us.
#include "bbm_mfma.h"
#include "bbm_prompt.h"

#include <algorithm>

namespace {

using bbm::bf16x8, bbm::buffer_of, bbm::copy_async, bbm::f32x16, bbm::global, bbm::IntC, bbm::lane_now, bbm::mfma_ring, bbm::operand, bbm::pack, bbm::Rows,
    bbm::scalar, bbm::TileAddr, bbm::TL;

constexpr float kLog2e = 1.4426950408889634f;

struct PromptBwdParams {
  Rows q, k, v, o, d_o, dq, dk, dv;
  const float* lse;
  float* nls;     // workspace [H][T]: -lse / scale, what the scores start at
  float* ndelta;  // workspace [H][T]: -<dO, O>
  float* partials;  // workspace [part][dV, dK][Hk][T][d], of more than one part
  const int32_t* cu;
  int32_t T, R, G, H, row_pieces, key_pieces, parts, key_wgs;
  float rc;  // softmax_scale * log2(e)
  float scale;
};
typedef bbm::InPlace<PromptBwdParams> Args;

// HALVES = 2: 64 rows a work-group, two waves share 32 of them and halve the keys of every tile, as in the forward.
// t_s0, t_s1: [K, V] tiles, one variable per parity.
template <int D, int HALVES>
__device__ __forceinline__ void dq_of(Args P, int wg, __bf16* t_s0, __bf16* t_s1) {
  using L = TL<D>;
  constexpr int NW = 4, BR = 32 * NW / HALVES, KB = 2 / HALVES, KS = D / 16, DB = D / 32;
  __bf16 *const k_s0 = t_s0, *const v_s0 = t_s0 + L::ELEMS, *const k_s1 = t_s1, *const v_s1 = t_s1 + L::ELEMS;

  const int lane = threadIdx.x & 63, lq = lane & 31, hh = lane >> 5;
  const int wave = (int)scalar(threadIdx.x >> 6);
  const int half = HALVES == 2 ? wave & 1 : 0;  // of the keys
  const bbm::Work work = bbm::work_of(wg, P->H);
  const int h = work.plane;
  if (work.number >= P->row_pieces) return;
  const bbm::Span s = bbm::find_piece(global(P->cu), P->R, P->T, 1, BR, P->row_pieces - 1 - work.number);
  const int n = s.end - s.begin, row0 = s.piece * BR;
  if (n <= 0) return;
  const int wrow = row0 + 32 * (wave / HALVES), wrows = max(0, min(32, n - wrow));
  const int n_tiles = (min(n, row0 + BR) + 63) / 64, n_full = row0 / 64 & ~1;
  const float rc = P->rc;

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

  // This lane's query as operands, Q by way of the buffers of parity 1.
  TileAddr<D> A;
  A.init(lane);
  bf16x8 qf[KS], dof[KS];
  float nl, nd;
  {
    __bf16* const stage = (wave / 2 == 0 ? k_s1 : v_s1) + wave % 2 * 32 * D;
    const int64_t t0 = s.begin + wrow;
    bbm::copy_slab<D>(global(P->q.p) + h * P->q.head + t0 * P->q.row, wrows, P->q.row, stage, lane);
    const __amdgpu_buffer_rsrc_t do_r = buffer_of(global(P->d_o.p) + h * P->d_o.head + t0 * P->d_o.row, wrows > 0 ? ((wrows - 1) * P->d_o.row + D) * 2 : 0);
    const int64_t row_at = (int64_t)h * P->T + t0;
    const float nls = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(buffer_of(P->nls + row_at, wrows * 4), lq * 4, 0, 0));
    nd = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(buffer_of(P->ndelta + row_at, wrows * 4), lq * 4, 0, 0));
#pragma unroll
    for (int t = 0; t < KS; ++t) dof[t] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(do_r, (lq * P->d_o.row + 16 * t + 8 * hh) * 2, 0, 0));
#pragma unroll
    for (int i = 0; i < 2 * LPW; ++i) copy_piece(0, rows_at(0), k_s0, v_s0, i);
    __builtin_amdgcn_s_waitcnt(0);
#pragma unroll
    for (int t = 0; t < KS; ++t) qf[t] = bbm::slab_frag<D>(stage, t, lane);
    nl = nls * rc;
  }
  for (int i = 0; i < 2; ++i) {  // this wave's keys of a tile
    A.ra[i] += half * (32 / L::NBLK) * D;
    A.ta[i] += 2 * half * (D == 64 ? 2 * D : D);
  }
  f32x16 dq[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
    for (int e = 0; e < 16; ++e) dq[db][e] = 0.0f;

  // One tile: a chain of matrix instructions over its two halves of 32 keys, S0, dP0, S1, dP1, dQ0, dQ1, with the exponentials of a half behind its
  // dP, dS0 behind S1, dS1 behind dQ0.
  auto step = [&](auto pb, auto part, int jt) __attribute__((always_inline)) {
    constexpr int PB = decltype(pb)::value;
    constexpr bool PART = decltype(part)::value != 0;
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    __bf16* const k_cur = PB ? k_s1 : k_s0;
    __bf16* const v_cur = PB ? v_s1 : v_s0;
    __bf16* const k_oth = PB ? k_s0 : k_s1;
    __bf16* const v_oth = PB ? v_s0 : v_s1;
    const int rows1 = rows_at(jt + 1);
    const bool live = wrows > 0 && (!PART || jt * 64 + 32 * half < wrow + wrows);
    if (!live) {
#pragma unroll
      for (int i = 0; i < 2 * LPW; ++i) copy_piece(jt + 1, rows1, k_oth, v_oth, i);
      return;
    }
    constexpr int N1 = KS, N2 = 2 * KS, N3 = 3 * KS, N4 = 2 * KB * KS, N5 = N4 + 2 * DB, N6 = N4 + 2 * KB * DB;
    constexpr int PER = D == 128 ? 4 : 8;  // elements behind a matrix instruction
    static_assert(PER * (KS - 2) >= 16 && PER * (2 * DB - 2) >= 16, "all 16 must find room");
    f32x16 sc[KB], dp[KB];
    uint32_t dsf[KB][2][4];  // dS of [half][16-key step], pairs of bf16
    uint32_t seen[2] = {0, 0};
    if constexpr (PART) {
      const uint64_t bits = bbm::bits_up_to(wrow + lq - jt * 64 - 32 * half) >> (4 * hh);
      seen[0] = (uint32_t)bits, seen[1] = (uint32_t)(bits >> 32);
    }
    auto start = [&](f32x16& acc, float x) {
      asm volatile("" : "+v"(x));
      for (int e = 0; e < 16; ++e) acc[e] = x;
    };
    auto exps = [&](int kb, int slot) {
#pragma unroll
      for (int e = slot * PER; e < min(16, (slot + 1) * PER); ++e) {
        if constexpr (PART) sc[kb][e] = bbm::keep_if(seen[kb], e, sc[kb][e]);
        sc[kb][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[kb][e], rc, nl));
      }
    };
    auto ds = [&](int kb, int slot) {
#pragma unroll
      for (int e = slot * PER; e < min(16, (slot + 1) * PER); e += 2)
        dsf[kb][e / 8][e % 8 / 2] = pack(sc[kb][e] * dp[kb][e], sc[kb][e + 1] * dp[kb][e + 1]);
    };
    mfma_ring<N6, 3>(
        [&](auto i) {
          constexpr int x = decltype(i)::value;
          if constexpr (x < N4)
            return A.row_frag(x / KS % 2 ? v_cur : k_cur, x / N2, x % KS);
          else
            return A.tr_frag(k_cur, (x - N4) / DB, (x - N4) % DB);
        },
        [&](auto i, bf16x8 f) {
          constexpr int x = decltype(i)::value;
          if constexpr (x % N2 == 0 && x < N4) {
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[x / N2][e] = 0.0f;
          }
          if constexpr (x == N1) start(dp[0], nd);
          if constexpr (KB == 2 && x == N3) start(dp[KB - 1], nd);
          if constexpr (x < N4 && x / KS % 2 == 0) {
            sc[x / N2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, qf[x % KS], sc[x / N2], 0, 0, 0);
          } else if constexpr (x < N4) {
            dp[x / N2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, dof[x % KS], dp[x / N2], 0, 0, 0);
          } else {
            constexpr int m = x - N4, u = m / DB;
            dq[m % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, operand(dsf[u / 2][u % 2]), dq[m % DB], 0, 0, 0);
          }
        },
        [&](auto i) {
          constexpr int x = decltype(i)::value;
          if constexpr (x < 2 * LPW) copy_piece(jt + 1, rows1, k_oth, v_oth, x);
          // a product is complete two matrix instructions after its last one was issued
          if constexpr (KB == 2) {
            if constexpr (x >= N1 + 2 && x < N2) exps(0, x - N1 - 2);
            if constexpr (x >= N2 + 2 && x < N3) ds(0, x - N2 - 2);
            if constexpr (x >= N3 + 2 && x < N4) exps(1, x - N3 - 2);
            if constexpr (x >= N4 + 2 && x < N5) ds(1, x - N4 - 2);
          } else {
            if constexpr (x >= N1 + 2 && x < N2) exps(0, x - N1 - 2);
            if constexpr (x == N2 - 1) {
#pragma unroll
              for (int i = 0; i < 16 / PER; ++i) ds(0, i);
            }
          }
        });
  };
#pragma unroll 1
  for (int jt = 0; jt < n_full; jt += 2) {
    step(IntC<0>{}, IntC<0>{}, jt);
    step(IntC<1>{}, IntC<0>{}, jt + 1);
  }
  step(IntC<0>{}, IntC<1>{}, n_full);
  if (n_full + 1 < n_tiles) step(IntC<1>{}, IntC<1>{}, n_full + 1);
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();  // the result is staged in the tile buffers
  if constexpr (HALVES == 2) {
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    static_assert(32 * D * sizeof(float) <= L::ELEMS * sizeof(__bf16), "a wave's sums must fit in a tile buffer");
    f32x4* const sums = reinterpret_cast<f32x4*>(wave / 2 == 0 ? k_s1 : v_s1) + lane;
    if (half == 1) {
#pragma unroll
      for (int i = 0; i < 4 * DB; ++i) sums[i * 64] = f32x4{dq[i / 4][i % 4 * 4], dq[i / 4][i % 4 * 4 + 1], dq[i / 4][i % 4 * 4 + 2], dq[i / 4][i % 4 * 4 + 3]};
    }
    __syncthreads();
    if (half == 1) return;
#pragma unroll
    for (int i = 0; i < 4 * DB; ++i) {
      const f32x4 y = sums[i * 64];
      for (int e = 0; e < 4; ++e) dq[i / 4][i % 4 * 4 + e] += y[e];
    }
  }
  if (wrows == 0) return;
  __bf16* const stage = (wave / 2 == 0 ? k_s0 : v_s0) + wave % 2 * 32 * D;
  bbm::store_strided<D>(dq, P->scale, stage, global(P->dq.p) + h * P->dq.head + (int64_t)(s.begin + wrow) * P->dq.row, wrows, P->dq.row, lane);
}

// Registers are what this form lives by.  D = 128: 256, two pieces of the K operand in LDS, two waves a SIMD; D = 64: 168, three.
// t_s0, t_s1: [Q, dO] tiles, one variable per parity; st_s0, st_s1: [-lse / scale, -D] of the tile's queries; kl_s: the last pieces of the K operand, which find
// no room in the registers.
template <int D>
constexpr int kPiecesInLds = D == 128 ? 2 : 0;
template <int D>
__device__ __forceinline__ void dkv_of(Args P, int wg, __bf16* t_s0, __bf16* t_s1, float* st_s0, float* st_s1, bf16x8 (*kl_s)[4][64]) {
  using L = TL<D>;
  constexpr int NW = 4, KS = D / 16, DB = D / 32, REGS = DB * 16, KL = kPiecesInLds<D>;
  static_assert(2 * 32 * D <= L::ELEMS, "two 32 x D slabs must fit in a tile buffer");

  const int lane = threadIdx.x & 63;
  const int wave = (int)scalar(threadIdx.x >> 6);
  const int kh = wave & 1;   // key half of the tile
  const int qh = wave >> 1;  // query half of a tile; behind the last one, 0: this wave writes dV, 1: dK
  const float rc = P->rc;
  const int parts = P->parts;
  const bbm::Work work = bbm::work_of(wg, P->H / P->G * parts);
  const int hk = work.plane / parts, part = work.plane - hk * parts;
  if (work.number >= P->key_pieces) return;
  const bbm::Span s = bbm::find_piece(global(P->cu), P->R, P->T, 1, 64, work.number);  // (early keys first: most queries see them)
  const int n = s.end - s.begin, j = s.piece;
  if (n <= 0) return;
  const int head0 = part * P->G / parts, heads = (part + 1) * P->G / parts - head0;  // this part's heads of the group
  const int per_head = (n + 63) / 64 - j, n_steps = per_head * heads;               // tiles of queries from the diagonal on

  const int q_row = P->q.row, g_row = P->d_o.row, T = P->T;
  const __bf16* const qg = global(P->q.p) + ((int64_t)hk * P->G + head0) * P->q.head + (int64_t)s.begin * q_row;
  const __bf16* const gg = global(P->d_o.p) + ((int64_t)hk * P->G + head0) * P->d_o.head + (int64_t)s.begin * g_row;
  const int64_t st0 = ((int64_t)hk * P->G + head0) * T + s.begin;
  const int64_t q_head = P->q.head, g_head = P->d_o.head;
  constexpr int LPW = bbm::TileCopy<D, NW>::PIECES;
  // the queries from row `row` on of head g of the group; queries past the end come as zeros everywhere, and add exact zeros
  // (where a lane copies what is found anew for every tile: its registers are free for the rest of the step)
  bbm::TileCopy<D, NW> qc, gc;
  auto copy_from = [&]() __attribute__((always_inline)) {
    const int ln = lane_now();
    qc.init(wave, ln, q_row);
    gc.init(wave, ln, g_row);
  };
  auto copy_piece = [&](int g, int row, int rows, __bf16* td, int i) {
    if (i < LPW)
      qc.piece(qg + g * q_head + (int64_t)row * q_row, rows, q_row, td, i, wave);
    else
      gc.piece(gg + g * g_head + (int64_t)row * g_row, rows, g_row, td + L::ELEMS, i - LPW, wave);
  };
  auto copy_stats = [&](int g, int row, int rows, float* sts) __attribute__((always_inline)) {
    if (qh == 0) copy_async<4>((kh == 0 ? global(P->nls) : global(P->ndelta)) + st0 + (int64_t)g * T + row, rows * 4, lane_now() * 4, sts + kh * 64);
  };

  TileAddr<D> A;
  A.init(lane);
  bf16x8 kf[KS - KL], vf[KS];
  f32x16 dk[DB], dv[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
    for (int e = 0; e < 16; ++e) dk[db][e] = dv[db][e] = 0.0f;
  {
    const int rows0 = bbm::rows_of_tile(j * 64, n);
    copy_stats(0, j * 64, rows0, st_s0);
    copy_from();
#pragma unroll
    for (int i = 0; i < 2 * LPW; ++i) copy_piece(0, j * 64, rows0, t_s0, i);
    // K and V come through the buffers of parity 1
    bbm::TileCopy<D, NW> c;
    c.init(wave, lane, P->k.row);
#pragma unroll
    for (int i = 0; i < LPW; ++i) c.piece(global(P->k.p) + hk * P->k.head + (int64_t)(s.begin + j * 64) * P->k.row, rows0, P->k.row, t_s1, i, wave);
    c.init(wave, lane, P->v.row);
#pragma unroll
    for (int i = 0; i < LPW; ++i) c.piece(global(P->v.p) + hk * P->v.head + (int64_t)(s.begin + j * 64) * P->v.row, rows0, P->v.row, t_s1 + L::ELEMS, i, wave);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    // this lane's key: K and V as operands
#pragma unroll
    for (int t = 0; t < KS; ++t) {
      const bf16x8 kt = A.row_frag(t_s1, kh, t);
      vf[t] = A.row_frag(t_s1 + L::ELEMS, kh, t);
      if (t >= KS - KL)
        kl_s[t - (KS - KL)][wave][lane] = kt;  // (read back by this wave alone)
      else
        kf[t < KS - KL ? t : 0] = kt;
    }
  }
  for (int i = 0; i < 2; ++i) {  // from here on, this wave's half of the queries
    A.ra[i] += qh * (32 / L::NBLK) * D;
    A.ta[i] += 2 * qh * (D == 64 ? 2 * D : D);
  }

  // Head by head, the tile on the diagonal first.  i0: this tile's place among the head's; g1, i1: the next one's.
  int i0 = 0, g1 = 0, i1 = 0;
  auto step = [&](auto pb) __attribute__((always_inline)) {
    constexpr int PB = decltype(pb)::value;
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    __bf16* const q_cur = PB ? t_s1 : t_s0;
    __bf16* const g_cur = q_cur + L::ELEMS;
    __bf16* const t_oth = PB ? t_s0 : t_s1;
    const float* const nl_cur = (PB ? st_s1 : st_s0) + 32 * qh;
    const float* const nd_cur = nl_cur + 64;
    const bool diagonal = i0 == 0;
    if (++i1 == per_head) i1 = 0, ++g1;
    i0 = i1;
    const bool more = g1 < heads;
    const int gn = more ? g1 : 0, row1 = more ? (j + i1) * 64 : 0, rows1 = more ? bbm::rows_of_tile(row1, n) : 0;
    if (more) copy_stats(gn, row1, rows1, PB ? st_s0 : st_s1);
    copy_from();
    const bool live = scalar(!diagonal || kh <= qh) != 0;  // else all queries are in front of this wave's keys.  (As a scalar the compiler
    // leaves the test as it is; threaded through the steps it put 90 registers into scratch memory.)
    if (!live) {
#pragma unroll
      for (int i = 0; i < 2 * LPW; ++i) copy_piece(gn, row1, rows1, t_oth, i);
    }
    if (live) {
      f32x16 sc, dp;
      constexpr int N1 = KS, N2 = 2 * KS, N3 = N2 + 2 * DB, N4 = N3 + 2 * DB;
      constexpr int PER = D == 128 ? 4 : 8;
      static_assert(PER * (KS - 2) >= 16 && PER * (2 * DB - 2) >= 16, "all 16 must find room");
      uint32_t pf[2][4], dsf[2][4];  // pairs of bf16
      bf16x8 kl[2];
      {
        const float* const p = nl_cur + (lane_now() >> 5 << 2);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float4 y = *reinterpret_cast<const float4*>(p + 8 * g);
          sc[4 * g + 0] = y.x, sc[4 * g + 1] = y.y, sc[4 * g + 2] = y.z, sc[4 * g + 3] = y.w;
        }
        // A pair that is not seen starts at -infinity and stays there.  (Behind the product the test costs 1 to 7 % in the kernels under masks.)
        if (diagonal && kh == qh) {
          const int ln = lane_now(), late = (ln & 31) - (ln >> 5 << 2);  // element e's query is 8 * (e / 4) + e % 4 - late rows behind this lane's key
#pragma unroll
          for (int e = 0; e < 16; ++e) sc[e] = 8 * (e / 4) + e % 4 < late ? -INFINITY : sc[e];
        }
      }
      mfma_ring<N4, 3>(
          [&](auto i) {
            constexpr int x = decltype(i)::value;
            if constexpr (x < N2)
              return A.row_frag(x < N1 ? q_cur : g_cur, 0, x % KS);
            else
              return A.tr_frag(x < N3 ? g_cur : q_cur, (x - N2) % (2 * DB) / DB, x % DB);
          },
          [&](auto i, bf16x8 f) {
            constexpr int x = decltype(i)::value, db = x % DB, u = (x - N2) % (2 * DB) / DB;
            if constexpr (x < N1 - KL)
              sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, kf[x], sc, 0, 0, 0);
            else if constexpr (x < N1)
              sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, kl[x & 1], sc, 0, 0, 0);
            else if constexpr (x < N2)
              dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, vf[x - N1], dp, 0, 0, 0);
            else if constexpr (x < N3)
              dv[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, operand(pf[u]), dv[db], 0, 0, 0);
            else
              dk[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, operand(dsf[u]), dk[db], 0, 0, 0);
          },
          [&](auto i) {
            constexpr int x = decltype(i)::value;
            static_assert(2 * LPW == KS, "one copy behind every matrix instruction of S");
            if constexpr (x < N1) copy_piece(gn, row1, rows1, t_oth, x);
            if constexpr (x >= N1 - KL - 2 && x < N1 - 2) kl[x & 1] = kl_s[x - (N1 - KL - 2)][wave][lane_now()];
            if constexpr (x == N1 - 2) {
              const float* const nd = nd_cur + (lane_now() >> 5 << 2);
#pragma unroll
              for (int g = 0; g < 4; ++g) {
                const float4 y = *reinterpret_cast<const float4*>(nd + 8 * g);
                dp[4 * g + 0] = y.x, dp[4 * g + 1] = y.y, dp[4 * g + 2] = y.z, dp[4 * g + 3] = y.w;
              }
            }
            if constexpr (x >= N1 + 2 && x < N2) {
#pragma unroll
              for (int e = (x - N1 - 2) * PER; e < min(16, (x - N1 - 1) * PER); e += 2) {
                sc[e] = __builtin_amdgcn_exp2f(sc[e] * rc);
                sc[e + 1] = __builtin_amdgcn_exp2f(sc[e + 1] * rc);
                pf[e / 8][e % 8 / 2] = pack(sc[e], sc[e + 1]);
              }
            }
            if constexpr (x >= N2 + 2 && x < N3) {
#pragma unroll
              for (int e = (x - N2 - 2) * PER; e < min(16, (x - N2 - 1) * PER); e += 2) {
                dsf[e / 8][e % 8 / 2] = pack(sc[e] * dp[e], sc[e + 1] * dp[e + 1]);
              }
            }
          });
    }
  };
  for (int t = 0; t < n_steps; t += 2) {
    step(IntC<0>{});
    if (t + 1 < n_steps) step(IntC<1>{});
  }
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();

  // The two waves of a key half exchange: query half 0 hands over its dK and receives dV, query half 1 the other way round.
  float4* const mine = reinterpret_cast<float4*>(qh == 0 ? t_s0 : t_s1) + kh * (REGS / 4) * 64;
  const float4* const theirs = reinterpret_cast<const float4*>(qh == 0 ? t_s1 : t_s0) + kh * (REGS / 4) * 64;
  static_assert(2 * REGS * 64 * sizeof(float) <= 2 * L::ELEMS * sizeof(__bf16), "two waves' sums must fit in the tile buffers of a parity");
#pragma unroll
  for (int db = 0; db < DB; ++db)
    for (int g = 0; g < 4; ++g) {
      float4 x;
      x.x = qh ? dv[db][4 * g + 0] : dk[db][4 * g + 0];
      x.y = qh ? dv[db][4 * g + 1] : dk[db][4 * g + 1];
      x.z = qh ? dv[db][4 * g + 2] : dk[db][4 * g + 2];
      x.w = qh ? dv[db][4 * g + 3] : dk[db][4 * g + 3];
      mine[(db * 4 + g) * 64 + lane] = x;
    }
  __syncthreads();
#pragma unroll
  for (int db = 0; db < DB; ++db)
    for (int g = 0; g < 4; ++g) {
      const float4 x = theirs[(db * 4 + g) * 64 + lane];
      dk[db][4 * g + 0] = x.x + (qh ? dk[db][4 * g + 0] : dv[db][4 * g + 0]);
      dk[db][4 * g + 1] = x.y + (qh ? dk[db][4 * g + 1] : dv[db][4 * g + 1]);
      dk[db][4 * g + 2] = x.z + (qh ? dk[db][4 * g + 2] : dv[db][4 * g + 2]);
      dk[db][4 * g + 3] = x.w + (qh ? dk[db][4 * g + 3] : dv[db][4 * g + 3]);
    }
  __syncthreads();  // the results are staged in the same buffers
  const int row0 = j * 64 + kh * 32, rows = max(0, min(32, n - row0));
  if (parts > 1) {  // fp32 rows for the kernel that adds the parts up
    if ((lane & 31) < rows) {
      float* const to = global(P->partials) + (((int64_t)(part * 2 + qh) * (P->H / P->G) + hk) * T + s.begin + row0 + (lane & 31)) * D + 4 * (lane >> 5);
#pragma unroll
      for (int db = 0; db < DB; ++db)
        for (int g = 0; g < 4; ++g) *reinterpret_cast<float4*>(to + 32 * db + 8 * g) = make_float4(dk[db][4 * g], dk[db][4 * g + 1], dk[db][4 * g + 2], dk[db][4 * g + 3]);
    }
    return;
  }
  if (qh == 0)
    bbm::store_strided<D>(dk, 1.0f, t_s0 + L::ELEMS + kh * 32 * D, global(P->dv.p) + hk * P->dv.head + (int64_t)(s.begin + row0) * P->dv.row, rows, P->dv.row, lane);
  else
    bbm::store_strided<D>(dk, P->scale, t_s0 + kh * 32 * D, global(P->dk.p) + hk * P->dk.head + (int64_t)(s.begin + row0) * P->dk.row, rows, P->dk.row, lane);
}

// Both gradients side by side, dK and dV, whose steps are longer, first.  One behind the other (the first one forming the statistics) / side by side, forward and
// backward, us: 1 x 1024 tokens, 16 heads of 64, 42 / 36; 1 x 4096, 32 / 8 heads of 128, 669 / 605; 8 x 1024, 32 / 8 of 128, 321 / 308; but 300 x 100, 8 heads of 64, 103 / 109.
template <int D, int HALVES>
__global__ __launch_bounds__(256, D == 128 ? 2 : 3) void prompt_both_kernel(const PromptBwdParams) {
  Args P = bbm::kernel_args<PromptBwdParams>();
  __shared__ __attribute__((aligned(16))) __bf16 t_s0[2 * TL<D>::ELEMS];
  __shared__ __attribute__((aligned(16))) __bf16 t_s1[2 * TL<D>::ELEMS];
  __shared__ __attribute__((aligned(16))) float st_s0[2 * 64];
  __shared__ __attribute__((aligned(16))) float st_s1[2 * 64];
  __shared__ __attribute__((aligned(16))) bf16x8 kl_s[kPiecesInLds<D> ? kPiecesInLds<D> : 1][4][64];
  const int wg = blockIdx.x, keys = P->key_wgs;
  if (wg < keys)
    dkv_of<D>(P, wg, t_s0, t_s1, st_s0, st_s1, kl_s);
  else
    dq_of<D, HALVES>(P, wg - keys, t_s0, t_s1);
}

// -lse / scale and -D of all rows, a row of a head for D / 8 lanes.  (Of rows of nobody too, from whatever they hold: nobody reads those.)
template <int D>
__global__ __launch_bounds__(256) void prompt_stats_kernel(const PromptBwdParams P) {
  constexpr int RC = D / 8;
  const int64_t at = (int64_t)blockIdx.x * (256 / RC) + threadIdx.x / RC;
  const int t = (int)(at / P.H), h = (int)(at - (int64_t)t * P.H), chunk = threadIdx.x % RC;
  if (t >= P.T) return;  // (whole rows)
  const bf16x8 g = *reinterpret_cast<const bf16x8*>(P.d_o.p + h * P.d_o.head + (int64_t)t * P.d_o.row + chunk * 8);
  const bf16x8 o = *reinterpret_cast<const bf16x8*>(P.o.p + h * P.o.head + (int64_t)t * P.o.row + chunk * 8);
  const int64_t row_at = (int64_t)h * P.T + t;
  const float lse = P.lse[row_at];
  float x = 0.0f;
  for (int e = 0; e < 8; ++e) x += (float)g[e] * (float)o[e];
  x = bbm::row_sum<RC>(x);
  if (chunk == 0) {
    P.nls[row_at] = -lse / P.scale;
    P.ndelta[row_at] = -x;
  }
}

// Adds the parts of dK and dV up, in their order; eight elements of a row a thread.
template <int D>
__global__ __launch_bounds__(256) void prompt_sum_kernel(const PromptBwdParams P) {
  const int Hk = P.H / P.G, T = P.T;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int chunk = (int)(at % (D / 8)), t = (int)(at / (D / 8) % T), rest = (int)(at / (D / 8) / T), hk = rest % Hk, which = rest / Hk;
  if (which > 1 || t < P.cu[0] || t >= P.cu[P.R]) return;  // (rows of nobody are left as they are)
  const float* from = P.partials + (((int64_t)which * Hk + hk) * T + t) * D + chunk * 8;
  const int64_t stride = (int64_t)2 * Hk * T * D;
  float x[8] = {};
  for (int p = 0; p < P.parts; ++p, from += stride) {
    const float4 a = *reinterpret_cast<const float4*>(from), b = *reinterpret_cast<const float4*>(from + 4);
    x[0] += a.x, x[1] += a.y, x[2] += a.z, x[3] += a.w, x[4] += b.x, x[5] += b.y, x[6] += b.z, x[7] += b.w;
  }
  const Rows& to = which ? P.dk : P.dv;
  bf16x8 y;
  for (int e = 0; e < 8; ++e) y[e] = (__bf16)(which ? x[e] * P.scale : x[e]);
  *reinterpret_cast<bf16x8*>(to.p + hk * to.head + (int64_t)t * to.row + chunk * 8) = y;
}

// Parts of a group's heads whose dK and dV are formed side by side: one key head's walk over all heads of its group is as long as they are many, and a
// chip that is not full waits for it.  Worth the fp32 sums in memory where the walk is long.  Forward and backward, one / several parts, us: 1 x 1024
// tokens, 8 / 2 heads of 128, 90 / 53; 1 x 4096, 8 / 2 of 64, 237 / 126; 1 x 2048, 32 / 8 of 128, 221 / 198; 12 x 214 on average and 1000 at most, 12 / 4 of 128, 85 / 76;
// 6 x 125, 8 / 1 of 64, 30 / 21; but 8 x 248, 16 / 4 of 128, 52 / 60 (cut up by this rule all the same, the slower side there); 30 x 81, 8 / 2 of 64, 23 / 29 (not cut up).
constexpr int64_t kDkvWgs = 512, kLongWalk = 512;  // work-groups, two a CU; queries of all heads of a group
inline int64_t head_parts(int64_t T, int64_t R, int64_t H, int64_t Hk) {
  if (H / Hk * T < kLongWalk * R) return 1;
  return std::min(H / Hk, std::max<int64_t>(1, kDkvWgs / (bbm::ceil_div(T, 64) * Hk)));
}
inline size_t partial_bytes(int64_t T, int64_t R, int64_t H, int64_t Hk, int d) {
  const int64_t parts = head_parts(T, R, H, Hk);
  return parts > 1 ? (size_t)(2 * parts * Hk * T * d) * sizeof(float) : 0;
}
inline size_t stats_bytes(int64_t T, int64_t H) { return ((size_t)(T * H) * sizeof(float) + 255) / 256 * 256; }

}  // namespace

extern "C" __attribute__((visibility("default"))) size_t bbm_prompt_attn_bwd_workspace_bytes(int64_t T, int64_t R, int64_t H, int64_t Hk, int d) {
  if (T < 1 || R < 1 || R > bbm::kMaxTokens || H < 1 || Hk < 1 || H % Hk || T > bbm::kMaxTokens || H > 65535 || (d != 64 && d != 128)) return 0;
  return 2 * stats_bytes(T, H) + partial_bytes(T, R, H, Hk, d);
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
    if (int rc = check_rows(fn, a.name, a.x, T, a.heads, d, a.output)) return rc;
  if ((T > 0 && !lse) || !aligned(lse, 4)) return fail(BBM_EINVAL, "%s: lse must be a non-NULL 4-byte aligned pointer", fn);
  if (int rc = check_scale(fn, softmax_scale)) return rc;
  const size_t need = bbm_prompt_attn_bwd_workspace_bytes(T, R, H, Hk, d);
  if (need > 0 && (!workspace || workspace_bytes < need))
    return fail(BBM_EWORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need, workspace ? workspace_bytes : (size_t)0);
  if (!aligned(workspace, 16)) return fail(BBM_EINVAL, "%s: workspace must be 16-byte aligned", fn);
  if (T == 0) return BBM_OK;
  if (int rc = check_apart(fn, {dq->ptr, dk->ptr, dv->ptr, workspace}, {q->ptr, k->ptr, v->ptr, o->ptr, d_o->ptr, lse, cu})) return rc;
  PromptBwdParams P;
  Rows* const to[] = {&P.q, &P.k, &P.v, &P.o, &P.d_o, &P.dq, &P.dk, &P.dv};
  for (int i = 0; i < 8; ++i) *to[i] = rows_of(all[i].x, T, d);
  P.lse = lse, P.nls = static_cast<float*>(workspace), P.ndelta = reinterpret_cast<float*>(static_cast<char*>(workspace) + stats_bytes(T, H)), P.cu = cu;
  P.T = (int32_t)T, P.R = (int32_t)R, P.G = (int32_t)(H / Hk), P.H = (int32_t)H, P.rc = softmax_scale * kLog2e, P.scale = softmax_scale;
  P.parts = (int32_t)head_parts(T, R, H, Hk);
  P.partials = reinterpret_cast<float*>(static_cast<char*>(workspace) + 2 * stats_bytes(T, H));
  const bool halves = split_keys(T, R, H);
  const int64_t row_pieces = count_pieces(T, R, 1, halves ? 64 : 128), key_pieces = count_pieces(T, R, 1, 64);
  const int64_t rows = work_groups(H, row_pieces), keys = work_groups(Hk * P.parts, key_pieces), sums = P.parts > 1 ? ceil_div(2 * Hk * T * (d / 8), 256) : 0, stats = ceil_div(T * H * (d / 8), 256);
  if (rows + keys >= kMaxWgs || stats >= kMaxWgs || sums >= kMaxWgs) return fail(BBM_EUNSUPPORTED, "%s: problem too large (T=%lld, H=%lld)", fn, (long long)T, (long long)H);
  P.row_pieces = (int32_t)row_pieces, P.key_pieces = (int32_t)key_pieces, P.key_wgs = (int32_t)keys;
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto go = [&](auto size) {
    constexpr int D = decltype(size)::value;
    prompt_stats_kernel<D><<<(unsigned)stats, 256, 0, s>>>(P);
    if (halves) prompt_both_kernel<D, 2><<<(unsigned)(rows + keys), 256, 0, s>>>(P);
    else prompt_both_kernel<D, 1><<<(unsigned)(rows + keys), 256, 0, s>>>(P);
    if (P.parts > 1) prompt_sum_kernel<D><<<(unsigned)sums, 256, 0, s>>>(P);
  };
  if (d == 64) go(IntC<64>{});
  else go(IntC<128>{});
  return launch_status(fn);
}
