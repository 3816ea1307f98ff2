// Attention of new tokens over the 4-bit cache (include/bbm_tokens.h).
//
// Bound by the cache's bytes when few queries read it: 17/32 byte an element.  A piece is 16 * QT query columns of a request and a key head (column
// c: query token c / G, head c % G of the group), so that the heads of a group and several new tokens share what is read.  A work-group takes a
// piece and a part of the keys, its four waves blocks of 32 keys in turn; there is no barrier and no LDS in the loop:
//   S^T = K Q^T       (16 keys x 16 columns x 32 elements an instruction): lane (n, q) = (l % 16, l / 16) of an A operand is key n, and what it
//                     loads, D / 4 elements from q * D / 4 on, is the operand of all D / 32 steps once the codes are converted (with the group's scale, exactly);
//   O^T += V^T P^T    over 32 keys: lane (n, q) loads elements n * D / 16 .. of the keys 4 q .. 4 q + 3 of both blocks of 16, converts pairs of elements,
//                     and pairs the keys by byte permutes; row n of instruction j is element n * D / 16 + j.  The lane's scores are of the same eight keys
//                     (the layout of the first product's result), so P goes from one product to the other in place.
// The waves' results meet in LDS, those of parts in the workspace, where a second kernel joins them in the order of parts.
#include "bbm_kv4.h"
#include "bbm_tile.h"

#include <algorithm>

namespace {

using bbm::bf16x2, bbm::bf16x8, bbm::Kv4, bbm::scalar;
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLazy = 8.0f;
constexpr int NW = 4;
constexpr int kStep = 32 * NW;  // keys of a work-group's step

struct Kv4AttnParams {
  Kv4 c;
  const __bf16* q;
  __bf16* o;
  float* lse;
  int64_t q_row, q_head, o_row, o_head, table_stride;
  const int32_t *cu, *lens, *table;
  const uint64_t* mask;
  float* partials;  // [piece][key head][part]: 16 * QT rows of D sums, then of a (maximum, sum) pair
  int32_t T, R, G, max_pages, mask_words, pieces, parts, part_keys;
  float rc;  // softmax_scale * log2(e)
};

// What a work-group and the one that joins its parts both need to know.
struct Piece {
  bbm::Span s;
  int cols, col0;    // columns of the request; the piece's first
  int len, prefix;   // keys that can be seen at all; keys in front of the new tokens
  int parts, keys;   // parts of this request, keys of one
};
__device__ __forceinline__ Piece piece_of(const Kv4AttnParams& P, int number, int width) {
  Piece x;
  x.s = bbm::find_piece(P.cu, P.R, P.T, P.G, width, number);
  const int n = x.s.end - x.s.begin, len = (int)scalar(P.lens[x.s.r]);
  x.cols = n * P.G;
  x.col0 = x.s.piece * width;
  x.prefix = len - n;
  x.len = (int)max((int64_t)0, min((int64_t)len, (int64_t)P.max_pages << P.c.page_shift));
  x.keys = max(P.part_keys, (int)(((int64_t)x.len + P.parts - 1) / P.parts + kStep - 1) / kStep * kStep);
  x.parts = max(1, (x.len + x.keys - 1) / x.keys);
  return x;
}

template <int X>
__device__ __forceinline__ float other_max(float x) {  // over lanes l and l ^ X
  auto r = X == 32 ? __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false)
                   : __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <int X>
__device__ __forceinline__ float other_sum(float x) {
  auto r = X == 32 ? __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false)
                   : __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Writes D / 16 values of column `col`, from element e0 on.
template <int D>
__device__ __forceinline__ void put_column(const Kv4AttnParams& P, const Piece& x, int hk, int col, int e0, const float (&v)[D / 16], float m, float l) {
  const int i = col / P.G, h = hk * P.G + (col - i * P.G), t = x.s.begin + i;
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  typedef __bf16 out_t __attribute__((ext_vector_type(D / 16)));
  out_t y;
#pragma unroll
  for (int e = 0; e < D / 16; ++e) y[e] = (__bf16)(v[e] * inv);
  *reinterpret_cast<out_t*>(P.o + (int64_t)t * P.o_row + h * P.o_head + e0) = y;
  if (P.lse && e0 == 0) P.lse[(int64_t)h * P.T + t] = l > 0.0f ? (m + __log2f(l)) * kLn2 : -INFINITY;
}

template <int D, int QT>
__global__ __launch_bounds__(64 * NW, QT == 4 ? 1 : QT == 2 ? 2 : 3) void kv4_attn_kernel(const Kv4AttnParams P) {
  constexpr int KD = D / 4;        // elements of K a lane loads of its key
  constexpr int KS = D / 32;       // steps of the first product
  constexpr int VD = D / 16;       // elements of V a lane loads of a key, instructions of the second product
  constexpr int LD = D + 4;        // row of the results in LDS
  __shared__ __attribute__((aligned(16))) float o_s[NW][16][LD];
  __shared__ float m_s[NW][16], l_s[NW][16];

  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, kq = lane >> 4;
  const int wave = (int)scalar(tid >> 6);
  const int at = bbm::logical_wg(blockIdx.x, gridDim.x);
  const int number = at % P.pieces, rest = at / P.pieces, part = rest % P.parts, hk = rest / P.parts;
  const Piece x = piece_of(P, number, 16 * QT);
  if (x.s.end <= x.s.begin || part >= x.parts) return;
  const int first = part * x.keys, last = min(x.len, first + x.keys);

  // this lane's columns: Q as operands, how far each sees
  bf16x8 qf[QT][KS];
  int sees[QT];               // of the new tokens, causal: keys 0 .. sees
  const uint64_t* words[QT];  // with a mask: the row's
  float m_run[QT], l_run[QT], nm[QT];
  f32x4 acc[QT][VD];
#pragma unroll
  for (int u = 0; u < QT; ++u) {
    const int col = min(x.col0 + 16 * u + n, x.cols - 1);  // (columns behind the last repeat it; they are not written)
    const int i = col / P.G, t = x.s.begin + i;
    const __bf16* const row = P.q + (int64_t)t * P.q_row + (hk * P.G + (col - i * P.G)) * P.q_head + kq * KD;
#pragma unroll
    for (int j = 0; j < KS; ++j) qf[u][j] = *reinterpret_cast<const bf16x8*>(row + 8 * j);
    sees[u] = x.prefix + i;
    words[u] = P.mask + (int64_t)t * P.mask_words;
    m_run[u] = -INFINITY, l_run[u] = 0.0f, nm[u] = 0.0f;
#pragma unroll
    for (int j = 0; j < VD; ++j) acc[u][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  const int sees_all = P.mask ? x.prefix - 1 : x.prefix + x.col0 / P.G;  // the last key that every column of the piece sees

  // 16 keys as they lie in the cache
  struct Block {
    uint32_t k[KD / 8], ks, v[4], vs;
    int valid;  // keys that are there: 16, or fewer at the end, or none (a page outside the cache)
  };
  const int32_t* const table = P.table + x.s.r * P.table_stride;
  auto page_at = [&](int j) { return (int)scalar(j < last ? table[j >> P.c.page_shift] : -1); };
  auto load = [&](Block& b, int j, int page) __attribute__((always_inline)) {
    const bool there = page >= 0 && page < P.c.pages;
    b.valid = there ? min(16, last - j) : 0;
    const int64_t head = (int64_t)(there ? page : 0) * P.c.Hk + hk;
    const int in_page = j & (P.c.page - 1);
    const int64_t key = head * P.c.page + in_page;
    const uint8_t* const kp = P.c.k + key * (D / 2);
    const uint8_t* const vp = P.c.v + key * (D / 2);
    if constexpr (D == 128) {
      const uint4 w = *reinterpret_cast<const uint4*>(kp + (uint32_t)(n * (D / 2) + kq * 16));
      b.k[0] = w.x, b.k[1] = w.y, b.k[2] = w.z, b.k[3] = w.w;
    } else {
      const uint2 w = *reinterpret_cast<const uint2*>(kp + (uint32_t)(n * (D / 2) + kq * 8));
      b.k[0] = w.x, b.k[1] = w.y;
    }
    b.ks = (P.c.k_scale + key * (D / 32))[(uint32_t)(n * (D / 32) + kq * KD / 32)];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint8_t* const p = vp + (uint32_t)((4 * kq + r) * (D / 2) + n * (VD / 2));
      b.v[r] = D == 128 ? *reinterpret_cast<const uint32_t*>(p) : *reinterpret_cast<const uint16_t*>(p);
    }
    b.vs = *reinterpret_cast<const uint32_t*>(P.c.v_scale + head * (D / 32) * P.c.page + in_page + (uint32_t)(n * VD / 32 * P.c.page + 4 * kq));
  };

  auto compute = [&](Block& a, Block& b, int j0) __attribute__((always_inline)) {
    const bool full = a.valid == 16 && b.valid == 16 && j0 + 31 <= sees_all;
    f32x4 sa[QT], sb[QT];
#pragma unroll
    for (int u = 0; u < QT; ++u) sa[u] = sb[u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const float ka = bbm::scale_of(a.ks), kb = bbm::scale_of(b.ks);
#pragma unroll
    for (int j = 0; j < KS; ++j) {
      const bf16x8 fa = bbm::values_of(a.k[j], ka), fb = bbm::values_of(b.k[j], kb);
#pragma unroll
      for (int u = 0; u < QT; ++u) {
        sa[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa, qf[u][j], sa[u], 0, 0, 0);
        sb[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb, qf[u][j], sb[u], 0, 0, 0);
      }
    }
    if (!full) {
      // keys that are not there get scores of -infinity, and scales of 0, since a NaN would survive a probability of 0
      auto there = [&](Block& z, f32x4 (&sz)[QT], int j) {
        const int have = max(0, min(4, z.valid - 4 * kq));
        z.vs &= have == 4 ? ~0u : (1u << (8 * have)) - 1u;
#pragma unroll
        for (int u = 0; u < QT; ++u) {
          uint32_t bits;  // which of the lane's four keys its column sees
          const int k0 = j + 4 * kq;
          if (!P.mask) {
            bits = k0 + 3 <= sees[u] ? 15u : k0 > sees[u] ? 0u : (2u << (sees[u] - k0)) - 1u;
          } else {
            const int w0 = k0 - x.prefix;  // among the new tokens
            auto word = [&](int i) { return i < P.mask_words ? words[u][i] : 0ull; };
            if (w0 >= 0) {
              const int sh = w0 & 63;
              bits = (uint32_t)(word(w0 >> 6) >> sh);
              if (sh > 60) bits |= (uint32_t)(word((w0 >> 6) + 1) << (64 - sh));
            } else {
              bits = w0 <= -4 ? 15u : ((1u << -w0) - 1u) | (uint32_t)(word(0) << -w0);
            }
          }
          bits &= (1u << have) - 1u;
#pragma unroll
          for (int r = 0; r < 4; ++r) sz[u][r] = bits >> r & 1 ? sz[u][r] : -INFINITY;
        }
      };
      there(a, sa, j0);
      there(b, sb, j0 + 16);
    }
    bf16x8 pf[QT];
#pragma unroll
    for (int u = 0; u < QT; ++u) {
      float mx = fmaxf(fmaxf(fmaxf(sa[u][0], sa[u][1]), fmaxf(sa[u][2], sa[u][3])), fmaxf(fmaxf(sb[u][0], sb[u][1]), fmaxf(sb[u][2], sb[u][3])));
      mx = other_max<16>(other_max<32>(mx)) * P.rc;
      if (__any(mx > m_run[u] + kLazy ? 1 : 0)) {
        const float m_new = fmaxf(m_run[u], mx), m_fin = m_new == -INFINITY ? 0.0f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m_run[u] - m_fin);
        l_run[u] *= alpha;
        m_run[u] = m_new;
        nm[u] = -m_fin;
#pragma unroll
        for (int j = 0; j < VD; ++j) acc[u][j] *= alpha;
      }
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(r < 4 ? sa[u][r & 3] : sb[u][r & 3], P.rc, nm[u]));
        l_run[u] += p;
        pf[u][r] = (__bf16)p;
      }
    }
    uint32_t va[4][VD / 2], vb[4][VD / 2];  // pairs of elements of a key
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float fa = bbm::scale_of(a.vs >> (8 * r) & 255), fb = bbm::scale_of(b.vs >> (8 * r) & 255);
      va[r][0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(a.v[r], fa, 0));
      va[r][1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(a.v[r], fa, 1));
      vb[r][0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(b.v[r], fb, 0));
      vb[r][1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(b.v[r], fb, 1));
      if constexpr (D == 128) {
        va[r][2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(a.v[r], fa, 2));
        va[r][3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(a.v[r], fa, 3));
        vb[r][2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(b.v[r], fb, 2));
        vb[r][3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(b.v[r], fb, 3));
      }
    }
#pragma unroll
    for (int j = 0; j < VD; ++j) {
      const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;  // the pair's second or first element of two keys
      const uint32_t w[4] = {__builtin_amdgcn_perm(va[1][j / 2], va[0][j / 2], sel), __builtin_amdgcn_perm(va[3][j / 2], va[2][j / 2], sel),
                             __builtin_amdgcn_perm(vb[1][j / 2], vb[0][j / 2], sel), __builtin_amdgcn_perm(vb[3][j / 2], vb[2][j / 2], sel)};
      const bf16x8 f = bbm::operand(w);
#pragma unroll
      for (int u = 0; u < QT; ++u) acc[u][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, pf[u], acc[u][j], 0, 0, 0);
    }
  };

  int j0 = first + 32 * wave;
  if (j0 < last) {
    // the next 32 keys are asked for before these are used, their pages a step before that
    Block a[2], b[2];
    int pa = page_at(j0), pb = page_at(j0 + 16);
    load(a[0], j0, pa);
    load(b[0], j0 + 16, pb);
    pa = page_at(j0 + kStep), pb = page_at(j0 + kStep + 16);
#pragma unroll 1
    for (;;) {
      load(a[1], j0 + kStep, pa);
      load(b[1], j0 + kStep + 16, pb);
      pa = page_at(j0 + 2 * kStep), pb = page_at(j0 + 2 * kStep + 16);
      compute(a[0], b[0], j0);
      j0 += kStep;
      if (j0 >= last) break;
      load(a[0], j0 + kStep, pa);
      load(b[0], j0 + kStep + 16, pb);
      pa = page_at(j0 + 2 * kStep), pb = page_at(j0 + 2 * kStep + 16);
      compute(a[1], b[1], j0);
      j0 += kStep;
      if (j0 >= last) break;
    }
  }

  // The waves' results meet: columns on threads, 16 threads a column.
  const int c = tid >> 4, e0 = (tid & 15) * VD;
  float* const rec = x.parts > 1 ? P.partials + (((int64_t)number * P.c.Hk + hk) * P.parts + part) * (16 * QT * (D + 2)) : nullptr;
#pragma unroll
  for (int u = 0; u < QT; ++u) {
    if (u > 0) __syncthreads();
    const float l = other_sum<16>(other_sum<32>(l_run[u]));
    if (kq == 0) m_s[wave][n] = m_run[u], l_s[wave][n] = l;
    // lane (n, kq): rows 4 kq + r of instruction j, element (4 kq + r) * VD + j
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < VD; j += 4) *reinterpret_cast<f32x4*>(&o_s[wave][n][(4 * kq + r) * VD + j]) = f32x4{acc[u][j][r], acc[u][j + 1][r], acc[u][j + 2][r], acc[u][j + 3][r]};
    __syncthreads();
    const int col = x.col0 + 16 * u + c;
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) m = fmaxf(m, m_s[w][c]);
    const float m_fin = m == -INFINITY ? 0.0f : m;
    float sum = 0.0f, v[VD] = {};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = __builtin_amdgcn_exp2f(m_s[w][c] - m_fin);
      sum += f * l_s[w][c];
#pragma unroll
      for (int e = 0; e < VD; ++e) v[e] += f * o_s[w][c][e0 + e];
    }
    if (col >= x.cols) continue;
    if (!rec) {
      put_column<D>(P, x, hk, col, e0, v, m, sum);
    } else {
#pragma unroll
      for (int e = 0; e < VD; e += 4) *reinterpret_cast<f32x4*>(rec + (16 * u + c) * D + e0 + e) = f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]};
      if (e0 == 0) *reinterpret_cast<float2*>(rec + 16 * QT * D + 2 * (16 * u + c)) = make_float2(m, sum);
    }
  }
}

// Joins the parts of a piece's 16 columns, in their order.
template <int D, int QT>
__global__ __launch_bounds__(256) void kv4_join_kernel(const Kv4AttnParams P) {
  constexpr int VD = D / 16;
  const int number = blockIdx.x, hk = blockIdx.y, u = blockIdx.z, c = 16 * u + (threadIdx.x >> 4), e0 = (threadIdx.x & 15) * VD;
  const Piece x = piece_of(P, number, 16 * QT);
  if (x.s.end <= x.s.begin || x.parts == 1 || x.col0 + c >= x.cols) return;
  const int64_t stride = 16 * QT * (D + 2);
  const float* const rec = P.partials + ((int64_t)number * P.c.Hk + hk) * P.parts * stride;
  float m = -INFINITY, l = 0.0f, v[VD] = {};
  for (int p = 0; p < x.parts; ++p) m = fmaxf(m, rec[p * stride + 16 * QT * D + 2 * c]);
  const float m_fin = m == -INFINITY ? 0.0f : m;
#pragma unroll 4
  for (int p = 0; p < x.parts; ++p) {
    const float2 ml = *reinterpret_cast<const float2*>(rec + p * stride + 16 * QT * D + 2 * c);
    const float f = __builtin_amdgcn_exp2f(ml.x - m_fin);
    l += f * ml.y;
#pragma unroll
    for (int e = 0; e < VD; e += 4) {
      const f32x4 y = *reinterpret_cast<const f32x4*>(rec + p * stride + c * D + e0 + e);
      for (int i = 0; i < 4; ++i) v[e + i] += f * y[i];
    }
  }
  put_column<D>(P, x, hk, x.col0 + c, e0, v, m, l);
}

// How a call is cut: 16 * QT columns a piece, at most `parts` parts of the keys, of at least part_keys each.
struct Plan {
  int qt;
  int64_t pieces, parts, part_keys;
};
constexpr int64_t kFill = 2048;     // work-groups that keep the chip busy to the end of a call
constexpr int64_t kPartKeys = 256;  // fewer keys than this are not worth a part of their own
inline Plan plan_of(int64_t T, int64_t R, int64_t G, int64_t Hk, int64_t max_len) {
  Plan p;
  const int64_t cols = bbm::ceil_div(T * G, R);
  p.qt = cols <= 16 ? 1 : cols <= 32 ? 2 : 4;
  p.pieces = bbm::count_pieces(T, R, G, 16 * p.qt);
  const int64_t busy = std::max<int64_t>(1, std::min(p.pieces, bbm::ceil_div(T * G, 16 * p.qt) + R / 2)) * Hk;
  p.parts = std::max<int64_t>(1, std::min(bbm::ceil_div(kFill, busy), max_len / kPartKeys));
  p.part_keys = bbm::ceil_div(bbm::ceil_div(max_len, p.parts), kStep) * kStep;
  p.parts = bbm::ceil_div(max_len, p.part_keys);
  return p;
}
inline bool sizes_ok(int64_t T, int64_t R, int64_t H, int64_t Hk, int64_t max_len) {
  return T >= 1 && R >= 1 && H >= 1 && Hk >= 1 && H % Hk == 0 && max_len >= 1 && T <= bbm::kMaxTokens && R <= bbm::kMaxTokens && H <= 65535;
}

template <int D, int QT>
void launch(const Kv4AttnParams& P, hipStream_t s) {
  kv4_attn_kernel<D, QT><<<(unsigned)((int64_t)P.pieces * P.c.Hk * P.parts), 64 * NW, 0, s>>>(P);
  if (P.parts > 1) kv4_join_kernel<D, QT><<<dim3((unsigned)P.pieces, (unsigned)P.c.Hk, QT), 256, 0, s>>>(P);
}

}  // namespace

extern "C" __attribute__((visibility("default"))) size_t bbm_kv4_attn_workspace_bytes(int64_t T, int64_t R, int64_t H, int64_t Hk, int d, int64_t max_len) {
  if (!sizes_ok(T, R, H, Hk, max_len) || (d != 64 && d != 128)) return 0;
  const Plan p = plan_of(T, R, H / Hk, Hk, std::min<int64_t>(max_len, 0x7fffffff));
  return p.parts == 1 ? 0 : (size_t)(p.pieces * Hk * p.parts * 16 * p.qt * (d + 2)) * sizeof(float);
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
  P.T = (int32_t)T, P.R = (int32_t)R, P.G = (int32_t)(H / cache->Hk), P.max_pages = (int32_t)max_pages, P.mask_words = (int32_t)mask_words;
  P.rc = softmax_scale * kLog2e;
  const Plan p = plan_of(T, R, P.G, cache->Hk, std::min<int64_t>(max_len, 0x7fffffff));
  if (p.pieces * cache->Hk * p.parts >= 1ll << 31) return fail(BBM_EUNSUPPORTED, "%s: problem too large (T=%lld, R=%lld, H=%lld)", fn, (long long)T, (long long)R, (long long)H);
  P.partials = static_cast<float*>(workspace);
  P.pieces = (int32_t)p.pieces, P.parts = (int32_t)p.parts, P.part_keys = (int32_t)p.part_keys;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (cache->d == 64)
    p.qt == 1 ? launch<64, 1>(P, s) : p.qt == 2 ? launch<64, 2>(P, s) : launch<64, 4>(P, s);
  else
    p.qt == 1 ? launch<128, 1>(P, s) : p.qt == 2 ? launch<128, 2>(P, s) : launch<128, 4>(P, s);
  return launch_status(fn);
}
