// Attention of new tokens over the 4-bit cache (include/bbm_tokens.h).
//
// The queries of a request and a key head are columns: column c is query token c / G, head c % G of the group, so that the heads of a group and
// several new tokens share what is read.  A work-group takes a piece of the columns and a part of the keys; parts meet in the workspace, where a
// second kernel joins them.  With few columns (the narrow kernel, 16 a piece) the cache's bytes are the bound, 17/32 byte an element; with many (the
// wide kernel, 128 a piece) converting the codes and the products are.
// Narrow: the four waves take blocks of 32 keys in turn; there is no barrier and no LDS in the loop:
//   S^T = K Q^T       (16 keys x 16 columns x 32 elements an instruction): lane (n, q) = (l % 16, l / 16) of an A operand is key n, and what it
//                     loads, D / 4 elements from q * D / 4 on, is the operand of all D / 32 steps once the codes are converted (with the group's scale, exactly);
//   O^T += V^T P^T    over 32 keys: lane (n, q) loads elements n * D / 16 .. of the keys 4 q .. 4 q + 3 of both blocks of 16, converts pairs of elements,
//                     and pairs the keys by byte permutes; row n of instruction j is element n * D / 16 + j.  The lane's scores are of the same eight keys
//                     (the layout of the first product's result), so P goes from one product to the other in place.
// Sums, maxima and O are fp32 until O's one rounding.  P is rounded to bf16 for its product, which the matrix instruction asks for: that puts O off by as much again as its own rounding does, no more.
// Measured: one token each of 64 requests of 9.8 to 16 thousand keys, 32 / 8 heads of 128 (861 MB), narrow, 162 - 176 us, 4.9 - 5.3 TB/s (a large copy reaches
// 4.8), and 5.2 for the join; trees of 256 nodes of 8 requests, 32 heads, over 805 to 1280 keys, wide, 52 us, 0.65 PFLOP/s counted as the products of all pairs.
// Behind shared prefixes (include/bbm_cache.h) a group's requests together are columns over the keys that they share, and each for itself over the rest; the parts of both meet in the join.
// 67 requests of one token behind 8192 common keys, 500 to 1000 of their own, 32 / 8 heads of 128: 32 us and 6 for the join; 256 requests behind 32768: 170 to 190 in all, of which the join is 16.
#include "bbm_cache.h"
#include "bbm_kv4.h"
#include "bbm_softmax.h"
#include "bbm_tile.h"

#include <algorithm>

namespace {

using bbm::bf16x8, bbm::f32x16, bbm::Kv4, bbm::scalar;
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
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
  float* partials;  // [piece][key head][part]: `width` rows of D sums, then as many (maximum, sum) pairs
  int32_t T, R, G, max_pages, mask_words, width, pieces, parts, part_keys;
  float rc;    // softmax_scale * log2(e)
  float lazy;  // kLazy as a difference of scores
  // Of calls with shared prefixes (SHARED of what follows); partials then are [part of a group, then part of a request][key head][column of all T * G],
  // D sums each, and behind all of them the (maximum, sum) pairs in the same order.
  const int32_t *group_cu, *shared_lens;
  int32_t S, group_pieces, group_parts, group_part_keys;
  int32_t group_wgs, own_wgs;  // work-groups of this launch for pieces of groups (they come first, up to a multiple of 8) and of requests
};

// Which piece, part and key head a work-group has; `group`: of a group's shared keys.
struct Item {
  int number, part, hk;
  bool group, none;
};
template <bool SHARED>
__device__ __forceinline__ Item item_of(const Kv4AttnParams& P) {
  const int ahead = SHARED ? (P.group_wgs + 7) & ~7 : 0;  // (a multiple of 8, so that both kinds spread over the XCDs alike)
  const bool group = SHARED && (int)blockIdx.x < ahead;
  const int wg = (int)blockIdx.x - (group ? 0 : ahead), total = !SHARED ? (int)gridDim.x : group ? P.group_wgs : P.own_wgs;
  const int pieces = group ? P.group_pieces : P.pieces, parts = group ? P.group_parts : P.parts;
  Item x;
  x.none = wg >= total;
  const int at = x.none ? 0 : bbm::logical_wg(wg, total), rest = at / pieces;
  x.number = at % pieces, x.part = rest % parts, x.hk = rest / parts, x.group = group;
  return x;
}

// What a work-group and the one that joins its parts both need to know.
struct Piece {
  bbm::Span s;
  int cols, col0;    // columns of the request; the piece's first
  int len, prefix;   // keys that can be seen at all; keys in front of the new tokens (causal: of the first one that has a row here)
  int from;          // the first key that is this piece's: those in front of it are its group's
  int parts, keys;   // parts of this request, keys of one
  int group_parts;   // parts of the keys that its group shares
};
template <bool SHARED>
__device__ __forceinline__ void cut_keys(const Kv4AttnParams& P, Piece& x, int parts, int part_keys) {
  const int n = x.len - (SHARED ? x.from : 0);
  x.keys = max(part_keys, (int)(((int64_t)n + parts - 1) / parts + kStep - 1) / kStep * kStep);
  x.parts = n > 0 ? (n - 1) / x.keys + 1 : 1;
}
// The keys that group g shares, in whole blocks of 16: what is left over is each request's own.
__device__ __forceinline__ int shared_keys(const Kv4AttnParams& P, int keys) {
  return (int)max((int64_t)0, min((int64_t)keys, (int64_t)P.max_pages << P.c.page_shift)) & ~15;
}
__device__ __forceinline__ int request_at(const Kv4AttnParams& P, int g) { return min(max(P.group_cu[g], 0), P.R); }
__device__ __forceinline__ Piece group_piece_of(const Kv4AttnParams& P, int number, int width) {
  Piece x;
  x.s = bbm::find_piece_of([&](int g) __attribute__((always_inline)) { return P.cu[request_at(P, g)]; }, P.S, P.T, P.G, width, number);
  x.len = x.s.end > x.s.begin ? shared_keys(P, (int)scalar(P.shared_lens[x.s.r])) : 0;
  x.s.r = min((int)scalar(request_at(P, x.s.r)), P.R - 1);  // (the first request's row of the table)
  x.cols = (x.s.end - x.s.begin) * P.G;
  x.col0 = x.s.piece * width;
  x.prefix = x.len;
  x.from = 0;
  x.group_parts = 0;
  cut_keys<true>(P, x, P.group_parts, P.group_part_keys);
  if (x.len == 0) x.s.end = x.s.begin;  // nothing to do
  return x;
}
template <bool SHARED>
__device__ __forceinline__ Piece piece_of(const Kv4AttnParams& P, int number, int width) {
  Piece x;
  x.s = bbm::find_piece(P.cu, P.R, P.T, P.G, width, number);
  const int n = x.s.end - x.s.begin, len = (int)scalar(P.lens[x.s.r]);
  const int c0 = (int)scalar(P.cu[x.s.r]), c1 = (int)scalar(P.cu[x.s.r + 1]);  // (rows outside 0 .. T are not here, but their tokens are in the cache)
  x.cols = n * P.G;
  x.col0 = x.s.piece * width;
  x.prefix = (int)((uint32_t)len - (uint32_t)max(0, c1 - c0) + (P.mask ? 0u : (uint32_t)x.s.begin - (uint32_t)c0));
  x.len = (int)max((int64_t)0, min((int64_t)len, (int64_t)P.max_pages << P.c.page_shift));
  x.from = 0;
  x.group_parts = 0;
  if constexpr (SHARED) {
    const int shared = shared_keys(P, bbm::group_of(P.group_cu, P.shared_lens, P.S, x.s.r).keys);
    if (shared > 0) {
      Piece all;
      all.len = shared, all.from = 0;
      cut_keys<true>(P, all, P.group_parts, P.group_part_keys);
      x.group_parts = all.parts;
      x.from = min(shared, x.len);
    }
  }
  cut_keys<SHARED>(P, x, P.parts, P.part_keys);
  return x;
}

using bbm::Table;
__device__ __forceinline__ Table table_of(const Kv4AttnParams& P, const Piece& x) { return (Table)(uintptr_t)(P.table + x.s.r * P.table_stride); }

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

// Where a part's sums of column c of its piece lie, and their (maximum, sum).
struct Record {
  float *sums, *pair;
};
template <int D, bool SHARED>
__device__ __forceinline__ Record record_of(const Kv4AttnParams& P, const Piece& x, int number, int hk, int part, int c) {
  if constexpr (SHARED) {  // (part: a group's parts, then the request's)
    const int64_t all = (int64_t)P.T * P.G, at = ((int64_t)part * P.c.Hk + hk) * all + (int64_t)x.s.begin * P.G + x.col0 + c;
    return {P.partials + at * D, P.partials + (P.group_parts + P.parts) * P.c.Hk * all * D + 2 * at};
  }
  float* const rec = P.partials + (((int64_t)number * P.c.Hk + hk) * P.parts + part) * (P.width * (D + 2));
  return {rec + c * D, rec + P.width * D + 2 * c};
}

// Whether a piece's columns are done with this part; the place of its record among the others of a column.
template <bool SHARED>
__device__ __forceinline__ bool alone(const Piece& x, const Item& item) { return x.parts == 1 && !(SHARED && (item.group || x.group_parts > 0)); }
template <bool SHARED>
__device__ __forceinline__ int slot_of(const Kv4AttnParams& P, const Item& item) { return item.part + (SHARED && !item.group ? P.group_parts : 0); }

__device__ __forceinline__ uint64_t seen_from(const Kv4AttnParams& P, const Piece& x, int i, int j0) {
  return bbm::seen_from(P.mask ? P.mask + (int64_t)(x.s.begin + i) * P.mask_words : nullptr, P.mask_words, i, j0 - x.prefix);
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
  if (P.lse && e0 == 0) P.lse[(int64_t)h * P.T + t] = l > 0.0f ? bbm::log_sum(m, l, P.rc) : -INFINITY;
}

// lds_a, lds_b: 16 columns' results of two waves each.
template <int D>
constexpr int kNarrowLd = D + 4;  // row of the results in LDS
template <int D, bool SHARED>
__device__ __forceinline__ void narrow(const Kv4AttnParams& P, const Item& item, float* lds_a, float* lds_b, float (*m_s)[16], float (*l_s)[16]) {
  constexpr int KD = D / 4;        // elements of K a lane loads of its key
  constexpr int KS = D / 32;       // steps of the first product
  constexpr int VD = D / 16;       // elements of V a lane loads of a key, instructions of the second product
  constexpr int LD = kNarrowLd<D>;
  auto o_s = [&](int w, int c) { return (w < 2 ? lds_a : lds_b) + ((w & 1) * 16 + c) * LD; };

  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, kq = lane >> 4;
  const int wave = (int)scalar(tid >> 6);
  const int number = item.number, part = item.part, hk = item.hk;
  const Piece x = SHARED && item.group ? group_piece_of(P, number, 16) : piece_of<SHARED>(P, number, 16);
  if (x.s.end <= x.s.begin || part >= x.parts) return;
  const int first = (SHARED ? x.from : 0) + part * x.keys, last = first + min(x.keys, x.len - first);

  // this lane's column: Q as operands, how far it sees (columns behind the last repeat it; they are not written)
  const int my_i = min(x.col0 + n, x.cols - 1) / P.G, my_h = hk * P.G + (min(x.col0 + n, x.cols - 1) - my_i * P.G), my_t = x.s.begin + my_i;
  bf16x8 qf[KS];
  f32x4 acc[VD];
  bbm::RunningMax top;
  float l_run = 0.0f;
  {
    const __bf16* const row = P.q + (int64_t)my_t * P.q_row + my_h * P.q_head + kq * KD;
#pragma unroll
    for (int j = 0; j < KS; ++j) qf[j] = *reinterpret_cast<const bf16x8*>(row + 8 * j);
  }
#pragma unroll
  for (int j = 0; j < VD; ++j) acc[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const int sees_all = P.mask ? x.prefix - 1 : x.prefix + x.col0 / P.G;  // the last key that every column of the piece sees

  // 16 keys as they lie in the cache.  Each array's bytes of a block are a buffer of their own: what a lane loads is a constant away from a
  // scalar address, and of a block that is not there (behind the part's end, on a page outside the cache) zeros come.
  struct Block {
    uint32_t k[KD / 8], ks, v[4], vs;
    int valid;  // keys that are there: 16, or fewer at the end, or none
  };
  const Table table = table_of(P, x);
  auto page_at = [&](int j) { return table[scalar(min(j, last - 1) >> P.c.page_shift)]; };
  auto load = [&](Block& b, int j, int page) __attribute__((always_inline)) {
    const bool there = j < last && page >= 0 && page < P.c.pages;
    b.valid = (int)scalar(there ? min(16, last - j) : 0);
    const int64_t head = (int64_t)page * P.c.Hk + hk;
    const int in_page = j & (P.c.page - 1);
    const int64_t key = head * P.c.page + in_page;
    const int all = b.valid ? 16 * (D / 2) : 0;
    const __amdgpu_buffer_rsrc_t k_r = bbm::buffer_of(P.c.k + key * (D / 2), all), v_r = bbm::buffer_of(P.c.v + key * (D / 2), all);
    const __amdgpu_buffer_rsrc_t ks_r = bbm::buffer_of(P.c.k_scale + key * (D / 32), all / 16);
    const __amdgpu_buffer_rsrc_t vs_r = bbm::buffer_of(P.c.v_scale + head * (D / 32) * P.c.page + in_page, b.valid ? (D / 32 - 1) * P.c.page + 16 : 0);
    if constexpr (D == 128) {
      const bbm::u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(k_r, n * (D / 2) + kq * 16, 0, 0);
      for (int i = 0; i < 4; ++i) b.k[i] = w[i];
    } else {
      const bbm::u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(k_r, n * (D / 2) + kq * 8, 0, 0);
      for (int i = 0; i < 2; ++i) b.k[i] = w[i];
    }
    b.ks = __builtin_amdgcn_raw_buffer_load_b8(ks_r, n * (D / 32) + kq * KD / 32, 0, 0);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int at = 4 * kq * (D / 2) + n * (VD / 2) + r * (D / 2);
      if constexpr (D == 128) b.v[r] = __builtin_amdgcn_raw_buffer_load_b32(v_r, at, 0, 0);
      else b.v[r] = __builtin_amdgcn_raw_buffer_load_b16(v_r, at, 0, 0);
    }
    b.vs = __builtin_amdgcn_raw_buffer_load_b32(vs_r, n * VD / 32 * P.c.page + 4 * kq, 0, 0);
  };

  auto compute = [&](Block& a, Block& b, int j0) __attribute__((always_inline)) {
    const bool full = a.valid == 16 && b.valid == 16 && j0 + 31 <= sees_all;
    f32x4 sa = f32x4{0.0f, 0.0f, 0.0f, 0.0f}, sb = sa;
    const float ka = bbm::scale_of(a.ks), kb = bbm::scale_of(b.ks);
#pragma unroll
    for (int j = 0; j < KS; ++j) {
      sa = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bbm::values_of(a.k[j], ka), qf[j], sa, 0, 0, 0);
      sb = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bbm::values_of(b.k[j], kb), qf[j], sb, 0, 0, 0);
    }
    if (!full) {
      // keys that are not there get scores of -infinity, and scales of 0, since a NaN would survive a probability of 0
      auto there = [&](Block& z, f32x4& sz, int j) {
        const int have = max(0, min(4, z.valid - 4 * kq));
        z.vs &= have == 4 ? ~0u : (1u << (8 * have)) - 1u;
        const uint32_t bits = (uint32_t)seen_from(P, x, my_i, j + 4 * kq) & ((1u << have) - 1u);
#pragma unroll
        for (int r = 0; r < 4; ++r) sz[r] = bits >> r & 1 ? sz[r] : -INFINITY;
      };
      there(a, sa, j0);
      there(b, sb, j0 + 16);
    }
    float mx = fmaxf(fmaxf(fmaxf(sa[0], sa[1]), fmaxf(sa[2], sa[3])), fmaxf(fmaxf(sb[0], sb[1]), fmaxf(sb[2], sb[3])));
    top.update(other_max<16>(other_max<32>(mx)), P.lazy, P.rc, [&](float alpha) __attribute__((always_inline)) {
      l_run *= alpha;
#pragma unroll
      for (int j = 0; j < VD; ++j) acc[j] *= alpha;
    });
    // The far form for all rows (bbm_softmax.h): the test for it and the two forms behind it cost the kernel of D = 64 registers in scratch memory.  One token each of 64
    // requests of 8 to 16 thousand keys, 32 / 8 heads of 64: 104 us, as with the near form alone; with the test 117.
    const float off = top.m == -INFINITY ? 0.0f : top.m;
    bf16x8 pf;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const float p = __builtin_amdgcn_exp2f(((r < 4 ? sa[r & 3] : sb[r & 3]) - off) * P.rc);
      l_run += p;
      pf[r] = (__bf16)p;
    }
    // (byte r in the exponent's place, whatever lies around it, see scale_of)
    float fa[4], fb[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      fa[r] = __uint_as_float(r < 3 ? a.vs << (23 - 8 * r) : a.vs >> 1);
      fb[r] = __uint_as_float(r < 3 ? b.vs << (23 - 8 * r) : b.vs >> 1);
    }
    bbm::for_each_n(
        [&](auto pair) {
          constexpr int i = decltype(pair)::value;  // two neighbouring elements of each key
          uint32_t va[4], vb[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            va[r] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(a.v[r], fa[r], i));
            vb[r] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(b.v[r], fb[r], i));
          }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t sel = e ? 0x07060302u : 0x05040100u;  // the first or the second of them, of two keys
            const uint32_t w[4] = {__builtin_amdgcn_perm(va[1], va[0], sel), __builtin_amdgcn_perm(va[3], va[2], sel), __builtin_amdgcn_perm(vb[1], vb[0], sel),
                                   __builtin_amdgcn_perm(vb[3], vb[2], sel)};
            acc[2 * i + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bbm::operand(w), pf, acc[2 * i + e], 0, 0, 0);
          }
          if constexpr (D == 128) __builtin_amdgcn_sched_barrier(0);  // (not all of them at once: registers)
        },
        std::make_integer_sequence<int, VD / 2>{});
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
  const float l = other_sum<16>(other_sum<32>(l_run));
  if (kq == 0) m_s[wave][n] = top.m, l_s[wave][n] = l;
  // lane (n, kq): rows 4 kq + r of instruction j, element (4 kq + r) * VD + j
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int j = 0; j < VD; j += 4) *reinterpret_cast<f32x4*>(o_s(wave, n) + (4 * kq + r) * VD + j) = f32x4{acc[j][r], acc[j + 1][r], acc[j + 2][r], acc[j + 3][r]};
  __syncthreads();
  const int c = tid >> 4, e0 = (tid & 15) * VD, col = x.col0 + c;
  if (col >= x.cols) return;
  float m = -INFINITY;
#pragma unroll
  for (int w = 0; w < NW; ++w) m = fmaxf(m, m_s[w][c]);
  const float m_fin = m == -INFINITY ? 0.0f : m;
  float sum = 0.0f, v[VD] = {};
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const float f = bbm::weight(m_s[w][c], m_fin, P.rc);
    sum += f * l_s[w][c];
#pragma unroll
    for (int e = 0; e < VD; ++e) v[e] += f * o_s(w, c)[e0 + e];
  }
  if (alone<SHARED>(x, item)) {
    put_column<D>(P, x, hk, col, e0, v, m, sum);
  } else {
    const Record rec = record_of<D, SHARED>(P, x, number, hk, slot_of<SHARED>(P, item), c);
#pragma unroll
    for (int e = 0; e < VD; e += 4) *reinterpret_cast<f32x4*>(rec.sums + e0 + e) = f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]};
    if (e0 == 0) *reinterpret_cast<float2*>(rec.pair) = make_float2(m, sum);
  }
}

// 128 columns of a piece, a wave 32 of them, one lane a column, with the products of the kernels for prompts: the codes of 64 keys at a time are converted once
// for all of them, on their way to LDS, where the tile is read as keys and values in bf16 are.
template <int D, bool SHARED>
__device__ __forceinline__ void wide(const Kv4AttnParams& P, const Item& item, __bf16* k_s0, __bf16* k_s1, __bf16* v_s0, __bf16* v_s1, uint32_t (*there_s)[NW]) {
  using L = bbm::TL<D>;
  constexpr int KS = D / 16, DB = D / 32, RC = D / 8, RPB = 64 / RC;
  constexpr int W = D / 32;  // 32-bit words of codes a thread converts of a tensor

  const int tid = threadIdx.x, lane = tid & 63, lq = lane & 31, hh = lane >> 5;
  const int wave = (int)scalar(tid >> 6);
  const int number = item.number, part = item.part, hk = item.hk;
  const Piece x = SHARED && item.group ? group_piece_of(P, number, 128) : piece_of<SHARED>(P, number, 128);
  if (x.s.end <= x.s.begin || part >= x.parts) return;
  const int first = (SHARED ? x.from : 0) + part * x.keys, last = first + min(x.keys, x.len - first);
  const int n_tiles = (last - first + 63) / 64;

  const int wcol = x.col0 + 32 * wave, my_col = min(wcol + lq, x.cols - 1), my_i = my_col / P.G, my_h = hk * P.G + (my_col - my_i * P.G);
  const int wcols = max(0, min(32, x.cols - wcol));
  const int sees_all = P.mask ? x.prefix - 1 : x.prefix + x.col0 / P.G;
  bf16x8 qf[KS];
  {
    const __bf16* const row = P.q + (int64_t)(x.s.begin + my_i) * P.q_row + my_h * P.q_head + hh * 8;
#pragma unroll
    for (int t = 0; t < KS; ++t) qf[t] = *reinterpret_cast<const bf16x8*>(row + 16 * t);
  }
  f32x16 oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
    for (int e = 0; e < 16; ++e) oacc[db][e] = 0.0f;
  bbm::RunningMax top;
  float l_run = 0.0f;
  bbm::TileAddr<D> A;
  A.init(lane);

  // A wave converts 16 keys of a tile, which lie on one page, a quarter of a key's elements a lane.  (Lanes take the keys in an order in which 16 of them
  // write to all banks: rows four apart differ in the turn of their chunks.)
  const Table table = table_of(P, x);
  const int row = (lane >> 2 & 3) * 4 + (lane >> 4), quarter = lane & 3;  // of the wave's 16
  struct Raw {
    uint32_t k[W], v[W], ks, vs;
    int valid;  // keys that are there
  };
  auto page_at = [&](int tile) { return table[scalar(min(first + tile * 64 + 16 * wave, max(0, last - 1)) >> P.c.page_shift)]; };
  auto load = [&](Raw& z, int tile, int page) __attribute__((always_inline)) {
    const int j = first + tile * 64 + 16 * wave;
    z.valid = (int)scalar(j < last && page >= 0 && page < P.c.pages ? min(16, last - j) : 0);
    const int64_t head = (int64_t)page * P.c.Hk + hk;
    const int in_page = j & (P.c.page - 1);
    const int64_t key = head * P.c.page + in_page;
    const int all = z.valid ? 16 * (D / 2) : 0, at = row * (D / 2) + quarter * (D / 8);
    const __amdgpu_buffer_rsrc_t k_r = bbm::buffer_of(P.c.k + key * (D / 2), all), v_r = bbm::buffer_of(P.c.v + key * (D / 2), all);
    const __amdgpu_buffer_rsrc_t ks_r = bbm::buffer_of(P.c.k_scale + key * (D / 32), all / 16);
    const __amdgpu_buffer_rsrc_t vs_r = bbm::buffer_of(P.c.v_scale + head * (D / 32) * P.c.page + in_page, z.valid ? (D / 32 - 1) * P.c.page + 16 : 0);
    if constexpr (D == 128) {
      const bbm::u32x4 a = __builtin_amdgcn_raw_buffer_load_b128(k_r, at, 0, 0), b = __builtin_amdgcn_raw_buffer_load_b128(v_r, at, 0, 0);
      for (int i = 0; i < W; ++i) z.k[i] = a[i], z.v[i] = b[i];
    } else {
      const bbm::u32x2 a = __builtin_amdgcn_raw_buffer_load_b64(k_r, at, 0, 0), b = __builtin_amdgcn_raw_buffer_load_b64(v_r, at, 0, 0);
      for (int i = 0; i < W; ++i) z.k[i] = a[i], z.v[i] = b[i];
    }
    z.ks = __builtin_amdgcn_raw_buffer_load_b8(ks_r, row * (D / 32) + quarter * D / 128, 0, 0);
    z.vs = __builtin_amdgcn_raw_buffer_load_b8(vs_r, quarter * D / 128 * P.c.page + row, 0, 0);
  };
  // piece i of 2 W of what a lane converts
  auto store_piece = [&](Raw& z, __bf16* kd, __bf16* vd, uint32_t* there_d, int i) __attribute__((always_inline)) {
    const int r = 16 * wave + row, base = r % L::NBLK * L::TBLK + r / L::NBLK * D, turn = r >> 2 & 3;
    const int chunk = (quarter * W + i % W) ^ turn;
    if (i < W)
      *reinterpret_cast<bf16x8*>(kd + base + chunk * 8) = bbm::values_of(z.k[i % W], bbm::scale_of(z.ks));
    else  // (a NaN would survive a probability of 0)
      *reinterpret_cast<bf16x8*>(vd + base + chunk * 8) = bbm::values_of(z.v[i % W], bbm::scale_of(row < z.valid ? z.vs : 0));
    if (i == 2 * W - 1 && lane == 0) there_d[wave] = (1u << z.valid) - 1u;
  };

  Raw raw[2];  // of the tile behind the one in use, and of the next: asked for two steps before they are converted
  auto step = [&](auto pb, int tile, int& page) __attribute__((always_inline)) {
    constexpr int PB = decltype(pb)::value;
    __syncthreads();  // the tile is there, and everyone is done with the one in the other buffers
    __bf16* const k_cur = PB ? k_s1 : k_s0;
    __bf16* const v_cur = PB ? v_s1 : v_s0;
    __bf16* const k_oth = PB ? k_s0 : k_s1;
    __bf16* const v_oth = PB ? v_s0 : v_s1;
    const int j0 = first + tile * 64;
    f32x16 sc[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
      for (int e = 0; e < 16; ++e) sc[kb][e] = 0.0f;
    // The next tile is converted behind the matrix instructions of the first product.  (Behind the last tile too, of which zeros are loaded and stored:
    // with loads behind a branch the compiler cannot count those under way, and waits for all of them.)
    bbm::mfma_ring<2 * KS, 4>([&](auto i) { return A.row_frag(k_cur, decltype(i)::value & 1, decltype(i)::value >> 1); },
                              [&](auto i, bf16x8 f) {
                                constexpr int y = decltype(i)::value;
                                sc[y & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, qf[y >> 1], sc[y & 1], 0, 0, 0);
                              },
                              [&](auto i) {
                                constexpr int y = decltype(i)::value, GAP = KS / W;
                                if constexpr (y % GAP == 0) store_piece(raw[PB ^ 1], k_oth, v_oth, there_s[PB ^ 1], y / GAP);
                              });
    load(raw[PB ^ 1], tile + 3, page);
    page = page_at(tile + 4);
    {
      const uint4 t4 = *reinterpret_cast<const uint4*>(there_s[PB]);
      const uint32_t t_lo = scalar(t4.x | t4.y << 16), t_hi = scalar(t4.z | t4.w << 16);
      if ((t_lo & t_hi) != ~0u || j0 + 63 > sees_all) {
        const uint64_t seen = seen_from(P, x, my_i, j0) & ((uint64_t)t_hi << 32 | t_lo);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          const uint32_t w = (uint32_t)(seen >> (32 * kb)) >> (4 * hh);
#pragma unroll
          for (int e = 0; e < 16; ++e) sc[kb][e] = bbm::keep_if(w, e, sc[kb][e]);
        }
      }
      float mx = sc[0][0];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
        for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sc[kb][e]);
      top.update(other_max<32>(mx), P.lazy, P.rc, [&](float alpha) __attribute__((always_inline)) {
        l_run *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db)
          for (int e = 0; e < 16; ++e) oacc[db][e] *= alpha;
      });
      if (top.far) {
        const float off = top.offset(P.rc);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
          for (int e = 0; e < 16; ++e) sc[kb][e] -= off;
      }
      bf16x8 pf[2];
      auto exps = [&](int u, int e0, int e1) {
#pragma unroll
        for (int e = e0; e < e1; ++e) {
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[u / 2][8 * (u % 2) + e], P.rc, top.nm));
          l_run += p;
          pf[u & 1][e] = (__bf16)p;
        }
      };
      exps(0, 0, 8);
      bbm::mfma_ring<4 * DB, 3>([&](auto i) { return A.tr_frag(v_cur, decltype(i)::value / DB, decltype(i)::value % DB); },
                                [&](auto i, bf16x8 f) {
                                  constexpr int y = decltype(i)::value;
                                  oacc[y % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, pf[y / DB & 1], oacc[y % DB], 0, 0, 0);
                                },
                                [&](auto i) {
                                  constexpr int y = decltype(i)::value, PER = 8 / DB;
                                  if constexpr (y / DB < 3) exps(y / DB + 1, y % DB * PER, (y % DB + 1) * PER);
                                });
    }
  };
  if (n_tiles > 0) {
    load(raw[0], 0, page_at(0));
    load(raw[1], 1, page_at(1));
    int page = page_at(2);
#pragma unroll
    for (int i = 0; i < 2 * W; ++i) store_piece(raw[0], k_s0, v_s0, there_s[0], i);
    __builtin_amdgcn_sched_barrier(0);  // (tile 1 is asked for before tile 2: the first step waits for the older loads)
    load(raw[0], 2, page);
    page = page_at(3);
    // (Q is waited for here; in the loop, where the compiler would have it, the wait takes the next tile's loads with it)
#pragma unroll
    for (int t = 0; t < KS; ++t) asm volatile("" : "+v"(qf[t]));
#pragma unroll 1
    for (int tile = 0; tile + 1 < n_tiles; tile += 2) {  // (with a way around the second step the compiler is not sure which loads are the older ones)
      step(bbm::IntC<0>{}, tile, page);
      step(bbm::IntC<1>{}, tile + 1, page);
    }
    if (n_tiles & 1) step(bbm::IntC<0>{}, n_tiles - 1, page);
  }
  __syncthreads();  // the result is staged in the tile buffers
  if (wcols == 0) return;
  const float l = other_sum<32>(l_run);
  if (!alone<SHARED>(x, item)) {
    if (lq < wcols) {
      const Record rec = record_of<D, SHARED>(P, x, number, hk, slot_of<SHARED>(P, item), 32 * wave + lq);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<f32x4*>(rec.sums + 32 * db + 8 * g + 4 * hh) = f32x4{oacc[db][4 * g], oacc[db][4 * g + 1], oacc[db][4 * g + 2], oacc[db][4 * g + 3]};
      if (hh == 0) *reinterpret_cast<float2*>(rec.pair) = make_float2(top.m, l);
    }
    return;
  }
  __bf16* const stage = (wave / 2 == 0 ? k_s0 : v_s0) + wave % 2 * 32 * D;
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      bbm::bf16x4 y;
      for (int e = 0; e < 4; ++e) y[e] = (__bf16)(oacc[db][4 * g + e] * inv);
      *reinterpret_cast<bbm::bf16x4*>(stage + lq * D + (((4 * db + g) ^ (lq % RC)) * 8) + 4 * hh) = y;
    }
#pragma unroll
  for (int i = 0; i < 32 / RPB; ++i) {
    const int r = i * RPB + lane / RC, col = wcol + r, tok = col / P.G, h = hk * P.G + (col - tok * P.G);
    if (r < wcols)
      *reinterpret_cast<bf16x8*>(P.o + (int64_t)(x.s.begin + tok) * P.o_row + h * P.o_head + lane % RC * 8) = *reinterpret_cast<const bf16x8*>(stage + r * D + (lane % RC ^ r % RC) * 8);
  }
  if (P.lse && hh == 0 && lq < wcols) P.lse[(int64_t)my_h * P.T + x.s.begin + my_i] = l > 0.0f ? bbm::log_sum(top.m, l, P.rc) : -INFINITY;
}

template <int D, bool SHARED>
__global__ __launch_bounds__(64 * NW, D == 128 ? 3 : 5) void kv4_narrow_kernel(const Kv4AttnParams P) {
  __shared__ __attribute__((aligned(16))) float o_s[NW][16][kNarrowLd<D>];
  __shared__ float m_s[NW][16], l_s[NW][16];
  const Item item = item_of<SHARED>(P);
  if (SHARED && item.none) return;
  narrow<D, SHARED>(P, item, &o_s[0][0][0], &o_s[2][0][0], m_s, l_s);
}

// (there_s: which of a tile's keys are there, 16 a wave)
#define BBM_WIDE_LDS                                                             \
  using L = bbm::TL<D>;                                                          \
  __shared__ __attribute__((aligned(16))) __bf16 k_s0[L::ELEMS];                 \
  __shared__ __attribute__((aligned(16))) __bf16 k_s1[L::ELEMS];                 \
  __shared__ __attribute__((aligned(16))) __bf16 v_s0[L::ELEMS];                 \
  __shared__ __attribute__((aligned(16))) __bf16 v_s1[L::ELEMS];                 \
  __shared__ __attribute__((aligned(16))) uint32_t there_s[2][NW]

template <int D, bool SHARED>
__global__ __launch_bounds__(64 * NW, 2) void kv4_wide_kernel(const Kv4AttnParams P) {
  BBM_WIDE_LDS;
  const Item item = item_of<SHARED>(P);
  if (SHARED && item.none) return;
  wide<D, SHARED>(P, item, k_s0, k_s1, v_s0, v_s1, there_s);
}

// Groups of many columns side by side with requests of few, in the same LDS.
template <int D>
__global__ __launch_bounds__(64 * NW, 2) void kv4_both_kernel(const Kv4AttnParams P) {
  BBM_WIDE_LDS;
  static_assert(2 * 16 * kNarrowLd<D> * sizeof(float) <= sizeof(k_s0) && 2 * NW * 16 * sizeof(float) <= sizeof(k_s1), "the results of two waves, and all statistics, must fit in a tile buffer");
  const Item item = item_of<true>(P);
  if (item.none) return;
  if (item.group) {
    wide<D, true>(P, item, k_s0, k_s1, v_s0, v_s1, there_s);
  } else {
    float(*const m_s)[16] = reinterpret_cast<float(*)[16]>(k_s1);
    narrow<D, true>(P, item, reinterpret_cast<float*>(k_s0), reinterpret_cast<float*>(v_s0), m_s, m_s + NW);
  }
}
#undef BBM_WIDE_LDS

// Joins the parts of a piece's columns in a fixed order, 16 lanes a column.  With many parts (SIDE = 4) a wave takes one column and four parts side by
// side, whose sums meet at the end; with few, a column for every 16 lanes: a wave costs more to start than to add up four records.
template <int D, int SIDE, bool SHARED>
__global__ __launch_bounds__(256) void kv4_join_kernel(const Kv4AttnParams P) {
  constexpr int VD = D / 16;
  const int lane = threadIdx.x & 63, number = blockIdx.x, hk = blockIdx.y, e0 = (lane & 15) * VD;
  const int c = SIDE == 4 ? 4 * blockIdx.z + (threadIdx.x >> 6) : 16 * blockIdx.z + (threadIdx.x >> 4);
  const Piece x = piece_of<SHARED>(P, number, SHARED ? (SIDE == 4 ? 4 : 16) : P.width);
  const int parts = x.parts + x.group_parts;
  if (x.s.end <= x.s.begin || parts == 1 || x.col0 + c >= x.cols) return;
  // (a part's records are `stride` apart, its pairs `pairs`; a request's own lie behind all that a group may have)
  const Record rec = record_of<D, SHARED>(P, x, number, hk, 0, c);
  const int64_t stride = SHARED ? P.c.Hk * ((int64_t)P.T * P.G) * D : (int64_t)P.width * (D + 2), pairs = SHARED ? P.c.Hk * ((int64_t)P.T * P.G) * 2 : stride;
  auto slot = [&](int p) { return SHARED && p >= x.group_parts ? p - x.group_parts + P.group_parts : p; };
  float m = -INFINITY, l = 0.0f, v[VD] = {};
#pragma unroll 1
  for (int p = SIDE == 4 ? lane >> 4 : 0; p < parts; p += 4 * SIDE) {  // four records' loads in flight
    float2 ml[4];
    f32x4 y[4][VD / 4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = slot(min(p + SIDE * i, parts - 1));
      ml[i] = *reinterpret_cast<const float2*>(rec.pair + at * pairs);
      if (p + SIDE * i >= parts) ml[i] = make_float2(-INFINITY, 0.0f);
#pragma unroll
      for (int e = 0; e < VD / 4; ++e) y[i][e] = *reinterpret_cast<const f32x4*>(rec.sums + at * stride + e0 + 4 * e);
    }
    const float m_new = fmaxf(fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x)), m), m_fin = m_new == -INFINITY ? 0.0f : m_new;
    const float keep = bbm::weight(m, m_fin, P.rc);
    m = m_new;
    l *= keep;
#pragma unroll
    for (int e = 0; e < VD; ++e) v[e] *= keep;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float f = bbm::weight(ml[i].x, m_fin, P.rc);
      l += f * ml[i].y;
#pragma unroll
      for (int e = 0; e < VD; ++e) v[e] += f * y[i][e / 4][e % 4];
    }
  }
  if constexpr (SIDE == 4) {
    const float m_all = other_max<16>(other_max<32>(m)), f = bbm::weight(m, m_all == -INFINITY ? 0.0f : m_all, P.rc);
    l = other_sum<16>(other_sum<32>(l * f));
#pragma unroll
    for (int e = 0; e < VD; ++e) v[e] = other_sum<16>(other_sum<32>(v[e] * f));
    m = m_all;
  }
  if (SIDE == 1 || lane < 16) put_column<D>(P, x, hk, x.col0 + c, e0, v, m, l);
}

// How a call is cut: pieces of `width` columns, at most `parts` parts of the keys, of at least part_keys each.
struct Plan {
  int width;
  int64_t pieces, parts, part_keys;
};
// Work-groups that occupy the chip, and that keep it busy to the end of a call whose requests differ in length; the keys that a part is worth for
// either.  (Every part costs its record and a share of the join.)  D = 128, 32 / 8 heads, us: one token each of 128 requests of 2048 keys whole / in two
// parts 49 / 56; of 64 requests of 16384 in 1 / 2 / 4 parts 206 / 182 / 173; of 8 requests of 8192 in 8 parts of 1024 / 16 of 512 22.3 / 20.7;
// of one request of 32768 in 32 parts of 1024 / 64 of 512 16.4 / 18.0.
constexpr int64_t kOccupy = 512, kBusy = 2048, kPartKeys = 1024, kLongPartKeys = 4096;
// The wide kernel takes 128 columns at 1.5 us for 64 keys and has few work-groups; the narrow one reads the keys again for every 16 columns.
// 32 / 8 heads over 4096 keys, us, narrow / wide: 16 requests of 8 tokens (32 columns) 30 / 42, of 16 40 / 44, of 32 (16 x 32 x 32 rows) 61 / 51; 4 requests
// of 64 35 / 43; 3 of 32 over 1000 keys 10 / 25; trees of 256 nodes, 8 x 32 heads, 88 / 53.
constexpr int64_t kWideColumns = 64, kWideRows = 16384;
inline Plan plan_of(int64_t T, int64_t R, int64_t G, int64_t Hk, int64_t max_len) {
  Plan p;
  const bool wide = T * G >= kWideColumns * R && T * G * Hk >= kWideRows;
  p.width = wide ? 128 : 16;
  p.pieces = bbm::count_pieces(T, R, G, p.width);
  const int64_t busy = std::max(std::min(T, R), bbm::ceil_div(T * G, p.width)) * Hk;  // pieces that belong to a request, or few fewer
  p.parts = std::min(bbm::ceil_div(kOccupy, busy), max_len / kPartKeys);
  if (!wide) p.parts = std::max(p.parts, std::min(bbm::ceil_div(kBusy, busy), max_len / kLongPartKeys));
  p.parts = std::max<int64_t>(p.parts, 1);
  p.part_keys = bbm::ceil_div(bbm::ceil_div(max_len, p.parts), kStep) * kStep;
  p.parts = bbm::ceil_div(max_len, p.part_keys);
  return p;
}
inline bool sizes_ok(int64_t T, int64_t R, int64_t H, int64_t Hk, int64_t max_len) {
  return T >= 1 && R >= 1 && H >= 1 && Hk >= 1 && H % Hk == 0 && max_len >= 1 && T <= bbm::kMaxTokens && R <= bbm::kMaxTokens && H <= 65535;
}

template <int D>
void launch(const Kv4AttnParams& P, hipStream_t s) {
  const unsigned wgs = (unsigned)((int64_t)P.pieces * P.c.Hk * P.parts);
  if (P.width == 16) kv4_narrow_kernel<D, false><<<wgs, 64 * NW, 0, s>>>(P);
  else kv4_wide_kernel<D, false><<<wgs, 64 * NW, 0, s>>>(P);
  if (P.parts > 4) kv4_join_kernel<D, 4, false><<<dim3((unsigned)P.pieces, (unsigned)P.c.Hk, (unsigned)P.width / 4), 256, 0, s>>>(P);
  else if (P.parts > 1) kv4_join_kernel<D, 1, false><<<dim3((unsigned)P.pieces, (unsigned)P.c.Hk, (unsigned)P.width / 16), 256, 0, s>>>(P);
}

}  // namespace

extern "C" __attribute__((visibility("default"))) size_t bbm_kv4_attn_workspace_bytes(int64_t T, int64_t R, int64_t H, int64_t Hk, int d, int64_t max_len) {
  if (!sizes_ok(T, R, H, Hk, max_len) || (d != 64 && d != 128)) return 0;
  const Plan p = plan_of(T, R, H / Hk, Hk, std::min<int64_t>(max_len, bbm::kMaxTokens));
  return p.parts == 1 ? 0 : (size_t)(p.pieces * Hk * p.parts * p.width * (d + 2)) * sizeof(float);
}

namespace {

// A call's arguments as both entry points have them.
struct Call {
  const bbm_packed *q, *o;
  float* lse;
  int64_t T, R;
  const int32_t *cu, *lens, *table;
  int64_t table_stride, max_pages;
  const uint64_t* mask;
  int64_t mask_words;
  const bbm_kv4_cache* cache;
  int64_t H;
  float softmax_scale;
  void* workspace;
  size_t workspace_bytes;
};
int check_call(const char* fn, const Call& a) {
  using namespace bbm;
  if (int rc = check_kv4(fn, a.cache)) return rc;
  if (int rc = check_tokens(fn, a.T, a.R, a.cu, a.H, a.cache->Hk)) return rc;
  if (int rc = check_packed(fn, "q", a.q, a.T, a.H, a.cache->d, false)) return rc;
  if (int rc = check_packed(fn, "o", a.o, a.T, a.H, a.cache->d, true)) return rc;
  if (!aligned(a.lse, 4)) return fail(BBM_EINVAL, "%s: lse must be 4-byte aligned", fn);
  if (int rc = check_table(fn, a.lens, a.table, a.table_stride, a.max_pages, a.cache->page)) return rc;
  if (int rc = check_mask(fn, a.mask, a.mask_words)) return rc;
  if (a.T * (a.H / a.cache->Hk) > kMaxTokens) return fail(BBM_EUNSUPPORTED, "%s: problem too large (T=%lld, H=%lld)", fn, (long long)a.T, (long long)a.H);
  return check_scale(fn, a.softmax_scale);
}
int check_workspace(const char* fn, const Call& a, size_t need) {
  using namespace bbm;
  if (need > 0 && (!a.workspace || a.workspace_bytes < need))
    return fail(BBM_EWORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need, a.workspace ? a.workspace_bytes : (size_t)0);
  if (!aligned(a.workspace, 16)) return fail(BBM_EINVAL, "%s: workspace must be 16-byte aligned", fn);
  return BBM_OK;
}
Kv4AttnParams params_of(const Call& a) {
  using namespace bbm;
  Kv4AttnParams P = {};
  P.c = kv4_of(a.cache);
  P.q = static_cast<const __bf16*>(a.q->ptr), P.o = static_cast<__bf16*>(a.o->ptr), P.lse = a.lse;
  P.q_row = a.q->row_stride, P.q_head = a.q->head_stride, P.o_row = a.o->row_stride, P.o_head = a.o->head_stride, P.table_stride = a.table_stride;
  P.cu = a.cu, P.lens = a.lens, P.table = a.table, P.mask = a.mask, P.partials = static_cast<float*>(a.workspace);
  P.T = (int32_t)a.T, P.R = (int32_t)a.R, P.G = (int32_t)(a.H / a.cache->Hk), P.max_pages = (int32_t)a.max_pages, P.mask_words = (int32_t)a.mask_words;
  P.rc = a.softmax_scale * kLog2e, P.lazy = kLazy / P.rc;
  return P;
}

}  // namespace

extern "C" __attribute__((visibility("default"))) int bbm_kv4_attn(const bbm_packed* q, const bbm_packed* o, float* lse, int64_t T, int64_t R, const int32_t* cu,
                                                                   const int32_t* lens, const int32_t* block_table, int64_t table_stride, int64_t max_pages,
                                                                   const uint64_t* mask, int64_t mask_words, const bbm_kv4_cache* cache, int64_t H,
                                                                   float softmax_scale, int64_t max_len, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace bbm;
  const char* fn = "bbm_kv4_attn";
  clear_error();
  const Call a{q, o, lse, T, R, cu, lens, block_table, table_stride, max_pages, mask, mask_words, cache, H, softmax_scale, workspace, workspace_bytes};
  if (int rc = check_call(fn, a)) return rc;
  if (max_len < 1) return fail(BBM_EINVAL, "%s: max_len=%lld must be >= 1", fn, (long long)max_len);
  const size_t need = bbm_kv4_attn_workspace_bytes(T, R, H, cache->Hk, cache->d, max_len);
  if (int rc = check_workspace(fn, a, need)) return rc;
  if (T == 0) return BBM_OK;
  if (int rc = check_apart(fn, {o->ptr, lse, need > 0 ? workspace : nullptr}, {q->ptr, cu, lens, block_table, mask, cache->k, cache->k_scale, cache->v, cache->v_scale})) return rc;
  Kv4AttnParams P = params_of(a);
  const Plan p = plan_of(T, R, P.G, cache->Hk, std::min<int64_t>(max_len, bbm::kMaxTokens));
  if (p.pieces >= kMaxWgs || p.pieces * cache->Hk * p.parts >= kMaxWgs) return fail(BBM_EUNSUPPORTED, "%s: problem too large (T=%lld, R=%lld, H=%lld)", fn, (long long)T, (long long)R, (long long)H);
  P.width = p.width, P.pieces = (int32_t)p.pieces, P.parts = (int32_t)p.parts, P.part_keys = (int32_t)p.part_keys;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (cache->d == 64) launch<64>(P, s);
  else launch<128>(P, s);
  return launch_status(fn);
}

namespace {

// Of a call with shared prefixes: the groups' cut and the requests'.
struct SharedPlan {
  Plan group, own;
  bool apart;  // each request for itself, as without groups
};
// Short prefixes of few requests are better read for each of them: one launch and no join.  32 / 8 heads of 128, us, by groups / apart: 4 requests behind 512 keys 10.5 / 7.9, behind 1024
// 10.6 / 10.8, behind 2048 11.1 / 13.5; 32 requests 11.9 / 8.3, 12.2 / 11.6, 15.8 / 18.3 (20, 38 and 74 MB read apart).  Heads of 64: 9.8 / 7.3, 9.9 / 9.8, 10.2 / 12.4; 10.8 / 7.6,
// 11.0 / 10.2, 13.7 / 16.5.
constexpr int64_t kApartKeys = 1152, kApartBytes = 40 << 20;
// Groups take the wide kernel from this many columns of a group on, on average.  32 / 8 heads of 128, us, narrow / wide: 16 requests of one token behind 8192 common keys (64 columns) 19 / 23,
// 32 (128 columns) 26 / 28, 67 (268) 43 / 37, 256 behind 32768 (1024) 263 / 185; heads of 64, 64 columns 16.3 / 16.6, 128 22.5 / 26.6, 192 25.6 / 26.0, 268 33.5 / 32.5, 1024 247 / 124.
// (The columns are an average over the groups, rows that are in none counted in: one large group among groups of few columns gets the narrow kernel too.)
// The narrow one's parts have at least 512 keys (groups are few, and the join has to be there anyway): 32 requests behind 1024 keys 15.1 us, of 1024 16.2; four heads of 64 behind 8192 11.4 / 13.0.
constexpr int64_t kGroupWideColumns = 192, kGroupPartKeys = 512;
// The wide one's are chosen by what they take: a tile of 64 keys of a work-group that has a CU to itself, of two that share one, and a MB of records, written and read, in us.  (With
// 512 keys a part and no more than 512 work-groups instead: 67 requests behind 8192 keys 41 us, with this 37; 32 requests behind 4096 keys, eight heads over one of 128, 25 and 17.)  They are
// times of heads of 128, used for heads of 64 too.  What is chosen / the best of 13 numbers of parts from 1 to 64, us: 67 requests behind 8192 keys 33.6 / 33.2, of 64 30.9 / 27.3; 256 behind 32768
// 190 / 180, 134 / 122; 100 behind 16384 72 / 57, 52 / 43; 32 behind 4096, eight heads over one, 16.2 / 16.5, 12.7 / 12.8.
constexpr double kTileAlone = 1.4, kTileShared = 2.2, kRecordMB = 0.25;
inline int64_t wide_parts(int64_t pieces, int64_t max_keys, double record_mb) {
  int64_t best = 1;
  double least = 0.0;
  for (int64_t parts = 1; parts <= std::min<int64_t>(64, bbm::ceil_div(max_keys, kStep)); ++parts) {
    const int64_t keys = bbm::ceil_div(bbm::ceil_div(max_keys, parts), kStep) * kStep, wgs = pieces * bbm::ceil_div(max_keys, keys);
    const double cost = (double)(keys / 64) * (wgs <= 256 ? kTileAlone : kTileShared * (double)bbm::ceil_div(wgs, 512)) + (double)parts * record_mb * kRecordMB;
    if (parts == 1 || cost < least) best = parts, least = cost;
  }
  return best;
}
inline SharedPlan shared_plan_of(int64_t T, int64_t R, int64_t S, int64_t G, int64_t Hk, int d, int64_t max_shared, int64_t max_own) {
  SharedPlan p;
  p.apart = S > 0 && max_shared + max_own <= kApartKeys && R * (max_shared + max_own) * Hk <= kApartBytes / (d * 17 / 16);
  p.own = plan_of(T, R, G, Hk, p.apart ? max_shared + max_own : max_own);
  if (S == 0 || p.apart) {
    p.group = Plan{p.own.width, 0, 0, kStep};
    return p;
  }
  const bool wide = p.own.width == 128 || T * G >= kGroupWideColumns * S;
  p.group.width = wide ? 128 : 16;
  p.group.pieces = bbm::count_pieces(T, S, G, p.group.width);
  const int64_t busy = std::max(std::min(T, S), bbm::ceil_div(T * G, p.group.width)) * Hk;
  p.group.parts = wide ? wide_parts(S * bbm::ceil_div(T * G, 128 * S) * Hk, max_shared, (double)T * (double)(G * Hk) * (d + 2) * 8e-6)
                       : std::max<int64_t>(1, std::min(bbm::ceil_div(kOccupy, busy), max_shared / kGroupPartKeys));
  p.group.part_keys = bbm::ceil_div(bbm::ceil_div(max_shared, p.group.parts), kStep) * kStep;
  p.group.parts = bbm::ceil_div(max_shared, p.group.part_keys);
  return p;
}
inline size_t shared_workspace(const SharedPlan& p, int64_t T, int64_t H, int d) {
  return p.group.parts + p.own.parts <= 1 ? 0 : (size_t)((p.group.parts + p.own.parts) * T * H) * (size_t)(d + 2) * sizeof(float);
}

template <int D>
void launch_shared(Kv4AttnParams P, const SharedPlan& p, hipStream_t s) {
  const int64_t group = p.group.pieces * P.c.Hk * p.group.parts, own = p.own.pieces * P.c.Hk * p.own.parts;
  P.group_wgs = (int32_t)group, P.own_wgs = (int32_t)own;
  const unsigned wgs = (unsigned)(((group + 7) & ~7ll) + own);
  if (p.own.width == 128) kv4_wide_kernel<D, true><<<wgs, 64 * NW, 0, s>>>(P);
  else if (p.group.width == 128 && group > 0) kv4_both_kernel<D><<<wgs, 64 * NW, 0, s>>>(P);
  else kv4_narrow_kernel<D, true><<<wgs, 64 * NW, 0, s>>>(P);
  if (p.group.parts + p.own.parts > 4)
    kv4_join_kernel<D, 4, true><<<dim3((unsigned)bbm::count_pieces(P.T, P.R, P.G, 4), (unsigned)P.c.Hk), 256, 0, s>>>(P);
  else if (p.group.parts + p.own.parts > 1)
    kv4_join_kernel<D, 1, true><<<dim3((unsigned)bbm::count_pieces(P.T, P.R, P.G, 16), (unsigned)P.c.Hk), 256, 0, s>>>(P);
}

}  // namespace

extern "C" __attribute__((visibility("default"))) size_t bbm_kv4_shared_attn_workspace_bytes(int64_t T, int64_t R, int64_t S, int64_t H, int64_t Hk, int d, int64_t max_shared,
                                                                                             int64_t max_own) {
  if (!sizes_ok(T, R, H, Hk, std::min(max_shared, max_own)) || S < 0 || S > R || (d != 64 && d != 128)) return 0;
  return shared_workspace(shared_plan_of(T, R, S, H / Hk, Hk, d, std::min<int64_t>(max_shared, bbm::kMaxTokens), std::min<int64_t>(max_own, bbm::kMaxTokens)), T, H, d);
}

extern "C" __attribute__((visibility("default"))) int bbm_kv4_shared_attn(const bbm_packed* q, const bbm_packed* o, float* lse, int64_t T, int64_t R, const int32_t* cu,
                                                                          const int32_t* lens, const int32_t* block_table, int64_t table_stride, int64_t max_pages, int64_t S,
                                                                          const int32_t* group_cu, const int32_t* shared_lens, const uint64_t* mask, int64_t mask_words,
                                                                          const bbm_kv4_cache* cache, int64_t H, float softmax_scale, int64_t max_shared, int64_t max_own,
                                                                          void* workspace, size_t workspace_bytes, void* stream) {
  using namespace bbm;
  const char* fn = "bbm_kv4_shared_attn";
  clear_error();
  const Call a{q, o, lse, T, R, cu, lens, block_table, table_stride, max_pages, mask, mask_words, cache, H, softmax_scale, workspace, workspace_bytes};
  if (int rc = check_call(fn, a)) return rc;
  if (int rc = check_groups(fn, R, S, group_cu, shared_lens, max_shared, max_own)) return rc;
  const size_t need = bbm_kv4_shared_attn_workspace_bytes(T, R, S, H, cache->Hk, cache->d, max_shared, max_own);
  if (int rc = check_workspace(fn, a, need)) return rc;
  if (T == 0) return BBM_OK;
  if (int rc = check_apart(fn, {o->ptr, lse, need > 0 ? workspace : nullptr},
                           {q->ptr, cu, lens, block_table, mask, cache->k, cache->k_scale, cache->v, cache->v_scale, S > 0 ? group_cu : nullptr, S > 0 ? shared_lens : nullptr}))
    return rc;
  Kv4AttnParams P = params_of(a);
  const SharedPlan p = shared_plan_of(T, R, S, P.G, cache->Hk, cache->d, std::min<int64_t>(max_shared, kMaxTokens), std::min<int64_t>(max_own, kMaxTokens));
  for (const Plan& x : {p.group, p.own})
    if (x.pieces >= kMaxWgs || x.pieces * cache->Hk * std::max<int64_t>(x.parts, 1) >= kMaxWgs / 2)
      return fail(BBM_EUNSUPPORTED, "%s: problem too large (T=%lld, R=%lld, H=%lld)", fn, (long long)T, (long long)R, (long long)H);
  if (count_pieces(T, R, P.G, 4) * cache->Hk >= kMaxWgs) return fail(BBM_EUNSUPPORTED, "%s: problem too large (T=%lld, R=%lld, H=%lld)", fn, (long long)T, (long long)R, (long long)H);
  P.width = p.own.width, P.pieces = (int32_t)p.own.pieces, P.parts = (int32_t)p.own.parts, P.part_keys = (int32_t)p.own.part_keys;
  P.S = p.apart ? 0 : (int32_t)S, P.group_cu = group_cu, P.shared_lens = shared_lens;
  P.group_pieces = (int32_t)p.group.pieces, P.group_parts = (int32_t)p.group.parts, P.group_part_keys = (int32_t)p.group.part_keys;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (cache->d == 64) launch_shared<64>(P, p, s);
  else launch_shared<128>(P, p, s);
  return launch_status(fn);
}
