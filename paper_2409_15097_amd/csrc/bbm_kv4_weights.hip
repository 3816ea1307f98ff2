// Weights that the keys of the 4-bit cache gather (include/bbm_cache.h): out = decay * weights + the sum of exp(scale <q, k> - lse) over the queries that see a key.
//
// A work-group owns its keys: no sums pass between work-groups, and nothing depends on an order.  The queries of a request (of a group, for its shared keys) and a key head are
// columns: column c is query token c / G, head c % G of the group.
// Narrow, for few columns: bound by the cache's bytes (half of the attention's, values are not read: 17/32 byte an element, and 8 a key).  A wave takes 64 keys at a time, the next ones
// under way while these are used, and 16 columns: S = K Q^T by 16 keys x 16 columns x 32 elements an instruction; lane (n, q) = (l % 16, l / 16) loads D / 4 elements of key n from
// q * D / 4 on, and of column n likewise, and has the scores of keys 4 q .. 4 q + 3 with column n.
// Wide, for many: bound by the exponentials and the products.  A work-group takes 128 keys, whose codes are converted once into operands in registers, and walks tiles of 64 columns
// through LDS; a wave has 32 of the keys and 32 columns of every tile.
// Either way a lane adds up the exponentials of its column, and lanes meet once, behind the last column.
// Measured, 32 / 8 heads of 128: one token each of 64 requests of 4 to 8 thousand keys (240 MB), narrow, 60 us, 4.0 TB/s (a large copy reaches 5.2); prompts of 1500, 420 and 839 tokens over up
// to 6000 keys, wide, 143 us, 0.74 PFLOP/s (a large product 1.26; the vector pipe is busy for 55 % of the cycles, the matrix pipe for 30: a tile's products stand in front of its exponentials).
// Heads of 64, the same requests of one token, 133 MB: 46 us, 2.9 TB/s: what a wave does for a key does not shrink with its bytes.
#include "bbm_cache.h"
#include "bbm_kv4.h"
#include "bbm_prompt.h"

#include <algorithm>

namespace {

using bbm::bf16x8, bbm::f32x16, bbm::Kv4, bbm::scalar;
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr int NW = 8;
constexpr int NB = 4;                // blocks of 16 keys that a wave of the narrow kernel has
constexpr int kStep = 16 * NB * NW;  // keys of its work-group's step
constexpr int kWideKeys = 128, kWideCols = 64;

struct WeightParams {
  Kv4 c;
  const __bf16* q;
  const uint32_t* lse;  // (its bits)
  const float* weights;
  float* out;
  int64_t q_row, q_head, table_stride;
  const int32_t *cu, *lens, *table, *group_cu, *shared_lens;
  const uint64_t* mask;
  int32_t T, R, S, G, max_pages, mask_words;
  int32_t group_parts, own_parts;  // work-groups of a group and key head, of a request and key head
  int32_t group_wgs, own_wgs;      // of all of them in this launch (the groups' come first)
  int32_t tile_tokens, tile_heads; // of the wide kernel: what the columns of a tile are
  float rc, decay;                 // softmax_scale * log2(e)
};

typedef bbm::InPlace<WeightParams> Args;

// Whose keys a work-group has, and who looks at them.
struct Owner {
  int r;            // row of the block table
  int begin, end;   // rows of the queries
  int from, len;    // its keys
  int prefix;       // keys in front of the new tokens (causal: of the first one that has a row here)
  int fresh;        // from this key on, new tokens
};
__device__ __forceinline__ int max_keys(Args P) { return (int)min((int64_t)P->max_pages << P->c.page_shift, (int64_t)0x7fffffff); }
// The keys that a group shares, in whole pages: a page shared in part is another one for each request, since requests go on in it, and what is left over lies there for each of them.
__device__ __forceinline__ int shared_keys(Args P, int keys) { return max(0, min(keys, max_keys(P))) & ~(P->c.page - 1); }
__device__ __forceinline__ int row_cut(Args P, int c) { return min(max(c, 0), P->T); }
__device__ __forceinline__ int request_cut(Args P, int g) { return min(max(bbm::global(P->group_cu)[g], 0), P->R); }
__device__ __forceinline__ Owner owner_of_group(Args P, int g) {
  const int r0 = request_cut(P, g), r1 = request_cut(P, g + 1), shared = (int)scalar(bbm::global(P->shared_lens)[g]);
  Owner x;
  x.begin = (int)scalar(row_cut(P, bbm::global(P->cu)[r0])), x.end = (int)scalar(row_cut(P, bbm::global(P->cu)[r1]));
  x.r = min((int)scalar(r0), P->R - 1);
  x.from = 0;
  x.len = x.prefix = x.fresh = shared_keys(P, shared);
  return x;
}
__device__ __forceinline__ Owner owner_of_request(Args P, int r) {
  const bbm::Group shared = bbm::group_of(bbm::global(P->group_cu), bbm::global(P->shared_lens), P->S, r);  // (one trip to memory for all that is known of a request)
  const int c0 = (int)scalar(bbm::global(P->cu)[r]), c1 = (int)scalar(bbm::global(P->cu)[r + 1]), len = (int)scalar(bbm::global(P->lens)[r]);
  Owner x;
  x.r = r;
  x.begin = row_cut(P, c0), x.end = row_cut(P, c1);
  x.fresh = (int)((uint32_t)len - (uint32_t)max(0, c1 - c0));
  x.prefix = bbm::global(P->mask) ? x.fresh : (int)((uint32_t)x.fresh + (uint32_t)x.begin - (uint32_t)c0);
  x.len = max(0, min(len, max_keys(P)));
  x.from = min(shared_keys(P, shared.keys), x.len);
  return x;
}

// Which keys a work-group begins with, and how far the next ones are.
struct Share {
  Owner x;
  int hk, part, parts, cols;
};
// Of up to 64 owners number `at` in the order of their work (queries times keys), the most first: the longest prompt's work-groups are not to be the last ones that start.
__device__ __forceinline__ int by_work(Args P, bool group, int owners, int at) {
  if (owners > 64 || owners == 1) return at;
  const int lane = threadIdx.x & 63, o = min(lane, owners - 1);
  const int r0 = group ? request_cut(P, o) : o, r1 = group ? request_cut(P, o + 1) : o + 1;
  const int rows = max(0, row_cut(P, bbm::global(P->cu)[r1]) - row_cut(P, bbm::global(P->cu)[r0])), keys = max(0, group ? bbm::global(P->shared_lens)[o] : bbm::global(P->lens)[o]);
  const float work = lane < owners ? (float)rows * (float)keys : -1.0f;
  int rank = 0;
  for (int j = 0; j < owners; ++j) {
    const float other = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(work), j));
    rank += other > work || (other == work && j < lane);
  }
  return min(__ffsll((unsigned long long)__ballot(lane < owners && rank == at)) - 1, owners - 1);
}

// Of the wide kernel an owner's work-groups lie one behind the other, those of a key head on one XCD, whose cache holds their queries (all of a request on one XCD: three prompts of 1500,
// 420 and 839 tokens were on a third of the chip each, and took 254 us; in the order of the requests instead of their work, 168).
template <bool WIDE>
__device__ __forceinline__ Share share_of(Args P, bool group) {
  const int wg = (int)blockIdx.x - (group ? 0 : P->group_wgs);
  Share y = {};
  y.parts = group ? P->group_parts : P->own_parts;
  int owner;
  if (WIDE) {
    const int owners = group ? P->S : P->R, each = 8 * P->c.Hk * ((y.parts + 7) / 8), at = wg / each;
    const bbm::Work w = bbm::work_of(wg - at * each, P->c.Hk);
    y.hk = w.plane, y.part = w.number;
    if (y.part >= y.parts) return y;
    owner = by_work(P, group, owners, at);
  } else {
    const int rest = wg / y.parts;
    y.part = wg % y.parts, y.hk = rest % P->c.Hk, owner = rest / P->c.Hk;
  }
  y.x = group ? owner_of_group(P, owner) : owner_of_request(P, owner);
  y.cols = max(0, y.x.end - y.x.begin) * P->G;
  return y;
}

// A column, and where its query and its log-sum-exp lie; `ahead` columns further, cut to (tokens, heads).
struct Column {
  int col, i, g;
  const __bf16* q;
  const uint32_t* lse;  // its bits
};
struct Stride {
  int cols, i, g;
};
__device__ __forceinline__ Stride stride_of(Args P, int cols) { return {cols, cols / P->G, cols % P->G}; }
__device__ __forceinline__ Column column_of(Args P, const __bf16* q0, const uint32_t* lse0, int c) {
  Column y;
  y.col = c, y.i = c / P->G, y.g = c - y.i * P->G;
  y.q = q0 + y.i * P->q_row + y.g * P->q_head;
  y.lse = lse0 + (int64_t)y.g * P->T + y.i;
  return y;
}
__device__ __forceinline__ void advance(Args P, Column& y, const Stride& s) {
  y.col += s.cols, y.i += s.i;
  y.q += s.i * P->q_row + s.g * P->q_head;
  y.lse += (int64_t)s.g * P->T + s.i;
  if (s.g != 0) {  // (of a group of 1, 2, 4 .. heads the head stays)
    y.g += s.g;
    const bool over = y.g >= P->G;
    y.g -= over ? P->G : 0, y.i += over;
    y.q += over ? P->q_row - P->G * P->q_head : 0;
    y.lse += over ? 1 - (int64_t)P->G * P->T : 0;
  }
}
// A row that saw nothing, whose log-sum-exp is -infinity, gives nothing.  (That is told from the bits as they lie in memory: as floats the compiler takes all for numbers.)
__device__ __forceinline__ bool gives_nothing(uint32_t lse) { return lse == 0xff800000u; }
__device__ __forceinline__ float minus_lse(uint32_t lse) { return gives_nothing(lse) ? -INFINITY : __uint_as_float(lse) * -kLog2e; }
// Which of the keys from j on the new token of a column sees.
__device__ __forceinline__ uint64_t seen_by(Args P, const Owner& x, int i, int j) {
  i = min(i, x.end - x.begin - 1);
  return bbm::seen_from(bbm::global(P->mask) ? bbm::global(P->mask) + (int64_t)(x.begin + i) * P->mask_words : nullptr, P->mask_words, i, j - x.prefix);
}

template <int D>
__device__ __forceinline__ void narrow(Args P, const Share& own) {
  constexpr int KS = D / 32;  // steps of a product, and words of codes that a lane loads of a key
  const int lane = threadIdx.x & 63, n = lane & 15, kq = lane >> 4;
  const int wave = (int)scalar(threadIdx.x >> 6);
  const Owner& x = own.x;
  const int hk = own.hk, cols = own.cols;
  if (cols == 0) return;

  struct Raw {
    uint32_t k[NB][KS], ks[NB];
    f32x4 old;       // of the four keys that this lane writes: 4 kq .. of block n (n < NB)
    int64_t place;   // where they lie
    int have;        // how many of them are there
  };
  const bbm::Table table = (bbm::Table)(uintptr_t)(bbm::global(P->table) + x.r * P->table_stride);
  struct Pages {
    int p[NB];
  };
  auto pages_at = [&](int j) __attribute__((always_inline)) {
    Pages y;
#pragma unroll
    for (int b = 0; b < NB; ++b) y.p[b] = table[scalar(min(j + 16 * b, x.len - 1) >> P->c.page_shift)];
    return y;
  };
  // the wave's 64 keys from j on; of those that are not there zeros, and of the weights the cache's first
  auto load = [&](Raw& z, int j, const Pages& pages, const float* weights) __attribute__((always_inline)) {
    z.have = 0;
    z.place = 0;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int jb = j + 16 * b, page = pages.p[b];
      const bool there = jb < x.len && page >= 0 && page < P->c.pages;
      const int64_t key = ((int64_t)page * P->c.Hk + hk) * P->c.page + (jb & (P->c.page - 1));
      const __amdgpu_buffer_rsrc_t k_r = bbm::buffer_of(bbm::global(P->c.k) + key * (D / 2), there ? 16 * (D / 2) : 0), ks_r = bbm::buffer_of(bbm::global(P->c.k_scale) + key * (D / 32), there ? D / 2 : 0);
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
    z.old = *reinterpret_cast<const f32x4*>(weights + z.place);
  };
  auto store = [&](const Raw& z, int j, f32x4 (&sum)[NB], float keep, int fresh_from) __attribute__((always_inline)) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) sum[b][r] = bbm::row_sum<16>(sum[b][r]);
    f32x4 y = n == 0 ? sum[0] : n == 1 ? sum[1] : n == 2 ? sum[2] : sum[3];
    const int fresh = fresh_from - (j + 16 * n + 4 * kq);  // how many of the four were there before
#pragma unroll
    for (int r = 0; r < 4; ++r) y[r] += r < fresh ? keep * z.old[r] : 0.0f;
    if (z.have == 4) {
      *reinterpret_cast<f32x4*>(bbm::global(P->out) + z.place) = y;
    } else {
#pragma unroll
      for (int r = 0; r < 3; ++r)
        if (r < z.have) bbm::global(P->out)[z.place + r] = y[r];
    }
  };

  const __bf16* const q0 = bbm::global(P->q) + (int64_t)x.begin * P->q_row + (int64_t)hk * P->G * P->q_head + kq * (D / 4);
  const uint32_t* const lse0 = bbm::global(P->lse) + (int64_t)hk * P->G * P->T + x.begin;
  struct Query {
    bf16x8 q[KS];
    float nl;  // what is added to its exponents
  };
  // (columns behind the last read the first one's query, and add nothing: a zero's product and -infinity give nothing whatever the query holds, as for a row that saw nothing)
  auto fetch = [&](const Column& y) __attribute__((always_inline)) {
    Query z;
    const bool there = y.col < cols;
    const __bf16* const p = there ? y.q : q0;
    const uint32_t l = *(there ? y.lse : lse0);
    const bool nothing = !there || gives_nothing(l);
    z.nl = nothing ? -INFINITY : minus_lse(l);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const bbm::u32x4 w = *reinterpret_cast<const bbm::u32x4*>(p + 8 * s);
      z.q[s] = __builtin_bit_cast(bf16x8, nothing ? bbm::u32x4{} : w);
    }
    return z;
  };
  // 64 keys from j on with 16 columns; all_see: the last key that all of them see
  auto use = [&](const Raw& a, f32x4 (&sum)[NB], const Query& z, const Column& y, int j, int all_see) __attribute__((always_inline)) {
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      f32x4 s = f32x4{0.0f, 0.0f, 0.0f, 0.0f}, p;
#pragma unroll
      for (int i = 0; i < KS; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bbm::values_of(a.k[b][i], bbm::scale_of(a.ks[b])), z.q[i], s, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], P->rc, z.nl));
      if (j + 16 * b + 15 > all_see) {
        const uint32_t seen = (uint32_t)seen_by(P, x, y.i, j + 16 * b + 4 * kq);
#pragma unroll
        for (int r = 0; r < 4; ++r) p[r] = seen >> r & 1 ? p[r] : 0.0f;
      }
      sum[b] = p;
    }
  };

  const int j0 = x.from + own.part * kStep + wave * (16 * NB), next = own.parts * kStep;
  if (j0 >= x.len) return;
  Column y = column_of(P, q0, lse0, n);
  const Stride ahead = stride_of(P, 16);
  // 16 columns at a time over all keys; those behind the first 16 are added to what was stored.
#pragma unroll 1
  for (int c = 0; c < cols; c += 16) {
    const Query z = fetch(y);
    const int all_see = P->mask ? x.prefix - 1 : x.prefix + c / P->G;
    const float* const old = c == 0 ? bbm::global(P->weights) : bbm::global(P->out);
    const float keep = c == 0 ? P->decay : 1.0f;
    const int fresh = c == 0 ? x.fresh : x.len;
    auto step = [&](const Raw& a, int j) __attribute__((always_inline)) {
      f32x4 sum[NB];
      use(a, sum, z, y, j, all_see);
      store(a, j, sum, keep, fresh);
    };
    // the next keys are asked for before these are used, their pages a step before that
    Raw a, b;
    int j = j0;
    load(a, j, pages_at(j), old);
    Pages pages = pages_at(j + next);
#pragma unroll 1
    for (;;) {
      load(b, j + next, pages, old);
      pages = pages_at(j + 2 * next);
      step(a, j);
      j += next;
      if (j >= x.len) break;
      load(a, j + next, pages, old);
      pages = pages_at(j + 2 * next);
      step(b, j);
      j += next;
      if (j >= x.len) break;
    }
    advance(P, y, ahead);
  }
}

template <int D>
__device__ __forceinline__ void wide(Args P, const Share& own) {
  using L = bbm::TL<D>;
  constexpr int KS = D / 16, RC = D / 8;
  constexpr int ROWS = 64 * NW / RC, PIECES = kWideCols / ROWS;  // rows of a tile that the threads fetch at a time
  __shared__ __attribute__((aligned(16))) __bf16 q_s[2][L::ELEMS];
  __shared__ float sum_s[2][kWideKeys];
  const int tid = threadIdx.x, lane = tid & 63, lq = lane & 31, hh = lane >> 5;
  const int wave = (int)scalar(tid >> 6), key_part = wave >> 1, col_half = wave & 1;
  const Owner& x = own.x;
  const int hk = own.hk;
  if (own.cols == 0) return;
  const int32_t* const table = bbm::global(P->table) + x.r * P->table_stride;
  bbm::TileAddr<D> A;
  A.init(lane);
  // the slot of a key in what has a number for each token and head, -1 if it is not there
  auto slot_of = [&](int j) -> int64_t {
    const int page = table[min(j, x.len - 1) >> P->c.page_shift];
    return j < x.len && page >= 0 && page < P->c.pages ? (((int64_t)page * P->c.Hk + hk) << P->c.page_shift) + (j & (P->c.page - 1)) : -1;
  };

  // A tile's columns are `heads` heads of `tokens` tokens, side by side (of 64 columns those behind them are not used, and repeat the first one): what a thread fetches of a tile lies
  // at the same distance from the tile's first query every time.
  const int tokens = P->tile_tokens, heads = P->tile_heads, n = x.end - x.begin, G = P->G;
  const int64_t q_row = P->q_row, q_head = P->q_head;
  const float rc = P->rc;
  const bool masked = P->mask != nullptr;
  uint32_t off[PIECES];
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    const int c = tid / RC + ROWS * p, t = c / heads;
    off[p] = (uint32_t)((t < tokens ? t * q_row + (c - t * heads) * q_head : 0) + tid % RC * 8) * 2u;
  }
  const int c = 32 * col_half + lq;
  const bool used = c < tokens * heads;
  const int my_t = used ? c / heads : 0, my_h = used ? c - my_t * heads : 0;
  const uint32_t* const lse0 = bbm::global(P->lse) + (int64_t)hk * G * P->T + x.begin;
  const int64_t my_lse = (int64_t)my_h * P->T + my_t;
  const __bf16* const q0 = bbm::global(P->q) + (int64_t)x.begin * q_row + (int64_t)hk * G * q_head;
  struct Tile {
    int i, h;  // its first token and head
  };
  auto after = [&](Tile t) __attribute__((always_inline)) {
    t.h += heads;
    if (t.h >= G) t.h = 0, t.i += tokens;
    return t;
  };

#pragma unroll 1
  for (int j0 = x.from + own.part * kWideKeys; j0 < x.len; j0 += own.parts * kWideKeys) {
    // (a causal key is seen by no token in front of its own)
    Tile now = {masked ? 0 : min(max(0, j0 - x.prefix), n - 1) / tokens * tokens, 0}, next = now;
    bf16x8 staged[PIECES];
    uint32_t l;
    auto fetch = [&]() __attribute__((always_inline)) {  // (of tokens and heads that are not there: zeros, or what lies between those that are)
      const int ts = min(tokens, n - next.i), hs = min(heads, G - next.h);
      const __amdgpu_buffer_rsrc_t r = bbm::buffer_of(q0 + next.i * q_row + next.h * q_head, ts > 0 ? (int)(((ts - 1) * q_row + (hs - 1) * q_head + D) * 2) : 0);
#pragma unroll
      for (int p = 0; p < PIECES; ++p) staged[p] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(r, off[p], 0, 0));
      l = lse0[my_t < ts && my_h < hs ? my_lse + (int64_t)next.h * P->T + next.i : 0];
      next = after(next);
    };
    auto put = [&](__bf16* dst) __attribute__((always_inline)) {
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        const int r = tid / RC + ROWS * p;
        *reinterpret_cast<bf16x8*>(dst + r % L::NBLK * L::TBLK + r / L::NBLK * D + (tid % RC ^ (r >> 2 & 3)) * 8) = staged[p];
      }
    };
    // A tile is asked for two steps before it is used, and goes to LDS one step before.
    fetch();
    // This wave's keys as operands: lane (l % 32, l / 32) has elements 16 t + 8 (l / 32) .. of key l % 32; and the key that this thread writes.  (What is read for one that is not there,
    // the cache's first, is left out of what is written.)
    const int64_t mine = slot_of(j0 + 32 * key_part + lq), place = tid < kWideKeys ? slot_of(j0 + tid) : -1;
    const int64_t from = max(mine, (int64_t)0);
    const uint32_t* const codes = reinterpret_cast<const uint32_t*>(bbm::global(P->c.k) + from * (D / 2)) + hh;
    uint32_t w[KS], scales;
#pragma unroll
    for (int t = 0; t < KS; ++t) w[t] = codes[2 * t];
    if constexpr (D == 128) scales = *reinterpret_cast<const uint32_t*>(bbm::global(P->c.k_scale) + from * 4);
    else scales = *reinterpret_cast<const uint16_t*>(bbm::global(P->c.k_scale) + from * 2);
    const float held = bbm::global(P->weights)[max(place, (int64_t)0)], old = j0 + tid < x.fresh ? P->decay * held : 0.0f;
    bf16x8 k[KS];
#pragma unroll
    for (int t = 0; t < KS; ++t) k[t] = bbm::values_of(w[t], bbm::scale_of(scales >> (8 * (t / 2)) & 0xff));
    f32x16 sum;
    for (int e = 0; e < 16; ++e) sum[e] = 0.0f;

    put(q_s[0]);
    uint32_t l_now = l;
    fetch();
    int buf = 0;
#pragma unroll 1
    for (; now.i < n; now = after(now), buf ^= 1) {
      const bool nothing = gives_nothing(l_now);  // (what that costs: 2 to 4 %; sums that are added up again where one is no number took 1 % less of these prompts, and 4 % more of 64 tokens each)
      const float nl = used ? minus_lse(l_now) : -INFINITY;
      __syncthreads();  // the tile is there, and everyone is done with the other buffer
      const __bf16* const tile = q_s[0] + buf * L::ELEMS;
      f32x16 s;
      for (int e = 0; e < 16; ++e) s[e] = 0.0f;
#pragma unroll
      for (int t = 0; t < KS; ++t) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[t], A.row_frag(tile, col_half, t), s, 0, 0, 0);
      put(q_s[0] + (buf ^ 1) * L::ELEMS);
      l_now = l;
      fetch();
      const int j = j0 + 32 * key_part, all_see = masked ? x.prefix - 1 : x.prefix + now.i;
      // (A row that saw nothing may hold no number, which times nothing is none; so may the first one, which columns that are not used repeat, but then all that it sees has none.)
      if (j + 31 <= all_see && now.i + tokens <= n && now.h + heads <= G && !__any(nothing)) {
#pragma unroll
        for (int e = 0; e < 16; ++e) sum[e] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], rc, nl));
      } else {
        const bool there = used && !nothing && now.i + my_t < n && now.h + my_h < G;
        const uint32_t seen = (there ? (uint32_t)seen_by(P, x, now.i + my_t, j) : 0) >> (4 * hh);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], rc, nl));
          sum[e] += seen >> (8 * (e / 4) + e % 4) & 1 ? p : 0.0f;
        }
      }
    }
    // over the columns: 32 lanes, then the two waves of the same keys
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float y = bbm::row_sum<16>(sum[e]);
      const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(y), __float_as_uint(y), false, false);
      const float both = __uint_as_float(r[0]) + __uint_as_float(r[1]);
      if (lq == 0) sum_s[col_half][32 * key_part + 8 * (e / 4) + 4 * hh + e % 4] = both;
    }
    __syncthreads();
    if (place >= 0) bbm::global(P->out)[place] = sum_s[0][tid] + sum_s[1][tid] + old;
    __syncthreads();
  }
}

template <int D, bool WIDE>
__global__ __launch_bounds__(64 * NW, 4) void kv4_weights_kernel(const WeightParams) {
  Args P = bbm::kernel_args<WeightParams>();
  const Share own = share_of<WIDE>(P, (int)blockIdx.x < P->group_wgs);
  if constexpr (WIDE) wide<D>(P, own);
  else narrow<D>(P, own);
}
// The groups' keys have many columns, the requests' few: both side by side.
template <int D>
__global__ __launch_bounds__(64 * NW, 4) void kv4_weights_both_kernel(const WeightParams) {
  Args P = bbm::kernel_args<WeightParams>();
  if ((int)blockIdx.x < P->group_wgs) wide<D>(P, share_of<true>(P, true));
  else narrow<D>(P, share_of<false>(P, false));
}

// Work-groups of an owner: of the narrow kernel enough to fill the chip, of the wide one as many as it has pieces (a launch counts threads in 32 bits: of many owners or a long table fewer,
// which then take several pieces each).
constexpr int64_t kFill = 512, kMaxParts = 1 << 17, kMaxOwners = 1 << 19, kMaxWideWgs = 1 << 21;  // (two steps of kMaxParts behind a key are still a 32-bit number)
inline int64_t parts_of(int64_t owners, int64_t Hk, int64_t keys, bool wide) {
  keys = std::min<int64_t>(keys, bbm::kMaxTokens);
  if (!wide) return std::min(bbm::ceil_div(keys, kStep), bbm::ceil_div(kFill, owners * Hk));
  return std::min({bbm::ceil_div(keys, kWideKeys), kMaxParts, std::max<int64_t>(8, kMaxWideWgs / (owners * Hk) / 8 * 8)});
}
// Columns of an owner, on average, from which on its codes are converted once.  32 / 8 heads of 128, us, narrow / wide: one request of 8192 keys, 16 columns 6.1 / 10.1, 32 8.8 / 10.4, 48
// 11.8 / 10.5, 64 14.5 / 9.9, 256 50 / 15; a group behind 8192 keys, 32 columns 8.9 / 13.9, 64 15.0 / 13.7, 268 53 / 25; heads of 64 alike (32 8.5 / 8.1, 48 11.3 / 8.2; 32 8.5 / 11.6, 64 13.9 / 11.2).
// That is the border for few owners.  Of many the wide kernel's work-groups, one for every 128 keys, cost more than their columns do: 16 requests of 2048 to 4096 keys, 32 columns 21 / 63, 48
// 29 / 64, 64 36 / 61, 128 68 / 69, 256 127 / 84; 64 of 1024 to 2048, 64 columns 56 / 151, 256 199 / 202.
constexpr int64_t kWideFrom = 32;

template <int D>
void launch(const WeightParams& P, bool group_wide, bool own_wide, hipStream_t s) {
  const unsigned wgs = (unsigned)(P.group_wgs + P.own_wgs);
  if (own_wide) kv4_weights_kernel<D, true><<<wgs, 64 * NW, 0, s>>>(P);
  else if (group_wide) kv4_weights_both_kernel<D><<<wgs, 64 * NW, 0, s>>>(P);
  else kv4_weights_kernel<D, false><<<wgs, 64 * NW, 0, s>>>(P);
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
  if (T * G > kMaxTokens || R * cache->Hk >= kMaxOwners) return fail(BBM_EUNSUPPORTED, "%s: problem too large (T=%lld, R=%lld, H=%lld)", fn, (long long)T, (long long)R, (long long)H);
  if (T == 0) return BBM_OK;
  if (int rc = check_apart(fn, {out}, {q->ptr, lse, cu, lens, block_table, mask, cache->k, cache->k_scale, S > 0 ? group_cu : nullptr, S > 0 ? shared_lens : nullptr})) return rc;
  WeightParams P = {};
  P.c = kv4_of(cache);
  P.q = static_cast<const __bf16*>(q->ptr), P.lse = reinterpret_cast<const uint32_t*>(lse), P.weights = weights, P.out = out;
  P.q_row = q->row_stride, P.q_head = q->head_stride, P.table_stride = table_stride;
  P.cu = cu, P.lens = lens, P.table = block_table, P.group_cu = group_cu, P.shared_lens = shared_lens, P.mask = mask;
  P.T = (int32_t)T, P.R = (int32_t)R, P.S = (int32_t)S, P.G = (int32_t)G, P.max_pages = (int32_t)max_pages, P.mask_words = (int32_t)mask_words;
  P.rc = softmax_scale * kLog2e, P.decay = decay;
  const bool own_wide = T * G > kWideFrom * R, group_wide = S > 0 && T * G > kWideFrom * S;  // (of the requests only if of the groups, S <= R)
  const int64_t group_parts = S > 0 ? parts_of(S, cache->Hk, max_shared, group_wide) : 1, own_parts = parts_of(R, cache->Hk, max_own, own_wide);
  auto count = [&](int64_t owners, int64_t parts, bool wide) { return owners * (wide ? work_groups(cache->Hk, parts) : cache->Hk * parts); };
  const int64_t group_wgs = count(S, group_parts, group_wide), own_wgs = count(R, own_parts, own_wide);
  // (heads of a tile that a buffer's 31 bits reach: of rows up to 2^22 elements apart 64 tokens are within 2^29 bytes)
  const int64_t reach = q->head_stride > 0 ? 1 + (1ll << 29) / q->head_stride : kWideCols;
  P.tile_heads = (int32_t)std::min({G, (int64_t)kWideCols, reach}), P.tile_tokens = kWideCols / P.tile_heads;
  P.group_parts = (int32_t)group_parts, P.own_parts = (int32_t)own_parts, P.group_wgs = (int32_t)group_wgs, P.own_wgs = (int32_t)own_wgs;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (cache->d == 64) launch<64>(P, group_wide, own_wide, s);
  else launch<128>(P, group_wide, own_wide, s);
  return launch_status(fn);
}
