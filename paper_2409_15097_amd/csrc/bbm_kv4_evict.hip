// Eviction from the 4-bit cache by the weights that its keys gathered (include/bbm_cache.h).
//
// A work-group takes a request and a key head: it finds the smallest weight that stays by counting (11, 11 and 10 bits of the weights as ordered integers, each pass over those that
// agree with the bits before), writes down which of the places that remain become free, a bit each, in LDS, and moves: a kept key from behind finds the place of its number by
// bisection over the counts of 64 places, then by counting bits.  Where the moves of the first kind end they read nothing that they write, so their order does not matter; the last
// keys are shifted by whole rounds of all waves, with a barrier between a round's loads and its stores, in ascending order.
// The pages go back by a wave for each request, behind the sum of what the requests in front of it give: of up to 256 requests in one more work-group, else by a second kernel.
// Measured on caches that nothing has thinned (a second call on the same keys and weights finds most of the chosen ones in front, and moves half as many).  Bound by latency: 1040 keys to
// 1024, 4 heads of 64, 11.5 us, 64 requests of up to 2112 keys to 2048, 8 heads of 128, 17; 16 requests of up to 32000 keys to 4000, 118 us, 1.2 TB/s of what has to move, 4 such requests
// 108: a work-group takes 100 us, of which reading the weights is 18, the rest of the choice 7, places 7, the moves of 3000 keys and the last 500 67.  (250 with weights read from memory in every
// pass and pages given back by a second launch; 140 with the pages from memory.)  One request of 100 thousand keys to 8000, whose weights do not fit into LDS, 382 us.
#include "bbm_cache.h"
#include "bbm_kv4.h"

#include <algorithm>

namespace {

using bbm::Kv4, bbm::scalar;

constexpr int NT = 1024, NWAVES = NT / 64;
constexpr int kBins = 2048;
constexpr int kGiveTogether = 256;  // requests whose pages one work-group gives back, while the others move keys
constexpr int64_t kMaxBudget = 1 << 19;  // places that are bits and counts in LDS: 96 KiB
// Of the 160 KiB of a CU's LDS: what a work-group may ask for without more, and what two and one of them may have beside 17 KiB of bins, sums and moves.
constexpr int64_t kPlain = 44 << 10, kTwo = 62 << 10, kOne = 140 << 10;

struct EvictParams {
  Kv4 c;
  float* weights;
  const int32_t *lens, *table, *first, *free_at;
  int32_t *new_lens, *free_pages, *free_next;
  int32_t* given;  // [R] pages that a request gives back; NULL if the first work-group sees to them
  int64_t table_stride, n_free;
  int32_t R, max_keys, budget, recent;
  int32_t held, held_pages;  // keys whose weights, and entries of the table, that LDS has room for
};

// What stays of a request: keys f .. f + between - 1 are chosen from, `chosen` of them stay.
struct Cut {
  int n, b, f, edge, between, chosen;
};
__device__ __forceinline__ Cut cut_of(const EvictParams& P, int r) {
  Cut x;
  x.n = max(0, min(P.lens[r], P.max_keys));
  const int f = P.first ? max(0, P.first[r]) : 0;
  const int64_t b = max((int64_t)P.budget, (int64_t)f + P.recent);
  x.b = (int)min(b, (int64_t)x.n);
  x.f = min(f, x.n);
  x.edge = x.b - P.recent;  // (of use if x.n > x.b, as are the others)
  x.between = x.n - P.recent - x.f;
  x.chosen = x.edge - x.f;
  return x;
}

__device__ __forceinline__ int wave_sum(int x) { return __builtin_amdgcn_readlane(bbm::wave_prefix_sum(x), 63); }

// By a wave: the pages that request r gives back; those, behind the `before` of `all` that the requests in front of it give, and the request's length.
__device__ __forceinline__ int pages_given(const EvictParams& P, int r) {
  const Cut x = cut_of(P, r);
  const int32_t* const table = P.table + r * P.table_stride;
  int count = 0;
  for (int at = ((x.b + P.c.page - 1) >> P.c.page_shift) + (threadIdx.x & 63); at < (x.n + P.c.page - 1) >> P.c.page_shift; at += 64) count += table[at] >= 0 && table[at] < P.c.pages;
  return wave_sum(count);
}
__device__ __forceinline__ void give(const EvictParams& P, int r, int before, int all) {
  const int lane = threadIdx.x & 63;
  const Cut x = cut_of(P, r);
  if (P.free_at) {
    const int64_t first = min((int64_t)*P.free_at, P.n_free) - all;  // (a list that was too short has nothing behind its end)
    if (r == 0 && lane == 0) *P.free_next = (int32_t)first;
    const int32_t* const table = P.table + r * P.table_stride;
    int64_t to = first + before;
    const int end = (x.n + P.c.page - 1) >> P.c.page_shift;
    for (int at = (x.b + P.c.page - 1) >> P.c.page_shift; at < end; at += 64) {
      const int page = at + lane < end ? table[at + lane] : -1;
      const uint64_t real = __ballot(page >= 0 && page < P.c.pages);
      const int64_t mine = to + __popcll(real & ((1ull << lane) - 1ull));
      if ((real >> lane & 1) && mine >= 0 && mine < P.n_free) P.free_pages[mine] = page;
      to += __popcll(real);
    }
  }
  if (lane == 0) P.new_lens[r] = x.b;
}

// Weights as integers of the same order; a NaN is 1, a key without a page 0.
__device__ __forceinline__ uint32_t ordered(uint32_t bits) {
  if ((bits & 0x7fffffffu) > 0x7f800000u) return 1u;
  if (bits == 0x80000000u) bits = 0u;
  return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}

template <int D>
__global__ __launch_bounds__(NT) void kv4_evict_kernel(const EvictParams P) {
  // free places, a bit each, 64 a word; the number of those in front of each word; the request's pages (P.held_pages); the weights of the keys between (P.held of them)
  extern __shared__ __attribute__((aligned(16))) uint32_t dynamic_s[];
  __shared__ int wave_s[3][NWAVES];
  __shared__ uint32_t found_s[3][3];         // of each pass the bin, what is still to be chosen from it, what it holds
  __shared__ int2 moves_s[NWAVES][2 * 64];  // of a wave: from and to, as slots
  uint32_t* const bins = reinterpret_cast<uint32_t*>(moves_s);
  static_assert(sizeof(moves_s) >= kBins * sizeof(uint32_t) && sizeof(moves_s) >= kGiveTogether * sizeof(int), "bins, and pages of requests, lie in the place of moves");
  const int tid = threadIdx.x, lane = tid & 63, wave = (int)scalar(tid >> 6);
  const int wg = (int)blockIdx.x - (P.given ? 0 : 1);
  if (wg < 0) {
    int* const given_s = reinterpret_cast<int*>(moves_s);
    for (int r = wave; r < P.R; r += NWAVES) {
      const int n = P.free_at ? pages_given(P, r) : 0;
      if (lane == 0) given_s[r] = n;
    }
    __syncthreads();
    for (int r = wave; r < P.R; r += NWAVES) {
      int before = 0, all = 0;
      for (int i = lane; i < P.R; i += 64) all += given_s[i], before += i < r ? given_s[i] : 0;
      give(P, r, wave_sum(before), wave_sum(all));
    }
    return;
  }
  const int r = wg / P.c.Hk, hk = wg % P.c.Hk;
  const Cut x = cut_of(P, r);
  const int32_t* const table = P.table + r * P.table_stride;
  if (P.given && hk == 0 && wave == 0 && P.free_at) {
    const int n = pages_given(P, r);
    if (lane == 0) P.given[r] = n;
  }
  if (x.n <= x.b) return;

  const int words = (x.chosen + 63) / 64, pages = (x.n + P.c.page - 1) >> P.c.page_shift;
  uint64_t* const free_s = reinterpret_cast<uint64_t*>(dynamic_s);
  int* const before_s = reinterpret_cast<int*>(free_s + words);
  int32_t* const pages_s = before_s + words;
  const bool pages_held = pages <= P.held_pages;
  if (pages_held) {
    for (int i = tid; i < pages; i += NT) pages_s[i] = table[i];
    __syncthreads();
  }
  auto page_of = [&](int j) { return pages_held ? pages_s[j >> P.c.page_shift] : table[j >> P.c.page_shift]; };
  // the slot of a key in the cache, for all that has a number for each token and head; -1 if it has no page
  auto slot_of = [&](int j) -> int64_t {
    const int page = page_of(j);
    return page >= 0 && page < P.c.pages ? (((int64_t)page * P.c.Hk + hk) << P.c.page_shift) + (j & (P.c.page - 1)) : -1;
  };
  uint32_t* const held_s = reinterpret_cast<uint32_t*>(pages_s + P.held_pages);
  const bool held = x.between <= P.held;
  auto weight_in_memory = [&](int i) -> uint32_t {  // of key f + i
    const int64_t s = slot_of(x.f + i);
    return s < 0 ? 0u : ordered(__float_as_uint(P.weights[max(s, (int64_t)0)]));
  };
  auto weight_of = [&](int i) -> uint32_t { return held ? held_s[i] : weight_in_memory(i); };

  // What the waves in front of this one wrote down.
  auto in_front = [&](const int* of_waves) {
    const int v = lane < NWAVES ? of_waves[lane] : 0, sum = bbm::wave_prefix_sum(v);
    return wave > 0 ? __builtin_amdgcn_readlane(sum, max(wave - 1, 0)) : 0;
  };

  // The smallest weight that stays, and how many that equal it do.
  uint32_t low = 0, need = (uint32_t)x.chosen, equal = 0;
  if (x.chosen > 0) {
    constexpr int SHIFT[3] = {21, 10, 0}, BITS[3] = {11, 11, 10};
    for (int i = tid; i < kBins; i += NT) bins[i] = 0;
    __syncthreads();
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const uint32_t above = pass == 0 ? 0u : ~0u << (pass == 1 ? 21 : 10);
      auto count = [&](auto at_once) __attribute__((always_inline)) {
        constexpr int U = decltype(at_once)::value;  // so many loads of a thread under way
        for (int i0 = tid; i0 < x.between; i0 += U * NT) {
          uint32_t u[U];
#pragma unroll
          for (int n = 0; n < U; ++n) {
            const int i = min(i0 + n * NT, x.between - 1);
            u[n] = pass == 0 ? weight_in_memory(i) : weight_of(i);
          }
#pragma unroll
          for (int n = 0; n < U; ++n) {
            if (i0 + n * NT >= x.between) continue;
            if (pass == 0 && held) held_s[i0 + n * NT] = u[n];
            if (((u[n] ^ low) & above) == 0) atomicAdd(&bins[u[n] >> SHIFT[pass] & ((1u << BITS[pass]) - 1u)], 1u);
          }
        }
      };
      if (x.between <= 2 * NT) count(bbm::IntC<2>{});  // (of 1000 and up to 2112 keys with eight 17.3 and 20.1 us a call, with two 15.9 and 17.6)
      else count(bbm::IntC<8>{});
      __syncthreads();
      // two bins a thread, the highest first; who reads them clears them for the next pass
      uint2* const mine = reinterpret_cast<uint2*>(bins) + (NT - 1 - tid);
      const uint32_t c0 = mine->y, c1 = mine->x;
      *mine = make_uint2(0, 0);
      int sum = bbm::wave_prefix_sum((int)(c0 + c1));
      if (lane == 63) wave_s[0][wave] = sum;
      __syncthreads();
      sum += in_front(wave_s[0]);
      const uint32_t before = (uint32_t)sum - c0 - c1;
      if (before < need && need <= (uint32_t)sum) {
        const bool second = before + c0 < need;
        found_s[pass][0] = (uint32_t)(kBins - 1 - 2 * tid) - second;
        found_s[pass][1] = need - before - (second ? c0 : 0u);
        found_s[pass][2] = second ? c1 : c0;
      }
      __syncthreads();
      low |= found_s[pass][0] << SHIFT[pass];
      need = found_s[pass][1];
      equal = found_s[pass][2];
    }
  } else {
    low = ~0u;
  }

  // Each wave takes a stretch of the keys between.  Of those that equal the smallest the first `need` stay: how many lie in front of each stretch.
  const int blocks = (x.between + 63) / 64, per = (blocks + NWAVES - 1) / NWAVES, block0 = min(blocks, wave * per), block1 = min(blocks, block0 + per);
  int ties = 0;  // in front of this wave's
  if (equal > need) {
    int mine = 0;
    for (int k = block0; k < block1; ++k) {
      const int i = 64 * k + lane;
      mine += __popcll(__ballot(i < x.between && weight_of(min(i, x.between - 1)) == low));
    }
    if (lane == 0) wave_s[1][wave] = mine;
    __syncthreads();
    ties = in_front(wave_s[1]);
  }
  // f(block, which of its 64 keys stay) for the blocks of this wave from `from` on in order, the weights of four of them read together; before: the equal ones in front of the next block.
  auto for_kept = [&](int from, int& before, auto f) __attribute__((always_inline)) {
    constexpr int U = 4;
    for (int k0 = from; k0 < block1; k0 += U) {
      uint32_t u[U];
#pragma unroll
      for (int n = 0; n < U; ++n) u[n] = weight_of(min(64 * (k0 + n) + lane, x.between - 1));
#pragma unroll
      for (int n = 0; n < U; ++n) {
        if (k0 + n >= block1) continue;
        const bool in = 64 * (k0 + n) + lane < x.between && x.chosen > 0;
        uint64_t stay = __ballot(in && u[n] >= low);
        if (equal > need) {
          const uint64_t same = __ballot(in && u[n] == low);
          const int rank = before + __popcll(same & ((1ull << lane) - 1ull));
          stay &= ~__ballot(in && u[n] == low && rank >= (int)need);
          before += __popcll(same);
        }
        f(k0 + n, stay);
      }
    }
  };
  // Places: bit i of the first `chosen` is free if key f + i does not stay there.
  // The moves begin in the block where the places end, with what stays there and the equal ones behind it as they are now: weights in memory change under those who would read them again.
  const int edge_block = x.chosen / 64;
  uint64_t edge_stay = 0;
  int edge_ties = ties, before = ties;
  int behind = 0;  // kept ones of this wave's that have to move
  for_kept(block0, before, [&](int k, uint64_t stay) __attribute__((always_inline)) {
    if (k == edge_block) edge_stay = stay, edge_ties = before;
    const int left = x.chosen - 64 * k;  // places among these
    const uint64_t places = left >= 64 ? ~0ull : left <= 0 ? 0ull : (1ull << left) - 1ull;
    if (lane == 0 && places) free_s[k] = places & ~stay;
    behind += __popcll(stay & ~places);
  });
  if (lane == 0) wave_s[0][wave] = behind;
  __syncthreads();
  int rank = in_front(wave_s[0]);  // of this wave's first move
  {
    const int each = (words + NT - 1) / NT, w0 = min(words, tid * each), w1 = min(words, w0 + each);
    int mine = 0;
    for (int w = w0; w < w1; ++w) mine += __popcll(free_s[w]);
    int sum = bbm::wave_prefix_sum(mine);
    if (lane == 63) wave_s[2][wave] = sum;
    __syncthreads();
    sum += in_front(wave_s[2]) - mine;
    for (int w = w0; w < w1; ++w) {
      before_s[w] = sum;
      sum += __popcll(free_s[w]);
    }
  }
  __syncthreads();
  // the place of number n
  auto place_of = [&](int n) {
    int lo = 0, hi = words;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (before_s[mid] <= n) lo = mid;
      else hi = mid;
    }
    uint64_t bits = free_s[lo];
    n -= before_s[lo];
    int at = 0;  // bit n of those that are set: by halves
#pragma unroll
    for (int half = 32; half > 0; half >>= 1) {
      const int c = __popcll(bits & ((1ull << half) - 1ull));
      if (n >= c) n -= c, at += half, bits >>= half;
      else bits &= (1ull << half) - 1ull;
    }
    return 64 * lo + at;
  };

  // Eight lanes carry a key: the codes of K and V, 16 bytes each (of D = 64, four lanes), then scales and weight.
  constexpr int LK = D / 32;  // lanes of a key's codes, groups
  struct Load {
    uint4 codes;
    uint32_t small;
    uint8_t v_scale;
  };
  const int sub = lane & 7;
  auto carry = [&](int64_t s) __attribute__((always_inline)) {
    Load y = {};
    if (s < 0) return y;
    if (sub < 2 * LK) y.codes = *reinterpret_cast<const uint4*>((sub < LK ? P.c.k : P.c.v) + s * (D / 2) + sub % LK * 16);
    if (sub == 0) {
      if constexpr (D == 128) y.small = *reinterpret_cast<const uint32_t*>(P.c.k_scale + s * 4);
      else y.small = *reinterpret_cast<const uint16_t*>(P.c.k_scale + s * 2);
    }
    if (sub == 7) y.small = __float_as_uint(P.weights[s]);
    if (sub < LK) y.v_scale = P.c.v_scale[((s >> P.c.page_shift) * LK + sub << P.c.page_shift) + (s & (P.c.page - 1))];
    return y;
  };
  auto put = [&](int64_t s, const Load& y) __attribute__((always_inline)) {
    if (s < 0) return;
    if (sub < 2 * LK) *reinterpret_cast<uint4*>((sub < LK ? P.c.k : P.c.v) + s * (D / 2) + sub % LK * 16) = y.codes;
    if (sub == 0) {
      if constexpr (D == 128) *reinterpret_cast<uint32_t*>(P.c.k_scale + s * 4) = y.small;
      else *reinterpret_cast<uint16_t*>(P.c.k_scale + s * 2) = (uint16_t)y.small;
    }
    if (sub == 7) P.weights[s] = __uint_as_float(y.small);
    if (sub < LK) P.c.v_scale[((s >> P.c.page_shift) * LK + sub << P.c.page_shift) + (s & (P.c.page - 1))] = y.v_scale;
  };

  // Kept keys from behind to the free places: a wave writes down its moves until it has 64, and makes them, four times eight under way together.
  auto token_slot = [&](int j) {
    const int page = page_of(j);
    return page >= 0 && page < P.c.pages ? (page << P.c.page_shift) + (j & (P.c.page - 1)) : -1;
  };
  auto row_of = [&](int slot) -> int64_t { return (((int64_t)(slot >> P.c.page_shift) * P.c.Hk + hk) << P.c.page_shift) + (slot & (P.c.page - 1)); };
  constexpr int U = 4;
  int waiting = 0;
  auto make_moves = [&](int count) __attribute__((always_inline)) {
    for (int m0 = 0; m0 < count; m0 += 8 * U) {
      int64_t to[U];
      Load y[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int m = m0 + 8 * u + (lane >> 3);
        const int2 move = moves_s[wave][min(m, count - 1)];
        const bool real = m < count && move.x >= 0 && move.y >= 0;
        to[u] = real ? row_of(move.y) : -1;
        y[u] = carry(real ? row_of(move.x) : -1);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) put(to[u], y[u]);
    }
  };
  before = ties;
  for_kept(max(block0, edge_block), before, [&](int k, uint64_t stay) __attribute__((always_inline)) {
    if (k == edge_block) stay = edge_stay, before = edge_ties;
    const int left = x.chosen - 64 * k;
    const uint64_t go = left >= 64 ? 0ull : left <= 0 ? stay : stay & (~0ull << left);
    const int count = __popcll(go);
    if (count == 0) return;
    if (go >> lane & 1) {
      const int at = __popcll(go & ((1ull << lane) - 1ull));
      moves_s[wave][waiting + at] = make_int2(token_slot(x.f + 64 * k + lane), token_slot(x.f + place_of(rank + at)));
    }
    rank += count;
    waiting += count;
    if (waiting < 64) return;
    make_moves(64);
    waiting -= 64;
    const int2 rest = moves_s[wave][64 + lane];
    moves_s[wave][lane] = rest;
  });
  if (waiting > 0) make_moves(waiting);
  bbm::hand_over();

  // The last keys, in order, by n - b to the front.
  constexpr int ROUND = NWAVES * 8 * U;
  for (int i0 = 0; i0 < P.recent; i0 += ROUND) {
    int64_t to[U];
    Load y[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + (u * NWAVES + wave) * 8 + (lane >> 3);
      to[u] = -1;
      if (i < P.recent) {
        const int64_t from = slot_of(x.n - P.recent + i), s = slot_of(x.edge + i);
        to[u] = from < 0 ? -1 : s;
        y[u] = carry(s < 0 ? -1 : from);
      }
    }
    bbm::hand_over();
#pragma unroll
    for (int u = 0; u < U; ++u) put(to[u], y[u]);
  }
}

// Lengths, and the pages that requests give back, by a kernel of its own behind the other.
__global__ __launch_bounds__(256) void kv4_give_kernel(const EvictParams P) {
  const int lane = threadIdx.x & 63, r = (int)scalar(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (r >= P.R) return;
  int before = 0, all = 0;
  for (int i = lane; P.free_at && i < P.R; i += 64) {
    const int c = P.given[i];
    all += c;
    before += i < r ? c : 0;
  }
  give(P, r, wave_sum(before), wave_sum(all));
}

inline bool sizes_ok(int64_t R, int64_t Hk, int64_t max_keys) { return R >= 1 && R <= BBM_SLOTS_MAX_REQUESTS && Hk >= 1 && max_keys >= 1; }

}  // namespace

extern "C" __attribute__((visibility("default"))) size_t bbm_kv4_evict_workspace_bytes(int64_t R, int64_t Hk, int64_t max_keys) {
  return sizes_ok(R, Hk, max_keys) ? (size_t)R * sizeof(int32_t) : 0;
}

extern "C" __attribute__((visibility("default"))) int bbm_kv4_evict(const bbm_kv4_cache* cache, float* weights, int64_t R, const int32_t* lens, const int32_t* block_table,
                                                                    int64_t table_stride, int64_t max_pages, int64_t budget, int64_t recent, const int32_t* first,
                                                                    int32_t* new_lens, int32_t* free_pages, int64_t n_free, const int32_t* free_at, int32_t* free_next,
                                                                    int64_t max_len, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace bbm;
  const char* fn = "bbm_kv4_evict";
  clear_error();
  if (int rc = check_kv4(fn, cache)) return rc;
  if (R < 1 || budget < 1 || recent < 0 || max_len < 1)
    return fail(BBM_EINVAL, "%s: R=%lld, budget=%lld, max_len=%lld must be >= 1, recent=%lld >= 0", fn, (long long)R, (long long)budget, (long long)max_len, (long long)recent);
  if (int rc = check_table(fn, lens, block_table, table_stride, max_pages, cache->page)) return rc;
  if (!weights || !aligned(weights, 16)) return fail(BBM_EINVAL, "%s: weights must be a non-NULL 16-byte aligned pointer", fn);
  if (!new_lens || !aligned(new_lens, 4) || !aligned(first, 4)) return fail(BBM_EINVAL, "%s: new_lens and first must be 4-byte aligned, new_lens not NULL", fn);
  if ((free_at != nullptr) != (free_next != nullptr) || n_free < 0 || (n_free > 0) > (free_pages != nullptr) || (free_pages != nullptr) > (free_at != nullptr) || !aligned(free_pages, 4) || !aligned(free_at, 4) || !aligned(free_next, 4))
    return fail(BBM_EINVAL, "%s: free_pages (of n_free=%lld pages), free_at and free_next are given together, 4-byte aligned", fn, (long long)n_free);
  if (R > BBM_SLOTS_MAX_REQUESTS) return fail(BBM_EUNSUPPORTED, "%s: R=%lld requests, more than %d", fn, (long long)R, BBM_SLOTS_MAX_REQUESTS);
  if (R * cache->Hk > (1 << 21)) return fail(BBM_EUNSUPPORTED, "%s: problem too large (R=%lld, Hk=%lld)", fn, (long long)R, (long long)cache->Hk);
  const int64_t max_keys = max_pages * cache->page;
  if (std::min(budget, max_keys) > kMaxBudget) return fail(BBM_EUNSUPPORTED, "%s: budget=%lld is beyond %lld", fn, (long long)budget, (long long)kMaxBudget);
  const size_t need = bbm_kv4_evict_workspace_bytes(R, cache->Hk, max_keys);
  if (!workspace || workspace_bytes < need) return fail(BBM_EWORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need, workspace ? workspace_bytes : (size_t)0);
  if (!aligned(workspace, 16)) return fail(BBM_EINVAL, "%s: workspace must be 16-byte aligned", fn);
  if (int rc = check_apart(fn, {cache->k, cache->k_scale, cache->v, cache->v_scale, weights, new_lens, free_pages, free_next, workspace}, {block_table, first, free_at})) return rc;
  if (int rc = check_apart(fn, {cache->k, cache->k_scale, cache->v, cache->v_scale, weights, free_pages, free_next, workspace}, {lens})) return rc;
  EvictParams P = {};
  P.c = kv4_of(cache), P.weights = weights;
  P.lens = lens, P.table = block_table, P.first = first, P.free_at = free_at, P.new_lens = new_lens, P.free_pages = free_pages, P.free_next = free_next;
  // (lengths that are written over would be read by work-groups of the same launch)
  const bool together = R <= kGiveTogether && new_lens != lens;
  P.given = together ? nullptr : static_cast<int32_t*>(workspace);
  P.table_stride = table_stride, P.n_free = n_free, P.R = (int32_t)R, P.max_keys = (int32_t)max_keys;
  // (more than there are keys is as good as all of them)
  P.budget = (int32_t)std::min(budget, max_keys), P.recent = (int32_t)std::min(recent, max_keys);
  // Pages and weights in LDS: of what a request may have at most, if they leave room for two work-groups a CU, or for one; else as many weights as leave room for two.
  const int64_t places = ceil_div(P.budget, 64) * 12, keys = std::min(max_len, max_keys), table_bytes = ceil_div(keys, cache->page) * 4;
  const int64_t bytes = places + table_bytes <= kTwo ? table_bytes : 0, most = places + bytes + 4 * keys;
  P.held_pages = (int32_t)(bytes / 4);
  P.held = (int32_t)(most <= kOne ? keys : std::max<int64_t>(0, kTwo - places - bytes) / 4);
  const size_t lds = (size_t)(places + bytes + 4 * (int64_t)P.held);
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto kernel = cache->d == 64 ? kv4_evict_kernel<64> : kv4_evict_kernel<128>;
  if (lds > (size_t)kPlain) {
    // (of the function on the current device; a repeated call changes nothing)
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)std::max(kOne, kMaxBudget / 64 * 12));
    if (e != hipSuccess) return fail(BBM_EHIP, "%s: %s", fn, hipGetErrorString(e));
  }
  kernel<<<(unsigned)(R * cache->Hk + together), NT, lds, s>>>(P);
  if (!together) kv4_give_kernel<<<(unsigned)ceil_div(R, 4), 256, 0, s>>>(P);
  return launch_status(fn);
}
