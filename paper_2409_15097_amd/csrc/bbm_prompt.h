// What the kernels of attention over packed prompts share: strided rows, copies of their tiles, and which work-group does what.
#pragma once
#include "bbm_packed.h"
#include "bbm_tile.h"

namespace bbm {

struct Rows {
  __bf16* p;
  int64_t head;
  int32_t row;  // strides in elements
};
inline Rows rows_of(const bbm_packed* x, int64_t T, int d) {
  return Rows{static_cast<__bf16*>(x->ptr), x->head_stride, (int32_t)(T > 1 ? x->row_stride : d)};
}
// Rows behind a sequence's end are kept out by the bounds of a buffer, which needs rows that do not lie upon each other.
inline int check_rows(const char* fn, const char* name, const bbm_packed* x, int64_t T, int64_t heads, int d, bool output) {
  if (int rc = check_packed(fn, name, x, T, heads, d, output)) return rc;
  if (T > 1 && x->row_stride < d) return fail(BBM_EUNSUPPORTED, "%s: rows of %s overlap (stride %lld): make it contiguous", fn, name, (long long)x->row_stride);
  return BBM_OK;
}

// Work-groups go to the eight XCDs in turn, each with a cache of its own.  An XCD gets whole heads where there are eight or more, so that the
// pieces which read the same keys (or queries) meet in one cache; the pieces of a head that several XCDs share go to them in turn, so that all XCDs
// get as much work.  Heads (planes) that are neighbours run side by side, as those of a group, which share their keys, have to.  In a plane
// the pieces come in the order of `number`.  launch: 8 * planes * ceil(pieces / 8) work-groups.
struct Work {
  int plane, number;
};
__device__ __forceinline__ Work work_of(int wg, int planes) {
  const int xcd = wg & 7, slot = wg >> 3, rank = slot / planes, unit = xcd * planes + (slot - rank * planes);
  return Work{unit >> 3, rank * 8 + (unit & 7)};
}
inline int64_t work_groups(int64_t planes, int64_t pieces) { return 8 * planes * ceil_div(pieces, 8); }

// With few pieces the longest sequence is what a launch waits for: two waves then share the keys of every tile (HALVES of the kernels), which makes twice as
// many work-groups of steps half as long.  Whole / halved, us, a training step with the backward pass either way: 13 packed sequences of 213 on average, 16 heads of
// 64 (352 pieces of 128 rows), 54 / 50; 1 x 2048, 16 heads of 64 (256), 74 / 67; but 4096 and 3277, 32 / 8 heads of 128 (1856), 962 / 989; 200 x 22, 8 / 2 of 128, 59 / 61.
// Forward alone: 37 sequences of 59, 16 heads of 64 (288), 10.5 / 12.0; 1 x 4096, 32 heads of 128 (1024), 153 / 179.
inline bool split_keys(int64_t T, int64_t R, int64_t H) { return ceil_div(T, 128) * H <= 384 && T >= 128 * R; }

// Asynchronous copies of up to 64 strided rows to a tile in LDS (layout TL), NBLK / NW instructions a wave; rows from `rows` on come as zeros.
template <int D, int NW>
struct TileCopy {
  typedef TL<D> L;
  static constexpr int PIECES = L::NBLK / NW;
  uint32_t row_off;
  int chunk;
  __device__ __forceinline__ void init(int wave, int lane, int stride) {
    const int slot = lane / L::RC;
    row_off = (uint32_t)((wave + L::NBLK * slot) * stride) * 2u;
    chunk = lane % L::RC ^ (L::NBLK * slot >> 2 & 3);
  }
  // instruction n of the wave, for the tile whose first row is at `tile`
  __device__ __forceinline__ void piece(const __bf16* tile, int rows, int stride, __bf16* dst, int n, int wave) const {
    static_assert(NW == 4 || NW == 2, "the block's part of the chunk position does not depend on the wave");
    const int blk = n * NW + wave, part = n * NW >> 2 & 3;
    const int bytes = rows > 0 ? ((rows - 1) * stride + D) * 2 : 0;
    uint32_t at = row_off;
    asm volatile("" : "+v"(at));  // one register, not one for every instruction
    copy_async<16>(tile, bytes, at + (uint32_t)(n * NW * stride) * 2u + ((uint32_t)(chunk ^ part) << 4), dst + blk * L::TBLK);
  }
};

// A wave's 32 x D slab of strided rows (zeros from `rows` on) to LDS: 16-byte chunk c of row r at chunk position c ^ (r % RC).
template <int D>
__device__ __forceinline__ void copy_slab(const __bf16* first, int rows, int stride, __bf16* stage, int lane) {
  constexpr int RC = D / 8, RPB = 64 / RC;
  const int bytes = rows > 0 ? ((rows - 1) * stride + D) * 2 : 0;
#pragma unroll
  for (int n = 0; n < 32 / RPB; ++n) {
    const int r = n * RPB + lane / RC;
    copy_async<16>(first, bytes, (uint32_t)(r * stride + (lane % RC ^ r % RC) * 8) * 2u, stage + n * 512);
  }
}
template <int D>
__device__ __forceinline__ bf16x8 slab_frag(const __bf16* stage, int t, int lane) {
  constexpr int RC = D / 8;
  return *reinterpret_cast<const bf16x8*>(stage + (lane & 31) * D + ((2 * t + (lane >> 5)) ^ (lane & 31) % RC) * 8);
}

// acc * mult, rounded, to the first `rows` of 32 strided rows: lane l holds row l % 32, columns 32 * db + 8 * (e / 4) + 4 * (l / 32) + e % 4.  By way of
// LDS (`stage`, 32 x D of this wave's own), so that whole rows are stored; rows that are not there lie outside the buffer.
template <int D>
__device__ __forceinline__ void store_strided(const f32x16 (&acc)[D / 32], float mult, __bf16* stage, __bf16* first, int rows, int stride, int lane) {
  constexpr int RC = D / 8, RPB = 64 / RC;
  asm volatile("" : "+v"(lane));  // (the addresses are not to be formed in front of the loop over tiles)
  const int lq = lane & 31, hh = lane >> 5;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      bf16x4 x;
      for (int e = 0; e < 4; ++e) x[e] = (__bf16)(acc[db][4 * g + e] * mult);
      *reinterpret_cast<bf16x4*>(stage + lq * D + (((4 * db + g) ^ (lq % RC)) * 8) + 4 * hh) = x;
    }
  const __amdgpu_buffer_rsrc_t out = buffer_of(first, rows > 0 ? ((rows - 1) * stride + D) * 2 : 0);
#pragma unroll
  for (int n = 0; n < 32 / RPB; ++n) {
    const int r = n * RPB + lane / RC;
    const u32x4 x = *reinterpret_cast<const u32x4*>(stage + r * D + (lane % RC ^ r % RC) * 8);
    __builtin_amdgcn_raw_buffer_store_b128(x, out, (r * stride + lane % RC * 8) * 2, 0, 0);
  }
}

}  // namespace bbm
