// Tiles of 64 rows in LDS as the attention kernels copy, read and store them.
#pragma once
#include "bbm_mfma.h"

namespace bbm {

// Sum over each group of RC = 8 or 16 consecutive lanes, in all of them.
template <int RC>
__device__ __forceinline__ float row_sum(float x) {
  auto other = [](float v, auto ctrl) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  x += other(x, IntC<0xB1>{});              // lane ^ 1
  x += other(x, IntC<0x4E>{});              // lane ^ 2
  x += other(x, IntC<0x141>{});             // mirrored within 8 lanes
  if constexpr (RC == 16) x += other(x, IntC<0x140>{});  // mirrored within 16 lanes
  return x;
}

// LDS layout of a 64-row x D tile, shared by every tile of these kernels.  One asynchronous copy instruction of a wave
// fills one 1 KiB block with RPB rows that lie NBLK rows apart: row r sits in block r % NBLK at slot r / NBLK; blocks
// are 1 KiB + 64 B apart, and the 16-byte chunk c of row r sits at chunk position c ^ ((r >> 2) & 3).  With that both
// access patterns are free of bank conflicts: 16 lanes reading the same chunk of 16 consecutive rows (A operand from
// tile rows), and 32 lanes reading 64 contiguous bytes of 4 consecutive rows (transposing read).
template <int D>
struct TL {
  static constexpr int RC = D / 8;          // 16-byte chunks per row
  static constexpr int RPB = 64 / RC;       // rows per 1 KiB block
  static constexpr int NBLK = 64 / RPB;     // blocks per tile
  static constexpr int TBLK = 512 + 32;     // block stride in elements
  static constexpr int ELEMS = NBLK * TBLK;
};

// Two floats rounded to bf16, the first in the low half; eight of them as a matrix operand.
__device__ __forceinline__ uint32_t pack(float a, float b) {
  const bf16x2 v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ bf16x8 operand(const uint32_t (&w)[4]) {
  const uint4 v = make_uint4(w[0], w[1], w[2], w[3]);
  return __builtin_bit_cast(bf16x8, v);
}

// The lane's number, found anew at each use: for what is needed once a step and not worth a register throughout the loop.
__device__ __forceinline__ int lane_now() {
  int x;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(x));
  return x;
}

// An asynchronous copy of SIZE bytes per lane into LDS, from byte `off` (per lane) of the `bytes` bytes at the wave-uniform p;
// lanes whose bytes lie past those write zeros (the bounds check of the buffer resource).  The buffer form also matters to the
// compiler: it counts the global form as possibly touching LDS through the flat path, and with one in flight it waits for ALL
// outstanding LDS reads at every use of one, which undoes the reads that run ahead (mfma_ring).
template <int SIZE>
__device__ __forceinline__ void copy_async(const void* p, int bytes, uint32_t off, void* dst) {
  static_assert(SIZE == 16 || SIZE == 4, "the builtin wants literal sizes");
  auto* const lds = (void __attribute__((address_space(3)))*)dst;
  const __amdgpu_buffer_rsrc_t src = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)scalar(bytes), 0x00027000);
  if constexpr (SIZE == 16)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(src, lds, 16, off, 0, 0, 0);
  else
    __builtin_amdgcn_raw_ptr_buffer_load_lds(src, lds, 4, off, 0, 0, 0);
}

// Asynchronous global -> LDS copy of the first `rows` (0 .. 64) of the 64 rows of a [..][D] matrix at `tile`; zeros for the rest.
// This is copy instruction n of the NBLK / NW of a wave.  Lane l of a copy instruction lands at block base + 16*l, i.e. slot
// l / RC, chunk position l % RC.  One address register per lane (`base`, from tile_copy_base) serves all instructions: the XOR
// of the chunk position splits into a part of the lane and one of the block.
template <int D, int NW>
__device__ __forceinline__ uint32_t tile_copy_base(int wave, int lane) {
  using L = TL<D>;
  static_assert(L::NBLK % 16 == 0 || L::NBLK == 8, "(row >> 2) & 3 must be the XOR of the lane's part and the block's part");
  const int slot = lane / L::RC, pos = lane % L::RC;
  return (uint32_t)((wave + L::NBLK * slot) * D + (pos ^ ((L::NBLK * slot >> 2) & 3)) * 8) * 2u;
}
template <int D, int NW>
__device__ __forceinline__ void tile_copy_piece(const __bf16* __restrict__ tile, int rows, uint32_t base, __bf16* dst, int n, int wave) {
  using L = TL<D>;
  static_assert(L::NBLK % NW == 0, "tile must split evenly over the waves");
  const int blk = n * NW + wave;
  asm volatile("" : "+v"(base));  // one register throughout the tile loop, not one per block
  copy_async<16>(tile, rows * D * 2, (base ^ (uint32_t)(((blk >> 2) & 3) << 4)) + n * NW * D * 2, dst + blk * L::TBLK);
}
// How many of the 64 rows from row0 on lie below N.  (A scalar by force: the compiler clamps in a vector register, and a buffer
// resource in one costs a loop around every copy.)
__device__ __forceinline__ int rows_of_tile(int row0, int N) { return (int)scalar(max(0, min(64, N - row0))); }

// Per-lane base addresses (in elements) of the two read patterns.
template <int D>
struct TileAddr {
  int ra[2];  // A operand from tile rows: row 32*blk + lane%32, chunk 2t + lane/32; ra[t & 1] + (t >> 1)*32 + blk*(32/NBLK)*D
  int ta[2];  // transposing read of 16-row step u, half a, column block db: ta[a] + u*(D == 64 ? 2*D : D) + db*32
  __device__ __forceinline__ void init(int lane) {
    using L = TL<D>;
    const int lq = lane & 31, hh = lane >> 5;
    const int hq = (lq >> 2) & 3;
    const int rowbase = (lq % L::NBLK) * L::TBLK + (lq / L::NBLK) * D;
    const int x = hh ^ (hq & 1), y = hq >> 1;
    ra[0] = rowbase + (2 * y + x) * 8;
    ra[1] = rowbase + (2 * (1 ^ y) + x) * 8;
    const int vy = (lane & 15) >> 2, vg = (lane >> 4) & 1, vx = (lane & 3) >> 1;
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      const int blockrow = D == 64 ? (4 * hh + vy) * L::TBLK + a * D : (8 * a + 4 * hh + vy) * L::TBLK;
      ta[a] = blockrow + (2 * (vg ^ a) + (vx ^ hh)) * 8 + 4 * (lane & 1);
    }
  }
  __device__ __forceinline__ bf16x8 row_frag(const __bf16* tile, int blk, int t) const {
    using L = TL<D>;
    return *reinterpret_cast<const bf16x8*>(tile + ra[t & 1] + (t >> 1) * 32 + blk * (32 / L::NBLK) * D);
  }
  // rows 16u + 8a + 4*(lane/32) + 0..3 (a = 0, 1) of column 32*db + lane%32: the order in which a lane's accumulator
  // registers 8*(u%2) .. 8*(u%2)+7 of row block u/2 list the rows of a 32x32 product
  __device__ __forceinline__ bf16x8 tr_frag(const __bf16* tile, int u, int db) const {
    s16x4 part[2];
#pragma unroll
    for (int a = 0; a < 2; ++a)
      part[a] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (s16x4 __attribute__((address_space(3)))*)(tile + ta[a] + u * (D == 64 ? 2 * D : D) + db * 32));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// acc * mult, rounded to bf16, to rows row0 .. of a [N][D] matrix: lane l holds row l%32 of the wave's 32-row slab,
// columns 32*db + 8*(e/4) + 4*(l/32) + e%4.  The slab is staged in LDS (`stage`, 32*D elements, this wave's own) so
// that the global stores are whole rows: 16-byte chunk ch of row r sits at chunk position ch ^ (r % RC).  (With the forward's
// store_rows, by buffer, more registers of these kernels lie in scratch memory: 1 to 2 % slower at D = 64.)
template <int D>
__device__ __forceinline__ void store_slab(const f32x16 (&acc)[D / 32], float mult, __bf16* stage, __bf16* __restrict__ dst,
                                           int row0, int N, int lane) {
  using L = TL<D>;
  // behind an optimisation barrier: otherwise the staging addresses are hoisted out of the loop over items and stay in
  // registers (or in scratch memory) throughout the tile loop
  asm volatile("" : "+v"(lane));
  const int lq = lane & 31, hh = lane >> 5, gro = lane / L::RC, gco = lane % L::RC;
#pragma unroll
  for (int db = 0; db < D / 32; ++db) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      bf16x4 ov;
      for (int e = 0; e < 4; ++e) ov[e] = (__bf16)(acc[db][4 * g + e] * mult);
      *reinterpret_cast<bf16x4*>(stage + lq * D + (((4 * db + g) ^ (lq % L::RC)) * 8) + 4 * hh) = ov;
    }
  }
  __bf16* og = dst + (int64_t)row0 * D;
#pragma unroll
  for (int n = 0; n < 32 / L::RPB; ++n) {
    const int r = n * L::RPB + gro;
    const bf16x8 ov = *reinterpret_cast<const bf16x8*>(stage + r * D + ((gco ^ (r % L::RC)) * 8));
    if (row0 + r < N) *reinterpret_cast<bf16x8*>(og + r * D + gco * 8) = ov;
  }
}

// (On the bits: the kernels are compiled with a flag that lets the compiler take any number for not a NaN.)
__device__ __forceinline__ bool is_nan(float x) {
  uint32_t bits = __float_as_uint(x);
  asm volatile("" : "+v"(bits));
  return (bits & 0x7fffffffu) > 0x7f800000u;
}

// The `bytes` bytes at the wave-uniform p: loads past them give zeros, stores are dropped.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)scalar(bytes), 0x00027000);
}

// XCD-aware logical work-group id: work-groups are handed to the 8 XCDs round-robin; give each XCD a contiguous range
// of logical ids so that the work-groups of one head (which share its tensors) meet in one XCD's L2.
__device__ __forceinline__ int logical_wg(int wg, int total) {
  const int xcd = wg & 7, slot = wg >> 3;
  const int per = total >> 3, rem = total & 7;
  return xcd * per + (xcd < rem ? xcd : rem) + slot;
}

// Bits 0 .. lim of 64.
__device__ __forceinline__ uint64_t bits_up_to(int lim) { return lim >= 63 ? ~0ull : lim < 0 ? 0ull : (2ull << lim) - 1ull; }
// x where bit 8 * (e / 4) + e % 4 of w is set, else -infinity (by bits: x may be anything).
__device__ __forceinline__ float keep_if(uint32_t w, int e, float x) {
  const uint32_t keep = (uint32_t)((int32_t)(w << (31 - (8 * (e / 4) + e % 4))) >> 31);
  return __uint_as_float((__float_as_uint(x) & keep) | (0xff800000u & ~keep));
}

}  // namespace bbm
