// Tiles of keys and values for the matrix-core kernels of attention among a history's items (bf16): how they come into LDS, from
// packed rows or from the pages of a cache, and how they are read as operands.
#pragma once

#include "history.h"
#include "sta_mfma_tile.h"

namespace laser {

// A buffer descriptor: `bytes` from `base` on can be read, what lies behind reads as zeros and touches no memory
__device__ __forceinline__ u32x4 buffer_of(const void* base, unsigned bytes) {
  const unsigned long long b = reinterpret_cast<unsigned long long>(base);
  return u32x4{(unsigned)__builtin_amdgcn_readfirstlane((unsigned)b),
               (unsigned)__builtin_amdgcn_readfirstlane((unsigned)(b >> 32)) & 0xffffu,
               (unsigned)__builtin_amdgcn_readfirstlane(bytes), 0x00027000u};
}

// 16 bytes per lane from a buffer at the lane's offset to LDS (uniform address + 16 * lane). Outside the compiler's sight: whoever
// reads them waits (vmcnt) and passes a barrier first.
__device__ __forceinline__ void buffer_to_lds16(u32x4 buf, unsigned voff, unsigned lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds\n" ::"s"(lds_addr), "v"(voff), "s"(buf)
               : "memory");
}

constexpr unsigned NO_COLUMN = 0x80000000u;   // an offset behind every buffer's end

// A tile row of DP bf16 is CH pieces of 16 bytes, piece c of row r at place c ^ kswz(r) of a key row and c ^ 4 vswz(r) of a value
// row: what an operand read takes at once (16 rows at one piece; four rows at four pieces) then lies in all banks.
template <int CH> __device__ __forceinline__ int tile_kswz(int r) { return ((r * CH) >> 4) & (CH - 1); }
template <int CH> __device__ __forceinline__ int tile_vswz(int r) { return ((r * CH) >> 4) & (CH / 4 - 1); }

// Offsets of a lane's pieces: each wave-wide request brings 64 pieces, RPI rows
template <int DP>
struct TileShape {
  static constexpr int ROW = DP * 2, CH = DP / 8, RPI = 64 / CH, BYTES = TI * ROW, GROUPS = TI / RPI;
};

// pages[] through the scalar cache: `at` is the same for all lanes
__device__ __forceinline__ int scalar_int(const int32_t* p, int at) {
  typedef const __attribute__((address_space(4))) int32_t* scalar_ptr;
  return ((scalar_ptr)(unsigned long long)p)[__builtin_amdgcn_readfirstlane(at)];
}

// K rows as the A operand of a product over the width: item 32 b + lane % 32, pieces 2 s + lane / 32
template <int DP>
__device__ __forceinline__ bf16x8 tile_k(unsigned at, int b, int s, int l32, int h) {
  constexpr int CH = DP / 8;
  const int row = b * 32 + l32;
  return lds_read16(lds_at(at + row * (DP * 2) + (((2 * s + h) ^ tile_kswz<CH>(row)) << 4)));
}

// V^T as the A operand of a product over items: columns 32 db .., items 16 s + {4h .. 4h+3, 8+4h .. 8+4h+3} (the order in which a
// score block's accumulators hold them)
template <int DP>
__device__ __forceinline__ bf16x8 tile_vt(unsigned at, int s, int db, int lane) {
  constexpr int CH = DP / 8;
  const int h = lane >> 5, i16 = lane & 15, vrow = h * 4 + (i16 >> 2), vlow = 2 * ((lane & 31) >> 4) + ((i16 & 3) >> 1);
  auto half = [&](int r) {
    const unsigned a = at + r * (DP * 2) + (((vlow + 4 * db) ^ (4 * tile_vswz<CH>(r))) << 4) + (i16 & 1) * 8;
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)lds_at(a));
  };
  const s16x4 lo = half(s * 16 + vrow), hi = half(s * 16 + 8 + vrow);
  return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// x of the other half of the wave: max and sum over the two lanes that share a row
__device__ __forceinline__ float half_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ unsigned pack_bf16(float a, float b) {
  const bf16x2 c = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(unsigned, c);
}

}  // namespace laser
