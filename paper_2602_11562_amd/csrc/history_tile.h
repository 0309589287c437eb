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

// Which tile of which of `per` (sequence, head) pairs a workgroup takes. Workgroups go to the eight dies in turn, and a die's 4 MB of
// cache serve the tiles of a pair that run on it at once. So `run` tiles of a pair in a row are one die's, and the runs are dealt to the
// dies turned by one from row of runs to row of runs (with a multiple of eight pairs, a long sequence would otherwise be one die's).
struct Deal {
  int per, tiles, run;
  MulDiv by_run, by_per;
  unsigned grid;
};
inline long long tiles_a_run(long long tiles) {
  // (16 histories of 920 to 4000 items, tiles a run 1, 2, 4, 8, 16: dq 537, 496, 481, 512, 506 us; 512 of 40 to 200, at most two tiles
  // each, 1 and 2: dq 49 and 58 us, dk and dv 51 and 69)
  return tiles >= 32 ? 4 : 1;
}
inline Deal deal(long long per, long long tiles) {
  const long long run = tiles_a_run(tiles), runs = (tiles + run - 1) / run * per, grid = (runs + 7) / 8 * 8 * run;
  return Deal{(int)per, (int)tiles, (int)run, mul_div((unsigned)run), mul_div((unsigned)per), (unsigned)grid};
}
// How many sequences of `tiles` tiles for each of Hkv heads one launch holds, which has fewer than 2^32 threads (the grid grows with the
// longest sequence, whatever the rows are in all). 0: the N of the call have more than 2^31 - 1 workgroups, or one has too many.
inline int sequences_a_launch(int N, int Hkv, long long tiles, int threads) {
  if ((long long)N * Hkv > 0x7fffffffLL / tiles) return 0;
  const long long run = tiles_a_run(tiles), runs = (tiles + run - 1) / run, most = 0xffffffffLL / threads / (8 * run) * 8 / (runs * Hkv);
  return most < N ? (int)most : N;
}
// The call in as many launches as that takes, mostly one. go(part, n): a launch for sequences n and on, part.N of them
template <typename Args, typename Go>
laser_status launch_dealt(const Args& a, long long tiles, int threads, Go&& go) {
  const int most = sequences_a_launch(a.N, a.Hkv, tiles, threads);
  if (most <= 0) return LASER_ERR_SHAPE;
  for (long long n = 0; n < a.N; n += most) {
    Args part = a;
    part.N = a.N - n < most ? (int)(a.N - n) : most;
    part.off = a.off + n;
    part.deal = deal((long long)part.N * a.Hkv, tiles);
    go(part, n);
    const laser_status s = launch_status();
    if (s != LASER_OK) return s;
  }
  return LASER_OK;
}
struct Place { int rank, pair; };   // the how manieth tile of which pair; rank >= tiles: none
__device__ __forceinline__ Place place_of(const Deal& d, unsigned block) {
  const unsigned at = block >> 3, row = d.by_run.div(at), chunk = row * 8 + (block & 7), turn = d.by_per.div(chunk);
  const unsigned turned = chunk - turn * d.per + turn;
  return Place{(int)(turn * d.run + at - row * d.run), (int)(turned - d.by_per.div(turned) * d.per)};
}

constexpr unsigned NO_COLUMN = 0x80000000u;   // an offset behind every buffer's end

// A tile row of DP bf16 is CH pieces of 16 bytes, piece c of row r at place c ^ tile_swz(r). Both ways of reading then find all
// banks: 16 rows at one piece (operands over the width), four rows at four pieces (the transpose load).
template <int CH> __device__ __forceinline__ int tile_swz(int r) {
  const int q = (r * CH) >> 4;   // 256-byte lines of all banks
  return CH == 16 ? (q & 3) * 4 + ((q >> 2) & 3) : CH == 8 ? (q & 1) * 4 + ((q >> 1) & 3) : q & 3;
}

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

// How a lane reads tiles as the A operand of its products. Tiles start at multiples of 256 bytes, so a piece's place can be flipped in
// the sum with the tile's address; place() does so once for all reads of a tile (or of several, `more` bytes behind it), whose rows are
// then the reads' immediate offsets.
template <int DP>
struct TileReader {
  static constexpr int ROW = DP * 2, CH = DP / 8, KS = DP / 16, DB = DP / 32;
  unsigned row, lo, hi;
  unsigned rows_at[KS], lo_at[DB], hi_at[DB];
  __device__ __forceinline__ explicit TileReader(int lane) {
    const int l32 = lane & 31, h = lane >> 5, i16 = lane & 15, r = h * 4 + (i16 >> 2), c = 2 * (l32 >> 4) + ((i16 & 3) >> 1);
    row = l32 * ROW + ((h ^ tile_swz<CH>(l32)) << 4);
    lo = r * ROW + ((c ^ tile_swz<CH>(r)) << 4) + (i16 & 1) * 8;
    hi = (r + 8) * ROW + ((c ^ tile_swz<CH>(r + 8)) << 4) + (i16 & 1) * 8;
  }
  __device__ __forceinline__ void place_rows(unsigned at) {
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      rows_at[s] = (at + row) ^ (s << 5);
      asm volatile("" : "+v"(rows_at[s]));
    }
  }
  __device__ __forceinline__ void place_cols(unsigned at) {
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      lo_at[db] = (at + lo) ^ (db << 6);
      hi_at[db] = (at + hi) ^ (db << 6);
      asm volatile("" : "+v"(lo_at[db]), "+v"(hi_at[db]));
    }
  }
  __device__ __forceinline__ void place(unsigned at) {
    place_rows(at);
    place_cols(at);
  }
  // a product over the width: row 32 b + lane % 32, pieces 2 s + lane / 32
  __device__ __forceinline__ bf16x8 rows(int more, int b, int s) const { return lds_read16(lds_at(rows_at[s]) + more + b * 32 * ROW); }
  // a product over the rows, of the transpose: columns 32 db .., rows 16 s + {4h .. 4h+3, 8+4h .. 8+4h+3} (the order in which a score
  // block's accumulators hold them)
  __device__ __forceinline__ bf16x8 cols(int more, int s, int db) const {
    auto half = [&](unsigned x) {
      return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(lds_at(x) + more + s * 16 * ROW));
    };
    const s16x4 a = half(lo_at[db]), b = half(hi_at[db]);
    return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

__device__ __forceinline__ unsigned pack_bf16(float a, float b) {
  const bf16x2 c = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(unsigned, c);
}

// Four bytes per lane to LDS (uniform address + 4 * lane)
__device__ __forceinline__ void buffer_to_lds4(u32x4 buf, unsigned voff, unsigned lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds\n" ::"s"(lds_addr), "v"(voff), "s"(buf)
               : "memory");
}

// Tiles of packed keys and values: request x of wave w brings rows (w + x NW) RPI and on, of both. These are STEP rows apart from request to
// request, which leaves a lane's offset as it is where STEP rows are whole turns of tile_swz: the buffer begins that much later.
template <int DP, int NW>
struct PackedTiles {
  using Sh = TileShape<DP>;
  static constexpr int RPW = Sh::GROUPS / NW, STEP = NW * Sh::RPI;
  static constexpr int OFFS = STEP * Sh::CH % 256 == 0 ? 1 : RPW;   // offsets that differ
  static_assert(Sh::GROUPS % NW == 0, "whole requests");
  unsigned koff[OFFS], voff[OFFS], to;
  __device__ __forceinline__ void init(int D, long long kp, long long vp, int wave, int lane) {
    to = wave * 1024;
    const int r = wave * Sh::RPI + lane / Sh::CH;
#pragma unroll
    for (int x = 0; x < OFFS; ++x) {
      const int c = (lane % Sh::CH) ^ tile_swz<Sh::CH>(r + x * STEP);
      koff[x] = c * 8 < D ? (unsigned)(r * (int)kp * 2 + c * 16) : NO_COLUMN;
      voff[x] = c * 8 < D ? (unsigned)(r * (int)vp * 2 + c * 16) : NO_COLUMN;
    }
  }
  // rows k, v and on (`left` of them are the sequence's); keys to `at`, values behind them
  __device__ __forceinline__ void fetch(const unsigned short* k, const unsigned short* v, long long kp, long long vp, int D, int left,
                                        unsigned at) const {
    left = left < TI ? left : TI;
#pragma unroll
    for (int x = 0; x < RPW; ++x) {
      const int rest = left - x * STEP;
      buffer_to_lds16(buffer_of(k + x * STEP * kp, rest > 0 ? (unsigned)(((rest - 1) * (int)kp + D) * 2) : 0u), koff[x % OFFS], at + to + x * NW * 1024);
      buffer_to_lds16(buffer_of(v + x * STEP * vp, rest > 0 ? (unsigned)(((rest - 1) * (int)vp + D) * 2) : 0u), voff[x % OFFS],
                      at + to + Sh::BYTES + x * NW * 1024);
    }
  }
};

// A block of 32 rows that the accumulators hold transposed (column 32 db + 8 g + 4 h + e of row lane % 32), times `by`, through an
// LDS patch of the wave's own so that it leaves in 16-byte pieces; to(r): where row r goes, rows from `rows` on go nowhere
template <int DP, typename To>
__device__ __forceinline__ void store_block(const f32x16* acc, float by, unsigned char* patch, int rows, int D, int lane, const To& to) {
  constexpr int OP = DP * 2 + 16, CH = DP / 8;
  const int l32 = lane & 31, h = lane >> 5;
#pragma unroll
  for (int db = 0; db < DP / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const u32x2 o = {pack_bf16(acc[db][g * 4] * by, acc[db][g * 4 + 1] * by),
                       pack_bf16(acc[db][g * 4 + 2] * by, acc[db][g * 4 + 3] * by)};
      *reinterpret_cast<u32x2*>(patch + l32 * OP + (db * 32 + g * 8 + h * 4) * 2) = o;
    }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll 2
  for (int x = lane; x < 32 * CH; x += 64) {
    const int r = x / CH, c = x % CH;
    if (r < rows && c * 8 < D) *reinterpret_cast<u32x4*>(to(r) + c * 8) = *reinterpret_cast<const u32x4*>(patch + r * OP + c * 16);
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
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

}  // namespace laser
