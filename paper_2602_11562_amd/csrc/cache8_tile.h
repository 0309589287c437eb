// Tiles of 8-bit keys and values for the matrix-core kernels over a cache of 8-bit blocks: how they come into LDS, and how they are read
// as bf16 operands. Every e4m3 number times its block's power of two is a bf16 number, so nothing is rounded on the way.
#pragma once

#include "cache8.h"
#include "history_tile.h"

namespace laser {

// A tile row of DP bytes is CH pieces of 16, piece c of row r at place c ^ swz8(r). The reads of 16 rows at one piece (keys), and the
// transpose loads of rows {0..3, 8..11} or {4..7, 12..15} at two pieces (values), then find all banks.
template <int CH> __device__ __forceinline__ int swz8(int r) {
  return CH == 8 ? ((r >> 1) & 1) * 2 + ((r >> 3) & 1) * 4 + ((r >> 2) & 1) : CH == 4 ? (r >> 2) & 3 : (r >> 3) & 1;
}
// The same for reads of rows {0..3, 8..11, 16..19, 24..27} (+ 4), the lanes of 16 at one piece and those of the next 16 at the next, and transpose
// loads of rows 0..15 or 16..31 at one
template <int CH> __device__ __forceinline__ int swz8_octets(int r) {
  const int b1 = (r >> 1) & 1, b2 = (r >> 2) & 1, b3 = (r >> 3) & 1, b4 = (r >> 4) & 1;
  return CH == 8 ? b1 + b3 * 2 + (b2 ^ b4) * 4 : CH == 4 ? (b2 ^ b4) + (b3 ^ b4) * 2 : b3;
}

// 8 e4m3 numbers, the first four times a, the others times b (powers of two)
__device__ __forceinline__ bf16x8 wide8(unsigned lo, unsigned hi, float a, float b) {
  const bf16x2 x0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, a, false), x1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, a, true),
               x2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, b, false), x3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, b, true);
  return __builtin_bit_cast(bf16x8, u32x4{__builtin_bit_cast(unsigned, x0), __builtin_bit_cast(unsigned, x1),
                                          __builtin_bit_cast(unsigned, x2), __builtin_bit_cast(unsigned, x3)});
}

// Scales of a tile: group g of 8 items has its key scale at 16 (g / 2) + 4 (g % 2) and its value scale 8 bytes behind it. Four bytes per
// lane from the lane's address to LDS (uniform address + 4 * lane), outside the compiler's sight as buffer_to_lds16.
__device__ __forceinline__ void global_to_lds4(const void* p, unsigned lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off\n" ::"s"(lds_addr), "v"(p) : "memory");
}

// Waits until at most n of this wave's vector-memory operations are outstanding: the requests of a tile ahead (3, 5 or 9), or of two of 16 rows (6 or 10)
__device__ __forceinline__ void wait_requests(int n) {
  switch (n) {
#define LASER_VM_CASE(i) case i: __builtin_amdgcn_s_waitcnt(vmcnt_imm(i)); break;
    LASER_VM_CASE(3) LASER_VM_CASE(5) LASER_VM_CASE(6) LASER_VM_CASE(9) LASER_VM_CASE(10)
#undef LASER_VM_CASE
    default: __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
  }
}

// What a wave brings of a tile: ROWS rows of keys and of values and their scales. Pages hold PART items or more each (8 or 16), which then
// share where they come from: a lone wave issues an instruction every 5 to 9 cycles, and those for the addresses of 32 rows were as many
// as for their products (one token for 128 users x up to 4096 by parts of 8 and of 16: 26.0 and 24.4 us).
template <int DP, int ROWS, int PART, bool OCTETS = false>
struct Tiles8 {
  static constexpr int CH = DP / 16, RPI = 64 / CH < ROWS ? 64 / CH : ROWS, REQ = ROWS / RPI, IDS = ROWS / PART, EACH = PART / RPI;
  unsigned off[REQ];
  int ids[IDS];            // pages of the next rows: of their items 0, PART, ..
  int part;                // rows of a request that are on one page
  __device__ __forceinline__ void init(int D, int page_log2, int row0, int lane) {
    part = (1 << page_log2) < RPI ? 1 << page_log2 : RPI;
#pragma unroll
    for (int x = 0; x < REQ; ++x) {
      const int in = lane / CH, r = row0 + x * RPI + in, c = (lane % CH) ^ (OCTETS ? swz8_octets<CH>(r) : swz8<CH>(r));
      off[x] = c * 16 < D && in < RPI ? (unsigned)(((EACH > 1 ? x % EACH * RPI : 0) + in) * D + c * 16) : NO_COLUMN;
    }
  }
  __device__ __forceinline__ int requests() const { return 2 * REQ * (RPI / part) + 1; }
  __device__ __forceinline__ void look_up(const int32_t* table, int j, int end, int page_log2) {
#pragma unroll
    for (int x = 0; x < IDS; ++x) ids[x] = j + x * PART < end ? scalar_int(table, (j + x * PART) >> page_log2) : -1;
  }
  // items j and on (behind `end` there are none: zeros); keys to k_at, values to v_at, scales to s_at
  __device__ __forceinline__ void fetch(const Cache8Args& a, int hk, int j, int end, unsigned k_at, unsigned v_at, unsigned s_at, int lane) const {
    const CacheArgs& c = a.c;
    const int mask = (1 << c.page_log2) - 1;
    // items at .. at + count - 1, on page id, for a request's rows skip and on
    auto rows = [&](int id, int at, int skip, int count, auto&& to) __attribute__((always_inline)) {
      const int left = end - at < count ? end - at : count;
      const bool ok = left > 0 && (unsigned)id < (unsigned)c.P;
      const long long row = ok ? (((long long)id * c.Hkv + hk) << c.page_log2) + (at & mask) - skip : 0;
      const unsigned bytes = ok ? (unsigned)((skip + left) * c.D) : 0u;
      to(buffer_of(static_cast<const unsigned char*>(c.k) + row * c.D, bytes), buffer_of(static_cast<const unsigned char*>(c.v) + row * c.D, bytes));
    };
    auto ask = [&](int x) __attribute__((always_inline)) {
      return [&, x](u32x4 k, u32x4 v) __attribute__((always_inline)) {
        buffer_to_lds16(k, off[x], k_at + x * 1024);
        buffer_to_lds16(v, off[x], v_at + x * 1024);
      };
    };
    if constexpr (EACH >= 1) {
#pragma unroll
      for (int p = 0; p < IDS; ++p)
        rows(ids[p], j + p * PART, 0, PART, [&](u32x4 k, u32x4 v) __attribute__((always_inline)) {
#pragma unroll
          for (int x = p * EACH; x < (p + 1) * EACH; ++x)
            if (RPI * CH == 64 || lane < RPI * CH) ask(x)(k, v);
        });
    } else {
#pragma unroll
      for (int x = 0; x < REQ; ++x) {
        if (part == RPI) {
          if (RPI * CH == 64 || lane < RPI * CH) rows(ids[x * RPI / PART], j + x * RPI, 0, RPI, ask(x));
        } else {   // several pages a request: the lanes of each from its own
#pragma unroll
          for (int p = 0; p < RPI / PART; ++p)
            if (p * PART % part == 0 && (lane / CH) / part == p * PART / part)
              rows(ids[x * RPI / PART + p], j + x * RPI + p * PART, p * PART, part, ask(x));
        }
      }
    }
    if (lane < ROWS / 4) {
      const int g = (lane >> 2) * 2 + (lane & 1);
      int id = ids[0];
#pragma unroll
      for (int x = 1; x < IDS; ++x) id = g >= x * PART / 8 ? ids[x] : id;
      const bool ok = (unsigned)id < (unsigned)c.P;
      const long long s = ok ? (((long long)id * c.Hkv + hk) << (c.page_log2 - a.block_log2)) + (((j + g * 8) & mask) >> a.block_log2) : 0;
      global_to_lds4((lane & 2 ? a.v_scale : a.k_scale) + s, s_at);
    }
  }
};

// How a lane reads tiles as the A operand of its products
template <int DP>
struct TileReader8 {
  static constexpr int CH = DP / 16, KS = DP / 16, DB = DP / 32;
  unsigned row, cols, ks;
  __device__ __forceinline__ explicit TileReader8(int lane) {
    const int l32 = lane & 31, h = lane >> 5, k = (lane & 15) >> 1, r = k < 4 ? 4 * h + k : 4 + 4 * h + k;
    row = l32 * DP + ((h ^ swz8<CH>(l32)) << 4);
    cols = r * DP + (((l32 >> 4) ^ swz8<CH>(r)) << 4) + (lane & 1) * 8;
    ks = (l32 >> 4) * 16 + ((l32 >> 3) & 1) * 4;
  }
  // a product over the width: row lane % 32, columns 32 i + 16 (lane / 32) and on; two operands of eight columns
  __device__ __forceinline__ u32x4 rows(unsigned at, int i) const {
    return __builtin_bit_cast(u32x4, lds_read16(lds_at((at + row) ^ (i << 5))));
  }
  __device__ __forceinline__ float key_scale(unsigned at) const {
    return *reinterpret_cast<const __attribute__((address_space(3))) float*>(lds_at(at + ks));
  }
  // a product over the rows, of the transpose: columns 32 db + lane % 32, rows 16 s + {4h .. 4h+3, 8+4h .. 8+4h+3}
  __device__ __forceinline__ u32x2 columns(unsigned at, int s, int db) const {
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(
        (__attribute__((address_space(3))) i32x2*)(lds_at(((at + cols) ^ (db << 5)) + s * 16 * DP))));
  }
  __device__ __forceinline__ u32x2 value_scales(unsigned at, int s) const {   // of rows 16 s .. +7 and the next eight
    return *reinterpret_cast<const __attribute__((address_space(3))) u32x2*>(lds_at(at + s * 16 + 8));
  }
};

// max and sum over the four lanes that share a row of 16
__device__ __forceinline__ float quarter_max(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return half_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float quarter_sum(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return half_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// A number of 24 bits as a sum of bf16 numbers, the largest first: products with them and with e4m3 numbers are exact
template <int NP>
__device__ __forceinline__ void split_bf16(float x, __bf16* part) {
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    part[i] = (__bf16)x;
    x -= (float)part[i];
  }
}

// Probabilities r and r + 1 of a block, of the operands p
template <int NP>
__device__ __forceinline__ void split_pair(float a, float b, int r, bf16x8 (*p)[2]) {
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const bf16x2 c = {(__bf16)a, (__bf16)b};
    p[i][r >> 3][r & 7] = c[0];
    p[i][r >> 3][(r & 7) + 1] = c[1];
    a -= (float)c[0];
    b -= (float)c[1];
  }
}

// Values that are NaN of items that not every row sees: 0 * NaN would make NaN of rows ahead of them. Of a tile with such items (the few that rows of
// a chunk end in) the codes are looked at ahead of the products: rows that see a NaN get it by a count, products of ones, and zeros take
// the codes' place. Without NaN it costs nothing that was measured (512 new items x up to 10000, 16 users of 128 205 us without and 199 so, when a lane's masks
// had become shifts of one register; 300 x up to 3000, 24 of 64 48.6 and 48.9; 4 x 2000, 256 of 128 35.1 and 35.0).
__device__ __forceinline__ u32x2 nan_codes(u32x2 w) {   // the top bit of each of 8 codes that is NaN
  return u32x2{((w[0] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u, ((w[1] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u};
}
__device__ __forceinline__ bf16x8 ones_at(u32x2 nan) { return wide8((nan[0] >> 7) * 0x38u, (nan[1] >> 7) * 0x38u, 1.0f, 1.0f); }   // (code 0x38 is 1)
template <int BYTES>   // of a wave, from `at` on
__device__ __forceinline__ bool any_nan(unsigned at, int lane) {
  unsigned any = 0;
#pragma unroll
  for (int x = 0; x < BYTES / 512; ++x) {
    const u32x2 nan = nan_codes(*reinterpret_cast<const __attribute__((address_space(3))) u32x2*>(lds_at(at + (x * 64 + lane) * 8)));
    any |= nan[0] | nan[1];
  }
  return __any(any != 0);
}
template <int BYTES>
__device__ __forceinline__ void clear_nan(unsigned at, int lane) {
#pragma unroll
  for (int x = 0; x < BYTES / 512; ++x) {
    auto* p = reinterpret_cast<__attribute__((address_space(3))) u32x2*>(lds_at(at + (x * 64 + lane) * 8));
    const u32x2 w = *p, nan = nan_codes(w);
    *p = u32x2{w[0] & ~((nan[0] >> 7) * 0xffu), w[1] & ~((nan[1] >> 7) * 0xffu)};
  }
  asm volatile("" ::: "memory");
}
// Of 32 items; seen: the place of the last that the lane's row sees, less 4 (lane / 32). (The barriers keep the counts of one piece of the columns at a time.)
template <int DP>
__device__ __forceinline__ void nan_seen32(const TileReader8<DP>& read, unsigned at_v, int seen, f32x16* acc) {
  bf16x8 sees[2];
#pragma unroll
  for (int r = 0; r < 16; ++r) sees[r >> 3][r & 7] = (__bf16)(8 * (r >> 2) + (r & 3) <= seen ? 1.0f : 0.0f);
#pragma unroll
  for (int db = 0; db < DP / 32; ++db) {
    f32x16 count = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < 2; ++s) count = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ones_at(nan_codes(read.columns(at_v, s, db))), sees[s], count, 0, 0, 0);
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[db][r] = count[r] > 0.0f ? __builtin_nanf("") : acc[db][r];
    __builtin_amdgcn_sched_barrier(0);
  }
}

// A row's sum in units of 2^m, as the logarithm to 2: nothing seen -inf; a sum that is NaN stays that, and is +inf in a part of a row, of which
// the join makes NaN whatever the other parts hold
__device__ __forceinline__ float log_sum(float m, float sum, bool in_part) {
  return sum == 0.0f ? -INFINITY : sum != sum && in_part ? INFINITY : m + log2f(sum);
}

// Where the maximum of a row is raised: probabilities may stand up to 2^8 above it meanwhile, sums and outputs are in its units
constexpr float MAX_SLACK = 8.0f;

// The query of a lane's row as B operands in the order of TileReader8::rows; bf16 as it is, fp32 in three parts
template <int DP, int NP, typename T>
__device__ __forceinline__ void load_query(const T* qr, int D, int h, bf16x8 (*q)[DP / 16]) {
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) {
    const int d = (2 * (s >> 1) + h) * 16 + (s & 1) * 8;
    if constexpr (NP == 1) {
      u32x4 raw = {0u, 0u, 0u, 0u};
      if (d < D) raw = *reinterpret_cast<const u32x4*>(qr + d);
      q[0][s] = __builtin_bit_cast(bf16x8, raw);
    } else {
      u32x4 raw[2] = {u32x4{0u, 0u, 0u, 0u}, u32x4{0u, 0u, 0u, 0u}};
      if (d < D) {
        raw[0] = *reinterpret_cast<const u32x4*>(qr + d);
        raw[1] = *reinterpret_cast<const u32x4*>(qr + d + 4);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        __bf16 part[NP];
        split_bf16<NP>(__uint_as_float(raw[j >> 2][j & 3]), part);
#pragma unroll
        for (int i = 0; i < NP; ++i) q[i][s][j] = part[i];
      }
    }
  }
}

}  // namespace laser
