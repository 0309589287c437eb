// Gradients of attention among the items of histories on the matrix cores (bf16).
//
//   p = exp2(c q.k - lse), dp = d_o . v, ds = p (dp - delta), delta = d_o . o
// Two kernels, each of which recomputes p and dp, so that every sum is one workgroup's and its order is fixed:
//   dq: a wave owns 32 rows (token and head, packed as in the forward pass) and walks the items they see.
//       Sc^T = K Q^T, dP^T = V dO^T (rows in lanes: lse and delta are one register each), dQ^T += K^T dS^T
//   dk, dv: a wave owns 32 items of a key-value head and walks the rows that see them, of all its query heads.
//       Sc = Q K^T, dP = dO V^T (items in lanes), dV^T += dO^T P, dK^T += Q^T dS
// Seven products where five would do with one kernel, which would have to add one of the gradients up across workgroups.
// p and ds are rounded to bf16 ahead of their products, which take their operands so (in 32 bits they would take 16 times as long); the sums are
// fp32. dq and dk are then off by 1.43 to 1.45 times what their own rounding costs, dv by 1.37 (root mean square).
//
// Bound: as the forward pass, by products with their exponentials. Width 128: dq 380 us for 16 histories of 920 to 4000 items, 8 heads over
// 2 (900 TFLOP/s of its three products), dk and dv 560 (810 of their four), whose first items' workgroups run longest. Widths to 64
// over histories of 40 to 200 items are bound by memory: 47 and 50 us where their bytes take 40 each at a copy's rate.
#include "history_tile.h"

namespace laser {

struct BwdArgs {
  const unsigned short* q;
  const unsigned short* k;
  const unsigned short* v;
  const unsigned short* o;
  const unsigned short* go;
  long long qp, kp, vp;
  const int32_t* off;
  int N, T, L, H, Hkv, D, G;
  MulDiv by_group;       // / G
  Deal deal;
  float scale, gamma, inv_gamma;   // scale: log2(e) / gamma
  const float* lse;
  float* rows;           // [T,H,2]: -lse gamma and -delta, by the first kernel for the second
  unsigned short* dq;
  unsigned short* dk;
  unsigned short* dv;
  long long dqp, dkp, dvp;
};

// The waves are NG groups of NW, which own the same rows, take the tiles in turn and are summed up at the end: where workgroups are few,
// the longest walk is what counts.
template <int DP, int NW, int NG>
__global__ __launch_bounds__(64 * NW * NG, 2) void history_dq_kernel(const BwdArgs a) {
  using Sh = TileShape<DP>;
  constexpr int KS = DP / 16, DB = DP / 32, ROWS = NW * 32, OP = DP * 2 + 16, STAGE = 2 * Sh::BYTES, PATCH = NW * 32 * OP;
  constexpr int JOIN = NG > 1 ? ROWS * DP * 4 : 0, LAST = PATCH > JOIN ? PATCH : JOIN, TILES = 2 * NG * STAGE;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[TILES > LAST ? TILES : LAST];
  const unsigned lds = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem);
  const Place place = place_of(a.deal, blockIdx.x);
  if (place.rank >= a.deal.tiles) return;
  const int tile = a.deal.tiles - 1 - place.rank;   // (the longest first)
  const int n_seq = place.pair / a.Hkv, hk = place.pair - n_seq * a.Hkv;
  const CandRange cr = cand_range(a.off, n_seq, a.L, a.T);
  const int n = cr.count, rows = n * a.G, row0 = tile * ROWS;
  if (row0 >= rows) return;
  const int wave_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = wave_all / NW, wave = wave_all % NW;
  const int lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;

  bf16x8 qreg[KS], greg[KS];
  float lse2, delta;
  int last;
  const int first = row0 + wave * 32;
  {
    int r = first + l32;
    r = r < rows ? r : rows - 1;
    last = (int)a.by_group.div(r);
    const int head = hk * a.G + r - last * a.G;
    const size_t tok = (size_t)cr.first + last, at = (tok * a.H + head) * a.D;
    float sum = 0.0f;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int c = s * 16 + h * 8;
      u32x4 x = {0u, 0u, 0u, 0u}, y = x, z = x;
      if (c < a.D) {
        x = *reinterpret_cast<const u32x4*>(a.q + tok * a.qp + (size_t)head * a.D + c);
        y = *reinterpret_cast<const u32x4*>(a.go + at + c);
        z = *reinterpret_cast<const u32x4*>(a.o + at + c);
      }
      qreg[s] = __builtin_bit_cast(bf16x8, x);
      greg[s] = __builtin_bit_cast(bf16x8, y);
      const bf16x8 o = __builtin_bit_cast(bf16x8, z);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fmaf((float)greg[s][e], (float)o[e], sum);
    }
    delta = half_sum(sum);
    lse2 = a.lse[tok * a.H + head] * LOG2E;
  }
  const int wave_first = __builtin_amdgcn_readlane(last, 0), wave_last = __builtin_amdgcn_readlane(last, 31);
  // o is as stored, in bf16, and what that costs delta weighs most where a row sees few items (against dq, 2^-9 / sqrt of their number).
  // Rows that see one block have their delta from that block instead, as the sum of p dp.
  const bool one_block = wave_last < 32;
  const int end = (int)a.by_group.div(row0 + ROWS < rows ? row0 + ROWS - 1 : rows - 1) + 1;

  f32x16 acc[DB];
  const f32x16 zero = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = zero;
  TileReader<DP> read(lane);

  // A block of 32 items: scores, dp behind which the exponentials are made, then its share of dq. What is left without a product
  // beside it is the other wave's time.
  auto block = [&](int t0, int ib) __attribute__((always_inline)) {
    f32x16 sc, dp;
    unsigned ds[8];
    bf16x8 kf[KS], vf[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) kf[s] = read.rows(0, ib, s);
#pragma unroll
    for (int s = 0; s < KS; ++s) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s], qreg[s], s == 0 ? zero : sc, 0, 0, 0);
#pragma unroll
    for (int s = 0; s < KS; ++s) vf[s] = read.rows(Sh::BYTES, ib, s);
    __builtin_amdgcn_sched_barrier(0);
    if (t0 + 31 > wave_first) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (t0 + 8 * (r >> 2) + 4 * h + (r & 3) > last) sc[r] = -INFINITY;
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < KS; ++s) dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[s], greg[s], s == 0 ? zero : dp, 0, 0, 0);
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[r] = __builtin_amdgcn_exp2f(fmaf(sc[r], a.scale, -lse2));
#pragma unroll
    for (int x = 0; x < KS; ++x) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x402, 32 / KS, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (one_block) {
      float sum = 0.0f;
#pragma unroll
      for (int r = 0; r < 16; ++r) sum = fmaf(sc[r], dp[r], sum);
      delta = half_sum(sum);
    }
    bf16x8 kt[2][DB];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int db = 0; db < DB; ++db) kt[s][db] = read.cols(0, ib * 2 + s, db);
#pragma unroll
    for (int r = 0; r < 16; r += 2) ds[r >> 1] = pack_bf16(sc[r] * (dp[r] - delta), sc[r + 1] * (dp[r + 1] - delta));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const u32x4 b = {ds[s * 4], ds[s * 4 + 1], ds[s * 4 + 2], ds[s * 4 + 3]};
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kt[s][db], __builtin_bit_cast(bf16x8, b), acc[db], 0, 0, 0);
      }
  };

  PackedTiles<DP, NW> tiles;
  tiles.init(a.D, a.kp, a.vp, wave, lane);
  auto fetch = [&](int t0, unsigned at) __attribute__((always_inline)) {
    const size_t row = (size_t)(cr.first + t0);
    tiles.fetch(a.k + row * a.kp + (size_t)hk * a.D, a.v + row * a.vp + (size_t)hk * a.D, a.kp, a.vp, a.D, n - t0, at);
  };
  unsigned at = lds + group * 2 * STAGE, other = at + STAGE;
  if (group * TI < end) fetch(group * TI, at);
  for (int t0 = group * TI, turn = 0; turn < end; t0 += NG * TI, turn += NG * TI) {   // (every group the same number of turns)
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    barrier_lds();
    if (t0 + NG * TI < end) fetch(t0 + NG * TI, other);
    read.place(at);
    if (t0 <= wave_last) block(t0, 0);
    if (t0 + 32 <= wave_last) block(t0 + 32, 1);
    const unsigned x = at;
    at = other;
    other = x;
  }
  if (group == 0 && h == 0 && first + l32 < rows) {   // (a row that sees one block saw it in the first tile)
    const int head = hk * a.G + first + l32 - last * a.G;
    float* row = a.rows + ((size_t)(cr.first + last) * a.H + head) * 2;
    row[0] = -lse2 * LN2 * a.gamma;
    row[1] = -delta;
  }
  barrier_lds();
  if constexpr (NG > 1) {   // the other groups' sums to the first, lane by lane, in their order
    float* mine = reinterpret_cast<float*>(smem) + (size_t)wave * 32 * DP + lane;
#pragma unroll 1
    for (int g = 1; g < NG; ++g) {
      if (group == g) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) mine[(db * 16 + r) * 64] = acc[db][r];
      }
      __syncthreads();
      if (group == 0) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[db][r] += mine[(db * 16 + r) * 64];
      }
      __syncthreads();
    }
    if (group > 0) return;
  }
  store_block<DP>(acc, a.inv_gamma, smem + wave * 32 * OP, rows - first, a.D, lane, [&](int r) {
    const int i = (int)a.by_group.div(first + r), head = hk * a.G + first + r - i * a.G;
    return a.dq + (size_t)(cr.first + i) * a.dqp + (size_t)head * a.D;
  });
}

// RT rows a tile. The width 128 leaves no registers for the values at two waves a SIMD: they stay in LDS (V_LDS) and are read as operands.
// The first items of a long history have all its rows to walk, and such a workgroup would still run when the others are done: its waves
// are NG groups of NW, which own the same items, take the tiles in turn and are summed up at the end.
template <int DP, int NW, int NG, int RT>
__global__ __launch_bounds__(64 * NW * NG, 2) void history_dkv_kernel(const BwdArgs a) {
  using Sh = TileShape<DP>;
  constexpr bool V_LDS = DP > 64;
  constexpr int KS = DP / 16, DB = DP / 32, ITEMS = NW * 32, OP = DP * 2 + 16, HALF = RT * Sh::ROW, GROUPS = RT / Sh::RPI;
  constexpr int GPW = (GROUPS + NW - 1) / NW;
  constexpr int STAGE = 2 * HALF + 1024, VALUES = V_LDS ? ITEMS * Sh::ROW : 0;   // (1024: what a row brings, and whole lines)
  constexpr int PATCH = NW * 32 * OP, JOIN = NG > 1 ? ITEMS * DP * 4 : 0, LAST = PATCH > JOIN ? PATCH : JOIN, TILES = 2 * NG * STAGE + VALUES;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[TILES > LAST ? TILES : LAST];
  const unsigned lds = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem);
  const Place place = place_of(a.deal, blockIdx.x);
  if (place.rank >= a.deal.tiles) return;
  const int tile = place.rank, n_seq = place.pair / a.Hkv, hk = place.pair - n_seq * a.Hkv;   // (the first items have the most rows)
  const CandRange cr = cand_range(a.off, n_seq, a.L, a.T);
  const int n = cr.count, item0 = tile * ITEMS;
  if (item0 >= n) return;
  const int wave_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = wave_all / NW, wave = wave_all % NW;
  const int lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
  const int rows = n * a.G, first = item0 + wave * 32;

  // tiles of rows: queries, behind them d_o, behind them what the first kernel left of each row; rows behind the last read as zeros and
  // add nothing. Where a tile is a whole number of tokens, a lane's offsets are the same in every tile.
  const bool whole_tokens = RT % a.G == 0;
  const int head0 = hk * a.G;
  unsigned qoff[GPW], goff[GPW], soff;
  auto offsets = [&](int r0, int i0) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < GPW; ++x) {
      const int in = (wave + x * NW) * Sh::RPI + lane / Sh::CH, c = (lane % Sh::CH) ^ tile_swz<Sh::CH>(in), r = r0 + in;
      const int i = (int)a.by_group.div(r), head = r - i * a.G, tk = i - i0;
      qoff[x] = c * 8 < a.D ? (unsigned)((tk * (int)a.qp + head * a.D + c * 8) * 2) : NO_COLUMN;
      goff[x] = c * 8 < a.D ? (unsigned)(((tk * a.H + head) * a.D + c * 8) * 2) : NO_COLUMN;
    }
    const int r = r0 + (RT == 64 ? lane : l32), i = (int)a.by_group.div(r);
    soff = (unsigned)((i - i0) * a.H + r - i * a.G) * 8 + (RT == 64 ? wave : h) * 4;
  };
  constexpr int ROW_WAVES = RT == 64 ? 2 : 1;   // waves that ask for the rows' two numbers
  if (whole_tokens) offsets(0, 0);
  auto fetch = [&](int r0, unsigned at) __attribute__((always_inline)) {
    const int i0 = (int)a.by_group.div(r0);
    if (!whole_tokens) offsets(r0, i0);
    const size_t tok = (size_t)cr.first + i0;
    const int more = n - 1 - i0 < RT ? n - 1 - i0 : RT;   // whole tokens within reach behind the first
    const u32x4 qb = buffer_of(a.q + tok * a.qp + (size_t)head0 * a.D, (unsigned)((more * (int)a.qp + a.G * a.D) * 2));
    const u32x4 gb = buffer_of(a.go + (tok * a.H + head0) * a.D, (unsigned)((more * a.H + a.G) * a.D * 2));
#pragma unroll
    for (int x = 0; x < GPW; ++x) {
      const int g = wave + x * NW;
      if (GROUPS % NW != 0 && g >= GROUPS) break;
      buffer_to_lds16(qb, qoff[x], at + g * 1024);
      buffer_to_lds16(gb, goff[x], at + HALF + g * 1024);
    }
    if (wave < ROW_WAVES)
      buffer_to_lds4(buffer_of(a.rows + (tok * a.H + head0) * 2, (unsigned)(more * a.H + a.G) * 8), soff, at + 2 * HALF + wave * 256);
  };

  // From the last rows to the first that see an item: what runs beside this workgroup on the die then reads the same rows at about the
  // same time, wherever its own items begin.
  const int start = item0 * a.G / RT * RT;   // (rows before it see no item of this workgroup)
  const int turns = (rows - start + RT - 1) / RT;
  unsigned at = lds + group * 2 * STAGE, other = at + STAGE;
  if (turns - 1 - group >= 0) fetch(start + (turns - 1 - group) * RT, at);
  const unsigned values = lds + 2 * NG * STAGE + wave * 32 * Sh::ROW;
  if (V_LDS && group == 0) {   // 32 for each wave of a group
#pragma unroll
    for (int g = 0; g < 32 / Sh::RPI; ++g) {
      const int in = g * Sh::RPI + lane / Sh::CH, c = (lane % Sh::CH) ^ tile_swz<Sh::CH>(in);
      const int left = n - first;
      buffer_to_lds16(buffer_of(a.v + (size_t)(cr.first + (left > 0 ? first : 0)) * a.vp + (size_t)hk * a.D,
                                left > 0 ? (unsigned)((((left < 32 ? left : 32) - 1) * (int)a.vp + a.D) * 2) : 0u),
                      c * 8 < a.D ? (unsigned)(in * (int)a.vp * 2 + c * 16) : NO_COLUMN, values + g * 1024);
    }
  }

  bf16x8 kreg[KS], vreg[V_LDS ? 1 : KS];
  int from;   // the first row that sees this lane's item
  {
    int j = first + l32;
    j = j < n ? j : n - 1;
    from = j * a.G;
    const size_t tok = (size_t)cr.first + j;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int c = s * 16 + h * 8;
      u32x4 x = {0u, 0u, 0u, 0u}, y = x;
      if (c < a.D) {
        x = *reinterpret_cast<const u32x4*>(a.k + tok * a.kp + (size_t)hk * a.D + c);
        if constexpr (!V_LDS) y = *reinterpret_cast<const u32x4*>(a.v + tok * a.vp + (size_t)hk * a.D + c);
      }
      kreg[s] = __builtin_bit_cast(bf16x8, x);
      if constexpr (!V_LDS) vreg[s] = __builtin_bit_cast(bf16x8, y);
    }
  }
  const int wave_from = __builtin_amdgcn_readlane(from, 0), wave_to = __builtin_amdgcn_readlane(from, 31);
  const int floor = first < n ? wave_from - 32 : 0x7fffffff;   // blocks of rows from above this on see an item of the wave

  f32x16 dk[DB], dv[DB];
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  const f32x16 zero = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int db = 0; db < DB; ++db) dk[db] = dv[db] = zero;
  TileReader<DP> read(lane);
  const unsigned value_row = values + read.row;

  // A block of 32 rows. Scores start from -lse gamma and dp from -delta, so that p = exp2(scale x) and ds = p dp.
  auto block = [&](int r0, unsigned at, int rb) __attribute__((always_inline)) {
    f32x16 sc, dp;
    auto of_rows = [&](f32x16& x, int kind) __attribute__((always_inline)) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 y = *reinterpret_cast<const __attribute__((address_space(3))) f32x4*>(
            lds_at(at + 2 * HALF + kind * RT * 4 + (rb * 32 + g * 8 + h * 4) * 4));
#pragma unroll
        for (int e = 0; e < 4; ++e) x[g * 4 + e] = y[e];
      }
    };
    of_rows(sc, 0);
    {
      bf16x8 qf[KS];
#pragma unroll
      for (int s = 0; s < KS; ++s) qf[s] = read.rows(0, rb, s);
      of_rows(dp, 1);
#pragma unroll
      for (int s = 0; s < KS; ++s) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[s], kreg[s], sc, 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (r0 < wave_to) {   // rows that do not see all of the wave's items
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (r0 + 8 * (r >> 2) + 4 * h + (r & 3) < from) sc[r] = -INFINITY;
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const bf16x8 gf = read.rows(HALF, rb, s);
      bf16x8 vf;
      if constexpr (V_LDS) vf = lds_read16(lds_at(value_row ^ (s << 5)));
      else vf = vreg[s];
      dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(gf, vf, dp, 0, 0, 0);
    }
    unsigned p[8], ds[8];
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[r] = __builtin_amdgcn_exp2f(sc[r] * a.scale);
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      p[r] = pack_bf16(sc[2 * r], sc[2 * r + 1]);
      asm volatile("" : "+v"(p[r]));
    }
    __builtin_amdgcn_sched_group_barrier(0x100, V_LDS ? 4 : 2, 0);
#pragma unroll
    for (int x = 0; x < KS; ++x) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, V_LDS ? 2 : 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x402, 40 / KS, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    auto add = [&](f32x16* to, const unsigned* w, int more) __attribute__((always_inline)) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const u32x4 b = {w[s * 4], w[s * 4 + 1], w[s * 4 + 2], w[s * 4 + 3]};
          to[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read.cols(more, rb * 2 + s, db), __builtin_bit_cast(bf16x8, b), to[db], 0, 0, 0);
        }
    };
    add(dv, p, HALF);
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      ds[r] = pack_bf16(sc[2 * r] * dp[2 * r], sc[2 * r + 1] * dp[2 * r + 1]);
      asm volatile("" : "+v"(ds[r]));
    }
    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
    for (int x = 0; x < 2 * DB; ++x) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      __builtin_amdgcn_sched_group_barrier(0x402, 12 / DB, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    add(dk, ds, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
    for (int x = 0; x < 2 * DB; ++x) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  for (int t = turns - 1 - group, left = (turns + NG - 1) / NG; left > 0; --left, t -= NG) {
    const int r0 = start + t * RT;
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    barrier_lds();
    if (t >= NG) fetch(r0 - NG * RT, other);
    read.place(at);
    if (t >= 0) {
      if constexpr (RT == 64)
        if (r0 + 32 > floor) block(r0 + 32, at, 1);
      if (r0 > floor) block(r0, at, 0);
    }
    const unsigned x = at;
    at = other;
    other = x;
  }
  barrier_lds();
  if constexpr (NG > 1) {   // the other groups' sums to the first, lane by lane, in their order
    float* mine = reinterpret_cast<float*>(smem) + (size_t)wave * 32 * DP + lane;
#pragma unroll 1
    for (int g = 1; g < NG; ++g)
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        f32x16* acc = which == 0 ? dk : dv;
        if (group == g) {
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) mine[(db * 16 + r) * 64] = acc[db][r];
        }
        __syncthreads();
        if (group == 0) {
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[db][r] += mine[(db * 16 + r) * 64];
        }
        __syncthreads();
      }
    if (group > 0) return;
  }
  unsigned char* patch = smem + wave * 32 * OP;
  store_block<DP>(dk, a.inv_gamma, patch, n - first, a.D, lane,
                  [&](int r) { return a.dk + (size_t)(cr.first + first + r) * a.dkp + (size_t)hk * a.D; });
  store_block<DP>(dv, 1.0f, patch, n - first, a.D, lane,
                  [&](int r) { return a.dv + (size_t)(cr.first + first + r) * a.dvp + (size_t)hk * a.D; });
}

template <int DP, int NW, int NG, int RT = (DP > 64 ? 32 : 64)>
static laser_status dkv_launch(const BwdArgs& a, hipStream_t stream) {
  return launch_dealt(a, ((long long)a.L + NW * 32 - 1) / (NW * 32), 64 * NW * NG, [&](const BwdArgs& part, long long) {
    history_dkv_kernel<DP, NW, NG, RT><<<part.deal.grid, 64 * NW * NG, 0, stream>>>(part);
  });
}

template <int DP, int NW, int NG>
static laser_status dq_launch(const BwdArgs& a, hipStream_t stream) {
  return launch_dealt(a, ((long long)a.L * a.G + NW * 32 - 1) / (NW * 32), 64 * NW * NG, [&](const BwdArgs& part, long long) {
    history_dq_kernel<DP, NW, NG><<<part.deal.grid, 64 * NW * NG, 0, stream>>>(part);
  });
}

template <int DP>
static laser_status bwd_launch(const BwdArgs& a, hipStream_t stream) {
  const long long per = (long long)a.N * a.Hkv;
  // (before anything is launched; the forms with smaller tiles or more threads are those of few workgroups)
  if (sequences_a_launch(a.N, a.Hkv, ((long long)a.L * a.G + 127) / 128, 256) <= 0 ||
      sequences_a_launch(a.N, a.Hkv, ((long long)a.L + 127) / 128, 256) <= 0)
    return LASER_ERR_SHAPE;
  // dq has two groups (of four waves, width 128) or four (of two) where its workgroups of 128 rows would leave much of the machine idle,
  // and at width 128 also where there are a few more, but long. Forward and backward without and with: one history of 2894 items, 4 heads
  // of 32 over 2 (92 workgroups) 74 and 54 us; of 64 104 and 78; four of 300, 4 of 64 over 2 (40) 27.0 and 26.4; two of 2635, 4 of 128 over
  // one (166) 218 and 204; two of 4096, 8 of 128 over 2 (512) 359 and 334; but eight of 1000 (512, of 4000 rows) 107 and 110.
  const long long rows = (long long)a.L * a.G, row_workgroups = per * ((rows + 127) / 128);
  const bool few = row_workgroups <= 256 && rows >= 256;
  laser_status s;
  if constexpr (DP > 64) s = few || (row_workgroups <= 512 && rows >= 8192) ? dq_launch<DP, 4, 2>(a, stream) : dq_launch<DP, 4, 1>(a, stream);
  else s = few ? dq_launch<DP, 2, 4>(a, stream) : dq_launch<DP, 4, 1>(a, stream);
  if (s != LASER_OK) return s;
  // How many groups of waves share the items of a workgroup, by how many workgroups of 128 items there are and how many rows the first
  // has to walk. Forward and backward, one, two (of four waves) and four groups (of two): 16 histories up to 4096 of 8 heads of 128 over 2
  // (1024 workgroups) 1209, 1130, 1168 us; two of 4096 (128) 740, 585, 451; 64 up to 1024 of 4 heads over 4 (2048) 250, 277, 345; 256 up to
  // 200 of 4 over 2 (1024) 112, 126, 151. (Four groups at width 128 spill five registers, 24 bytes of scratch a lane, all the same.)
  // Few workgroups, four groups of two and one of four: 16 histories of 500, 2 of 64 over 2 (128) 24 and 26 us; four of 300, 4 over 2 (24)
  // 21.6 and 26.5; 64 of 200, 4 over 2 (256, of 400 rows) 34 and 28. Eight groups of one wave, where even those of 32 items are few: one of
  // 2894, 4 of 32 over 2 (182 of them) 44 us, with four groups of two 54; eight of 1000, 8 of 64 over 2 (512) 70 and 67.
  const long long workgroups = per * ((a.L + 127) / 128);
  if constexpr (DP <= 64)
    if (per * ((a.L + 31) / 32) <= 256 && rows >= 1024) return dkv_launch<DP, 1, 8, 32>(a, stream);
  if ((workgroups <= 256 && rows >= 1024) || (workgroups <= 128 && rows >= 384)) return dkv_launch<DP, 2, 4>(a, stream);
  if constexpr (DP > 64)
    if (workgroups < 1536 && rows >= 4096) return dkv_launch<DP, 4, 2>(a, stream);
  return dkv_launch<DP, 4, 1>(a, stream);
}

laser_status history_bwd_tile_launch(const HistoryBwdArgs& b) {
  const HistoryArgs& h = b.f;
  BwdArgs a{};
  a.q = static_cast<const unsigned short*>(h.q);
  a.k = static_cast<const unsigned short*>(h.k);
  a.v = static_cast<const unsigned short*>(h.v);
  a.o = static_cast<const unsigned short*>(h.o);
  a.go = static_cast<const unsigned short*>(b.go);
  a.qp = h.qp, a.kp = h.kp, a.vp = h.vp;
  a.off = h.off;
  a.N = h.N, a.T = h.T, a.L = h.L, a.H = h.H, a.Hkv = h.Hkv, a.D = h.D, a.G = h.H / h.Hkv;
  a.by_group = mul_div(a.G);
  a.scale = LOG2E / h.gamma;
  a.gamma = h.gamma;
  a.inv_gamma = 1.0f / h.gamma;
  a.lse = h.lse;
  a.rows = b.work;
  a.dq = static_cast<unsigned short*>(b.dq);
  a.dk = static_cast<unsigned short*>(b.dk);
  a.dv = static_cast<unsigned short*>(b.dv);
  a.dqp = b.dqp, a.dkp = b.dkp, a.dvp = b.dvp;
  if (a.D > 64) return bwd_launch<128>(a, h.stream);
  if (a.D > 32) return bwd_launch<64>(a, h.stream);
  return bwd_launch<32>(a, h.stream);
}

}  // namespace laser
