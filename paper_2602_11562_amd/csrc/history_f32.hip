// Attention among the items of histories in single precision, on the matrix cores' fp32 products: the forms of history_mfma.hip,
// history_backward.hip and cache_weights.hip, whose mathematics and layout of products they share.
//
// v_mfma_f32_32x32x2_f32 takes two steps of the contraction at a time, one from each half of the wave. Over the width a lane's 16-byte
// piece feeds four of them; over the items register r of a score block is, as it stands, the B operand for items 8 (r / 4) + r % 4 and
// four further, and the A operand is one float a lane, 32 columns side by side. Products take 16 times as long as bf16's, so tiles of
// 32 rows, no second tile of registers and no ordering by hand: everything else is behind them (a large product in this
// precision reaches 154 TFLOP/s on this card).
//
// Every kernel but the weights' has two forms. Wide: the four waves of a workgroup own 32 rows (items) each and share the tiles they walk.
// SPLIT: the workgroup owns 32, its waves take the tiles in turn, each through a place of its own, and are summed up at the end; four
// times the workgroups with a quarter of the way, for calls whose wide workgroups would not fill the machine.
#include "history_tile.h"

namespace laser {

constexpr int FI = 32;   // rows of a tile

typedef float f32x4 __attribute__((ext_vector_type(4)));

// A row of DP floats is CH pieces of 16 bytes; piece c of row r stands at place c ^ swz(r). Sixteen rows at one piece are in all banks,
// and so are 32 columns of two rows four apart (rows of 256 bytes and more).
template <int DP>
struct F32Tile {
  static constexpr int ROW = DP * 4, CH = DP / 4, RPI = 64 / CH, BYTES = FI * ROW;
  static __device__ __forceinline__ int swz(int r) {
    return CH >= 16 ? (r & 3) | ((r >> 3) & 1) << 2 | ((r >> 2) & 1) << 3 : (r >> 1) & 7;
  }
  // four steps over the width: row l32, pieces 2 a + h
  static __device__ __forceinline__ f32x4 rows(unsigned at, int a, int lane) {
    const int r = lane & 31;
    return *reinterpret_cast<const __attribute__((address_space(3))) f32x4*>(lds_at(at + r * ROW + (((2 * a + (lane >> 5)) ^ swz(r)) << 4)));
  }
  // a step over the rows: columns 32 db + l32 of rows 8 (r / 4) + r % 4 + 4 h
  static __device__ __forceinline__ float col(unsigned at, int r, int db, int lane) {
    const int row = 8 * (r >> 2) + (r & 3) + 4 * (lane >> 5), d = db * 32 + (lane & 31);
    return *reinterpret_cast<const __attribute__((address_space(3))) float*>(lds_at(at + row * ROW + (((d >> 2) ^ swz(row)) << 4) + (d & 3) * 4));
  }
};

struct F32Args {
  const float* q;
  const float* k;
  const float* v;
  long long qp, kp, vp;
  const int32_t* off;
  const int32_t* pages;
  const int32_t* lens;
  int N, T, L, C, H, Hkv, D, log2, P, max_pages, G, tiles, chunk, runs;
  MulDiv by_group;
  Deal deal;
  float scale, inv_gamma;
  bool causal, add;
  float* o;
  float* lse;
  float* work;
  float* weight;
  // backward
  const float* go;
  float* dq;
  float* dk;
  float* dv;
  long long dqp, dkp, dvp;
};

// Products over the width: x[row or item in lane] += tile rows . regs, four steps a piece
template <int DP>
__device__ __forceinline__ f32x16 over_width(unsigned at, const f32x4* regs, f32x16 x, int lane) {
#pragma unroll
  for (int a = 0; a < DP / 8; ++a) {
    const f32x4 t = F32Tile<DP>::rows(at, a, lane);
#pragma unroll
    for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_32x32x2f32(t[e], regs[a][e], x, 0, 0, 0);
  }
  return x;
}
// and over the tile's rows: acc[column, lane] += tile^T . w
template <int DP>
__device__ __forceinline__ void over_rows(unsigned at, const f32x16& w, f32x16* acc, int lane) {
#pragma unroll
  for (int r = 0; r < 16; ++r)
#pragma unroll
    for (int db = 0; db < DP / 32; ++db) acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(F32Tile<DP>::col(at, r, db, lane), w[r], acc[db], 0, 0, 0);
}
// 16-byte pieces 2 a + h of a row of D floats, zeros behind its end
template <int DP>
__device__ __forceinline__ void load_row(f32x4* regs, const float* row, int D, int h) {
#pragma unroll
  for (int a = 0; a < DP / 8; ++a) regs[a] = a * 8 < D ? *reinterpret_cast<const f32x4*>(row + a * 8 + h * 4) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
}
// A lane's row of the transposed accumulators: columns 32 db + 8 x + 4 h and on, times `by`
template <int DP>
__device__ __forceinline__ void store_row(float* row, const f32x16* acc, float by, int D, int h) {
#pragma unroll
  for (int db = 0; db < DP / 32; ++db)
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int c = db * 32 + x * 8 + h * 4;
      if (c < D) *reinterpret_cast<f32x4*>(row + c) = f32x4{acc[db][x * 4] * by, acc[db][x * 4 + 1] * by, acc[db][x * 4 + 2] * by, acc[db][x * 4 + 3] * by};
    }
}

__device__ __forceinline__ f32x16 splat(float x) { return f32x16{x, x, x, x, x, x, x, x, x, x, x, x, x, x, x, x}; }

// Requests for tiles of items, in eights of rows, which a page of eight or more holds together: of a shared tile wave w brings the
// eight w, of a tile of its own all four
template <int DP, bool PAGED, bool SPLIT>
struct F32Items {
  using Sh = F32Tile<DP>;
  static constexpr int EIGHTS = SPLIT ? 4 : 1, PER = 8 / Sh::RPI;
  unsigned koff[EIGHTS][PER], voff[EIGHTS][PER];
  int wave, ids[EIGHTS];
  __device__ __forceinline__ int row_of(int x) const { return SPLIT ? x * 8 : wave * 8; }
  __device__ __forceinline__ void init(const F32Args& a, int wave_, int lane) {
    wave = wave_;
#pragma unroll
    for (int x = 0; x < EIGHTS; ++x)
#pragma unroll
      for (int y = 0; y < PER; ++y) {
        const int in = y * Sh::RPI + lane / Sh::CH, c = (lane % Sh::CH) ^ Sh::swz(row_of(x) + in);
        koff[x][y] = c * 4 < a.D ? (unsigned)((in * (PAGED ? a.D : (int)a.kp) + c * 4) * 4) : NO_COLUMN;
        voff[x][y] = c * 4 < a.D ? (unsigned)((in * (PAGED ? a.D : (int)a.vp) + c * 4) * 4) : NO_COLUMN;
      }
  }
  __device__ __forceinline__ void look_up(const F32Args& a, const int32_t* table, int t0, int n) {
    if (PAGED)
#pragma unroll
      for (int x = 0; x < EIGHTS; ++x) {
        const int j = t0 + row_of(x);
        ids[x] = j < n ? scalar_int(table, j >> a.log2) : -1;
      }
  }
  // items t0 and on of n
  __device__ __forceinline__ void fetch(const F32Args& a, size_t first, int hk, int t0, int n, unsigned at) const {
#pragma unroll
    for (int x = 0; x < EIGHTS; ++x) {
      const int j = t0 + row_of(x);
      int left = n - j < 8 ? n - j : 8;
      const float *k, *v;
      if constexpr (PAGED) {
        if ((unsigned)ids[x] >= (unsigned)a.P) left = 0;
        const size_t row = left > 0 ? (((size_t)ids[x] * a.Hkv + hk) << a.log2) + (j & ((1 << a.log2) - 1)) : 0;
        k = a.k + row * a.D;
        v = a.v + row * a.D;
      } else {
        const size_t row = left > 0 ? first + j : first;
        k = a.k + row * a.kp + (size_t)hk * a.D;
        v = a.v + row * a.vp + (size_t)hk * a.D;
      }
      const int kp = PAGED ? a.D : (int)a.kp, vp = PAGED ? a.D : (int)a.vp;
      const u32x4 kb = buffer_of(k, left > 0 ? (unsigned)(((left - 1) * kp + a.D) * 4) : 0u);
      const u32x4 vb = buffer_of(v, left > 0 ? (unsigned)(((left - 1) * vp + a.D) * 4) : 0u);
      const unsigned to = at + row_of(x) * Sh::ROW;
#pragma unroll
      for (int y = 0; y < PER; ++y) {
        buffer_to_lds16(kb, koff[x][y], to + y * 1024);
        buffer_to_lds16(vb, voff[x][y], to + Sh::BYTES + y * 1024);
      }
    }
  }
};

// SPLIT: the waves' accumulators in LDS, [column][32 rows], row r of column d at r ^ d % 32, in the place of each wave's tile
template <int DP>
__device__ __forceinline__ void leave(unsigned char* place, const f32x16* acc, int lane) {
  float* out = reinterpret_cast<float*>(place);
#pragma unroll
  for (int db = 0; db < DP / 32; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int d = 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
      out[(db * 32 + d) * 32 + ((lane & 31) ^ d)] = acc[db][r];
    }
}
__device__ __forceinline__ float left_by(const unsigned char* place, int r, int d) {
  return reinterpret_cast<const float*>(place)[d * 32 + (r ^ (d & 31))];
}

template <int DP, bool PAGED, bool SPLIT>
__global__ __launch_bounds__(256, SPLIT && DP > 64 ? 1 : 2) void history_f32_kernel(const F32Args a) {
  using Sh = F32Tile<DP>;
  constexpr int DB = DP / 32, ROWS = SPLIT ? 32 : 128, STAGE = 2 * Sh::BYTES;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[(SPLIT ? 4 : 2) * STAGE];
  __shared__ float join_m[SPLIT ? 4 : 1][32], join_l[SPLIT ? 4 : 1][32];
  const unsigned lds = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem);
  const Place place = place_of(a.deal, blockIdx.x);
  if (place.rank >= a.deal.tiles) return;
  int tile = place.rank, run = 0;
  if (PAGED && a.runs > 1) {
    run = tile / a.tiles;
    tile -= run * a.tiles;
  }
  tile = a.tiles - 1 - tile;   // (the longest first)
  const int n_seq = place.pair / a.Hkv, hk = place.pair - n_seq * a.Hkv;
  const CandRange cr = cand_range(a.off, n_seq, a.C, a.T);
  const int rows = cr.count * a.G, row0 = tile * ROWS;
  if (row0 >= rows) return;
  const int n = PAGED ? cache_len(a.lens, n_seq, a.L, a.max_pages, a.log2) : cr.count;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
  int end;   // one past the last item that a row of this workgroup sees
  {
    const int r = row0 + ROWS < rows ? row0 + ROWS - 1 : rows - 1;
    end = a.causal ? n - cr.count + (int)a.by_group.div(r) + 1 : n;
  }
  const bool joined = PAGED && a.runs > 1 && n > a.chunk;   // others write their part of the result too
  int begin = 0;
  if (PAGED && a.runs > 1) {
    begin = run * a.chunk;
    if (run > 0 && begin >= end) return;
    end = end < begin + a.chunk ? end : begin + a.chunk;
  }
  const int32_t* table = PAGED ? a.pages + (size_t)n_seq * a.max_pages : nullptr;
  F32Items<DP, PAGED, SPLIT> items;
  items.init(a, wave, lane);
  const int first_tile = begin + (SPLIT ? wave * FI : 0), stride = SPLIT ? 4 * FI : FI;
  unsigned at = lds + (SPLIT ? wave * STAGE : 0), other = at + STAGE;
  if (end > first_tile) {
    items.look_up(a, table, first_tile, n);
    items.fetch(a, (size_t)cr.first, hk, first_tile, n, at);
    items.look_up(a, table, first_tile + stride, n);
  }

  const int mine = row0 + (SPLIT ? 0 : wave * 32) + l32, r = mine < rows ? mine : rows - 1, i = (int)a.by_group.div(r), head = hk * a.G + r - i * a.G;
  const size_t tok = (size_t)cr.first + i;
  const bool busy = SPLIT || row0 + wave * 32 < rows;
  const int last = a.causal ? n - cr.count + i : n - 1;
  const int wave_first = __builtin_amdgcn_readlane(last, 0), wave_last = busy ? __builtin_amdgcn_readlane(last, 31) : -1;
  f32x4 q[DP / 8];
  load_row<DP>(q, a.q + tok * a.qp + (size_t)head * a.D, a.D, h);
  bool whole_pages = true;
  if constexpr (PAGED) {
    bool bad = false;
    if (end > begin)
      for (int x = (begin >> a.log2) + lane; x <= (end - 1) >> a.log2; x += 64) bad |= (unsigned)table[x] >= (unsigned)a.P;
    whole_pages = __ballot(bad) == 0;
  }
  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = splat(0.0f);
  float m = -INFINITY, l = 0.0f;
  for (int t0 = first_tile; t0 < end; t0 += stride) {
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    if constexpr (!SPLIT) {
      barrier_lds();
      if (t0 + FI < end) {
        items.fetch(a, (size_t)cr.first, hk, t0 + FI, n, other);
        items.look_up(a, table, t0 + 2 * FI, n);
      }
    } else {
      asm volatile("" ::: "memory");
    }
    if (t0 <= wave_last) {
      f32x16 sc = over_width<DP>(at, q, splat(0.0f), lane);
      if (!whole_pages || t0 + FI - 1 > wave_first || t0 + FI > n) {
        bool in = l32 < n - t0;
        if (PAGED && !whole_pages) in = in && (unsigned)table[(t0 + (in ? l32 : 0)) >> a.log2] < (unsigned)a.P;
        const unsigned there = (unsigned)__ballot(in) >> (4 * h);
        const int seen = last - t0 - 4 * h;
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const int i0 = 8 * (x >> 2) + (x & 3);
          if (i0 > seen || !((there >> i0) & 1)) sc[x] = -INFINITY;
        }
      }
      float top = sc[0];
#pragma unroll
      for (int x = 1; x < 16; ++x) top = fmaxf(top, sc[x]);
      top = half_max(top) * a.scale;
      if (__any(top > m)) {
        const float next = fmaxf(m, top), c = next == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - next);
        m = next;
        l *= c;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int x = 0; x < 16; ++x) acc[db][x] *= c;
      }
      const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        sc[x] = __builtin_amdgcn_exp2f(fmaf(sc[x], a.scale, -base));
        l += sc[x];
      }
      over_rows<DP>(at + Sh::BYTES, sc, acc, lane);
    }
    if constexpr (SPLIT) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the tile has been read: its place may be asked for again
      if (t0 + stride < end) {
        items.fetch(a, (size_t)cr.first, hk, t0 + stride, n, at);
        items.look_up(a, table, t0 + 2 * stride, n);
      }
    } else {
      const unsigned x = at;
      at = other;
      other = x;
    }
  }
  if constexpr (SPLIT) {
    l = half_sum(l);
    leave<DP>(smem + wave * STAGE, acc, lane);
    if (h == 0) {
      join_m[wave][l32] = m;
      join_l[wave][l32] = l;
    }
    __syncthreads();
    const int here = rows - row0 < 32 ? rows - row0 : 32;
    for (int e = threadIdx.x; e < here * a.D; e += 256) {
      const int x = e / a.D, d = e - x * a.D;
      float top = -INFINITY, sum = 0.0f, o = 0.0f;
#pragma unroll
      for (int w = 0; w < 4; ++w) top = fmaxf(top, join_m[w][x]);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float mw = join_m[w][x], c = mw == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mw - top);
        sum = fmaf(join_l[w][x], c, sum);
        o = fmaf(left_by(smem + w * STAGE, x, d), c, o);
      }
      const float by = sum > 0.0f ? 1.0f / sum : 0.0f, z = sum > 0.0f ? top + log2f(sum) : -INFINITY;
      const int tk = (int)a.by_group.div(row0 + x);
      const size_t to = (size_t)(cr.first + tk) * a.H + hk * a.G + row0 + x - tk * a.G;
      if (joined) {
        const size_t all = (size_t)a.T * a.H;
        a.work[(run * all + to) * a.D + d] = o * by;
        if (d == 0) a.work[a.runs * all * a.D + run * all + to] = z;
      } else {
        a.o[to * a.D + d] = o * by;
        if (d == 0 && a.lse != nullptr) a.lse[to] = z * LN2;
      }
    }
    return;
  }
  if (mine >= rows) return;
  const float sum = half_sum(l), inv = sum > 0.0f ? 1.0f / sum : 0.0f, z = sum > 0.0f ? m + log2f(sum) : -INFINITY;
  const size_t row = tok * a.H + head;
  if (joined) {
    const size_t all = (size_t)a.T * a.H;
    store_row<DP>(a.work + (run * all + row) * a.D, acc, inv, a.D, h);
    if (h == 0) a.work[a.runs * all * a.D + run * all + row] = z;
  } else {
    store_row<DP>(a.o + row * a.D, acc, inv, a.D, h);
    if (h == 0 && a.lse != nullptr) a.lse[row] = z * LN2;
  }
}

template <int DP, bool SPLIT>
__global__ __launch_bounds__(256, 1) void history_dq_f32_kernel(const F32Args a) {
  using Sh = F32Tile<DP>;
  constexpr int DB = DP / 32, ROWS = SPLIT ? 32 : 128, STAGE = 2 * Sh::BYTES;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[(SPLIT ? 4 : 2) * STAGE];
  const unsigned lds = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem);
  const Place place = place_of(a.deal, blockIdx.x);
  if (place.rank >= a.deal.tiles) return;
  const int tile = a.deal.tiles - 1 - place.rank, n_seq = place.pair / a.Hkv, hk = place.pair - n_seq * a.Hkv;
  const CandRange cr = cand_range(a.off, n_seq, a.L, a.T);
  const int n = cr.count, rows = n * a.G, row0 = tile * ROWS;
  if (row0 >= rows) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
  const int end = (int)a.by_group.div(row0 + ROWS < rows ? row0 + ROWS - 1 : rows - 1) + 1;
  F32Items<DP, false, SPLIT> items;
  items.init(a, wave, lane);
  const int first_tile = SPLIT ? wave * FI : 0, stride = SPLIT ? 4 * FI : FI;
  unsigned at = lds + (SPLIT ? wave * STAGE : 0), other = at + STAGE;
  if (end > first_tile) items.fetch(a, (size_t)cr.first, hk, first_tile, n, at);

  const int mine = row0 + (SPLIT ? 0 : wave * 32) + l32, r = mine < rows ? mine : rows - 1, last = (int)a.by_group.div(r), head = hk * a.G + r - last * a.G;
  const size_t tok = (size_t)cr.first + last, row = tok * a.H + head;
  const int wave_first = __builtin_amdgcn_readlane(last, 0);
  const int wave_last = SPLIT || row0 + wave * 32 < rows ? __builtin_amdgcn_readlane(last, 31) : -1;
  f32x4 q[DP / 8], go[DP / 8], o[DP / 8];
  load_row<DP>(q, a.q + tok * a.qp + (size_t)head * a.D, a.D, h);
  load_row<DP>(go, a.go + row * a.D, a.D, h);
  load_row<DP>(o, a.o + row * a.D, a.D, h);
  float delta = 0.0f;
#pragma unroll
  for (int x = 0; x < DP / 8; ++x)
#pragma unroll
    for (int e = 0; e < 4; ++e) delta = fmaf(go[x][e], o[x][e], delta);
  delta = half_sum(delta);
  const float lse2 = a.lse[row] * LOG2E;
  if (h == 0 && mine < rows && (!SPLIT || wave == 0)) {
    a.work[row * 2] = -lse2;
    a.work[row * 2 + 1] = -delta;
  }
  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = splat(0.0f);
  for (int t0 = first_tile; t0 < end; t0 += stride) {
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    if constexpr (!SPLIT) {
      barrier_lds();
      if (t0 + FI < end) items.fetch(a, (size_t)cr.first, hk, t0 + FI, n, other);
    } else {
      asm volatile("" ::: "memory");
    }
    if (t0 <= wave_last) {
      f32x16 sc = over_width<DP>(at, q, splat(0.0f), lane);
      const f32x16 dp = over_width<DP>(at + Sh::BYTES, go, splat(-delta), lane);
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        sc[x] = __builtin_amdgcn_exp2f(fmaf(sc[x], a.scale, -lse2)) * dp[x];
        if (t0 + FI - 1 > wave_first && t0 + 8 * (x >> 2) + 4 * h + (x & 3) > last) sc[x] = 0.0f;
      }
      over_rows<DP>(at, sc, acc, lane);
    }
    if constexpr (SPLIT) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (t0 + stride < end) items.fetch(a, (size_t)cr.first, hk, t0 + stride, n, at);
    } else {
      const unsigned x = at;
      at = other;
      other = x;
    }
  }
  if constexpr (SPLIT) {
    leave<DP>(smem + wave * STAGE, acc, lane);
    __syncthreads();
    const int here = rows - row0 < 32 ? rows - row0 : 32;
    for (int e = threadIdx.x; e < here * a.D; e += 256) {
      const int x = e / a.D, d = e - x * a.D, tk = (int)a.by_group.div(row0 + x);
      float sum = 0.0f;
#pragma unroll
      for (int w = 0; w < 4; ++w) sum += left_by(smem + w * STAGE, x, d);
      a.dq[(size_t)(cr.first + tk) * a.dqp + (size_t)(hk * a.G + row0 + x - tk * a.G) * a.D + d] = sum * a.inv_gamma;
    }
    return;
  }
  if (mine < rows) store_row<DP>(a.dq + tok * a.dqp + (size_t)head * a.D, acc, a.inv_gamma, a.D, h);
}

// Requests for tiles of a group's rows, of one tensor: `pitch` between tokens of p (at the tile's first token i0 and the group's first
// head), `more` tokens within reach behind the first; the eight `eight` of the tile
template <int DP>
__device__ __forceinline__ void fetch_rows(const F32Args& a, const float* p, int pitch, int r0, int i0, int more, unsigned at, int eight, int lane) {
  using Sh = F32Tile<DP>;
  const u32x4 b = buffer_of(p, (unsigned)((more * pitch + a.G * a.D) * 4));
#pragma unroll
  for (int x = 0; x < 8 / Sh::RPI; ++x) {
    const int in = eight * 8 + x * Sh::RPI + lane / Sh::CH, c = (lane % Sh::CH) ^ Sh::swz(in), r = r0 + in;
    const int i = (int)a.by_group.div(r), head = r - i * a.G;
    buffer_to_lds16(b, c * 4 < a.D ? (unsigned)(((i - i0) * pitch + head * a.D + c * 4) * 4) : NO_COLUMN, at + eight * 8 * Sh::ROW + x * 1024);
  }
}

template <int DP, bool SPLIT>
__global__ __launch_bounds__(256, 1) void history_dkv_f32_kernel(const F32Args a) {
  using Sh = F32Tile<DP>;
  constexpr int DB = DP / 32, ITEMS = SPLIT ? 32 : 128, STAGE = 2 * Sh::BYTES + 1024;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[(SPLIT ? 4 : 2) * STAGE];
  const unsigned lds = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem);
  const Place place = place_of(a.deal, blockIdx.x);
  if (place.rank >= a.deal.tiles) return;
  const int tile = place.rank, n_seq = place.pair / a.Hkv, hk = place.pair - n_seq * a.Hkv;
  const CandRange cr = cand_range(a.off, n_seq, a.L, a.T);
  const int n = cr.count, item0 = tile * ITEMS;
  if (item0 >= n) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
  const int rows = n * a.G, first = item0 + (SPLIT ? 0 : wave * 32), head0 = hk * a.G;
  auto fetch = [&](int r0, unsigned at) {
    const int i0 = (int)a.by_group.div(r0), more = n - 1 - i0 < FI ? n - 1 - i0 : FI;
    const size_t tok = (size_t)cr.first + i0;
#pragma unroll
    for (int x = 0; x < (SPLIT ? 4 : 1); ++x) {
      const int eight = SPLIT ? x : wave;
      fetch_rows<DP>(a, a.q + tok * a.qp + (size_t)head0 * a.D, (int)a.qp, r0, i0, more, at, eight, lane);
      fetch_rows<DP>(a, a.go + (tok * a.H + head0) * a.D, a.H * a.D, r0, i0, more, at + Sh::BYTES, eight, lane);
    }
    if (SPLIT || wave == 0) {
      const int r = r0 + l32, i = (int)a.by_group.div(r);
      buffer_to_lds4(buffer_of(a.work + (tok * a.H + head0) * 2, (unsigned)(more * a.H + a.G) * 8),
                     (unsigned)((i - i0) * a.H + r - i * a.G) * 8 + h * 4, at + 2 * Sh::BYTES);
    }
  };
  const int start = item0 * a.G / FI * FI, turns = (rows - start + FI - 1) / FI;
  const int first_turn = turns - 1 - (SPLIT ? wave : 0), stride = SPLIT ? 4 : 1;
  unsigned at = lds + (SPLIT ? wave * STAGE : 0), other = at + STAGE;
  if (first_turn >= 0) fetch(start + first_turn * FI, at);
  const int mine = first + l32, j = mine < n ? mine : n - 1, from = j * a.G;
  const size_t item = (size_t)cr.first + j;
  const int wave_from = __builtin_amdgcn_readlane(from, 0);
  const int floor = first < n ? wave_from - 32 : 0x7fffffff;
  f32x4 k[DP / 8], v[DP / 8];
  load_row<DP>(k, a.k + item * a.kp + (size_t)hk * a.D, a.D, h);
  load_row<DP>(v, a.v + item * a.vp + (size_t)hk * a.D, a.D, h);
  f32x16 dk[DB], dv[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dk[db] = dv[db] = splat(0.0f);
  for (int t = first_turn; t >= 0; t -= stride) {
    const int r0 = start + t * FI;
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    if constexpr (!SPLIT) {
      barrier_lds();
      if (t > 0) fetch(r0 - FI, other);
    } else {
      asm volatile("" ::: "memory");
    }
    if (r0 > floor) {
      auto of_rows = [&](int g, int kind) {   // -lse log2(e), and -delta, of rows 8 g + 4 h and on
        return *reinterpret_cast<const __attribute__((address_space(3))) f32x4*>(lds_at(at + 2 * Sh::BYTES + kind * FI * 4 + (g * 8 + h * 4) * 4));
      };
      // (scores begin at zero: begun at the row's log-sum, their sum would lose what is below its half step, up to 2^-17 of p at width 128)
      f32x16 sc = over_width<DP>(at, k, splat(0.0f), lane), dp;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 d = of_rows(g, 1);
#pragma unroll
        for (int e = 0; e < 4; ++e) dp[g * 4 + e] = d[e];
      }
      dp = over_width<DP>(at + Sh::BYTES, v, dp, lane);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 z = of_rows(g, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int x = g * 4 + e;
          sc[x] = __builtin_amdgcn_exp2f(fmaf(sc[x], a.scale, z[e]));
          if (r0 + 8 * g + 4 * h + e < from) sc[x] = 0.0f;
          dp[x] *= sc[x];
        }
      }
      over_rows<DP>(at + Sh::BYTES, sc, dv, lane);
      over_rows<DP>(at, dp, dk, lane);
    }
    if constexpr (SPLIT) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (t >= stride) fetch(r0 - stride * FI, at);
    } else {
      const unsigned x = at;
      at = other;
      other = x;
    }
  }
  if constexpr (SPLIT) {
    leave<DP>(smem + wave * STAGE, dk, lane);
    leave<DP>(smem + wave * STAGE + Sh::BYTES, dv, lane);
    __syncthreads();
    const int here = n - item0 < 32 ? n - item0 : 32;
    for (int e = threadIdx.x; e < here * a.D; e += 256) {
      const int x = e / a.D, d = e - x * a.D;
      float k_sum = 0.0f, v_sum = 0.0f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        k_sum += left_by(smem + w * STAGE, x, d);
        v_sum += left_by(smem + w * STAGE + Sh::BYTES, x, d);
      }
      const size_t to = (size_t)(cr.first + item0 + x);
      a.dk[to * a.dkp + (size_t)hk * a.D + d] = k_sum * a.inv_gamma;
      a.dv[to * a.dvp + (size_t)hk * a.D + d] = v_sum;
    }
    return;
  }
  if (mine >= n) return;
  store_row<DP>(a.dk + item * a.dkp + (size_t)hk * a.D, dk, a.inv_gamma, a.D, h);
  store_row<DP>(a.dv + item * a.dvp + (size_t)hk * a.D, dv, 1.0f, a.D, h);
}

template <int DP>
__global__ __launch_bounds__(256, 2) void cache_weights_f32_kernel(const F32Args a) {
  using Sh = F32Tile<DP>;
  constexpr int STAGE = Sh::BYTES + 1024;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * STAGE];
  const unsigned lds = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem);
  const int u = blockIdx.y;
  const CandRange cr = cand_range(a.off, u, a.C, a.T);
  const int n = cache_len(a.lens, u, a.L, a.max_pages, a.log2), item0 = (int)((blockIdx.x + u) % gridDim.x) * 128;   // (see cache_weights.hip)
  if (item0 >= n) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
  const int rows = cr.count * a.G, first = item0 + wave * 32, mine = first + l32, j = mine < n ? mine : n - 1;
  const int page = a.pages[(size_t)u * a.max_pages + (j >> a.log2)], place = j & ((1 << a.log2) - 1);
  const bool there = (unsigned)page < (unsigned)a.P;
  const size_t slot = there ? (size_t)page : 0;
  int from = a.causal ? (j - (n - cr.count)) * a.G : 0, start = a.causal ? (item0 - (n - cr.count)) * a.G : 0;
  from = from < 0 ? 0 : from;
  start = start < 0 ? 0 : start / FI * FI;
  const int wave_from = __builtin_amdgcn_readlane(from, 0);
  auto fetch = [&](int hk, int r0, unsigned at) {
    const int i0 = (int)a.by_group.div(r0), more = cr.count - 1 - i0 < FI ? cr.count - 1 - i0 : FI;
    const size_t tok = (size_t)cr.first + i0, head0 = (size_t)hk * a.G;
    fetch_rows<DP>(a, a.q + tok * a.qp + head0 * a.D, (int)a.qp, r0, i0, more, at, wave, lane);
    if (wave == 0) {
      const int r = r0 + l32, i = (int)a.by_group.div(r);
      buffer_to_lds4(buffer_of(a.lse + tok * a.H + head0, (unsigned)(more * a.H + a.G) * 4), (unsigned)((i - i0) * a.H + r - i * a.G) * 4,
                     at + Sh::BYTES);
    }
  };
  float sum = 0.0f;
  f32x4 k[DP / 8];
  if (rows > start) {
    fetch(0, start, lds);
    unsigned at = lds, other = lds + STAGE;
    for (int hk = 0; hk < a.Hkv; ++hk) {
      load_row<DP>(k, a.k + (((slot * a.Hkv + hk) << a.log2) + place) * (size_t)a.D, a.D, h);
      for (int r0 = start; r0 < rows; r0 += FI) {
        __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
        barrier_lds();
        if (r0 + FI < rows) fetch(hk, r0 + FI, other);
        else if (hk + 1 < a.Hkv) fetch(hk + 1, start, other);
        if (first < n && r0 + FI > wave_from) {
          const f32x16 sc = over_width<DP>(at, k, splat(0.0f), lane);
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const f32x4 z = *reinterpret_cast<const __attribute__((address_space(3))) f32x4*>(lds_at(at + Sh::BYTES + (g * 8 + h * 4) * 4));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int r = r0 + g * 8 + h * 4 + e;
              const float p = __builtin_amdgcn_exp2f(fmaf(sc[g * 4 + e], a.scale, -z[e] * LOG2E));
              sum += r < from || r >= rows ? 0.0f : p;
            }
          }
        }
        const unsigned x = at;
        at = other;
        other = x;
      }
    }
  }
  sum = half_sum(sum);
  if (h == 0 && mine < n && there) {
    float* w = a.weight + (slot << a.log2) + place;
    if (a.add) unsafeAtomicAdd(w, sum);
    else *w = sum;
  }
}

static F32Args of_history(const HistoryArgs& h) {
  F32Args a{};
  a.q = static_cast<const float*>(h.q);
  a.k = static_cast<const float*>(h.k);
  a.v = static_cast<const float*>(h.v);
  a.qp = h.qp, a.kp = h.kp, a.vp = h.vp;
  a.off = h.off;
  a.N = h.N, a.T = h.T, a.L = a.C = h.L, a.H = h.H, a.Hkv = h.Hkv, a.D = h.D, a.G = h.H / h.Hkv;
  a.by_group = mul_div(a.G);
  a.scale = LOG2E / h.gamma, a.inv_gamma = 1.0f / h.gamma;
  a.causal = true;
  a.runs = 1;
  a.o = static_cast<float*>(h.o);
  a.lse = h.lse;
  return a;
}
static F32Args of_cache(const CacheArgs& c) {
  F32Args a{};
  a.q = static_cast<const float*>(c.q);
  a.k = static_cast<const float*>(c.k);
  a.v = static_cast<const float*>(c.v);
  a.qp = c.qp;
  a.off = c.off, a.pages = c.pages, a.lens = c.lens;
  a.N = c.U, a.T = c.T, a.L = c.L, a.C = c.C, a.H = c.H, a.Hkv = c.Hkv, a.D = c.D, a.G = c.H / c.Hkv;
  a.log2 = c.page_log2, a.P = c.P, a.max_pages = c.max_pages;
  a.by_group = mul_div(a.G);
  a.scale = LOG2E / c.gamma;
  a.causal = c.causal, a.add = c.add;
  a.o = static_cast<float*>(c.o);
  a.lse = c.lse;
  a.weight = c.weight;
  return a;
}

// Workgroups of 128 rows, or items, that have any: `longest` of them in each of `per` pairs, `all` in the whole batch
static long long in_128(long long longest, long long per, long long all) {
  const long long a = (longest + 127) / 128 * per, b = (all + 127) / 128;
  return a < b ? a : b;
}
// When the split form: the wide form's workgroups against the items that one walks, whose tiles its four waves share; two split
// workgroups of width 128 do not fit a compute unit. us wide and split, full histories, 4 heads over 4:
//   items, workgroups        30, 60       60, 60       120, 56      120, 240     500, 125     500, 688     3000, 656    3000, 2344
//   width 64, forward        6.8, 9.6     9.6, 9.5     15.9, 9.6    17, 26       49, 24       80, 106      387, 303     1002, 1058
//   width 128, forward       10.5, 15.8   16.5, 16.3   28, 16       32, 65       97, 53       151, 264     709, 758     2139, 2752
//   width 128, gradients with dq wide and split: 33, 37; 53, 49; 94, 74; 100, 133; 326, 255; 670, 715; 2804, 2655; 9088, 8989
static bool splits(long long workgroups, long long walk, int D) { return walk > FI && workgroups * (D > 64 ? 2 : 1) <= walk; }
// dk, dv: the rows of all heads of the group are walked; the split form of width 128 spills (296 bytes of scratch a lane). Gradients with
// dk, dv wide and split: width 64, 1000 items, 4 heads over 2: 782 workgroups (of 128 items) 1030 and 997 us, 344 of 250 items 212 and
// 176; width 128: 1000 items, 187 workgroups 989 and 740, 344 of them 1177 and 1288; 500 items, 4 over 4, 125 326 and 264, 250 328 and 387;
// 3000 items, 281 1817 and 1713, 375 1820 and 2061. Also where items keep one or two waves of the wide form busy and many rows see them:
// 1000 histories, widths 64 and 128: 20 items, 4 over 2, 156, 331 and 112, 290; 45 items, 8 over 2, 433, 968 and 331, 929; 2250 of 64, 4
// over 2, 686, 1471 and 568, 1597; 1125 of 60, 4 over 4, 436, 962 and 485, 1221.
static bool splits_items(long long workgroups, long long items, long long walk, int D) {
  if (items <= 64 && walk > FI && walk >= (D > 64 && items > FI ? 4 : 2) * items) return true;
  return D > 64 ? workgroups * 3 <= walk && workgroups < 320 : walk > FI && workgroups <= walk;
}
// Over a cache histories are cut into runs, of 128 items or more, until workgroups are enough; of lengths below the longest the runs at the
// end are empty. Split also where the rows of a head keep one or two waves of the wide form busy and the runs are longer than two tiles.
// us wide and split, 2 heads of widths 32, 64, 128: 2 rows over 2000 items, 256 users: 62, 161, 369 and 45, 84, 190; 32 rows over 2000, 100
// users: 32, 72, 156 and 29, 49, 110; 64 over 2000, 60 users: 33, 54, 136 and 31, 55, 129; 64 over 64, 500 users: 14, 27, 53 and 21, 48, 130;
// 400 over 1000, 1 user (64 workgroups): 15, 21, 35 and 12, 15, 23; 800 over 1000, 2 users (200): 16, 23, 40 and 19, 30, 70.
static bool splits_over_cache(long long workgroups, long long rows, long long walk, int D) {
  return walk > FI && ((D > 64 ? workgroups * 4 <= walk * 3 : workgroups <= walk) || (rows <= 64 && walk > 2 * FI));
}

template <int DP, bool PAGED>
static laser_status forward_typed(F32Args a, hipStream_t stream) {
  const long long rows = (long long)a.C * a.G, per = (long long)a.N * a.Hkv, walk = a.runs > 1 ? a.chunk : a.L;
  long long workgroups = in_128(rows, per, (long long)a.T * a.H) * a.runs;
  if (PAGED && a.causal) workgroups -= workgroups * (a.C < a.L ? a.C : a.L) / (2LL * a.L);   // (of the runs behind a row's own item)
  const bool split = PAGED ? splits_over_cache(workgroups, rows, walk, a.D) : splits(workgroups, walk, a.D);
  a.tiles = (int)((rows + (split ? 31 : 127)) / (split ? 32 : 128));
  return launch_dealt(a, (long long)a.tiles * a.runs, 256, [&](F32Args& part, long long n) {
    if constexpr (PAGED) {
      part.pages += n * a.max_pages;
      part.lens += n;
    }
    if (split) history_f32_kernel<DP, PAGED, true><<<part.deal.grid, 256, 0, stream>>>(part);
    else history_f32_kernel<DP, PAGED, false><<<part.deal.grid, 256, 0, stream>>>(part);
  });
}
laser_status history_f32_launch(const HistoryArgs& h) {
  const F32Args a = of_history(h);
  return a.D > 64 ? forward_typed<128, false>(a, h.stream) : a.D > 32 ? forward_typed<64, false>(a, h.stream) : forward_typed<32, false>(a, h.stream);
}
laser_status cache_f32_launch(const CacheArgs& c, const CacheRuns& r) {
  F32Args a = of_cache(c);
  a.chunk = r.chunk, a.runs = r.runs, a.work = c.work;
  const laser_status s = a.D > 64 ? forward_typed<128, true>(a, c.stream) : a.D > 32 ? forward_typed<64, true>(a, c.stream) : forward_typed<32, true>(a, c.stream);
  return s == LASER_OK && r.runs > 1 ? cache_join_launch(c, r.chunk, r.runs) : s;
}

template <int DP>
static laser_status backward_typed(const F32Args& a, hipStream_t stream) {
  const long long per = (long long)a.N * a.Hkv, rows = (long long)a.L * a.G;
  const bool split_rows = splits(in_128(rows, per, (long long)a.T * a.H), a.L, a.D);
  const bool split_items = splits_items(in_128(a.L, per, (long long)a.T * a.Hkv), a.L, rows, a.D);
  const long long row_tiles = (rows + (split_rows ? 31 : 127)) / (split_rows ? 32 : 128);
  const long long item_tiles = ((long long)a.L + (split_items ? 31 : 127)) / (split_items ? 32 : 128);
  // (both before anything is launched)
  if (sequences_a_launch(a.N, a.Hkv, row_tiles, 256) <= 0 || sequences_a_launch(a.N, a.Hkv, item_tiles, 256) <= 0) return LASER_ERR_SHAPE;
  const laser_status s = launch_dealt(a, row_tiles, 256, [&](const F32Args& part, long long) {
    if (split_rows) history_dq_f32_kernel<DP, true><<<part.deal.grid, 256, 0, stream>>>(part);
    else history_dq_f32_kernel<DP, false><<<part.deal.grid, 256, 0, stream>>>(part);
  });
  if (s != LASER_OK) return s;
  return launch_dealt(a, item_tiles, 256, [&](const F32Args& part, long long) {
    if (split_items) history_dkv_f32_kernel<DP, true><<<part.deal.grid, 256, 0, stream>>>(part);
    else history_dkv_f32_kernel<DP, false><<<part.deal.grid, 256, 0, stream>>>(part);
  });
}
laser_status history_bwd_f32_launch(const HistoryBwdArgs& b) {
  F32Args a = of_history(b.f);
  a.go = static_cast<const float*>(b.go);
  a.dq = static_cast<float*>(b.dq);
  a.dk = static_cast<float*>(b.dk);
  a.dv = static_cast<float*>(b.dv);
  a.dqp = b.dqp, a.dkp = b.dkp, a.dvp = b.dvp;
  a.work = b.work;
  return a.D > 64 ? backward_typed<128>(a, b.f.stream) : a.D > 32 ? backward_typed<64>(a, b.f.stream) : backward_typed<32>(a, b.f.stream);
}

template <int DP>
static laser_status weights_typed(const F32Args& a, hipStream_t stream) {
  for (long long u = 0; u < a.N; u += 65535) {
    F32Args part = a;
    part.off = a.off + u;
    part.lens = a.lens + u;
    part.pages = a.pages + (size_t)u * a.max_pages;
    cache_weights_f32_kernel<DP><<<dim3((a.L + 127) / 128, a.N - u < 65535 ? a.N - u : 65535), 256, 0, stream>>>(part);
  }
  return launch_status();
}
laser_status cache_weights_f32_launch(const CacheArgs& c) {
  const F32Args a = of_cache(c);
  return a.D > 64 ? weights_typed<128>(a, c.stream) : a.D > 32 ? weights_typed<64>(a, c.stream) : weights_typed<32>(a, c.stream);
}

}  // namespace laser
