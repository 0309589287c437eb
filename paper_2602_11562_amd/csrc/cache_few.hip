// A few rows per key-value head over a paged cache (bf16): one new item or a handful of candidates a user. The cache is read once
// and everything else is small, so this is bound by memory.
//
// A workgroup owns (user, key-value head, run of items); its four waves take tiles of 32 items in turn, each with tiles of its own
// in LDS and no barrier while it streams. Up to width 64 two of them, so that requests run a tile ahead of the arithmetic; beyond there is
// room for one, whose successor is asked for behind its last read, and what runs meanwhile are the other seven waves of the compute unit.
// The rows (at most 32: every new item's query heads of the group) are one column block of the products of history_mfma.hip, with the same
// rounding of P. At the end the waves' maxima, sums and outputs are joined in LDS. Histories longer than a run are cut into several
// workgroups' runs, whose results go to the work buffer (outputs normalised, with log2 of their sums) and are joined by a second launch.
// 128 users of up to 4096 items, 8 heads of 128 over 2: 27 us for 128 MB; one user of 65000, 16 heads over 2: 17 us for 67 MB (4.7 and
// 3.9 TB/s; a large copy reaches 5.2). The joins are a launch each, 4 to 6 us.
#include "history_tile.h"

namespace laser {

typedef float f32x4 __attribute__((ext_vector_type(4)));

template <int DP>
struct FewShape {
  static constexpr int ROW = DP * 2, CH = DP / 8, RPI = 64 / CH, TILE = 32 * ROW, GROUPS = 32 / RPI;
  static constexpr int REQ = 2 * GROUPS;                  // requests a tile
  static constexpr int NST = DP == 128 ? 1 : 2;           // tiles of a wave
  static constexpr int WAVE = NST * 2 * TILE;             // its bytes
  static constexpr int JOIN = DP * 32 * 4;                // what it joins with: [column][32 rows] of fp32, row r at r ^ column % 32
  static_assert(JOIN <= WAVE, "the outputs take the tiles' place");
};

template <int DP>
__global__ __launch_bounds__(256, 2) void cache_few_kernel(const CacheArgs a, int G, MulDiv by_group, float scale, int chunk, int splits) {
  using Sh = FewShape<DP>;
  constexpr int KS = DP / 16, DB = DP / 32;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * Sh::WAVE];
  __shared__ float join_m[4][32], join_l[4][32];
  const int per = a.U * a.Hkv;
  // (turned by one from run to run: a user's runs are not all one die's)
  const int split = blockIdx.x / per, uh = (blockIdx.x + split) % per, u = uh / a.Hkv, hk = uh % a.Hkv;
  const CandRange cr = cand_range(a.off, u, a.C, a.T);
  const int rows = cr.count * G;
  if (rows == 0) return;
  const int n = cache_len(a.lens, u, a.L, a.max_pages, a.page_log2);
  const int lo = split * chunk, hi = n < lo + chunk ? n : lo + chunk;
  if (lo >= n && split > 0) return;   // (the first run of an empty history still writes)
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, h = lane >> 5;
  const unsigned lds = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem) + wave * Sh::WAVE;
  const unsigned short* q = static_cast<const unsigned short*>(a.q);
  const unsigned short* kc = static_cast<const unsigned short*>(a.k);
  const unsigned short* vc = static_cast<const unsigned short*>(a.v);
  const int32_t* table = a.pages + (size_t)u * a.max_pages;

  unsigned off[Sh::GROUPS];
#pragma unroll
  for (int g = 0; g < Sh::GROUPS; ++g) {
    const int in = lane / Sh::CH, c = (lane % Sh::CH) ^ tile_swz<Sh::CH>(g * Sh::RPI + in);
    off[g] = c * 8 < a.D ? (unsigned)(in * a.D * 2 + c * 16) : NO_COLUMN;
  }
  int ids[4];   // pages of the next tile: of its items 0, 8, 16 and 24
  auto look_up = [&](int t0) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < 4; ++x) ids[x] = t0 + x * 8 < hi ? scalar_int(table, (t0 + x * 8) >> a.page_log2) : -1;
  };
  auto fetch = [&](int t0, unsigned at) __attribute__((always_inline)) {
#pragma unroll
    for (int g = 0; g < Sh::GROUPS; ++g) {
      auto part = [&](int id, int j, int count, int skip) __attribute__((always_inline)) {
        const int left = hi - j < count ? hi - j : count;
        const bool ok = left > 0 && (unsigned)id < (unsigned)a.P;
        const size_t row = ok ? (((size_t)id * a.Hkv + hk) << a.page_log2) + (j & ((1 << a.page_log2) - 1)) : 0;
        const unsigned bytes = ok ? (unsigned)((skip + left) * a.D * 2) : 0u;
        const long long base = ((long long)row - (ok ? skip : 0)) * a.D;
        buffer_to_lds16(buffer_of(kc + base, bytes), off[g], at + g * 1024);
        buffer_to_lds16(buffer_of(vc + base, bytes), off[g], at + Sh::TILE + g * 1024);
      };
      const int j = t0 + g * Sh::RPI;
      if (Sh::RPI > 8 && a.page_log2 == 3) {   // two pages a request: each half of the lanes from its own
        if (lane < 32) part(ids[g * 2], j, 8, 0);
        else part(ids[g * 2 + 1], j + 8, 8, 8);
      } else {
        part(ids[g * Sh::RPI / 8], j, Sh::RPI, 0);
      }
    }
  };
  // (what a request brings: its own count on the page of two, twice as many)
  const int requests = Sh::RPI > 8 && a.page_log2 == 3 ? 2 * Sh::REQ : Sh::REQ;

  const int step_items = 4 * 32;
  int ask = lo + wave * 32, mine = ask;
  int pending = 0, slot_in = 0, slot_out = 0;
  look_up(ask);
  auto request = [&]() __attribute__((always_inline)) {
    fetch(ask, lds + slot_in * 2 * Sh::TILE);
    slot_in = slot_in + 1 == Sh::NST ? 0 : slot_in + 1;
    ask += step_items;
    ++pending;
    look_up(ask);
  };
  for (int x = 0; x < Sh::NST && ask < hi; ++x) request();

  bf16x8 qreg[KS];
  int last;
  {
    const int r = l32 < rows ? l32 : rows - 1, i = (int)by_group.div(r), g = r - i * G;
    last = a.causal ? n - cr.count + i : n - 1;
    const unsigned short* qr = q + (size_t)(cr.first + i) * a.qp + (size_t)(hk * G + g) * a.D;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      u32x4 raw = {0u, 0u, 0u, 0u};
      if (s * 16 + h * 8 < a.D) raw = *reinterpret_cast<const u32x4*>(qr + s * 16 + h * 8);
      qreg[s] = __builtin_bit_cast(bf16x8, raw);
    }
  }
  const int first_seen = __builtin_amdgcn_readlane(last, 0);
  bool whole_pages;
  {
    bool bad = false;
    for (int x = (lo >> a.page_log2) + lane; x <= (hi - 1) >> a.page_log2 && lo < hi; x += 64) bad |= (unsigned)table[x] >= (unsigned)a.P;
    whole_pages = __ballot(bad) == 0;
  }

  const f32x16 zero = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = zero;
  float m = -INFINITY, l = 0.0f;
  TileReader<DP> read(lane);

  for (; mine < hi; mine += step_items) {
    // loads return in order: with `pending` tiles asked for, the oldest is there when those of the others are all that is left
    wait_vm((pending - 1) * requests);
    asm volatile("" ::: "memory");
    const unsigned at = lds + slot_out * 2 * Sh::TILE;
    read.place(at);
    f32x16 sc;
#pragma unroll
    for (int s = 0; s < KS; ++s)
      sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read.rows(0, 0, s), qreg[s], s == 0 ? zero : sc, 0, 0, 0);
    if (!whole_pages || mine + 31 > first_seen || mine + 32 > hi) {
      const int left = hi - mine;
      bool in = l32 < left;
      if (!whole_pages) in = in && (unsigned)table[(mine + (in ? l32 : 0)) >> a.page_log2] < (unsigned)a.P;
      const unsigned items = (unsigned)__ballot(in) >> (4 * h);
      const int seen = last - mine - 4 * h;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int i0 = 8 * (r >> 2) + (r & 3);
        if (i0 > seen || !((items >> i0) & 1)) sc[r] = -INFINITY;
      }
    }
    float top = sc[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, sc[r]);
    top = half_max(top) * scale;
    if (__any(top > m)) {
      const float next = fmaxf(m, top), c = next == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - next);
      m = next;
      l *= c;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[db][r] *= c;
    }
    const float base = m == -INFINITY ? 0.0f : m;
    unsigned p[8];
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
      const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[r], scale, -base)), p1 = __builtin_amdgcn_exp2f(fmaf(sc[r + 1], scale, -base));
      l += p0 + p1;
      p[r >> 1] = pack_bf16(p0, p1);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const u32x4 b = {p[s * 4], p[s * 4 + 1], p[s * 4 + 2], p[s * 4 + 3]};
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read.cols(Sh::TILE, s, db), __builtin_bit_cast(bf16x8, b), acc[db], 0, 0, 0);
      }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the tile has been read: its place may be asked for again
    --pending;
    slot_out = slot_out + 1 == Sh::NST ? 0 : slot_out + 1;
    if (ask < hi) request();
  }

  // the waves' results, in the place of the tiles
  float* out = reinterpret_cast<float*>(smem + wave * Sh::WAVE);
  l = half_sum(l);
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int d = 8 * (r >> 2) + 4 * h + (r & 3);
      out[(db * 32 + d) * 32 + (l32 ^ d)] = acc[db][r];
    }
  if (h == 0) {
    join_m[wave][l32] = m;
    join_l[wave][l32] = l;
  }
  __syncthreads();
  const bool final = n <= chunk;
  for (int e = tid; e < rows * a.D; e += 256) {
    const int r = e / a.D, d = e - r * a.D;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, join_m[w][r]);
    float sum = 0.0f, x = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float mw = join_m[w][r], c = mw == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mw - top);
      sum = fmaf(join_l[w][r], c, sum);
      x = fmaf(reinterpret_cast<const float*>(smem + w * Sh::WAVE)[d * 32 + (r ^ (d & 31))], c, x);
    }
    x = sum > 0.0f ? x / sum : 0.0f;
    const float z = sum > 0.0f ? top + log2f(sum) : -INFINITY;
    const int i = (int)by_group.div(r), g = r - i * G;
    const size_t row = (size_t)(cr.first + i) * a.H + hk * G + g;
    if (final) {
      static_cast<unsigned short*>(a.o)[row * a.D + d] = f32_to_bf16_bits(x);
      if (d == 0 && a.lse != nullptr) a.lse[row] = z * LN2;
    } else {
      const size_t all = (size_t)a.T * a.H;
      a.work[(split * all + row) * a.D + d] = x;
      if (d == 0) a.work[splits * all * a.D + split * all + row] = z;
    }
  }
}

// Joins the runs' results of a row, a workgroup each: the runs' shares first, then their
// outputs, 16 bytes a lane and as many runs at a time as there are lanes for.
constexpr int MOST_RUNS = 1024;

template <typename T>
__global__ __launch_bounds__(256) void cache_join_kernel(const CacheArgs a, int chunk, int splits) {
  constexpr int NT = 256;
  __shared__ float share[MOST_RUNS];
  __shared__ __attribute__((aligned(16))) float part[NT * 4];
  __shared__ float wave_top[NT / 64], wave_sum[NT / 64];
  const int u = blockIdx.y, tid = threadIdx.x;
  const CandRange cr = cand_range(a.off, u, a.C, a.T);
  const int n = cache_len(a.lens, u, a.L, a.max_pages, a.page_log2);
  if (n <= chunk) return;   // one run: it has written the result
  const size_t all = (size_t)a.T * a.H;
  const float* z = a.work + splits * all * a.D;
  const int pieces = a.D / 4, groups = NT / pieces, group = tid / pieces, piece = tid - group * pieces;
  for (long long x = blockIdx.x; x < (long long)cr.count * a.H; x += gridDim.x) {
    const int i = (int)(x / a.H);
    const size_t row = (size_t)cr.first * a.H + x;
    const int seen = a.causal ? n - cr.count + i + 1 : n;
    const int runs = seen <= 0 ? 0 : (seen + chunk - 1) / chunk;
    float mine[MOST_RUNS / NT], top = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int s = 0; s < MOST_RUNS / NT; ++s) {
      mine[s] = s * NT + tid < runs ? z[(s * NT + tid) * all + row] : -INFINITY;
      top = fmaxf(top, mine[s]);
    }
    for (int m = 32; m; m >>= 1) top = fmaxf(top, __shfl_xor(top, m));
    if ((tid & 63) == 0) wave_top[tid >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) top = fmaxf(top, wave_top[w]);
#pragma unroll
    for (int s = 0; s < MOST_RUNS / NT; ++s)
      if (s * NT + tid < runs) {
        const float c = mine[s] == -INFINITY ? 0.0f : exp2f(mine[s] - top);
        share[s * NT + tid] = c;
        sum += c;
      }
    for (int m = 32; m; m >>= 1) sum += __shfl_xor(sum, m);
    if ((tid & 63) == 0) wave_sum[tid >> 6] = sum;
    __syncthreads();
    sum = 0.0f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) sum += wave_sum[w];
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    if (group < groups) {
      const float* at = a.work + row * a.D + piece * 4;
      for (int s0 = group; s0 < runs; s0 += 4 * groups) {
        f32x4 y[4];
        float c[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {   // (behind the last run: the last one again, with no share)
          const int s = s0 + e * groups, k = s < runs ? s : runs - 1;
          c[e] = s < runs ? share[k] : 0.0f;
          y[e] = *reinterpret_cast<const f32x4*>(at + k * all * a.D);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int d = 0; d < 4; ++d) o[d] = fmaf(c[e], y[e][d], o[d]);
      }
      *reinterpret_cast<f32x4*>(part + (group * pieces + piece) * 4) = o;
    }
    __syncthreads();
    const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
    for (int d = tid; d < a.D; d += NT) {
      float y = 0.0f;
      for (int g = 0; g < groups; ++g) y += part[g * a.D + d];
      store_from_f32<T>(static_cast<T*>(a.o), row * a.D + d, y * by);
    }
    if (tid == 0 && a.lse != nullptr) a.lse[row] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * LN2;
    __syncthreads();
  }
}

// The same for few runs: a thread per row and 16 bytes
template <typename T>
__global__ __launch_bounds__(256) void cache_join_few_kernel(const CacheArgs a, int chunk, int splits, MulDiv by_pieces, MulDiv by_heads) {
  const int u = blockIdx.y;
  const CandRange cr = cand_range(a.off, u, a.C, a.T);
  const int n = cache_len(a.lens, u, a.L, a.max_pages, a.page_log2);
  if (n <= chunk) return;
  const size_t all = (size_t)a.T * a.H;
  const float* z = a.work + splits * all * a.D;
  const unsigned pieces = a.D / 4, e = blockIdx.x * 256 + threadIdx.x, x = by_pieces.div(e), piece = e - x * pieces;
  if (x >= (unsigned)(cr.count * a.H)) return;
  const int i = (int)by_heads.div(x);
  const size_t row = (size_t)cr.first * a.H + x;
  const int seen = a.causal ? n - cr.count + i + 1 : n;
  const int runs = seen <= 0 ? 0 : (seen + chunk - 1) / chunk;
  const float* at = a.work + row * a.D + piece * 4;
  float top = -INFINITY, sum = 0.0f;
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s0 = 0; s0 < runs; s0 += 4) {
    float zs[4];
    f32x4 y[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {   // (behind the last run: the last one again, with no share)
      const int k = s0 + s < runs ? s0 + s : runs - 1;
      zs[s] = z[k * all + row];
      y[s] = *reinterpret_cast<const f32x4*>(at + k * all * a.D);
    }
    float next = top;
#pragma unroll
    for (int s = 0; s < 4; ++s) next = fmaxf(next, zs[s]);
    if (next == -INFINITY) continue;
    const float old = exp2f(top - next);
    top = next;
    sum *= old;
#pragma unroll
    for (int d = 0; d < 4; ++d) o[d] *= old;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const float c = s0 + s < runs ? exp2f(zs[s] - top) : 0.0f;
      sum += c;
#pragma unroll
      for (int d = 0; d < 4; ++d) o[d] = fmaf(c, y[s][d], o[d]);
    }
  }
  const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<f32x4*>(static_cast<float*>(a.o) + row * a.D + piece * 4) = f32x4{o[0] * by, o[1] * by, o[2] * by, o[3] * by};
  } else {
    *reinterpret_cast<u32x2*>(static_cast<unsigned short*>(a.o) + row * a.D + piece * 4) = u32x2{pack_bf16(o[0] * by, o[1] * by), pack_bf16(o[2] * by, o[3] * by)};
  }
  if (piece == 0 && a.lse != nullptr) a.lse[row] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * LN2;
}

laser_status cache_join_launch(const CacheArgs& a, int chunk, int splits) {
  const long long rows = (long long)a.C * a.H;
  for (long long u = 0; u < a.U; u += 65535) {
    CacheArgs part = a;
    part.off = a.off + u;
    part.lens = a.lens + u;
    const unsigned users = a.U - u < 65535 ? a.U - u : 65535;
    if (splits > 16) {   // (16 rows of 128 columns in 127 runs: 5.3 us; 40000 rows in four runs: 18 us by the other, 31 by this one)
      const dim3 grid((unsigned)(rows < 65536 ? rows : 65536), users);
      if (a.dt == LASER_F32) cache_join_kernel<float><<<grid, 256, 0, a.stream>>>(part, chunk, splits);
      else cache_join_kernel<unsigned short><<<grid, 256, 0, a.stream>>>(part, chunk, splits);
    } else {
      const dim3 grid((unsigned)((rows * (a.D / 4) + 255) / 256), users);   // (rows are few enough to be cut into runs)
      const MulDiv pieces = mul_div(a.D / 4), heads = mul_div(a.H);
      if (a.dt == LASER_F32) cache_join_few_kernel<float><<<grid, 256, 0, a.stream>>>(part, chunk, splits, pieces, heads);
      else cache_join_few_kernel<unsigned short><<<grid, 256, 0, a.stream>>>(part, chunk, splits, pieces, heads);
    }
  }
  return launch_status();
}

// How the longest history is cut into runs of whole tiles, of `least` items or more: into as many as make `want` workgroups of all
// users' histories together. Sizes alone decide, which the caller who provides the work buffer knows too.
CacheRuns cache_runs(long long workgroups, int L, int want, int least, int tile) {
  const long long wanted = (want + workgroups - 1) / workgroups;
  const int most = (L + least - 1) / least;
  int runs = wanted < most ? (int)wanted : most;
  runs = runs < MOST_RUNS ? runs : MOST_RUNS;
  const int chunk = ((L + runs - 1) / runs + tile - 1) / tile * tile;
  return CacheRuns{chunk, (L + chunk - 1) / chunk};
}

template <int DP>
static laser_status few_typed(const CacheArgs& a, const CacheRuns& r) {
  const int G = a.H / a.Hkv;
  const long long each = (long long)a.Hkv * r.runs;   // workgroups of a user
  if (a.U * each > 0x7fffffffLL) return LASER_ERR_SHAPE;
  const long long most = 0xffffffffLL / 256 / each;   // (a launch has fewer than 2^32 threads; a user has Hkv * runs <= 2^20 workgroups)
  for (long long u = 0; u < a.U; u += most) {
    CacheArgs part = a;
    part.U = a.U - u < most ? (int)(a.U - u) : (int)most;
    part.off = a.off + u;
    part.pages = a.pages + u * a.max_pages;
    part.lens = a.lens + u;
    cache_few_kernel<DP><<<(unsigned)(part.U * each), 256, 0, a.stream>>>(part, G, mul_div(G), LOG2E / a.gamma, r.chunk, r.runs);
    const laser_status s = launch_status();
    if (s != LASER_OK) return s;
  }
  return r.runs > 1 ? cache_join_launch(a, r.chunk, r.runs) : LASER_OK;
}
laser_status cache_few_launch(const CacheArgs& a, const CacheRuns& r) {
  if (a.D > 64) return few_typed<128>(a, r);
  if (a.D > 32) return few_typed<64>(a, r);
  return few_typed<32>(a, r);
}

}  // namespace laser
