// Attention among the items of histories on the matrix cores (bf16): packed sequences, and rows over a paged cache.
//
// The rows of a key-value head are its G = H / H_kv query heads of every token, row r = token r / G, head r % G: shared keys and
// values are then read once for all of them. A workgroup owns NW * RB * 32 consecutive rows of one head of one sequence and
// walks the items that the last of them sees in tiles of 64; a wave owns RB blocks of 32 rows, whose queries stay in registers.
//   Sc^T[item, row] = K . Q^T             A = K from LDS, B = Q^T
//   P^T = exp2(Sc^T c - m)                the running maximum m and sum l of a row are one lane's (and its other half's) registers
//   acc^T[column, row] += V^T . P^T       A = V^T by the LDS transpose load, B = P^T as the accumulators hold it
// Tiles come by direct loads to LDS, the next one behind the current one's arithmetic, one barrier a tile. Rows behind the valid
// ones read as zeros (the buffer's end), so padding that holds NaN never enters; their scores are masked.
#include <type_traits>

#include "history_tile.h"

namespace laser {

struct TileArgs {
  const unsigned short* q;
  const unsigned short* k;
  const unsigned short* v;
  long long qp, kp, vp;
  const int32_t* off;
  const int32_t* pages;
  const int32_t* lens;
  int N, T, L, C, H, Hkv, D, log2, P, max_pages;
  MulDiv by_group;       // / G
  int G, tiles;
  float scale;           // log2(e) / gamma
  bool causal;
  unsigned short* o;
  float* lse;
  int chunk, runs;       // over a cache: items a workgroup walks, and into how many such runs the longest history is cut
  float* work;           // their results where a history has several
};

// Where the maximum of a row is raised: probabilities may stand up to 2^8 above it meanwhile, sums and outputs are in its units
constexpr float MAX_SLACK = 8.0f;

template <int DP, int NW, int RB, bool PAGED>
__global__ __launch_bounds__(64 * NW, (DP * RB <= 128 ? 2 : 1)) void history_tile_kernel(const TileArgs a) {
  using Sh = TileShape<DP>;
  constexpr int KS = DP / 16, DB = DP / 32, ROWS = NW * RB * 32, GPW = (Sh::GROUPS + NW - 1) / NW, OP = DP * 2 + 16;
  constexpr int STAGE = 2 * Sh::BYTES, PATCH = NW * 32 * OP;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * STAGE > PATCH ? 2 * STAGE : PATCH];
  const unsigned lds = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem);

  const int per = a.N * a.Hkv;
  int tile = (int)(blockIdx.x / per), run = 0;
  if (PAGED && a.runs > 1) {
    run = tile / a.tiles;
    tile -= run * a.tiles;
  }
  tile = a.tiles - 1 - tile;   // (the longest first)
  const int nh = blockIdx.x % per, n_seq = nh / a.Hkv, hk = nh % a.Hkv;
  const CandRange cr = cand_range(a.off, n_seq, a.C, a.T);
  const int rows = cr.count * a.G, row0 = tile * ROWS;
  if (row0 >= rows) return;
  const int n = PAGED ? cache_len(a.lens, n_seq, a.L, a.max_pages, a.log2) : cr.count;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, h = lane >> 5;

  // this lane's rows and the last item each sees
  int last[RB];
  bf16x8 qreg[RB][KS];
  int wave_last = -1, wave_first = 0x7fffffff;
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    int r = row0 + (wave * RB + b) * 32 + l32;
    r = r < rows ? r : rows - 1;
    const int i = (int)a.by_group.div(r), g = r - i * a.G;
    last[b] = a.causal ? n - cr.count + i : n - 1;
    const unsigned short* qr = a.q + (size_t)(cr.first + i) * a.qp + (size_t)(hk * a.G + g) * a.D;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      u32x4 raw = {0u, 0u, 0u, 0u};
      if (s * 16 + h * 8 < a.D) raw = *reinterpret_cast<const u32x4*>(qr + s * 16 + h * 8);
      qreg[b][s] = __builtin_bit_cast(bf16x8, raw);
    }
    const int lo = __builtin_amdgcn_readlane(last[b], 0), hi = __builtin_amdgcn_readlane(last[b], 31);
    wave_first = lo < wave_first ? lo : wave_first;
    wave_last = hi > wave_last ? hi : wave_last;
  }
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

  // requests: wave w brings groups w, w + NW, .. of a tile, of keys and of values
  PackedTiles<DP, NW> packed;
  unsigned paged_off[GPW];
  if constexpr (PAGED) {
#pragma unroll
    for (int x = 0; x < GPW; ++x) {
      const int in = lane / Sh::CH, c = (lane % Sh::CH) ^ tile_swz<Sh::CH>((wave + x * NW) * Sh::RPI + in);
      paged_off[x] = c * 8 < a.D ? (unsigned)(in * a.D * 2 + c * 16) : NO_COLUMN;
    }
  } else {
    packed.init(a.D, a.kp, a.vp, wave, lane);
  }
  const int32_t* table = PAGED ? a.pages + (size_t)n_seq * a.max_pages : nullptr;
  int ids[GPW][2];   // pages of the next tile's groups (a second one where a page is shorter than a group)
  auto look_up = [&](int t0) __attribute__((always_inline)) {
    if constexpr (PAGED) {
#pragma unroll
      for (int x = 0; x < GPW; ++x)
#pragma unroll
        for (int e = 0; e < (Sh::RPI > 8 ? 2 : 1); ++e) {
          const int j = t0 + (wave + x * NW) * Sh::RPI + e * 8;
          ids[x][e] = j < n ? scalar_int(table, j >> a.log2) : -1;
        }
    }
  };
  auto fetch = [&](int t0, unsigned at) __attribute__((always_inline)) {
    if constexpr (PAGED) {
#pragma unroll
      for (int x = 0; x < GPW; ++x) {
        const int g = wave + x * NW;
        if (Sh::GROUPS % NW != 0 && g >= Sh::GROUPS) break;
        const int j = t0 + g * Sh::RPI;
        auto half = [&](int id, int j, int rows_here, int skip) __attribute__((always_inline)) {
          const int left = n - j < rows_here ? n - j : rows_here;
          const bool ok = left > 0 && (unsigned)id < (unsigned)a.P;
          const size_t row = ok ? (((size_t)id * a.Hkv + hk) << a.log2) + (j & ((1 << a.log2) - 1)) : 0;
          // (offsets count from the group's first row: the base of a second page's rows lies `skip` rows ahead of them)
          const unsigned bytes = ok ? (unsigned)((skip + left) * a.D * 2) : 0u;
          const long long base = ((long long)row - (ok ? skip : 0)) * a.D;
          buffer_to_lds16(buffer_of(a.k + base, bytes), paged_off[x], at + g * 1024);
          buffer_to_lds16(buffer_of(a.v + base, bytes), paged_off[x], at + Sh::BYTES + g * 1024);
        };
        if (Sh::RPI > 8 && a.log2 == 3) {   // two pages a group: each half of the lanes from its own
          if (lane < 32) half(ids[x][0], j, 8, 0);
          else half(ids[x][1], j + 8, 8, 8);
        } else {
          half(ids[x][0], j, Sh::RPI, 0);
        }
      }
    } else {
      const size_t row = (size_t)(cr.first + t0);
      packed.fetch(a.k + row * a.kp + (size_t)hk * a.D, a.v + row * a.vp + (size_t)hk * a.D, a.kp, a.vp, a.D, n - t0, at);
    }
  };
  // is every page of the user's items one of the pool? (then only the last tile has places without items)
  bool whole_pages = true;
  if constexpr (PAGED) {
    const int used = end > 0 ? ((end - 1) >> a.log2) + 1 : 0;
    bool bad = false;
    for (int x = lane; x < used; x += 64) bad |= (unsigned)table[x] >= (unsigned)a.P;
    whole_pages = __ballot(bad) == 0;
  }
  auto items_of = [&](int t0) {   // bit i: item t0 + i is there
    const int left = n - t0;
    if (PAGED && !whole_pages) {
      const bool in = lane < left && (unsigned)table[(t0 + (lane < left ? lane : 0)) >> a.log2] < (unsigned)a.P;
      return (unsigned long long)__ballot(in);
    }
    return left >= TI ? ~0ull : (1ull << left) - 1;
  };

  f32x16 acc[RB][DB];
  float m[RB], l[RB];
  const f32x16 zero = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    m[b] = -INFINITY;
    l[b] = 0.0f;
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[b][db] = zero;
  }

  const TileReader<DP> read(lane);
  auto step = [&](int t0, unsigned at, unsigned long long items, auto masked) __attribute__((always_inline)) {
    constexpr bool MASKED = decltype(masked)::value;
    f32x16 sc[RB][2];
#pragma unroll
    for (int ib = 0; ib < 2; ++ib)
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const bf16x8 kf = read.rows(at, ib, s);
#pragma unroll
        for (int b = 0; b < RB; ++b)
          sc[b][ib] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qreg[b][s], s == 0 ? zero : sc[b][ib], 0, 0, 0);
      }
    unsigned p[RB][2][8];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      if (MASKED) {
        const int seen = last[b] - t0;
        const unsigned long long mine = items >> (4 * h);
#pragma unroll
        for (int ib = 0; ib < 2; ++ib)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int i0 = ib * 32 + 8 * (r >> 2) + (r & 3);
            if (i0 + 4 * h > seen || !((mine >> i0) & 1)) sc[b][ib][r] = -INFINITY;
          }
      }
      float top = sc[b][0][0];
#pragma unroll
      for (int ib = 0; ib < 2; ++ib)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, sc[b][ib][r]);
      top = half_max(top) * a.scale;
      if (__any(top > m[b] + MAX_SLACK)) {   // (the first tile: m is -inf)
        const float next = fmaxf(m[b], top), c = next == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[b] - next);
        m[b] = next;
        l[b] *= c;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[b][db][r] *= c;
      }
      const float base = m[b] == -INFINITY ? 0.0f : m[b];
      float sum = 0.0f;
#pragma unroll
      for (int ib = 0; ib < 2; ++ib)
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
          const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[b][ib][r], a.scale, -base));
          const float p1 = __builtin_amdgcn_exp2f(fmaf(sc[b][ib][r + 1], a.scale, -base));
          sum += p0 + p1;
          p[b][ib][r >> 1] = pack_bf16(p0, p1);
        }
      l[b] += sum;
    }
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const bf16x8 vf = read.cols(at + Sh::BYTES, s, db);
#pragma unroll
        for (int b = 0; b < RB; ++b) {
          const unsigned* w = &p[b][s >> 1][(s & 1) * 4];
          const u32x4 pf = {w[0], w[1], w[2], w[3]};
          acc[b][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, __builtin_bit_cast(bf16x8, pf), acc[b][db], 0, 0, 0);
        }
      }
  };

  if (end > begin) {
    look_up(begin);
    fetch(begin, lds);
    look_up(begin + TI);
    unsigned at = lds, other = lds + STAGE;
    for (int t0 = begin; t0 < end; t0 += TI) {
      __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
      barrier_lds();   // the tile is there, and every wave is through with the one before
      if (t0 + TI < end) {
        fetch(t0 + TI, other);
        look_up(t0 + 2 * TI);
      }
      if (t0 <= wave_last) {
        const unsigned long long items = items_of(t0);
        if (items == ~0ull && t0 + TI - 1 <= wave_first) step(t0, at, items, std::false_type{});
        else step(t0, at, items, std::true_type{});
      }
      const unsigned x = at;
      at = other;
      other = x;
    }
    barrier_lds();
  }

  // out: a block's rows through a patch of the wave's own, so that they leave in whole 16-byte pieces
  unsigned char* patch = smem + wave * 32 * OP;
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const float sum = half_sum(l[b]), inv = sum > 0.0f ? 1.0f / sum : 0.0f;
    const int first = row0 + (wave * RB + b) * 32;
    const int r = first + l32;
    if (joined) {
      if (r >= rows) continue;
      const int i = (int)a.by_group.div(r), g = r - i * a.G;
      const size_t all = (size_t)a.T * a.H, row = (size_t)(cr.first + i) * a.H + hk * a.G + g;
      float* to = a.work + (run * all + row) * a.D;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int c = db * 32 + x * 8 + h * 4;
          typedef float f32x4 __attribute__((ext_vector_type(4)));
          if (c < a.D) *reinterpret_cast<f32x4*>(to + c) = f32x4{acc[b][db][x * 4] * inv, acc[b][db][x * 4 + 1] * inv,
                                                                 acc[b][db][x * 4 + 2] * inv, acc[b][db][x * 4 + 3] * inv};
        }
      if (h == 0) a.work[a.runs * all * a.D + run * all + row] = sum > 0.0f ? m[b] + log2f(sum) : -INFINITY;
      continue;
    }
    if (a.lse != nullptr && h == 0 && r < rows) {
      const int i = (int)a.by_group.div(r), g = r - i * a.G;
      a.lse[(size_t)(cr.first + i) * a.H + hk * a.G + g] = sum > 0.0f ? (m[b] + log2f(sum)) * LN2 : -INFINITY;
    }
    store_block<DP>(acc[b], inv, patch, rows - first, a.D, lane, [&](int r) {
      const int i = (int)a.by_group.div(first + r), g = first + r - i * a.G;
      return a.o + ((size_t)(cr.first + i) * a.H + hk * a.G + g) * a.D;
    });
  }
}

template <int DP, int NW, int RB, bool PAGED>
static laser_status tile_launch(TileArgs a, hipStream_t stream) {
  constexpr int ROWS = NW * RB * 32;
  a.tiles = (int)(((long long)a.C * a.G + ROWS - 1) / ROWS);
  const long long grid = (long long)a.tiles * a.N * a.Hkv * a.runs;
  if (grid > 0x7fffffffLL) return LASER_ERR_SHAPE;
  history_tile_kernel<DP, NW, RB, PAGED><<<(unsigned)grid, 64 * NW, 0, stream>>>(a);
  return launch_status();
}
template <bool PAGED>
static laser_status tile_launch_any(const TileArgs& a, hipStream_t stream) {
  const int form = tuning_int("LASER_HIST_FORM", 0);
  if (a.D > 64) {
    if (form == 1) return tile_launch<128, 8, 1, PAGED>(a, stream);
    if (form == 2) return tile_launch<128, 4, 2, PAGED>(a, stream);
    return tile_launch<128, 4, 1, PAGED>(a, stream);
  }
  if (a.D > 32) {
    if (form == 1) return tile_launch<64, 8, 1, PAGED>(a, stream);
    if (form == 2) return tile_launch<64, 4, 2, PAGED>(a, stream);
    return tile_launch<64, 4, 1, PAGED>(a, stream);
  }
  return tile_launch<32, 4, 1, PAGED>(a, stream);
}

laser_status history_tile_launch(const HistoryArgs& h) {
  TileArgs a{};
  a.q = static_cast<const unsigned short*>(h.q);
  a.k = static_cast<const unsigned short*>(h.k);
  a.v = static_cast<const unsigned short*>(h.v);
  a.qp = h.qp, a.kp = h.kp, a.vp = h.vp;
  a.off = h.off;
  a.N = h.N, a.T = h.T, a.L = a.C = h.L, a.H = h.H, a.Hkv = h.Hkv, a.D = h.D, a.G = h.H / h.Hkv;
  a.by_group = mul_div(a.G);
  a.scale = LOG2E / h.gamma;
  a.causal = true;
  a.runs = 1;
  a.o = static_cast<unsigned short*>(h.o);
  a.lse = h.lse;
  return tile_launch_any<false>(a, h.stream);
}

laser_status cache_tile_launch(const CacheArgs& c, const CacheRuns& r) {
  TileArgs a{};
  a.q = static_cast<const unsigned short*>(c.q);
  a.k = static_cast<const unsigned short*>(c.k);
  a.v = static_cast<const unsigned short*>(c.v);
  a.qp = c.qp;
  a.off = c.off, a.pages = c.pages, a.lens = c.lens;
  a.N = c.U, a.T = c.T, a.L = c.L, a.C = c.C, a.H = c.H, a.Hkv = c.Hkv, a.D = c.D, a.G = c.H / c.Hkv;
  a.log2 = c.page_log2, a.P = c.P, a.max_pages = c.max_pages;
  a.by_group = mul_div(a.G);
  a.scale = LOG2E / c.gamma;
  a.causal = c.causal;
  a.o = static_cast<unsigned short*>(c.o);
  a.lse = c.lse;
  a.chunk = r.chunk, a.runs = r.runs;
  a.work = c.work;
  const laser_status s = tile_launch_any<true>(a, c.stream);
  return s == LASER_OK && r.runs > 1 ? cache_join_launch(c, r.chunk, r.runs) : s;
}

}  // namespace laser
