// Many rows over a cache of 8-bit blocks: chunks of new items, and candidates. The split of history_mfma.hip: a workgroup of four waves
// owns 128 rows of a key-value head and walks the items that the last of them sees in tiles of 64, which come by direct loads to LDS as
// the bytes that they are; a wave owns 32 rows (SPLIT: of half of the items) and makes its operands of the bytes in registers. (Scores of bf16 queries, as two numbers of
// 8 bits each, straight from the bytes by the products of 8-bit operands: 215 us would be 202 for 512 new items x up to 10000, but those products
// sum in fewer than 32 bits: errors of lse 4e-6 against 4e-7.)
// Bound by the vector units beside the products: an exponential, a product and a sum for a score of one, and the values' bytes. Ragged
// histories leave a part of the chip without work behind the others' end, hence the order below.
#include "cache8_tile.h"

namespace laser {

struct Tile8Args {
  Cache8Args a;
  const int32_t* off;
  int N, Hkv;
  MulDiv by_group;       // / G
  int G, tiles, rows_log2;   // tiles of the longest sequence's rows, of 128 or 64
  Deal deal;             // of (tile, run) to workgroups
  float scale;           // log2(e) / gamma
  int chunk, runs;       // items a workgroup walks, and into how many such runs the longest history is cut
  bool ranked;           // workgroups by what they have to do, the most first
};

// Which tile of rows of which user and head, and which run of its items, a workgroup has
struct Part8 { int user, head, tile, run, first, count, n; };   // (and the user's rows and items)
__device__ __forceinline__ bool part_in_turn(const Tile8Args& t, Part8* p) {
  const Place place = place_of(t.deal, blockIdx.x);
  if (place.rank >= t.deal.tiles) return false;
  p->run = t.runs > 1 ? place.rank / t.tiles : 0;
  p->tile = t.tiles - 1 - (place.rank - p->run * t.tiles);   // (the longest first)
  p->user = place.pair / t.Hkv;
  p->head = place.pair - p->user * t.Hkv;
  const CandRange cr = cand_range(t.off, p->user, t.a.c.C, t.a.c.T);
  p->first = cr.first;
  p->count = cr.count;
  if (p->tile << t.rows_log2 >= cr.count * t.G) return false;
  p->n = cache_len(t.a.c.lens, p->user, t.a.c.L, t.a.c.max_pages, t.a.c.page_log2);
  return true;
}
// At most 64 users, a lane for each: the whole runs of all of them come first, then what is left of each, the longest first, since workgroups
// are started in the order of their numbers. Against the order of users (us, with the join): 512 new items x up to 10000, 16 users of 128 229
// and 191; 256 rows x up to 4096, 32 of 64 80.3 and 65.1; 128 x up to 4096, 64 of 128 122 and 100; equal lengths 360 and 365; 1000 x up to
// 1500, 50 of 128 (3200 workgroups, four or more for each place, which even out by themselves) 130 and 134.
// Workgroups of whole runs go to the eighths of the chip, each with an L2 cache of its own, in even parts, so that the tiles of a run meet
// there (against the plain order 193 and 191, 119 and 116 for 400 x up to 9000, 12 of 128).
__device__ __forceinline__ bool part_by_length(const Tile8Args& t, int lane, Part8* p) {
  const CacheArgs& a = t.a.c;
  const int u = lane < t.N ? lane : t.N - 1;
  const CandRange cr = cand_range(t.off, u, a.C, a.T);
  const int n = cache_len(a.lens, u, a.L, a.max_pages, a.page_log2), tiles = lane < t.N ? (cr.count * t.G + (1 << t.rows_log2) - 1) >> t.rows_log2 : 0;
  const int whole = t.runs > 1 ? n / t.chunk : 0, rest = n - whole * t.chunk;
  int at = blockIdx.x, behind = whole * tiles * t.Hkv;   // the workgroups of whole runs up to this user's last
  const int mine = behind;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int other = __shfl_up(behind, d);
    behind += lane >= d ? other : 0;
  }
  const int all = __builtin_amdgcn_readlane(behind, 63);
  int first, last_run = 0;
  unsigned long long found;
  if (at < all) {
    const int eighth = all >> 3;
    if (at < eighth * 8) at = (at & 7) * eighth + (at >> 3);
    first = behind - mine;
    found = __ballot(at >= first && at < behind);
  } else {
    at -= all;
    const int w = rest > 0 || n == 0 ? tiles * t.Hkv : 0;
    first = 0;
    for (int v = 0; v < t.N; ++v) {
      const int r = __builtin_amdgcn_readlane(rest, v), x = __builtin_amdgcn_readlane(w, v);
      first += r > rest || (r == rest && v < lane) ? x : 0;
    }
    found = __ballot(at >= first && at < first + w);
    last_run = 1;
  }
  if (found == 0) return false;
  const int who = __builtin_ctzll(found), count = __builtin_amdgcn_readlane(tiles, who);
  at -= __builtin_amdgcn_readlane(first, who);
  p->user = who;
  const int pair = at / count;
  p->tile = count - 1 - (at - pair * count);   // (the longest first)
  const int run = pair / t.Hkv;
  p->head = pair - run * t.Hkv;
  p->run = last_run ? __builtin_amdgcn_readlane(whole, who) : run;
  p->first = __builtin_amdgcn_readlane(cr.first, who);
  p->count = __builtin_amdgcn_readlane(cr.count, who);
  p->n = __builtin_amdgcn_readlane(n, who);
  return true;
}

template <int DP, int SLOTS, int NP, int PART, int SPLIT, typename T>
__global__ __launch_bounds__(256, 2) void cache8_tile_kernel(const Tile8Args t) {
  constexpr int KS = DP / 16, DB = DP / 32, NW = 4, BLOCKS = NW / SPLIT, ROWS = BLOCKS * 32, KB = TI * DP, SLOT = 2 * KB, OP = DP * 2 + 16, PATCH = NW * 32 * OP;
  static_assert(SLOTS <= 4, "wait_requests knows the requests of two tiles ahead at most");
  constexpr bool PATCHED = sizeof(T) == 2;   // (fp32 rows leave from the registers)
  __shared__ __attribute__((aligned(1024))) unsigned char smem[SLOTS * SLOT > PATCH || !PATCHED ? SLOTS * SLOT : PATCH];
  __shared__ __attribute__((aligned(16))) float scales[SLOTS][TI / 8 * 2];
  __shared__ int odd[2][NW];
  const CacheArgs& a = t.a.c;
  const unsigned lds = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem);
  const unsigned lds_s = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(__attribute__((address_space(3))) float*)&scales[0][0]);
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, h = lane >> 5;
  Part8 part;
  if (!(t.ranked ? part_by_length(t, lane, &part) : part_in_turn(t, &part))) return;
  const int u_seq = part.user, hk = part.head, run = part.run, n = part.n, rows = part.count * t.G, row0 = part.tile * ROWS;

  int end;   // one past the last item that a row of this workgroup sees
  {
    const int r = row0 + ROWS < rows ? row0 + ROWS - 1 : rows - 1;
    end = a.causal ? n - part.count + (int)t.by_group.div(r) + 1 : n;
  }
  const bool joined = t.runs > 1 && n > t.chunk;   // others write their part of the result too
  int begin = 0;
  if (t.runs > 1) {
    begin = run * t.chunk;
    if (run > 0 && begin >= end) return;
    end = end < begin + t.chunk ? end : begin + t.chunk;
  }
  const int turns = end > begin ? (end - begin + TI - 1) / TI : 0;
  const int32_t* table = a.pages + (size_t)u_seq * a.max_pages;

  Tiles8<DP, 16, PART> tiles;
  tiles.init(a.D, a.page_log2, wave * 16, lane);
  const int requests = tiles.requests();
  int asked = 0, in = 0;
  auto request = [&]() __attribute__((always_inline)) {
    const unsigned at = lds + in * SLOT + wave * 16 * DP;
    tiles.fetch(t.a, hk, begin + asked * TI + wave * 16, n, at, at + KB, lds_s + in * (TI / 8 * 8) + wave * 16, lane);
    in = in + 1 == SLOTS ? 0 : in + 1;
    ++asked;
    tiles.look_up(table, begin + asked * TI + wave * 16, end, a.page_log2);
  };
  if (turns > 0) {
    tiles.look_up(table, begin + wave * 16, end, a.page_log2);
    for (int x = 0; x < SLOTS - 1 && x < turns; ++x) request();
  }

  // this lane's row and the last item it sees
  const int first = row0 + wave % BLOCKS * 32;
  int last;
  bf16x8 qreg[NP][KS];
  {
    int r = first + l32;
    r = r < rows ? r : rows - 1;
    const int i = (int)t.by_group.div(r), g = r - i * t.G;
    last = a.causal ? n - part.count + i : n - 1;
    load_query<DP, NP>(static_cast<const T*>(a.q) + (size_t)(part.first + i) * a.qp + (size_t)(hk * t.G + g) * a.D, a.D, h, qreg);
  }
  const int all_see = a.causal ? n - part.count + (int)t.by_group.div(row0) : 0x7fffffff;   // up to this item all rows see all that is there
  const int wave_first = __builtin_amdgcn_readlane(last, 0), wave_last = first < rows ? __builtin_amdgcn_readlane(last, 31) : -1;   // (without rows: none)
  bool whole_pages;
  {
    bool bad = false;
    if (turns > 0)
      for (int x = (begin >> a.page_log2) + lane; x <= (end - 1) >> a.page_log2; x += 64) bad |= (unsigned)table[x] >= (unsigned)a.P;
    whole_pages = __ballot(bad) == 0;
  }

  const f32x16 zero = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = zero;
  float m = -INFINITY, l = 0.0f;
  const TileReader8<DP> read(lane);

  auto block = [&](int t0, unsigned at, unsigned at_s) __attribute__((always_inline)) {
    f32x16 sc = zero;
    const float ks = read.key_scale(at_s);
#pragma unroll
    for (int i = 0; i < KS / 2; ++i) {
      const u32x4 w = read.rows(at, i);
      const bf16x8 k0 = wide8(w[0], w[1], ks, ks), k1 = wide8(w[2], w[3], ks, ks);
#pragma unroll
      for (int p = NP - 1; p >= 0; --p) {
        sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k0, qreg[p][2 * i], sc, 0, 0, 0);
        sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k1, qreg[p][2 * i + 1], sc, 0, 0, 0);
      }
    }
    const bool whole = whole_pages && t0 + 31 <= wave_first && t0 + 32 <= end;
    unsigned items = ~0u;
    if (!whole) {   // places without an item, and items behind a row's own
      bool in = l32 < end - t0;
      if (!whole_pages) in = in && (unsigned)table[(t0 + (in ? l32 : 0)) >> a.page_log2] < (unsigned)a.P;
      items = (unsigned)__ballot(in);
      const int seen = last - t0 - 4 * h;
      const unsigned mine = items >> (4 * h);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int i0 = 8 * (r >> 2) + (r & 3);
        if (i0 > seen || !((mine >> i0) & 1)) sc[r] = -INFINITY;
      }
    }
    float top = sc[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, sc[r]);
    top = half_max(top) * t.scale;
    if (__any(top > m + MAX_SLACK)) {   // (the first tile: m is -inf)
      const float next = fmaxf(m, top), c = next == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - next);
      m = next;
      l *= c;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[db][r] *= c;
    }
    const float base = m == -INFINITY ? 0.0f : m;
    bf16x8 p[NP][2];
    float sum = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
      const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[r], t.scale, -base)), p1 = __builtin_amdgcn_exp2f(fmaf(sc[r + 1], t.scale, -base));
      sum += p0 + p1;
      split_pair<NP>(p0, p1, r, p);
    }
    l += sum;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const u32x2 vs = read.value_scales(at_s, s);
      float v0 = __uint_as_float(vs[0]), v1 = __uint_as_float(vs[1]);
      if (!whole) {   // (a block without items has no scale; its codes came as zeros)
        v0 = (items >> (16 * s)) & 1 ? v0 : 1.0f;
        v1 = (items >> (16 * s + 8)) & 1 ? v1 : 1.0f;
      }
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const u32x2 w = read.columns(at + KB, s, db);
        const bf16x8 v = wide8(w[0], w[1], v0, v1);
#pragma unroll
        for (int i = NP - 1; i >= 0; --i) acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[i][s], acc[db], 0, 0, 0);
      }
    }
  };
  int out = 0;
  for (int u = 0; u < turns; ++u) {
    wait_requests((asked - u - 1) * requests);
    const unsigned at = lds + out * SLOT, at_s = lds_s + out * (TI / 8 * 8);
    const int t0 = begin + u * TI;
    const bool hidden = t0 + TI - 1 > all_see;
    if (hidden) {
      asm volatile("" ::: "memory");
      const bool any = any_nan<16 * DP>(at + KB + wave * 16 * DP, lane);
      if (lane == 0) odd[u & 1][wave] = any;
    }
    barrier_lds();   // tile u is there, and every wave is through with the one before, whose slot is asked for again
    if (asked < turns) request();
    out = out + 1 == SLOTS ? 0 : out + 1;
    if (hidden && __builtin_amdgcn_readfirstlane(odd[u & 1][0] | odd[u & 1][1] | odd[u & 1][2] | odd[u & 1][3])) {
      const int half = SPLIT == 1 ? 0 : wave / BLOCKS * 32;
#pragma unroll 1
      for (int x = half; x < (SPLIT == 1 ? TI : half + 32); x += 32) nan_seen32<DP>(read, at + KB + x * DP, last - t0 - x - 4 * h, acc);
      barrier_lds();   // every wave has seen the codes
      clear_nan<16 * DP>(at + KB + wave * 16 * DP, lane);
      barrier_lds();
    }
    if constexpr (SPLIT == 1) {
      if (t0 <= wave_last) block(t0, at, at_s);
      if (t0 + 32 <= wave_last) block(t0 + 32, at + 32 * DP, at_s + 32);
    } else {
      const int half = wave / BLOCKS * 32;
      if (t0 + half <= wave_last) block(t0 + half, at + half * DP, at_s + half);
    }
  }
  barrier_lds();
  if constexpr (SPLIT == 2) {   // the second halves' results to the waves of the first
    constexpr int BOX = DP * 32 + 128;
    static_assert(BLOCKS * BOX * 4 <= SLOTS * SLOT, "they take the tiles' place");
    float* box = reinterpret_cast<float*>(smem) + wave % BLOCKS * BOX + lane;
    if (wave >= BLOCKS) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) box[(db * 16 + r) * 64] = acc[db][r];
      box[DP * 32] = m;
      box[DP * 32 + 64] = l;
    }
    barrier_lds();
    if (wave < BLOCKS) {
      const float other = box[DP * 32], next = fmaxf(m, other);
      const float c = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - next), c2 = other == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(other - next);
      m = next;
      l = fmaf(box[DP * 32 + 64], c2, l * c);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[db][r] = fmaf(box[(db * 16 + r) * 64], c2, acc[db][r] * c);
    }
    barrier_lds();
    if (wave >= BLOCKS) return;
  }

  const float sum = half_sum(l), inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  const int r = first + l32;
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  if (joined || !PATCHED) {
    if (r >= rows) return;
    const int i = (int)t.by_group.div(r), g = r - i * t.G;
    const size_t all = (size_t)a.T * a.H, row = (size_t)(part.first + i) * a.H + hk * t.G + g;
    float* to = joined ? a.work + (run * all + row) * a.D : static_cast<float*>(a.o) + row * a.D;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int c = db * 32 + x * 8 + h * 4;
        if (c < a.D) *reinterpret_cast<f32x4*>(to + c) = f32x4{acc[db][x * 4] * inv, acc[db][x * 4 + 1] * inv, acc[db][x * 4 + 2] * inv,
                                                               acc[db][x * 4 + 3] * inv};
      }
    const float z = log_sum(m, sum, joined);
    if (h == 0 && joined) a.work[t.runs * all * a.D + run * all + row] = z;
    if (h == 0 && !joined && a.lse != nullptr) a.lse[row] = z * LN2;
    return;
  }
  if (a.lse != nullptr && h == 0 && r < rows) {
    const int i = (int)t.by_group.div(r), g = r - i * t.G;
    a.lse[(size_t)(part.first + i) * a.H + hk * t.G + g] = log_sum(m, sum, false) * LN2;
  }
  store_block<DP>(acc, inv, smem + wave * 32 * OP, rows - first, a.D, lane, [&](int r) {
    const int i = (int)t.by_group.div(first + r), g = first + r - i * t.G;
    return static_cast<unsigned short*>(a.o) + ((size_t)(part.first + i) * a.H + hk * t.G + g) * a.D;
  });
}

template <int DP, int SLOTS, int NP, int SPLIT, typename T>
static laser_status tile8_split(Tile8Args t) {
  const CacheArgs& c = t.a.c;
  t.rows_log2 = SPLIT == 2 ? 6 : 7;
  t.tiles = (int)(((long long)c.C * t.G + 128 / SPLIT - 1) / (128 / SPLIT));
  const long long most = (long long)t.N * t.Hkv * t.tiles * t.runs;
  t.ranked = t.N <= CACHE8_RANKED && most <= 2560;   // (ten a compute unit)
  if (t.ranked) {
    if (c.page_log2 >= 4) cache8_tile_kernel<DP, SLOTS, NP, 16, SPLIT, T><<<(unsigned)most, 256, 0, c.stream>>>(t);
    else cache8_tile_kernel<DP, SLOTS, NP, 8, SPLIT, T><<<(unsigned)most, 256, 0, c.stream>>>(t);
    return launch_status();
  }
  return launch_dealt(t, (long long)t.tiles * t.runs, 256, [&](Tile8Args& part, long long n) {
    part.a.c.pages += n * c.max_pages;
    part.a.c.lens += n;
    if (c.page_log2 >= 4) cache8_tile_kernel<DP, SLOTS, NP, 16, SPLIT, T><<<part.deal.grid, 256, 0, c.stream>>>(part);
    else cache8_tile_kernel<DP, SLOTS, NP, 8, SPLIT, T><<<part.deal.grid, 256, 0, c.stream>>>(part);
  });
}
// Two waves have the same 32 rows, and a half of each tile's items, where a head has at most 64 rows (us by four waves of rows and so: 64 rows x up
// to 4096, 32 users of 128 32.0 and 27.5, of 64 26.2 and 22.6; 40 x up to 3000, 64 of 64 28.5 and 24.7; fp32, 64 x up to 3000, 16 of 128 24.7 and
// 21.6), and where the tiles of 128 rows are one a compute unit or fewer: the way of each is then half as long, of twice as many (400 rows x 1000,
// 1 of 64 14.0 and 12.4; 800 x 3000, 2 of 128 29.1 and 26.7; 1200 x up to 600, 3 of 128 18.8 and 15.8; of 480 tiles 400 x 30000, 1 of 128 40.0 and
// 42.7, 100 x up to 3000, 20 of 64 24.8 and 22.4).
template <int DP, int SLOTS, int NP, typename T>
static laser_status tile8_typed(const Tile8Args& t) {
  const long long rows = (long long)t.a.c.C * t.G, workgroups = (rows + 127) / 128 * t.N * t.Hkv * t.runs;
  return rows <= 64 || workgroups <= 256 ? tile8_split<DP, SLOTS, NP, 2, T>(t) : tile8_split<DP, SLOTS, NP, 1, T>(t);
}
template <int NP, typename T>
static laser_status tile8_width(const Tile8Args& t) {
  if (t.a.c.D > 64) return tile8_typed<128, 3, NP, T>(t);
  if (t.a.c.D > 32) return tile8_typed<64, 4, NP, T>(t);
  return tile8_typed<32, 4, NP, T>(t);
}

laser_status cache8_tile_launch(const Cache8Args& a, const CacheRuns& r) {
  Tile8Args t{};
  t.a = a;
  t.off = a.c.off, t.N = a.c.U, t.Hkv = a.c.Hkv;
  t.G = a.c.H / a.c.Hkv;
  t.by_group = mul_div(t.G);
  t.scale = LOG2E / a.c.gamma;
  t.chunk = r.chunk, t.runs = r.runs;
  const laser_status s = a.c.dt == LASER_F32 ? tile8_width<3, float>(t) : tile8_width<1, unsigned short>(t);
  return s == LASER_OK && r.runs > 1 ? cache8_join_launch(a.c, r) : s;
}

}  // namespace laser
