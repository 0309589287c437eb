// Attention among the items of histories on the matrix cores (bf16): packed sequences, and rows over a paged cache.
//
// The rows of a key-value head are its G = H / H_kv query heads of every token, row r = token r / G, head r % G: shared keys and
// values are then read once for all of them. A workgroup of four waves owns 128 consecutive rows of one head of one sequence and
// walks the items that the last of them sees in tiles of 64; a wave owns 32 rows, whose queries stay in registers.
//   Sc^T[item, row] = K . Q^T             A = K from LDS, B = Q^T
//   P^T = exp2(Sc^T c - m)                the running maximum m and sum l of a row are one lane's (and its other half's) registers
//   acc^T[column, row] += V^T . P^T       A = V^T by the LDS transpose load, B = P^T as the accumulators hold it
// Tiles come by direct loads to LDS, the next ones behind the current one's arithmetic, one barrier a tile. Rows behind the valid
// ones read as zeros (the buffer's end), so padding that holds NaN never enters; their scores are masked.
//
// P is rounded to bf16 ahead of its product, which takes its operands so (in 32 bits it would take 16 times as long); l is the sum of P
// unrounded, in fp32. o is then off by 1.2 to 1.41 times what its own rounding costs (root mean square).
//
// Bound: products and exponentials together. A block of 32 items costs a wave of width 128 512 cycles of products and about 360 of vector
// arithmetic beside them, two waves share a SIMD, and the matrix cores are busy 52 % of the time.
// Histories of 3000 to 9000 items, 16 heads of 128 over 4: 683 to 697 us, 970 TFLOP/s (1250 us without the pipeline of block(); 1100 with it
// and every long sequence on one or two dies; 745 before a tile's read addresses were made once). Workgroups of eight waves 700 us
// and 64 rows a wave 760; over caches both are 10 to 35 % slower.
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
  int G, tiles;          // tiles of the longest sequence's rows
  Deal deal;             // of (tile, run) to workgroups
  float scale;           // log2(e) / gamma
  bool causal;
  unsigned short* o;
  float* lse;
  int chunk, runs;       // over a cache: items a workgroup walks, and into how many such runs the longest history is cut
  float* work;           // their results where a history has several
};

// Where the maximum of a row is raised: probabilities may stand up to 2^8 above it meanwhile, sums and outputs are in its units
constexpr float MAX_SLACK = 8.0f;

// Tiles come as pairs: values of items 64 u and on, keys of 32 items later (what turn u reads), pair u to slot u % SLOTS of a ring. Pair -1
// is the first 32 keys. A wave brings 16 rows of either kind.
constexpr int NW = 4;
template <int DP>
struct PairShape {
  static constexpr int ROW = DP * 2, CH = DP / 8, RPI = 64 / CH, KB = TI * ROW, SLOT = 2 * KB;
};

template <int DP, int SLOTS, bool PAGED>
__global__ __launch_bounds__(64 * NW, 2) void history_tile_kernel(const TileArgs a) {
  using Sh = PairShape<DP>;
  constexpr int KS = DP / 16, DB = DP / 32, ROWS = NW * 32, OP = DP * 2 + 16, PATCH = NW * 32 * OP;
  constexpr int MINE = TI / NW, RPW = MINE / Sh::RPI;   // a wave's rows of a tile, and its requests for them
  static_assert(MINE % Sh::RPI == 0 && MINE == 16, "whole requests, at most two pages of eight items");
  __shared__ __attribute__((aligned(1024))) unsigned char smem[SLOTS * Sh::SLOT > PATCH ? SLOTS * Sh::SLOT : PATCH];
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
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, h = lane >> 5;

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
  const int turns = end > begin ? (end - begin + TI - 1) / TI : 0;

  unsigned koff[RPW], voff[RPW];
#pragma unroll
  for (int x = 0; x < RPW; ++x) {
    const int in = x * Sh::RPI + lane / Sh::CH, r = wave * MINE + in, c = (lane % Sh::CH) ^ tile_swz<Sh::CH>(r);
    koff[x] = c * 8 < a.D ? (unsigned)((PAGED ? in * a.D : r * (int)a.kp) * 2 + c * 16) : NO_COLUMN;
    voff[x] = c * 8 < a.D ? (unsigned)((PAGED ? in * a.D : r * (int)a.vp) * 2 + c * 16) : NO_COLUMN;
  }
  const int32_t* table = PAGED ? a.pages + (size_t)n_seq * a.max_pages : nullptr;
  const bool short_pages = PAGED && a.log2 == 3;   // a wave's rows are on two pages
  // The table's next 64 entries wait in the lanes of a register, and those of the next pair are read from there: a scalar load under way
  // would make every wait for LDS in between a wait for it and for all of them.
  int ids[2][2], window = 0, window_at = -64;
  auto first_of = [&](int u, int kind) { return begin + (u < 0 ? 0 : u * TI + (kind ? 0 : 32)) + wave * MINE; };
  auto look_up = [&](int u) __attribute__((always_inline)) {
    if constexpr (PAGED) {
      const int lowest = first_of(u, 1) >> a.log2, highest = (first_of(u, 0) + 8) >> a.log2;
      if (highest >= window_at + 64) {
        window_at = lowest;
        const int x = window_at + lane, most = (end - 1) >> a.log2;
        window = table[x < most ? x : most];
      }
#pragma unroll
      for (int kind = 0; kind < 2; ++kind) {
        const int j = first_of(u, kind);
        ids[kind][0] = j < end ? __builtin_amdgcn_readlane(window, (j >> a.log2) - window_at) : -1;
        if (short_pages) ids[kind][1] = j + 8 < end ? __builtin_amdgcn_readlane(window, ((j + 8) >> a.log2) - window_at) : -1;
      }
    }
  };
  const unsigned page_bytes = PAGED ? (unsigned)((a.Hkv << a.log2) * a.D * 2) : 0, head_bytes = PAGED ? (unsigned)((hk << a.log2) * a.D * 2) : 0;
  auto fetch = [&](int u, unsigned at) __attribute__((always_inline)) {
    at += wave * MINE * Sh::ROW;
    if constexpr (PAGED) {
#pragma unroll
      for (int kind = 0; kind < 2; ++kind) {
        const int j = first_of(u, kind);
        const char* cache = reinterpret_cast<const char*>(kind ? a.v : a.k) + head_bytes;
        // rows j and on of a page, `skip` rows into the wave's own; places behind the last item read as zeros, like a page outside the pool
        auto page = [&](int id, int j, int count, int skip) __attribute__((always_inline)) {
          int left = n - j < count ? n - j : count;
          if ((unsigned)id >= (unsigned)a.P || (kind && u < 0)) left = -skip;
          const unsigned place = (unsigned)(j & ((1 << a.log2) - 1)) * a.D * 2;
          return buffer_of(cache + ((unsigned long long)(id < 0 ? 0 : id) * page_bytes + place) - skip * a.D * 2,
                           left + skip > 0 ? (unsigned)((left + skip) * a.D * 2) : 0u);
        };
        const unsigned* off = kind ? voff : koff;
        const unsigned to = at + (kind ? Sh::KB : 0);
        if (!short_pages) {
          const u32x4 b = page(ids[kind][0], j, MINE, 0);
#pragma unroll
          for (int x = 0; x < RPW; ++x) buffer_to_lds16(b, off[x], to + x * 1024);
        } else if constexpr (Sh::RPI > 8) {   // both pages in one request: each half of the lanes from its own
          if (lane < 32) buffer_to_lds16(page(ids[kind][0], j, 8, 0), off[0], to);
          else buffer_to_lds16(page(ids[kind][1], j + 8, 8, 8), off[0], to);
        } else {
          const u32x4 b0 = page(ids[kind][0], j, 8, 0), b1 = page(ids[kind][1], j + 8, 8, 8);
#pragma unroll
          for (int x = 0; x < RPW; ++x) buffer_to_lds16(x * Sh::RPI < 8 ? b0 : b1, off[x], to + x * 1024);
        }
      }
    } else {
      const int tk = u < 0 ? 0 : u * TI + 32, tv = u < 0 ? 0 : u * TI;
      int kl = end - tk, vl = u < 0 ? 0 : end - tv;
      kl = kl < TI ? kl : TI;
      vl = vl < TI ? vl : TI;
      const u32x4 kb = buffer_of(a.k + (size_t)(cr.first + tk) * a.kp + (size_t)hk * a.D, kl > 0 ? (unsigned)(((kl - 1) * (int)a.kp + a.D) * 2) : 0u);
      const u32x4 vb = buffer_of(a.v + (size_t)(cr.first + tv) * a.vp + (size_t)hk * a.D, vl > 0 ? (unsigned)(((vl - 1) * (int)a.vp + a.D) * 2) : 0u);
#pragma unroll
      for (int x = 0; x < RPW; ++x) {
        buffer_to_lds16(kb, koff[x], at + x * 1024);
        buffer_to_lds16(vb, voff[x], at + Sh::KB + x * 1024);
      }
    }
  };
  int asked = -1, in = SLOTS - 1;   // the next pair to ask for, and its slot
  auto request = [&]() __attribute__((always_inline)) {
    fetch(asked, lds + in * Sh::SLOT);
    in = in + 1 == SLOTS ? 0 : in + 1;
    ++asked;
    look_up(asked);
  };
  const int requests = short_pages && Sh::RPI > 8 ? 4 * RPW : 2 * RPW;
  if (turns > 0) {
    look_up(-1);
    for (int x = 0; x < SLOTS && x <= turns; ++x) request();   // pairs -1 .. SLOTS - 2
  }

  // this lane's row and the last item it sees
  const int first = row0 + wave * 32;
  int last;
  bf16x8 qreg[KS];
  {
    int r = first + l32;
    r = r < rows ? r : rows - 1;
    const int i = (int)a.by_group.div(r), g = r - i * a.G;
    last = a.causal ? n - cr.count + i : n - 1;
    const unsigned short* qr = a.q + (size_t)(cr.first + i) * a.qp + (size_t)(hk * a.G + g) * a.D;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      u32x4 raw = {0u, 0u, 0u, 0u};
      if (s * 16 + h * 8 < a.D) raw = *reinterpret_cast<const u32x4*>(qr + s * 16 + h * 8);
      qreg[s] = __builtin_bit_cast(bf16x8, raw);
    }
  }
  const int wave_first = __builtin_amdgcn_readlane(last, 0), wave_last = __builtin_amdgcn_readlane(last, 31);
  // is every page of the user's items one of the pool? (then only the last block has places without items)
  bool whole_pages = true;
  if constexpr (PAGED) {
    bool bad = false;
    if (turns > 0)
      for (int x = (begin >> a.log2) + lane; x <= (end - 1) >> a.log2; x += 64) bad |= (unsigned)table[x] >= (unsigned)a.P;
    whole_pages = __ballot(bad) == 0;
  }

  f32x16 acc[DB], sa, sb;   // (scores of a block and of the next)
  float m = -INFINITY, l = 0.0f;
  unsigned p[8] = {};
  bf16x8 kf[KS], vf[2][DB];
  const f32x16 zero = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    acc[db] = zero;
    vf[0][db] = vf[1][db] = __builtin_bit_cast(bf16x8, u32x4{0u, 0u, 0u, 0u});
  }
  TileReader<DP> read(lane);

  auto read_k = [&](int half) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < KS; ++s) kf[s] = read.rows(0, half, s);
  };
  auto read_v = [&](int half) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int db = 0; db < DB; ++db) vf[s][db] = read.cols(Sh::KB, half * 2 + s, db);
  };
  auto scores = [&](f32x16& sc) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < KS; ++s) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s], qreg[s], s == 0 ? zero : sc, 0, 0, 0);
  };
  auto values = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const u32x4 pf = {p[s * 4], p[s * 4 + 1], p[s * 4 + 2], p[s * 4 + 3]};
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[s][db], __builtin_bit_cast(bf16x8, pf), acc[db], 0, 0, 0);
      }
  };
  // scores of places without an item, and of items behind a row's own, become -inf
  auto mask = [&](f32x16& sc, int t0) __attribute__((always_inline)) {
    if (whole_pages && t0 + 31 <= wave_first && t0 + 32 <= n) return;
    bool in = l32 < n - t0;
    if (PAGED && !whole_pages) in = in && (unsigned)table[(t0 + (in ? l32 : 0)) >> a.log2] < (unsigned)a.P;
    const unsigned items = (unsigned)__ballot(in) >> (4 * h);
    const int seen = last - t0 - 4 * h;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int i0 = 8 * (r >> 2) + (r & 3);
      if (i0 > seen || !((items >> i0) & 1)) sc[r] = -INFINITY;
    }
  };
  auto raise = [&](const f32x16& sc) __attribute__((always_inline)) {
    float top = sc[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, sc[r]);
    top = half_max(top) * a.scale;
    if (__any(top > m + MAX_SLACK)) {   // (the first block: m is -inf)
      const float next = fmaxf(m, top), c = next == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - next);
      m = next;
      l *= c;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[db][r] *= c;
    }
  };
  auto weigh = [&](const f32x16& sc) __attribute__((always_inline)) {
    const float base = m == -INFINITY ? 0.0f : m;
    float sum = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
      const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[r], a.scale, -base));
      const float p1 = __builtin_amdgcn_exp2f(fmaf(sc[r + 1], a.scale, -base));
      sum += p0 + p1;
      p[r >> 1] = pack_bf16(p0, p1);
      asm volatile("" : "+v"(p[r >> 1]));   // (here, not where the next turn reads it)
    }
    l += sum;
    asm volatile("" : "+v"(l));
  };

  // A block of 32 items, half of a tile: its scores are there, those of the next block are made behind its exponentials, the last
  // block's sum of values behind its maximum
  auto block = [&](f32x16& sc, f32x16& next, int t0, int half) __attribute__((always_inline)) {
    read_k(half);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);   // (ahead of a wave at its barrier or its masks: 696 -> 688 us of the histories above)
    values();
    raise(sc);
    __builtin_amdgcn_sched_barrier(0);
    read_v(half);
    scores(next);
    weigh(sc);
#pragma unroll
    for (int x = 0; x < KS; ++x) {   // one product, then its share of the reads and of the exponentials
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 4 * DB / KS, 0);
      __builtin_amdgcn_sched_group_barrier(0x402, 64 / KS, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(0);
    mask(next, t0 + 32);
  };
  if (turns > 0) {
    wait_vm(asked * requests);
    barrier_lds();
    read.place_rows(lds + (SLOTS - 1) * Sh::SLOT);
    read_k(0);
    scores(sa);
    mask(sa, begin);
    int out = 0;
    for (int u = 0; u < turns; ++u) {
      wait_vm((asked - u - 1) * requests);
      barrier_lds();   // pair u is there, and every wave is through with the one before, whose slot is asked for again
      if (asked < turns) request();
      read.place(lds + out * Sh::SLOT);
      out = out + 1 == SLOTS ? 0 : out + 1;
      const int t0 = begin + u * TI;
      if (t0 <= wave_last) block(sa, sb, t0, 0);
      if (t0 + 32 <= wave_last) block(sb, sa, t0 + 32, 1);
    }
    values();
    barrier_lds();
  }

  // out: through a patch of the wave's own, so that the rows leave in whole 16-byte pieces
  const float sum = half_sum(l), inv = sum > 0.0f ? 1.0f / sum : 0.0f;
  const int r = first + l32;
  if (joined) {
    if (r >= rows) return;
    const int i = (int)a.by_group.div(r), g = r - i * a.G;
    const size_t all = (size_t)a.T * a.H, row = (size_t)(cr.first + i) * a.H + hk * a.G + g;
    float* to = a.work + (run * all + row) * a.D;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int c = db * 32 + x * 8 + h * 4;
        typedef float f32x4 __attribute__((ext_vector_type(4)));
        if (c < a.D) *reinterpret_cast<f32x4*>(to + c) = f32x4{acc[db][x * 4] * inv, acc[db][x * 4 + 1] * inv, acc[db][x * 4 + 2] * inv,
                                                               acc[db][x * 4 + 3] * inv};
      }
    if (h == 0) a.work[a.runs * all * a.D + run * all + row] = sum > 0.0f ? m + log2f(sum) : -INFINITY;
    return;
  }
  if (a.lse != nullptr && h == 0 && r < rows) {
    const int i = (int)a.by_group.div(r), g = r - i * a.G;
    a.lse[(size_t)(cr.first + i) * a.H + hk * a.G + g] = sum > 0.0f ? (m + log2f(sum)) * LN2 : -INFINITY;
  }
  store_block<DP>(acc, inv, smem + wave * 32 * OP, rows - first, a.D, lane, [&](int r) {
    const int i = (int)a.by_group.div(first + r), g = first + r - i * a.G;
    return a.o + ((size_t)(cr.first + i) * a.H + hk * a.G + g) * a.D;
  });
}

// The same over packed sequences where workgroups are few and the longest one's way is what counts: the waves are NG groups of NW, which own
// the same rows, take the tiles in turn, each with its own maximum and sum, and are joined at the end in their order.
template <int DP, int NW, int NG>
__global__ __launch_bounds__(64 * NW * NG, 2) void history_groups_kernel(const TileArgs a) {
  using Sh = TileShape<DP>;
  constexpr int KS = DP / 16, DB = DP / 32, ROWS = NW * 32, OP = DP * 2 + 16, STAGE = 2 * Sh::BYTES, TILES = 2 * NG * STAGE;
  static_assert(ROWS * DP * 4 <= TILES && NW * 32 * OP <= TILES, "what is joined, and the patches, take the tiles' place");
  __shared__ __attribute__((aligned(1024))) unsigned char smem[TILES];
  __shared__ float join_m[ROWS], join_l[ROWS];
  const unsigned lds = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem);
  const Place place = place_of(a.deal, blockIdx.x);
  if (place.rank >= a.deal.tiles) return;
  const int tile = a.tiles - 1 - place.rank;   // (the longest first)
  const int n_seq = place.pair / a.Hkv, hk = place.pair - n_seq * a.Hkv;
  const CandRange cr = cand_range(a.off, n_seq, a.C, a.T);
  const int n = cr.count, rows = n * a.G, row0 = tile * ROWS;
  if (row0 >= rows) return;
  const int wave_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = wave_all / NW, wave = wave_all % NW;
  const int lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
  const int end = (int)a.by_group.div(row0 + ROWS < rows ? row0 + ROWS - 1 : rows - 1) + 1;   // behind the last item that is seen

  PackedTiles<DP, NW> tiles;
  tiles.init(a.D, a.kp, a.vp, wave, lane);
  auto fetch = [&](int t0, unsigned at) __attribute__((always_inline)) {
    const size_t row = (size_t)(cr.first + t0);
    tiles.fetch(a.k + row * a.kp + (size_t)hk * a.D, a.v + row * a.vp + (size_t)hk * a.D, a.kp, a.vp, a.D, n - t0, at);
  };
  unsigned at = lds + group * 2 * STAGE, other = at + STAGE;
  if (group * TI < end) fetch(group * TI, at);

  const int first = row0 + wave * 32;
  int last;
  bf16x8 qreg[KS];
  {
    int r = first + l32;
    r = r < rows ? r : rows - 1;
    last = (int)a.by_group.div(r);
    const unsigned short* qr = a.q + (size_t)(cr.first + last) * a.qp + (size_t)(hk * a.G + r - last * a.G) * a.D;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      u32x4 raw = {0u, 0u, 0u, 0u};
      if (s * 16 + h * 8 < a.D) raw = *reinterpret_cast<const u32x4*>(qr + s * 16 + h * 8);
      qreg[s] = __builtin_bit_cast(bf16x8, raw);
    }
  }
  const int wave_first = __builtin_amdgcn_readlane(last, 0), wave_last = __builtin_amdgcn_readlane(last, 31);

  f32x16 acc[DB];
  const f32x16 zero = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = zero;
  float m = -INFINITY, l = 0.0f;
  TileReader<DP> read(lane);
  auto block = [&](int t0, int ib) __attribute__((always_inline)) {
    f32x16 sc;
#pragma unroll
    for (int s = 0; s < KS; ++s) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read.rows(0, ib, s), qreg[s], s == 0 ? zero : sc, 0, 0, 0);
    bf16x8 vt[2][DB];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int db = 0; db < DB; ++db) vt[s][db] = read.cols(Sh::BYTES, ib * 2 + s, db);
    if (t0 + 31 > wave_first) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (t0 + 8 * (r >> 2) + 4 * h + (r & 3) > last) sc[r] = -INFINITY;
    }
    float top = sc[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, sc[r]);
    top = half_max(top) * a.scale;
    if (__any(top > m + MAX_SLACK)) {   // (the first block: m is -inf)
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
    float sum = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
      const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[r], a.scale, -base)), p1 = __builtin_amdgcn_exp2f(fmaf(sc[r + 1], a.scale, -base));
      sum += p0 + p1;
      p[r >> 1] = pack_bf16(p0, p1);
    }
    l += sum;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const u32x4 b = {p[s * 4], p[s * 4 + 1], p[s * 4 + 2], p[s * 4 + 3]};
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vt[s][db], __builtin_bit_cast(bf16x8, b), acc[db], 0, 0, 0);
      }
  };
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
  barrier_lds();
  l = half_sum(l);
  float* mine = reinterpret_cast<float*>(smem) + (size_t)wave * 32 * DP + lane;
#pragma unroll 1
  for (int g = 1; g < NG; ++g) {
    if (group == g) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) mine[(db * 16 + r) * 64] = acc[db][r];
      if (h == 0) {
        join_m[wave * 32 + l32] = m;
        join_l[wave * 32 + l32] = l;
      }
    }
    __syncthreads();
    if (group == 0) {   // (it has the first tile, of which every row sees an item: its maximum is finite)
      const float m2 = join_m[wave * 32 + l32], top = fmaxf(m, m2), c = __builtin_amdgcn_exp2f(m - top), c2 = __builtin_amdgcn_exp2f(m2 - top);
      m = top;
      l = fmaf(join_l[wave * 32 + l32], c2, l * c);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[db][r] = fmaf(mine[(db * 16 + r) * 64], c2, acc[db][r] * c);
    }
    __syncthreads();
  }
  if (group > 0) return;
  const int r = first + l32;
  if (a.lse != nullptr && h == 0 && r < rows)
    a.lse[(size_t)(cr.first + last) * a.H + hk * a.G + r - last * a.G] = (m + log2f(l)) * LN2;
  store_block<DP>(acc, 1.0f / l, smem + wave * 32 * OP, rows - first, a.D, lane, [&](int r) {
    const int i = (int)a.by_group.div(first + r), g = first + r - i * a.G;
    return a.o + ((size_t)(cr.first + i) * a.H + hk * a.G + g) * a.D;
  });
}

template <int DP, int NW, int NG>
static laser_status groups_launch(TileArgs a, hipStream_t stream) {
  a.tiles = (int)(((long long)a.C * a.G + NW * 32 - 1) / (NW * 32));
  return launch_dealt(a, a.tiles, 64 * NW * NG, [&](const TileArgs& part, long long) {
    history_groups_kernel<DP, NW, NG><<<part.deal.grid, 64 * NW * NG, 0, stream>>>(part);
  });
}

template <int DP, int SLOTS, bool PAGED>
static laser_status tile_launch(TileArgs a, hipStream_t stream) {
  a.tiles = (int)(((long long)a.C * a.G + NW * 32 - 1) / (NW * 32));
  return launch_dealt(a, (long long)a.tiles * a.runs, 64 * NW, [&](TileArgs& part, long long n) {
    if constexpr (PAGED) {
      part.pages += n * a.max_pages;
      part.lens += n;
    }
    history_tile_kernel<DP, SLOTS, PAGED><<<part.deal.grid, 64 * NW, 0, stream>>>(part);
  });
}
template <bool PAGED>
static laser_status tile_launch_any(const TileArgs& a, hipStream_t stream) {
  // (as many pairs on the way as leave LDS for the two or three workgroups that the registers allow)
  if (a.D > 64) return tile_launch<128, 2, PAGED>(a, stream);
  if (a.D > 32) return tile_launch<64, 3, PAGED>(a, stream);
  return tile_launch<32, 4, PAGED>(a, stream);
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
  // Groups of waves where workgroups of 128 rows would leave much of the machine idle; four of two waves down to 256 rows, or two of four,
  // at width 128 only these, and there also where there are a few more, but long (us by the ring, four groups, two groups): one history of
  // 2894 items, 4 heads of 64 over 2 (92 workgroups) 46, 23, 34; 30 of 200, 4 of 64 over 4 (240, of 200 rows) 9.0, 12.2, 7.4; eight of 1000,
  // 8 of 64 over 2 (512) 22, 33, 19; width 128: two of 2635, 4 over one (166) 57, two groups 44; two of 4096, 8 over 2 (512) 102 and 85;
  // eight of 1000, 8 over 2 (512, of 4000 rows) 31.3 and 31.4.
  const long long rows = (long long)h.L * a.G, workgroups = (rows + 127) / 128 * h.N * h.Hkv;
  if (a.D > 64) {
    if (workgroups <= 256 || (workgroups <= 512 && rows >= 8192)) return groups_launch<128, 4, 2>(a, h.stream);
  } else if (workgroups <= 512) {
    if (workgroups <= 256 && rows >= 256) return a.D > 32 ? groups_launch<64, 2, 4>(a, h.stream) : groups_launch<32, 2, 4>(a, h.stream);
    return a.D > 32 ? groups_launch<64, 4, 2>(a, h.stream) : groups_launch<32, 4, 2>(a, h.stream);
  }
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
