// A few rows per key-value head over a cache of 8-bit blocks: one new item or a handful of candidates a user. Bound by memory, as
// cache_few.hip, whose split it has: a workgroup owns (user, key-value head, run of items), its four or eight waves take tiles of 32 items in turn,
// each with two tiles of its own in LDS and no barrier while it streams; at the end the waves' maxima, sums and outputs are joined in
// LDS, and the runs of a long history by a second launch.
//
// Tiles stand in LDS as the bytes that they are. Keys are read by rows, values by the transpose load of bytes, and both become bf16 operands times
// their block's scale in registers, exactly, so that scores and P V need no factors. Rows in bf16: P is rounded to bf16 ahead of its product.
// Rows in fp32: the query and P are sums of three bf16 numbers each, whose products with the operands are exact.
#include "cache8_tile.h"

namespace laser {

// A tile's products, and the state of a wave's rows: a lane holds a row's scores of 16 of the tile's items.
template <int DP, int NP>
struct Rows32 {
  static constexpr int ROWS = 32, KS = DP / 16, DB = DP / 32;
  static constexpr bool OCTETS = false;
  const TileReader8<DP> read;
  bf16x8 q[NP][KS];
  f32x16 acc[DB];
  float m = -INFINITY, l = 0.0f;
  __device__ __forceinline__ explicit Rows32(int lane) : read(lane) {
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[db][r] = 0.0f;
  }
  template <typename T>
  __device__ __forceinline__ void load(const T* qr, int D, int lane) { load_query<DP, NP>(qr, D, lane >> 5, q); }
  // `items` and `last`, where not all rows see all of the tile: the tile's items that are there, and the place of the last that the row sees
  __device__ __forceinline__ void tile(unsigned at_k, unsigned at_v, unsigned at_s, float scale, bool whole, unsigned items, int last, int lane) {
    const int h = lane >> 5;
    f32x16 sc = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    const float ks = read.key_scale(at_s);
#pragma unroll
    for (int i = 0; i < KS / 2; ++i) {
      const u32x4 w = read.rows(at_k, i);
      const bf16x8 k0 = wide8(w[0], w[1], ks, ks), k1 = wide8(w[2], w[3], ks, ks);
#pragma unroll
      for (int p = NP - 1; p >= 0; --p) {
        sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k0, q[p][2 * i], sc, 0, 0, 0);
        sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k1, q[p][2 * i + 1], sc, 0, 0, 0);
      }
    }
    if (!whole) {
      const int seen = last - 4 * h;
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
    top = half_max(top) * scale;
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
      const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[r], scale, -base)), p1 = __builtin_amdgcn_exp2f(fmaf(sc[r + 1], scale, -base));
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
        const u32x2 w = read.columns(at_v, s, db);
        const bf16x8 v = wide8(w[0], w[1], v0, v1);
#pragma unroll
        for (int i = NP - 1; i >= 0; --i) acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[i][s], acc[db], 0, 0, 0);
      }
    }
  }
  __device__ __forceinline__ void see_nan(unsigned at_v, int last, int lane) { nan_seen32<DP>(read, at_v, last - 4 * (lane >> 5), acc); }
  // to [column][32 rows], row r at r ^ column % 32
  __device__ __forceinline__ void leave(float* out, float* to_m, float* to_l, int lane) {
    const int l32 = lane & 31, h = lane >> 5;
    l = half_sum(l);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int d = 8 * (r >> 2) + 4 * h + (r & 3);
        out[(db * 32 + d) * 32 + (l32 ^ d)] = acc[db][r];
      }
    if (h == 0) {
      to_m[l32] = m;
      to_l[l32] = l;
    }
  }
};

// At most 16 rows: a lane holds a row's scores of 8 of the items, half the exponentials and half the time of the products, and the values are
// read ahead of the scores, for which there are registers (us by 32 rows and by 16: one token for 128 users x up to 4096 24.6 and 21.6, fp32 for
// 5 x up to 777 10.3 and 7.8, 64 x 1000 11.8 and 10.1, 100 x up to 3000 of width 32
// 18.0 and 15.5; keys and values at once, with the tile's place asked for again ahead of the products: 22.5, 7.7, 10.3;
// four tiles a wave instead of two, with 32 rows of 64: 25.2 and 30.9 us for 64 x up to 8192). Product x of a
// tile's two has the items 8 (i / 4) + 4 x + i % 4 as its rows i, so that a lane of the scores, items 8 g + 4 x .. + 3 for g = lane / 16,
// has the octet 8 g .. 8 g + 7 that it is to have of the other factor.
template <int DP, int NP>
struct Rows16 {
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  static constexpr int ROWS = 16, CH = DP / 16, KC = DP > 32 ? DP / 64 : 1, KS = DP > 32 ? 2 : 1, DB = DP / 16;   // (width 32: one product of 32 columns)
  static constexpr bool OCTETS = true;
  unsigned row, cols, ks, vs;
  bf16x8 q[NP][KC][KS];
  f32x4 acc[DB];
  float m = -INFINITY, l = 0.0f;
  __device__ __forceinline__ explicit Rows16(int lane) {
    const int i = lane & 15, g = lane >> 4, r = 8 * (i >> 2) + (i & 3), k = 8 * g + (i >> 1);
    row = r * DP + (KS == 2 ? (g ^ swz8_octets<CH>(r)) << 4 : (((g >> 1) ^ swz8_octets<CH>(r)) << 4) + (g & 1) * 8);
    cols = k * DP + (swz8_octets<CH>(k) << 4) + (i & 1) * 8;
    ks = (i >> 3) * 16 + ((i >> 2) & 1) * 4;
    vs = (g >> 1) * 16 + (g & 1) * 4 + 8;
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[db] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  // columns 64 c + 16 (lane / 16) and on; of width 32 8 (lane / 16) and on
  template <typename T>
  __device__ __forceinline__ void load(const T* qr, int D, int lane) {
#pragma unroll
    for (int c = 0; c < KC; ++c)
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int d = c * 64 + (lane >> 4) * 8 * KS + s * 8;
        float x[8];
        bf16x8 part[NP];
        if constexpr (NP == 1) {
          u32x4 raw = {0u, 0u, 0u, 0u};
          if (d < D) raw = *reinterpret_cast<const u32x4*>(qr + d);
          part[0] = __builtin_bit_cast(bf16x8, raw);
        } else {
#pragma unroll
          for (int j = 0; j < 8; j += 4) {
            f32x4 raw = {0.0f, 0.0f, 0.0f, 0.0f};
            if (d < D) raw = *reinterpret_cast<const f32x4*>(qr + d + j);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[j + e] = raw[e];
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            __bf16 b[NP];
            split_bf16<NP>(x[j], b);
#pragma unroll
            for (int i = 0; i < NP; ++i) part[i][j] = b[i];
          }
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) q[i][c][s] = part[i];
      }
  }
  __device__ __forceinline__ u32x2 columns(unsigned at_v, int db) const {
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2*)(lds_at((at_v + cols) ^ (db << 4)))));
  }
  __device__ __forceinline__ void tile(unsigned at_k, unsigned at_v, unsigned at_s, float scale, bool whole, unsigned items, int last, int lane) {
    const int g = lane >> 4;
    f32x4 sc[2];
    const float k_scale = *reinterpret_cast<const __attribute__((address_space(3))) float*>(lds_at(at_s + ks));
    float v_scale = *reinterpret_cast<const __attribute__((address_space(3))) float*>(lds_at(at_s + vs));
    u32x4 kw[2][KC];
    u32x2 vw[DB];   // (read ahead of the scores, so that no product waits for LDS)
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int c = 0; c < KC; ++c) {   // (row + 4 x: its piece moves by the swizzle of bit 2 alone)
        if constexpr (KS == 2) {
          kw[x][c] = __builtin_bit_cast(u32x4, lds_read16(lds_at(((at_k + row) ^ (c << 6) ^ (x * (CH == 8 ? 4 : 1) << 4)) + x * 4 * DP)));
        } else {
          const u32x2 w = *reinterpret_cast<const __attribute__((address_space(3))) u32x2*>(lds_at(at_k + row + x * 4 * DP));
          kw[x][c] = u32x4{w[0], w[1], 0u, 0u};
        }
      }
#pragma unroll
    for (int db = 0; db < DB; ++db) vw[db] = columns(at_v, db);
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      sc[x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const u32x4 w = kw[x][c];
        const bf16x8 k0 = wide8(w[0], w[1], k_scale, k_scale), k1 = wide8(w[2], w[3], k_scale, k_scale);
#pragma unroll
        for (int p = NP - 1; p >= 0; --p) {
          sc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, q[p][c][0], sc[x], 0, 0, 0);
          if constexpr (KS == 2) sc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, q[p][c][1], sc[x], 0, 0, 0);
        }
      }
    }
    if (!whole) {
      const int seen = last - 8 * g;
      const unsigned mine = items >> (8 * g);
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (4 * x + r > seen || !((mine >> (4 * x + r)) & 1)) sc[x][r] = -INFINITY;
      v_scale = mine & 1 ? v_scale : 1.0f;   // (a block without items has no scale; its codes came as zeros)
    }
    float top = sc[0][0];
#pragma unroll
    for (int r = 1; r < 8; ++r) top = fmaxf(top, sc[r >> 2][r & 3]);
    top = quarter_max(top) * scale;
    if (__any(top > m + MAX_SLACK)) {   // (the first tile: m is -inf)
      const float next = fmaxf(m, top), c = next == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - next);
      m = next;
      l *= c;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[db][r] *= c;
    }
    const float base = m == -INFINITY ? 0.0f : m;
    bf16x8 p[NP][2];
    float sum = 0.0f;
#pragma unroll
    for (int r = 0; r < 8; r += 2) {
      const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[r >> 2][r & 3], scale, -base)), p1 = __builtin_amdgcn_exp2f(fmaf(sc[r >> 2][(r & 3) + 1], scale, -base));
      sum += p0 + p1;
      split_pair<NP>(p0, p1, r, p);
    }
    l += sum;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const bf16x8 v = wide8(vw[db][0], vw[db][1], v_scale, v_scale);
#pragma unroll
      for (int i = NP - 1; i >= 0; --i) acc[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[i][0], acc[db], 0, 0, 0);
    }
  }
  __device__ __forceinline__ void see_nan(unsigned at_v, int last, int lane) {
    bf16x8 sees;
#pragma unroll
    for (int r = 0; r < 8; ++r) sees[r] = (__bf16)(r <= last - 8 * (lane >> 4) ? 1.0f : 0.0f);
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const f32x4 count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones_at(nan_codes(columns(at_v, db))), sees, f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[db][r] = count[r] > 0.0f ? __builtin_nanf("") : acc[db][r];
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // to [column][16 rows], row r at r ^ column % 16
  __device__ __forceinline__ void leave(float* out, float* to_m, float* to_l, int lane) {
    const int i = lane & 15, g = lane >> 4;
    l = quarter_sum(l);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 4; ++r) out[(db * 16 + 4 * g + r) * 16 + (i ^ (4 * g + r))] = acc[db][r];
    if (g == 0) {
      to_m[i] = m;
      to_l[i] = l;
    }
  }
};

template <int DP>
struct Few8Shape {
  static constexpr int TILE = 32 * DP, STAGE = 2 * TILE, NST = 2, WAVE = NST * STAGE;
  static constexpr int JOIN = DP * 32 * 4;   // [column][32 rows] of fp32, row r at r ^ column % 32
  static_assert(JOIN <= WAVE, "the outputs take the tiles' place");
};

template <int DP, int NW, int PART, typename Rows, typename T>
__global__ __launch_bounds__(64 * NW, 2) void cache8_few_kernel(const Cache8Args a8, int G, MulDiv by_group, float scale, int chunk, int splits) {
  using Sh = Few8Shape<DP>;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[NW * Sh::WAVE];
  __shared__ __attribute__((aligned(16))) float scales[NW][Sh::NST][8];
  __shared__ float join_m[NW][Rows::ROWS], join_l[NW][Rows::ROWS];
  const CacheArgs& a = a8.c;
  const int per = a.U * a.Hkv;
  // (turned by one from run to run: a user's runs are not all one die's)
  const int split = blockIdx.x / per, uh = (blockIdx.x + split) % per, u = uh / a.Hkv, hk = uh % a.Hkv;
  const CandRange cr = cand_range(a.off, u, a.C, a.T);
  const int rows = cr.count * G;
  if (rows == 0) return;
  const int n = cache_len(a.lens, u, a.L, a.max_pages, a.page_log2);
  const int lo = split * chunk, hi = n < lo + chunk ? n : lo + chunk;
  if (lo >= n && split > 0) return;   // (the first run of an empty history still writes)
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const unsigned lds = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem) + wave * Sh::WAVE;
  const unsigned lds_s = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(__attribute__((address_space(3))) float*)&scales[wave][0][0]);
  const int32_t* table = a.pages + (size_t)u * a.max_pages;

  Tiles8<DP, 32, PART, Rows::OCTETS> tiles;
  tiles.init(a.D, a.page_log2, 0, lane);
  const int step_items = NW * 32, requests = tiles.requests();
  int ask = lo + wave * 32, mine = ask;
  int pending = 0, slot_in = 0, slot_out = 0;
  tiles.look_up(table, ask, hi, a.page_log2);
  auto request = [&]() __attribute__((always_inline)) {
    const unsigned at = lds + slot_in * Sh::STAGE;
    tiles.fetch(a8, hk, ask, hi, at, at + Sh::TILE, lds_s + slot_in * 32, lane);
    slot_in = slot_in + 1 == Sh::NST ? 0 : slot_in + 1;
    ask += step_items;
    ++pending;
    tiles.look_up(table, ask, hi, a.page_log2);
  };

  Rows mine_rows(lane);
  int last;
  {
    const int at = lane & (Rows::ROWS - 1), r = at < rows ? at : rows - 1, i = (int)by_group.div(r), g = r - i * G;
    last = a.causal ? n - cr.count + i : n - 1;
    mine_rows.load(static_cast<const T*>(a.q) + (size_t)(cr.first + i) * a.qp + (size_t)(hk * G + g) * a.D, a.D, lane);
  }
  const int first_seen = __builtin_amdgcn_readlane(last, 0);
  bool whole_pages;
  {
    bool bad = false;
    for (int x = (lo >> a.page_log2) + lane; x <= (hi - 1) >> a.page_log2 && lo < hi; x += 64) bad |= (unsigned)table[x] >= (unsigned)a.P;
    whole_pages = __ballot(bad) == 0;
  }
  for (int x = 0; x < Sh::NST && ask < hi; ++x) request();

  for (; mine < hi; mine += step_items) {
    // loads return in order: with a second tile asked for, the first is there when the second's requests are all that is left
    wait_requests(pending > 1 ? requests : 0);
    asm volatile("" ::: "memory");
    const unsigned at = lds + slot_out * Sh::STAGE, at_s = lds_s + slot_out * 32;
    const bool whole = whole_pages && mine + 31 <= first_seen && mine + 32 <= hi;
    unsigned items = ~0u;
    if (!whole) {
      const int at = lane & 31;
      bool in = at < hi - mine;
      if (!whole_pages) in = in && (unsigned)table[(mine + (in ? at : 0)) >> a.page_log2] < (unsigned)a.P;
      items = (unsigned)__ballot(in);
    }
    if ((mine + 32 < hi ? mine + 32 : hi) - 1 > first_seen && any_nan<Sh::TILE>(at + Sh::TILE, lane)) {   // (items that not every row sees)
      mine_rows.see_nan(at + Sh::TILE, last - mine, lane);
      clear_nan<Sh::TILE>(at + Sh::TILE, lane);
    }
    mine_rows.tile(at, at + Sh::TILE, at_s, scale, whole, items, last - mine, lane);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the tile has been read: its place may be asked for again
    --pending;
    slot_out = slot_out + 1 == Sh::NST ? 0 : slot_out + 1;
    if (ask < hi) request();
  }

  // the waves' results, in the place of the tiles
  mine_rows.leave(reinterpret_cast<float*>(smem + wave * Sh::WAVE), join_m[wave], join_l[wave], lane);
  __syncthreads();
  const bool final = n <= chunk;
  for (int e = tid; e < rows * a.D; e += 64 * NW) {
    const int r = e / a.D, d = e - r * a.D;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, join_m[w][r]);
    float sum = 0.0f, x = 0.0f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float mw = join_m[w][r], c = mw == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mw - top);
      sum = fmaf(join_l[w][r], c, sum);
      x = fmaf(reinterpret_cast<const float*>(smem + w * Sh::WAVE)[d * Rows::ROWS + (r ^ (d & (Rows::ROWS - 1)))], c, x);
    }
    x = sum == 0.0f ? 0.0f : x / sum;
    const float z = log_sum(top, sum, !final);
    const int i = (int)by_group.div(r), g = r - i * G;
    const size_t row = (size_t)(cr.first + i) * a.H + hk * G + g;
    if (final) {
      store_from_f32<T>(static_cast<T*>(a.o), row * a.D + d, x);
      if (d == 0 && a.lse != nullptr) a.lse[row] = z * LN2;
    } else {
      const size_t all = (size_t)a.T * a.H;
      a.work[(split * all + row) * a.D + d] = x;
      if (d == 0) a.work[splits * all * a.D + split * all + row] = z;
    }
  }
}

// Joins the parts of a row that are more than 16: a workgroup a row and 32 of its columns, eight lanes a part, 128 parts at a time, whose columns are
// asked for ahead of the parts' shares, so that a row is two loads behind one another and not three. For few rows: the call with it, captured, us, by
// cache_join_kernel and by this one: 16 rows of 128 columns in 127 parts 15.1 and 13.9 (fp32 17.8 and 16.2; calls in a row from Python are 15.7 by either,
// the host's part), 64 rows in 59 18.3 and 17.6, 64 rows of 8 users in 20 27.5 and 26.8; 800 rows in 59 39.7 and 41.0, 7200 rows of 64 in 34 110 and 118.
constexpr int JOIN_PARTS = 1024, JOIN_COLUMNS = 32;
template <typename T>
__global__ __launch_bounds__(256) void cache8_join_kernel(const CacheArgs a, int chunk, int splits, MulDiv by_slices, int slices) {
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  constexpr int NT = 256, LANES = JOIN_COLUMNS / 4, GROUPS = NT / LANES, AHEAD = 4, MINE = JOIN_PARTS / NT;
  __shared__ float share[JOIN_PARTS];
  __shared__ __attribute__((aligned(16))) float part[NT / 64][JOIN_COLUMNS];
  __shared__ float wave_top[NT / 64], wave_sum[NT / 64];
  const int u = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, group = tid / LANES;
  const CandRange cr = cand_range(a.off, u, a.C, a.T);
  const int x = (int)by_slices.div(blockIdx.x), d = ((int)blockIdx.x - x * slices) * JOIN_COLUMNS + tid % LANES * 4;
  const int n = cache_len(a.lens, u, a.L, a.max_pages, a.page_log2);
  if (n <= chunk || x >= cr.count * a.H) return;   // (one part: it has written the result)
  const size_t all = (size_t)a.T * a.H, row = (size_t)cr.first * a.H + x;
  const int seen = a.causal ? n - cr.count + x / a.H + 1 : n, parts = seen <= 0 ? 0 : (seen + chunk - 1) / chunk;
  const float* z = a.work + splits * all * a.D + row;
  const float* at = a.work + row * a.D + (d < a.D ? d : 0);
  f32x4 y[AHEAD];
#pragma unroll
  for (int e = 0; e < AHEAD; ++e) {   // (behind the last part: the last one again, with no share)
    const int s = group + e * GROUPS, k = s < parts ? s : parts > 0 ? parts - 1 : 0;
    y[e] = *reinterpret_cast<const f32x4*>(at + k * all * a.D);
  }
  float mine[MINE], top = -INFINITY, sum = 0.0f;
#pragma unroll
  for (int i = 0; i < MINE; ++i) {
    mine[i] = i * NT + tid < parts ? z[(i * NT + tid) * all] : -INFINITY;
    top = fmaxf(top, mine[i]);
  }
  for (int m = 32; m; m >>= 1) top = fmaxf(top, __shfl_xor(top, m));
  if (lane == 0) wave_top[wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) top = fmaxf(top, wave_top[w]);
#pragma unroll
  for (int i = 0; i < MINE; ++i)
    if (i * NT + tid < parts) {
      const float c = mine[i] == -INFINITY ? 0.0f : exp2f(mine[i] - top);
      share[i * NT + tid] = c;
      sum += c;
    }
  for (int m = 32; m; m >>= 1) sum += __shfl_xor(sum, m);
  if (lane == 0) wave_sum[wave] = sum;
  __syncthreads();
  sum = 0.0f;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) sum += wave_sum[w];
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s0 = 0; s0 < parts; s0 += AHEAD * GROUPS) {
#pragma unroll
    for (int e = 0; e < AHEAD; ++e) {
      const int s = s0 + group + e * GROUPS;
      const float c = s < parts ? share[s] : 0.0f;
      if (s < parts) {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = fmaf(c, y[e][i], o[i]);
      }
      const int next = s + AHEAD * GROUPS;
      if (next < parts) y[e] = *reinterpret_cast<const f32x4*>(at + next * all * a.D);
    }
  }
#pragma unroll
  for (int m = LANES; m < 64; m <<= 1)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += __shfl_xor(o[i], m);
  if (lane < LANES) *reinterpret_cast<f32x4*>(&part[wave][lane * 4]) = o;
  __syncthreads();
  const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
  const int c = d - tid % LANES * 4 + tid;
  if (tid < JOIN_COLUMNS && c < a.D) {
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) v += part[w][tid];
    store_from_f32<T>(static_cast<T*>(a.o), row * a.D + c, v * by);
    if (c == 0 && a.lse != nullptr) a.lse[row] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * LN2;
  }
}
laser_status cache8_join_launch(const CacheArgs& a, const CacheRuns& r) {
  const int slices = (a.D + JOIN_COLUMNS - 1) / JOIN_COLUMNS;
  const long long grid = (long long)a.C * a.H * slices;
  if (r.runs <= 16 || grid * a.U > 1024) return cache_join_launch(a, r.chunk, r.runs);
  const dim3 size((unsigned)grid, (unsigned)a.U);
  if (a.dt == LASER_F32) cache8_join_kernel<float><<<size, 256, 0, a.stream>>>(a, r.chunk, r.runs, mul_div(slices), slices);
  else cache8_join_kernel<unsigned short><<<size, 256, 0, a.stream>>>(a, r.chunk, r.runs, mul_div(slices), slices);
  return launch_status();
}

template <int DP, int NW, typename Rows, typename T>
static laser_status few8_typed(const Cache8Args& a, const CacheRuns& r) {
  const CacheArgs& c = a.c;
  const int G = c.H / c.Hkv;
  const long long each = (long long)c.Hkv * r.runs;   // workgroups of a user
  if (c.U * each > 0x7fffffffLL) return LASER_ERR_SHAPE;
  const long long most = 0xffffffffLL / (64 * NW) / each;   // (a launch has fewer than 2^32 threads; a user has Hkv * runs <= 2^20 workgroups)
  for (long long u = 0; u < c.U; u += most) {
    Cache8Args part = a;
    part.c.U = c.U - u < most ? (int)(c.U - u) : (int)most;
    part.c.off = c.off + u;
    part.c.pages = c.pages + u * c.max_pages;
    part.c.lens = c.lens + u;
    const unsigned grid = (unsigned)(part.c.U * each);
    const MulDiv by_group = mul_div(G);
    if (c.page_log2 >= 4) cache8_few_kernel<DP, NW, 16, Rows, T><<<grid, 64 * NW, 0, c.stream>>>(part, G, by_group, LOG2E / c.gamma, r.chunk, r.runs);
    else cache8_few_kernel<DP, NW, 8, Rows, T><<<grid, 64 * NW, 0, c.stream>>>(part, G, by_group, LOG2E / c.gamma, r.chunk, r.runs);
    const laser_status s = launch_status();
    if (s != LASER_OK) return s;
  }
  return r.runs > 1 ? cache8_join_launch(c, r) : LASER_OK;
}
template <int NP, int NW, typename T>
static laser_status few8_width(const Cache8Args& a, const CacheRuns& r) {
  const bool sixteen = a.c.C * (a.c.H / a.c.Hkv) <= 16;
  if (a.c.D > 64) return sixteen ? few8_typed<128, NW, Rows16<128, NP>, T>(a, r) : few8_typed<128, NW, Rows32<128, NP>, T>(a, r);
  if (a.c.D > 32) return sixteen ? few8_typed<64, NW, Rows16<64, NP>, T>(a, r) : few8_typed<64, NW, Rows32<64, NP>, T>(a, r);
  return sixteen ? few8_typed<32, NW, Rows16<32, NP>, T>(a, r) : few8_typed<32, NW, Rows32<32, NP>, T>(a, r);
}
laser_status cache8_few_launch(const Cache8Args& a, const CacheRuns& r) {
  if (cache8_waves(a.c.U, a.c.Hkv, r) == 8) return a.c.dt == LASER_F32 ? few8_width<3, 8, float>(a, r) : few8_width<1, 8, unsigned short>(a, r);
  return a.c.dt == LASER_F32 ? few8_width<3, 4, float>(a, r) : few8_width<1, 4, unsigned short>(a, r);
}

}  // namespace laser
