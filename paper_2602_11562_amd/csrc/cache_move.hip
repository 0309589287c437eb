// What moves rows of a paged cache: new items into it, and the items that stay into fresh pages.
#include "history.h"

namespace laser {

// New rows into the cache: user u's c rows are the last c of its lens[u] items. A thread moves 16 bytes of a key row and of a
// value row; consecutive threads run along a row, so every piece is whole and nothing is read twice. Bound by memory: 2 x the
// rows' bytes; 2.4 us of five rows, 5.4 of 8192 rows of 2 heads of 128 (17 MB in all, most of them in the caches).
__global__ __launch_bounds__(256) void cache_append_kernel(const unsigned char* __restrict__ k, const unsigned char* __restrict__ v,
                                                           long long k_row, long long v_row, unsigned char* __restrict__ kc,
                                                           unsigned char* __restrict__ vc, const int32_t* __restrict__ off,
                                                           const int32_t* __restrict__ pages, const int32_t* __restrict__ lens,
                                                           int T, int C, int L, int Hkv, int head_bytes, int log2, int P,
                                                           int max_pages, float* __restrict__ weight) {
  const int u = blockIdx.y;
  const CandRange r = cand_range(off, u, C, T);
  const int n = cache_len(lens, u, L, max_pages, log2);
  const int pieces = head_bytes >> 4;
  const int per_row = pieces * Hkv;
  const long long all = (long long)r.count * per_row;
  for (long long e = (long long)blockIdx.x * 256 + threadIdx.x; e < all; e += (long long)gridDim.x * 256) {
    const int i = (int)(e / per_row), x = (int)(e % per_row), h = x / pieces, piece = x % pieces;
    const int j = n - r.count + i;
    if (j < 0) continue;   // more new rows than items
    const int page = pages[(size_t)u * max_pages + (j >> log2)];
    if ((unsigned)page >= (unsigned)P) continue;
    const int place = j & ((1 << log2) - 1);
    const size_t to = (((((size_t)page * Hkv + h) << log2) + place) * pieces + piece) << 4;
    const size_t at = (size_t)h * head_bytes + piece * 16, tok = (size_t)r.first + i;
    *reinterpret_cast<stream16*>(kc + to) = *reinterpret_cast<const stream16*>(k + tok * k_row + at);
    *reinterpret_cast<stream16*>(vc + to) = *reinterpret_cast<const stream16*>(v + tok * v_row + at);
    if (weight != nullptr && x == 0) weight[((size_t)page << log2) + place] = 0.0f;
  }
}

laser_status cache_append_launch(const CacheAppendArgs& a) {
  const CacheArgs& c = a.c;
  const int e = c.dt == LASER_F32 ? 4 : 2;
  const long long most = (long long)c.C * c.Hkv * c.D * e / 16;   // pieces of a user with C rows
  const int gx = (int)((most + 255) / 256 < 256 ? (most + 255) / 256 : 256);
  for (long long u = 0; u < c.U; u += 65535) {
    const int users = c.U - u < 65535 ? c.U - u : 65535;
    cache_append_kernel<<<dim3(gx, users), 256, 0, c.stream>>>(
        static_cast<const unsigned char*>(a.k), static_cast<const unsigned char*>(a.v), a.kp * e, a.vp * e,
        static_cast<unsigned char*>(c.k), static_cast<unsigned char*>(c.v), c.off + u, c.pages + (size_t)u * c.max_pages,
        c.lens + u, c.T, c.C, c.L, c.Hkv, c.D * e, c.page_log2, c.P, c.max_pages, c.weight);
  }
  return launch_status();
}

// Which items stay: the `recent` last ones and, of the others, the budget - recent heaviest (of equal ones the first). A
// workgroup per user finds the weight of the last one that stays by four passes over the weights, eight bits of the key a pass
// (a key orders as its float does, NaN below everything), then lists the items that stay in order by counting them.
constexpr int SEL = 1024, HELD = 8;

__device__ __forceinline__ unsigned weight_key(float w) {
  if (w != w) return 0u;
  const unsigned b = __float_as_uint(w == 0.0f ? 0.0f : w);   // (the zeros are equal)
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// (lens and lens_out may be one array)
__global__ __launch_bounds__(SEL) void cache_select_kernel(const float* __restrict__ weight, const int32_t* __restrict__ pages,
                                                           const int32_t* lens, int L, int log2, int P,
                                                           int max_pages, int budget, int recent, int32_t* lens_out,
                                                           int32_t* __restrict__ kept) {
  __shared__ int hist[256];
  __shared__ int wave_keep[SEL / 64], wave_tie[SEL / 64];
  __shared__ int chosen, above;
  const int u = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = cache_len(lens, u, L, max_pages, log2);
  const int stay = n < budget ? n : budget;
  int32_t* out = kept + (size_t)u * budget;
  const int32_t* table = pages + (size_t)u * max_pages;
  __syncthreads();   // (every wave has its length before it is overwritten)
  if (tid == 0) lens_out[u] = stay;
  for (int i = stay + tid; i < budget; i += SEL) out[i] = -1;
  if (n <= budget) {
    for (int i = tid; i < n; i += SEL) out[i] = i;
    return;
  }
  const int old = n - recent;              // items that compete (recent <= budget < n)
  const int want = budget - recent;        // how many of them stay
  auto key_of = [&](int j) {
    const int page = table[j >> log2];
    return (unsigned)page < (unsigned)P ? weight_key(weight[((size_t)page << log2) + (j & ((1 << log2) - 1))]) : 0u;
  };
  // a thread's first keys wait in registers; a longer history's others are read again in every pass
  unsigned keys[HELD];
#pragma unroll
  for (int x = 0; x < HELD; ++x) keys[x] = x * SEL + tid < old ? key_of(x * SEL + tid) : 0u;
  auto each = [&](auto&& use) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < HELD; ++x)
      if (x * SEL + tid < old) use(keys[x]);
    for (int j = HELD * SEL + tid; j < old; j += SEL) use(key_of(j));
  };
  unsigned limit = 0xffffffffu;            // the smallest key that stays
  int ties = 0;                            // how many of the items with that key stay
  if (want > 0) {
    unsigned prefix = 0;
    int left = want;
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int b = tid; b < 256; b += SEL) hist[b] = 0;
      __syncthreads();
      each([&](unsigned key) {
        if (shift == 24 || (key >> (shift + 8)) == prefix) atomicAdd(&hist[(key >> shift) & 255], 1);
      });
      __syncthreads();
      if (tid < 64) {   // the digit in which the items counted from the heaviest reach `left`
        int mine[4], sum = 0;
        for (int b = 0; b < 4; ++b) sum += mine[b] = hist[255 - (tid * 4 + b)];
        int before = sum;
        for (int d = 1; d < 64; d <<= 1) {
          const int x = __shfl_up(before, d);
          if (tid >= d) before += x;
        }
        before -= sum;
        for (int b = 0; b < 4; ++b) {
          if (before < left && left <= before + mine[b]) {
            chosen = 255 - (tid * 4 + b);
            above = before;
          }
          before += mine[b];
        }
      }
      __syncthreads();
      prefix = prefix << 8 | (unsigned)chosen;
      left -= above;
      __syncthreads();
    }
    limit = prefix;
    ties = left;
  }
  int at = 0, tied = 0;                    // items listed so far, and those of them with the limit's key
  auto list = [&](int base, unsigned held, bool is_held) __attribute__((always_inline)) {
    const int j = base + tid;
    const unsigned key = is_held ? held : j < old ? key_of(j) : 0u;
    const bool tie = want > 0 && j < old && key == limit;
    const unsigned long long ties_here = __ballot(tie), under = (1ull << lane) - 1;
    if (lane == 0) wave_tie[wave] = __popcll(ties_here);
    __syncthreads();
    int tie_before = tied, tie_all = 0;
    for (int x = 0; x < SEL / 64; ++x) {
      if (x < wave) tie_before += wave_tie[x];
      tie_all += wave_tie[x];
    }
    const bool keep = j < n && (j >= old || (want > 0 && (key > limit || (tie && tie_before + __popcll(ties_here & under) < ties))));
    const unsigned long long keeps = __ballot(keep);
    if (lane == 0) wave_keep[wave] = __popcll(keeps);
    __syncthreads();
    int before = at, all = 0;
    for (int x = 0; x < SEL / 64; ++x) {
      if (x < wave) before += wave_keep[x];
      all += wave_keep[x];
    }
    if (keep) out[before + __popcll(keeps & under)] = j;
    at += all;
    tied += tie_all;
  };
#pragma unroll
  for (int x = 0; x < HELD; ++x)
    if (x * SEL < n) list(x * SEL, keys[x], true);
  for (int base = HELD * SEL; base < n; base += SEL) list(base, 0u, false);
}

// The items that stay into their new pages, with their weights: a thread per 16 bytes of a key row and of a value row. Bound by
// memory, each byte once in and once out: 48 users keep up to 2048 items of 2 heads of 128, 28 us for 180 MB (6.3 TB/s, what it writes
// standing in the last cache).
__global__ __launch_bounds__(256) void cache_move_kernel(unsigned char* k, unsigned char* v, float* weight,
                                                         const int32_t* __restrict__ pages, const int32_t* __restrict__ pages_out,
                                                         const int32_t* __restrict__ lens_out, const int32_t* __restrict__ kept,
                                                         int Hkv, int head_bytes, int log2, int P, int max_pages,
                                                         int max_pages_out, int budget) {
  const int u = blockIdx.y;
  int n = lens_out[u];   // (the selection's; whatever stands there, no more than kept has room for)
  n = n < 0 ? 0 : (n > budget ? budget : n);
  const int pieces = head_bytes >> 4, per_row = pieces * Hkv, mask = (1 << log2) - 1;
  const long long all = (long long)n * per_row;
  for (long long e = (long long)blockIdx.x * 256 + threadIdx.x; e < all; e += (long long)gridDim.x * 256) {
    const int i = (int)(e / per_row), x = (int)(e % per_row), h = x / pieces, piece = x % pieces;
    const int j = kept[(size_t)u * budget + i];
    const int from = pages[(size_t)u * max_pages + (j >> log2)], to = pages_out[(size_t)u * max_pages_out + (i >> log2)];
    if ((unsigned)from >= (unsigned)P || (unsigned)to >= (unsigned)P) continue;
    const size_t src = (((((size_t)from * Hkv + h) << log2) + (j & mask)) * pieces + piece) << 4;
    const size_t dst = (((((size_t)to * Hkv + h) << log2) + (i & mask)) * pieces + piece) << 4;
    *reinterpret_cast<stream16*>(k + dst) = *reinterpret_cast<const stream16*>(k + src);
    *reinterpret_cast<stream16*>(v + dst) = *reinterpret_cast<const stream16*>(v + src);
    if (x == 0) weight[((size_t)to << log2) + (i & mask)] = weight[((size_t)from << log2) + (j & mask)];
  }
}

laser_status cache_evict_launch(const CacheEvictArgs& a) {
  const CacheArgs& c = a.c;
  const int head_bytes = c.D * (c.dt == LASER_F32 ? 4 : 2);
  // (a launch holds fewer than 2^32 threads; rows are moved only once every list of them is under way)
  constexpr int USERS = 1 << 21;
  for (long long u = 0; u < c.U; u += USERS) {
    const int users = c.U - u < USERS ? (int)(c.U - u) : USERS;
    cache_select_kernel<<<users, SEL, 0, c.stream>>>(c.weight, c.pages + u * c.max_pages, c.lens + u, c.L, c.page_log2, c.P, c.max_pages, a.budget,
                                                     a.recent, a.lens_out + u, a.kept + u * a.budget);
    const laser_status s = launch_status();
    if (s != LASER_OK) return s;
  }
  const int rows = a.budget < c.L ? a.budget : c.L;
  const long long most = ((long long)rows * c.Hkv * head_bytes / 16 + 255) / 256;
  for (long long u = 0; u < c.U; u += 65535) {
    const int users = c.U - u < 65535 ? c.U - u : 65535;
    cache_move_kernel<<<dim3((unsigned)(most < 1024 ? most : 1024), users), 256, 0, c.stream>>>(
        static_cast<unsigned char*>(c.k), static_cast<unsigned char*>(c.v), c.weight, c.pages + (size_t)u * c.max_pages,
        a.pages_out + (size_t)u * a.max_pages_out, a.lens_out + u, a.kept + (size_t)u * a.budget, c.Hkv, head_bytes,
        c.page_log2, c.P, c.max_pages, a.max_pages_out, a.budget);
  }
  return launch_status();
}

}  // namespace laser
