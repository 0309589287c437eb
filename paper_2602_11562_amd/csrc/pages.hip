// The pages of a cache. refs[p] counts the tables that hold page p; a page with refs <= 0 is free, and free pages are taken from the
// lowest number up, users in order, so that the same calls give the same tables whatever the order of atomics.
//
// A plan is made by one workgroup that walks the counts (a page's number among the free ones is a sum over all before it), for the
// compaction of more than 4096 pages by one for each 2048, and leaves lists in the work buffer; copies and tables are then written by as many
// workgroups as that takes. Copies go piece by piece of 16 bytes over all parts of all listed pages, whatever a page's size. Bound by latency for small calls (two launches), by memory for large ones.
#include "pages.h"

namespace laser {

constexpr int PLAN = 1024;   // threads of the plan
// A wave looks at `runs` runs of 64 pages at a time, the workgroup at a chunk: many where one workgroup walks until it has enough, few where
// every page has something written and workgroups share them (10248 pages, the plan: one workgroup 9.3 us; runs of 2 in two launches, 5 workgroups, 42.3 us the call instead of 47.0)
constexpr int TAKE_RUNS = 8, COMPACT_RUNS = 2, CHUNK = PLAN * COMPACT_RUNS;

struct Tables {
  const int32_t* pages;
  const int32_t* lens;
  int32_t* refs;
  int U, P, log2, max_pages;
};

__device__ __forceinline__ int held_items(const Tables& t, int u) {   // of user u, within what its table can hold
  const int n = t.lens[u], room = t.max_pages << t.log2;
  return n < 0 ? 0 : n < room ? n : room;
}
__device__ __forceinline__ int pages_of(int n, int log2) { return (int)(((long long)n + (1 << log2) - 1) >> log2); }

// Sum of x over the threads before this one, and over all (every thread calls it)
__device__ __forceinline__ int sum_before(int x, int* all) {
  __shared__ int waves[PLAN / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int sum = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(sum, d);
    if (lane >= d) sum += y;
  }
  __syncthreads();   // (the last call's sums have been read)
  if (lane == 63) waves[wave] = sum;
  __syncthreads();
  int before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < PLAN / 64; ++w) {
    before += w < wave ? waves[w] : 0;
    total += waves[w];
  }
  *all = total;
  return before + sum - x;
}
// The same of a number that each wave has
__device__ __forceinline__ int waves_before(int x, int* all) {
  __shared__ int waves[PLAN / 64];
  const int wave = threadIdx.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) waves[wave] = x;
  __syncthreads();
  int before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < PLAN / 64; ++w) {
    before += w < wave ? waves[w] : 0;
    total += waves[w];
  }
  *all = total;
  return before;
}

// The counts of a wave's pages of a chunk: lane l holds those of pages 64 x + l
template <int RUNS> struct Counts { int c[RUNS]; };
template <int RUNS>
__device__ __forceinline__ Counts<RUNS> counts_of(const int32_t* refs, long long first, int P) {
  Counts<RUNS> x;
#pragma unroll
  for (int r = 0; r < RUNS; ++r) {
    const long long p = first + r * 64 + (threadIdx.x & 63);
    x.c[r] = p < P ? refs[p] : 0;
  }
  return x;
}
__device__ __forceinline__ int lanes_before(unsigned long long mask) { return __popcll(mask & ((1ull << (threadIdx.x & 63)) - 1)); }

template <int RUNS>
__device__ __forceinline__ int used_in(const Counts<RUNS>& x, unsigned long long* used) {
  int sum = 0;
#pragma unroll
  for (int r = 0; r < RUNS; ++r) {
    used[r] = __ballot(x.c[r] > 0);
    sum += __popcll(used[r]);
  }
  return sum;
}
// Pages in use of each chunk
template <int RUNS>
__global__ __launch_bounds__(PLAN) void used_kernel(const int32_t* __restrict__ refs, int P, int32_t* __restrict__ sums) {
  unsigned long long used[RUNS];
  int all;
  waves_before(used_in(counts_of<RUNS>(refs, (long long)blockIdx.x * PLAN * RUNS + (threadIdx.x >> 6) * 64 * RUNS, P), used), &all);
  if (threadIdx.x == 0) sums[blockIdx.x] = all;
}

// The first `want` free pages to fresh[], their counts set to 1; returns how many there were. One workgroup walks the pool by chunks of 8192
// pages; of a large pool (FULL) `used` says which chunks are full, and those are left out: 128 users that grow by a page each, the free
// ones last of 100000 pages 29 us without and 13 with, of 500000 117 and 14, of 10000 9 without. next: the counts of the first chunk, where it is not.
constexpr int TAKE_CHUNK = PLAN * TAKE_RUNS, FULL_POOL = 4 * TAKE_CHUNK;
struct Taken {
  int32_t *refs, *fresh;
  int P, want, got;
};
__device__ __forceinline__ void take_chunk(Taken& t, int p0, const Counts<TAKE_RUNS>& here) {
  const int mine = (int)(threadIdx.x >> 6) * 64 * TAKE_RUNS, lane = threadIdx.x & 63;
  unsigned long long free[TAKE_RUNS];
  int sum = 0;
#pragma unroll
  for (int r = 0; r < TAKE_RUNS; ++r) {
    free[r] = __ballot(here.c[r] <= 0 && (long long)p0 + mine + r * 64 + lane < t.P);
    sum += __popcll(free[r]);
  }
  int all;
  int rank = t.got + waves_before(sum, &all);
#pragma unroll
  for (int r = 0; r < TAKE_RUNS; ++r) {
    const int at = rank + lanes_before(free[r]);
    if ((free[r] >> lane & 1) && at < t.want) {
      const int p = p0 + mine + r * 64 + lane;
      t.fresh[at] = p;
      t.refs[p] = 1;
    }
    rank += __popcll(free[r]);
  }
  t.got += all;
}
template <bool FULL>
__device__ __forceinline__ int take_free(int32_t* refs, int P, int want, int32_t* fresh, Counts<TAKE_RUNS> next, const int32_t* used) {
  const int mine = (int)(threadIdx.x >> 6) * 64 * TAKE_RUNS;
  Taken t{refs, fresh, P, want, 0};
  if constexpr (FULL) {
    __shared__ int list[PLAN];
    const int chunks = (P + TAKE_CHUNK - 1) / TAKE_CHUNK;
    for (int c0 = 0; c0 < chunks && t.got < want; c0 += PLAN) {
      const int c = c0 + (int)threadIdx.x, size = c < chunks ? (P - c * TAKE_CHUNK < TAKE_CHUNK ? P - c * TAKE_CHUNK : TAKE_CHUNK) : 0;
      const bool has = size > 0 && used[c] < size;
      int count;
      const int at = sum_before(has, &count);
      if (has) list[at] = c;
      __syncthreads();
      if (count > 0) next = counts_of<TAKE_RUNS>(refs, (long long)list[0] * TAKE_CHUNK + mine, P);
      for (int k = 0; k < count && t.got < want; ++k) {
        const Counts<TAKE_RUNS> here = next;
        if (k + 1 < count) next = counts_of<TAKE_RUNS>(refs, (long long)list[k + 1] * TAKE_CHUNK + mine, P);
        take_chunk(t, list[k] * TAKE_CHUNK, here);
      }
      __syncthreads();   // (the list has been read)
    }
  } else {
    for (int p0 = 0; p0 < P && t.got < want; p0 += TAKE_CHUNK) {
      const Counts<TAKE_RUNS> here = next;
      next = counts_of<TAKE_RUNS>(refs, (long long)p0 + TAKE_CHUNK + mine, P);   // (asked for ahead of this chunk's sums)
      take_chunk(t, p0, here);
    }
  }
  return t.got < want ? t.got : want;
}

// Fork, the plan: history v of the new tables gets a fresh page where the history it comes from ends within a page. rank[v]: the fresh
// page's number, or -1
__device__ __forceinline__ int forked_items(const Tables& t, const int32_t* source, int v, int max_out) {
  const int u = source[v];
  if ((unsigned)u >= (unsigned)t.U) return 0;
  const int n = held_items(t, u), room = max_out << t.log2;
  return n < room ? n : room;
}
template <bool FULL>
__device__ __forceinline__ void fork_plan(const Tables& t, const int32_t* source, int V, int max_out, int32_t* rank, int32_t* fresh,
                                          int32_t* missing, const int32_t* used) {
  Counts<TAKE_RUNS> first = {};
  if (!FULL) first = counts_of<TAKE_RUNS>(t.refs, (threadIdx.x >> 6) * 64 * TAKE_RUNS, t.P);
  int want = 0;
  for_users(0, PLAN, V, [&](int v0) __attribute__((always_inline)) {
    const unsigned v = v0 + threadIdx.x;
    int need = 0;
    if (v < (unsigned)V) {
      const int n = forked_items(t, source, (int)v, max_out);
      if (n & ((1 << t.log2) - 1)) need = (unsigned)t.pages[(size_t)source[v] * t.max_pages + (n >> t.log2)] < (unsigned)t.P;
    }
    int all;
    const int before = sum_before(need, &all);
    if (v < (unsigned)V) rank[v] = need ? want + before : -1;
    want += all;
  });
  const int got = take_free<FULL>(t.refs, t.P, want, fresh, first, used);
  for_users(threadIdx.x, PLAN, V, [&](int v) __attribute__((always_inline)) {   // (a thread's own ranks)
    if (rank[v] >= got) rank[v] = -2;                                           // no page is left for it
  });
  if (threadIdx.x == 0) *missing = want - got;
}
template <bool FULL>
__global__ __launch_bounds__(PLAN) void fork_plan_kernel(const Tables t, const int32_t* __restrict__ source, int V, int max_out,
                                                         int32_t* rank, int32_t* fresh, int32_t* missing, const int32_t* __restrict__ used) {
  fork_plan<FULL>(t, source, V, max_out, rank, fresh, missing, used);
}

// Pieces of listed pages from src[] to dst[], every part of them
template <int N>
struct Moves {
  static constexpr int PARTS = N;
  PageParts<N> parts;
  const int32_t* count;      // entries, where the host does not know
  MulDiv by_all;             // / parts.all
};
template <typename T>
__device__ __forceinline__ void move_piece(unsigned char* base, unsigned page_bytes, int src, int dst, unsigned piece) {
  const long long bytes = page_bytes;
  reinterpret_cast<T*>(base + dst * bytes)[piece] = reinterpret_cast<const T*>(base + src * bytes)[piece];
}
// entry(e, &src, &dst): false where the entry moves nothing
template <int THREADS = 256, int N, typename Entry>
__device__ __forceinline__ void move_pages(const Moves<N>& m, long long entries, unsigned block, unsigned blocks, const Entry& entry) {
  const PageParts<N>& parts = m.parts;
  const long long all = entries * parts.all;
  for (long long g = (long long)block * THREADS + threadIdx.x; g < all; g += (long long)blocks * THREADS) {
    const long long e = all <= 0x7fffffffLL ? (long long)m.by_all.div((unsigned)g) : g / parts.all;
    unsigned piece = (unsigned)(g - e * parts.all);
    int src, dst, i = 0;
    if (!entry(e, &src, &dst)) continue;
    for (unsigned here; piece >= (here = parts.bytes[i] >> parts.piece_log2[i]); ++i) piece -= here;
    if (parts.piece_log2[i] == 4) move_piece<stream16>(parts.at[i], parts.bytes[i], src, dst, piece);
    else if (parts.piece_log2[i] == 2) move_piece<unsigned>(parts.at[i], parts.bytes[i], src, dst, piece);
    else move_piece<unsigned char>(parts.at[i], parts.bytes[i], src, dst, piece);
  }
}

// Fork, the rest: where a page that is copied comes from and goes to, and entry j of table v
struct Fork {
  const int32_t *source, *rank, *fresh;
  int32_t *pages_out, *lens_out;
  int V, max_out;
};
__device__ __forceinline__ bool forked_page(const Tables& t, const Fork& f, int v, int* src, int* dst) {
  const int r = f.rank[v];
  if (r < 0) return false;
  const int n = forked_items(t, f.source, v, f.max_out);
  *src = t.pages[(size_t)f.source[v] * t.max_pages + (n >> t.log2)];
  *dst = f.fresh[r];
  return true;
}
__device__ __forceinline__ void forked_entry(const Tables& t, const Fork& f, int v, int j, int n) {
  int p = -1;
  if (j < pages_of(n, t.log2)) {
    p = t.pages[(size_t)f.source[v] * t.max_pages + j];
    if (j >= n >> t.log2) {
      if ((unsigned)p < (unsigned)t.P) p = f.rank[v] >= 0 ? f.fresh[f.rank[v]] : -1;
    } else if ((unsigned)p < (unsigned)t.P) {
      atomicAdd(t.refs + p, 1);
    }
  }
  f.pages_out[(size_t)v * f.max_out + j] = p;
  if (j == 0) f.lens_out[v] = n;
}
// The first `copies` workgroups copy pages, the others write a table each
template <int N>
__global__ __launch_bounds__(256) void fork_kernel(const Tables t, const Fork f, unsigned copies, bool tables, const Moves<N> m) {
  if (blockIdx.x < copies) {
    move_pages(m, f.V, blockIdx.x, copies, [&](long long v, int* src, int* dst) __attribute__((always_inline)) { return forked_page(t, f, (int)v, src, dst); });
    return;
  }
  if (!tables) return;
  for_users(blockIdx.x - copies, gridDim.x - copies, f.V, [&](int v) __attribute__((always_inline)) {
    const int n = forked_items(t, f.source, v, f.max_out);
    for (int j = threadIdx.x; j < f.max_out; j += 256) forked_entry(t, f, v, j, n);
  });
}
// A small fork, plan and rest in one launch
__global__ __launch_bounds__(PLAN) void fork_small_kernel(const Tables t, const Fork f, int32_t* rank, int32_t* fresh, int32_t* missing,
                                                          MulDiv by_out, const Moves<FEW_PARTS> m) {
  fork_plan<false>(t, f.source, f.V, f.max_out, rank, fresh, missing, nullptr);
  __syncthreads();   // ranks, fresh pages and their counts are written
  move_pages<PLAN>(m, f.V, 0, 1, [&](long long v, int* src, int* dst) __attribute__((always_inline)) { return forked_page(t, f, (int)v, src, dst); });
  for (int x = threadIdx.x; x < f.V * f.max_out; x += PLAN) {
    const int v = (int)by_out.div((unsigned)x);
    forked_entry(t, f, v, x - v * f.max_out, forked_items(t, f.source, v, f.max_out));
  }
}

constexpr int OWN_ENTRIES = 16;
// Grow: user u's table gets the pages that its next c items ask for
template <bool FULL>
__global__ __launch_bounds__(PLAN) void grow_kernel(const Tables t, const int32_t* __restrict__ off, int32_t* pages, int32_t* lens,
                                                    int32_t* __restrict__ rank, int32_t* __restrict__ fresh, int32_t* __restrict__ missing,
                                                    const int32_t* __restrict__ used) {
  auto grown = [&](int u, int n) {
    const long long c = (long long)off[u + 1] - off[u], room = (long long)t.max_pages << t.log2, m = n + (c > 0 ? c : 0);
    return (int)(m < room ? m : room);
  };
  Counts<TAKE_RUNS> ahead = {};
  if (!FULL) ahead = counts_of<TAKE_RUNS>(t.refs, (threadIdx.x >> 6) * 64 * TAKE_RUNS, t.P);
  int want = 0;
  for_users(0, PLAN, t.U, [&](int u0) __attribute__((always_inline)) {
    const unsigned u = u0 + threadIdx.x;
    int need = 0;
    if (u < (unsigned)t.U) {
      const int n = held_items(t, (int)u);
      need = pages_of(grown((int)u, n), t.log2) - pages_of(n, t.log2);
    }
    int all;
    const int before = sum_before(need, &all);
    if (u < (unsigned)t.U) rank[u] = want + before;
    want += all;
  });
  const int got = take_free<FULL>(t.refs, t.P, want, fresh, ahead, used);
  __syncthreads();
  // A user's first entries by a thread, the others by its wave, where few users are dealt to all waves (65000 items of one user in pages of
  // 8: 822 us by the thread alone and 27 so, 16 users' 5000 in pages of 16 49 and 14, 128 users' 1000 23 and 16).
  const bool deal = t.U <= PLAN / 4;
  for_users(0, PLAN, t.U, [&](int u0) __attribute__((always_inline)) {
    const unsigned lane = threadIdx.x & 63, at = u0 + (deal ? lane * (PLAN / 64) + (threadIdx.x >> 6) : threadIdx.x);
    const int u = (int)at;
    int first = 0, last = 0, r = 0;
    if (at < (unsigned)t.U) {
      const int n = held_items(t, u), m = grown(u, n);
      first = pages_of(n, t.log2), last = pages_of(m, t.log2), r = rank[u] - first;
      lens[u] = m;
    }
    auto entry = [&](int u, int r, int j) { pages[(size_t)u * t.max_pages + j] = r + j < got ? fresh[r + j] : -1; };
    for (int j = first; j < last && j < first + OWN_ENTRIES; ++j) entry(u, r, j);
    for (unsigned long long more = __ballot(last - first > OWN_ENTRIES); more != 0; more &= more - 1) {
      const int l = __builtin_ctzll(more), end = __builtin_amdgcn_readlane(last, l), their_u = __builtin_amdgcn_readlane(u, l),
                their_r = __builtin_amdgcn_readlane(r, l);
      for (int j = __builtin_amdgcn_readlane(first, l) + OWN_ENTRIES + lane; j < end; j += 64) entry(their_u, their_r, j);
    }
  });
  if (threadIdx.x == 0) *missing = want - got;
}

// Free: a workgroup gives back the pages of a user
__global__ __launch_bounds__(256) void free_kernel(const Tables t, const int32_t* __restrict__ gone, int32_t* lens) {
  for_users(blockIdx.x, gridDim.x, t.U, [&](int u) __attribute__((always_inline)) {
    if (gone != nullptr && gone[u] == 0) return;
    const int used = pages_of(held_items(t, u), t.log2);
    for (int j = threadIdx.x; j < used; j += 256) {
      const int p = t.pages[(size_t)u * t.max_pages + j];
      // (never below 0, should a page be given back more often than it is held)
      if ((unsigned)p < (unsigned)t.P && atomicSub(t.refs + p, 1) <= 0) atomicAdd(t.refs + p, 1);
    }
    __syncthreads();   // (every wave has the length)
    if (threadIdx.x == 0) lens[u] = 0;
  });
}

// Compact, the plan: of M pages in use, those numbered M and more go to the free ones below M, in order. With `sums`, pages in use of each
// chunk, a workgroup a chunk; otherwise one workgroup for all of them, a few.
constexpr int CHUNKS_AT_ONCE = 2, WAVE_PAGES = 64 * COMPACT_RUNS;
struct CompactPlan {
  int32_t *src, *dst, *place, *moved, *in_use;
};
// A wave's pages of a chunk that begins with page p0; before: pages in use ahead of the wave's, below: those below M
__device__ __forceinline__ void plan_wave(const CompactPlan& o, const unsigned long long* used, int p0, int P, int M, int before, int below) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int r = 0; r < COMPACT_RUNS; ++r) {
    const int p = p0 + (int)(threadIdx.x >> 6) * WAVE_PAGES + r * 64 + lane, rank = before + lanes_before(used[r]);
    if (p < P) {
      if (used[r] >> lane & 1) {
        if (p >= M) o.src[rank - below] = p;
        o.place[p] = p >= M ? below - rank - 1 : p;   // (below 0: where the list says, which may not be whole yet)
      } else {
        if (p < M) o.dst[p - rank] = p;
        o.place[p] = p;
      }
    }
    before += __popcll(used[r]);
  }
}
__global__ __launch_bounds__(PLAN) void compact_plan_kernel(const int32_t* __restrict__ refs, int P, const CompactPlan o) {
  unsigned long long used[CHUNKS_AT_ONCE][COMPACT_RUNS];
  int before[CHUNKS_AT_ONCE], M = 0;
  const int wave = (int)(threadIdx.x >> 6);
  Counts<COMPACT_RUNS> x[CHUNKS_AT_ONCE];
#pragma unroll
  for (int c = 0; c < CHUNKS_AT_ONCE; ++c) x[c] = counts_of<COMPACT_RUNS>(refs, (long long)c * CHUNK + wave * WAVE_PAGES, P);
#pragma unroll
  for (int c = 0; c < CHUNKS_AT_ONCE; ++c) {
    int all;
    before[c] = M + waves_before(used_in(x[c], used[c]), &all);
    M += all;
  }
  int below = 0;   // pages in use below M
#pragma unroll
  for (int c = 0; c < CHUNKS_AT_ONCE; ++c)
#pragma unroll
    for (int r = 0; r < COMPACT_RUNS; ++r) {
      const int left = M - (c * CHUNK + wave * WAVE_PAGES + r * 64);
      below += left >= 64 ? __popcll(used[c][r]) : left > 0 ? __popcll(used[c][r] & ((1ull << left) - 1)) : 0;
    }
  int all;
  waves_before(below, &all);
  below = all;
#pragma unroll
  for (int c = 0; c < CHUNKS_AT_ONCE; ++c) plan_wave(o, used[c], c * CHUNK, P, M, before[c], below);
  if (threadIdx.x == 0) {
    *o.moved = M - below;
    *o.in_use = M;
  }
}
// ALONE: without sums, every workgroup counts all pages, where they are few (the call without contents, captured, us by sums of a launch ahead
// and alone: 4097 pages 8.7 and 7.8, 10248 9.5 and 9.0, 16384 9.3 and 8.5, 32768 9.3 and 9.7, 131072 11.2 and 18.8)
constexpr int CHUNKS_ALONE = 8;
template <bool ALONE>
__global__ __launch_bounds__(PLAN) void compact_chunk_kernel(const int32_t* __restrict__ refs, int P, const int32_t* __restrict__ sums,
                                                             int chunks, const CompactPlan o) {
  const int chunk = blockIdx.x, wave = (int)(threadIdx.x >> 6);
  const Counts<COMPACT_RUNS> x = counts_of<COMPACT_RUNS>(refs, (long long)chunk * CHUNK + wave * WAVE_PAGES, P);
  int total = 0, ahead = 0, M, before;
  if constexpr (ALONE) {
#pragma unroll 8
    for (int p = threadIdx.x; p < P; p += PLAN) {
      const int y = refs[p] > 0;
      total += y;
      ahead += p < chunk * CHUNK ? y : 0;
    }
  } else {
    for (int c = threadIdx.x; c < chunks; c += PLAN) {
      const int y = sums[c];
      total += y;
      ahead += c < chunk ? y : 0;
    }
  }
  sum_before(total, &M);
  sum_before(ahead, &before);
  // pages in use below M: of whole chunks, and of the one that M is in
  const int last = ALONE ? 0 : M / CHUNK;
  int below = 0, all;
  if constexpr (!ALONE)
    for (int c = threadIdx.x; c < last; c += PLAN) below += sums[c];
#pragma unroll 8
  for (int p = last * CHUNK + threadIdx.x; p < M; p += PLAN) below += refs[p] > 0;
  sum_before(below, &all);
  below = all;
  unsigned long long used[COMPACT_RUNS];
  before += waves_before(used_in(x, used), &all);
  plan_wave(o, used, chunk * CHUNK, P, M, before, below);
  if (chunk == 0 && threadIdx.x == 0) {
    *o.moved = M - below;
    *o.in_use = M;
  }
}
// Where page p goes
__device__ __forceinline__ int place_of_page(const int32_t* place, const int32_t* dst, int p) {
  const int x = place[p];
  return x < 0 ? dst[-1 - x] : x;
}

// Compact, the rest: the first `copies` workgroups copy pages, the others write tables and counts
template <int N>
__global__ __launch_bounds__(256) void compact_kernel(const Tables t, const int32_t* __restrict__ src, const int32_t* __restrict__ dst,
                                                      const int32_t* __restrict__ place, int32_t* __restrict__ pages_out,
                                                      int32_t* __restrict__ refs_out, const int32_t* __restrict__ in_use,
                                                      unsigned copies, bool tables, const Moves<N> m) {
  if (blockIdx.x < copies) {
    move_pages(m, *m.count, blockIdx.x, copies, [&](long long i, int* from, int* to) __attribute__((always_inline)) {
      *from = src[i];
      *to = dst[i];
      return true;
    });
    return;
  }
  if (!tables) return;
  const unsigned first = blockIdx.x - copies, step = gridDim.x - copies;
  for_users(first, step, t.U, [&](int u) __attribute__((always_inline)) {
    const int used = pages_of(held_items(t, u), t.log2);
    for (int j = threadIdx.x; j < t.max_pages; j += 256) {
      int p = -1;
      if (j < used) {
        p = t.pages[(size_t)u * t.max_pages + j];
        if ((unsigned)p < (unsigned)t.P) p = place_of_page(place, dst, p);
      }
      pages_out[(size_t)u * t.max_pages + j] = p;
    }
  });
  // a page in use has its count where it goes to; what lies behind the last of them is free
  const int M = *in_use;
  for (long long p = (long long)first * 256 + threadIdx.x; p < t.P; p += (long long)step * 256) {
    const int count = t.refs[p];
    if (count > 0) refs_out[place_of_page(place, dst, (int)p)] = count;
    if (p >= M) refs_out[p] = 0;
  }
}

template <int N>
__global__ __launch_bounds__(256) void copy_kernel(const int32_t* __restrict__ src, const int32_t* __restrict__ dst, int n, int P,
                                                   const Moves<N> m) {
  move_pages(m, n, blockIdx.x, gridDim.x, [&](long long i, int* from, int* to) __attribute__((always_inline)) {
    *from = src[i];
    *to = dst[i];
    return (unsigned)*from < (unsigned)P && (unsigned)*to < (unsigned)P;
  });
}

// ---------------------------------------------------------------- launchers
size_t pages_work_ints(int U, int P) { return (size_t)U + 3 * (size_t)P + (P + CHUNK - 1) / CHUNK + 16; }

static Tables tables_of(const PagesArgs& a) { return Tables{a.pages, a.lens, a.refs, a.U, a.P, a.page_log2, a.max_pages}; }

// The parts from `first` on that one launch moves, with their pieces
template <int N>
static Moves<N> moves_of(const PagesArgs& a, int first, const int32_t* count) {
  Moves<N> m{};
  PageParts<N>& p = m.parts;
  for (int i = first; i < a.n_parts && p.n < N; ++i, ++p.n) {
    const unsigned long long x = reinterpret_cast<unsigned long long>(a.parts[i]) | (unsigned long long)a.part_bytes[i];
    p.at[p.n] = static_cast<unsigned char*>(a.parts[i]);
    p.bytes[p.n] = (unsigned)a.part_bytes[i];
    p.piece_log2[p.n] = x % 16 == 0 ? 4 : x % 4 == 0 ? 2 : 0;
    p.all += p.bytes[p.n] >> p.piece_log2[p.n];
  }
  m.count = count;
  m.by_all = mul_div(p.all > 0 ? p.all : 1);
  return m;
}
// go(moves, workgroups that copy, first): a launch for every N parts
template <int N, typename Go>
static laser_status over_parts_by(const PagesArgs& a, long long entries, const int32_t* count, Go&& go) {
  for (int i = 0; i == 0 || i < a.n_parts; i += N) {
    const Moves<N> m = moves_of<N>(a, i, count);
    const long long groups = (entries * m.parts.all + 255) / 256;
    go(m, (unsigned)(groups < 16384 ? groups : 16384), i == 0);
    const laser_status s = launch_status();
    if (s != LASER_OK) return s;
  }
  return LASER_OK;
}
template <typename Go>
static laser_status over_parts(const PagesArgs& a, long long entries, const int32_t* count, Go&& go) {
  return a.n_parts <= FEW_PARTS ? over_parts_by<FEW_PARTS>(a, entries, count, go) : over_parts_by<PARTS_A_LAUNCH>(a, entries, count, go);
}

// Of a large pool, pages in use of each chunk that pages are taken from
static laser_status full_chunks(const PagesArgs& a, int32_t* sums, const int32_t** used) {
  *used = nullptr;
  if (a.P <= FULL_POOL) return LASER_OK;
  used_kernel<TAKE_RUNS><<<(a.P + TAKE_CHUNK - 1) / TAKE_CHUNK, PLAN, 0, a.stream>>>(a.refs, a.P, sums);
  *used = sums;
  return launch_status();
}

// Of so many pieces and entries a fork is one workgroup's, plan and all: the GPU takes as long (three histories of 63 pages, two parts of
// 4096 bytes: 9.3 us by two launches and 9.5 by one, with the release of the forks), the host less (a fork, a growth and a release: 17.1 and 15.7)
constexpr int SMALL_FORK = 2 * PLAN;
laser_status pages_fork_launch(const PagesArgs& a) {
  int32_t *rank = a.work, *fresh = a.work + a.V;
  const Tables t = tables_of(a);
  const Fork f{a.source, rank, fresh, a.pages_out, a.lens_out, a.V, a.max_out};
  if (a.P <= FULL_POOL && a.n_parts <= FEW_PARTS && (long long)a.V * a.max_out <= SMALL_FORK) {
    const Moves<FEW_PARTS> m = moves_of<FEW_PARTS>(a, 0, nullptr);
    if ((long long)a.V * m.parts.all <= SMALL_FORK) {
      fork_small_kernel<<<1, PLAN, 0, a.stream>>>(t, f, rank, fresh, a.missing, mul_div(a.max_out), m);
      return launch_status();
    }
  }
  laser_status s;
  const int32_t* used;
  if ((s = full_chunks(a, fresh + a.P, &used)) != LASER_OK) return s;
  if (used != nullptr) fork_plan_kernel<true><<<1, PLAN, 0, a.stream>>>(t, a.source, a.V, a.max_out, rank, fresh, a.missing, used);
  else fork_plan_kernel<false><<<1, PLAN, 0, a.stream>>>(t, a.source, a.V, a.max_out, rank, fresh, a.missing, nullptr);
  if ((s = launch_status()) != LASER_OK) return s;
  return over_parts(a, a.V, nullptr, [&](const auto& m, unsigned copies, bool first) {
    const unsigned more = first ? (a.V < 4096 ? a.V : 4096) : 0;
    if (copies + more > 0) fork_kernel<<<copies + more, 256, 0, a.stream>>>(t, f, copies, first, m);
  });
}

laser_status pages_grow_launch(const PagesArgs& a) {
  const Tables t = tables_of(a);
  int32_t *rank = a.work, *fresh = a.work + a.U, *pages = const_cast<int32_t*>(a.pages);
  const int32_t* used;
  const laser_status s = full_chunks(a, fresh + a.P, &used);
  if (s != LASER_OK) return s;
  if (used != nullptr) grow_kernel<true><<<1, PLAN, 0, a.stream>>>(t, a.off, pages, a.lens_out, rank, fresh, a.missing, used);
  else grow_kernel<false><<<1, PLAN, 0, a.stream>>>(t, a.off, pages, a.lens_out, rank, fresh, a.missing, nullptr);
  return launch_status();
}

laser_status pages_free_launch(const PagesArgs& a) {
  free_kernel<<<a.U < 65536 ? a.U : 65536, 256, 0, a.stream>>>(tables_of(a), a.gone, a.lens_out);
  return launch_status();
}

laser_status pages_compact_launch(const PagesArgs& a) {
  int32_t *src = a.work, *dst = src + a.P, *place = dst + a.P, *moved = place + a.P, *sums = moved + 1;
  const CompactPlan o{src, dst, place, moved, a.in_use};
  const Tables t = tables_of(a);
  const int chunks = (a.P + CHUNK - 1) / CHUNK;
  laser_status s;
  if (chunks <= CHUNKS_AT_ONCE) {
    compact_plan_kernel<<<1, PLAN, 0, a.stream>>>(a.refs, a.P, o);
  } else if (chunks <= CHUNKS_ALONE) {
    compact_chunk_kernel<true><<<chunks, PLAN, 0, a.stream>>>(a.refs, a.P, nullptr, chunks, o);
  } else {
    used_kernel<COMPACT_RUNS><<<chunks, PLAN, 0, a.stream>>>(a.refs, a.P, sums);
    if ((s = launch_status()) != LASER_OK) return s;
    compact_chunk_kernel<false><<<chunks, PLAN, 0, a.stream>>>(a.refs, a.P, sums, chunks, o);
  }
  if ((s = launch_status()) != LASER_OK) return s;
  return over_parts(a, a.P / 2, moved, [&](const auto& m, unsigned copies, bool first) {
    const unsigned more = first ? 1024 : 0;
    if (copies + more > 0)
      compact_kernel<<<copies + more, 256, 0, a.stream>>>(t, src, dst, place, a.pages_out, a.refs_out, a.in_use, copies, first, m);
  });
}

laser_status pages_copy_launch(const PagesArgs& a, const int32_t* src, const int32_t* dst, int n) {
  return over_parts(a, n, nullptr, [&](const auto& m, unsigned copies, bool) {
    if (copies > 0) copy_kernel<<<copies, 256, 0, a.stream>>>(src, dst, n, a.P, m);
  });
}

}  // namespace laser
