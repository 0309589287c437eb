// Attention among the items of histories: arguments after validation, the launchers, and how the kernels find their rows.
#pragma once

#include "laser_internal.h"

namespace laser {

// Packed sequences: sequence n owns rows off[n] .. off[n+1]-1 of q, k, v (at most L of them, T rows in all).
struct HistoryArgs {
  const void* q;
  const void* k;
  const void* v;
  long long qp, kp, vp;    // elements from one token's row to the next
  const int32_t* off;
  int N, T, L, H, Hkv, D;
  float gamma;
  laser_dtype dt;
  void* o;                 // [T,H,D]
  float* lse;              // [T,H], may be nullptr
  hipStream_t stream;
};
laser_status history_forward_launch(const HistoryArgs& a);
laser_status history_tile_launch(const HistoryArgs& a);   // bf16
laser_status history_f32_launch(const HistoryArgs& a);

struct HistoryBwdArgs {
  HistoryArgs f;           // the forward pass's arguments; o and lse are inputs here
  const void* go;          // d loss / d o [T,H,D]
  void* dq;
  void* dk;
  void* dv;
  long long dqp, dkp, dvp;
  float* work;             // history_backward_work_bytes() bytes
};
size_t history_backward_work_bytes(int N, int T, int L, int H, int Hkv, int D, laser_dtype dt);
laser_status history_backward_launch(const HistoryBwdArgs& a);
laser_status history_bwd_tile_launch(const HistoryBwdArgs& a);   // bf16
laser_status history_bwd_f32_launch(const HistoryBwdArgs& a);

// A paged cache: item j of user u stands in page pages[u * max_pages + j / page], at place j % page of every key-value head.
struct CacheArgs {
  const void* q;           // [T,H,D], rows off[u] .. off[u+1]-1 are user u's (at most C of them)
  long long qp;
  void* k;                 // [P,Hkv,page,D]
  void* v;
  const int32_t* off;
  const int32_t* pages;    // [U,max_pages]
  const int32_t* lens;     // [U]
  int U, T, C, L, H, Hkv, D, page_log2, P, max_pages;
  float gamma;
  bool causal;
  laser_dtype dt;
  void* o;                 // [T,H,D]
  float* lse;              // [T,H]
  hipStream_t stream;
  float* work;             // cache_attention_work_bytes() bytes
  float* weight;           // [P,page]
  bool add;
};
size_t cache_attention_work_bytes(int U, int T, int C, int L, int H, int Hkv, int D, laser_dtype dt);
laser_status cache_attention_launch(const CacheArgs& a);
struct CacheRuns { int chunk, runs; };   // histories of up to L items are cut into runs of `chunk`
CacheRuns cache_runs(long long workgroups, int L, int want, int least, int tile);
laser_status cache_join_launch(const CacheArgs& a, int chunk, int splits);
laser_status cache_few_launch(const CacheArgs& a, const CacheRuns& r);    // bf16, at most 32 rows a key-value head
laser_status cache_tile_launch(const CacheArgs& a, const CacheRuns& r);   // bf16
laser_status cache_f32_launch(const CacheArgs& a, const CacheRuns& r);
laser_status cache_weights_tile_launch(const CacheArgs& a);               // bf16
laser_status cache_weights_f32_launch(const CacheArgs& a);
laser_status cache_weights_launch(const CacheArgs& a);   // q, lse and k in, weight out

struct CacheAppendArgs {
  const void* k;           // [T,Hkv,D]
  const void* v;
  long long kp, vp;
  CacheArgs c;
};
laser_status cache_append_launch(const CacheAppendArgs& a);

struct CacheEvictArgs {
  CacheArgs c;             // k, v, weight, pages, lens and the sizes
  const int32_t* pages_out;   // [U,max_pages_out]
  int max_pages_out, budget, recent;
  int32_t* lens_out;       // [U]
  int32_t* kept;           // [U,budget]
};
laser_status cache_evict_launch(const CacheEvictArgs& a);

// ---------------------------------------------------------------- device helpers
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// Items of user u in the cache: what lens says, within L and what the page table can hold
__device__ __forceinline__ int cache_len(const int32_t* lens, int u, int L, int max_pages, int page_log2) {
  const long long room = (long long)max_pages << page_log2;
  return valid_len(lens, u, room < L ? (int)room : L);
}

}  // namespace laser
