// Attention among the items of histories, the plain kernels: a wave per row, any shape and either storage type.
#include "history.h"

namespace laser {

// How a kernel finds item j of its sequence or user, for one key-value head. row() is only asked for items that ok() accepts.
template <typename T>
struct PackedRows {
  const T* k;
  const T* v;
  long long kp, vp;
  __device__ __forceinline__ bool ok(int) const { return true; }
  __device__ __forceinline__ const T* krow(int j) const { return k + j * kp; }
  __device__ __forceinline__ const T* vrow(int j) const { return v + j * vp; }
};
template <typename T>
struct PagedRows {
  const T* k;
  const T* v;
  const int32_t* pages;   // the user's
  int P, Hkv, head, D, log2;
  __device__ __forceinline__ bool ok(int j) const { return (unsigned)pages[j >> log2] < (unsigned)P; }
  __device__ __forceinline__ size_t at(int j) const {
    return ((((size_t)pages[j >> log2] * Hkv + head) << log2) + (j & ((1 << log2) - 1))) * D;
  }
  __device__ __forceinline__ const T* krow(int j) const { return k + at(j); }
  __device__ __forceinline__ const T* vrow(int j) const { return v + at(j); }
};

__device__ __forceinline__ float wave_max64(float x) {
  for (int m = 32; m; m >>= 1) x = fmaxf(x, __shfl_xor(x, m));
  return x;
}
__device__ __forceinline__ float wave_sum64(float x) {
  for (int m = 32; m; m >>= 1) x += __shfl_xor(x, m);
  return x;
}
template <typename T>
__device__ __forceinline__ float dot_row(const float* a, const T* b, int D) {
  float s = 0.0f;
  for (int d = 0; d < D; ++d) s = fmaf(a[d], load_as_f32<T>(b, d), s);
  return s;
}

// One query row against items 0 .. n-1: lane = item for the scores, lane = column for the sum of values
template <typename T, typename Rows>
__device__ __forceinline__ void attend_row(const float* q, const Rows& rows, int n, int D, float scale, T* o, float* lse) {
  const int lane = threadIdx.x & 63;
  float m = -INFINITY, l = 0.0f, a0 = 0.0f, a1 = 0.0f;
  for (int t = 0; t < n; t += 64) {
    const int j = t + lane;
    const bool in = j < n && rows.ok(j);
    const float s = in ? dot_row<T>(q, rows.krow(j), D) * scale : -INFINITY;
    const float mt = fmaxf(m, wave_max64(s));
    if (mt == -INFINITY) continue;
    const float p = in ? exp2f(s - mt) : 0.0f, c = exp2f(m - mt);
    m = mt;
    l = l * c + wave_sum64(p);
    a0 *= c;
    a1 *= c;
    for (int i = 0; i < 64; ++i) {
      const float pi = __shfl(p, i);
      if (t + i >= n || !rows.ok(t + i)) continue;
      const T* v = rows.vrow(t + i);
      if (lane < D) a0 = fmaf(pi, load_as_f32<T>(v, lane), a0);
      if (lane + 64 < D) a1 = fmaf(pi, load_as_f32<T>(v, lane + 64), a1);
    }
  }
  const float r = l == 0.0f ? 0.0f : 1.0f / l;
  if (lane < D) store_from_f32<T>(o, lane, a0 * r);
  if (lane + 64 < D) store_from_f32<T>(o, lane + 64, a1 * r);
  if (lse != nullptr && lane == 0) *lse = l == 0.0f ? -INFINITY : (m + log2f(l)) * LN2;
}

template <typename T>
__global__ __launch_bounds__(64) void history_forward_generic(const T* q, const T* k, const T* v, long long qp, long long kp,
                                                              long long vp, const int32_t* off, int T_all, int L, int H,
                                                              int Hkv, int D, float scale, T* o, float* lse) {
  __shared__ float qs[128];
  const int h = blockIdx.y, n = blockIdx.z;
  const CandRange r = cand_range(off, n, L, T_all);
  for (int i = blockIdx.x; i < r.count; i += gridDim.x) {
    const size_t tok = (size_t)r.first + i;
    __syncthreads();
    for (int d = threadIdx.x; d < D; d += 64) qs[d] = load_as_f32<T>(q + tok * qp + (size_t)h * D, d);
    __syncthreads();
    const int hk = h / (H / Hkv);
    const PackedRows<T> rows{k + r.first * kp + (size_t)hk * D, v + r.first * vp + (size_t)hk * D, kp, vp};
    attend_row<T>(qs, rows, i + 1, D, scale, o + (tok * H + h) * D, lse ? lse + tok * H + h : nullptr);
  }
}

template <typename T>
__global__ __launch_bounds__(64) void cache_attention_generic(const T* q, long long qp, const T* k, const T* v,
                                                              const int32_t* off, const int32_t* pages, const int32_t* lens,
                                                              int T_all, int C, int L, int H, int Hkv, int D, int log2, int P,
                                                              int max_pages, float scale, bool causal, T* o, float* lse) {
  __shared__ float qs[128];
  const int h = blockIdx.y, u = blockIdx.z;
  const CandRange r = cand_range(off, u, C, T_all);
  const int n = cache_len(lens, u, L, max_pages, log2);
  for (int i = blockIdx.x; i < r.count; i += gridDim.x) {
    const size_t tok = (size_t)r.first + i;
    __syncthreads();
    for (int d = threadIdx.x; d < D; d += 64) qs[d] = load_as_f32<T>(q + tok * qp + (size_t)h * D, d);
    __syncthreads();
    const PagedRows<T> rows{k, v, pages + (size_t)u * max_pages, P, Hkv, h / (H / Hkv), D, log2};
    attend_row<T>(qs, rows, causal ? n - r.count + i + 1 : n, D, scale, o + (tok * H + h) * D, lse ? lse + tok * H + h : nullptr);
  }
}

// What the items of a user's cache receive: a wave per item, lane = row
template <typename T>
__global__ __launch_bounds__(64) void cache_weights_generic(const T* q, long long qp, const T* k, const float* lse,
                                                            const int32_t* off, const int32_t* pages, const int32_t* lens,
                                                            int T_all, int C, int L, int H, int Hkv, int D, int log2, int P,
                                                            int max_pages, float scale, bool causal, float* weight, bool add) {
  __shared__ float ks[128];
  const int u = blockIdx.y, lane = threadIdx.x;
  const CandRange r = cand_range(off, u, C, T_all);
  const int n = cache_len(lens, u, L, max_pages, log2), G = H / Hkv;
  for (int j = blockIdx.x; j < n; j += gridDim.x) {
    float sum = 0.0f;
    const PagedRows<T> rows{k, k, pages + (size_t)u * max_pages, P, Hkv, 0, D, log2};
    if (!rows.ok(j)) continue;
    for (int hk = 0; hk < Hkv; ++hk) {
      __syncthreads();
      PagedRows<T> mine = rows;
      mine.head = hk;
      for (int d = lane; d < D; d += 64) ks[d] = load_as_f32<T>(mine.krow(j), d);
      __syncthreads();
      for (int x = lane; x < r.count * G; x += 64) {
        const int i = x / G, h = hk * G + x % G;
        if (causal && j > n - r.count + i) continue;
        const size_t tok = (size_t)r.first + i;
        const float z = lse[tok * H + h];
        if (z == -INFINITY) continue;
        sum += exp2f(dot_row<T>(ks, q + tok * qp + (size_t)h * D, D) * scale - z * LOG2E);
      }
    }
    sum = wave_sum64(sum);
    float* w = weight + ((size_t)pages[(size_t)u * max_pages + (j >> log2)] << log2) + (j & ((1 << log2) - 1));
    if (lane == 0) {
      if (add) atomicAdd(w, sum);
      else *w = sum;
    }
  }
}

// Gradients of the queries: a wave per row
template <typename T>
__global__ __launch_bounds__(64) void history_dq_generic(const T* q, const T* k, const T* v, long long qp, long long kp,
                                                         long long vp, const int32_t* off, int T_all, int L, int H, int Hkv,
                                                         int D, float inv_gamma, const T* o, const float* lse, const T* go,
                                                         T* dq, long long dqp, float* delta) {
  __shared__ float qs[128], gs[128];
  const int h = blockIdx.y, n = blockIdx.z, lane = threadIdx.x, hk = h / (H / Hkv);
  const CandRange r = cand_range(off, n, L, T_all);
  for (int i = blockIdx.x; i < r.count; i += gridDim.x) {
    const size_t tok = (size_t)r.first + i, row = (tok * H + h) * D;
    __syncthreads();
    float dl = 0.0f;
    for (int d = lane; d < D; d += 64) {
      qs[d] = load_as_f32<T>(q + tok * qp + (size_t)h * D, d);
      gs[d] = load_as_f32<T>(go + row, d);
      dl += gs[d] * load_as_f32<T>(o + row, d);
    }
    __syncthreads();
    dl = wave_sum64(dl);
    if (lane == 0) delta[tok * H + h] = dl;
    const float z = lse[tok * H + h] * LOG2E;
    float a0 = 0.0f, a1 = 0.0f;
    for (int t = 0; t <= i; t += 64) {
      const int j = t + lane;
      float ds = 0.0f;
      if (j <= i) {
        const float s = dot_row<T>(qs, k + (r.first + (size_t)j) * kp + (size_t)hk * D, D) * inv_gamma * LOG2E;
        ds = exp2f(s - z) * (dot_row<T>(gs, v + (r.first + (size_t)j) * vp + (size_t)hk * D, D) - dl) * inv_gamma;
      }
      for (int x = 0; x < 64 && t + x <= i; ++x) {
        const float dx = __shfl(ds, x);
        const T* kr = k + (r.first + (size_t)(t + x)) * kp + (size_t)hk * D;
        if (lane < D) a0 = fmaf(dx, load_as_f32<T>(kr, lane), a0);
        if (lane + 64 < D) a1 = fmaf(dx, load_as_f32<T>(kr, lane + 64), a1);
      }
    }
    if (lane < D) store_from_f32<T>(dq + tok * dqp + (size_t)h * D, lane, a0);
    if (lane + 64 < D) store_from_f32<T>(dq + tok * dqp + (size_t)h * D, lane + 64, a1);
  }
}

// Gradients of keys and values: a wave per (item, key-value head), which walks the rows of all its heads
template <typename T>
__global__ __launch_bounds__(64) void history_dkv_generic(const T* q, const T* k, const T* v, long long qp, long long kp,
                                                          long long vp, const int32_t* off, int T_all, int L, int H, int Hkv,
                                                          int D, float inv_gamma, const float* lse, const T* go,
                                                          const float* delta, T* dk, T* dv, long long dkp, long long dvp) {
  __shared__ float ks[128], vs[128];
  const int hk = blockIdx.y, n = blockIdx.z, lane = threadIdx.x, G = H / Hkv;
  const CandRange r = cand_range(off, n, L, T_all);
  for (int j = blockIdx.x; j < r.count; j += gridDim.x) {
    const size_t item = (size_t)r.first + j;
    __syncthreads();
    for (int d = lane; d < D; d += 64) {
      ks[d] = load_as_f32<T>(k + item * kp + (size_t)hk * D, d);
      vs[d] = load_as_f32<T>(v + item * vp + (size_t)hk * D, d);
    }
    __syncthreads();
    float k0 = 0.0f, k1 = 0.0f, v0 = 0.0f, v1 = 0.0f;
    const int rows = (r.count - j) * G;
    for (int t = 0; t < rows; t += 64) {
      const int x = t + lane;
      float p = 0.0f, ds = 0.0f;
      if (x < rows) {
        const size_t tok = item + x / G;
        const int h = hk * G + x % G;
        const float s = dot_row<T>(ks, q + tok * qp + (size_t)h * D, D) * inv_gamma * LOG2E;
        p = exp2f(s - lse[tok * H + h] * LOG2E);
        ds = p * (dot_row<T>(vs, go + (tok * H + h) * D, D) - delta[tok * H + h]) * inv_gamma;
      }
      for (int y = 0; y < 64 && t + y < rows; ++y) {
        const float py = __shfl(p, y), dy = __shfl(ds, y);
        const size_t tok = item + (t + y) / G;
        const int h = hk * G + (t + y) % G;
        const T* qr = q + tok * qp + (size_t)h * D;
        const T* gr = go + (tok * H + h) * D;
        if (lane < D) {
          k0 = fmaf(dy, load_as_f32<T>(qr, lane), k0);
          v0 = fmaf(py, load_as_f32<T>(gr, lane), v0);
        }
        if (lane + 64 < D) {
          k1 = fmaf(dy, load_as_f32<T>(qr, lane + 64), k1);
          v1 = fmaf(py, load_as_f32<T>(gr, lane + 64), v1);
        }
      }
    }
    if (lane < D) {
      store_from_f32<T>(dk + item * dkp + (size_t)hk * D, lane, k0);
      store_from_f32<T>(dv + item * dvp + (size_t)hk * D, lane, v0);
    }
    if (lane + 64 < D) {
      store_from_f32<T>(dk + item * dkp + (size_t)hk * D, lane + 64, k1);
      store_from_f32<T>(dv + item * dvp + (size_t)hk * D, lane + 64, v1);
    }
  }
}

static int at_most(int x, int lim) { return x < lim ? x : lim; }

template <typename T>
static laser_status forward_typed(const HistoryArgs& a) {
  for (int n = 0; n < a.N; n += 65535) {
    const dim3 grid(at_most(a.L, 4096), a.H, at_most(a.N - n, 65535));
    history_forward_generic<T><<<grid, 64, 0, a.stream>>>(
        static_cast<const T*>(a.q), static_cast<const T*>(a.k), static_cast<const T*>(a.v), a.qp, a.kp, a.vp, a.off + n, a.T,
        a.L, a.H, a.Hkv, a.D, LOG2E / a.gamma, static_cast<T*>(a.o), a.lse);
  }
  return launch_status();
}
laser_status history_forward_launch(const HistoryArgs& a) {
  return a.dt == LASER_F32 ? forward_typed<float>(a) : history_tile_launch(a);
}

template <typename T>
static laser_status backward_typed(const HistoryBwdArgs& b) {
  const HistoryArgs& a = b.f;
  const T *q = static_cast<const T*>(a.q), *k = static_cast<const T*>(a.k), *v = static_cast<const T*>(a.v);
  for (int n = 0; n < a.N; n += 65535) {
    const dim3 grid(at_most(a.L, 4096), a.H, at_most(a.N - n, 65535));
    history_dq_generic<T><<<grid, 64, 0, a.stream>>>(q, k, v, a.qp, a.kp, a.vp, a.off + n, a.T, a.L, a.H, a.Hkv, a.D,
                                                     1.0f / a.gamma, static_cast<const T*>(a.o), a.lse,
                                                     static_cast<const T*>(b.go), static_cast<T*>(b.dq), b.dqp, b.work);
    history_dkv_generic<T><<<dim3(grid.x, a.Hkv, grid.z), 64, 0, a.stream>>>(
        q, k, v, a.qp, a.kp, a.vp, a.off + n, a.T, a.L, a.H, a.Hkv, a.D, 1.0f / a.gamma, a.lse, static_cast<const T*>(b.go),
        b.work, static_cast<T*>(b.dk), static_cast<T*>(b.dv), b.dkp, b.dvp);
  }
  return launch_status();
}
size_t history_backward_work_bytes(int, int T, int, int H, int, int, laser_dtype) { return (size_t)T * H * 8; }
laser_status history_backward_launch(const HistoryBwdArgs& a) {
  return a.f.dt == LASER_F32 ? backward_typed<float>(a) : history_bwd_tile_launch(a);
}

template <typename T>
static laser_status cache_attention_typed(const CacheArgs& a) {
  for (int u = 0; u < a.U; u += 65535) {
    const dim3 grid(at_most(a.C, 4096), a.H, at_most(a.U - u, 65535));
    cache_attention_generic<T><<<grid, 64, 0, a.stream>>>(
        static_cast<const T*>(a.q), a.qp, static_cast<const T*>(a.k), static_cast<const T*>(a.v), a.off + u,
        a.pages + (size_t)u * a.max_pages, a.lens + u, a.T, a.C, a.L, a.H, a.Hkv, a.D, a.page_log2, a.P, a.max_pages,
        LOG2E / a.gamma, a.causal, static_cast<T*>(a.o), a.lse);
  }
  return launch_status();
}
static bool few_rows(int C, int H, int Hkv) { return (long long)C * (H / Hkv) <= 32; }
static CacheRuns runs_of(int U, int C, int L, int H, int Hkv, laser_dtype dt) {
  if (dt == LASER_F32) return CacheRuns{L, 1};
  const long long tiles = few_rows(C, H, Hkv) ? 1 : ((long long)C * (H / Hkv) + 127) / 128, all = tiles * U * Hkv;
  return cache_runs(all < 512 ? (int)all : 512, L, few_rows(C, H, Hkv) ? 512 : 256, few_rows(C, H, Hkv) ? 128 : 64);
}
size_t cache_attention_work_bytes(int U, int T, int C, int L, int H, int Hkv, int D, laser_dtype dt) {
  const CacheRuns r = runs_of(U, C, L, H, Hkv, dt);
  return r.runs > 1 ? (size_t)r.runs * T * H * (D + 1) * 4 : 16;
}
laser_status cache_attention_launch(const CacheArgs& a) {
  if (a.dt == LASER_F32) return cache_attention_typed<float>(a);
  const CacheRuns r = runs_of(a.U, a.C, a.L, a.H, a.Hkv, a.dt);
  return few_rows(a.C, a.H, a.Hkv) ? cache_few_launch(a, r) : cache_tile_launch(a, r);
}

template <typename T>
static laser_status cache_weights_typed(const CacheArgs& a) {
  for (int u = 0; u < a.U; u += 65535) {
    const dim3 grid(at_most(a.L, 65535), at_most(a.U - u, 65535));
    cache_weights_generic<T><<<grid, 64, 0, a.stream>>>(
        static_cast<const T*>(a.q), a.qp, static_cast<const T*>(a.k), a.lse, a.off + u, a.pages + (size_t)u * a.max_pages,
        a.lens + u, a.T, a.C, a.L, a.H, a.Hkv, a.D, a.page_log2, a.P, a.max_pages, LOG2E / a.gamma, a.causal, a.weight, a.add);
  }
  return launch_status();
}
laser_status cache_weights_launch(const CacheArgs& a) {
  return a.dt == LASER_F32 ? cache_weights_typed<float>(a) : cache_weights_tile_launch(a);
}

}  // namespace laser
