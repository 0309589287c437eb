// Host side of the entry points for attention among the items of histories: argument validation (GPU-free) and dispatch.
#include <initializer_list>

#include "history.h"

namespace laser {

static bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

static int element_bytes(laser_dtype dt) { return dt == LASER_F32 ? 4 : 2; }

// Sequences or users, rows, the longest of them, heads and their width
static bool sizes_fit(int N, int T, int L, int H, int Hkv, int D) {
  if (N <= 0 || T <= 0 || L <= 0 || H <= 0 || Hkv <= 0 || D <= 0) return false;
  if (D > 128 || D % 8 != 0 || H > 1024 || H % Hkv != 0) return false;
  return (long long)L * H <= 0x3fffffffLL && (long long)T * H <= 0x7fffffffLL;
}

// Elements from one token's row to the next: rows do not overlap, 16-byte pieces stay whole, and 128 rows are within reach of a
// 32-bit byte offset
static bool pitch_fits(long long pitch, int heads, int D, laser_dtype dt) {
  return pitch >= (long long)heads * D && pitch <= (1 << 22) && pitch * element_bytes(dt) % 16 == 0;
}

// log2(e) / gamma, and 1 / gamma of the gradients, are fp32 numbers
static bool gamma_fits(float gamma) { return gamma >= 0x1p-126f && gamma < INFINITY; }

static laser_status validate_history(const void* q, int64_t qp, const void* k, int64_t kp, const void* v, int64_t vp,
                                     const int32_t* off, int N, int T, int L, int H, int Hkv, int D, float gamma, laser_dtype dt,
                                     const void* o, const float* lse, void* stream, HistoryArgs* out) {
  if (!q || !k || !v || !off || !o) return LASER_ERR_NULL;
  if (dt != LASER_F32 && dt != LASER_BF16) return LASER_ERR_DTYPE;
  if (!sizes_fit(N, T, L, H, Hkv, D) || !gamma_fits(gamma)) return LASER_ERR_SHAPE;
  if (!pitch_fits(qp, H, D, dt) || !pitch_fits(kp, Hkv, D, dt) || !pitch_fits(vp, Hkv, D, dt)) return LASER_ERR_SHAPE;
  for (const void* p : {q, k, v, o})
    if (!aligned(p, 16)) return LASER_ERR_ALIGN;
  if (!aligned(off, 4) || !aligned(lse, 4)) return LASER_ERR_ALIGN;
  *out = HistoryArgs{q, k, v, qp, kp, vp, off, N, T, L, H, Hkv, D, gamma, dt, const_cast<void*>(o), const_cast<float*>(lse),
                     static_cast<hipStream_t>(stream)};
  return LASER_OK;
}

// What every entry point of the cache has in common: the cache itself, its table and the users' lengths
static laser_status validate_cache(const void* k_cache, const void* v_cache, const int32_t* pages, const int32_t* lens, int U,
                                   int P, int page, int max_pages, int L, int Hkv, int D, laser_dtype dt, void* stream,
                                   CacheArgs* out) {
  if (!k_cache || !v_cache || !pages || !lens) return LASER_ERR_NULL;
  if (dt != LASER_F32 && dt != LASER_BF16) return LASER_ERR_DTYPE;
  if (!sizes_fit(U, 1, L, Hkv, Hkv, D) || P <= 0 || max_pages <= 0) return LASER_ERR_SHAPE;
  if (page < 8 || page > 4096 || (page & (page - 1)) != 0) return LASER_ERR_SHAPE;
  if (!aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(pages, 4) || !aligned(lens, 4)) return LASER_ERR_ALIGN;
  CacheArgs a{};
  a.k = const_cast<void*>(k_cache);
  a.v = const_cast<void*>(v_cache);
  a.pages = pages;
  a.lens = lens;
  a.U = U;
  a.P = P;
  for (a.page_log2 = 3; (1 << a.page_log2) < page;) ++a.page_log2;
  a.max_pages = max_pages;
  a.L = L;
  a.H = a.Hkv = Hkv;
  a.D = D;
  a.dt = dt;
  a.stream = static_cast<hipStream_t>(stream);
  *out = a;
  return LASER_OK;
}

// The rows beside the cache (queries, or new keys and values): packed by off, at most C a user
static laser_status validate_rows(const void* rows, int64_t pitch, int heads, const int32_t* off, int T, int C, CacheArgs* a) {
  if (!rows || !off) return LASER_ERR_NULL;
  if (T <= 0 || C <= 0 || heads <= 0 || heads % a->Hkv != 0 || !sizes_fit(a->U, T, C, heads, a->Hkv, a->D) ||
      !sizes_fit(a->U, T, a->L, heads, a->Hkv, a->D) || !pitch_fits(pitch, heads, a->D, a->dt))
    return LASER_ERR_SHAPE;
  if (!aligned(rows, 16) || !aligned(off, 4)) return LASER_ERR_ALIGN;
  a->off = off;
  a->T = T;
  a->C = C;
  a->H = heads;
  return LASER_OK;
}

// What the backward pass keeps of every row between its two kernels
size_t history_backward_work_bytes(int, int T, int, int H, int, int, laser_dtype) { return (size_t)T * H * 8; }

laser_status history_forward_launch(const HistoryArgs& a) { return a.dt == LASER_F32 ? history_f32_launch(a) : history_tile_launch(a); }
laser_status history_backward_launch(const HistoryBwdArgs& a) {
  return a.f.dt == LASER_F32 ? history_bwd_f32_launch(a) : history_bwd_tile_launch(a);
}
laser_status cache_weights_launch(const CacheArgs& a) {
  return a.dt == LASER_F32 ? cache_weights_f32_launch(a) : cache_weights_tile_launch(a);
}

// Rows of a key-value head that one column block holds: the streaming kernel (bf16). us by it and by the kernel of tiles: 64 users of up to
// 4000 items, 8 heads of 128 over 2, 4 rows 46 and 57, 8 rows 50 and 58 (of 64 28 and 34); 300 of 1000, 8 rows of 64 31 and 39; two of
// 30000, 8 rows of 128 22.5 and 20.9.
static bool few_rows(int C, int H, int Hkv, laser_dtype dt) { return dt == LASER_BF16 && (long long)C * (H / Hkv) <= 32; }
// Into how many runs: workgroups wanted, the fewest items of a run and the items that it is a whole number of. us, 8 heads over 2, rows x
// items, users:
//   single rows, 512 / 1024 / 2048 wanted: 1 x 20000, 8 of 128: 24.0, 23.8, 24.1; 1 x 5000, 64 of 64: 23.0, 26.8, 25.8, of 128 63, 66, 69;
//     2 x 3000, 200 of 128: 41.6, 40.0, 41.6; 256 / 512 / 1024 items: 1 x 30000, 1 of 128: 16.4, 16.9, 21.4; 1 x 20000, 8: 28.4, 24.1, 27.1
//   tiles of rows, 1024 / 2048 wanted: 200 x 20000, 8 of 128: 138, 132; 300 x 3000, 24 of 64: 57.2, 55.1; 400 new items x 9000, 12 of 128: 151, 146;
//     256 / 512 / 1024 items: 100 x 1000, 1 of 64: 13.9, 18.0, 23.0; 100 x 3000, 1 of 128: 19, 24, 36; 100 x 30000 (118 runs, joined by
//     the form for many): 45, 35, 40
//   fp32, 512 / 1024 / 2048 wanted: 1 x 20000, 4 of 128: 54, 44, 46; 1 x 3000, 32 of 64: 25, 31, 32; 2 x 3000, 100 of 128: 81, 72, 79; 128 / 256 /
//     512 items (its tiles are 32 items, one for each of four waves): 1 x 700, 5 of 64 (4 heads): 11.5, 13.2, 15.2; 1 x 20000, 1 of 64: 17.3, 16.1, 20.6
static CacheRuns runs_of(int U, int C, int L, int H, int Hkv, laser_dtype dt) {
  const bool few = few_rows(C, H, Hkv, dt);
  const long long pairs = (long long)U * Hkv, rows = (long long)C * (H / Hkv);
  if (dt == LASER_F32) return cache_runs((rows + 127) / 128 * pairs, L, 1024, 128, 128);
  return few ? cache_runs(pairs, L, 1024, 512, 128) : cache_runs((rows + 127) / 128 * pairs, L, 2048, 256, 64);
}
size_t cache_attention_work_bytes(int U, int T, int C, int L, int H, int Hkv, int D, laser_dtype dt) {
  const CacheRuns r = runs_of(U, C, L, H, Hkv, dt);
  return r.runs > 1 ? (size_t)r.runs * T * H * (D + 1) * 4 : 16;
}
laser_status cache_attention_launch(const CacheArgs& a) {
  const CacheRuns r = runs_of(a.U, a.C, a.L, a.H, a.Hkv, a.dt);
  if (a.dt == LASER_F32) return cache_f32_launch(a, r);
  return few_rows(a.C, a.H, a.Hkv, a.dt) ? cache_few_launch(a, r) : cache_tile_launch(a, r);
}

}  // namespace laser

using namespace laser;

extern "C" {

laser_status laser_history_attention_forward(const void* q, int64_t q_pitch, const void* k, int64_t k_pitch, const void* v,
                                             int64_t v_pitch, const int32_t* off, int N, int T, int L_max, int H, int H_kv, int D,
                                             float gamma, laser_dtype dt, void* o_out, float* lse_out, void* stream) {
  HistoryArgs a;
  const laser_status s = validate_history(q, q_pitch, k, k_pitch, v, v_pitch, off, N, T, L_max, H, H_kv, D, gamma, dt, o_out,
                                          lse_out, stream, &a);
  return s != LASER_OK ? s : history_forward_launch(a);
}

size_t laser_history_attention_backward_work_bytes(int N, int T, int L_max, int H, int H_kv, int D, laser_dtype dt) {
  if ((dt != LASER_F32 && dt != LASER_BF16) || !sizes_fit(N, T, L_max, H, H_kv, D)) return 0;
  return history_backward_work_bytes(N, T, L_max, H, H_kv, D, dt);
}

laser_status laser_history_attention_backward(const void* q, int64_t q_pitch, const void* k, int64_t k_pitch, const void* v,
                                              int64_t v_pitch, const void* o, const float* lse, const void* d_o,
                                              const int32_t* off, int N, int T, int L_max, int H, int H_kv, int D, float gamma,
                                              laser_dtype dt, void* dq_out, int64_t dq_pitch, void* dk_out, int64_t dk_pitch,
                                              void* dv_out, int64_t dv_pitch, void* work, size_t work_bytes, void* stream) {
  if (!lse || !d_o || !dq_out || !dk_out || !dv_out || !work) return LASER_ERR_NULL;
  HistoryBwdArgs a;
  const laser_status s = validate_history(q, q_pitch, k, k_pitch, v, v_pitch, off, N, T, L_max, H, H_kv, D, gamma, dt, o, lse,
                                          stream, &a.f);
  if (s != LASER_OK) return s;
  if (gamma > 0x1p120f) return LASER_ERR_SHAPE;   // (bf16 scores start at -gamma lse, lse up to log(L_max) < 21 past the largest)
  if (!pitch_fits(dq_pitch, H, D, dt) || !pitch_fits(dk_pitch, H_kv, D, dt) || !pitch_fits(dv_pitch, H_kv, D, dt))
    return LASER_ERR_SHAPE;
  for (const void* p : {d_o, (const void*)dq_out, (const void*)dk_out, (const void*)dv_out, (const void*)work})
    if (!aligned(p, 16)) return LASER_ERR_ALIGN;
  if (work_bytes < history_backward_work_bytes(N, T, L_max, H, H_kv, D, dt)) return LASER_ERR_SHAPE;
  a.go = d_o;
  a.dq = dq_out;
  a.dk = dk_out;
  a.dv = dv_out;
  a.dqp = dq_pitch;
  a.dkp = dk_pitch;
  a.dvp = dv_pitch;
  a.work = static_cast<float*>(work);
  return history_backward_launch(a);
}

laser_status laser_cache_append(const void* k, int64_t k_pitch, const void* v, int64_t v_pitch, void* k_cache, void* v_cache,
                                const int32_t* off, const int32_t* pages, const int32_t* lens, int U, int T, int C_max, int P,
                                int page, int max_pages, int L_max, int H_kv, int D, laser_dtype dt, float* weight,
                                void* stream) {
  CacheAppendArgs a;
  laser_status s = validate_cache(k_cache, v_cache, pages, lens, U, P, page, max_pages, L_max, H_kv, D, dt, stream, &a.c);
  if (s == LASER_OK) s = validate_rows(k, k_pitch, H_kv, off, T, C_max, &a.c);
  if (s == LASER_OK) s = validate_rows(v, v_pitch, H_kv, off, T, C_max, &a.c);
  if (s != LASER_OK) return s;
  if (!aligned(weight, 4)) return LASER_ERR_ALIGN;
  a.k = k;
  a.v = v;
  a.kp = k_pitch;
  a.vp = v_pitch;
  a.c.weight = weight;
  return cache_append_launch(a);
}

size_t laser_cache_attention_work_bytes(int U, int T, int C_max, int L_max, int H, int H_kv, int D, laser_dtype dt) {
  if ((dt != LASER_F32 && dt != LASER_BF16) || !sizes_fit(U, T, L_max, H, H_kv, D) || !sizes_fit(U, T, C_max, H, H_kv, D))
    return 0;
  return cache_attention_work_bytes(U, T, C_max, L_max, H, H_kv, D, dt);
}

laser_status laser_cache_attention_forward(const void* q, int64_t q_pitch, const void* k_cache, const void* v_cache,
                                           const int32_t* off, const int32_t* pages, const int32_t* lens, int U, int T, int C_max,
                                           int P, int page, int max_pages, int L_max, int H, int H_kv, int D, float gamma,
                                           int causal, laser_dtype dt, void* o_out, float* lse_out, void* work,
                                           size_t work_bytes, void* stream) {
  if (!o_out || !work) return LASER_ERR_NULL;
  CacheArgs a;
  laser_status s = validate_cache(k_cache, v_cache, pages, lens, U, P, page, max_pages, L_max, H_kv, D, dt, stream, &a);
  if (s == LASER_OK) s = validate_rows(q, q_pitch, H, off, T, C_max, &a);
  if (s != LASER_OK) return s;
  if (!gamma_fits(gamma)) return LASER_ERR_SHAPE;
  if (!aligned(o_out, 16) || !aligned(lse_out, 4) || !aligned(work, 16)) return LASER_ERR_ALIGN;
  if (work_bytes < cache_attention_work_bytes(U, T, C_max, L_max, H, H_kv, D, dt)) return LASER_ERR_SHAPE;
  a.q = q;
  a.qp = q_pitch;
  a.gamma = gamma;
  a.causal = causal != 0;
  a.o = o_out;
  a.lse = lse_out;
  a.work = static_cast<float*>(work);
  return cache_attention_launch(a);
}

laser_status laser_cache_weights(const void* q, int64_t q_pitch, const float* lse, const void* k_cache, const int32_t* off,
                                 const int32_t* pages, const int32_t* lens, int U, int T, int C_max, int P, int page,
                                 int max_pages, int L_max, int H, int H_kv, int D, float gamma, int causal, int add,
                                 laser_dtype dt, float* weight, void* stream) {
  if (!lse || !weight) return LASER_ERR_NULL;
  CacheArgs a;
  laser_status s = validate_cache(k_cache, k_cache, pages, lens, U, P, page, max_pages, L_max, H_kv, D, dt, stream, &a);
  if (s == LASER_OK) s = validate_rows(q, q_pitch, H, off, T, C_max, &a);
  if (s != LASER_OK) return s;
  if (!gamma_fits(gamma)) return LASER_ERR_SHAPE;
  if (!aligned(lse, 4) || !aligned(weight, 4)) return LASER_ERR_ALIGN;
  a.q = q;
  a.qp = q_pitch;
  a.gamma = gamma;
  a.causal = causal != 0;
  a.lse = const_cast<float*>(lse);
  a.weight = weight;
  a.add = add != 0;
  return cache_weights_launch(a);
}

laser_status laser_cache_evict(void* k_cache, void* v_cache, float* weight, const int32_t* pages, const int32_t* lens,
                               const int32_t* pages_out, int U, int P, int page, int max_pages, int max_pages_out, int L_max,
                               int budget, int recent, int H_kv, int D, laser_dtype dt, int32_t* lens_out, int32_t* kept_out,
                               void* stream) {
  if (!weight || !pages_out || !lens_out || !kept_out) return LASER_ERR_NULL;
  CacheEvictArgs a;
  const laser_status s = validate_cache(k_cache, v_cache, pages, lens, U, P, page, max_pages, L_max, H_kv, D, dt, stream, &a.c);
  if (s != LASER_OK) return s;
  if (budget <= 0 || recent < 0 || recent > budget || max_pages_out <= 0 || (long long)U * budget > 0x7fffffffLL)
    return LASER_ERR_SHAPE;
  const long long held = (long long)max_pages * page < L_max ? (long long)max_pages * page : L_max;   // most items of a user
  if ((long long)max_pages_out * page < (budget < held ? budget : held)) return LASER_ERR_SHAPE;
  for (const void* p : {(const void*)weight, (const void*)pages_out, (const void*)lens_out, (const void*)kept_out})
    if (!aligned(p, 4)) return LASER_ERR_ALIGN;
  a.c.weight = weight;
  a.pages_out = pages_out;
  a.max_pages_out = max_pages_out;
  a.budget = budget;
  a.recent = recent;
  a.lens_out = lens_out;
  a.kept = kept_out;
  return cache_evict_launch(a);
}

}  // extern "C"
