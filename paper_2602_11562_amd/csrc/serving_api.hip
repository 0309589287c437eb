// Host side of the entry points for positions, the cache in 8 bits and the pages of a cache: argument validation (GPU-free) and dispatch.
#include "cache8.h"
#include "history_checks.h"
#include "pages.h"
#include "rotary.h"

namespace laser {

static laser_status rotary(const void* q, int64_t qp, const void* k, int64_t kp, const int32_t* pos, const double* freq, int T, int H, int Hkv,
                           int D, int R, laser_rotary_layout layout, float scale, laser_dtype dt, void* q_out, int64_t qop, void* k_out,
                           int64_t kop, bool back, void* stream) {
  const bool keys = Hkv != 0;
  if (!q || !q_out || !pos || !freq || (keys != (k != nullptr)) || (keys != (k_out != nullptr))) return LASER_ERR_NULL;
  if (dt != LASER_F32 && dt != LASER_BF16) return LASER_ERR_DTYPE;
  if (layout != LASER_ROTARY_HALF && layout != LASER_ROTARY_INTERLEAVED) return LASER_ERR_UNSUPPORTED;
  if (!sizes_fit(1, T, 1, H, 1, D) || Hkv < 0 || (keys && !sizes_fit(1, T, 1, Hkv, 1, D))) return LASER_ERR_SHAPE;
  if (R < 2 || R > D || R % 2 != 0 || !(fabsf(scale) < INFINITY)) return LASER_ERR_SHAPE;
  if (!pitch_fits(qp, H, D, dt) || !pitch_fits(qop, H, D, dt)) return LASER_ERR_SHAPE;
  if (keys && (!pitch_fits(kp, Hkv, D, dt) || !pitch_fits(kop, Hkv, D, dt))) return LASER_ERR_SHAPE;
  if ((q == q_out && qp != qop) || (keys && k == k_out && kp != kop)) return LASER_ERR_SHAPE;
  for (const void* p : {q, (const void*)q_out, k, (const void*)k_out})
    if (!aligned(p, 16)) return LASER_ERR_ALIGN;
  if (!aligned(pos, 4) || !aligned(freq, 8)) return LASER_ERR_ALIGN;
  return rotary_launch(RotaryArgs{{q, k}, {q_out, k_out}, {qp, kp}, {qop, kop}, {H, Hkv}, pos, freq, T, D, R,
                                  layout == LASER_ROTARY_INTERLEAVED, back, scale, dt, static_cast<hipStream_t>(stream)});
}

// A cache of 8-bit blocks
static laser_status validate_cache8(const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale, const int32_t* pages,
                                    const int32_t* lens, int U, int P, int page, int block, int max_pages, int L, int Hkv, int D,
                                    laser_dtype dt, void* stream, Cache8Args* out) {
  if (!k_scale || !v_scale) return LASER_ERR_NULL;
  Cache8Args a{};
  const laser_status s = validate_cache(k_cache, v_cache, pages, lens, U, P, page, max_pages, L, Hkv, D, dt, stream, &a.c);
  if (s != LASER_OK) return s;
  if (D % 16 != 0 || block < 8 || block > page || (block & (block - 1)) != 0) return LASER_ERR_SHAPE;
  if (!aligned(k_scale, 4) || !aligned(v_scale, 4)) return LASER_ERR_ALIGN;
  for (a.block_log2 = 3; (1 << a.block_log2) < block;) ++a.block_log2;
  a.k_scale = const_cast<float*>(k_scale);
  a.v_scale = const_cast<float*>(v_scale);
  *out = a;
  return LASER_OK;
}

// Rows of a key-value head that one column block holds: the streaming kernel
static bool few8_rows(int C, int H, int Hkv) { return (long long)C * (H / Hkv) <= 32; }
// Into how many runs. A cut costs a join, 4 to 6 us, and what its parts weigh.
// Many rows: two workgroups for each place that the chip has for them (three a compute unit of heads of 128, four of 64), which come by their
// lengths (us by 1024, 1536 and 2048 wanted; 8 heads over 2, rows x longest history, users: 512 x 10000, 16 of 128 211, 191, 200; 400 x 9000, 12
// of 128 112, 118, 123; 200 x 20000, 8 of 128 98, 96, 112; 256 x 4096, 32 of 64 71.5, 70.8, 67.7; more users, in their own order: 64 x 4096, 100
// of 128 -, 116, 111), of 512 items or more, of 256 where the longest history has few runs anyway and for fp32 (us by 256 and 512: 100 x
// 30000, 1 of 128 49.1, 41.6; 300 x 5000, 4 of 128 45.1, 41.3; 100 x 1000, 1 of 64 17.4, 21.3; fp32, 100 x 3000, 4 of 128 30.6, 38.1). None where the histories are short and two tiles of rows a compute
// unit (512) without a cut: 32 x 1000, 256 of 128, in four runs and whole: all of that length 117, 54, of lengths up to it 63, 50, most short 40, 43; 128 x 1000, 32
// of 128 (256 tiles) 33, 44. Nor where they are very short (two runs and whole: 50 x up to 300, 20 of 64 12.5, 11.0; 40 x 500, 4 of 64 11.8, 12.5).
// Few rows, us by one run a history and runs of 1024 and 512 items (heads of 128 over 2 key-value heads unless said otherwise):
//   1 x 65000, 16 heads (2 pairs)  307, 15.8, 15.2;  30 x 2000 (60)  13.1, 11.9, 9.8;  8 x 20000 (16)  88, 17.3, 17.9;  40 x 3000 fp32 (80)  25.7, 16.9, 17.7;
//   5 x 777 fp32 (10)  7.7, -, 9.2;  32 x 1000, 8 over 8 of 64 (256)  7.8, -, 10.4;  100 x 2000 (200)  16.9, 19.2, 22.1;  100 x 3000 (200)  21.8,
//   23.4, 26.8, most of them short 18.0, 18.5, 16.6;  128 x 4096 (256)  31.2, 37.9, 39.9, most short 24.6, 21.1, 24.0;  256 x 2000, four rows (512)  33.6, 42.9, 48.8
// Rules: none where the histories alone are two workgroups a compute unit, or short, or one for every other unit and of medium length; else
// runs of 512 while they are one workgroup a compute unit, and of 1024 beyond.
CacheRuns cache8_runs_of(int U, int C, int L, int H, int Hkv, int D, laser_dtype dt) {
  const long long pairs = (long long)U * Hkv, rows = (long long)C * (H / Hkv);
  const long long tiles = (rows + 127) / 128 * pairs;
  if (!few8_rows(C, H, Hkv)) {
    if (L <= (tiles >= 512 ? 1024 : 384)) return CacheRuns{(L + 63) / 64 * 64, 1};
    return cache_runs(tiles, L, D > 64 && U <= CACHE8_RANKED ? 1536 : 2048, L > 2048 && dt != LASER_F32 ? 512 : 256, 64);
  }
  if (pairs >= 512 || L <= (pairs > 128 ? 3200 : 1024)) return CacheRuns{(L + 255) / 256 * 256, 1};
  return cache_runs(pairs, L, 1024, pairs * ((L + 511) / 512) <= 256 ? 512 : 1024, 256);
}
// Eight waves where there is about one workgroup a compute unit, whose way is then half as long (us by four and eight: 1 x 65000 15.5 and
// 14.8, 40 x 3000 fp32 18.7 and 17.0, 32 x 1000 9.4 and 7.8); four beyond, two workgroups of which share a compute unit (128 x 4096, most
// of them short, 21.5 and 25.0, 256 x 2000, four rows, 34.2 and 36.2).
int cache8_waves(int U, int Hkv, const CacheRuns& r) { return (long long)U * Hkv * r.runs <= 320 ? 8 : 4; }
size_t cache8_attention_work_bytes(int U, int T, int C, int L, int H, int Hkv, int D, laser_dtype dt) {
  const CacheRuns r = cache8_runs_of(U, C, L, H, Hkv, D, dt);
  return r.runs > 1 ? (size_t)r.runs * T * H * (D + 1) * 4 : 16;
}
laser_status cache8_attention_launch(const Cache8Args& a) {
  const CacheRuns r = cache8_runs_of(a.c.U, a.c.C, a.c.L, a.c.H, a.c.Hkv, a.c.D, a.c.dt);
  return few8_rows(a.c.C, a.c.H, a.c.Hkv) ? cache8_few_launch(a, r) : cache8_tile_launch(a, r);
}

constexpr int MOST_PAGES = 1 << 26, MOST_PARTS = 1024;
constexpr int64_t MOST_PAGE_BYTES = 1 << 27;

// The counts, and users' tables
static laser_status validate_pages(const int32_t* pages, const int32_t* lens, const int32_t* refs, int U, int P, int page, int max_pages,
                                   const void* work, bool needs_work, size_t work_bytes, void* stream, PagesArgs* a) {
  if (!pages || !lens || !refs || (needs_work && !work)) return LASER_ERR_NULL;
  if (U <= 0 || P <= 0 || P > MOST_PAGES || max_pages <= 0 || page < 8 || page > 4096 || (page & (page - 1)) != 0) return LASER_ERR_SHAPE;
  if ((long long)U * max_pages > 0x7fffffffLL || (long long)max_pages * page > 0x7fffffffLL) return LASER_ERR_SHAPE;
  for (const void* p : {(const void*)pages, (const void*)lens, (const void*)refs, work})
    if (!aligned(p, 4)) return LASER_ERR_ALIGN;
  if (needs_work && work_bytes < pages_work_ints(U, P) * 4) return LASER_ERR_SHAPE;
  a->pages = pages;
  a->lens = lens;
  a->refs = const_cast<int32_t*>(refs);
  a->U = U;
  a->P = P;
  for (a->page_log2 = 3; (1 << a->page_log2) < page;) ++a->page_log2;
  a->max_pages = max_pages;
  a->stream = static_cast<hipStream_t>(stream);
  a->work = static_cast<int32_t*>(const_cast<void*>(work));
  return LASER_OK;
}
static laser_status validate_parts(void* const* parts, const int64_t* part_bytes, int n_parts, bool some, PagesArgs* a) {
  if (n_parts < 0 || n_parts > MOST_PARTS || (some && n_parts == 0)) return LASER_ERR_SHAPE;
  if (n_parts > 0 && (!parts || !part_bytes)) return LASER_ERR_NULL;
  for (int i = 0; i < n_parts; ++i) {
    if (!parts[i]) return LASER_ERR_NULL;
    if (part_bytes[i] <= 0 || part_bytes[i] > MOST_PAGE_BYTES) return LASER_ERR_SHAPE;
  }
  a->parts = parts;
  a->part_bytes = part_bytes;
  a->n_parts = n_parts;
  return LASER_OK;
}

}  // namespace laser

using namespace laser;

extern "C" {

laser_status laser_rotary_frequencies(int R, double base, laser_rotary_scaling scaling, double factor, double length, double low, double high,
                                      double* freq_out, void* stream) {
  if (!freq_out) return LASER_ERR_NULL;
  if (scaling < LASER_ROTARY_NONE || scaling > LASER_ROTARY_PARTS) return LASER_ERR_UNSUPPORTED;
  if (R < 2 || R > 128 || R % 2 != 0 || !(base > 0.0 && base < INFINITY)) return LASER_ERR_SHAPE;
  if (scaling != LASER_ROTARY_NONE && !(factor > 0.0 && factor < INFINITY)) return LASER_ERR_SHAPE;
  if (scaling == LASER_ROTARY_PARTS && !(length > 0.0 && length < INFINITY && low >= 0.0 && low < high && high < INFINITY)) return LASER_ERR_SHAPE;
  if (!aligned(freq_out, 8)) return LASER_ERR_ALIGN;
  return rotary_frequencies_launch(RotaryFrequencies{freq_out, R, base, factor, scaling, length, low, high, static_cast<hipStream_t>(stream)});
}

laser_status laser_rotary_forward(const void* q, int64_t q_pitch, const void* k, int64_t k_pitch, const int32_t* pos, const double* freq, int T,
                                  int H, int H_kv, int D, int R, laser_rotary_layout layout, float scale, laser_dtype dt, void* q_out,
                                  int64_t q_out_pitch, void* k_out, int64_t k_out_pitch, void* stream) {
  return rotary(q, q_pitch, k, k_pitch, pos, freq, T, H, H_kv, D, R, layout, scale, dt, q_out, q_out_pitch, k_out, k_out_pitch, false, stream);
}

laser_status laser_rotary_backward(const void* d_q, int64_t d_q_pitch, const void* d_k, int64_t d_k_pitch, const int32_t* pos, const double* freq,
                                   int T, int H, int H_kv, int D, int R, laser_rotary_layout layout, float scale, laser_dtype dt, void* dq_out,
                                   int64_t dq_pitch, void* dk_out, int64_t dk_pitch, void* stream) {
  return rotary(d_q, d_q_pitch, d_k, d_k_pitch, pos, freq, T, H, H_kv, D, R, layout, scale, dt, dq_out, dq_pitch, dk_out, dk_pitch, true, stream);
}

laser_status laser_cache8_append(const void* k, int64_t k_pitch, const void* v, int64_t v_pitch, void* k_cache, void* v_cache, float* k_scale,
                                 float* v_scale, const int32_t* off, const int32_t* pages, const int32_t* lens, int U, int T, int C_max, int P,
                                 int page, int block, int max_pages, int L_max, int H_kv, int D, laser_dtype dt, void* stream) {
  Cache8Args a;
  laser_status s = validate_cache8(k_cache, v_cache, k_scale, v_scale, pages, lens, U, P, page, block, max_pages, L_max, H_kv, D, dt, stream, &a);
  if (s == LASER_OK) s = validate_rows(k, k_pitch, H_kv, off, T, C_max, &a.c);
  if (s == LASER_OK) s = validate_rows(v, v_pitch, H_kv, off, T, C_max, &a.c);
  if (s != LASER_OK) return s;
  a.k_new = k;
  a.v_new = v;
  a.kp = k_pitch;
  a.vp = v_pitch;
  return cache8_append_launch(a);
}

size_t laser_cache8_attention_work_bytes(int U, int T, int C_max, int L_max, int H, int H_kv, int D, laser_dtype dt) {
  if ((dt != LASER_F32 && dt != LASER_BF16) || !sizes_fit(U, T, L_max, H, H_kv, D) || !sizes_fit(U, T, C_max, H, H_kv, D)) return 0;
  return cache8_attention_work_bytes(U, T, C_max, L_max, H, H_kv, D, dt);
}

laser_status laser_cache8_attention_forward(const void* q, int64_t q_pitch, const void* k_cache, const void* v_cache, const float* k_scale,
                                            const float* v_scale, const int32_t* off, const int32_t* pages, const int32_t* lens, int U, int T,
                                            int C_max, int P, int page, int block, int max_pages, int L_max, int H, int H_kv, int D,
                                            float gamma, int causal, laser_dtype dt, void* o_out, float* lse_out, void* work,
                                            size_t work_bytes, void* stream) {
  if (!o_out || !work) return LASER_ERR_NULL;
  Cache8Args a;
  laser_status s = validate_cache8(k_cache, v_cache, k_scale, v_scale, pages, lens, U, P, page, block, max_pages, L_max, H_kv, D, dt, stream, &a);
  if (s == LASER_OK) s = validate_rows(q, q_pitch, H, off, T, C_max, &a.c);
  if (s != LASER_OK) return s;
  if (!gamma_fits(gamma)) return LASER_ERR_SHAPE;
  if (!aligned(o_out, 16) || !aligned(lse_out, 4) || !aligned(work, 16)) return LASER_ERR_ALIGN;
  if (work_bytes < cache8_attention_work_bytes(U, T, C_max, L_max, H, H_kv, D, dt)) return LASER_ERR_SHAPE;
  a.c.q = q;
  a.c.qp = q_pitch;
  a.c.gamma = gamma;
  a.c.causal = causal != 0;
  a.c.o = o_out;
  a.c.lse = lse_out;
  a.c.work = static_cast<float*>(work);
  return cache8_attention_launch(a);
}

size_t laser_pages_work_bytes(int U, int P) { return U <= 0 || P <= 0 || P > MOST_PAGES ? 0 : pages_work_ints(U, P) * 4; }

laser_status laser_pages_copy(void* const* parts, const int64_t* part_bytes, int n_parts, const int32_t* from, const int32_t* to, int n, int P,
                              void* stream) {
  if (!from || !to) return LASER_ERR_NULL;
  PagesArgs a{};
  const laser_status s = validate_parts(parts, part_bytes, n_parts, true, &a);
  if (s != LASER_OK) return s;
  if (n <= 0 || P <= 0 || P > MOST_PAGES) return LASER_ERR_SHAPE;
  if (!aligned(from, 4) || !aligned(to, 4)) return LASER_ERR_ALIGN;
  a.P = P;
  a.stream = static_cast<hipStream_t>(stream);
  return pages_copy_launch(a, from, to, n);
}

laser_status laser_pages_grow(int32_t* pages, int32_t* lens, const int32_t* off, int32_t* refs, int U, int P, int page, int max_pages,
                              int32_t* missing_out, void* work, size_t work_bytes, void* stream) {
  if (!off || !missing_out) return LASER_ERR_NULL;
  PagesArgs a{};
  const laser_status s = validate_pages(pages, lens, refs, U, P, page, max_pages, work, true, work_bytes, stream, &a);
  if (s != LASER_OK) return s;
  if (!aligned(off, 4) || !aligned(missing_out, 4)) return LASER_ERR_ALIGN;
  a.off = off;
  a.lens_out = lens;
  a.missing = missing_out;
  return pages_grow_launch(a);
}

laser_status laser_pages_fork(void* const* parts, const int64_t* part_bytes, int n_parts, const int32_t* pages, const int32_t* lens,
                              const int32_t* source, int32_t* refs, int U, int V, int P, int page, int max_pages, int max_pages_out,
                              int32_t* pages_out, int32_t* lens_out, int32_t* missing_out, void* work, size_t work_bytes, void* stream) {
  if (!source || !pages_out || !lens_out || !missing_out) return LASER_ERR_NULL;
  PagesArgs a{};
  laser_status s = validate_parts(parts, part_bytes, n_parts, false, &a);
  if (s == LASER_OK) s = validate_pages(pages, lens, refs, U, P, page, max_pages, work, true, work_bytes, stream, &a);
  if (s != LASER_OK) return s;
  if (V <= 0 || max_pages_out <= 0 || (long long)V * max_pages_out > 0x7fffffffLL || (long long)max_pages_out * page > 0x7fffffffLL ||
      work_bytes < pages_work_ints(V, P) * 4)
    return LASER_ERR_SHAPE;
  for (const void* p : {(const void*)source, (const void*)pages_out, (const void*)lens_out, (const void*)missing_out})
    if (!aligned(p, 4)) return LASER_ERR_ALIGN;
  a.source = source;
  a.V = V;
  a.max_out = max_pages_out;
  a.pages_out = pages_out;
  a.lens_out = lens_out;
  a.missing = missing_out;
  return pages_fork_launch(a);
}

laser_status laser_pages_free(const int32_t* pages, int32_t* lens, const int32_t* gone, int32_t* refs, int U, int P, int page, int max_pages,
                              void* stream) {
  PagesArgs a{};
  const laser_status s = validate_pages(pages, lens, refs, U, P, page, max_pages, nullptr, false, 0, stream, &a);
  if (s != LASER_OK) return s;
  if (!aligned(gone, 4)) return LASER_ERR_ALIGN;
  a.gone = gone;
  a.lens_out = lens;
  return pages_free_launch(a);
}

laser_status laser_pages_compact(void* const* parts, const int64_t* part_bytes, int n_parts, const int32_t* pages, const int32_t* lens,
                                 const int32_t* refs, int U, int P, int page, int max_pages, int32_t* pages_out, int32_t* refs_out,
                                 int32_t* in_use_out, void* work, size_t work_bytes, void* stream) {
  if (!pages_out || !refs_out || !in_use_out) return LASER_ERR_NULL;
  PagesArgs a{};
  laser_status s = validate_parts(parts, part_bytes, n_parts, false, &a);
  if (s == LASER_OK) s = validate_pages(pages, lens, refs, U, P, page, max_pages, work, true, work_bytes, stream, &a);
  if (s != LASER_OK) return s;
  for (const void* p : {(const void*)pages_out, (const void*)refs_out, (const void*)in_use_out})
    if (!aligned(p, 4)) return LASER_ERR_ALIGN;
  a.pages_out = pages_out;
  a.refs_out = refs_out;
  a.in_use = in_use_out;
  return pages_compact_launch(a);
}

}  // extern "C"
