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
// Into how many runs the longest history is cut. A cut costs a join, 4 to 6 us, and what its parts weigh; sizes alone decide, which whoever
// provides the work buffer knows too. Figures: us of captured calls; users x history, bf16 over 2 key-value heads of 128 unless said
// otherwise; "full": all histories that long, "up to": of all lengths up to it, "spread": over decades of lengths.
//
// Many rows: two workgroups for each place that the chip has for them (three a compute unit of heads of 128, four of 64), which come by their
// lengths; more users, in their own order, a few more. By 1024, 1536 and 2048 wanted, 8 heads, new rows a user ahead:
//   512, 16 x up to 10000       210, 192, 196      256, 32 x up to 4096 of 64    76.1, 68.7, 65.5
//   400, 12 x up to 9000        112, 117, 120      64, 100 x up to 4096          108, 105, 104
//   200, 8 x up to 20000        95.8, 93.9, 109
// Runs of 512 items or more, of 256 where the longest history has few runs anyway (100, 1 x 30000 by 256 and 512: 44.7, 40.2; 300, 4 x up to
// 5000: 42.0, 39.7; 100, 1 x 1000 of 64: 12.1, 15.5) and for fp32 (100, 4 x 3000: 40.0, 37.5, spread 24.6, 24.7; 300, 8 x up to 3000 64.2,
// 57.4: since two waves may share their rows, 512 would do there too). None where the histories are short and the tiles of rows two a compute unit (512)
// without a cut (in four runs and whole: 32, 256 x 1000 109, 51.5, up to 1000 59.3, 45.9, spread 37.8, 39.2; 256 tiles, 128, 32 x up to 1000, 30.4,
// 31.8). Nor where they are very short (in two runs and whole: 50, 20 x up to 300 of 64 13.2, 11.8; 40, 4 x 500 of 64 12.4, 13.1).
//
// Few rows, by one run a history, runs of 1024 and of 512 items (pairs of a user and a key-value head in brackets):
//   1 x 65000, 16 heads (2)     296, 15.7, 13.7    32 x 1000, 8 of 64 (256)      9.0, -, 11.8
//   30 x 2000 (60)              14.6, 13.5, 11.1   100 x 2000 (200)              20.6, 24.0, 27.6
//   8 x 20000 (16)              96, 26.8, 25.3     100 x 3000 (200)              27.3, 36.4, 35.9, spread 18.6, 19.4, 16.6
//   40 x 3000 fp32 (80)         26.1, 19.8, 20.8   256 x 2000, four rows (512)   46.7, 56.6, 65.1, spread 25.6, 28.6, 29.4
//   5 x 777 of 64 fp32 (10)     8.6, -, 9.6
// None where the histories alone are two workgroups a compute unit, or short, or one for every other unit and of medium length; else runs of 512
// while they are one workgroup a compute unit, and of 1024 beyond. Between 129 and 511 pairs sizes do not tell full histories, for which a cut costs
// up to a quarter, from spread ones, which wait for their longest: whole and cut, full, up to and spread
//   128 x 4096 (256)   43.3, 49.4   31.6, 37.8   25.4, 21.5      80 x 8000 (160)    59.9, 64.6   43.6, 44.0   40.3, 23.8
//   100 x 4096 (200)   34.8, 41.2   27.4, 34.0   24.5, 19.6      200 x 8000 (400)   143, 160     112, 105     72.7, 43.5
//   200 x 3500 (400)   66.3, 79.5   42.9, 43.7   36.1, 25.6      250 x 4096 (500)   94.8, 103    62.7, 66.7   40.1, 35.2
// so beyond 3200 items the rule goes by the spread ones, where the wait is up to two fifths.
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
