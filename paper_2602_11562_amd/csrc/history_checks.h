// What the entry points around attention among the items of histories check on the host before they launch anything (GPU-free).
#pragma once

#include <initializer_list>

#include "history.h"

namespace laser {

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

inline int element_bytes(laser_dtype dt) { return dt == LASER_F32 ? 4 : 2; }

// Sequences or users, rows, the longest of them, heads and their width
inline bool sizes_fit(int N, int T, int L, int H, int Hkv, int D) {
  if (N <= 0 || T <= 0 || L <= 0 || H <= 0 || Hkv <= 0 || D <= 0) return false;
  if (D > 128 || D % 8 != 0 || H > 1024 || H % Hkv != 0) return false;
  return (long long)L * H <= 0x3fffffffLL && (long long)T * H <= 0x7fffffffLL;
}

// Elements from one token's row to the next: rows do not overlap, 16-byte pieces stay whole, and 128 rows are within reach of a
// 32-bit byte offset
inline bool pitch_fits(long long pitch, int heads, int D, laser_dtype dt) {
  return pitch >= (long long)heads * D && pitch <= (1 << 22) && pitch * element_bytes(dt) % 16 == 0;
}

// log2(e) / gamma, and 1 / gamma of the gradients, are fp32 numbers
inline bool gamma_fits(float gamma) { return gamma >= 0x1p-126f && gamma < INFINITY; }

// What every entry point of the cache has in common: the cache itself, its table and the users' lengths
inline laser_status validate_cache(const void* k_cache, const void* v_cache, const int32_t* pages, const int32_t* lens, int U,
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
inline laser_status validate_rows(const void* rows, int64_t pitch, int heads, const int32_t* off, int T, int C, CacheArgs* a) {
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

}  // namespace laser
