// A paged cache of keys and values in 8 bits: items are e4m3 numbers (4 bits of exponent, 3 of mantissa), of which each block of
// 2^block_log2 items of a key-value head has a power of two for its scale. Arguments after validation, and the launchers.
#pragma once

#include "history.h"

namespace laser {

struct Cache8Args {
  CacheArgs c;             // k and v are bytes [P,Hkv,page,D]; dt is the type of the rows beside the cache
  float* k_scale;          // [P,Hkv,page / block]
  float* v_scale;
  int block_log2;
  const void* k_new;       // append: [T,Hkv,D]
  const void* v_new;
  long long kp, vp;
};
laser_status cache8_append_launch(const Cache8Args& a);
CacheRuns cache8_runs_of(int U, int C, int L, int H, int Hkv, int D, laser_dtype dt);
int cache8_waves(int U, int Hkv, const CacheRuns& r);    // of a workgroup of the kernel for few rows
size_t cache8_attention_work_bytes(int U, int T, int C, int L, int H, int Hkv, int D, laser_dtype dt);
laser_status cache8_attention_launch(const Cache8Args& a);
laser_status cache8_few_launch(const Cache8Args& a, const CacheRuns& r);    // at most 32 rows a key-value head
laser_status cache8_join_launch(const CacheArgs& a, const CacheRuns& r);
constexpr int CACHE8_RANKED = 64;                        // so many users the tiles of rows come by their lengths, a lane for each
laser_status cache8_tile_launch(const Cache8Args& a, const CacheRuns& r);

constexpr float E4M3_MAX = 448.0f;                       // 1.75 * 2^8
constexpr int LEAST_SCALE = -100, MOST_SCALE = 119;      // exponents; with the largest, the largest item is 1.75 * 2^127

}  // namespace laser
