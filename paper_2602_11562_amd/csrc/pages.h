// The pages of a cache: who holds them, and copies of them. Arguments after validation, and the launchers.
#pragma once

#include "laser_internal.h"

namespace laser {

// go(u) for users first, first + step, .. below U, which may be 2^31 - 1 of tables of one page: the step behind the last (of 2^16 at most) does
// not fit an int, which would go on below 0 and still be less than U
template <typename Go>
__host__ __device__ __forceinline__ void for_users(unsigned first, unsigned step, int U, Go&& go) {
  for (unsigned u = first; u < (unsigned)U; u += step) go((int)u);
}

// Arrays [P, page bytes] that a page is made of, at most N a launch. (4 or 16: 100 bytes of arguments cost a launch 0.2 us)
constexpr int FEW_PARTS = 4, PARTS_A_LAUNCH = 16;
template <int N>
struct PageParts {
  unsigned char* at[N];
  unsigned bytes[N];         // of a page
  unsigned char piece_log2[N];   // bytes of a piece: 4 (16 bytes), 2 or 0
  int n;
  unsigned all;              // pieces of a page in all parts
};

struct PagesArgs {
  void* const* parts;        // host arrays
  const int64_t* part_bytes;
  int n_parts;
  const int32_t* pages;      // [U,max_pages]
  const int32_t* lens;       // [U]
  int32_t* refs;             // [P]
  int U, P, page_log2, max_pages;
  hipStream_t stream;
  int32_t* work;             // pages_work_ints() of them
  // fork
  const int32_t* source;     // [V]
  int V, max_out;
  int32_t* pages_out;        // [V,max_out], compact: [U,max_pages]
  int32_t* lens_out;         // [V], grow: lens itself
  int32_t* missing;          // [1]
  // grow
  const int32_t* off;        // [U + 1]
  // free
  const int32_t* gone;       // [U], nullptr: all of them
  // compact
  int32_t* refs_out;         // [P]
  int32_t* in_use;           // [1]
};
size_t pages_work_ints(int U, int P);
laser_status pages_fork_launch(const PagesArgs& a);
laser_status pages_grow_launch(const PagesArgs& a);
laser_status pages_free_launch(const PagesArgs& a);
laser_status pages_compact_launch(const PagesArgs& a);
laser_status pages_copy_launch(const PagesArgs& a, const int32_t* src, const int32_t* dst, int n);

}  // namespace laser
