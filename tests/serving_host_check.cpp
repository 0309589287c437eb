// Host-side check of rotary positions, the cache in 8 bits and the pages of a cache under AddressSanitizer and UndefinedBehaviorSanitizer (no
// GPU needed): every size at the edges of int and of its documented limits, alone and in pairs, through validation, the choice of forms and
// the launchers, whose launches are recorded (launch_recorder.cpp). Device pointers are never dereferenced on the host. Built by
// paper_2602_11562_amd.build.build_serving_host_check(), run by tests/test_serving_host_cpu.py. Exit status 0: every call returned what its
// sizes call for, and every launch holds fewer than 2^32 threads (a sanitizer report aborts).
#include <climits>
#include <cstdint>
#include <cstdio>
#include <functional>
#include <vector>

#include "laser.h"

struct LaunchRecord {
  const char* kernel;
  unsigned grid, block;
  unsigned long long lds;
  int limit;
};
extern "C" int launch_count();
extern "C" void launch_clear();
extern "C" const LaunchRecord* launch_record(int i);

static int failures = 0, accepted = 0, refused = 0;

// status of a call; nothing is launched on an error, something that a launch holds otherwise
static void look(const char* what, laser_status s, const std::vector<int>& sizes) {
  bool bad = (s == LASER_OK) != (launch_count() > 0) || (s != LASER_OK && s != LASER_ERR_SHAPE);
  for (int i = 0; i < launch_count(); ++i) {
    const LaunchRecord* r = launch_record(i);
    bad = bad || r->grid == 0 || r->block == 0 || (unsigned long long)r->grid * r->block >= 1ull << 32;
  }
  launch_clear();
  ++(s == LASER_OK ? accepted : refused);
  if (!bad) return;
  ++failures;
  std::printf("%s: status %d, sizes", what, (int)s);
  for (int x : sizes) std::printf(" %d", x);
  std::printf("\n");
}

// `call` with its base sizes, and with one and two of them at every edge
static void edges(const char* what, std::vector<int> base, const std::function<laser_status(const std::vector<int>&)>& call) {
  const int at[] = {INT_MIN, -1, 0, 1, 7, 8, 31, 33, 64, 65, 128, 1024, 4096, 65536, 1 << 20, 1 << 22, 1 << 24, (1 << 30) - 1, 1 << 30, INT_MAX - 65535, INT_MAX};
  look(what, call(base), base);
  for (size_t i = 0; i < base.size(); ++i)
    for (int x : at) {
      std::vector<int> one = base;
      one[i] = x;
      look(what, call(one), one);
      if (i == 0 && x > 1 << 20) continue;   // (so many users go out in up to tens of thousands of launches: once is enough)
      for (size_t j = i + 1; j < base.size(); ++j)
        for (int y : at) {
          std::vector<int> two = one;
          two[j] = y;
          look(what, call(two), two);
        }
    }
}

int main() {
  void* const A = reinterpret_cast<void*>(0x10000);
  int32_t* const I = reinterpret_cast<int32_t*>(0x10000);
  float* const F = reinterpret_cast<float*>(0x10000);
  double* const X = reinterpret_cast<double*>(0x10000);
  for (laser_dtype dt : {LASER_F32, LASER_BF16}) {
    auto pitch = [](int heads, int D) { return (int64_t)heads * D; };
    // T, H, H_kv, D, R
    for (const auto& base : {std::vector<int>{7, 4, 2, 64, 64}, std::vector<int>{70000, 1, 1, 128, 100}, std::vector<int>{1 << 22, 8, 8, 8, 6}})
      for (laser_rotary_layout layout : {LASER_ROTARY_HALF, LASER_ROTARY_INTERLEAVED})
        edges("laser_rotary_forward", base, [&](const std::vector<int>& s) {
          void* const k = s[2] == 0 ? nullptr : A;
          return laser_rotary_forward(A, pitch(s[1], s[3]), k, pitch(s[2], s[3]), I, X, s[0], s[1], s[2], s[3], s[4], layout, 1.0f, dt, A, pitch(s[1], s[3]),
                                      k, pitch(s[2], s[3]), nullptr);
        });
    // U, T, C_max, P, page, block, max_pages, L_max, H, H_kv, D
    const std::vector<int> cached[] = {{3, 9, 3, 100, 16, 8, 20, 300, 8, 2, 64}, {90, 9000, 200, 5000, 64, 32, 64, 4000, 4, 4, 128},
                                       {64, 6400, 100, 5000, 32, 32, 200, 6000, 8, 2, 64}, {70000, 70000, 1, 100000, 8, 8, 9, 70, 2, 1, 32}};
    for (const auto& base : cached) {
      edges("laser_cache8_append", base, [&](const std::vector<int>& s) {
        return laser_cache8_append(A, pitch(s[9], s[10]), A, pitch(s[9], s[10]), A, A, F, F, I, I, I, s[0], s[1], s[2], s[3], s[4], s[5], s[6], s[7], s[9],
                                   s[10], dt, nullptr);
      });
      edges("laser_cache8_attention_forward", base, [&](const std::vector<int>& s) {
        const size_t room = laser_cache8_attention_work_bytes(s[0], s[1], s[2], s[7], s[8], s[9], s[10], dt);
        return laser_cache8_attention_forward(A, pitch(s[8], s[10]), A, A, F, F, I, I, I, s[0], s[1], s[2], s[3], s[4], s[5], s[6], s[7], s[8], s[9], s[10],
                                              1.0f, 1, dt, A, F, A, room, nullptr);
      });
    }
  }
  edges("laser_rotary_frequencies", {64}, [&](const std::vector<int>& s) {
    return laser_rotary_frequencies(s[0], 10000.0, LASER_ROTARY_BASE, 4.0, 0.0, 0.0, 0.0, X, nullptr);
  });
  // U, V, P, page, max_pages, max_pages_out, n_parts
  void* parts[1024];
  int64_t bytes[1024];
  for (int i = 0; i < 1024; ++i) {
    parts[i] = A;
    bytes[i] = i % 3 == 0 ? 4096 : i % 3 == 1 ? 1 << 27 : 13;
  }
  for (const auto& base : {std::vector<int>{3, 5, 100, 16, 20, 30, 2}, std::vector<int>{70000, 100000, 1 << 20, 8, 4, 5, 40}, std::vector<int>{1, 1, 1, 4096, 1, 1, 0}}) {
    edges("laser_pages_fork", base, [&](const std::vector<int>& s) {
      const size_t room = laser_pages_work_bytes(s[0] > s[1] ? s[0] : s[1], s[2]);
      return laser_pages_fork(parts, bytes, s[6], I, I, I, I, s[0], s[1], s[2], s[3], s[4], s[5], I, I, I, A, room, nullptr);
    });
    edges("laser_pages_grow", {base[0], base[2], base[3], base[4]}, [&](const std::vector<int>& s) {
      return laser_pages_grow(I, I, I, I, s[0], s[1], s[2], s[3], I, A, laser_pages_work_bytes(s[0], s[1]), nullptr);
    });
    edges("laser_pages_free", {base[0], base[2], base[3], base[4]}, [&](const std::vector<int>& s) {
      return laser_pages_free(I, I, I, I, s[0], s[1], s[2], s[3], nullptr);
    });
    edges("laser_pages_compact", {base[0], base[2], base[3], base[4], base[6]}, [&](const std::vector<int>& s) {
      return laser_pages_compact(parts, bytes, s[4], I, I, I, s[0], s[1], s[2], s[3], I, I, I, A, laser_pages_work_bytes(s[0], s[1]), nullptr);
    });
    edges("laser_pages_copy", {base[1], base[2], base[6] + 1}, [&](const std::vector<int>& s) {
      return laser_pages_copy(parts, bytes, s[2], I, I, s[0], s[1], nullptr);
    });
  }
  std::printf("%d failure(s), %d calls accepted, %d refused\n", failures, accepted, refused);
  return failures != 0;
}
