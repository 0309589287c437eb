// Host-side check of the entry points for attention among a history's items under AddressSanitizer and UndefinedBehaviorSanitizer (no
// GPU needed): every size at the edges of int and of its documented limits, alone and in pairs, through validation, the choice of forms and
// the launchers, whose launches are recorded (launch_recorder.cpp). Pointers are never dereferenced on the host. Built by
// paper_2602_11562_amd.build.build_history_host_check(), run by tests/test_history_host_cpu.py. Exit status 0: every call returned what its
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
  for (laser_dtype dt : {LASER_F32, LASER_BF16}) {
    auto pitch = [](int heads, int D) { return (int64_t)heads * D; };
    // N, T, L_max, H, H_kv, D
    const std::vector<int> packed[] = {{3, 500, 200, 4, 2, 64}, {2000, 70000, 90, 8, 8, 128}, {70000, 100000, 5000, 2, 1, 32}};
    for (const auto& base : packed) {
      edges("laser_history_attention_forward", base, [&](const std::vector<int>& s) {
        return laser_history_attention_forward(A, pitch(s[3], s[5]), A, pitch(s[4], s[5]), A, pitch(s[4], s[5]), I, s[0], s[1], s[2], s[3], s[4], s[5], 1.0f,
                                               dt, A, F, nullptr);
      });
      edges("laser_history_attention_backward", base, [&](const std::vector<int>& s) {
        const size_t room = laser_history_attention_backward_work_bytes(s[0], s[1], s[2], s[3], s[4], s[5], dt);
        const int64_t q = pitch(s[3], s[5]), k = pitch(s[4], s[5]);
        return laser_history_attention_backward(A, q, A, k, A, k, A, F, A, I, s[0], s[1], s[2], s[3], s[4], s[5], 1.0f, dt, A, q, A, k, A, k, A, room, nullptr);
      });
    }
    // U, T, C_max, P, page, max_pages, L_max, H, H_kv, D
    const std::vector<int> cached[] = {{3, 9, 3, 100, 16, 20, 300, 8, 2, 64}, {90, 9000, 200, 5000, 64, 64, 4000, 4, 4, 128},
                                       {70000, 70000, 1, 100000, 8, 9, 70, 2, 1, 32}};
    for (const auto& base : cached) {
      edges("laser_cache_append", base, [&](const std::vector<int>& s) {
        return laser_cache_append(A, pitch(s[8], s[9]), A, pitch(s[8], s[9]), A, A, I, I, I, s[0], s[1], s[2], s[3], s[4], s[5], s[6], s[8], s[9], dt, F, nullptr);
      });
      edges("laser_cache_attention_forward", base, [&](const std::vector<int>& s) {
        const size_t room = laser_cache_attention_work_bytes(s[0], s[1], s[2], s[6], s[7], s[8], s[9], dt);
        return laser_cache_attention_forward(A, pitch(s[7], s[9]), A, A, I, I, I, s[0], s[1], s[2], s[3], s[4], s[5], s[6], s[7], s[8], s[9], 1.0f, 1, dt, A, F,
                                             A, room, nullptr);
      });
      edges("laser_cache_weights", base, [&](const std::vector<int>& s) {
        return laser_cache_weights(A, pitch(s[7], s[9]), F, A, I, I, I, s[0], s[1], s[2], s[3], s[4], s[5], s[6], s[7], s[8], s[9], 1.0f, 0, 1, dt, F, nullptr);
      });
    }
    // U, P, page, max_pages, max_pages_out, L_max, budget, recent, H_kv, D
    const std::vector<int> evicted[] = {{3, 100, 16, 20, 10, 300, 100, 20, 2, 64}, {70000, 900000, 8, 9, 9, 70, 1, 0, 1, 32}};
    for (const auto& base : evicted)
      edges("laser_cache_evict", base, [&](const std::vector<int>& s) {
        return laser_cache_evict(A, A, F, I, I, I, s[0], s[1], s[2], s[3], s[4], s[5], s[6], s[7], s[8], s[9], dt, I, I, nullptr);
      });
  }
  std::printf("history_host_check: %d failure(s), %d calls accepted, %d refused\n", failures, accepted, refused);
  return failures == 0 ? 0 : 1;
}
