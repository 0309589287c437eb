// Rotary positions: pair i of the first R columns of every head is turned by the angle pos * freq[i],
//   (a, b) -> scale (a c - b s, a s + b c),   c, s = cos, sin(pos freq[i]),
// pairs being columns (i, i + R/2) or (2i, 2i + 1); the transpose (s -> -s) carries gradients back. One launch turns queries and keys.
//
// Bound by memory: what is turned comes in and goes out once, in pieces of 16 bytes (201 MB of bf16 rows in 38 us, 5.3 TB/s, what a large
// copy reaches; pairs side by side 42 us; halves that are no whole pieces take up to twice as long). Results are stored for whoever reads them next: with
// the non-temporal hint the launch alone is 0 to 10 us shorter, attention behind it 4 to 8 us longer than that. A workgroup takes a few tokens, makes their cosines
// and sines once for all heads, in LDS, and walks heads and pieces. An angle of a far position is many turns: it is formed in fp64 and
// reduced to an eighth of a turn there (fp32 would be off by 4e-3 at position 65000), then cosine and sine are Taylor sums in fp32.
#include "rotary.h"

#include <type_traits>

namespace laser {

// cos and sin of x radians: the nearest whole number of quarter turns comes off in fp64, the rest is within pi/4, where the first term
// left out is 1e-10 (cos) and 2e-9 of the result (sin)
__device__ __forceinline__ float2 cos_sin(double x) {
  const double quarters = x * 0.63661977236758134308, whole = rint(quarters);
  const float t = (float)((quarters - whole) * 1.57079632679489661923), t2 = t * t;
  const float s = fmaf(t * t2, fmaf(t2, fmaf(t2, fmaf(t2, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6), t);
  const float c = fmaf(t2, fmaf(t2, fmaf(t2, fmaf(t2, fmaf(t2, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
  const int turn = (int)(whole - 4.0 * floor(whole * 0.25));   // 0 .. 3
  const float a = turn & 1 ? s : c, b = turn & 1 ? c : s;
  return float2{turn == 1 || turn == 2 ? -a : a, turn >= 2 ? -b : b};
}

// 16 bytes of a row, at any element (the second halves of pairs start at column R / 2)
template <typename T>
struct Piece {
  static constexpr int N = 16 / sizeof(T);
  typedef unsigned int words __attribute__((ext_vector_type(4), aligned(2)));
  T v[N];
  __device__ __forceinline__ void load(const T* p) { *reinterpret_cast<words*>(v) = *reinterpret_cast<const words*>(p); }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<words*>(p) = *reinterpret_cast<const words*>(v); }
  __device__ __forceinline__ float get(int j) const { return load_as_f32<T>(v, j); }
  __device__ __forceinline__ void set(int j, float x) { store_from_f32<T>(v, j, x); }
};

// The last elements of a row, fewer than a piece: by halves of one, quarters, .., of which `left` has each once or not at all, M elements from
// the element on that the larger ones end at; they stand in a Piece from N - 2 M on
template <typename T, int M, typename Go>
__device__ __forceinline__ void over_rest(int left, const Go& go) {
  if constexpr (M > 0) {
    if (left & M) go(std::integral_constant<int, M>(), left & ~(2 * M - 1));
    over_rest<T, M / 2>(left, go);
  }
}
template <typename T, int M>
struct Some {
  typedef T type __attribute__((ext_vector_type(M), aligned(sizeof(T) < 2 ? 1 : 2)));
  static __device__ __forceinline__ void copy(T* to, const T* from) { *reinterpret_cast<type*>(to) = *reinterpret_cast<const type*>(from); }
};

constexpr int ROTARY_TOKENS = 16;   // of a workgroup, at most

// Cosines and sines of a workgroup's tokens, and which of them have a position
__device__ __forceinline__ void make_turns(const RotaryArgs& a, int t0, int count, const MulDiv& by_half, float2* turn, int* there) {
  const int half = a.R / 2;
  for (unsigned e = threadIdx.x; e < (unsigned)(count * half); e += 256) {
    const int t = (int)by_half.div(e), i = (int)e - t * half, pos = a.pos[t0 + t];
    const float2 cs = cos_sin((double)pos * a.freq[i]);
    turn[t * half + i] = float2{cs.x * a.scale, (a.back ? -cs.y : cs.y) * a.scale};
    if (i == 0) there[t] = pos >= 0;
  }
  __syncthreads();
}

// What a thread has of a head: HALF pairs, a piece of either half; SIDE by side, two pieces in a row. Columns from R on are copied.
// (x and y may be the same rows: a thread reads what it writes, and nobody else does)
template <typename T, bool SIDE>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryArgs a, int tokens, MulDiv by_half, MulDiv by_units, MulDiv by_heads, int units) {
  typedef Piece<T> P;
  constexpr int N = P::N;
  __shared__ float2 turn[ROTARY_TOKENS * 64];
  __shared__ int there[ROTARY_TOKENS];
  const int t0 = blockIdx.x * tokens, count = a.T - t0 < tokens ? a.T - t0 : tokens, half = a.R / 2;
  make_turns(a, t0, count, by_half, turn, there);
  const int heads = a.heads[0] + a.heads[1];
  for (unsigned e = threadIdx.x; e < (unsigned)(count * heads * units); e += 256) {
    const unsigned row = by_units.div(e), unit = e - row * units, t = by_heads.div(row);
    if (!there[t]) continue;
    unsigned head = row - t * heads;
    const int which = head >= (unsigned)a.heads[0];
    head -= which ? a.heads[0] : 0;
    const T* x = static_cast<const T*>(a.x[which]) + (size_t)(t0 + t) * a.xp[which] + head * a.D;
    T* y = static_cast<T*>(a.y[which]) + (size_t)(t0 + t) * a.yp[which] + head * a.D;
    const float2* cs = turn + t * half;
    if constexpr (SIDE) {
      const int c = unit * 2 * N;
      const bool both = c + N < a.D;
      P p[2];
      p[0].load(x + c);
      if (both) p[1].load(x + c + N);
#pragma unroll
      for (int w = 0; w < 2; ++w) {
#pragma unroll
        for (int j = 0; j < N; j += 2) {
          const int i = (c + w * N + j) / 2;
          if (i < half) {
            const float u = p[w].get(j), v = p[w].get(j + 1);
            p[w].set(j, fmaf(u, cs[i].x, -(v * cs[i].y)));
            p[w].set(j + 1, fmaf(u, cs[i].y, v * cs[i].x));
          }
        }
      }
      p[0].store(y + c);
      if (both) p[1].store(y + c + N);
    } else {
      const int c = unit * N, left = half - c;
      if (left >= N) {
        P p, r;
        p.load(x + c);
        r.load(x + half + c);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float u = p.get(j), v = r.get(j), cj = cs[c + j].x, sj = cs[c + j].y;
          p.set(j, fmaf(u, cj, -(v * sj)));
          r.set(j, fmaf(u, sj, v * cj));
        }
        p.store(y + c);
        r.store(y + half + c);
      } else if (left > 0) {   // the last pairs, fewer than a piece
        P p, r;
        over_rest<T, N / 2>(left, [&](auto m, int o) __attribute__((always_inline)) {
          constexpr int M = decltype(m)::value;
          Some<T, M>::copy(p.v + N - 2 * M, x + c + o);
          Some<T, M>::copy(r.v + N - 2 * M, x + half + c + o);
        });
        over_rest<T, N / 2>(left, [&](auto m, int o) __attribute__((always_inline)) {
          constexpr int M = decltype(m)::value;
#pragma unroll
          for (int j = N - 2 * M; j < N - M; ++j) {
            const float2 f = cs[c + o + j - (N - 2 * M)];
            const float u = p.get(j), v = r.get(j);
            p.set(j, fmaf(u, f.x, -(v * f.y)));
            r.set(j, fmaf(u, f.y, v * f.x));
          }
          Some<T, M>::copy(y + c + o, p.v + N - 2 * M);
          Some<T, M>::copy(y + half + c + o, r.v + N - 2 * M);
        });
      } else {                 // columns from R on, where they have to be copied
        const int from = a.R + (int)(unit - (half + N - 1) / N) * N;
        if (from + N <= a.D) {
          P p;
          p.load(x + from);
          p.store(y + from);
        } else {
          P p;
          over_rest<T, N / 2>(a.D - from, [&](auto m, int o) __attribute__((always_inline)) {
            Some<T, decltype(m)::value>::copy(p.v + N - 2 * decltype(m)::value, x + from + o);
          });
          over_rest<T, N / 2>(a.D - from, [&](auto m, int o) __attribute__((always_inline)) {
            Some<T, decltype(m)::value>::copy(y + from + o, p.v + N - 2 * decltype(m)::value);
          });
        }
      }
    }
  }
}

// Halves that are no whole pieces, to other rows than they come from: a thread has a piece of the result, whole and aligned, and reads the
// piece's own columns and the other halves of its pairs, wherever they start. (Bound by requests: 20000 tokens, 10 heads of 128, 100 columns
// turned, 37 us against 39.5 by the kernel above, which is left with rows in place; fp32, 38 of 80, 36 against 49. Whole halves 21.)
template <typename T>
__global__ __launch_bounds__(256) void rotary_apart_kernel(const RotaryArgs a, int tokens, MulDiv by_half, MulDiv by_units, MulDiv by_heads, int units) {
  typedef Piece<T> P;
  constexpr int N = P::N;
  __shared__ float2 turn[ROTARY_TOKENS * 64];
  __shared__ int there[ROTARY_TOKENS];
  const int t0 = blockIdx.x * tokens, count = a.T - t0 < tokens ? a.T - t0 : tokens, half = a.R / 2;
  make_turns(a, t0, count, by_half, turn, there);
  const int heads = a.heads[0] + a.heads[1];
  for (unsigned e = threadIdx.x; e < (unsigned)(count * heads * units); e += 256) {
    const unsigned row = by_units.div(e), unit = e - row * units, t = by_heads.div(row);
    if (!there[t]) continue;
    unsigned head = row - t * heads;
    const int which = head >= (unsigned)a.heads[0], c = unit * N;
    head -= which ? a.heads[0] : 0;
    const T* x = static_cast<const T*>(a.x[which]) + (size_t)(t0 + t) * a.xp[which] + head * a.D;
    T* y = static_cast<T*>(a.y[which]) + (size_t)(t0 + t) * a.yp[which] + head * a.D;
    const float2* cs = turn + t * half;
    P p, r;
    p.load(x + c);
    if (c < a.R) {
      if (c + N <= half) r.load(x + c + half);
      else if (c >= half) r.load(x + c - half);
      else {   // on both sides of the middle
#pragma unroll
        for (int j = 0; j < N; ++j) r.v[j] = x[c + j < half ? c + j + half : c + j < a.R ? c + j - half : c + j];
      }
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int i = c + j;
        if (i < a.R) {
          const float2 f = cs[i < half ? i : i - half];
          const float u = p.get(j), v = r.get(j);
          p.set(j, i < half ? fmaf(u, f.x, -(v * f.y)) : fmaf(v, f.y, u * f.x));
        }
      }
    }
    p.store(y + c);
  }
}

template <typename T, bool SIDE>
static laser_status rotary_typed(const RotaryArgs& a) {
  constexpr int N = Piece<T>::N;
  const int heads = a.heads[0] + a.heads[1], half = a.R / 2;
  // (rows turned in place keep their other columns: those pieces are left out. A tensor in place beside one that is not copies onto itself.)
  const bool in_place = a.y[0] == a.x[0] && a.y[1] == a.x[1];
  const bool apart = !SIDE && half % N != 0 && (a.x[0] == nullptr || a.y[0] != a.x[0]) && (a.x[1] == nullptr || a.y[1] != a.x[1]);
  const int units = apart ? a.D / N : SIDE ? ((in_place ? a.R : a.D) + 2 * N - 1) / (2 * N) : (half + N - 1) / N + (in_place ? 0 : (a.D - a.R + N - 1) / N);
  // Tokens that give each thread a piece or two, and a few workgroups for each compute unit (39322 tokens of 10 heads of 128, 80 threads
  // each: by 16 tokens 42.6 us, by 4 38.2; 100000 of 2 heads, 16 threads each: by 16 24.6, by 4 26.2)
  int tokens = (320 + heads * units - 1) / (heads * units);
  tokens = tokens < a.T / 2048 ? tokens : a.T / 2048;
  tokens = tokens < 1 ? 1 : tokens > ROTARY_TOKENS ? ROTARY_TOKENS : tokens;
  const unsigned grid = (unsigned)((a.T + (long long)tokens - 1) / tokens);
  // (a launch has fewer than 2^32 threads: 2^24 workgroups and more go out in several)
  constexpr unsigned MOST = 0xffffff;
  for (unsigned b = 0; b < grid; b += MOST) {
    RotaryArgs part = a;
    const long long t0 = (long long)b * tokens;
    for (int w = 0; w < 2; ++w) {
      if (a.x[w] == nullptr) continue;
      part.x[w] = static_cast<const T*>(a.x[w]) + t0 * a.xp[w];
      part.y[w] = static_cast<T*>(a.y[w]) + t0 * a.yp[w];
    }
    part.pos = a.pos + t0;
    const unsigned here = grid - b < MOST ? grid - b : MOST;
    part.T = b + here < grid ? (int)((long long)here * tokens) : (int)(a.T - t0);
    if (apart) rotary_apart_kernel<T><<<here, 256, 0, a.stream>>>(part, tokens, mul_div(half), mul_div(units), mul_div(heads), units);
    else rotary_kernel<T, SIDE><<<here, 256, 0, a.stream>>>(part, tokens, mul_div(half), mul_div(units), mul_div(heads), units);
    const laser_status s = launch_status();
    if (s != LASER_OK) return s;
  }
  return LASER_OK;
}

laser_status rotary_launch(const RotaryArgs& a) {
  if (a.dt == LASER_F32) return a.interleaved ? rotary_typed<float, true>(a) : rotary_typed<float, false>(a);
  return a.interleaved ? rotary_typed<unsigned short, true>(a) : rotary_typed<unsigned short, false>(a);
}

// freq[i] = base^(-2i/R), for longer contexts than those of training stretched one way or another
__global__ __launch_bounds__(64) void rotary_frequencies_kernel(const RotaryFrequencies a) {
  const int i = threadIdx.x;
  if (i >= a.R / 2) return;
  double base = a.base;
  // (the slowest pair is stretched by the factor, the fastest not at all; a single pair is both, and stays)
  if (a.scaling == LASER_ROTARY_BASE && a.R > 2) base *= pow(a.factor, (double)a.R / (a.R - 2));
  double f = pow(base, -2.0 * i / a.R);
  if (a.scaling == LASER_ROTARY_LINEAR) f /= a.factor;
  if (a.scaling == LASER_ROTARY_PARTS) {   // by the turns that a pair makes within the length of training
    const double share = (a.length * f * 0.15915494309189533577 - a.low) / (a.high - a.low);
    const double kept = share < 0.0 ? 0.0 : share > 1.0 ? 1.0 : share;
    f *= kept + (1.0 - kept) / a.factor;
  }
  a.freq[i] = f;
}

laser_status rotary_frequencies_launch(const RotaryFrequencies& a) {
  rotary_frequencies_kernel<<<1, 64, 0, a.stream>>>(a);
  return launch_status();
}

}  // namespace laser
