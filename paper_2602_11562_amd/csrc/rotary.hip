// Rotary positions: pair i of the first R columns of every head is turned by the angle pos * freq[i],
//   (a, b) -> scale (a c - b s, a s + b c),   c, s = cos, sin(pos freq[i]),
// pairs being columns (i, i + R/2) or (2i, 2i + 1); the transpose (s -> -s) carries gradients back. One launch turns queries and keys.
//
// Bound by memory: what is turned comes in and goes out once, in pieces of 16 bytes. A workgroup takes a few tokens, makes their cosines
// and sines once for all heads, in LDS, and walks heads and pieces. An angle of a far position is many turns: it is formed in fp64 and
// reduced to an eighth of a turn there (fp32 would be off by 4e-3 at position 65000), then cosine and sine are Taylor sums in fp32.
#include "rotary.h"

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

template <typename T, int N> struct Piece { T v[N]; };
template <typename T, int N>
__device__ __forceinline__ Piece<T, N> load_piece(const T* p) {
  Piece<T, N> x;
  if constexpr (sizeof(T) * N == 16) *reinterpret_cast<stream16*>(&x) = *reinterpret_cast<const stream16*>(p);
  else if constexpr (sizeof(T) * N == 8) *reinterpret_cast<uint2*>(&x) = *reinterpret_cast<const uint2*>(p);
  else if constexpr (sizeof(T) * N == 4) *reinterpret_cast<unsigned*>(&x) = *reinterpret_cast<const unsigned*>(p);
  else x.v[0] = *p;
  return x;
}
template <typename T, int N>
__device__ __forceinline__ void store_piece(T* p, const Piece<T, N>& x) {
  if constexpr (sizeof(T) * N == 16) *reinterpret_cast<stream16*>(p) = *reinterpret_cast<const stream16*>(&x);
  else if constexpr (sizeof(T) * N == 8) *reinterpret_cast<uint2*>(p) = *reinterpret_cast<const uint2*>(&x);
  else if constexpr (sizeof(T) * N == 4) *reinterpret_cast<unsigned*>(p) = *reinterpret_cast<const unsigned*>(&x);
  else *p = x.v[0];
}

constexpr int ROTARY_TOKENS = 16;   // of a workgroup, at most

// N: elements of a piece. Pairs of halves: the largest power of two that divides R / 2, at most 16 bytes, so that both pieces of a
// pair are whole; columns from R on are then whole pieces too. Pairs side by side: always 16 bytes.
// (x and y may be the same rows: a thread reads what it writes, and nobody else does)
template <typename T, int N, bool SIDE>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryArgs a, int tokens, MulDiv by_half, MulDiv by_units, MulDiv by_heads, int units) {
  __shared__ float2 turn[ROTARY_TOKENS * 64];
  __shared__ int there[ROTARY_TOKENS];
  const int t0 = blockIdx.x * tokens, count = a.T - t0 < tokens ? a.T - t0 : tokens, half = a.R / 2;
  for (unsigned e = threadIdx.x; e < (unsigned)(count * half); e += 256) {
    const int t = (int)by_half.div(e), i = (int)e - t * half, pos = a.pos[t0 + t];
    float2 cs = cos_sin((double)pos * a.freq[i]);
    turn[t * half + i] = float2{cs.x * a.scale, (a.back ? -cs.y : cs.y) * a.scale};
    if (i == 0) there[t] = pos >= 0;
  }
  __syncthreads();
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
      Piece<T, N> p = load_piece<T, N>(x + unit * N);
#pragma unroll
      for (int j = 0; j < N; j += 2) {
        const int i = unit * (N / 2) + j / 2;
        if (i < half) {
          const float u = load_as_f32<T>(p.v, j), v = load_as_f32<T>(p.v, j + 1);
          store_from_f32<T>(p.v, j, fmaf(u, cs[i].x, -(v * cs[i].y)));
          store_from_f32<T>(p.v, j + 1, fmaf(u, cs[i].y, v * cs[i].x));
        }
      }
      store_piece<T, N>(y + unit * N, p);
    } else {
      const int c = unit * N;
      if (c < half) {
        Piece<T, N> p = load_piece<T, N>(x + c), r = load_piece<T, N>(x + half + c);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float u = load_as_f32<T>(p.v, j), v = load_as_f32<T>(r.v, j), cj = cs[c + j].x, sj = cs[c + j].y;
          store_from_f32<T>(p.v, j, fmaf(u, cj, -(v * sj)));
          store_from_f32<T>(r.v, j, fmaf(u, sj, v * cj));
        }
        store_piece<T, N>(y + c, p);
        store_piece<T, N>(y + half + c, r);
      } else {   // columns from R on, where they have to be copied
        store_piece<T, N>(y + half + c, load_piece<T, N>(x + half + c));
      }
    }
  }
}

template <typename T, int N, bool SIDE>
static laser_status rotary_typed(const RotaryArgs& a) {
  const int heads = a.heads[0] + a.heads[1], half = a.R / 2;
  // (rows turned in place keep their other columns: those pieces are left out. A tensor in place beside one that is not copies onto itself.)
  const bool in_place = a.y[0] == a.x[0] && a.y[1] == a.x[1];
  const int units = SIDE ? ((in_place ? a.R : a.D) + N - 1) / N : (in_place ? half : a.D - half) / N;
  int tokens = a.T / 2048;   // (a few workgroups for each compute unit)
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
    part.T = (int)(a.T - t0);
    const unsigned here = grid - b < MOST ? grid - b : MOST;
    if (b + here < grid) part.T = (int)((long long)here * tokens);
    rotary_kernel<T, N, SIDE><<<here, 256, 0, a.stream>>>(part, tokens, mul_div(half), mul_div(units), mul_div(heads), units);
    const laser_status s = launch_status();
    if (s != LASER_OK) return s;
  }
  return LASER_OK;
}

template <typename T>
static laser_status rotary_width(const RotaryArgs& a) {
  constexpr int MOST = 16 / sizeof(T);
  if (a.interleaved) return rotary_typed<T, MOST, true>(a);
  const int half = a.R / 2;
  if (half % MOST == 0) return rotary_typed<T, MOST, false>(a);
  if constexpr (MOST == 8) {
    if (half % 4 == 0) return rotary_typed<T, 4, false>(a);
  }
  return half % 2 == 0 ? rotary_typed<T, 2, false>(a) : rotary_typed<T, 1, false>(a);
}

laser_status rotary_launch(const RotaryArgs& a) {
  return a.dt == LASER_F32 ? rotary_width<float>(a) : rotary_width<unsigned short>(a);
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
