// New items into a cache of 8-bit blocks. A block's scale is the smallest power of two with which its largest item fits e4m3's range, so
// items lose nothing but their rounding to 4 significant bits (a power of two moves no bits; against scales of any value it leaves at most one of
// the 18 binades unused). Items that come later may be larger: the scale then grows and the items that are there are encoded anew, exact but for the
// smallest ones, whose last bits fall off.
//
// A workgroup owns a block that new items come into (the first of a user's may hold older ones), for a head's keys or values: largest
// new item, scale, codes. Bound by loads behind one another: offset, length and page, then the rows twice, for the largest and for the codes (the second
// time from the L2 cache): 2.5 us for one item of 5 users, 4.3 of 128, 7.5 for 512 items of 16 (8 MB in and out, 1.6 us at a copy's rate).
#include "cache8.h"

namespace laser {

__device__ __forceinline__ float needed_scale(float largest) {
  const unsigned b = __float_as_uint(largest);
  int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u);
  e = e < LEAST_SCALE ? LEAST_SCALE : e > MOST_SCALE ? MOST_SCALE : e;
  return __uint_as_float((unsigned)(e + 127) << 23);
}
// x, y as e4m3 in the low 16 bits: to nearest, of two equally near the even one, at most +-448 (infinities too), NaN stays
__device__ __forceinline__ unsigned encode2(float x, float y) {
  x = x != x ? x : fminf(fmaxf(x, -E4M3_MAX), E4M3_MAX);
  y = y != y ? y : fminf(fmaxf(y, -E4M3_MAX), E4M3_MAX);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(x, y, 0, false) & 0xffffu;
}

// 8 elements of a row as fp32
__device__ __forceinline__ void load8(const float* p, float* x) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const stream16 w = *reinterpret_cast<const stream16*>(p + i * 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[i * 4 + j] = __uint_as_float(w[j]);
  }
}
__device__ __forceinline__ void load8(const unsigned short* p, float* x) {
  const stream16 w = *reinterpret_cast<const stream16*>(p);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[2 * j] = __uint_as_float(w[j] << 16);
    x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void cache8_append_kernel(const Cache8Args a, MulDiv by_pieces) {
  __shared__ float wave_largest[4];
  const CacheArgs& c = a.c;
  const int u = blockIdx.z, hk = blockIdx.y >> 1, tid = threadIdx.x;
  const bool values = blockIdx.y & 1;
  const CandRange r = cand_range(c.off, u, c.C, c.T);
  const int n = cache_len(c.lens, u, c.L, c.max_pages, c.page_log2), old = n - r.count;   // (below 0: the first rows have no place)
  const int first = old > 0 ? old : 0, block = 1 << a.block_log2;
  const int j0 = (int)((((unsigned)first >> a.block_log2) + blockIdx.x) << a.block_log2);
  const int lo = j0 > first ? j0 : first, hi = n - j0 < block ? n : j0 + block;
  if (lo >= hi) return;
  const int page = c.pages[(size_t)u * c.max_pages + (j0 >> c.page_log2)];
  if ((unsigned)page >= (unsigned)c.P) return;
  const int place = j0 & ((1 << c.page_log2) - 1);
  const size_t head = (size_t)page * c.Hkv + hk;
  unsigned char* to = static_cast<unsigned char*>(values ? c.v : c.k) + ((head << c.page_log2) + place) * c.D;
  float* scale_at = (values ? a.v_scale : a.k_scale) + (head << (c.page_log2 - a.block_log2)) + (place >> a.block_log2);
  const long long pitch = values ? a.vp : a.kp;
  const T* from = static_cast<const T*>(values ? a.v_new : a.k_new) + (size_t)(r.first + lo - old) * pitch + (size_t)hk * c.D;
  const unsigned pieces = c.D / 8, all = (unsigned)(hi - lo) * pieces;

  float largest = 0.0f;
  for (unsigned e = tid; e < all; e += 256) {
    const unsigned i = by_pieces.div(e);
    float x[8];
    load8(from + i * pitch + (e - i * pieces) * 8, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float y = fabsf(x[j]);
      largest = y < INFINITY ? fmaxf(largest, y) : largest;   // (infinities and NaN ask for no scale)
    }
  }
#pragma unroll
  for (int m = 32; m; m >>= 1) largest = fmaxf(largest, __shfl_xor(largest, m));
  if ((tid & 63) == 0) wave_largest[tid >> 6] = largest;
  const float was = j0 < first ? *scale_at : 0.0f;   // (a block without older items has no scale yet)
  __syncthreads();
  largest = fmaxf(fmaxf(wave_largest[0], wave_largest[1]), fmaxf(wave_largest[2], wave_largest[3]));
  const float scale = fmaxf(needed_scale(largest), was), by = 1.0f / scale;
  for (unsigned e = tid; e < all; e += 256) {
    const unsigned i = by_pieces.div(e), piece = e - i * pieces;
    float x[8];
    load8(from + i * pitch + piece * 8, x);
    uint2 w;
    w.x = encode2(x[0] * by, x[1] * by) | encode2(x[2] * by, x[3] * by) << 16;
    w.y = encode2(x[4] * by, x[5] * by) | encode2(x[6] * by, x[7] * by) << 16;
    *reinterpret_cast<uint2*>(to + (size_t)(lo - j0 + i) * c.D + piece * 8) = w;
  }
  if (j0 < first && scale > was) {
    const float less = was * by;
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    for (unsigned e = tid; e < (unsigned)(first - j0) * (c.D / 4); e += 256) {
      unsigned* at = reinterpret_cast<unsigned*>(to) + e;
      const unsigned w = *at;
      const f32x2 x = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), y = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
      *at = encode2(x[0] * less, x[1] * less) | encode2(y[0] * less, y[1] * less) << 16;
    }
  }
  if (tid == 0) *scale_at = scale;
}

laser_status cache8_append_launch(const Cache8Args& a) {
  const CacheArgs& c = a.c;
  const int least = c.C < c.L ? c.C : c.L;
  const long long rows = least < c.T ? least : c.T, blocks = (rows + 2 * (1 << a.block_log2) - 2) >> a.block_log2;   // that a user's rows touch
  // (a launch has fewer than 2^32 threads, and 65535 of a grid's second and third sides)
  const long long most = 0xffffffffLL / 256 / (blocks * c.Hkv * 2);
  if (most <= 0) return LASER_ERR_SHAPE;
  for (long long u = 0; u < c.U;) {
    long long users = c.U - u < most ? c.U - u : most;
    if (users > 65535) users = 65535;
    Cache8Args part = a;
    part.c.off = c.off + u;
    part.c.pages = c.pages + u * c.max_pages;
    part.c.lens = c.lens + u;
    const dim3 grid((unsigned)blocks, c.Hkv * 2, (unsigned)users);
    const MulDiv pieces = mul_div(c.D / 8);
    if (c.dt == LASER_F32) cache8_append_kernel<float><<<grid, 256, 0, c.stream>>>(part, pieces);
    else cache8_append_kernel<unsigned short><<<grid, 256, 0, c.stream>>>(part, pieces);
    const laser_status s = launch_status();
    if (s != LASER_OK) return s;
    u += users;
  }
  return LASER_OK;
}

}  // namespace laser
