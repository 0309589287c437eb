// What the items of a cache receive from rows that attended to them (bf16, on the matrix cores): weight_j = sum over rows r and heads
// of exp2(c q_r . k_j - lse_r).
//
// A wave owns 32 items; for each key-value head their keys are loaded once, straight into registers as the A operand, and the rows of the
// head's group pass through LDS in tiles of 64 that the workgroup's four waves share:
//   Sc^T[item, row] = K Q^T,  then exp2 and a sum for every accumulator (an item), over the lanes only at the end.
// For few rows this reads the keys and little else: 128 users of up to 4096 items, 8 heads of 128 over 2, one row each 22 us for 65 MB
// (2.9 TB/s; a wave's keys of one head wait for each other). For a chunk it costs half of the attention's products and its exponentials:
// 512 rows for 16 users of up to 10000 items 130 us, where the attention takes 240; the matrix cores are busy 30 % of the time.
#include <type_traits>

#include "history_tile.h"

namespace laser {

template <int DP>
__global__ __launch_bounds__(256, 2) void cache_weights_kernel(const CacheArgs a, int G, MulDiv by_group, float scale) {
  using Sh = TileShape<DP>;
  constexpr int KS = DP / 16, NW = 4, GPW = (Sh::GROUPS + NW - 1) / NW, STAGE = Sh::BYTES + 1024;
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * STAGE];
  const unsigned lds = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem);
  const int u = blockIdx.y;   // (users are turned against each other: their first items are not all one die's)
  const CandRange cr = cand_range(a.off, u, a.C, a.T);
  const int n = cache_len(a.lens, u, a.L, a.max_pages, a.page_log2), item0 = (int)((blockIdx.x + u) % gridDim.x) * NW * 32;
  if (item0 >= n) return;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, h = lane >> 5;
  const int rows = cr.count * G, first = item0 + wave * 32;
  const unsigned short* q = static_cast<const unsigned short*>(a.q);
  const unsigned short* k = static_cast<const unsigned short*>(a.k);

  int j = first + l32;
  const bool inside = j < n;
  j = inside ? j : n - 1;
  const int page = a.pages[(size_t)u * a.max_pages + (j >> a.page_log2)];
  const bool there = (unsigned)page < (unsigned)a.P;
  const int place = j & ((1 << a.page_log2) - 1);
  const size_t slot = there ? (size_t)page : 0;
  // the first row that sees the lane's item, and the wave's first and last of these
  int from = a.causal ? (j - (n - cr.count)) * G : 0;
  from = from < 0 ? 0 : from;
  const int wave_from = __builtin_amdgcn_readlane(from, 0), wave_to = __builtin_amdgcn_readlane(from, 31);
  int start = a.causal ? (item0 - (n - cr.count)) * G : 0;
  start = start < 0 ? 0 : start / TI * TI;
  const int tiles = rows > start ? (rows - start + TI - 1) / TI : 0;   // of each key-value head

  // (offsets as in history_backward.hip: the same in every tile of whole tokens)
  const bool whole_tokens = TI % G == 0;
  unsigned qoff[GPW], zoff;
  auto offsets = [&](int r0, int i0) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < GPW; ++x) {
      const int in = (wave + x * NW) * Sh::RPI + lane / Sh::CH, c = (lane % Sh::CH) ^ tile_swz<Sh::CH>(in), r = r0 + in;
      const int i = (int)by_group.div(r), head = r - i * G;
      qoff[x] = c * 8 < a.D ? (unsigned)(((i - i0) * (int)a.qp + head * a.D + c * 8) * 2) : NO_COLUMN;
    }
    const int r = r0 + lane, i = (int)by_group.div(r);
    zoff = (unsigned)((i - i0) * a.H + r - i * G) * 4;
  };
  if (whole_tokens) offsets(0, 0);
  auto fetch = [&](int hk, int r0, unsigned at) __attribute__((always_inline)) {
    const int i0 = (int)by_group.div(r0);
    if (!whole_tokens) offsets(r0, i0);
    const size_t tok = (size_t)cr.first + i0, head0 = (size_t)hk * G;
    const int more = cr.count - 1 - i0 < TI ? cr.count - 1 - i0 : TI;   // whole tokens within reach behind the first
    const u32x4 qb = buffer_of(q + tok * a.qp + head0 * a.D, (unsigned)((more * (int)a.qp + G * a.D) * 2));
#pragma unroll
    for (int x = 0; x < GPW; ++x) {
      const int g = wave + x * NW;
      if (Sh::GROUPS % NW != 0 && g >= Sh::GROUPS) break;
      buffer_to_lds16(qb, qoff[x], at + g * 1024);
    }
    if (wave == 0) buffer_to_lds4(buffer_of(a.lse + tok * a.H + head0, (unsigned)(more * a.H + G) * 4), zoff, at + Sh::BYTES);
  };
  TileReader<DP> read(lane);
  const f32x16 zero = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  bf16x8 kreg[KS];
  // Sc^T[item, row] = K Q^T: rows in lanes, so a row's lse is one register and the items' sums stay apart until the end
  f32x16 sums = zero;
  const int wave_item = first - (n - cr.count);   // (causal: row r sees item j of the wave if r / G >= wave_item + j)
  auto step = [&](int r0, unsigned at, auto masked) __attribute__((always_inline)) {
    read.place_rows(at);
#pragma unroll
    for (int rb = 0; rb < 2; ++rb) {
      if (decltype(masked)::value && (r0 + rb * 32 >= rows || r0 + rb * 32 + 32 <= wave_from)) continue;
      const float z = *reinterpret_cast<const __attribute__((address_space(3))) float*>(lds_at(at + Sh::BYTES + (rb * 32 + l32) * 4)) * LOG2E;
      f32x16 sc;
#pragma unroll
      for (int s = 0; s < KS; ++s) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kreg[s], read.rows(0, rb, s), s == 0 ? zero : sc, 0, 0, 0);
      const int r = r0 + rb * 32 + l32, seen = a.causal ? (int)by_group.div(r) - wave_item - 4 * h : 32;
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const float p = __builtin_amdgcn_exp2f(fmaf(sc[x], scale, -z));
        if (decltype(masked)::value && (r >= rows || 8 * (x >> 2) + (x & 3) > seen)) continue;
        sums[x] += p;
      }
    }
  };

  if (tiles > 0) {
    fetch(0, start, lds);
    unsigned at = lds, other = lds + STAGE;
    for (int hk = 0; hk < a.Hkv; ++hk) {
      const unsigned short* kr = k + ((((slot * a.Hkv + hk) << a.page_log2) + place) * (size_t)a.D);
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        u32x4 raw = {0u, 0u, 0u, 0u};
        if (s * 16 + h * 8 < a.D) raw = *reinterpret_cast<const u32x4*>(kr + s * 16 + h * 8);
        kreg[s] = __builtin_bit_cast(bf16x8, raw);
      }
      for (int r0 = start; r0 < rows; r0 += TI) {
        __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
        barrier_lds();
        if (r0 + TI < rows) fetch(hk, r0 + TI, other);
        else if (hk + 1 < a.Hkv) fetch(hk + 1, start, other);
        if (first < n && r0 + TI > wave_from) {
          if (r0 >= wave_to && r0 + TI <= rows) step(r0, at, std::false_type{});
          else step(r0, at, std::true_type{});
        }
        const unsigned x = at;
        at = other;
        other = x;
      }
    }
  }
  // over the 32 lanes of a half: with every step a lane keeps half of its items, at last lane l the sum of accumulator l / 2
#pragma unroll
  for (int step = 16, left = 8; step > 1; step >>= 1, left >>= 1)
#pragma unroll
    for (int x = 0; x < 8; ++x)
      if (x < left) {
        const float keep = l32 & step ? sums[x + left] : sums[x], give = l32 & step ? sums[x] : sums[x + left];
        sums[x] = keep + __shfl_xor(give, step);
      }
  sums[0] += __shfl_xor(sums[0], 1);
  const float sum = __shfl(sums[0], ((l32 >> 2) & 1) * 32 + 2 * ((l32 >> 3) * 4 + (l32 & 3)));   // to the lane that has the item
  if (h == 0 && inside && there) {
    float* w = a.weight + (slot << a.page_log2) + place;
    if (a.add) unsafeAtomicAdd(w, sum);
    else *w = sum;
  }
}

template <int DP>
static laser_status weights_typed(const CacheArgs& a) {
  const int G = a.H / a.Hkv;
  for (long long u = 0; u < a.U; u += 65535) {
    CacheArgs part = a;
    part.off = a.off + u;
    part.lens = a.lens + u;
    part.pages = a.pages + (size_t)u * a.max_pages;
    cache_weights_kernel<DP><<<dim3((a.L + 127) / 128, a.U - u < 65535 ? a.U - u : 65535), 256, 0, a.stream>>>(part, G, mul_div(G),
                                                                                                              LOG2E / a.gamma);
  }
  return launch_status();
}
laser_status cache_weights_tile_launch(const CacheArgs& a) {
  if (a.D > 64) return weights_typed<128>(a);
  if (a.D > 32) return weights_typed<64>(a);
  return weights_typed<32>(a);
}

}  // namespace laser
