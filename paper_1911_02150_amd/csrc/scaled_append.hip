// New rows into paged caches of 8 bits.
//
// A block of `block` positions and a head has one scale for K and one for V.  Of a block that gets rows, with a the largest finite |x| of its new rows and Q the
// type's largest number: s' = the smallest power of two >= 2^-126 with a <= Q s'; its scale becomes s' where its first row is new, else max(s_old, s'), and the
// rows that it had are rounded again, from q to round(q s_old / s), where that is more than s_old.  (Powers of two: the quotients are exact, so that rounding them again and again is off by less
// than a step, and e4m3, whose steps go by the number's own size, loses nothing over other scales; int8 loses half a bit on average.)
#include "paged.hpp"
#include "scaled.hpp"

namespace mqa {
namespace {

__device__ __forceinline__ float finite_size(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.f;
}

constexpr int kHeld = 8;

// A unit, (sequence, one of the blocks that its new rows reach, head, K or V), is THREADS threads' work: 64, 256 or 1024.  Its rows are one run of
// memory in the pool, and h_kv apart in the new rows.  HBM bounds it, five bytes a value (64 prompts of 640, two widths of 128, 52 MB: 13 us = 4.0 TB/s in blocks of 16 or 64), and for a token each the launch
// and three reads in a row: length, entry, scale (128 sequences: 3.7 us).
template <bool E4M3, int THREADS>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS)
void scaled_append_kernel(ScaledAppend p, int reach) {
  constexpr int WAVES = THREADS / 64, GROUP = THREADS < 256 ? 256 : THREADS;
  __shared__ float s_most[WAVES];
  const PagedCache& c = p.a.c;
  const int lane = threadIdx.x % THREADS;
  unsigned unit = blockIdx.x * (unsigned)(GROUP / THREADS) + threadIdx.x / THREADS;
  if (unit >= (unsigned)p.a.b * reach * c.h_kv * 2) return;
  const bool is_v = unit & 1;
  unit >>= 1;
  const int e = (int)(unit % (unsigned)c.h_kv);
  unit /= (unsigned)c.h_kv;
  const int turn = (int)(unit % (unsigned)reach), i = (int)(unit / (unsigned)reach);
  const int L = p.a.lens_in[i];
  const int count = p.a.counts ? min(max(p.a.counts[i], 0), p.a.n) : p.a.n;
  const bool fits = L >= 0 && L <= c.positions() - count;
  if (lane == 0 && turn == 0 && e == 0 && !is_v) p.a.lens_out[i] = fits ? L + count : L;
  if (!fits) return;
  const int first = (L / p.block + turn) * p.block;              // the block's first position, and its rows that are new
  const int begin = max(first, L), end = min(first + p.block, L + count);
  if (begin >= end) return;
  const int w4 = (is_v ? c.v : c.k) >> 2;
  const float4* const fresh = reinterpret_cast<const float4*>(is_v ? p.a.v_new : p.a.k_new) + (((size_t)i * p.a.n + (begin - L)) * c.h_kv + e) * w4;
  const int older = (begin - first) * w4, all = (end - begin) * w4;
  const int step = (c.h_kv - 1) * w4;                            // from one row's end to the next one's beginning
  const bool power4 = (w4 & (w4 - 1)) == 0;
  const int shift = __builtin_ctz(w4);
  auto new4 = [&](int x) { return fresh[x + (step == 0 ? 0 : (power4 ? x >> shift : x / w4) * step)]; };
  auto most_of = [](float most, const float4& y) {
    return fmaxf(most, fmaxf(fmaxf(finite_size(y.x), finite_size(y.y)), fmaxf(finite_size(y.z), finite_size(y.w))));
  };
  // A thread's first kHeld fours stay in registers; a block that has more of them is read twice (64 prompts of 100 to 1000, 42 MB: all of them twice 17.5 us, once 11.6).
  float4 mine[kHeld];
#pragma unroll
  for (int u = 0; u < kHeld; ++u) mine[u] = new4(min(lane + u * THREADS, all - 1));
  const int row = paged_row(c, c.table + (size_t)i * c.max_pages, e, first);
  if (row < 0) return;
  float* const scale_at = (is_v ? p.V_scales : p.K_scales) + row / p.block;
  uint32_t* const held = static_cast<uint32_t*>(is_v ? c.V : c.K) + (size_t)row * w4;
  const float had = older > 0 ? *scale_at : 0.f;
  float most = 0.f;
#pragma unroll
  for (int u = 0; u < kHeld; ++u) most = most_of(most, mine[u]);
  for (int x = lane + kHeld * THREADS; x < all; x += THREADS) most = most_of(most, new4(x));
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) most = fmaxf(most, __shfl_xor(most, off));
  if constexpr (WAVES > 1) {
    if ((lane & 63) == 0) s_most[lane >> 6] = most;
    __syncthreads();                                             // (and every wave has read the scale)
#pragma unroll
    for (int w = 0; w < WAVES; ++w) most = fmaxf(most, s_most[w]);
  }
  float s = scale_of<E4M3>(most);
  if (had > s) s = had;                                          // (a scale that is no number gives way)
  const bool power = (__float_as_uint(s) & 0x007fffffu) == 0 && s >= 0x1p-126f && s <= 0x1p126f;
  const float inv = power ? inverse_of(s) : 0.f;
  if (older > 0 && s != had) {
    const float ratio = had / s;
    for (int x = lane; x < older; x += THREADS) {
      float4 y = values4<E4M3>(held[x]);
      y.x *= ratio; y.y *= ratio; y.z *= ratio; y.w *= ratio;
      held[x] = round4<E4M3>(y);
    }
  }
  auto put = [&](int x, float4 y) {
    if (power) { y.x *= inv; y.y *= inv; y.z *= inv; y.w *= inv; }
    else { y.x /= s; y.y /= s; y.z /= s; y.w /= s; }             // (a scale that the caller has written)
    held[older + x] = round4<E4M3>(y);
  };
#pragma unroll
  for (int u = 0; u < kHeld; ++u)
    if (lane + u * THREADS < all) put(lane + u * THREADS, mine[u]);
  for (int x = lane + kHeld * THREADS; x < all; x += THREADS) put(x, new4(x));
  if (lane == 0 && (older == 0 || s != had)) *scale_at = s;
}

}  // namespace

// As few threads as hold a unit's values, 32 each, in registers.  64 prompts of 640, two widths of 128, 64 / 256 / 1024 threads: blocks of 8 14.7 / 30.8 / 85.8 us, 16 13.0 / 18.6 / 47.6,
// 32 16.7 / 14.2 / 28.3, 64 28.1 / 13.1 / 18.4, 128 51 / 16.6 / 15.1, 256 96 / 29 / 16.7; one prompt in blocks of 16 4.3 / 3.7 / 4.8, of 256 53 / 14.9 / 6.5; 128 tokens 3.7 / 3.8 / 5.1.
template <bool E4M3>
static void launch_units(const ScaledAppend& p, int reach, unsigned units, long long values, hipStream_t st) {
  // (grids of less than 2^32 threads)
  if (values > 256 * 4 * kHeld && units < 1u << 22) hipLaunchKernelGGL((scaled_append_kernel<E4M3, 1024>), dim3(units), dim3(1024), 0, st, p, reach);
  else if (values > 64 * 4 * kHeld && units < 1u << 24) hipLaunchKernelGGL((scaled_append_kernel<E4M3, 256>), dim3(units), dim3(256), 0, st, p, reach);
  else hipLaunchKernelGGL((scaled_append_kernel<E4M3, 64>), dim3((units + 3) / 4), dim3(256), 0, st, p, reach);
}

hipError_t launch_scaled_append(const ScaledAppend& p, int is_e4m3, hipStream_t st) {
  const int reach = (p.a.n + p.block - 2) / p.block + 1;         // blocks that n rows reach, at most
  const unsigned units = (unsigned)p.a.b * reach * p.a.c.h_kv * 2;
  const int wide = p.a.c.k > p.a.c.v ? p.a.c.k : p.a.c.v;
  const long long values = (long long)(p.block < p.a.n ? p.block : p.a.n) * wide;
  if (is_e4m3) launch_units<true>(p, reach, units, values, st);
  else launch_units<false>(p, reach, units, values, st);
  return hipGetLastError();
}

}  // namespace mqa
