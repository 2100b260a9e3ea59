// New rows into a paged cache, and the eviction of rows from one.
#include "paged.hpp"

namespace mqa {
namespace {

// Eight neighbouring values of a new row a thread: two 16-byte loads, one store of 16 (bf16) or two (float32).  What bounds a step's rows is the chain
// length -> table -> store behind the launch; of prompts, HBM.
__device__ __forceinline__ void store8(uint16_t* at, const float4& a, const float4& b) {
  uint4 w;
  w.x = pack_bf16_pair(a.x, a.y); w.y = pack_bf16_pair(a.z, a.w);
  w.z = pack_bf16_pair(b.x, b.y); w.w = pack_bf16_pair(b.z, b.w);
  *reinterpret_cast<uint4*>(at) = w;
}
__device__ __forceinline__ void store8(float* at, const float4& a, const float4& b) {
  reinterpret_cast<float4*>(at)[0] = a;
  reinterpret_cast<float4*>(at)[1] = b;
}

template <typename T>
__global__ __launch_bounds__(256)
void paged_append_kernel(PagedAppend p) {
  const int k8 = p.c.k >> 3, w8 = k8 + (p.c.v >> 3);              // eights of a K row, and of both rows
  const size_t idx = (size_t)blockIdx.x * 256 + threadIdx.x;
  const size_t line = idx / w8;                                   // (sequence, new row, head)
  const int c8 = (int)(idx - line * w8);
  const size_t row = line / p.c.h_kv;
  if (row >= (size_t)p.b * p.n) return;
  const int e = (int)(line - row * p.c.h_kv), i = (int)(row / p.n), r = (int)(row - (size_t)i * p.n);
  const bool is_v = c8 >= k8;
  const float* src = is_v ? p.v_new + line * p.c.v + 8 * (c8 - k8) : p.k_new + line * p.c.k + 8 * c8;
  const int L = p.lens_in[i];
  const int count = p.counts ? min(max(p.counts[i], 0), p.n) : p.n;
  const bool fits = L >= 0 && L <= p.c.positions() - count;
  if (r == 0 && e == 0 && c8 == 0) p.lens_out[i] = fits ? L + count : L;
  if (!fits || r >= count) return;
  const float4 a = reinterpret_cast<const float4*>(src)[0], b = reinterpret_cast<const float4*>(src)[1];
  const int at = paged_row(p.c, p.c.table + (size_t)i * p.c.max_pages, e, L + r);
  if (at < 0) return;
  T* dst = is_v ? static_cast<T*>(p.c.V) + (size_t)at * p.c.v + 8 * (c8 - k8) : static_cast<T*>(p.c.K) + (size_t)at * p.c.k + 8 * c8;
  store8(dst, a, b);
}

// ---------------------------------------------------------------- eviction
// Scores as integers in the same order: the larger the score the larger its key; -0 as 0, NaN as -inf (0 is no score's key).
__device__ __forceinline__ uint32_t score_key(float x) {
  if (x != x) x = -INFINITY;
  if (x == 0.f) x = 0.f;
  const uint32_t u = __float_as_uint(x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int kSelectThreads = 1024;
constexpr int kBins = 2048;

// Sum of x over the workgroup's threads before this one; *total: over all.
__device__ __forceinline__ int before_me(int x, int* waves, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int incl = x;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int y = __shfl_up(incl, off);
    if (lane >= off) incl += y;
  }
  __syncthreads();
  if (lane == 63) waves[wave] = incl;
  __syncthreads();
  int before = 0, all = 0;
  for (int w = 0; w < kSelectThreads / 64; ++w) {
    if (w < wave) before += waves[w];
    all += waves[w];
  }
  *total = all;
  return before + incl - x;
}

// Which positions of (sequence, head) stay: the latest `recent`, and of the older ones the largest scores up to the budget, the lower position among
// equals.  A radix selection over the keys, 11 + 11 + 10 bits from the top: a histogram of the keys that agree with the threshold so far, and the bin in
// which the wanted rank lies.  One workgroup per (sequence, head).
__global__ __launch_bounds__(kSelectThreads)
void evict_select_kernel(PagedEvict p) {
  __shared__ int bins[kBins];
  __shared__ int waves[kSelectThreads / 64];
  __shared__ int s_bin, s_above;
  const int tid = threadIdx.x;
  const int g = blockIdx.x, i = g / p.c.h_kv;
  const int L = paged_length(p.c, p.lens_in[i]);
  const int32_t* table = p.c.table + (size_t)i * p.c.max_pages;
  const float* score = p.scores_in + (size_t)g * p.c.positions();
  const int old = max(0, L - p.recent);
  auto there = [&](int pos) { return (unsigned)table[(unsigned)pos / (unsigned)p.c.page_size] < (unsigned)p.c.num_pages; };
  auto key_of = [&](int pos) -> uint32_t { return pos < old && there(pos) ? score_key(score[pos]) : 0u; };      // 0: not one of the older ones
  int n_old = 0, n_recent = 0;
  for (int pos = tid; pos < L; pos += kSelectThreads)
    if (there(pos)) (pos < old ? n_old : n_recent) += 1;
  int all_old, all_recent;
  before_me(n_old, waves, &all_old);
  before_me(n_recent, waves, &all_recent);
  int want = min(all_old, p.budget - min(all_recent, p.budget));
  uint32_t threshold = 0;              // keys above it stay, and of those equal to it the first `ties`
  int ties = 0;
  if (want == all_old) {
    threshold = 0;                     // (every one: their keys are above 0)
  } else if (want == 0) {
    threshold = 0xffffffffu;
  } else {
    int rank = want;                   // the rank of the threshold among the keys that agree with its upper bits
    const int shifts[3] = {21, 10, 0}, sizes[3] = {11, 11, 10};
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = shifts[pass], count = 1 << sizes[pass];
      const uint32_t agree = pass == 0 ? 0u : ~0u << (shift + sizes[pass]);
      for (int x = tid; x < count; x += kSelectThreads) bins[x] = 0;
      __syncthreads();
      for (int pos = tid; pos < old; pos += kSelectThreads) {
        const uint32_t key = key_of(pos);
        if (key != 0 && (key & agree) == (threshold & agree)) atomicAdd(&bins[(key >> shift) & (count - 1)], 1);
      }
      __syncthreads();
      // bins from the top: thread t has the two (or the one) from count - 1 - 2t down
      const int top = count - 1 - 2 * tid;
      const int x0 = top >= 0 ? bins[top] : 0, x1 = top >= 1 ? bins[top - 1] : 0;
      int total;
      const int above = before_me(x0 + x1, waves, &total);
      if (above < rank && rank <= above + x0) { s_bin = top; s_above = above; }
      if (above + x0 < rank && rank <= above + x0 + x1) { s_bin = top - 1; s_above = above + x0; }
      __syncthreads();
      threshold |= (uint32_t)s_bin << shift;
      rank -= s_above;
      __syncthreads();
    }
    ties = rank;
  }
  // the positions that stay, in order
  int32_t* kept = p.kept + (size_t)g * p.budget;
  float* score_out = p.scores_out + (size_t)g * p.max_pages_out * p.c.page_size;
  int done = 0, tied = 0;
  for (int base = 0; base < L; base += kSelectThreads) {
    const int pos = base + tid;
    const uint32_t key = pos < old ? key_of(pos) : 0u;
    const bool equal = key != 0 && key == threshold;
    int total;
    const int equals_before = tied + before_me(equal ? 1 : 0, waves, &total);
    tied += total;
    const bool stays = pos < L && (pos < old ? key > threshold || (equal && equals_before < ties) : there(pos));
    const int slot = done + before_me(stays ? 1 : 0, waves, &total);
    done += total;
    if (stays && slot < p.budget) {
      kept[slot] = pos;
      score_out[slot] = score[pos];
    }
  }
  done = min(done, p.budget);
  for (int slot = done + tid; slot < p.budget; slot += kSelectThreads) kept[slot] = -1;
  if (g % p.c.h_kv == 0 && tid == 0) p.lens_out[i] = done;
}

// The rows that stay, 16 bytes a thread.
__global__ __launch_bounds__(256)
void evict_copy_kernel(PagedEvict p, int k16, int v16) {
  const int w16 = k16 + v16;
  const size_t idx = (size_t)blockIdx.x * 256 + threadIdx.x;
  const size_t line = idx / w16;                                  // (sequence, head, slot)
  const size_t g = line / p.budget;
  if (g >= (size_t)p.b * p.c.h_kv) return;
  const int x = (int)(idx - line * w16), slot = (int)(line - g * p.budget);
  const int i = (int)(g / p.c.h_kv), e = (int)(g - (size_t)i * p.c.h_kv);
  const int pos = p.kept[line];
  if (pos < 0) return;
  const int from = paged_row(p.c, p.c.table + (size_t)i * p.c.max_pages, e, pos);
  const int to = paged_row(p.c, p.table_out + (size_t)i * p.max_pages_out, e, slot);
  if (from < 0 || to < 0) return;
  uint4* pool = static_cast<uint4*>(x < k16 ? p.c.K : p.c.V);
  const int width = x < k16 ? k16 : v16, at = x < k16 ? x : x - k16;
  pool[(size_t)to * width + at] = pool[(size_t)from * width + at];
}

}  // namespace

hipError_t launch_paged_append(const PagedAppend& p, int is_bf16, hipStream_t st) {
  const size_t threads = (size_t)p.b * p.n * p.c.h_kv * ((p.c.k >> 3) + (p.c.v >> 3));
  const dim3 grid((unsigned)((threads + 255) / 256)), block(256);
  if (is_bf16) hipLaunchKernelGGL(paged_append_kernel<uint16_t>, grid, block, 0, st, p);
  else hipLaunchKernelGGL(paged_append_kernel<float>, grid, block, 0, st, p);
  return hipGetLastError();
}

hipError_t launch_paged_evict(const PagedEvict& p, int is_bf16, hipStream_t st) {
  const int groups = p.b * p.c.h_kv, esz = is_bf16 ? 2 : 4;
  hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)groups), dim3(kSelectThreads), 0, st, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int k16 = p.c.k * esz / 16, v16 = p.c.v * esz / 16;
  const size_t threads = (size_t)groups * p.budget * (k16 + v16);
  hipLaunchKernelGGL(evict_copy_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, st, p, k16, v16);
  return hipGetLastError();
}

}  // namespace mqa
