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

// Sum of x over the workgroup's threads before this one; *total: over all.  `waves` is the call's own until two barriers later.
__device__ __forceinline__ int before_me(int x, int* waves, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int incl = x;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int y = __shfl_up(incl, off);
    if (lane >= off) incl += y;
  }
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
// which the wanted rank lies, until all of a bin stays (one sequence of 100 in two passes 8.1 us, in three 10.8).  One workgroup per (sequence, head), which is bound by the latency of its steps: a thread's KEEP positions
// (tid, tid + 1024, ...) are read once and stay in registers, and what stays is put in order by two sums over all of them, not two
// for every 1024 (8192 positions: 36 -> 12 us).  Capacities beyond (KEEP = 0) are gone over again for every step, eight positions a thread on their way together
// (one sequence of 130000: 164 us, one position at a time 379).
template <int KEEP>
__global__ __launch_bounds__(kSelectThreads)
void evict_select_kernel(PagedEvict p) {
  constexpr int kWaves = kSelectThreads / 64;
  __shared__ int bins[kBins];
  __shared__ int waves[8][kWaves];     // a scan's each; those of the loops in turn
  __shared__ int s_bin, s_above, s_all;
  __shared__ int s_count[2][(KEEP > 0 ? KEEP : 1) * kWaves + 1];      // of a wave's 64 positions: those at the threshold, those that stay
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int g = blockIdx.x, i = g / p.c.h_kv;
  const int L = paged_length(p.c, p.lens_in[i]);
  const int32_t* table = p.c.table + (size_t)i * p.c.max_pages;
  const float* score = p.scores_in + (size_t)g * p.c.positions();
  const int old = max(0, L - p.recent);
  constexpr int kStep = 8 * kSelectThreads;
  const unsigned size = p.c.page_size, step = kSelectThreads / size, more = kSelectThreads % size;
  struct Walk { unsigned page, inside; };      // of positions tid, tid + 1024, ...
  const Walk start{(unsigned)tid / size, (unsigned)tid % size};
  auto next = [&](Walk& w) {
    w.page += step;
    w.inside += more;
    if (w.inside >= size) { w.inside -= size; ++w.page; }
  };
  // see(position, whether it is there, its score) for all positions below `end`, and some that are not, eight on their way at a time
  auto go_over = [&](int end, auto&& see) {
    Walk w = start;
    for (int base = 0; base < end; base += kStep) {
      int32_t entry[8];
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {    // (past the end: the first entry and score, which are there)
        const int pos = base + u * kSelectThreads + tid;
        entry[u] = table[pos < end ? w.page : 0u];
        x[u] = score[pos < end ? pos : 0];
        next(w);
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int pos = base + u * kSelectThreads + tid;
        see(pos, pos < end && (unsigned)entry[u] < (unsigned)p.c.num_pages, x[u]);
      }
    }
  };
  for (int x = tid; x < kBins; x += kSelectThreads) bins[x] = 0;
  uint32_t keys[KEEP > 0 ? KEEP : 1];
  float values[KEEP > 0 ? KEEP : 1];
  uint32_t late = 0;                   // bit u: the thread's u-th position is one of the latest, and there
  int n_old = 0, n_recent = 0;
  if constexpr (KEEP > 0) {
    Walk w = start;
#pragma unroll
    for (int u = 0; u < KEEP; ++u) {   // (past the length: the first entry and score, which are there)
      const int pos = tid + u * kSelectThreads;
      keys[u] = (uint32_t)table[pos < L ? w.page : 0u];
      values[u] = score[pos < L ? pos : 0];
      next(w);
    }
#pragma unroll
    for (int u = 0; u < KEEP; ++u) {
      const int pos = tid + u * kSelectThreads;
      const bool is = pos < L && keys[u] < (unsigned)p.c.num_pages;
      keys[u] = is && pos < old ? score_key(values[u]) : 0u;
      late |= (uint32_t)(is && pos >= old) << u;
      n_old += keys[u] != 0;
    }
    n_recent = __popc(late);
  } else {
    go_over(L, [&](int pos, bool is, float) {
      n_old += is && pos < old;
      n_recent += is && pos >= old;
    });
  }
  int all_old, all_recent;
  if constexpr (KEEP > 0) {            // (both in one: up to 24576 each)
    int all;
    before_me(n_old | n_recent << 16, waves[0], &all);
    all_old = all & 0xffff;
    all_recent = (int)((unsigned)all >> 16);
  } else {
    before_me(n_old, waves[0], &all_old);
    before_me(n_recent, waves[1], &all_recent);
  }
  const int want = min(all_old, p.budget - min(all_recent, p.budget));
  uint32_t threshold = 0;              // keys above it stay, and of those equal to it the first `ties`
  int ties = 0;
  if (want == 0) {
    threshold = 0xffffffffu;
  } else if (want < all_old) {         // (else every one: their keys are above 0)
    int rank = want;                   // the rank of the threshold among the keys that agree with its upper bits
    const int shifts[3] = {21, 10, 0}, sizes[3] = {11, 11, 10};
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = shifts[pass], count = 1 << sizes[pass];
      const uint32_t agree = pass == 0 ? 0u : ~0u << (shift + sizes[pass]);
      auto add = [&](uint32_t key) {
        if (key != 0 && (key & agree) == (threshold & agree)) atomicAdd(&bins[(key >> shift) & (count - 1)], 1);
      };
      if constexpr (KEEP > 0) {
#pragma unroll
        for (int u = 0; u < KEEP; ++u) add(keys[u]);
      } else {
        go_over(old, [&](int, bool is, float x) { add(is ? score_key(x) : 0u); });
      }
      __syncthreads();
      // bins from the top: thread t has the two (or the one) from count - 1 - 2t down
      const int top = count - 1 - 2 * tid;
      int x0 = 0, x1 = 0;
      if (top >= 0) {                  // (count is even)
        x0 = bins[top];
        x1 = bins[top - 1];
        bins[top] = bins[top - 1] = 0; // (for the next pass)
      }
      int total;
      const int above = before_me(x0 + x1, waves[2 + pass], &total);
      if (above < rank && rank <= above + x0) { s_bin = top; s_above = above; s_all = x0; }
      if (above + x0 < rank && rank <= above + x0 + x1) { s_bin = top - 1; s_above = above + x0; s_all = x1; }
      __syncthreads();
      threshold |= (uint32_t)s_bin << shift;
      rank -= s_above;
      if (rank == s_all) {             // the whole bin stays: every key from its first on  (no key is 0 in the first pass' bits)
        --threshold;
        rank = 0;
        break;
      }
    }
    ties = rank;
  }
  // the positions that stay, in order
  int32_t* kept = p.kept + (size_t)g * p.budget;
  float* score_out = p.scores_out + (size_t)g * p.max_pages_out * p.c.page_size;
  int done = 0;
  if constexpr (KEEP > 0) {
    // in order: by u, then by wave, then by lane
    const unsigned long long below = (1ull << lane) - 1;
    auto in_order = [&](int which) {   // the counts of all waves in the place of their running sum; the last: of all
      constexpr int all = KEEP * kWaves;
      static_assert(all <= kSelectThreads, "a count a thread");
      __syncthreads();
      int total;
      const int before = before_me(tid < all ? s_count[which][tid] : 0, waves[5 + which], &total);
      if (tid < all) s_count[which][tid] = before;
      if (tid == 0) s_count[which][all] = total;
      __syncthreads();
    };
    uint32_t equal = 0, stays = late;
#pragma unroll
    for (int u = 0; u < KEEP; ++u) {
      equal |= (uint32_t)(keys[u] != 0 && keys[u] == threshold) << u;
      stays |= (uint32_t)(keys[u] > threshold) << u;
    }
    if (ties > 0) {
#pragma unroll
      for (int u = 0; u < KEEP; ++u) {
        const unsigned long long those = __ballot(equal >> u & 1);
        if (lane == 0) s_count[0][u * kWaves + wave] = __popcll(those);
      }
      in_order(0);
#pragma unroll
      for (int u = 0; u < KEEP; ++u) {
        const unsigned long long those = __ballot(equal >> u & 1);
        if ((equal >> u & 1) && s_count[0][u * kWaves + wave] + __popcll(those & below) < ties) stays |= 1u << u;
      }
    }
#pragma unroll
    for (int u = 0; u < KEEP; ++u) {
      const unsigned long long those = __ballot(stays >> u & 1);
      if (lane == 0) s_count[1][u * kWaves + wave] = __popcll(those);
    }
    in_order(1);
#pragma unroll
    for (int u = 0; u < KEEP; ++u) {
      const unsigned long long those = __ballot(stays >> u & 1);
      const int slot = s_count[1][u * kWaves + wave] + __popcll(those & below);
      if ((stays >> u & 1) && slot < p.budget) {
        kept[slot] = tid + u * kSelectThreads;
        score_out[slot] = values[u];
      }
    }
    done = s_count[1][KEEP * kWaves];
  } else {
    int tied = 0;
    for (int base = 0; base < L; base += kStep) {
      const int first = base + 8 * tid;
      Walk w{(unsigned)first / size, (unsigned)first % size};
      float x[8];
      int32_t entry[8];
      uint32_t is = 0, stays = 0, equal = 0;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        entry[u] = table[first + u < L ? w.page : 0u];
        x[u] = score[first + u < L ? first + u : 0];
        if (++w.inside == size) { w.inside = 0; ++w.page; }
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) is |= (uint32_t)(first + u < L && (unsigned)entry[u] < (unsigned)p.c.num_pages) << u;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const uint32_t key = score_key(x[u]);
        const bool late = first + u >= old;
        stays |= (uint32_t)(late || key > threshold) << u;
        equal |= (uint32_t)(!late && key == threshold) << u;
      }
      stays &= is;
      equal &= is;
      int total;
      if (ties > 0) {                  // (the same in all threads)
        int rank = tied + before_me(__popc(equal), waves[5], &total);
        tied += total;
#pragma unroll
        for (int u = 0; u < 8; ++u)
          if (equal >> u & 1) stays |= (uint32_t)(rank++ < ties) << u;
      }
      int slot = done + before_me(__popc(stays), waves[6], &total);
      done += total;
      __syncthreads();                 // (the scans' places are the next round's)
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (stays >> u & 1) {
          if (slot < p.budget) {
            kept[slot] = first + u;
            score_out[slot] = x[u];
          }
          ++slot;
        }
    }
  }
  done = min(done, p.budget);
  for (int slot = done + tid; slot < p.budget; slot += kSelectThreads) kept[slot] = -1;
  if (g % p.c.h_kv == 0 && tid == 0) p.lens_out[i] = done;
}

// The rows that stay: 16 lanes a row, a word of K and one of V of each on their way together.  A row costs a chain (kept position -> two table entries -> row)
// that other waves cover: 56000 rows of 512 bytes 13 us (4.6 TB/s read and written), where a thread with two rows takes 24 and one with a single word 19.
// (Without branches around the loads, which would wait for one another: what is not to be copied is read from the pool's first row.)
constexpr int kCopyLanes = 16, kCopyEach = 256 / kCopyLanes;      // lanes of a row, rows of a workgroup
__global__ __launch_bounds__(256)
void evict_copy_kernel(PagedEvict p, int k16, int v16, int pieces) {
  const int g = (int)(blockIdx.x / (unsigned)pieces), piece = (int)blockIdx.x - g * pieces;
  const int i = g / p.c.h_kv, e = g - i * p.c.h_kv;
  const int mine = piece * kCopyEach + (int)threadIdx.x / kCopyLanes, slot = min(mine, p.budget - 1);
  const int pos = p.kept[(size_t)g * p.budget + slot];
  const int from = paged_row(p.c, p.c.table + (size_t)i * p.c.max_pages, e, max(pos, 0));
  const int to = paged_row(p.c, p.table_out + (size_t)i * p.max_pages_out, e, slot);
  const bool copied = mine < p.budget && pos >= 0 && from >= 0 && to >= 0;
  const size_t src = max(from, 0), dst = max(to, 0);
  uint4 *K = static_cast<uint4*>(p.c.K), *V = static_cast<uint4*>(p.c.V);
  for (int x = threadIdx.x & (kCopyLanes - 1); x < max(k16, v16); x += kCopyLanes) {
    const uint4 kw = K[src * k16 + min(x, k16 - 1)], vw = V[src * v16 + min(x, v16 - 1)];
    if (copied && x < k16) K[dst * k16 + x] = kw;
    if (copied && x < v16) V[dst * v16 + x] = vw;
  }
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
  const int groups = p.b * p.c.h_kv, esz = is_bf16 ? 2 : 4, each = (p.c.positions() + kSelectThreads - 1) / kSelectThreads;
  const dim3 grid((unsigned)groups), block(kSelectThreads);
  // As few positions a thread as hold the capacity, since a thread goes over all that it could have (one sequence of 700: 8.7 us with 3, 11.1 with 10, 15.6 with 24, gone
  // over again 12.9; 6000: 11.9 with 10, 16.4, 16.1; 24000: 19.9 with 24, 36.7).
  if (each <= 3) hipLaunchKernelGGL(evict_select_kernel<3>, grid, block, 0, st, p);
  else if (each <= 10) hipLaunchKernelGGL(evict_select_kernel<10>, grid, block, 0, st, p);
  else if (each <= 24) hipLaunchKernelGGL(evict_select_kernel<24>, grid, block, 0, st, p);
  else hipLaunchKernelGGL(evict_select_kernel<0>, grid, block, 0, st, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int pieces = (p.budget + kCopyEach - 1) / kCopyEach;
  hipLaunchKernelGGL(evict_copy_kernel, dim3((unsigned)groups * pieces), dim3(256), 0, st, p, p.c.k * esz / 16, p.c.v * esz / 16, pieces);
  return hipGetLastError();
}

}  // namespace mqa
