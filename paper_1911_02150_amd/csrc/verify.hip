// Drafted tokens against the target's probabilities (speculative decoding; also, with no drafts, one token drawn from given logits).
//
// p_j = softmax(logits[j] / temperature), q_j = softmax(draft_logits[j] / temperature), or all of it on the drafted token.  Draft j stands while those before
// it do and u[j] q_j(t_j) < p_j(t_j); behind the last that stands comes one token drawn by u[n] from what p has over q, max(p - q, 0) over its sum (from p
// where no draft was refused): the lowest index at which the running sum exceeds u[n] times the whole.
//
// The indices are what comes out, so that everything between is held in float64: a running sum over 32768 probabilities in float32 is off by more than many of
// them are.  Its exponential is the Taylor series of 2^x on [-1/2, 1/2]; the sums of the rows cost about as long as reading them.
#include "paged.hpp"

namespace mqa {
namespace {

constexpr int kThreads = 256;
constexpr int kEach = 16;                          // logits of a thread
constexpr int kChunk = kThreads * kEach;           // of a workgroup

// What a chunk of a row of logits adds up to.
struct ChunkStats { double sum; float most; int at; };       // sum of e^((x - most) / temperature); the largest logit and its lowest index

// -inf for NaN, and +inf as the largest number: a row always has a distribution unless it is -inf throughout.
__device__ __forceinline__ float tame(float x) { return x != x ? -INFINITY : fminf(x, 3.402823466e+38f); }

// 2^x for x <= 0: the series sum (x ln 2)^k / k! to k = 13 (the next term is below 2^-54 of the sum on [-1/2, 1/2])
__device__ __forceinline__ double exp2_of(double x) {
  if (!(x > -1000.)) return 0.;                    // (2^-1000 of the largest: nothing in any sum; -inf)
  const double whole = rint(x), y = (x - whole) * 0.6931471805599453094;
  double s = 1. / 6227020800.;
  s = fma(s, y, 1. / 479001600.);
  s = fma(s, y, 1. / 39916800.);
  s = fma(s, y, 1. / 3628800.);
  s = fma(s, y, 1. / 362880.);
  s = fma(s, y, 1. / 40320.);
  s = fma(s, y, 1. / 5040.);
  s = fma(s, y, 1. / 720.);
  s = fma(s, y, 1. / 120.);
  s = fma(s, y, 1. / 24.);
  s = fma(s, y, 1. / 6.);
  s = fma(s, y, 0.5);
  s = fma(s, y, 1.);
  s = fma(s, y, 1.);
  return ldexp(s, (int)whole);
}
// e^((x - most) / temperature), `per` = log2(e) / temperature
__device__ __forceinline__ double weight(float x, float most, double per) { return most == -INFINITY ? 0. : exp2_of(((double)x - (double)most) * per); }

__device__ __forceinline__ void better(float& x, int& i, float y, int j) {
  if (y > x || (y == x && j < i)) { x = y; i = j; }
}

__device__ __forceinline__ double block_sum(double x, double* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

__device__ __forceinline__ int drafts_of(const Verify& p, int i) { return p.counts ? min(max(p.counts[i], 0), p.n) : p.n; }

// rows of a sequence: n + 1 of the target, then n of the draft
__global__ __launch_bounds__(kThreads)
void verify_stats_kernel(Verify p, int chunks, int rows, ChunkStats* stats) {
  __shared__ double red[4];
  __shared__ float s_most[4];
  __shared__ int s_at[4];
  const int chunk = blockIdx.x % chunks, row = blockIdx.x / chunks % rows, i = blockIdx.x / chunks / rows;
  const int count = drafts_of(p, i);
  const bool drafted = row > p.n;
  const int j = drafted ? row - p.n - 1 : row;
  if (drafted ? j >= count : j > count) return;
  const float* x = drafted ? p.draft_logits + ((size_t)i * p.n + j) * p.vocab : p.logits + ((size_t)i * (p.n + 1) + j) * p.vocab;
  const int first = chunk * kChunk;
  float val[kEach];
  float most = -INFINITY;
  int at = 0x7fffffff;
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const int idx = first + e * kThreads + threadIdx.x;
    val[e] = idx < p.vocab ? tame(x[idx]) : -INFINITY;
  }
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const int idx = first + e * kThreads + threadIdx.x;
    if (idx < p.vocab) better(most, at, val[e], idx);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) better(most, at, __shfl_xor(most, o), __shfl_xor(at, o));
  if ((threadIdx.x & 63) == 0) { s_most[threadIdx.x >> 6] = most; s_at[threadIdx.x >> 6] = at; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 4; ++w) better(most, at, s_most[w], s_at[w]);
  double sum = 0.;
  if (p.temperature > 0.f) {
    const double per = 1.4426950408889634074 / (double)p.temperature;
#pragma unroll
    for (int e = 0; e < kEach; ++e) sum += weight(val[e], most, per);
    sum = block_sum(sum, red);
  }
  if (threadIdx.x == 0) stats[((size_t)i * rows + row) * chunks + chunk] = ChunkStats{sum, most, at};
}

struct RowStats { double sum; float most; int at; };
__device__ __forceinline__ RowStats row_stats(const ChunkStats* s, int chunks, double per) {
  RowStats r{0., -INFINITY, 0x7fffffff};
  for (int c = 0; c < chunks; ++c) better(r.most, r.at, s[c].most, s[c].at);
  if (per > 0.)
    for (int c = 0; c < chunks; ++c) r.sum += s[c].sum * weight(s[c].most, r.most, per);
  return r;
}

// How many drafts stand, and the distribution of the token behind them: all threads of the workgroup together.
struct Choice { int accepted; bool refused; int drafted; RowStats p, q; };
__device__ __forceinline__ Choice choose(const Verify& p, int i, int chunks, int rows, const ChunkStats* stats, int* s_first) {
  const int count = drafts_of(p, i);
  const double per = p.temperature > 0.f ? 1.4426950408889634074 / (double)p.temperature : 0.;
  const ChunkStats* mine = stats + (size_t)i * rows * chunks;
  if (threadIdx.x == 0) *s_first = count;
  __syncthreads();
  for (int j = threadIdx.x; j < count; j += kThreads) {
    const int t = p.drafts[(size_t)i * p.n + j];
    const RowStats a = row_stats(mine + (size_t)j * chunks, chunks, per);
    bool stands = false;
    if (t >= 0 && t < p.vocab) {
      if (per == 0.) {
        stands = t == (a.at < p.vocab ? a.at : 0);
      } else {
        const double u = p.u[(size_t)i * (p.n + 1) + j];
        const double pt = weight(tame(p.logits[((size_t)i * (p.n + 1) + j) * p.vocab + t]), a.most, per);
        if (p.draft_logits) {
          const RowStats d = row_stats(mine + (size_t)(p.n + 1 + j) * chunks, chunks, per);
          const double qt = weight(tame(p.draft_logits[((size_t)i * p.n + j) * p.vocab + t]), d.most, per);
          stands = u * qt * a.sum < pt * d.sum;
        } else {
          stands = u * a.sum < pt;
        }
      }
    }
    if (!stands) atomicMin(s_first, j);
  }
  __syncthreads();
  Choice c;
  c.accepted = *s_first;
  c.refused = c.accepted < count;
  c.drafted = c.refused ? p.drafts[(size_t)i * p.n + c.accepted] : -1;
  c.p = row_stats(mine + (size_t)c.accepted * chunks, chunks, per);
  c.q = RowStats{0., -INFINITY, 0};
  if (c.refused && p.draft_logits && per > 0.) c.q = row_stats(mine + (size_t)(p.n + 1 + c.accepted) * chunks, chunks, per);
  return c;
}

// What p has over q at index v, times the sum of p's row.
struct Rest {
  const float *x, *y;
  float most_p, most_q;
  double per, scale_q;
  int drafted;
  __device__ __forceinline__ Rest(const Verify& p, int i, const Choice& c) {
    per = 1.4426950408889634074 / (double)p.temperature;
    x = p.logits + ((size_t)i * (p.n + 1) + c.accepted) * p.vocab;
    y = c.refused && p.draft_logits ? p.draft_logits + ((size_t)i * p.n + c.accepted) * p.vocab : nullptr;
    most_p = c.p.most;
    most_q = c.q.most;
    scale_q = c.q.sum > 0. ? c.p.sum / c.q.sum : 0.;
    drafted = y ? -1 : c.drafted;
  }
  __device__ __forceinline__ double at(int v) const {
    if (v == drafted) return 0.;
    double r = weight(tame(x[v]), most_p, per);
    if (y) r = fmax(r - weight(tame(y[v]), most_q, per) * scale_q, 0.);
    return r;
  }
};

__global__ __launch_bounds__(kThreads)
void verify_rest_kernel(Verify p, int chunks, int rows, const ChunkStats* stats, double* rest) {
  __shared__ double red[4];
  __shared__ int s_first;
  const int chunk = blockIdx.x % chunks, i = blockIdx.x / chunks;
  const Choice c = choose(p, i, chunks, rows, stats, &s_first);
  const Rest r(p, i, c);
  double sum = 0.;
#pragma unroll 4
  for (int e = 0; e < kEach; ++e) {
    const int v = chunk * kChunk + e * kThreads + threadIdx.x;
    if (v < p.vocab) sum += r.at(v);
  }
  sum = block_sum(sum, red);
  if (threadIdx.x == 0) rest[(size_t)i * chunks + chunk] = sum;
}

__global__ __launch_bounds__(kThreads)
void verify_draw_kernel(Verify p, int chunks, int rows, const ChunkStats* stats, const double* rest) {
  __shared__ int s_first, s_token, s_last;
  __shared__ double s_waves[4];
  const int i = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Choice c = choose(p, i, chunks, rows, stats, &s_first);
  int token = c.p.at < p.vocab ? c.p.at : 0;             // the most probable (a row of -inf throughout: 0)
  if (p.temperature > 0.f) {
    const Rest r(p, i, c);
    double total = 0.;
    for (int x = 0; x < chunks; ++x) total += rest[(size_t)i * chunks + x];
    if (total > 0.) {
      const double goal = (double)p.u[(size_t)i * (p.n + 1) + p.n] * total;
      // the chunk in which the running sum exceeds the goal; past all of them (u is not below 1): the last that has anything
      int chunk = -1, last = 0;
      double before = 0., sum = 0.;
      for (int x = 0; x < chunks; ++x) {
        const double add = rest[(size_t)i * chunks + x];
        if (add > 0.) last = x;
        if (chunk < 0 && sum + add > goal) { chunk = x; before = sum; }
        sum += add;
      }
      const bool inside = chunk >= 0;
      if (!inside) chunk = last;
      if (tid == 0) { s_token = 0x7fffffff; s_last = -1; }
      double val[kEach], mine = 0.;
      const int v0 = chunk * kChunk + tid * kEach;
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        val[e] = v0 + e < p.vocab ? r.at(v0 + e) : 0.;
        mine += val[e];
      }
      double incl = mine;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const double y = __shfl_up(incl, off);
        if (lane >= off) incl += y;
      }
      if (lane == 63) s_waves[wave] = incl;
      __syncthreads();
      double run = before + (incl - mine);
      for (int w = 0; w < wave; ++w) run += s_waves[w];
      int found = 0x7fffffff, there = -1;
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        run += val[e];
        if (val[e] > 0.) {
          there = v0 + e;
          if (inside && run > goal && found == 0x7fffffff) found = v0 + e;
        }
      }
      if (found != 0x7fffffff) atomicMin(&s_token, found);
      if (there >= 0) atomicMax(&s_last, there);
      __syncthreads();
      if (s_token != 0x7fffffff) token = s_token;
      else if (s_last >= 0) token = s_last;
    }
  }
  for (int j = tid; j <= p.n; j += kThreads)
    p.tokens[(size_t)i * (p.n + 1) + j] = j < c.accepted ? p.drafts[(size_t)i * p.n + j] : j == c.accepted ? token : -1;
  if (tid == 0) p.accepted[i] = c.accepted;
}

int verify_chunks(int vocab) { return (vocab + kChunk - 1) / kChunk; }

}  // namespace

size_t verify_workspace_bytes(int b, int n, int vocab) {
  const size_t chunks = verify_chunks(vocab);
  return (size_t)b * (2 * (size_t)n + 1) * chunks * sizeof(ChunkStats) + (size_t)b * chunks * sizeof(double);
}

hipError_t launch_verify(const Verify& p, void* workspace, hipStream_t st) {
  const int chunks = verify_chunks(p.vocab), rows = p.draft_logits && p.temperature > 0.f ? 2 * p.n + 1 : p.n + 1;
  ChunkStats* stats = static_cast<ChunkStats*>(workspace);
  double* rest = reinterpret_cast<double*>(stats + (size_t)p.b * rows * chunks);
  hipLaunchKernelGGL(verify_stats_kernel, dim3((unsigned)((size_t)p.b * rows * chunks)), dim3(kThreads), 0, st, p, chunks, rows, stats);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (p.temperature > 0.f) {
    hipLaunchKernelGGL(verify_rest_kernel, dim3((unsigned)((size_t)p.b * chunks)), dim3(kThreads), 0, st, p, chunks, rows, stats, rest);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(verify_draw_kernel, dim3((unsigned)p.b), dim3(kThreads), 0, st, p, chunks, rows, stats, rest);
  return hipGetLastError();
}

}  // namespace mqa
