// Drafted tokens against the target's probabilities (speculative decoding; also, with no drafts, one token drawn from given logits).
//
// p_j = softmax(logits[j] / temperature), q_j = softmax(draft_logits[j] / temperature), or all of it on the drafted token.  Draft j stands while those before
// it do and u[j] q_j(t_j) < p_j(t_j); behind the last that stands comes one token drawn by u[n] from what p has over q, max(p - q, 0) over its sum (from p
// where no draft was refused): the lowest index at which the running sum exceeds u[n] times the whole.
//
// The indices are what comes out, so that everything between is held in float64: a running sum over 32768 probabilities in float32 is off by more than many of
// them are.  An exponential is some twenty float64 instructions, 2^x by its Taylor series around the nearest integer.  Three launches: the rows' sums
// (what reads, all but the drafts behind the count); the choice of the row that decides, and what is left of it in segments of 256 tokens; the segment that
// holds the goal, token by token.  (Shorter rows: what follows the sums in one launch, or all of it.)
#include "paged.hpp"

namespace mqa {
namespace {

constexpr int kThreads = 256;
constexpr int kEach = 16;                          // logits of a thread, or half as many: of a workgroup a chunk of 4096 or 2048

// What a chunk of a row of logits adds up to: the sum of e^((x - most) / temperature); the largest logit and (temperature 0) its lowest index.
// (at: not below vocab where nothing is comparable: a row of NaN)
struct ChunkStats { double sum; float most; int at; };
struct RowStats { double sum; float most; int at; };

// -inf for NaN, and +inf as the largest number: a row always has a distribution unless it is -inf throughout.
__device__ __forceinline__ float tame(float x) { return x != x ? -INFINITY : fminf(x, 3.402823466e+38f); }

// 2^x for x <= 0: with n the nearest integer (left in the low word by an addition that rounds to integers) and y = x - n the polynomial of degree 11 that equals 2^y
// at the twelve Chebyshev nodes of [-1/2, 1/2]: off by 2^-55.4 of 2^y at most, so that a weight is off by float64's own roundings (the series sum (y ln 2)^k / k! needs
// k = 13 for that; cut at k = 10, 2^-41.6, an index went wrong where the goal was that near a border); below 2^-1000 nothing.
__device__ __forceinline__ double exp2_of(double x) {
  const double shift = 6755399441055744.;          // 1.5 * 2^52
  const double n = x + shift, y = x - (n - shift);
  double s = 4.4558179083360645e-10;
  s = fma(s, y, 7.0741942972885214e-9);
  s = fma(s, y, 1.0178057087733941e-7);
  s = fma(s, y, 1.3215432535912375e-6);
  s = fma(s, y, 1.5252733841556773e-5);
  s = fma(s, y, 1.5403530463724353e-4);
  s = fma(s, y, 1.3333558146406470e-3);
  s = fma(s, y, 9.6181291075872560e-3);
  s = fma(s, y, 5.5504108664821625e-2);
  s = fma(s, y, 0.24022650695910158);
  s = fma(s, y, 0.69314718055994530);
  s = fma(s, y, 1.);
  const double z = __hiloint2double(__double2hiint(s) + (__double2loint(n) << 20), __double2loint(s));
  return x > -1000. ? z : 0.;                      // (-inf, and what a row of -inf throughout gives, NaN, are here)
}
// e^((x - most) / temperature), `per` = log2(e) / temperature
__device__ __forceinline__ double weight(float x, float most, double per) { return exp2_of(((double)x - (double)most) * per); }
__device__ __forceinline__ double per_of(const Verify& p) { return 1.4426950408889634074 / (double)p.temperature; }

__device__ __forceinline__ void better(float& x, int& i, float y, int j) {
  if (y > x || (y == x && j < i)) { x = y; i = j; }
}

__device__ __forceinline__ double block_sum(double x, double* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

__device__ __forceinline__ int drafts_of(const Verify& p, int i) { return p.counts ? min(max(p.counts[i], 0), p.n) : p.n; }

// A thread's logits of a chunk of THREADS * EACH, 16 bytes at a time (of rows that begin at any float: the memory pipe takes them so); past the end -inf.
// at(e): the index of the e-th.  RAW: as they are, for the largest one (comparisons pass NaN over, as in argmax_kernel).
template <int THREADS, int EACH, bool RAW = false>
struct Logits {
  typedef __attribute__((ext_vector_type(4), aligned(4))) float Four;
  static constexpr int kStep = 4 * THREADS;
  float x[EACH];
  int first;
  __device__ __forceinline__ Logits(const float* row, int chunk, int vocab) {
    first = chunk * THREADS * EACH + 4 * (int)threadIdx.x;
#pragma unroll
    for (int e = 0; e < EACH / 4; ++e) {
      const int v = first + e * kStep;
      Four y = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      if (v + 4 <= vocab) {
        y = *reinterpret_cast<const Four*>(row + v);
      } else {
#pragma unroll
        for (int z = 0; z < 3; ++z)
          if (v + z < vocab) y[z] = row[v + z];
      }
#pragma unroll
      for (int z = 0; z < 4; ++z) x[4 * e + z] = y[z];
    }
    if constexpr (!RAW) {
#pragma unroll
      for (int e = 0; e < EACH; ++e) x[e] = tame(x[e]);
    }
  }
  __device__ __forceinline__ int at(int e) const { return first + (e >> 2) * kStep + (e & 3); }
};

// rows of a sequence: n + 1 of the target, then n of the draft
template <bool GREEDY, int EACH>
__global__ __launch_bounds__(kThreads)
void verify_stats_kernel(Verify p, int chunks, int rows, ChunkStats* stats) {
  __shared__ double red[4];
  __shared__ float s_most[4];
  __shared__ int s_at[4];
  const unsigned line = blockIdx.x / (unsigned)chunks;
  const int chunk = (int)(blockIdx.x - line * chunks), i = (int)(line / (unsigned)rows), row = (int)line - i * rows;
  const int count = drafts_of(p, i);
  const bool drafted = row > p.n;
  const int j = drafted ? row - p.n - 1 : row;
  if (drafted ? j >= count : j > count) return;
  const Logits<kThreads, EACH, GREEDY> v(drafted ? p.draft_logits + ((size_t)i * p.n + j) * p.vocab : p.logits + ((size_t)i * (p.n + 1) + j) * p.vocab, chunk, p.vocab);
  float most = -INFINITY;
  int at = 0x7fffffff;
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    if constexpr (GREEDY) {
      if (v.at(e) < p.vocab) better(most, at, v.x[e], v.at(e));
    } else {
      most = fmaxf(most, v.x[e]);
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    if constexpr (GREEDY) better(most, at, __shfl_xor(most, o), __shfl_xor(at, o));
    else most = fmaxf(most, __shfl_xor(most, o));
  }
  if ((threadIdx.x & 63) == 0) { s_most[threadIdx.x >> 6] = most; s_at[threadIdx.x >> 6] = at; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if constexpr (GREEDY) better(most, at, s_most[w], s_at[w]);
    else most = fmaxf(most, s_most[w]);
  }
  double sum = 0.;
  if constexpr (!GREEDY) {
    const double per = per_of(p);
#pragma unroll
    for (int e = 0; e < EACH; ++e) sum += weight(v.x[e], most, per);
    sum = block_sum(sum, red);
  }
  if (threadIdx.x == 0) stats[(size_t)line * chunks + chunk] = ChunkStats{sum, most, at};
}

// A row's statistics from its chunks', by a group of `lanes` neighbouring threads (a power of two up to 64), of which this is the x-th; all get them.
template <bool GREEDY>
__device__ __forceinline__ RowStats row_stats(const ChunkStats* s, int chunks, double per, int x, int lanes) {
  RowStats r{0., -INFINITY, 0x7fffffff};
  if (chunks <= lanes) {                                   // a chunk each: the largest first, then one exponential
    ChunkStats y{0., -INFINITY, 0x7fffffff};
    if (x < chunks) y = s[x];
    r.most = y.most;
    r.at = y.at;
    for (int o = 1; o < lanes; o <<= 1) {
      if constexpr (GREEDY) better(r.most, r.at, __shfl_xor(r.most, o), __shfl_xor(r.at, o));
      else r.most = fmaxf(r.most, __shfl_xor(r.most, o));
    }
    if constexpr (!GREEDY) {
      r.sum = y.sum * weight(y.most, r.most, per);
      for (int o = 1; o < lanes; o <<= 1) r.sum += __shfl_xor(r.sum, o);
    }
    return r;
  }
  for (int c = x; c < chunks; c += lanes) {
    const ChunkStats y = s[c];
    if constexpr (GREEDY) {
      better(r.most, r.at, y.most, y.at);
    } else {
      const float most = fmaxf(r.most, y.most);
      r.sum = r.sum * weight(r.most, most, per) + y.sum * weight(y.most, most, per);
      r.most = most;
    }
  }
  for (int o = 1; o < lanes; o <<= 1) {
    const float most = __shfl_xor(r.most, o);
    if constexpr (GREEDY) {
      better(r.most, r.at, most, __shfl_xor(r.at, o));
    } else {
      const float both = fmaxf(r.most, most);
      r.sum = r.sum * weight(r.most, both, per) + __shfl_xor(r.sum, o) * weight(most, both, per);
      r.most = both;
    }
  }
  return r;
}

// How many drafts stand, and the distribution of the token behind them: all threads of the workgroup together.
struct Choice { RowStats p, q; int accepted, drafted; };      // drafted: the refused token; -1: none was refused
constexpr int kKept = 32;
struct ChooseLds { RowStats p[kKept], q[kKept]; int first; };
// mine: the statistics of the sequence's rows, `chunks` each.
template <bool GREEDY, int THREADS = kThreads>
__device__ __forceinline__ Choice choose(const Verify& p, int i, int chunks, const ChunkStats* mine, ChooseLds* lds) {
  const int count = drafts_of(p, i), tid = threadIdx.x;
  const double per = GREEDY ? 0. : per_of(p);
  int lanes = 64;
  while (lanes > 1 && lanes / 2 >= chunks) lanes >>= 1;
  const int x = tid & (lanes - 1), group = tid / lanes, groups = THREADS / lanes;
  if (tid == 0) lds->first = count;
  __syncthreads();
  for (int j0 = 0; j0 <= count; j0 += groups) {            // (all threads of a group, so that they can exchange; row `count` is behind the last draft)
    const int j = min(j0 + group, count), t = j < count ? p.drafts[(size_t)i * p.n + j] : -1;
    const bool token = t >= 0 && t < p.vocab;
    const float lp = token ? p.logits[((size_t)i * (p.n + 1) + j) * p.vocab + t] : -INFINITY;
    const RowStats a = row_stats<GREEDY>(mine + (size_t)j * chunks, chunks, per, x, lanes);
    RowStats d{0., -INFINITY, 0};
    bool stands = false;
    if constexpr (GREEDY) {
      stands = token && t == (a.at < p.vocab ? a.at : 0);
    } else if (j < count) {                                // (the same j, and draft_logits, in all of a group)
      const double u = p.u[(size_t)i * (p.n + 1) + j];
      const double pt = weight(tame(lp), a.most, per);
      if (p.draft_logits) {
        const float lq = token ? p.draft_logits[((size_t)i * p.n + j) * p.vocab + t] : -INFINITY;
        d = row_stats<false>(mine + (size_t)(p.n + 1 + j) * chunks, chunks, per, x, lanes);
        // (a draft row of -inf throughout: probabilities of 0)
        stands = pt > 0. && (d.sum == 0. || u * weight(tame(lq), d.most, per) * a.sum < pt * d.sum);
      } else {
        stands = pt > 0. && u * a.sum < pt;
      }
    }
    if (x == 0 && j < kKept) { lds->p[j] = a; lds->q[j] = d; }
    if (x == 0 && !stands && j < count) atomicMin(&lds->first, j);
  }
  __syncthreads();
  Choice c;
  c.accepted = lds->first;
  c.drafted = c.accepted < count ? p.drafts[(size_t)i * p.n + c.accepted] : -1;
  if (c.accepted < kKept) {
    c.p = lds->p[c.accepted];
    c.q = lds->q[c.accepted];
  } else {
    c.p = row_stats<GREEDY>(mine + (size_t)c.accepted * chunks, chunks, per, x, lanes);
    c.q = RowStats{0., -INFINITY, 0};
    if constexpr (!GREEDY)
      if (c.accepted < count && p.draft_logits) c.q = row_stats<false>(mine + (size_t)(p.n + 1 + c.accepted) * chunks, chunks, per, x, lanes);
  }
  if (c.accepted >= count) c.drafted = -1;
  else if (c.drafted < 0) c.drafted = 0x7fffffff;          // (refused, and no token)
  return c;
}

// What p has over q, times the sum of p's row.
struct Rest {
  const float *x, *y;      // the rows of logits; y null: nothing is taken off but the drafted token
  double per, scale_q;
  float most_p, most_q;
  int drafted;
  __device__ __forceinline__ Rest(const Verify& p, int i, const Choice& c) {
    per = per_of(p);
    x = p.logits + ((size_t)i * (p.n + 1) + c.accepted) * p.vocab;
    y = c.drafted >= 0 && p.draft_logits ? p.draft_logits + ((size_t)i * p.n + c.accepted) * p.vocab : nullptr;
    most_p = c.p.most;
    most_q = c.q.most;
    scale_q = c.q.sum > 0. ? c.p.sum / c.q.sum : 0.;
    drafted = y ? -1 : c.drafted;
  }
  __device__ __forceinline__ double of(int v, float lp, float lq) const {
    if (v == drafted) return 0.;
    const double r = weight(lp, most_p, per);
    return y ? fmax(r - weight(lq, most_q, per) * scale_q, 0.) : r;
  }
};

constexpr int kSegment = 256;                      // tokens; a chunk has EACH of them

// draft: the thread's own, of the first THREADS
template <int THREADS = kThreads>
__device__ __forceinline__ void write_tokens(const Verify& p, int i, int accepted, int token, int draft) {
  for (int j = threadIdx.x; j <= p.n; j += THREADS)
    p.tokens[(size_t)i * (p.n + 1) + j] = j < accepted ? (j < THREADS ? draft : p.drafts[(size_t)i * p.n + j]) : j == accepted ? token : -1;
  if (threadIdx.x == 0) p.accepted[i] = accepted;
}

__global__ __launch_bounds__(kThreads)
void verify_greedy_kernel(Verify p, int chunks, int rows, const ChunkStats* stats) {
  __shared__ ChooseLds lds;
  const int draft = (int)threadIdx.x < p.n ? p.drafts[(size_t)blockIdx.x * p.n + threadIdx.x] : -1;
  const Choice c = choose<true>(p, blockIdx.x, chunks, stats + (size_t)blockIdx.x * rows * chunks, &lds);
  write_tokens(p, blockIdx.x, c.accepted, c.p.at < p.vocab ? c.p.at : 0, draft);
}

// What is left of the row that decides, a chunk a workgroup, in segments.  (With the draw in the same launch, by the last of a sequence's workgroups, 19 us where
// the two took 9 and 9 (now 7 and 5): what orders writes and reads across the XCDs costs more than a launch.)
template <int EACH>
__global__ __launch_bounds__(kThreads)
void verify_rest_kernel(Verify p, int chunks, int rows, const ChunkStats* stats, double* rest, Choice* choice) {
  __shared__ ChooseLds lds;
  __shared__ double s_sum[EACH];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int i = (int)(blockIdx.x / (unsigned)chunks), chunk = (int)blockIdx.x - i * chunks;
  const Choice c = choose<false>(p, i, chunks, stats + (size_t)i * rows * chunks, &lds);
  if (chunk == 0 && tid == 0) choice[i] = c;
  const Rest r(p, i, c);
  double* left = rest + (size_t)i * chunks * EACH;
  {
    const Logits<kThreads, EACH> lp(r.x, chunk, p.vocab);
    double of[EACH];
    if (r.y) {
      const Logits<kThreads, EACH> lq(r.y, chunk, p.vocab);
#pragma unroll
      for (int e = 0; e < EACH; ++e) of[e] = r.of(lp.at(e), lp.x[e], lq.x[e]);
    } else {
#pragma unroll
      for (int e = 0; e < EACH; ++e) of[e] = r.of(lp.at(e), lp.x[e], 0.f);
    }
#pragma unroll
    for (int e = 0; e < EACH / 4; ++e) {                  // (a segment is a wave's 256 neighbouring tokens)
      double sum = (of[4 * e] + of[4 * e + 1]) + (of[4 * e + 2] + of[4 * e + 3]);
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
      if (lane == 0) s_sum[4 * e + wave] = sum;
    }
  }
  __syncthreads();
  if (tid < EACH) left[(size_t)chunk * EACH + tid] = s_sum[tid];
}

// Where there is nothing to draw from: the lowest index of the row's largest logit (all threads together).
template <int THREADS>
__device__ __forceinline__ int largest(const float* row, int vocab, float* s_most, int* s_at) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float most = -INFINITY;
  int at = 0x7fffffff;
  for (int v = threadIdx.x; v < vocab; v += THREADS) better(most, at, tame(row[v]), v);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) better(most, at, __shfl_xor(most, o), __shfl_xor(at, o));
  if (lane == 0) { s_most[wave] = most; s_at[wave] = at; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) better(most, at, s_most[w], s_at[w]);
  return most > -INFINITY ? at : 0;
}

// What is left of a wave's 256 tokens, four a lane.
struct Four {
  double of[4], upto;      // upto: of the tokens up to this lane's last
  int first;
  template <typename L, typename Q>
  __device__ __forceinline__ Four(const Rest& r, const L& lp, Q&& drafted) {
    first = lp.first;
    if (r.y) {
      const L lq = drafted();
#pragma unroll
      for (int e = 0; e < 4; ++e) of[e] = r.of(lp.at(e), lp.x[e], lq.x[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) of[e] = r.of(lp.at(e), lp.x[e], 0.f);
    }
    upto = (of[0] + of[1]) + (of[2] + of[3]);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double y = __shfl_up(upto, o);
      if ((int)(threadIdx.x & 63) >= o) upto += y;
    }
  }
  // The first token at which the running sum, `before` in front of the wave's, exceeds the goal, else the last that has anything (there is one).
  __device__ __forceinline__ int token(double before, double goal) const {
    double to = __shfl_up(upto, 1);
    to = before + ((threadIdx.x & 63) == 0 ? 0. : to);
    int found = -1, last = -1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      to += of[e];
      if (of[e] > 0.) {
        last = first + e;
        if (found < 0 && to > goal) found = last;
      }
    }
    const unsigned long long those = __ballot(found >= 0), any = __ballot(last >= 0);
    return those != 0 ? __shfl(found, __ffsll(those) - 1) : __shfl(last, any != 0 ? 63 - __clzll(any) : 0);
  }
};

// A wave a sequence, so that nothing waits at a barrier (four waves, the places by atomics in LDS 9.4 us, so 3): the segments, eight neighbouring ones a lane, then the tokens
// of the one that holds the goal, four a lane.
constexpr int kLine = 8, kRound = 64 * kLine;      // segments of a lane; gone over at a time, 131072 tokens
__global__ __launch_bounds__(64)
void verify_draw_kernel(Verify p, int stride, const double* rest, const Choice* choice) {
  __shared__ float s_most[1];
  __shared__ int s_at[1];
  const int i = blockIdx.x, lane = threadIdx.x;
  const int segments = (p.vocab + kSegment - 1) / kSegment;
  const double* sums = rest + (size_t)i * stride;
  double add[kLine], run;                                  // of a round: the lane's segments; those of the lanes up to this one
  auto load = [&](int x0) {
#pragma unroll
    for (int y = 0; y < kLine; ++y) {
      const int at = x0 + lane * kLine + y;
      const double x = sums[min(at, segments - 1)];
      add[y] = at < segments ? x : 0.;
    }
  };
  auto scan = [&]() {
    run = 0.;
#pragma unroll
    for (int y = 0; y < kLine; ++y) run += add[y];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double y = __shfl_up(run, o);
      if (lane >= o) run += y;
    }
  };
  load((segments - 1) / kRound * kRound);
  const float u = p.u[(size_t)i * (p.n + 1) + p.n];
  const int draft = lane < p.n ? p.drafts[(size_t)i * p.n + lane] : -1;
  const Choice c = choice[i];
  const Rest r(p, i, c);
  scan();
  double total = __shfl(run, 63);
  for (int x0 = ((segments - 1) / kRound - 1) * kRound; x0 >= 0; x0 -= kRound) {
    load(x0);
    scan();
    total += __shfl(run, 63);
  }
  int token;
  if (total > 0.) {
    const double goal = (double)u * total;
    // the segment in which the running sum exceeds the goal; past all of them (u is not below 1): the last that has anything
    double before = 0.;
    int segment = 0;
    bool inside = false;
    for (int x0 = 0;;) {
      double to = __shfl_up(run, 1), found_before = 0.;
      to = before + (lane == 0 ? 0. : to);
      int found = -1, last = -1;
#pragma unroll
      for (int y = 0; y < kLine; ++y) {
        if (add[y] > 0.) {
          last = x0 + lane * kLine + y;
          if (found < 0 && to + add[y] > goal) { found = last; found_before = to; }
        }
        to += add[y];
      }
      const unsigned long long those = __ballot(found >= 0), any = __ballot(last >= 0);
      if (those != 0) {
        const int at = __ffsll(those) - 1;
        segment = __shfl(found, at);
        before = __shfl(found_before, at);
        inside = true;
        break;
      }
      if (any != 0) segment = __shfl(last, 63 - __clzll(any));
      before += __shfl(run, 63);
      x0 += kRound;
      if (x0 >= segments) break;
      load(x0);
      scan();
    }
    const Four left(r, Logits<64, 4>(r.x, segment, p.vocab), [&]() { return Logits<64, 4>(r.y, segment, p.vocab); });      // (a chunk of 64 threads: a segment)
    token = left.token(before, inside ? goal : INFINITY);
  } else {                                                 // nothing to draw from: the largest logit
    token = largest<64>(r.x, p.vocab, s_most, s_at);
  }
  write_tokens<64>(p, i, c.accepted, token, draft);
}

// Rows that one workgroup's threads hold, four logits each of the target's and the draft's: what is left of the row that decides stays in registers, and the
// token is drawn from them: the waves' sums in order give the one that holds the goal, and it finds the token.  ALONE: the rows' sums as well, a wave a row.
constexpr int kNear = 1024, kNearEach = 4;         // threads, logits of one
constexpr int kAloneRows = 128;                    // rows of a sequence, at most
template <bool ALONE>
__global__ __launch_bounds__(kNear)
void verify_near_kernel(Verify p, int chunks, int rows, const ChunkStats* stats) {
  constexpr int kWaves = kNear / 64;
  __shared__ ChooseLds lds;
  __shared__ ChunkStats s_rows[ALONE ? kAloneRows : 1];
  __shared__ double s_sum[kWaves];
  __shared__ float s_most[kWaves];
  __shared__ int s_at[kWaves], s_token;
  const int i = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int draft = tid < p.n ? p.drafts[(size_t)i * p.n + tid] : -1;
  const float u = p.u[(size_t)i * (p.n + 1) + p.n];
  const ChunkStats* mine = stats + (size_t)i * rows * chunks;
  if constexpr (ALONE) {
    const int count = drafts_of(p, i);
    const double per = per_of(p);
    for (int row = wave; row < rows; row += kWaves) {
      const bool drafted = row > p.n;
      const int j = drafted ? row - p.n - 1 : row;
      if (drafted ? j >= count : j > count) continue;
      const float* x = drafted ? p.draft_logits + ((size_t)i * p.n + j) * p.vocab : p.logits + ((size_t)i * (p.n + 1) + j) * p.vocab;
      auto four = [&](int v0, float (&y)[4]) {             // (loads without branches around them: all on their way at once)
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = x[min(v0 + 64 * e, p.vocab - 1)];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = v0 + 64 * e < p.vocab ? tame(y[e]) : -INFINITY;
      };
      float y[4], most = -INFINITY;
      for (int v = lane; v < p.vocab; v += 256) {
        four(v, y);
        most = fmaxf(most, fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])));
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
      double sum = 0.;
      for (int v = lane; v < p.vocab; v += 256) {
        four(v, y);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += weight(y[e], most, per);
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
      if (lane == 0) s_rows[row] = ChunkStats{sum, most, 0};
    }
    mine = s_rows;
    __syncthreads();
  }
  const Choice c = choose<false, kNear>(p, i, ALONE ? 1 : chunks, mine, &lds);
  const Rest r(p, i, c);
  const Four left(r, Logits<kNear, kNearEach>(r.x, 0, p.vocab), [&]() { return Logits<kNear, kNearEach>(r.y, 0, p.vocab); });
  if (lane == 63) s_sum[wave] = left.upto;
  __syncthreads();
  const double mine_all = lane < kWaves ? s_sum[lane] : 0.;      // lane w: wave w's
  double run = mine_all;
#pragma unroll
  for (int o = 1; o < kWaves; o <<= 1) {
    const double y = __shfl_up(run, o);
    if (lane >= o) run += y;
  }
  const double total = __shfl(run, kWaves - 1);
  int token;
  if (total > 0.) {
    // the wave in whose tokens the running sum exceeds the goal; past all of them (u is not below 1): the last that has anything
    const double goal = (double)u * total;
    const unsigned long long those = __ballot(mine_all > 0. && run > goal), any = __ballot(mine_all > 0.);
    const bool inside = those != 0;
    const int segment = inside ? __ffsll(those) - 1 : 63 - __clzll(any);
    const double before = __shfl(run - mine_all, segment);
    if (wave == segment) {
      token = left.token(before, inside ? goal : INFINITY);
      if (lane == 0) s_token = token;
    }
    __syncthreads();
    token = s_token;
  } else {
    token = largest<kNear>(r.x, p.vocab, s_most, s_at);
  }
  write_tokens<kNear>(p, i, c.accepted, token, draft);
}

template <bool ALONE>
static void launch_near(const Verify& p, int chunks, int rows, const ChunkStats* stats, hipStream_t st) {
  hipLaunchKernelGGL(verify_near_kernel<ALONE>, dim3((unsigned)p.b), dim3(kNear), 0, st, p, chunks, rows, stats);
}

// Logits of a thread: half as many where the chunks would not be one for every compute unit (one sequence, four drafts, 32768 tokens: 21.8 us, so 19.9; above 256 of them no difference, above 4000 slower).
int verify_each(int b, int n, int vocab) {
  const long long chunks = (vocab + kThreads * kEach - 1) / (kThreads * kEach);
  return (long long)b * (2 * n + 1) * chunks <= 256 ? kEach / 2 : kEach;
}
int verify_chunks(int vocab, int each) { return (vocab + kThreads * each - 1) / (kThreads * each); }

template <bool GREEDY>
hipError_t launch_stats(const Verify& p, int each, int chunks, int rows, ChunkStats* stats, hipStream_t st) {
  const dim3 grid((unsigned)((size_t)p.b * rows * chunks)), block(kThreads);
  if (each == kEach) hipLaunchKernelGGL((verify_stats_kernel<GREEDY, kEach>), grid, block, 0, st, p, chunks, rows, stats);
  else hipLaunchKernelGGL((verify_stats_kernel<GREEDY, kEach / 2>), grid, block, 0, st, p, chunks, rows, stats);
  return hipGetLastError();
}

}  // namespace

size_t verify_workspace_bytes(int b, int n, int vocab) {
  const int each = verify_each(b, n, vocab);
  const size_t chunks = verify_chunks(vocab, each);
  return (size_t)b * ((2 * (size_t)n + 1) * chunks * sizeof(ChunkStats) + sizeof(Choice) + chunks * each * sizeof(double));
}

hipError_t launch_verify(const Verify& p, void* workspace, hipStream_t st) {
  const int each = verify_each(p.b, p.n, p.vocab), chunks = verify_chunks(p.vocab, each), rows = p.draft_logits && p.temperature > 0.f ? 2 * p.n + 1 : p.n + 1;
  ChunkStats* stats = static_cast<ChunkStats*>(workspace);
  Choice* choice = reinterpret_cast<Choice*>(stats + (size_t)p.b * rows * chunks);
  double* rest = reinterpret_cast<double*>(choice + p.b);
  const dim3 rests((unsigned)((size_t)p.b * chunks)), per_sequence((unsigned)p.b), block(kThreads);
  if (!(p.temperature > 0.f)) {
    const hipError_t e = launch_stats<true>(p, each, chunks, rows, stats, st);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(verify_greedy_kernel, per_sequence, block, 0, st, p, chunks, rows, stats);
    return hipGetLastError();
  }
  // One launch where the rows that a wave has in turn are short (four drafts, 300 tokens: 8.2 us, in two launches 9.8; of 2000 10.6 and 10.3), and for more
  // where the sequences are many (256 of two rows of 2000: 11.9 and 13.1; of 4000 19.5 and 14.2).
  static_assert(2048 <= kNear * kNearEach, "rows that the threads hold");
  if (rows <= kAloneRows && (long long)((rows + 15) / 16) * p.vocab <= (p.b >= 128 ? 2048 : 1024)) {
    launch_near<true>(p, chunks, rows, stats, st);
    return hipGetLastError();
  }
  hipError_t e = launch_stats<false>(p, each, chunks, rows, stats, st);
  if (e != hipSuccess) return e;
  // (two launches for three: four drafts, 4096 tokens 10.5 us and 12.5, 64 sequences 13.2 and 17.2; 16384 tokens, 16 a thread, 15.6 and 13.2)
  if (p.vocab <= kNear * kNearEach) {
    launch_near<false>(p, chunks, rows, stats, st);
    return hipGetLastError();
  }
  if (each == kEach) hipLaunchKernelGGL(verify_rest_kernel<kEach>, rests, block, 0, st, p, chunks, rows, stats, rest, choice);
  else hipLaunchKernelGGL(verify_rest_kernel<kEach / 2>, rests, block, 0, st, p, chunks, rows, stats, rest, choice);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(verify_draw_kernel, per_sequence, dim3(64), 0, st, p, chunks * each, rest, choice);
  return hipGetLastError();
}

}  // namespace mqa
