// Logits with penalties for repeated tokens, biases and the tokens that are allowed.
//
// Of row j of sequence i, token t: c: how often t is among the tokens that the sequence has from prompts[i] on and the drafts before row j; seen: whether it is among
// all that it has and those drafts.
//   x = logit;  seen: x = x > 0 ? x / repetition : x * repetition;  c > 0: x -= frequency c + presence;  x += bias;  not allowed: x = -infinity
// A workgroup has eight tokens a thread of a sequence's vocabulary and counts the sequence's tokens among them in LDS, once; then a thread has its tokens' counts and biases in registers and
// goes over the rows, a row's logits on their way while the one before is adjusted.  What bounds it is HBM, 8 bytes a logit (64 sequences, five rows of 32768, histories of 8192: 84 MB, 21.0 us = 4.0 TB/s
// with reads from L2 of 34 MB of histories for each 2048 tokens of the vocabulary), and for one sequence the launch and three reads in a row (4.4 us; with a history of 131072, which every workgroup
// reads, 17).  Rows of any length are read and written by 4 bytes (32767: 28.8 us).
#include "paged.hpp"

namespace mqa {
namespace {

constexpr int kMine = 8;
constexpr uint32_t kSeen = 0x80000000u;      // in a token's count: the prompt has it, and nothing else

template <int EACH, int THREADS>             // EACH: neighbouring logits of a thread: 4, or 1 where rows are not on 16 bytes
__global__ __launch_bounds__(THREADS)
void adjust_kernel(AdjustLogits p, int chunks, int each) {
  constexpr int GROUPS = kMine / EACH, kTokens = kMine * THREADS;
  extern __shared__ __align__(16) uint32_t s_count[];      // [kTokens] behind the prompt, [kTokens] in it
  uint32_t* const s_bias = s_count + 2 * kTokens;          // where there are biases, [kTokens]: 1 + the last of a token's
  const int tid = threadIdx.x, i = (int)(blockIdx.x / (unsigned)chunks), first = ((int)blockIdx.x - i * chunks) * kTokens;
  const int begin = (int)blockIdx.y * each, end = min(begin + each, p.n + 1);      // rows
  const int tokens = min(kTokens, p.vocab - first);
  const int words = (p.vocab + 31) >> 5;
  struct Row { float y[GROUPS][EACH]; uint32_t allowed[GROUPS]; };
  const size_t row0 = (size_t)i * (p.n + 1);
  auto load = [&](int j, Row* r) {
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) {
      const int x = min(EACH * (tid + THREADS * k), tokens - EACH);        // (past the end: some other logits, which are not stored)
      const float* const at = p.logits + (row0 + j) * p.vocab + first + x;
      if constexpr (EACH == 4) {
        const float4 v = *reinterpret_cast<const float4*>(at);
        r->y[k][0] = v.x; r->y[k][1] = v.y; r->y[k][2] = v.z; r->y[k][3] = v.w;
      } else {
        r->y[k][0] = *at;
      }
      r->allowed[k] = p.allowed ? p.allowed[(row0 + j) * words + ((first + x) >> 5)] >> ((first + x) & 31) : ~0u;
    }
  };
  Row next;
  load(begin, &next);
  // The history, four tokens a load from 16 bytes on (which may hold others before the row's first), four loads on their way, the first ones before the length is here.
  const int skew = (int)((size_t)i * p.cap & 3), last4 = (int)(((long long)p.cap + skew) >> 2) - 1;
  const int4* const history4 = reinterpret_cast<const int4*>(p.history + ((size_t)i * p.cap - skew));
  int4 y[4];
  if (last4 >= 0)
#pragma unroll
    for (int u = 0; u < 4; ++u) y[u] = history4[min(tid + u * THREADS, last4)];
  for (int x = tid; x < kTokens; x += THREADS) s_count[x] = s_count[kTokens + x] = 0;
  if (p.biases)
    for (int x = tid; x < kTokens; x += THREADS) s_bias[x] = 0;
  __syncthreads();
  const int len = min(max(p.lens[i], 0), p.cap), prompt = p.prompts ? p.prompts[i] : 0;
  const int32_t* const history = p.history + (size_t)i * p.cap;
  auto count_one = [&](int token, int at) {
    const unsigned x = (unsigned)token - (unsigned)first;
    if (x < (unsigned)tokens && (unsigned)at < (unsigned)len) atomicAdd(&s_count[at < prompt ? kTokens + x : x], 1u);
  };
  const int fours = (len + skew) >> 2;
  for (int base = tid; base < fours; base += 4 * THREADS) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int x = base + u * THREADS, at = x < fours ? 4 * x - skew : len;
      count_one(y[u].x, at);
      count_one(y[u].y, at + 1);
      count_one(y[u].z, at + 2);
      count_one(y[u].w, at + 3);
    }
    if (base + 4 * THREADS < fours)
#pragma unroll
      for (int u = 0; u < 4; ++u) y[u] = history4[min(base + (4 + u) * THREADS, last4)];
  }
  if (tid < (len + skew) - 4 * fours && 4 * fours - skew + tid >= 0) count_one(history[4 * fours - skew + tid], 4 * fours - skew + tid);
  for (int x = tid; x < begin; x += THREADS) {             // drafts before the first row
    const unsigned t = (unsigned)p.drafts[(size_t)i * p.n + x] - (unsigned)first;
    if (t < (unsigned)tokens) atomicAdd(&s_count[t], 1u);
  }
  for (int x = tid; x < p.biases; x += THREADS) {
    const unsigned t = (unsigned)p.bias_tokens[(size_t)i * p.biases + x] - (unsigned)first;
    if (t < (unsigned)tokens) atomicMax(&s_bias[t], (uint32_t)x + 1);
  }
  const float repetition = p.repetition ? p.repetition[i] : 1.f, frequency = p.frequency ? p.frequency[i] : 0.f, presence = p.presence ? p.presence[i] : 0.f;
  __syncthreads();
  uint32_t count[GROUPS][EACH];
  float bias[GROUPS][EACH];
#pragma unroll
  for (int k = 0; k < GROUPS; ++k)
#pragma unroll
    for (int z = 0; z < EACH; ++z) {
      const int x = EACH * (tid + THREADS * k) + z;
      count[k][z] = s_count[x] | (s_count[kTokens + x] ? kSeen : 0);
      bias[k][z] = 0.f;
    }
  if (p.biases)
#pragma unroll
    for (int k = 0; k < GROUPS; ++k)
#pragma unroll
      for (int z = 0; z < EACH; ++z) {
        const uint32_t b = s_bias[EACH * (tid + THREADS * k) + z];
        if (b) bias[k][z] = p.bias_values[(size_t)i * p.biases + b - 1];
      }
  for (int j = begin; j < end; ++j) {
    Row row = next;
    if (j + 1 < end) load(j + 1, &next);
    if (j > begin) {
      const int t = (int)((unsigned)p.drafts[(size_t)i * p.n + j - 1] - (unsigned)first);
#pragma unroll
      for (int k = 0; k < GROUPS; ++k)
#pragma unroll
        for (int z = 0; z < EACH; ++z) count[k][z] += t == EACH * (tid + THREADS * k) + z;      // (a token outside the vocabulary is none of these, or past the end)
    }
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) {
      const int x = EACH * (tid + THREADS * k);
      if (x >= tokens) continue;
#pragma unroll
      for (int z = 0; z < EACH; ++z) {
        float y = row.y[k][z];
        if (const uint32_t c = count[k][z]) {
          y = y > 0.f ? y / repetition : y * repetition;
          if (const uint32_t often = c & ~kSeen) y -= frequency * (float)often + presence;
        }
        if (bias[k][z] != 0.f) y += bias[k][z];
        if (!(row.allowed[k] >> z & 1)) y = -INFINITY;
        row.y[k][z] = y;
      }
      float* const at = p.out + (row0 + j) * p.vocab + first + x;
      if constexpr (EACH == 4) *reinterpret_cast<float4*>(at) = make_float4(row.y[k][0], row.y[k][1], row.y[k][2], row.y[k][3]);
      else *at = row.y[k][0];
    }
  }
}

}  // namespace

// Rows go to several workgroups, which count the history each, where there are few (4 sequences, 16 rows of 50257: 39.9 us by one, 12.8).
constexpr long long kEnough = 512 * 256;
template <int EACH, int THREADS>
static void launch_chunks(const AdjustLogits& p, hipStream_t st) {
  const int chunks = (p.vocab + kMine * THREADS - 1) / (kMine * THREADS);
  const long long groups = (long long)p.b * chunks;
  int each = p.n + 1;
  while (each > 1 && groups * ((p.n + each) / each) * THREADS < kEnough) each = (each + 1) / 2;
  hipLaunchKernelGGL((adjust_kernel<EACH, THREADS>), dim3((unsigned)groups, (unsigned)((p.n + each) / each)), dim3(THREADS), (size_t)kMine * THREADS * 4 * (p.biases ? 3 : 2), st, p,
                     chunks, each);
}

// Twice the threads, so that half as many workgroups read the history, where it is long beside a workgroup's rows (256 / 512 threads: 64 sequences, a history of 8192, one row 8.7 / 7.3 us, five
// 21.0 / 21.3; one sequence, 131072 27.5 / 17.1, 1024 4.6 / 4.8; 256 sequences, 4096 18.7 / 19.4).
hipError_t launch_adjust(const AdjustLogits& p, hipStream_t st) {
  const bool wide = p.cap / (p.n + 1) > 4096, fours = p.vocab % 4 == 0;
  if (fours) wide ? launch_chunks<4, 512>(p, st) : launch_chunks<4, 256>(p, st);
  else wide ? launch_chunks<1, 512>(p, st) : launch_chunks<1, 256>(p, st);
  return hipGetLastError();
}

}  // namespace mqa
