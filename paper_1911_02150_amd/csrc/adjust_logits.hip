// Logits with penalties for repeated tokens, biases and the tokens that are allowed.
//
// Of row j of sequence i, token t: c: how often t is among the tokens that the sequence has from prompts[i] on and the drafts before row j; seen: whether it is among
// all that it has and those drafts.
//   x = logit;  seen: x = x > 0 ? x / repetition : x * repetition;  c > 0: x -= frequency c + presence;  x += bias;  not allowed: x = -infinity
// A workgroup has kTokens of a sequence's vocabulary and counts the sequence's tokens among them in LDS, once; then a thread has its eight tokens' counts and biases in registers and goes
// over the rows, a row's logits on their way while the one before is adjusted.  What bounds it is HBM: 8 bytes a logit, and 4 a token of the history for each kTokens of the
// vocabulary, from L2.
#include "paged.hpp"

namespace mqa {
namespace {

constexpr int kTokens = 2048, kMine = kTokens / 256;
constexpr uint32_t kSeen = 0x80000000u;      // in a token's count: the prompt has it

template <int EACH>                          // neighbouring logits of a thread: 4, or 1 where rows are not on 16 bytes
__global__ __launch_bounds__(256)
void adjust_kernel(AdjustLogits p, int chunks) {
  constexpr int GROUPS = kMine / EACH;
  __shared__ __align__(16) uint32_t s_count[kTokens];
  __shared__ __align__(16) uint32_t s_bias[kTokens];       // 1 + the last of a token's biases
  const int tid = threadIdx.x, i = (int)(blockIdx.x / (unsigned)chunks), first = ((int)blockIdx.x - i * chunks) * kTokens;
  const int tokens = min(kTokens, p.vocab - first);
  const int words = (p.vocab + 31) >> 5;
  struct Row { float y[GROUPS][EACH]; uint32_t allowed[GROUPS]; };
  const size_t row0 = (size_t)i * (p.n + 1);
  auto load = [&](int j, Row* r) {
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) {
      const int x = min(EACH * (tid + 256 * k), tokens - EACH);        // (past the end: some other logits, which are not stored)
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
  load(0, &next);
  for (int x = tid; x < kTokens; x += 256) {
    s_count[x] = 0;
    s_bias[x] = 0;
  }
  __syncthreads();
  const int len = min(max(p.lens[i], 0), p.cap), prompt = p.prompts ? p.prompts[i] : 0;
  const int32_t* const history = p.history + (size_t)i * p.cap;
  for (int base = tid; base < len; base += 8 * 256) {
    unsigned t[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) t[u] = (unsigned)history[min(base + 256 * u, len - 1)] - (unsigned)first;
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (t[u] < (unsigned)tokens && base + 256 * u < len) {
        if (base + 256 * u < prompt) atomicOr(&s_count[t[u]], kSeen);
        else atomicAdd(&s_count[t[u]], 1u);
      }
  }
  for (int x = tid; x < p.biases; x += 256) {
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
      const int x = EACH * (tid + 256 * k) + z;
      count[k][z] = s_count[x];
      const uint32_t b = s_bias[x];
      bias[k][z] = b ? p.bias_values[(size_t)i * p.biases + b - 1] : 0.f;
    }
  for (int j = 0; j <= p.n; ++j) {
    Row row = next;
    if (j < p.n) load(j + 1, &next);
    if (j > 0) {
      const int t = (int)((unsigned)p.drafts[(size_t)i * p.n + j - 1] - (unsigned)first);
#pragma unroll
      for (int k = 0; k < GROUPS; ++k)
#pragma unroll
        for (int z = 0; z < EACH; ++z) count[k][z] += t == EACH * (tid + 256 * k) + z;      // (a token outside the vocabulary is none of these, or past the end)
    }
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) {
      const int x = EACH * (tid + 256 * k);
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

hipError_t launch_adjust(const AdjustLogits& p, hipStream_t st) {
  const int chunks = (p.vocab + kTokens - 1) / kTokens;
  if (p.vocab % 4 == 0) hipLaunchKernelGGL(adjust_kernel<4>, dim3((unsigned)(p.b * chunks)), dim3(256), 0, st, p, chunks);
  else hipLaunchKernelGGL(adjust_kernel<1>, dim3((unsigned)(p.b * chunks)), dim3(256), 0, st, p, chunks);
  return hipGetLastError();
}

}  // namespace mqa
