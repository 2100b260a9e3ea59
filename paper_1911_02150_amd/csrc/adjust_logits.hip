// Logits with penalties for repeated tokens, biases and the tokens that are allowed.
//
// Of row j of sequence i, token t: c: how often t is among the tokens that the sequence has from prompts[i] on and the drafts before row j; seen: whether it is among
// all that it has and those drafts.
//   x = logit;  seen: x = x > 0 ? x / repetition : x * repetition;  c > 0: x -= frequency c + presence;  x += bias;  not allowed: x = -infinity
// A workgroup has kTokens of a sequence's vocabulary, counts the sequence's tokens among them in LDS once, and goes over the rows, adding a draft at a time.
#include "paged.hpp"

namespace mqa {
namespace {

constexpr int kTokens = 2048;
constexpr uint32_t kSeen = 0x80000000u;      // in a token's count: the prompt has it

template <int EACH>                          // neighbouring logits of a thread: 4, or 1 where rows are not on 16 bytes
__global__ __launch_bounds__(256)
void adjust_kernel(AdjustLogits p, int chunks) {
  __shared__ uint32_t s_count[kTokens];
  __shared__ uint32_t s_bias[kTokens];       // 1 + the last of a token's biases
  const int tid = threadIdx.x, i = (int)(blockIdx.x / (unsigned)chunks), first = ((int)blockIdx.x - i * chunks) * kTokens;
  const int tokens = min(kTokens, p.vocab - first);
  for (int x = tid; x < kTokens; x += 256) {
    s_count[x] = 0;
    s_bias[x] = 0;
  }
  __syncthreads();
  const int len = min(max(p.lens[i], 0), p.cap), prompt = p.prompts ? p.prompts[i] : 0;
  for (int x = tid; x < len; x += 256) {
    const unsigned t = (unsigned)p.history[(size_t)i * p.cap + x] - (unsigned)first;
    if (t < (unsigned)tokens) {
      if (x < prompt) atomicOr(&s_count[t], kSeen);
      else atomicAdd(&s_count[t], 1u);
    }
  }
  for (int x = tid; x < p.biases; x += 256) {
    const unsigned t = (unsigned)p.bias_tokens[(size_t)i * p.biases + x] - (unsigned)first;
    if (t < (unsigned)tokens) atomicMax(&s_bias[t], (uint32_t)x + 1);
  }
  const float repetition = p.repetition ? p.repetition[i] : 1.f, frequency = p.frequency ? p.frequency[i] : 0.f, presence = p.presence ? p.presence[i] : 0.f;
  const int words = (p.vocab + 31) >> 5;
  for (int j = 0; j <= p.n; ++j) {
    __syncthreads();
    if (j > 0) {
      const unsigned t = (unsigned)p.drafts[(size_t)i * p.n + j - 1] - (unsigned)first;
      if (t < (unsigned)tokens && tid == 0) s_count[t] += 1;
      __syncthreads();
    }
    const size_t row = (size_t)i * (p.n + 1) + j;
    for (int x = EACH * tid; x < tokens; x += EACH * 256) {
      const size_t at = row * p.vocab + first + x;
      float y[EACH];
      if constexpr (EACH == 4) *reinterpret_cast<float4*>(y) = *reinterpret_cast<const float4*>(p.logits + at);
      else y[0] = p.logits[at];
      const uint32_t allowed = p.allowed ? p.allowed[row * words + ((first + x) >> 5)] >> ((first + x) & 31) : ~0u;
#pragma unroll
      for (int z = 0; z < EACH; ++z) {
        const uint32_t c = s_count[x + z], bias = s_bias[x + z];
        if (c) {
          y[z] = y[z] > 0.f ? y[z] / repetition : y[z] * repetition;
          const uint32_t count = c & ~kSeen;
          if (count) y[z] -= frequency * (float)count + presence;
        }
        if (bias) y[z] += p.bias_values[(size_t)i * p.biases + bias - 1];
        if (!(allowed >> z & 1)) y[z] = -INFINITY;
      }
      if constexpr (EACH == 4) *reinterpret_cast<float4*>(p.out + at) = *reinterpret_cast<const float4*>(y);
      else p.out[at] = y[0];
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
