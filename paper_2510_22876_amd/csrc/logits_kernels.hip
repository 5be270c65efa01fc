// Penalties for repeated tokens, biases and grammar masks on the logits of a
// verify window, ahead of verification (gfx950, wave64).  For logit x of token
// v in window slot r, with n(v) the occurrences of v among the answered tokens
// and the drafts before slot r, and held(v) whether v occurs at all (prompt
// included):
//
//   x = held ? (x > 0 ? x / repetition : x * repetition) : x
//   x = x - (frequency * n + presence * [n > 0])
//   x = x + bias(v)
//   x = allowed(v) ? x : -inf
//
// A workgroup takes one sequence and one chunk of the vocabulary and walks the
// window's slots: the counts of its chunk, built once from the token row in
// LDS, serve every slot, and each slot's draft is counted before the next.
#include "forward_common.h"

namespace specdec {
namespace {

constexpr uint32_t kBadPadIn = 0x1u, kEmptyMask = 0x80u;
constexpr uint32_t kPrompt = 0x80000000u;   // the token occurs in the prompt; the low bits count the answered ones
constexpr int kChunk = 4096;

struct LogitsArgs {
  LogitsLaunch p;
  int64_t base;      // first workgroup of this launch
  int64_t chunks;    // of the vocabulary
};

template <int kDtype>
__global__ __launch_bounds__(kThreads) void logits_kernel(LogitsArgs a) {
  typedef typename Element<kDtype>::type T;
  __shared__ uint32_t s_n[kChunk];
  __shared__ float s_bias[kChunk];
  const LogitsLaunch& p = a.p;
  const int64_t block = a.base + blockIdx.x, chunk = block % a.chunks, v0 = chunk * kChunk;
  const int i = static_cast<int>(block / a.chunks), tid = threadIdx.x;
  const int size = static_cast<int>(p.V - v0 < kChunk ? p.V - v0 : kChunk);
  const bool penal = p.repetition || p.presence || p.frequency;
  int64_t begin = 0, end = p.width, answered = 0;   // columns of the history; the first behind the prompt
  if (penal) {
    if (p.begin) begin = p.begin[i];
    if (p.lens) end = p.lens[i];
    if (begin < 0 || begin > end || end >= p.s_stride) {
      if (chunk == 0 && tid == 0 && p.dev_status) atomicOr(p.dev_status, kBadPadIn);
      return;
    }
  }
  for (int j = tid; j < size; j += kThreads) {
    s_n[j] = 0;
    s_bias[j] = 0.f;
  }
  __syncthreads();
  if (penal) {
    const int32_t* s = p.s + i * p.s_stride;
    answered = begin + (p.prompt ? p.prompt[i] : 0);
    for (int64_t j = begin + tid; j <= end; j += kThreads) {
      const int64_t v = s[j] - v0;
      if (v < 0 || v >= size) continue;
      if (j < answered) atomicOr(&s_n[v], kPrompt);
      else atomicAdd(&s_n[v], 1u);
    }
  }
  const int32_t* ids = p.bias_ids + static_cast<int64_t>(i) * p.n_bias;
  const float* bias = p.bias + static_cast<int64_t>(i) * p.n_bias;
  for (int j = tid; j < p.n_bias; j += kThreads) {
    const int64_t v = ids[j] - v0;
    if (v < 0 || v >= size) continue;
    // an id given more than once: its first place adds them up, in their order
    bool first = true;
    for (int e = 0; e < j; ++e) first = first && ids[e] != ids[j];
    if (!first) continue;
    float sum = bias[j];
    for (int e = j + 1; e < p.n_bias; ++e)
      if (ids[e] == ids[j]) sum += bias[e];
    s_bias[v] = sum;
  }
  const float rep = p.repetition ? p.repetition[i] : 1.f, pres = p.presence ? p.presence[i] : 0.f;
  const float freq = p.frequency ? p.frequency[i] : 0.f;
  const bool in_place = p.out == p.logits;
  for (int r = 0; r <= p.k; ++r) {
    __syncthreads();
    const int64_t row = static_cast<int64_t>(i) * (p.k + 1) + r;
    const T* x = static_cast<const T*>(p.logits) + row * p.V + v0;
    T* y = static_cast<T*>(p.out) + row * p.V + v0;
    const uint32_t* mask = p.mask ? p.mask + row * p.mask_stride : nullptr;
    for (int j = tid; j < size; j += kThreads) {
      const int64_t v = v0 + j;
      if (mask && !(mask[v >> 5] >> (v & 31) & 1u)) {
        y[j] = static_cast<T>(-__builtin_inff());
        continue;
      }
      const uint32_t n = s_n[j];
      if (in_place && n == 0 && s_bias[j] == 0.f) continue;
      float z = static_cast<float>(x[j]);
      if (p.repetition && n) z = z > 0.f ? z / rep : z * rep;
      const uint32_t told = n & ~kPrompt;
      if (told) z -= freq * static_cast<float>(told) + pres;
      y[j] = static_cast<T>(z + s_bias[j]);
    }
    if (mask && chunk == 0) {   // a slot that allows nothing
      int any = 0;
      for (int64_t w = tid; w * 32 < p.V; w += kThreads) {
        const uint32_t bits = p.V - w * 32 >= 32 ? ~0u : (1u << (p.V - w * 32)) - 1u;
        any |= (mask[w] & bits) != 0;
      }
      if (!__syncthreads_or(any) && tid == 0 && p.dev_status) atomicOr(p.dev_status, kEmptyMask);
    }
    __syncthreads();
    if (penal && r < p.k && tid == 0) {
      const int64_t v = p.draft[static_cast<int64_t>(i) * p.k + r] - v0;
      if (v >= 0 && v < size) {
        if (end + 1 + r < answered) s_n[v] |= kPrompt;
        else s_n[v] += 1u;
      }
    }
  }
}

}  // namespace

hipError_t launch_logits(const LogitsLaunch& p, hipStream_t stream) {
  LogitsArgs a{p, 0, (static_cast<int64_t>(p.V) + kChunk - 1) / kChunk};
  return launch_blocks(p.B * a.chunks, kThreads, [&](int64_t at, uint32_t n) {
    a.base = at;
    if (p.dtype == 0) logits_kernel<0><<<n, kThreads, 0, stream>>>(a);
    else if (p.dtype == 1) logits_kernel<1><<<n, kThreads, 0, stream>>>(a);
    else logits_kernel<2><<<n, kThreads, 0, stream>>>(a);
  });
}

}  // namespace specdec
