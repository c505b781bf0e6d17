// HIP kernel of the adjustments of logits for gfx950: penalties for tokens that occurred, biases, masks.
#include "ops.h"
#include "dev.h"
#include <algorithm>

namespace sprinter {

// What is known of a token stands in one word of LDS: how often it was generated (20 bits), whether it is in the prompt (1), and which of the bias
// list's entries is its (11, 0 none).  The entries come first, while the words are 0, so that the largest index wins whatever the order.
constexpr unsigned PROMPT = 1u << 20, BIAS_SHIFT = 21;
constexpr int SLICE = 4096;

// One row and SLICE tokens of the vocabulary per workgroup.
template <typename T>
__global__ __launch_bounds__(256) void k_adjust_logits(sprinter_logits a) {
  __shared__ unsigned word[SLICE];
  const int t = blockIdx.y, v0 = blockIdx.x * SLICE, n = min(SLICE, a.vocab - v0);
  int b = t, f0 = t, f1 = t + 1;
  if (a.first) {
    int lo = 0, hi = a.n_seq;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.first[mid] <= t) lo = mid; else hi = mid;
    }
    b = lo; f0 = a.first[lo]; f1 = min(a.first[lo + 1], a.n_rows);
    if (t < f0 || t >= f1) b = -1;
  }
  for (int i = threadIdx.x; i < SLICE; i += 256) word[i] = 0;
  __syncthreads();
  float rep = 1.f, pre = 0.f, freq = 0.f;
  if (b >= 0) {
    if (a.repetition) rep = a.repetition[b];
    if (a.presence) pre = a.presence[b];
    if (a.frequency) freq = a.frequency[b];
    if (a.bias_ids) {
      for (int i = threadIdx.x; i < a.n_bias; i += 256) {
        const int v = a.bias_ids[b * a.ld_bias_ids + i];
        if (v >= v0 && v - v0 < n) atomicMax(&word[v - v0], (unsigned)(i + 1) << BIAS_SHIFT);
      }
      __syncthreads();
    }
    if (a.tokens) {
      const int made = a.n_prompt ? a.n_prompt[b] : 0, end = a.n_token ? min(a.n_token[b], a.n_tokens) : a.n_tokens;
      for (int i = threadIdx.x; i < end; i += 256) {
        const int v = a.tokens[b * a.ld_tokens + i];
        if (v >= v0 && v - v0 < n) {
          if (i < made) atomicOr(&word[v - v0], PROMPT); else atomicAdd(&word[v - v0], 1u);
        }
      }
    }
    if (a.draft) {
      const int nodes = a.visible ? min(f1 - f0, 64 * a.n_words) : t - f0 + 1;
      for (int j = threadIdx.x; j < nodes; j += 256) {
        if (a.visible && !(a.visible[(long long)t * a.n_words + (j >> 6)] >> (j & 63) & 1)) continue;
        const int v = a.draft[f0 + j];
        if (v >= v0 && v - v0 < n) atomicAdd(&word[v - v0], 1u);
      }
    }
    __syncthreads();
  }
  const int row = a.mask ? (a.mask_row ? a.mask_row[t] : t) : -1;
  const int* mask = row >= 0 && row < a.n_mask ? a.mask + row * a.ld_mask : nullptr;
  const T* in = (const T*)a.logits + t * a.ld_logits + v0;
  T* out = (T*)a.out + t * a.ld_out + v0;
  for (int i = threadIdx.x; i < n; i += 256) {
    float x;
    if constexpr (sizeof(T) == 4) x = in[i]; else x = __uint_as_float((unsigned)in[i] << 16);
    const unsigned w = word[i];
    if (w) {
      const unsigned times = w & (PROMPT - 1), entry = w >> BIAS_SHIFT;
      if ((w & (2 * PROMPT - 1)) && a.repetition) x = x > 0.f ? x / rep : x * rep;
      if (times) x = x - freq * (float)times - pre;
      if (entry) x += a.bias[b * a.ld_bias + entry - 1];
    }
    if (mask && !(mask[(v0 + i) >> 5] >> ((v0 + i) & 31) & 1)) x = -INFINITY;
    if constexpr (sizeof(T) == 4) out[i] = x; else out[i] = f2bf(x);
  }
}

void launch_adjust_logits(const sprinter_logits& a, hipStream_t s) {
  const dim3 grid((a.vocab + SLICE - 1) / SLICE, a.n_rows);
  if (a.dtype == SPRINTER_F32) hipLaunchKernelGGL(k_adjust_logits<float>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(k_adjust_logits<bf16_t>, grid, dim3(256), 0, s, a);
}

}  // namespace sprinter
