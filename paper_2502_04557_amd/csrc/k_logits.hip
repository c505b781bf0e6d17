// HIP kernel of the adjustments of logits for gfx950: penalties for tokens that occurred, biases, masks.
#include "ops.h"
#include "dev.h"
#include <algorithm>
#include <type_traits>

namespace sprinter {

// What is known of a token stands in one word of LDS: how often it was generated (20 bits), whether it is in the prompt (1), and which of the bias
// list's entries is its (11, 0 none).  The entries come first, while the words are 0, so that the largest index wins whatever the order.
constexpr unsigned PROMPT = 1u << 20, BIAS_SHIFT = 21;

typedef unsigned Vec4 __attribute__((ext_vector_type(4), aligned(4)));   // 16 bytes at the alignment of one logit
typedef unsigned Vec2 __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ float logit_f32(float v) { return v; }
__device__ __forceinline__ float logit_f32(bf16_t v) { return __uint_as_float((unsigned)v << 16); }
__device__ __forceinline__ void put_logit(float* p, float v) { *p = v; }
__device__ __forceinline__ void put_logit(bf16_t* p, float v) { *p = f2bf(v); }

// The sequence of row t, by a whole wave, 64 places at a time: the last b with first[b] <= t, or -1 where t is no row of it.
__device__ __forceinline__ int row_sequence(const int* first, int n_seq, int n_rows, int t, int& f0, int& f1) {
  const int lane = threadIdx.x & 63;
  int b = 0;
  for (int n = n_seq; n > 0;) {                    // among b .. b + n - 1
    const int stride = (n + 63) >> 6;
    const int below = __popcll(__ballot((long long)lane * stride < n && first[min((long long)b + (long long)lane * stride, (long long)n_seq)] <= t));
    if (below == 0) return -1;
    b += (below - 1) * stride;
    n = stride == 1 ? 0 : min(stride, n - (below - 1) * stride);
  }
  if (n_seq < 1) return -1;
  f0 = max(first[b], 0);
  f1 = min(first[b + 1], n_rows);
  return t >= f0 && t < f1 ? b : -1;
}

// A workgroup takes `slice` tokens of the vocabulary of `per` rows one after the other.  What the history says of those tokens is counted once for all of its
// rows of one sequence; the tokens of a row's path are added for the row and taken out again.  Reads and writes 16 bytes a lane whatever the rows'
// alignment; all but a few words are 0, and their logits go through as they are.  Bound by HBM: 448 rows of 128256 float32, 460 MB in 101 us = 4.6 TB/s, of the 4.7
// that a large copy reaches; counting 2000 tokens of history for every third row is 8 us of them.
// MANY: past the caches (through them, 129 us), slices of up to MANY_SLICE tokens, all of a thread's pieces of a row on their way at once (6 in float32, 3 in bf16); else one
// piece a thread, and the logits stay in L2 for who draws from them.
constexpr int MANY_SLICE = 6144;
template <typename T, bool MANY>
__global__ __launch_bounds__(256) void k_adjust_logits(sprinter_logits a, int slice, int per) {
  extern __shared__ unsigned word[];               // [slice]
  constexpr int VEC = 16 / sizeof(T), RUN = 256 * VEC, UNROLL = MANY ? MANY_SLICE / RUN : 1;   // pieces of a thread: slice <= UNROLL * RUN
  static_assert(MANY_SLICE % RUN == 0, "whole pieces");
  using Vec = std::conditional_t<sizeof(T) == 4, Vec4, Vec2>;
  const int tid = threadIdx.x, v0 = blockIdx.y * slice, n = min(slice, a.vocab - v0), whole = n / VEC * VEC, t1 = min((int)(blockIdx.x + 1) * per, a.n_rows);
  int now = -2, b = -1, f0 = 0, f1 = 0;            // the sequence that the words are of
  float rep = 1.f, pre = 0.f, freq = 0.f;
  Vec x[UNROLL];
  auto fetch = [&](const T* in) {
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int i = tid * VEC + u * RUN;
      if (i >= whole) continue;
      if constexpr (MANY) x[u] = __builtin_nontemporal_load(reinterpret_cast<const Vec*>(in + i));
      else x[u] = *reinterpret_cast<const Vec*>(in + i);
    }
  };
  bool path_in = false;                            // the last row's path is among the words
  auto add_path = [&](int t, unsigned by) {
    const int nodes = a.visible ? min(f1 - f0, 64 * a.n_words) : t - f0 + 1;
    for (int j = tid; j < nodes; j += 256)
      if (!a.visible || (a.visible[(long long)t * a.n_words + (j >> 6)] >> (j & 63) & 1)) {
        const int v = a.draft[f0 + j];
        if (v >= v0 && v - v0 < n) atomicAdd(&word[v - v0], by);
      }
  };
  fetch((const T*)a.logits + (long long)blockIdx.x * per * a.ld_logits + v0);   // (on its way while the tokens are counted)
  for (int t = blockIdx.x * per; t < t1; ++t) {
    const T* in = (const T*)a.logits + t * a.ld_logits + v0;
    T* out = (T*)a.out + t * a.ld_out + v0;
    if (!a.first) { b = t; f0 = t; f1 = t + 1; }
    else if (now < -1 || t >= f1 || b < 0) b = row_sequence(a.first, a.n_seq, a.n_rows, t, f0, f1);
    if (b != now || now < 0) {
      path_in = false;
      for (int i = tid * 4; i < slice; i += 1024) *reinterpret_cast<uint4*>(&word[i]) = make_uint4(0, 0, 0, 0);
      now = b;
      __syncthreads();
      if (b >= 0) {
        if (a.repetition) rep = a.repetition[b];
        if (a.presence) pre = a.presence[b];
        if (a.frequency) freq = a.frequency[b];
        if (a.bias_ids) {
          for (int i = tid; i < a.n_bias; i += 256) {
            const int v = a.bias_ids[b * a.ld_bias_ids + i];
            if (v >= v0 && v - v0 < n) atomicMax(&word[v - v0], (unsigned)(i + 1) << BIAS_SHIFT);
          }
          __syncthreads();
        }
        if (a.tokens) {
          const int made = a.n_prompt ? a.n_prompt[b] : 0, end = a.n_token ? min(a.n_token[b], a.n_tokens) : a.n_tokens;
          const int* tokens = a.tokens + b * a.ld_tokens;
          for (int i0 = tid; i0 < end; i0 += 1024) {
            int v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = i0 + 256 * u < end ? tokens[i0 + 256 * u] : -1;
#pragma unroll
            for (int u = 0; u < 4; ++u)
              if (v[u] >= v0 && v[u] - v0 < n) {
                if (i0 + 256 * u < made) atomicOr(&word[v[u] - v0], PROMPT); else atomicAdd(&word[v[u] - v0], 1u);
              }
          }
        }
      }
      __syncthreads();
    }
    if (a.draft && b >= 0) {                       // (out and in at once: the sums are the same in any order)
      if (path_in) add_path(t - 1, ~0u);
      add_path(t, 1u);
      path_in = true;
      __syncthreads();
    }
    const int row = a.mask ? (a.mask_row ? a.mask_row[t] : t) : -1;
    const int* mask = row >= 0 && row < a.n_mask ? a.mask + row * a.ld_mask : nullptr;
    auto adjusted = [&](float y, unsigned w, bool allowed) {
      if (w) {
        const unsigned times = w & (PROMPT - 1), entry = w >> BIAS_SHIFT;
        if ((w & (2 * PROMPT - 1)) && a.repetition) y = y > 0.f ? y / rep : y * rep;
        if (times) y = y - freq * (float)times - pre;
        if (entry) y += a.bias[b * a.ld_bias + entry - 1];
      }
      return allowed ? y : -INFINITY;
    };
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int i = tid * VEC + u * RUN;
      if (i >= whole) continue;
      unsigned w[VEC], any = 0;
#pragma unroll
      for (int e = 0; e < VEC; e += 4) *reinterpret_cast<uint4*>(&w[e]) = *reinterpret_cast<const uint4*>(&word[i + e]);
#pragma unroll
      for (int e = 0; e < VEC; ++e) any |= w[e];
      const unsigned allowed = mask ? (unsigned)mask[(v0 + i) >> 5] >> ((v0 + i) & 31) : 0xffffffffu;
      if (any || mask) {                         // (what no step touches keeps its bits)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const bool touched = w[e] || !(allowed >> e & 1);
          if constexpr (sizeof(T) == 4) {
            if (touched) x[u][e] = __float_as_uint(adjusted(__uint_as_float(x[u][e]), w[e], allowed >> e & 1));
          } else if (touched) {
            const unsigned sh = 16 * (e & 1);
            const unsigned y = f2bf(adjusted(__uint_as_float(x[u][e >> 1] >> sh << 16), w[e], allowed >> e & 1));
            x[u][e >> 1] = (x[u][e >> 1] & ~(0xffffu << sh)) | y << sh;
          }
        }
      }
      if constexpr (MANY) __builtin_nontemporal_store(x[u], reinterpret_cast<Vec*>(out + i));
      else *reinterpret_cast<Vec*>(out + i) = x[u];
    }
    if (whole + tid < n) {                         // (the last few of the vocabulary)
      const int i = whole + tid;
      const bool allowed = !mask || mask[(v0 + i) >> 5] >> ((v0 + i) & 31) & 1;
      T y = in[i];
      if (word[i] || !allowed) put_logit(&y, adjusted(logit_f32(y), word[i], allowed));
      out[i] = y;
    }
    if (t + 1 < t1) {
      fetch(in + a.ld_logits);
      __syncthreads();                             // (this row's words have been read)
    }
  }
}

// Few rows: as many workgroups as the vocabulary has runs of 256 pieces, so that all of a row is on its way at once.  Many (from 8 MB on): slices of at most
// 6144 tokens, all of one size (24 KB of words, six workgroups on a compute unit: 103 us a call; 4096 / 8192: 123 / 112, the latter leaves a short slice at the end),
// and rows of a sequence share the count of its history, as long as 2048 workgroups are left.
void launch_adjust_logits(const sprinter_logits& a, hipStream_t s) {
  const int run = a.dtype == SPRINTER_F32 ? 1024 : 2048;
  const bool many = (long long)((a.vocab + run - 1) / run) * a.n_rows > 2048;
  const int slices = many ? (a.vocab + MANY_SLICE - 1) / MANY_SLICE : (a.vocab + run - 1) / run, slice = many ? round_up((a.vocab + slices - 1) / slices, 32) : run;
  const int per = (int)std::max(1ll, std::min(8ll, (long long)slices * a.n_rows / 2048));
  const dim3 grid((a.n_rows + per - 1) / per, slices);
  auto go = [&](auto type) {
    if (many) hipLaunchKernelGGL((k_adjust_logits<decltype(type), true>), grid, dim3(256), slice * 4, s, a, slice, per);
    else hipLaunchKernelGGL((k_adjust_logits<decltype(type), false>), grid, dim3(256), slice * 4, s, a, slice, per);
  };
  if (a.dtype == SPRINTER_F32) go(float()); else go(bf16_t());
}

}  // namespace sprinter
