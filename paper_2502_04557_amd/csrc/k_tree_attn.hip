// HIP kernels of the attention of trees of drafted tokens over a cache in pages, for gfx950.
#include "ops.h"
#include "dev.h"
#include <algorithm>

namespace sprinter {

// The sequence of row t: the last b with first[b] <= t, or -1 where t is no row of it.
__device__ __forceinline__ int sequence_of(const int* first, int n_seq, int t) {
  int lo = 0, hi = n_seq;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= t) lo = mid; else hi = mid;
  }
  return first[lo] <= t && t < first[lo + 1] ? lo : -1;
}

// One wave per row and head, four keys at a time: 16 lanes share a key, each group of them runs an online softmax of its own.
template <typename T, int DH>
__global__ __launch_bounds__(64) void k_tree_attn(AttendArgs a) {
  constexpr int N = DH / 16;
  const int t = blockIdx.x, h = blockIdx.y, lane = threadIdx.x, l16 = lane & 15, lq = lane >> 4;
  const int b = sequence_of(a.first, a.c.n_seq, t);
  if (b < 0) return;
  const int node = t - a.first[b], nodes = min(a.first[b + 1], a.T) - a.first[b], len = max(a.lens[b], 0);
  const int kvh = h / (a.H / a.c.KVH);
  float q[N], o[N], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const T v = ((const T*)a.q)[(long long)t * a.ld_q + h * DH + l16 * N + i];
    if constexpr (sizeof(T) == 4) q[i] = v * a.scale; else q[i] = __uint_as_float((unsigned)v << 16) * a.scale;
    o[i] = 0.f;
  }
  const long long total = min((long long)len + nodes, (long long)a.c.n_table << a.c.shift);
  for (int s0 = 0; s0 < total; s0 += 4) {
    const int s = s0 + lq;
    bool there = s < total;
    if (there && s >= len) {
      const int j = s - len;
      there = a.visible ? j < 64 * a.n_words && (a.visible[(long long)t * a.n_words + (j >> 6)] >> (j & 63) & 1) : j <= node;
    }
    int page = -1;
    if (there) page = a.c.table[(long long)b * a.c.ld_table + (s >> a.c.shift)];
    there = there && page >= 0 && page < a.c.n_page;
    float k[N], v[N], d = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) k[i] = v[i] = 0.f;
    if (there) {
      const long long at = ((((long long)page * a.c.KVH + kvh) << a.c.shift) + (s & ((1 << a.c.shift) - 1))) * DH + l16 * N;
      load_row((const T*)a.c.keys + at, k);
      load_row((const T*)a.c.values + at, v);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) d += q[i] * k[i];
    d = group_sum<16>(d);
    if (!there || d == -INFINITY) continue;
    const float mn = d != d ? d : fmaxf(m, d);
    const float corr = expf(m - mn), p = expf(d - mn);
    l = l * corr + p;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = o[i] * corr + p * v[i];
    m = mn;
  }
  float all = m;
  for (int x = 16; x < 64; x <<= 1) { const float y = __shfl_xor(all, x); all = all != all || y != y ? all + y : fmaxf(all, y); }
  const float w = m == -INFINITY ? 0.f : expf(m - all);
  l *= w;
#pragma unroll
  for (int i = 0; i < N; ++i) o[i] = m == -INFINITY ? 0.f : o[i] * w;
  for (int x = 16; x < 64; x <<= 1) {
    l += __shfl_xor(l, x);
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] += __shfl_xor(o[i], x);
  }
  if (lq) return;
  T* y = (T*)a.y + (long long)t * a.ld_y + h * DH + l16 * N;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float r = l == 0.f ? 0.f : o[i] / l;
    if constexpr (sizeof(T) == 4) y[i] = r; else y[i] = f2bf(r);
  }
}

size_t attend_workspace(int, int, int, int, int, int, long long) { return 0; }

void launch_cache_attend(const AttendArgs& a, void*, hipStream_t s) {
  const dim3 grid(a.T, a.H), block(64);
  if (a.type == X_F32) {
    if (a.c.dh == 64) hipLaunchKernelGGL((k_tree_attn<float, 64>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_tree_attn<float, 128>), grid, block, 0, s, a);
  } else {
    if (a.c.dh == 64) hipLaunchKernelGGL((k_tree_attn<bf16_t, 64>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_tree_attn<bf16_t, 128>), grid, block, 0, s, a);
  }
}

}  // namespace sprinter
