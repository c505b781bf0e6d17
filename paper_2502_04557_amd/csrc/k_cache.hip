// HIP kernels of the cache in pages for gfx950: appending keys and values with their rotation, and moving an accepted path's slots.
#include "ops.h"
#include "dev.h"
#include <algorithm>

namespace sprinter {

// The first element of slot `s` of sequence `b`, KV head 0, in an array of one layer; -1 where it is not there.
__device__ __forceinline__ long long slot_at(const PagedArgs& c, int b, int s) {
  if (s < 0 || (s >> c.shift) >= c.n_table) return -1;
  const int page = c.table[(long long)b * c.ld_table + (s >> c.shift)];
  if (page < 0 || page >= c.n_page) return -1;
  return ((((long long)page * c.KVH) << c.shift) + (s & ((1 << c.shift) - 1))) * c.dh;
}

// cos and sin of an angle in radians: reduced by whole turns in float64 (2 pi as a sum of two), evaluated in float32.
__device__ __forceinline__ float2 turn_of(double angle) {
  const double turns = rint(angle * 0.15915494309189535);
  const float r = (float)fma(-turns, 2.4492935982947064e-16, fma(-turns, 6.283185307179586, angle));
  float sn, cs;
  sincosf(r, &sn, &cs);
  return make_float2(cs, sn);
}

__device__ __forceinline__ float as_f32(float v) { return v; }
__device__ __forceinline__ float as_f32(bf16_t v) { return __uint_as_float((unsigned)v << 16); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16_t* p, float v) { *p = f2bf(v); }

// One token per workgroup; a thread takes one pair of columns at a time, reads both before it writes one.
template <typename X, typename C>
__global__ __launch_bounds__(256) void k_cache_append(AppendArgs a) {
  __shared__ float2 turn[64];
  const int t = blockIdx.x, dh = a.c.dh, half = a.n_turned / 2, b = a.seq[t];
  if (b < 0 || b >= a.c.n_seq) return;
  const int slot = a.slot[t];
  const long long to = slot_at(a.c, b, slot);
  if ((int)threadIdx.x < half) turn[threadIdx.x] = turn_of((double)(a.pos ? a.pos[t] : slot) * a.freq[threadIdx.x]);
  __syncthreads();
  const int heads = a.H + 2 * a.c.KVH;
  for (int u = threadIdx.x; u < heads * (dh / 2); u += 256) {
    const int head = u / (dh / 2), i = u % (dh / 2);
    const bool turned = i < half && head < a.H + a.c.KVH;
    const int c0 = i < half ? (a.pairs ? 2 * i : i) : 2 * i, c1 = i < half && !a.pairs ? i + half : c0 + 1;   // (columns beyond the turned ones: in order)
    const X* src;
    C* dst;
    if (head < a.H) {
      src = (const X*)a.q + (long long)t * a.ld_q + head * dh;
      dst = (C*)a.q_out + (long long)t * a.ld_q_out + head * dh;
    } else {
      const int kv = (head - a.H) % a.c.KVH;
      const bool value = head >= a.H + a.c.KVH;
      if (to < 0) continue;
      src = value ? (const X*)a.v + (long long)t * a.ld_v + kv * dh : (const X*)a.k + (long long)t * a.ld_k + kv * dh;
      dst = (C*)(value ? a.c.values : a.c.keys) + to + (((long long)kv * dh) << a.c.shift);
    }
    float x = as_f32(src[c0]), y = as_f32(src[c1]);
    if (turned) {
      const float2 cs = turn[i];
      const float z = x * cs.x - y * cs.y;
      y = x * cs.y + y * cs.x;
      x = z;
    }
    put(dst + c0, x);
    put(dst + c1, y);
  }
}

void launch_cache_append(const AppendArgs& a, hipStream_t s) {
  const dim3 grid(a.T), block(256);
  if (a.row_type == X_F32) {
    if (a.cache_type == X_F32) hipLaunchKernelGGL((k_cache_append<float, float>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_cache_append<float, bf16_t>), grid, block, 0, s, a);
  } else {
    if (a.cache_type == X_F32) hipLaunchKernelGGL((k_cache_append<bf16_t, float>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_cache_append<bf16_t, bf16_t>), grid, block, 0, s, a);
  }
}

// A thread owns 16 bytes of a column of slots (keys or values of a KV head) in one layer and goes through the path in order: since path[j] >= j, what
// it reads for j lies behind every slot it has written, and what lies before it has been read.
__global__ __launch_bounds__(256) void k_cache_keep(KeepArgs a) {
  const int b = blockIdx.x, pieces = a.c.dh * a.element / 16, u = blockIdx.z * 256 + threadIdx.x;
  if (u >= 2 * a.c.KVH * pieces) return;
  const int n = min(a.n_keep[b], a.n_path), len = a.lens[b], nodes = a.first[b + 1] - a.first[b];
  const int kv = u / pieces % a.c.KVH;
  char* base = (char*)(u / pieces >= a.c.KVH ? a.c.values : a.c.keys) + blockIdx.y * a.layer_bytes + (((long long)kv * a.c.dh * a.element) << a.c.shift) +
               u % pieces * 16;
  if (len < 0) return;
  for (int j = 0; j < n; ++j) {
    const int i = a.path[b * a.ld_path + j];
    if (i <= j || i >= nodes) continue;
    const long long from = slot_at(a.c, b, (int)min((long long)len + i, 0x7fffffffll)), to = slot_at(a.c, b, (int)min((long long)len + j, 0x7fffffffll));
    if (from < 0 || to < 0) continue;
    *(uint4*)(base + to * a.element) = *(const uint4*)(base + from * a.element);
  }
}

void launch_cache_keep(const KeepArgs& a, hipStream_t s) {
  const int units = 2 * a.c.KVH * a.c.dh * a.element / 16;
  hipLaunchKernelGGL(k_cache_keep, dim3(a.c.n_seq, a.n_layer, (units + 255) / 256), dim3(256), 0, s, a);
}

}  // namespace sprinter
