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

__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(bf16_t* p, const float (&x)[8]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pk_bf16(x[0], x[1]), pk_bf16(x[2], x[3]), pk_bf16(x[4], x[5]), pk_bf16(x[6], x[7]));
}
__device__ __forceinline__ void turn_pair(float& x, float& y, float2 cs) {
  const float z = x * cs.x - y * cs.y;
  y = x * cs.y + y * cs.x;
  x = z;
}

// One token per workgroup (few tokens: its heads dealt out to up to 4), its angles shared by all heads.  A thread takes pairs of columns in units of two
// pieces of N elements that turn together: its reads of a unit come before its writes, so that queries may be turned in place.  N = 8: rows are 16-byte
// aligned and n_turned a multiple of 16; N = 1: any.  Bound by HBM: 4091 tokens of 32 heads of 128 columns in bf16, 201 MB in 42 us = 4.8 TB/s, what a large
// copy reaches (a pair at a time: 69 us).
template <typename X, typename C, int N>
__global__ __launch_bounds__(256) void k_cache_append(AppendArgs a) {
  __shared__ float2 turn[64];
  const int t = blockIdx.x, dh = a.c.dh, half = a.n_turned / 2, tid = threadIdx.x, b = a.seq[t], slot = a.slot[t];
  if (b < 0 || b >= a.c.n_seq) return;
  if (tid < half) turn[tid] = turn_of((double)(a.pos ? a.pos[t] : slot) * a.freq[tid]);
  const long long to = slot_at(a.c, b, slot);
  __syncthreads();
  const int shift = (dh == 64 ? 5 : 6) - (N == 8 ? 3 : 0);       // units of a head
  const int heads = a.H + 2 * a.c.KVH, first = blockIdx.y * heads / gridDim.y, end = (blockIdx.y + 1) * heads / gridDim.y;
  for (int i = tid + (first << shift); i < end << shift; i += 256) {
    const int head = i >> shift, u = (i & ((1 << shift) - 1)) * N;   // pairs u .. u + N - 1
    const X* src;
    C* dst;
    bool turned = u < half;
    if (head < a.H) {
      src = (const X*)a.q + t * a.ld_q + head * dh;
      dst = (C*)a.q_out + t * a.ld_q_out + head * dh;
    } else {
      if (to < 0) continue;
      const bool value = head >= a.H + a.c.KVH;
      const int kv = head - a.H - (value ? a.c.KVH : 0);
      src = value ? (const X*)a.v + t * a.ld_v + kv * dh : (const X*)a.k + t * a.ld_k + kv * dh;
      dst = (C*)(value ? a.c.values : a.c.keys) + to + (((long long)kv * dh) << a.c.shift);
      turned = turned && !value;
    }
    const bool apart = u < half && !a.pairs;       // a unit's two pieces: half a turn apart, or neighbours (also beyond the turned columns)
    const int c0 = apart ? u : 2 * u, c1 = apart ? u + half : 2 * u + N;
    if constexpr (N == 8) {
      float x[8], y[8];
      load_row(src + c0, x);
      load_row(src + c1, y);
      if (turned) {
        if (apart) {
#pragma unroll
          for (int e = 0; e < 8; ++e) turn_pair(x[e], y[e], turn[u + e]);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            turn_pair(x[2 * e], x[2 * e + 1], turn[u + e]);
            turn_pair(y[2 * e], y[2 * e + 1], turn[u + 4 + e]);
          }
        }
      }
      store8(dst + c0, x);
      store8(dst + c1, y);
    } else {
      float x = as_f32(src[c0]), y = as_f32(src[c1]);
      if (turned) turn_pair(x, y, turn[u]);
      put(dst + c0, x);
      put(dst + c1, y);
    }
  }
}

void launch_cache_append(const AppendArgs& a, hipStream_t s) {
  const size_t in = a.row_type == X_F32 ? 4 : 2, out = a.cache_type == X_F32 ? 4 : 2;
  auto fits = [&](const void* p, long long ld, size_t es) { return (uintptr_t)p % 16 == 0 && (a.T < 2 || (ld * es) % 16 == 0); };
  const bool wide = a.n_turned % 16 == 0 && fits(a.k, a.ld_k, in) && fits(a.v, a.ld_v, in) && (!a.H || (fits(a.q, a.ld_q, in) && fits(a.q_out, a.ld_q_out, out)));
  const dim3 grid(a.T, a.T < 128 ? std::min(4, a.H + 2 * a.c.KVH) : 1), block(256);
  auto go = [&](auto x, auto c) {
    if (wide) hipLaunchKernelGGL((k_cache_append<decltype(x), decltype(c), 8>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_cache_append<decltype(x), decltype(c), 1>), grid, block, 0, s, a);
  };
  if (a.row_type == X_F32) { if (a.cache_type == X_F32) go(float(), float()); else go(float(), bf16_t()); }
  else { if (a.cache_type == X_F32) go(bf16_t(), float()); else go(bf16_t(), bf16_t()); }
}

// A workgroup takes 512 bytes of a slot (keys or values, all KV heads one after the other) in one layer, and 8 entries of the path at a time: their reads come
// before a barrier, their writes behind it, and since path[j] >= j, what later entries read lies behind every slot that is written.  Bound by its chain of loads
// (counts, path, table, slot): 64 trees, 16 layers of 8 heads of 64 columns 6.6 us, 1.6 of them a launch (a thread that goes through the path alone: 7.2).
__global__ __launch_bounds__(256) void k_cache_keep(KeepArgs a) {
  const int b = blockIdx.x, pieces = a.c.dh * a.element / 16, u = blockIdx.z * 32 + (threadIdx.x & 31);
  int j = threadIdx.x >> 5, i = a.path[b * a.ld_path + min(j, a.n_path - 1)];   // (requested with the counts)
  const int n = min(a.n_keep[b], a.n_path), len = a.lens[b], nodes = a.first[b + 1] - a.first[b];
  if (len < 0) return;
  const int head = u / pieces, kv = head % a.c.KVH;
  char* base = (char*)(head >= a.c.KVH ? a.c.values : a.c.keys) + blockIdx.y * a.layer_bytes + (((long long)kv * a.c.dh * a.element) << a.c.shift) + u % pieces * 16;
  for (int j0 = 0; j0 < n; j0 += 8, j += 8) {      // (the same for all threads)
    if (j0) i = a.path[b * a.ld_path + min(j, n - 1)];
    long long from = -1, to = -1;
    if (j < n && i > j && i < nodes && head < 2 * a.c.KVH) {     // (a node in its place stays)
      from = slot_at(a.c, b, (int)min((long long)len + i, 0x7fffffffll));
      to = slot_at(a.c, b, (int)min((long long)len + j, 0x7fffffffll));
    }
    const bool moves = from >= 0 && to >= 0;
    uint4 v;
    if (moves) v = *(const uint4*)(base + from * a.element);
    __syncthreads();
    if (moves) *(uint4*)(base + to * a.element) = v;
  }
}

void launch_cache_keep(const KeepArgs& a, hipStream_t s) {
  const int units = 2 * a.c.KVH * a.c.dh * a.element / 16;
  hipLaunchKernelGGL(k_cache_keep, dim3(a.c.n_seq, a.n_layer, (units + 31) / 32), dim3(256), 0, s, a);
}

}  // namespace sprinter
