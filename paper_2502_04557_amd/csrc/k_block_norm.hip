// HIP kernel of the norms around a block for gfx950: the norm of the block's output, its gate and residual scale, the residual row, and
// the norm that the next block reads, in one launch.
#include "ops.h"
#include "dev.h"
#include <algorithm>

namespace sprinter {

// u = norm(y; post) or y;  h' = h + scale gate u;  out = norm(h'; gain).  Statistics are two-pass float32: the mean first, then the
// squares of what lies around it.  k_block_norm takes any width and alignment, one row per workgroup, which stays in LDS between the steps.
template <int YT> struct RowType { using type = float; };
template <> struct RowType<X_BF16> { using type = bf16_t; };

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(bf16_t v) { return __uint_as_float((unsigned)v << 16); }

__device__ __forceinline__ float block_sum(float v, float* s4) {
  v = wave_total(v);
  __syncthreads();                                     // (the previous sum has been read)
  if ((threadIdx.x & 63) == 63) s4[threadIdx.x >> 6] = v;
  __syncthreads();
  return ((s4[0] + s4[1]) + s4[2]) + s4[3];
}
// mean (layer norm) and 1 / sqrt(variance + eps) of row[d]
__device__ __forceinline__ void statistics(const float* row, int d, int layer, float eps, float* s4, float& mean, float& rstd) {
  mean = 0.f;
  if (layer) {
    float s = 0.f;
    for (int c = threadIdx.x; c < d; c += 256) s += row[c];
    mean = block_sum(s, s4) / (float)d;
  }
  float q = 0.f;
  for (int c = threadIdx.x; c < d; c += 256) { const float v = row[c] - mean; q += v * v; }
  rstd = 1.0f / sqrtf(block_sum(q, s4) / (float)d + eps);
}

template <int YT>
__global__ __launch_bounds__(256) void k_block_norm(BlockNormArgs a) {
  extern __shared__ float row[];
  __shared__ float s4[4];
  using Y = typename RowType<YT>::type;
  const int r = blockIdx.x, d = a.d, layer = a.kind == 0;
  const Y* __restrict__ y = (const Y*)a.y + (long long)r * a.ldy;
  const float* __restrict__ h = a.h + (long long)r * a.ldh;
  for (int c = threadIdx.x; c < d; c += 256) row[c] = to_f32(y[c]);
  float mean = 0.f, rstd = 1.f;
  if (a.post_g) statistics(row, d, layer, a.eps, s4, mean, rstd);      // (each thread reads what it has written)
  for (int c = threadIdx.x; c < d; c += 256) {
    float u = row[c];
    if (a.post_g) u = (u - mean) * rstd * a.post_g[c];
    if (a.post_b) u += a.post_b[c];
    if (a.gate) u *= a.gate[(long long)r * a.gate_row + (long long)c * a.gate_col];
    const float v = h[c] + a.scale * u;
    row[c] = v;
    a.h_out[(long long)r * a.ld_h_out + c] = v;
  }
  statistics(row, d, layer, a.eps, s4, mean, rstd);
  for (int c = threadIdx.x; c < d; c += 256) {
    float v = (row[c] - mean) * rstd * a.g[c];
    if (a.b) v += a.b[c];
    if (a.out) {
      if (a.out_type == X_F32) ((float*)a.out)[(long long)r * a.ldo + c] = v;
      else ((bf16_t*)a.out)[(long long)r * a.ldo + c] = a.out_type == X_BF16 ? f2bf(v) : f2h(v);
    }
    if (a.tiles) act_store<bf16_t>((bf16_t*)a.tiles, r, c, d, v);
    if (a.f32) a.f32[(size_t)r * d + c] = v;
  }
}

// The same where rows, gains and gate lie at 16-byte addresses: a row in registers, 8 NI columns of 256 threads' chunks of 8 each, requested together
// while the row before is worked on.  A workgroup takes rows `stride` apart.  What bounds it: HBM; 4096 x 4096 with both norms and a gain per
// column 42 us, 201 MB at 4.8 TB/s, of inputs that change from call to call (37 of the same ones, which the cache behind L2 keeps in part; 4095
// columns through LDS, an element at a time: 96), one row 3.4 (12.4 through LDS).
template <int YT, int NI>
__global__ __launch_bounds__(256) void k_block_norm_rows(BlockNormArgs a, int stride) {
  using Y = typename RowType<YT>::type;
  __shared__ float sums[2][4][4];
  const int tid = threadIdx.x, n_chunks = a.d >> 3;
  const bool layer = a.kind == 0, post = a.post_g != nullptr;
  float y[NI][8], h[NI][8], gate[NI][8], next_y[NI][8], next_h[NI][8];
  auto chunk = [&](int i) { return min(tid + i * 256, n_chunks - 1) * 8; };
  auto fetch = [&](int r, float (&fy)[NI][8], float (&fh)[NI][8]) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      load_row((const Y*)a.y + (long long)r * a.ldy + chunk(i), fy[i]);
      load_row(a.h + (long long)r * a.ldh + chunk(i), fh[i]);
    }
  };
  // sum over the row of f(element); row parity and kind choose a place of their own: no barrier before the store
  auto total = [&](float v, int parity, int kind) {
    v = wave_total(v);
    if ((tid & 63) == 63) sums[parity][kind][tid >> 6] = v;
    __syncthreads();
    const float* s = sums[parity][kind];
    return ((s[0] + s[1]) + s[2]) + s[3];
  };
  auto statistics = [&](const float (&v)[NI][8], int parity, int kind, float& mean, float& rstd) {
    mean = 0.f;
    float s = 0.f;
    if (layer) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) s += tid + i * 256 < n_chunks ? v[i][e] : 0.f;
      mean = total(s, parity, kind) / (float)a.d;
    }
    s = 0.f;
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) { const float c = tid + i * 256 < n_chunks ? v[i][e] - mean : 0.f; s += c * c; }
    rstd = 1.0f / sqrtf(total(s, parity, kind + 1) / (float)a.d + a.eps);
  };
  int r = blockIdx.x;
  fetch(r, y, h);
  for (int parity = 0; r < a.T; parity ^= 1) {
    const int next = r + stride;
    float mean, rstd;
    if (a.gate && a.gate_col) {
#pragma unroll
      for (int i = 0; i < NI; ++i) load_row(a.gate + r * a.gate_row + chunk(i), gate[i]);
    }
    const float row_gate = a.gate && !a.gate_col ? a.gate[r * a.gate_row] : 1.f;
    if (next < a.T) fetch(next, next_y, next_h);
    if (post) {
      statistics(y, parity, 0, mean, rstd);
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        float g[8], b[8];
        load_row(a.post_g + chunk(i), g);
        if (a.post_b) load_row(a.post_b + chunk(i), b);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          y[i][e] = (y[i][e] - mean) * rstd * g[e];
          if (a.post_b) y[i][e] += b[e];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (a.gate) y[i][e] *= a.gate_col ? gate[i][e] : row_gate;
        h[i][e] = h[i][e] + a.scale * y[i][e];
      }
      const int c = (tid + i * 256) * 8;
      if (c < a.d) {
        float* to = a.h_out + (long long)r * a.ld_h_out + c;
        *reinterpret_cast<float4*>(to) = make_float4(h[i][0], h[i][1], h[i][2], h[i][3]);
        *reinterpret_cast<float4*>(to + 4) = make_float4(h[i][4], h[i][5], h[i][6], h[i][7]);
      }
    }
    statistics(h, parity, 2, mean, rstd);
    const int Kt = (a.d + 31) >> 5;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int c = (tid + i * 256) * 8;
      float g[8], b[8], o[8];
      load_row(a.g + chunk(i), g);
      if (a.b) load_row(a.b + chunk(i), b);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        o[e] = (h[i][e] - mean) * rstd * g[e];
        if (a.b) o[e] += b[e];
      }
      if (c >= a.d) continue;
      auto store_f32 = [&](float* to) {
        *reinterpret_cast<float4*>(to) = make_float4(o[0], o[1], o[2], o[3]);
        *reinterpret_cast<float4*>(to + 4) = make_float4(o[4], o[5], o[6], o[7]);
      };
      const uint4 half = make_uint4(pk_f16(o[0], o[1]), pk_f16(o[2], o[3]), pk_f16(o[4], o[5]), pk_f16(o[6], o[7]));
      if (a.out) {
        const long long at = (long long)r * a.ldo + c;
        if (a.out_type == X_F32) store_f32((float*)a.out + at);
        else if (a.out_type == X_F16) *reinterpret_cast<uint4*>((bf16_t*)a.out + at) = half;
        else *reinterpret_cast<uint4*>((bf16_t*)a.out + at) = make_uint4(pk_bf16(o[0], o[1]), pk_bf16(o[2], o[3]), pk_bf16(o[4], o[5]), pk_bf16(o[6], o[7]));
      }
      if (a.tiles) *reinterpret_cast<uint4*>((bf16_t*)a.tiles + ((size_t)(r >> 4) * Kt + (c >> 5)) * 512 + ((((c & 31) >> 3) << 4) + (r & 15)) * 8) = half;
      if (a.f32) store_f32(a.f32 + (size_t)r * a.d + c);
    }
    r = next;
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) { y[i][e] = next_y[i][e]; h[i][e] = next_h[i][e]; }
  }
}

template <int YT>
static void launch_rows(const BlockNormArgs& a, hipStream_t s) {
  const int wgs = std::min(a.T, 2048);
  if (a.d <= 2048) hipLaunchKernelGGL((k_block_norm_rows<YT, 1>), dim3(wgs), dim3(256), 0, s, a, wgs);
  else if (a.d <= 4096) hipLaunchKernelGGL((k_block_norm_rows<YT, 2>), dim3(wgs), dim3(256), 0, s, a, wgs);
  else if (a.d <= 8192) hipLaunchKernelGGL((k_block_norm_rows<YT, 4>), dim3(wgs), dim3(256), 0, s, a, wgs);
  else hipLaunchKernelGGL((k_block_norm_rows<YT, 8>), dim3(wgs), dim3(256), 0, s, a, wgs);
}

// Whether every row and parameter can be read and written 8 columns at a time.
static bool whole_chunks(const BlockNormArgs& a) {
  auto at16 = [](const void* p, long long ld, int size) { return ((uintptr_t)p & 15) == 0 && ld * size % 16 == 0; };
  auto param = [&](const float* p) { return at16(p, 0, 4); };
  return a.d % 8 == 0 && at16(a.h, a.ldh, 4) && at16(a.y, a.ldy, a.y_type == X_F32 ? 4 : 2) && at16(a.h_out, a.ld_h_out, 4) &&
         at16(a.out, a.ldo, a.out_type == X_F32 ? 4 : 2) && param(a.post_g) && param(a.post_b) && param(a.g) && param(a.b) &&
         (!a.gate || a.gate_col == 0 || (a.gate_col == 1 && at16(a.gate, a.gate_row, 4)));
}

void launch_block_norm(const BlockNormArgs& a, hipStream_t s) {
  if (whole_chunks(a)) {
    if (a.y_type == X_F32) launch_rows<X_F32>(a, s); else launch_rows<X_BF16>(a, s);
    return;
  }
  const size_t lds = (size_t)a.d * 4;
  if (a.y_type == X_F32) hipLaunchKernelGGL(k_block_norm<X_F32>, dim3(a.T), dim3(256), lds, s, a);
  else hipLaunchKernelGGL(k_block_norm<X_BF16>, dim3(a.T), dim3(256), lds, s, a);
}

}  // namespace sprinter
