// HIP kernel of the norms around a block for gfx950: the norm of the block's output, its gate and residual scale, the residual row, and
// the norm that the next block reads, in one launch.
#include "ops.h"
#include "dev.h"

namespace sprinter {

// u = norm(y; post) or y;  h' = h + scale gate u;  out = norm(h'; gain), one row per workgroup; the row stays in LDS between the steps.
// Statistics are two-pass float32: the mean first, then the squares of what lies around it.
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

void launch_block_norm(const BlockNormArgs& a, hipStream_t s) {
  const size_t lds = (size_t)a.d * 4;
  if (a.y_type == X_F32) hipLaunchKernelGGL(k_block_norm<X_F32>, dim3(a.T), dim3(256), lds, s, a);
  else hipLaunchKernelGGL(k_block_norm<X_BF16>, dim3(a.T), dim3(256), lds, s, a);
}

}  // namespace sprinter
