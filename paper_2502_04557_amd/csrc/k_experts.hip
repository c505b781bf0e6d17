// HIP kernels of the experts' products for gfx950.
#include "ops.h"
#include "dev.h"
#include <algorithm>

namespace sprinter {

// y[t] = sum_j w[t,j] W2[e] (silu(Wg[e] x_t) * (Wu[e] x_t)), e = ids[t,j].
//
// Every pair (t, j) with an expert gets a slot; an expert's slots lie together and begin at a multiple of 16, so that 16 slots are one
// row tile of the matrix instruction and belong to one expert.  Which of its expert's slots a pair takes is left to chance: a row's
// products do not depend on the rows beside it, and the sum over j runs in the order of j.
//   plan     slots of the pairs, the rows of the slots, the list of row blocks (expert, first slot, rows)
//   up       hidden[slot] = silu(Wg x) * (Wu x), float16 operand tiles (float32 mode: rows)
//   down     product[slot] = W2 hidden[slot], float32
//   combine  y[t] = sum over j
struct Block { int expert, slot, rows; };
struct Plan {
  int* n_blocks; Block* blocks; int* row_of; int* slot_of;             // row_of [slots], slot_of [T k]
};
constexpr int BLOCK_ROWS = 16;

__global__ __launch_bounds__(1024) void k_experts_plan(const int* __restrict__ ids, int pairs, int k, int E, Plan p) {
  __shared__ int count[MAX_EXPERTS], first[MAX_EXPERTS];
  const int tid = threadIdx.x;
  for (int e = tid; e < E; e += 1024) count[e] = 0;
  __syncthreads();
  for (int i = tid; i < pairs; i += 1024) {
    const int e = ids[i];
    if ((unsigned)e < (unsigned)E) atomicAdd(&count[e], 1);
  }
  __syncthreads();
  if (tid == 0) {
    int slot = 0, n = 0;
    for (int e = 0; e < E; ++e) {
      first[e] = slot;
      for (int r = 0; r < count[e]; r += BLOCK_ROWS) p.blocks[n++] = Block{e, slot + r, min(BLOCK_ROWS, count[e] - r)};
      slot += round_up(count[e], 16);
    }
    *p.n_blocks = n;
  }
  __syncthreads();
  for (int e = tid; e < E; e += 1024) count[e] = 0;
  __syncthreads();
  for (int i = tid; i < pairs; i += 1024) {
    const int e = ids[i];
    int slot = -1;
    if ((unsigned)e < (unsigned)E) {
      slot = first[e] + atomicAdd(&count[e], 1);
      p.row_of[slot] = i / k;
    }
    p.slot_of[i] = slot;
  }
}

// One lane's operand of a k tile.  bf16 mode: 8 float16 of 32 k; float32 mode: 4 float32 of 16 k, one per instruction of 4 k each.
template <int DT> struct Operand;
template <> struct Operand<SPRINTER_BF16> { using T = uint4; static constexpr int K = 32, PER = 8; };
template <> struct Operand<SPRINTER_F32> { using T = f32x4; static constexpr int K = 16, PER = 4; };
__device__ __forceinline__ f32x4 product(uint4 x, uint4 w, f32x4 c) { return mfma_f16(x, w, c); }
__device__ __forceinline__ f32x4 product(f32x4 x, f32x4 w, f32x4 c) {
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], w[i], c, 0, 0, 0);
  return c;
}
// 8 elements of a row as float16
__device__ __forceinline__ uint4 load_x(const bf16_t* p, int type) {
  uint4 v = *reinterpret_cast<const uint4*>(p);
  if (type == X_BF16) {
    unsigned* q = &v.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = pk_f16(__uint_as_float(q[i] << 16), __uint_as_float(q[i] & 0xffff0000u));
  }
  return v;
}
__device__ __forceinline__ f32x4 load_x(const float* p, int) { return *reinterpret_cast<const f32x4*>(p); }
template <int DT> using Elem = std::conditional_t<DT == SPRINTER_F32, float, bf16_t>;

// The weights of column tile nt, k tile kt: row n of expert e of a matrix [E][N][K]
template <int DT>
__device__ __forceinline__ typename Operand<DT>::T load_w(const void* W, int e, int N, int K, int nt, int kt, int lane) {
  if constexpr (DT == SPRINTER_BF16) {
    const int Kt = (K + 31) >> 5, Nt = (N + 15) >> 4;
    return ((const uint4*)W)[(((size_t)e * Nt + nt) * Kt + kt) * 64 + lane];
  } else {
    const int n = min(nt * 16 + (lane & 15), N - 1), k = kt * 16 + (lane >> 4) * 4;
    const f32x4 v = *reinterpret_cast<const f32x4*>((const float*)W + ((size_t)e * N + n) * K + min(k, K - 4));
    return k < K ? v : (f32x4){0.f, 0.f, 0.f, 0.f};
  }
}

// Sum of the four waves' accumulators, in wave 0
__device__ __forceinline__ f32x4 join(f32x4 v, f32x4 (*red)[64], int w, int lane) {
  red[w][lane] = v;
  __syncthreads();
  const f32x4 s = ((red[0][lane] + red[1][lane]) + red[2][lane]) + red[3][lane];
  __syncthreads();
  return s;
}

// A workgroup: one column tile (of col_tiles) of one row block.  Four waves share K.
template <int DT>
__global__ __launch_bounds__(256) void k_experts_up(ExpertsArgs a, Plan p, void* hidden, int col_tiles) {
  using O = Operand<DT>;
  __shared__ f32x4 red[4][64];
  const int lane = threadIdx.x & 63, w = wave_index(), id = blockIdx.x / col_tiles, nt = blockIdx.x - id * col_tiles;
  if (id >= *p.n_blocks) return;
  const Block b = p.blocks[id];
  const int r = min(lane & 15, b.rows - 1);
  const Elem<DT>* x = (const Elem<DT>*)a.x + (long long)p.row_of[b.slot + r] * a.ldx;
  const int Kt = (a.d + O::K - 1) / O::K;
  f32x4 g = {0.f, 0.f, 0.f, 0.f}, u = g;
  for (int kt = w; kt < Kt; kt += 4) {
    const int k = kt * O::K + (lane >> 4) * O::PER;
    typename O::T xv = {};
    if (k < a.d) xv = load_x(x + k, a.x_type);
    g = product(xv, load_w<DT>(a.wg, b.expert, a.ff, a.d, nt, kt, lane), g);
    u = product(xv, load_w<DT>(a.wu, b.expert, a.ff, a.d, nt, kt, lane), u);
  }
  g = join(g, red, w, lane);
  u = join(u, red, w, lane);
  const int n = nt * 16 + (lane & 15), m = (lane >> 4) * 4 + w;        // each wave finishes one of the four rows of a lane
  if (m < b.rows && n < a.ff) act_store<Elem<DT>>((Elem<DT>*)hidden, b.slot + m, n, a.ff, silu(g[w]) * u[w]);
}

template <int DT>
__global__ __launch_bounds__(256) void k_experts_down(ExpertsArgs a, Plan p, const void* hidden, float* out, int col_tiles) {
  using O = Operand<DT>;
  __shared__ f32x4 red[4][64];
  const int lane = threadIdx.x & 63, w = wave_index(), id = blockIdx.x / col_tiles, nt = blockIdx.x - id * col_tiles;
  if (id >= *p.n_blocks) return;
  const Block b = p.blocks[id];
  const int slot = b.slot + min(lane & 15, b.rows - 1), Kt = (a.ff + O::K - 1) / O::K;
  f32x4 c = {0.f, 0.f, 0.f, 0.f};
  for (int kt = w; kt < Kt; kt += 4) {
    const int k = kt * O::K + (lane >> 4) * O::PER;
    typename O::T xv = {};
    if (k < a.ff) xv = load_x((const Elem<DT>*)hidden + act_idx<Elem<DT>>(slot, k, a.ff), X_F16);
    c = product(xv, load_w<DT>(a.w2, b.expert, a.d, a.ff, nt, kt, lane), c);
  }
  c = join(c, red, w, lane);
  const int n = nt * 16 + (lane & 15), m = (lane >> 4) * 4 + w;
  if (m < b.rows && n < a.d) out[(size_t)(b.slot + m) * a.d + n] = c[w];
}

// One thread per 4 columns of a row.
__global__ __launch_bounds__(256) void k_experts_combine(ExpertsArgs a, const int* __restrict__ slot_of, const float* __restrict__ out, int parts) {
  const int t = blockIdx.x / parts, c = ((blockIdx.x - t * parts) * 256 + threadIdx.x) * 4;
  if (c >= a.d) return;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int j = 0; j < a.k; ++j) {
    const int slot = slot_of[(size_t)t * a.k + j];
    if (slot < 0) continue;
    const float w = a.weights[(size_t)t * a.k + j];
    const float4 v = *reinterpret_cast<const float4*>(out + (size_t)slot * a.d + c);
    s.x += w * v.x; s.y += w * v.y; s.z += w * v.z; s.w += w * v.w;
  }
  if (a.y_type == X_F32) *reinterpret_cast<float4*>((float*)a.y + (long long)t * a.ldy + c) = s;
  else *reinterpret_cast<uint2*>((bf16_t*)a.y + (long long)t * a.ldy + c) = make_uint2(pk_bf16(s.x, s.y), pk_bf16(s.z, s.w));
}

void launch_pack_experts(const void* w, void* out, int E, int N, int K, hipStream_t s) {
  for (int e = 0; e < E; ++e)
    launch_pack_bf16((const bf16_t*)w + (size_t)e * N * K, (bf16_t*)out + (size_t)e * expert_elems(N, K), N, K, s);
}

namespace {
struct Space {
  Plan plan; void* hidden; float* out; size_t bytes;
};
// pairs and experts bound the slots: every used expert rounds its own up to 16.
Space space(void* base, int dtype, int E, int d, int ff, long long T, int k) {
  const long long pairs = T * k, slots = (pairs + 15 * std::min<long long>(E, pairs) + 15) / 16 * 16;
  size_t at = 0;
  auto take = [&](size_t n) { void* p = (char*)base + at; at += (n + 255) & ~(size_t)255; return p; };
  Space s;
  s.plan.n_blocks = (int*)take(4);
  s.plan.blocks = (Block*)take((size_t)(slots / 16) * sizeof(Block));
  s.plan.row_of = (int*)take((size_t)slots * 4);
  s.plan.slot_of = (int*)take((size_t)pairs * 4);
  s.hidden = take((size_t)slots * (dtype == SPRINTER_F32 ? (size_t)ff * 4 : (size_t)round_up(ff, 32) * 2));
  s.out = (float*)take((size_t)slots * d * 4);
  s.bytes = at;
  return s;
}
}  // namespace

size_t experts_workspace(int dtype, int E, int d, int ff, long long T, int k) { return space(nullptr, dtype, E, d, ff, T, k).bytes; }

void launch_experts(const ExpertsArgs& a, void* workspace, hipStream_t s) {
  const Space w = space(workspace, a.dtype, a.E, a.d, a.ff, a.T, a.k);
  const int pairs = a.T * a.k, blocks = pairs / BLOCK_ROWS + std::min(a.E, pairs);
  hipLaunchKernelGGL(k_experts_plan, dim3(1), dim3(1024), 0, s, a.ids, pairs, a.k, a.E, w.plan);
  const int up = (a.ff + 15) / 16, down = (a.d + 15) / 16, parts = (a.d / 4 + 255) / 256;
  if (a.dtype == SPRINTER_F32) {
    hipLaunchKernelGGL(k_experts_up<SPRINTER_F32>, dim3(up * blocks), dim3(256), 0, s, a, w.plan, w.hidden, up);
    hipLaunchKernelGGL(k_experts_down<SPRINTER_F32>, dim3(down * blocks), dim3(256), 0, s, a, w.plan, w.hidden, w.out, down);
  } else {
    hipLaunchKernelGGL(k_experts_up<SPRINTER_BF16>, dim3(up * blocks), dim3(256), 0, s, a, w.plan, w.hidden, up);
    hipLaunchKernelGGL(k_experts_down<SPRINTER_BF16>, dim3(down * blocks), dim3(256), 0, s, a, w.plan, w.hidden, w.out, down);
  }
  hipLaunchKernelGGL(k_experts_combine, dim3(parts * a.T), dim3(256), 0, s, a, w.plan.slot_of, w.out, parts);
}

}  // namespace sprinter
