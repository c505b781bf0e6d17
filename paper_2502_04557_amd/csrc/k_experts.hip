// HIP kernels of the experts' products for gfx950: the plan of many rows, few rows, float32, and the sum over a row's experts.
#include "experts.h"
#include <algorithm>
#include <type_traits>

namespace sprinter {

// y[t] = sum_j w[t,j] W2[e] (silu(Wg[e] x_t) * (Wu[e] x_t)), e = ids[t,j].
//
// bf16 mode, up to 16 rows: they are one row tile of the matrix instruction, whoever names an expert.
//   up_few     hidden[e][t] = silu(Wg x_t) * (Wu x_t) for every expert that some row names (0 for rows that do not name it), and the
//              rows' weights for it
//   down_few   y[t] = sum over e of w W2[e] hidden[e][t]: one launch over a K of (experts named) x ff, an expert's sum joining the rows that
//              name it.  (The weight could ride in hidden, but small ones would push it below float16's normal numbers.)
// Else:
//   plan       slots of the pairs, the rows of the slots, the list of row blocks; beside it the rows as float16
//   up, down   hidden[slot], product[slot] (k_experts_tile.hip; float32 mode: here)
//   combine    y[t] = sum over j
// us of the launches, inputs and weights changing from call to call: 4096 rows, 2 of 8 experts of 4096 x 14336: 14 + 1730 + 857 + 28; 1789 rows,
// 8 of 64 of 2048 x 1024: 11 + 211 + 111 + 20; 61 rows, 2 of 8 of 4096 x 14336: 5 + 322 + 154 + 5 (2.8 GB at 5.9 TB/s); 1 row of them: 80 + 41
// (0.7 GB at 5.9); 16 rows, 8 of 64: 71 + 38 + 5 (49 experts are named: 0.63 GB at 5.7).

// ------------------------------------------------------------------------------------------------------------------ plan
// 8 elements of a row as float16
__device__ __forceinline__ uint4 as_f16(uint4 v) {
  unsigned* q = &v.x;
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] = pk_f16(__uint_as_float(q[i] << 16), __uint_as_float(q[i] & 0xffff0000u));
  return v;
}

// A counter per expert in LDS gives each pair its place among its expert's; the counts' prefix sums (rounded up to 16) are the experts'
// first slots.  Every workgroup counts all pairs, those before its own share apart, and writes the slots of its share: the scattered
// stores of one workgroup alone took 18 us for 14312 pairs, now 9.  The workgroups behind the `plans` of them copy x as float16 rows of whole k tiles.
__global__ __launch_bounds__(1024) void k_experts_plan(const int* __restrict__ ids, int pairs, int k, int E, int block_rows, int share, Plan p, int plans, int copies,
                                                       const bf16_t* __restrict__ x, long long ldx, uint4* __restrict__ rows, int T, int d) {
  __shared__ int count[MAX_EXPERTS], before[MAX_EXPERTS], slots[16], blocks[16];
  constexpr int N = 8;                                  // ids of a thread that are requested together
  const int tid = threadIdx.x, lane = tid & 63, p0 = blockIdx.x * share, p1 = min(p0 + share, pairs);
  if ((int)blockIdx.x >= plans) {
    const int octets = round_up(d, 32) >> 3;
    const long long n = (long long)T * octets, step = (long long)copies * 1024;
    for (long long i = (long long)(blockIdx.x - plans) * 1024 + tid; i < n; i += step) {
      const int t = (int)(i / octets), c = (int)(i - (long long)t * octets) * 8;
      rows[i] = c < d ? as_f16(*reinterpret_cast<const uint4*>(x + t * ldx + c)) : make_uint4(0u, 0u, 0u, 0u);
    }
    return;
  }
  count[tid] = before[tid] = 0;
  __syncthreads();
  auto load = [&](int i0, int end, int (&e)[N]) {
#pragma unroll
    for (int r = 0; r < N; ++r) {
      const int i = i0 + r * 1024 + tid;
      e[r] = i < end ? ids[i] : -1;
      if ((unsigned)e[r] >= (unsigned)E) e[r] = -1;
    }
  };
  int e[N];
  for (int i0 = 0; i0 < pairs; i0 += N * 1024) {
    load(i0, pairs, e);
#pragma unroll
    for (int r = 0; r < N; ++r) {
      if (e[r] < 0) continue;
      atomicAdd(&count[e[r]], 1);
      if (i0 + r * 1024 + tid < p0) atomicAdd(&before[e[r]], 1);
    }
  }
  __syncthreads();
  {
    const int c = tid < E ? count[tid] : 0, mine = round_up(c, 16), mine_b = (c + block_rows - 1) / block_rows;
    int s = mine, b = mine_b;
    for (int o = 1; o < 64; o <<= 1) {
      const int ps = __shfl_up(s, o), pb = __shfl_up(b, o);
      if (lane >= o) { s += ps; b += pb; }
    }
    if (lane == 63) { slots[tid >> 6] = s; blocks[tid >> 6] = b; }
    __syncthreads();
    int s0 = s - mine, b0 = b - mine_b;
    for (int q = 0; q < tid >> 6; ++q) { s0 += slots[q]; b0 += blocks[q]; }
    before[tid] += s0;
    if (blockIdx.x == 0) {
      for (int i = 0; i < mine_b; ++i) p.blocks[b0 + i] = Block{tid, s0 + i * block_rows, min(block_rows, c - i * block_rows), b0, mine_b};
      if (tid == 1023) *p.n_blocks = b0 + mine_b;
    }
  }
  __syncthreads();
  for (int i0 = p0; i0 < p1; i0 += N * 1024) {
    load(i0, p1, e);
#pragma unroll
    for (int r = 0; r < N; ++r) {
      const int i = i0 + r * 1024 + tid;
      if (i >= p1) continue;
      const int slot = e[r] < 0 ? -1 : atomicAdd(&before[e[r]], 1);
      p.slot_of[i] = slot;
      if (slot >= 0) p.row_of[slot] = i / k;
    }
  }
}

// -------------------------------------------------------------------------------------------------------------- few rows
constexpr int FEW_ROWS = 16;

// The rows that name each expert, as bits in LDS, from the ids [T, k]; experts that no row names have none.  named_expert: the j-th that is
// named, in rising order, for every wave by itself (-1: there are no more).
struct NamedExperts { unsigned rows[MAX_EXPERTS]; };
constexpr int FEW_THREADS = 512;                        // (no kernel here asks for its block's or grid's size, which would bring hidden arguments)
__device__ __forceinline__ void name_experts(NamedExperts& s, const int* __restrict__ ids, int T, int k, int E) {
  for (int e = threadIdx.x; e < E; e += FEW_THREADS) s.rows[e] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < T * k; i += FEW_THREADS) {
    const int e = ids[i];
    if ((unsigned)e < (unsigned)E) atomicOr(&s.rows[e], 1u << (i / k));
  }
  __syncthreads();
}
__device__ __forceinline__ int named_expert(const NamedExperts& s, int j, int E, int lane) {
  for (int e0 = 0; e0 < E; e0 += 64) {                  // (scalar)
    u64 named = __ballot(e0 + lane < E && s.rows[min(e0 + lane, E - 1)] != 0);
    const int n = __popcll(named);
    if (j < n) {
      for (; j > 0; --j) named &= named - 1;
      return e0 + __builtin_ctzll(named);
    }
    j -= n;
  }
  return -1;
}

// A workgroup: one expert's column tile of both matrices.  The 8 waves share K; 256 threads then finish an element each.  What bounds it: the
// weights, at 5.7 - 5.9 TB/s (two column tiles per workgroup: 5.5; eight k tiles in flight per wave for four: as many or less).
__global__ __launch_bounds__(FEW_THREADS) void k_experts_up_few(const void* wg, const void* wu, const void* x_, const int* __restrict__ ids, const float* __restrict__ weights,
                                                        int T, int k, int E, int d, int ff, long long ldx, int x_type, int col_tiles, uint4* hidden,
                                                        float* row_weights) {
  constexpr int U = 4;
  __shared__ NamedExperts named;
  __shared__ float red[8][2][4][64];
  const int tid = threadIdx.x, lane = tid & 63, w = wave_index();
  const int j = blockIdx.x / col_tiles, nt = blockIdx.x - j * col_tiles;
  name_experts(named, ids, T, k, E);
  const int e = named_expert(named, j, E, lane);
  if (e < 0) return;
  const int Kt = (d + 31) >> 5, Nt = (ff + 15) >> 4, row = lane & 15, oct = (lane >> 4) * 8;
  const size_t tile = ((size_t)e * Nt + min(nt, Nt - 1)) * Kt * 64 + lane;      // (the column tile behind the last one of an odd count: zeros)
  const uint4 *Wg = (const uint4*)wg + tile, *Wu = (const uint4*)wu + tile;
  const bf16_t* x = (const bf16_t*)x_ + (size_t)min(row, T - 1) * ldx;
  f32x4 g = {0.f, 0.f, 0.f, 0.f}, u = g;
  for (int kt = w; kt < Kt; kt += 8 * U) {
    uint4 a[U], b[U], v[U];
#pragma unroll
    for (int q = 0; q < U; ++q) {
      const int kc = min(kt + q * 8, Kt - 1);
      a[q] = Wg[(size_t)kc * 64]; b[q] = Wu[(size_t)kc * 64];
      v[q] = make_uint4(0u, 0u, 0u, 0u);
      if (row < T && kt + q * 8 < Kt && kc * 32 + oct < d) v[q] = *reinterpret_cast<const uint4*>(x + kc * 32 + oct);
    }
#pragma unroll
    for (int q = 0; q < U; ++q) {
      const uint4 h = x_type == X_BF16 ? as_f16(v[q]) : v[q];
      g = mfma_f16(h, a[q], g);
      u = mfma_f16(h, b[q], u);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) { red[w][0][i][lane] = g[i]; red[w][1][i][lane] = u[i]; }
  if (nt == 0) {                                        // the rows' weights for this expert: 32 threads to a row
    const int m = tid >> 5;
    float s = 0.f;
    if (m < T)
      for (int i = tid & 31; i < k; i += 32)
        if (ids[m * k + i] == e) s += weights[m * k + i];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) s += __shfl_xor(s, o);
    if ((tid & 31) == 0) row_weights[j * FEW_ROWS + m] = s;
  }
  __syncthreads();
  if (tid >= 256) return;
  // (row m, column c), in the order of the operand tile
  const int m = (tid >> 3) & 15, c = (tid >> 7) * 8 + (tid & 7), n = nt * 16 + c, i = m & 3, at = (m >> 2) * 16 + c;
  float gs = 0.f, us = 0.f;
#pragma unroll
  for (int q = 0; q < 8; ++q) { gs += red[q][0][i][at]; us += red[q][1][i][at]; }
  act_store<bf16_t>((bf16_t*)(hidden + (size_t)j * ((ff + 31) >> 5) * 64), m, n, ff, (named.rows[e] >> m & 1) && n < ff ? silu(gs) * us : 0.f);
}

// A workgroup: one column tile of y and one of `shares` shares of K = (experts named) x ff.  A row takes nothing from an expert that it does
// not name, not even 0 times an infinite weight: each expert's sum joins the rows that name it.
__global__ __launch_bounds__(FEW_THREADS) void k_experts_down_few(const void* w2, const uint4* __restrict__ hidden, const float* __restrict__ row_weights, const int* __restrict__ ids, int T, int k, int E, int d,
                                                          int ff, int shares, float* part, void* y, int y_type, long long ldy) {
  constexpr int U = 8;
  __shared__ NamedExperts named;
  __shared__ unsigned short list[MAX_EXPERTS];
  __shared__ float red[8][4][64];
  __shared__ int n_named;
  const int tid = threadIdx.x, lane = tid & 63, w = wave_index();
  const int Nt = (d + 15) >> 4, Kt = (ff + 31) >> 5, nt = blockIdx.x % Nt, share = blockIdx.x / Nt;
  name_experts(named, ids, T, k, E);
  if (w == 0) {
    int n = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {
      const bool on = e0 + lane < E && named.rows[min(e0 + lane, E - 1)] != 0;
      const u64 at = __ballot(on);
      if (on) list[n + __popcll(at & ((1ull << lane) - 1))] = (unsigned short)(e0 + lane);
      n += __popcll(at);
    }
    if (lane == 0) n_named = n;
  }
  __syncthreads();
  const int total = n_named * Kt, parts = shares * 8, me = share * 8 + w;
  const int q0 = (int)((long long)total * me / parts), q1 = (int)((long long)total * (me + 1) / parts);
  const bool live = (lane & 15) < T;
  f32x4 c = (f32x4){0.f, 0.f, 0.f, 0.f};
  for (int j = q0 / Kt, q = q0; q < q1; ++j) {          // expert by expert
    const int e = __builtin_amdgcn_readfirstlane((int)list[j]), end = min(q1, (j + 1) * Kt);
    const unsigned rows = named.rows[e];
    const float4 weight = *reinterpret_cast<const float4*>(row_weights + j * FEW_ROWS + (lane >> 4) * 4);
    const uint4* W = (const uint4*)w2 + (((size_t)e * Nt + nt) * Kt - (size_t)j * Kt) * 64 + lane;
    const uint4* H = hidden + lane;
    f32x4 p = (f32x4){0.f, 0.f, 0.f, 0.f};
    for (; q < end; q += U) {
      uint4 a[U], h[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int qc = min(q + i, end - 1);
        a[i] = W[(size_t)qc * 64];
        h[i] = make_uint4(0u, 0u, 0u, 0u);
        if (live && q + i < end) h[i] = H[(size_t)qc * 64];
      }
#pragma unroll
      for (int i = 0; i < U; ++i) p = mfma_f16(h[i], a[i], p);
    }
    q = end;
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] += rows >> ((lane >> 4) * 4 + i) & 1 ? (&weight.x)[i] * p[i] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) red[w][i][lane] = c[i];
  __syncthreads();
  if (tid >= 256) return;
  const int m = tid >> 4, n = nt * 16 + (tid & 15), at = (m >> 2) * 16 + (tid & 15);
  if (m >= T || n >= d) return;
  float s = 0.f;
#pragma unroll
  for (int q = 0; q < 8; ++q) s += red[q][m & 3][at];
  if (shares > 1) part[((size_t)share * FEW_ROWS + m) * d + n] = s;
  else if (y_type == X_F32) ((float*)y)[m * ldy + n] = s;
  else ((bf16_t*)y)[m * ldy + n] = f2bf(s);
}
__global__ __launch_bounds__(256) void k_experts_join(const float* __restrict__ part, int shares, int T, int d, void* y, int y_type, long long ldy) {
  const int parts = (d + 255) >> 8, m = blockIdx.x / parts, n = (blockIdx.x - m * parts) * 256 + threadIdx.x;
  if (n >= d) return;
  float s = 0.f;
#pragma unroll 8
  for (int q = 0; q < shares; ++q) s += part[((size_t)q * FEW_ROWS + m) * d + n];
  if (y_type == X_F32) ((float*)y)[m * ldy + n] = s;
  else ((bf16_t*)y)[m * ldy + n] = f2bf(s);
}

// --------------------------------------------------------------------------------------------------------------- float32
// One lane's operand of a k tile: 4 float32 of 16 k, one per instruction of 4 k each.
__device__ __forceinline__ f32x4 product(f32x4 x, f32x4 w, f32x4 c) {
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], w[i], c, 0, 0, 0);
  return c;
}
__device__ __forceinline__ f32x4 load4(const float* row, int k, int K) {
  const f32x4 v = *reinterpret_cast<const f32x4*>(row + min(k, K - 4));
  return k < K ? v : (f32x4){0.f, 0.f, 0.f, 0.f};
}
// A workgroup: one column tile (blockIdx.x) of one row block of 16 rows (blockIdx.y).  Eight waves share K.  up: out = silu(Wg x) * (Wu x) of the
// gathered rows.  What bounds it: the weights, 67 MB of 8 experts of 512 x 2048 in 16.7 us and 34 MB in 10.9, 4.0 and 3.1 TB/s: streams this
// short do not reach the rate of long ones.
template <bool UP>
__global__ __launch_bounds__(512) void k_experts_f32(const float* W, const float* W2, const float* X, long long ldx, int N, int K, Plan p, float* out) {
  constexpr int U = 4, MATS = UP ? 2 : 1;
  __shared__ f32x4 red[8][MATS][64];
  const int lane = threadIdx.x & 63, w = wave_index(), nt = blockIdx.x;
  if ((int)blockIdx.y >= *p.n_blocks) return;
  const Block b = p.blocks[blockIdx.y];
  const int slot = b.slot + min(lane & 15, b.rows - 1);
  const float* x = X + (UP ? p.row_of[slot] : slot) * ldx;
  const size_t at = ((size_t)b.expert * N + min(nt * 16 + (lane & 15), N - 1)) * K;
  f32x4 acc[MATS];
#pragma unroll
  for (int q = 0; q < MATS; ++q) acc[q] = (f32x4){0.f, 0.f, 0.f, 0.f};
  for (int kt = w; kt < (K + 15) >> 4; kt += 8 * U) {
    f32x4 wv[U][MATS], xv[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = (kt + u * 8) * 16 + (lane >> 4) * 4;               // (behind K: zeros)
      wv[u][0] = load4(W + at, k, K);
      if (UP) wv[u][MATS - 1] = load4(W2 + at, k, K);
      xv[u] = load4(x, k, K);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int q = 0; q < MATS; ++q) acc[q] = product(xv[u], wv[u][q], acc[q]);
  }
#pragma unroll
  for (int q = 0; q < MATS; ++q) red[w][q][lane] = acc[q];
  __syncthreads();
  if (threadIdx.x >= 256) return;
  // lane 16 (row / 4) + column of an accumulator holds four rows
  const int m = threadIdx.x >> 4, n = nt * 16 + (threadIdx.x & 15), from = (m >> 2) * 16 + (threadIdx.x & 15), i = m & 3;
  if (m >= b.rows || n >= N) return;
  float g = 0.f, u = 0.f;
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    g += red[q][0][from][i];
    if (UP) u += red[q][MATS - 1][from][i];
  }
  out[(size_t)(b.slot + m) * N + n] = UP ? silu(g) * u : g;
}

// The same for many rows: 64 rows x 64 columns (up: 32 of each matrix) per workgroup, both operands through LDS.  A stage is 32 k, 128 bytes
// of 64 rows of each operand; eight lanes next to each other fetch a row's 128 bytes (one cache line), whose 16-byte units lie exchanged
// by row % 8 in LDS, so that the fragment reads - 16 bytes of 16 rows - are free of bank conflicts.  A ring of four stages: at the top of
// stage kc the wave waits for its own loads of it and its own reads of kc - 1, the barrier makes that true for every wave and says that nobody reads stage kc - 1 any
// more, whose place takes the loads of kc + 3.
// KS = 2: half the columns, and two of the waves take the other 16 k of a stage, for outputs whose workgroups would not fill the chip.
template <bool UP, int KS>
__global__ __launch_bounds__(256, 2) void k_experts_f32_tile(const float* W, const float* W2, const float* X, long long ldx, int N, int K, Plan p, float* out) {
  constexpr int S = 4, WR = 64 / KS, COLS = UP ? WR / 2 : WR, PER = (64 + WR) / 32;
  __shared__ __attribute__((aligned(1024))) f32x4 ring[S][64 + WR][8]; // rows 0 - 63: x; then the weights (up: half of them of each matrix)
  if ((int)blockIdx.y >= *p.n_blocks) return;
  const Block b = p.blocks[blockIdx.y];
  const int lane = threadIdx.x & 63, w = wave_index(), n0 = blockIdx.x * COLS, stages = (K + 31) >> 5;
  const int unit = (lane & 7) ^ (lane >> 3);            // what this lane fetches of its rows' stage
  const float* src[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int r = (w * PER + i) * 8 + (lane >> 3);
    if ((w * PER + i) * 8 < 64) {                       // (scalar)
      const int slot = b.slot + min(r, b.rows - 1);
      src[i] = X + (UP ? p.row_of[slot] : slot) * ldx;
    } else {
      const int c = r - 64, n = min(n0 + c % COLS, N - 1);
      src[i] = (UP && c >= COLS ? W2 : W) + ((size_t)b.expert * N + n) * K;
    }
  }
  auto issue = [&](int kc) {                            // (units behind K: its last one again; stages behind the last one: never read)
    const int k = min(min(kc, stages - 1) * 32 + unit * 4, K - 4);
#pragma unroll
    for (int i = 0; i < PER; ++i)
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src[i] + k),
                                       (__attribute__((address_space(3))) void*)&ring[kc % S][(w * PER + i) * 8][0], 16, 0, 0);
  };
  const int l16 = lane & 15, q4 = lane >> 4, wm = (w & 1) * 32, wn = KS == 1 ? w >> 1 : 0, half = w >> 1;
  const int wr[2] = {64 + wn * (UP ? 16 : 32), UP ? 64 + COLS + wn * 16 : 80 + wn * 32};     // this wave's two weight tiles
  f32x4 sum[2 / KS][2][2];                              // a sum for each 16 k of a stage: half as long, half the roundings in a row
#pragma unroll
  for (int i = 0; i < 8 / KS; ++i) sum[i >> 2][i >> 1 & 1][i & 1] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < S - 1; ++i) issue(i);
  for (int kc = 0; kc < stages; ++kc) {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((S - 2) * PER) : "memory");
    issue(kc + S - 1);
    const auto& st = ring[kc % S];
    const bool tail = kc * 32 + 32 > K;                 // (scalar)
#pragma unroll
    for (int h = 0; h < 2 / KS; ++h) {
      const int u = (KS == 1 ? h : half) * 4 + q4, at = u ^ (l16 & 7);
      f32x4 xv[2], wv[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) { xv[i] = st[wm + i * 16 + l16][at]; wv[i] = st[wr[i] + l16][at]; }
      if (tail && kc * 32 + u * 4 >= K) {
#pragma unroll
        for (int i = 0; i < 2; ++i) xv[i] = wv[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) sum[h][i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(xv[i][e], wv[j][e], sum[h][i][j], 0, 0, 0);
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // the last stages' loads still write to LDS
  f32x4 acc[2][2];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    acc[i >> 1][i & 1] = sum[0][i >> 1][i & 1];
    if constexpr (KS == 1) acc[i >> 1][i & 1] += sum[1][i >> 1][i & 1];
  }
  if constexpr (KS == 2) {                              // the halves of K: the first two waves add the others' to theirs
    __syncthreads();
    f32x4(*other)[4][64] = reinterpret_cast<f32x4(*)[4][64]>(&ring[0][0][0]);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (half) other[w & 1][i][lane] = acc[i >> 1][i & 1];
    __syncthreads();
    if (half) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i >> 1][i & 1] += other[w][i][lane];
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int m = wm + i * 16 + q4 * 4 + v;
      if (m >= b.rows) continue;
      float* row = out + (size_t)(b.slot + m) * N;
      if (UP) {
        const int n = n0 + wn * 16 + l16;
        if (n < N) row[n] = silu(acc[i][0][v]) * acc[i][1][v];
      } else {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int n = n0 + wn * 32 + j * 16 + l16;
          if (n < N) row[n] = acc[i][j][v];
        }
      }
    }
}

// --------------------------------------------------------------------------------------------------------------- combine
// One thread per 4 columns of a row.  It reads what the product has just written: 117 MB in 20 us.
__global__ __launch_bounds__(256) void k_experts_combine(const int* __restrict__ slot_of, const float* __restrict__ weights, const float* __restrict__ out, int k, int d,
                                                         int parts, void* y, int y_type, long long ldy) {
  const int t = blockIdx.x / parts, c = ((blockIdx.x - t * parts) * 256 + threadIdx.x) * 4;
  if (c >= d) return;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int j = 0; j < k; ++j) {
    const int slot = slot_of[(size_t)t * k + j];
    if (slot < 0) continue;
    const float w = weights[(size_t)t * k + j];
    const float4 v = *reinterpret_cast<const float4*>(out + (size_t)slot * d + c);
    s.x += w * v.x; s.y += w * v.y; s.z += w * v.z; s.w += w * v.w;
  }
  if (y_type == X_F32) *reinterpret_cast<float4*>((float*)y + t * ldy + c) = s;
  else *reinterpret_cast<uint2*>((bf16_t*)y + t * ldy + c) = make_uint2(pk_bf16(s.x, s.y), pk_bf16(s.z, s.w));
}

void launch_pack_experts(const void* w, void* out, int E, int N, int K, hipStream_t s) {
  for (int e = 0; e < E; ++e)
    launch_pack_bf16((const bf16_t*)w + (size_t)e * N * K, (bf16_t*)out + (size_t)e * expert_elems(N, K), N, K, s);
}

namespace {
// Float32: rows of a block, by the rows r that an expert has in the mean.  us of up + down, 16 / 64: 8 experts of 512 x 2048 at r = 12 20 + 16 /
// 28 + 31, 24 28 + 18 / 29 + 31, 50 49 + 32 / 28 + 31; 16 of 1024 x 2048 at r = 16 86 + 48 / 96 + 50, 32 129 + 76 / 97 + 51, 128 418 + 248 / 236 + 142.
int f32_block_rows(int r) { return r > 24 ? 64 : 16; }
bool few(int dtype, long long T) { return dtype == SPRINTER_BF16 && T <= FEW_ROWS; }
// Shares of the K of down_few: a workgroup per compute unit.  us, 1 / 2 / 4 shares with the launch that joins them: 2 experts of 4096 x 14336
// 42 / 45 / 45, 56 of 2048 x 1024 (half as many column tiles) 65 / 45 / 46.  Fewer columns, whole calls of 16 rows and of 1, one share / this
// rule: 8 experts of 256 x 704 11.1 / 10.3 and 7.3 / 8.6 (16 shares), 8 of 512 x 1344 16.3 / 13.1 and 8.0 / 9.1, 64 of them 82 / 50 and 13.6 / 11.5 (8),
// 16 of 1024 x 2048 45 / 37 and 14.4 / 15.1 (4).
int few_shares(int d) { const int tiles = (d + 15) / 16; return (256 + tiles - 1) / tiles; }

struct Space {
  Plan plan; int slots, blocks; void *rows, *hidden; float *out, *row_weights; size_t bytes;
};
// pairs and experts bound the slots: every expert named rounds its own up to 16.
Space space(void* base, int dtype, int E, int d, int ff, long long T, int k) {
  const long long pairs = T * k, named = std::min<long long>(E, pairs);
  const bool bf = dtype == SPRINTER_BF16;
  size_t at = 0;
  auto take = [&](size_t n) { void* p = (char*)base + at; at += (n + 255) & ~(size_t)255; return p; };
  Space s{};
  if (few(dtype, T)) {
    s.hidden = take((size_t)named * FEW_ROWS * round_up(ff, 32) * 2);
    s.row_weights = (float*)take((size_t)named * FEW_ROWS * 4);
    s.out = (float*)take((size_t)few_shares(d) * FEW_ROWS * d * 4);
  } else {
    s.slots = (int)((pairs + 15 * named + 15) / 16 * 16);
    s.blocks = s.slots / 16;
    s.plan.n_blocks = (int*)take(4);
    s.plan.blocks = (Block*)take((size_t)s.blocks * sizeof(Block));
    s.plan.row_of = (int*)take((size_t)s.slots * 4);
    s.plan.slot_of = (int*)take((size_t)pairs * 4);
    s.rows = bf ? take((size_t)T * round_up(d, 32) * 2) : nullptr;
    s.hidden = take((size_t)s.slots * (bf ? (size_t)round_up(ff, 32) * 2 : (size_t)ff * 4));
    s.out = (float*)take((size_t)s.slots * d * 4);
  }
  s.bytes = at;
  return s;
}
}  // namespace

// Enough for any call of up to T rows.
size_t experts_workspace(int dtype, int E, int d, int ff, long long T, int k) {
  return std::max(space(nullptr, dtype, E, d, ff, T, k).bytes, space(nullptr, dtype, E, d, ff, std::min<long long>(T, FEW_ROWS), k).bytes);
}

void launch_experts(const ExpertsArgs& a, void* workspace, hipStream_t s) {
  const Space w = space(workspace, a.dtype, a.E, a.d, a.ff, a.T, a.k);
  const int pairs = a.T * a.k, named = std::min(a.E, pairs);
  if (few(a.dtype, a.T)) {
    const int up = (a.ff + 31) / 32 * 2, Nt = (a.d + 15) / 16, shares = few_shares(a.d);
    hipLaunchKernelGGL(k_experts_up_few, dim3(named * up), dim3(512), 0, s, a.wg, a.wu, a.x, a.ids, a.weights, a.T, a.k, a.E, a.d, a.ff, a.ldx, a.x_type, up,
                       (uint4*)w.hidden, w.row_weights);
    hipLaunchKernelGGL(k_experts_down_few, dim3(Nt * shares), dim3(512), 0, s, a.w2, (const uint4*)w.hidden, w.row_weights, a.ids, a.T, a.k, a.E, a.d, a.ff, shares, w.out, a.y, a.y_type, a.ldy);
    if (shares > 1)
      hipLaunchKernelGGL(k_experts_join, dim3(a.T * ((a.d + 255) / 256)), dim3(256), 0, s, w.out, shares, a.T, a.d, a.y, a.y_type, a.ldy);
    return;
  }
  const bool f32 = a.dtype == SPRINTER_F32, copy = !f32 && a.x_type != X_F16;
  const int tile = f32 ? 0 : expert_tile_choice(a.E, pairs, a.d, a.ff), block_rows = f32 ? f32_block_rows(pairs / named) : expert_tile_rows(tile);
  const int blocks = pairs / block_rows + named, parts = (a.d / 4 + 255) / 256;
  const int share = std::max(1024, ((pairs + 15) / 16 + 1023) / 1024 * 1024), plans = (pairs + share - 1) / share;       // up to 16 workgroups
  const int copies = copy ? (int)std::min<long long>(1024, ((long long)a.T * round_up(a.d, 32) / 8 + 1023) / 1024) : 0;
  hipLaunchKernelGGL(k_experts_plan, dim3(plans + copies), dim3(1024), 0, s, a.ids, pairs, a.k, a.E, block_rows, share, w.plan, plans, copies, (const bf16_t*)a.x, a.ldx,
                     (uint4*)w.rows, a.T, a.d);
  if (f32) {
    const float *x = (const float*)a.x, *hidden = (const float*)w.hidden;
    if (block_rows == 64) {
      // in halves where whole columns would give a compute unit less than two workgroups
      const int up = (a.ff + 31) / 32, down = (a.d + 63) / 64, live = pairs / 64 + (named + 1) / 2;
      if (up * live >= 512) hipLaunchKernelGGL((k_experts_f32_tile<true, 1>), dim3(up, blocks), dim3(256), 0, s, (const float*)a.wg, (const float*)a.wu, x, a.ldx, a.ff, a.d, w.plan, (float*)w.hidden);
      else hipLaunchKernelGGL((k_experts_f32_tile<true, 2>), dim3((a.ff + 15) / 16, blocks), dim3(256), 0, s, (const float*)a.wg, (const float*)a.wu, x, a.ldx, a.ff, a.d, w.plan, (float*)w.hidden);
      if (down * live >= 512) hipLaunchKernelGGL((k_experts_f32_tile<false, 1>), dim3(down, blocks), dim3(256), 0, s, (const float*)a.w2, nullptr, hidden, (long long)a.ff, a.d, a.ff, w.plan, w.out);
      else hipLaunchKernelGGL((k_experts_f32_tile<false, 2>), dim3((a.d + 31) / 32, blocks), dim3(256), 0, s, (const float*)a.w2, nullptr, hidden, (long long)a.ff, a.d, a.ff, w.plan, w.out);
    } else {
      hipLaunchKernelGGL(k_experts_f32<true>, dim3((a.ff + 15) / 16, blocks), dim3(512), 0, s, (const float*)a.wg, (const float*)a.wu, x, a.ldx, a.ff, a.d, w.plan,
                         (float*)w.hidden);
      hipLaunchKernelGGL(k_experts_f32<false>, dim3((a.d + 15) / 16, blocks), dim3(512), 0, s, (const float*)a.w2, nullptr, hidden, (long long)a.ff, a.d, a.ff, w.plan, w.out);
    }
  } else {
    launch_expert_tiles(tile, ExpertTiles{w.plan, blocks, w.slots, a.E, a.d, a.ff, a.wg, a.wu, a.w2, copy ? w.rows : a.x,
                                          copy ? (long long)round_up(a.d, 32) * 2 : a.ldx * 2, w.hidden, w.out}, s);
  }
  hipLaunchKernelGGL(k_experts_combine, dim3(parts * a.T), dim3(256), 0, s, w.plan.slot_of, a.weights, w.out, a.k, a.d, parts, a.y, a.y_type, a.ldy);
}

}  // namespace sprinter
