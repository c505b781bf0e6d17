// HIP kernels of the experts' products for gfx950: many rows, in row blocks of one expert each.
#include "gemm_tile.h"
#include "experts.h"
#include <algorithm>

namespace sprinter {

// up: hidden[slot] = silu(Wg x) * (Wu x) of the gathered rows, float16 operand tiles; down: out[slot] = W2 hidden[slot], float32.  The
// tiles and the loop are those of the dense products (gemm_tile.h); a row block's weights are its expert's.  How many blocks there are
// is only known on the device, so the grid is the most there can be; the workgroups behind them end at once.
struct TileArgs {
  const char *W, *W2; const void* X; size_t w_bytes;   // bytes of one expert's matrix
  int Kt, N, x_tiles, gn; const int* n_blocks; const Block* blocks; const int* row_of; long long row_bytes; void* out; int ldo;
};
template <typename T, int EPI>
__device__ __forceinline__ void expert_tile(const GemmArgs& a, const TileArgs& t, const Block& b, int bn, void* lds) {
  if constexpr (EPI == EPI_SWIGLU) gemm_tile<T, EPI>(a, t.x_tiles, 0, bn, 0, 1, lds, RowsGathered{b.slot >> 4, b.slot + b.rows, t.row_of, t.row_bytes});
  else gemm_tile<T, EPI>(a, t.x_tiles, 0, bn, 0, 1, lds, RowsOfTiles{b.slot >> 4, b.slot + b.rows});
}
template <typename T, int EPI>
__global__ __launch_bounds__(T::waves * 64, T::pinned ? 1 : 2) void k_expert_tile(TileArgs t) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[T::stages * (T::wm * T::mt + T::wn * T::nt) * 1024];
  const int tiles = *t.n_blocks * t.gn, rest = T::pinned ? tiles_in_halves(tiles) : 0, whole = tiles - rest, id = blockIdx.x;
  if (id >= whole + 2 * rest) return;
  // The tiles of an expert follow each other, in bands of equally many (up to 8) of its row blocks, those of a band together for each
  // column: what shares weights runs at one time on one XCD.  (In bands of 4, a fifth row block read all the weights for itself.)
  const int halves = T::pinned && id >= whole ? xcd_run(id - whole, 2 * rest) : 0, at = id < whole ? xcd_run(id, whole) : whole + (halves >> 1);
  Block b = t.blocks[at / t.gn];
  const int in = at - b.first * t.gn, bands = (b.count + 7) >> 3, height = (b.count + bands - 1) / bands, band = in / (height * t.gn);
  const int left = in - band * height * t.gn, rows = min(height, b.count - band * height), bn = left / rows;
  b = t.blocks[b.first + band * height + left - bn * rows];
  GemmArgs a;
  a.W = t.W + b.expert * t.w_bytes; a.W2 = EPI == EPI_SWIGLU ? t.W2 + b.expert * t.w_bytes : nullptr; a.X = t.X; a.bias = nullptr;
  a.Kt = t.Kt; a.N = t.N; a.n_tiles = (t.N + 15) >> 4; a.out_f32 = (float*)t.out; a.out_act = t.out; a.ldo = a.out_K = t.ldo;
  if constexpr (T::pinned) {
    if (id >= whole) { expert_tile<TileH, EPI>(a, t, b, 2 * bn + (halves & 1), lds); return; }
    if (b.rows <= 128) { expert_tile<TileT, EPI>(a, t, b, bn, lds); return; }
  }
  expert_tile<T, EPI>(a, t, b, bn, lds);
}

template <typename T>
static void launch_pair(const ExpertTiles& e, hipStream_t s) {
  const int up_cols = T::wn * T::nt * 8, down_cols = T::wn * T::nt * 16;
  TileArgs t{(const char*)e.wg, (const char*)e.wu, e.x, expert_elems(e.ff, e.d) * 2, (e.d + 31) / 32, e.ff, e.slots / 16, (e.ff + up_cols - 1) / up_cols,
             e.plan.n_blocks, e.plan.blocks, e.plan.row_of, e.row_bytes, e.hidden, e.ff};
  hipLaunchKernelGGL((k_expert_tile<T, EPI_SWIGLU>), dim3(e.max_blocks * t.gn + (T::pinned ? 128 : 0)), dim3(T::waves * 64), 0, s, t);
  t.W = (const char*)e.w2; t.X = e.hidden; t.w_bytes = expert_elems(e.d, e.ff) * 2; t.Kt = (e.ff + 31) / 32; t.N = e.d;
  t.gn = (e.d + down_cols - 1) / down_cols; t.out = e.out; t.ldo = e.d;
  hipLaunchKernelGGL((k_expert_tile<T, EPI_F32>), dim3(e.max_blocks * t.gn + (T::pinned ? 128 : 0)), dim3(T::waves * 64), 0, s, t);
}

int expert_tile_rows(int tile) {
  static const int rows[N_EXPERT_TILES] = {256, 128, 64, 64, 32};
  return rows[tile];
}

void launch_expert_tiles(int tile, const ExpertTiles& a, hipStream_t s) {
  switch (tile) {
    case 0: launch_pair<TileL>(a, s); break;
    case 1: launch_pair<TileM>(a, s); break;
    case 2: launch_pair<TileS>(a, s); break;
    case 3: launch_pair<TileX>(a, s); break;
    default: launch_pair<TileN>(a, s); break;
  }
}

// Per tile as for the dense products: workgroups a compute unit holds, microseconds before the first product and after the last, cycles
// per k tile of a workgroup alone and what each further one adds, PFLOP/s on a full chip.
struct Cost { int tm, tn, per_cu; float start_us, cycles, shared, rate; };
static float product_us(const Cost& c, int mats, float blocks, int E, int N, int K) {
  const int cols = c.tn / mats, Kt = (K + 31) / 32, slots = 256 * c.per_cu;
  const float wgs = blocks * ((N + cols - 1) / cols);
  const int full = (int)(wgs / slots), rest = (int)(wgs - (float)full * slots);
  float cycles = full * (c.cycles + c.shared * (c.per_cu - 1)) * Kt;
  if (rest) cycles += (c.cycles + c.shared * ((rest + 255) / 256 - 1)) * Kt;
  const float product = 2.f * wgs * c.tm * c.tn * Kt * 32 / c.rate * 1e-9f, memory = 64.f * N * Kt * mats * E / 6.0e6f;
  return c.start_us + std::max(cycles / 2400.f, std::max(product, memory));
}
int expert_tile_choice(int E, long long pairs, int d, int ff) {
  if (const char* v = getenv("ETILE")) return atoi(v);
  static const Cost cost[N_EXPERT_TILES] = {{256, 256, 1, 8.0f, 1355.f, 0.f, 1.22f}, {128, 128, 2, 5.4f, 608.f, 465.f, 1.10f},
                                            {64, 128, 2, 4.2f, 478.f, 200.f, 0.83f}, {64, 64, 2, 3.7f, 327.f, 517.f, 0.64f},
                                            {32, 64, 3, 3.4f, 290.f, 293.f, 1.23f}};
  const int used = (int)std::min<long long>(E, pairs);
  int best = 0;
  float best_us = 1e30f;
  for (int i = 0; i < N_EXPERT_TILES; ++i) {
    // an expert's last block is half empty in the mean
    const float blocks = std::max((float)used, (float)pairs / cost[i].tm + 0.5f * used);
    const float us = product_us(cost[i], 2, blocks, used, ff, d) + product_us(cost[i], 1, blocks, used, d, ff);
    if (us < best_us) { best_us = us; best = i; }
  }
  return best;
}

}  // namespace sprinter
