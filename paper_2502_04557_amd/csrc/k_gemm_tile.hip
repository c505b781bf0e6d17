// HIP kernel of the batched SPRINTER decode step for gfx950: the GEMMs of 17 and more rows (prefill chunks, work lists, larger
// batches).
#include "gemm_tile.h"
#include <algorithm>
#include <type_traits>
#include <cstring>

namespace sprinter {

// whole: workgroups with a whole tile; those behind them (256 x 256 tile only) take half a tile each.
template <typename T, int EPI>
__global__ __launch_bounds__(T::waves * 64, T::pinned ? 1 : 2) void k_gemm_tile(const void* W_, const void* X_, const void* second_, int Kt_, int N_, int x_tiles, int gm, int gn, int whole,
                                                                                  const int* n_rows_, void* out_, int ldo_, int rows_live_, int half_, int shares_, size_t part_stride_,
                                                                                  GemmMore<EPI> more_) {
  GemmArgs a;                                           // second: bias, or W2; out: EPI_PART: the shares' buffer; half_: workgroups with half a tile
  a.W = W_; a.X = X_; a.W2 = second_; a.bias = EPI == EPI_SWIGLU ? nullptr : (const float*)second_; a.Kt = Kt_; a.N = N_; a.n_tiles = (N_ + 15) >> 4;
  a.n_rows = n_rows_; a.out_f32 = a.part = (float*)out_; a.out_act = out_; a.ldo = a.out_K = ldo_; a.rows_live = rows_live_; a.part_stride = part_stride_;
  if constexpr (EPI == EPI_QKV) a.kv = more_;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[T::stages * (T::wm * T::mt + T::wn * T::nt) * 1024];
  const int id = blockIdx.x;
  int bm, bn;
  if constexpr (T::pinned && EPI != EPI_PART) {         // (partial products: several shares, never in halves)
    if (id >= whole) {                                  // (scalar)
      const int t = xcd_run(id - whole, half_);
      tile_place<T>(whole + (t >> 1), gm, gn, bm, bn);
      gemm_tile<TileH, EPI>(a, x_tiles, bm, 2 * bn + (t & 1), 0, 1, lds);
      return;
    }
  }
  tile_place<T>(xcd_run(id, whole), gm, gn, bm, bn);
  gemm_tile<T, EPI>(a, x_tiles, bm, bn, EPI == EPI_PART ? blockIdx.y : 0, EPI == EPI_PART ? shares_ : 1, lds);
}

// Which tile, and how many K shares (partial products), for a shape: the one with the smallest estimate of
//   start + max(rounds of workgroups x cycles, padded products / rate, weights and shares / HBM rate) + the shares' way into the norm.
// Per tile: workgroups a compute unit holds, microseconds before the first product and after the last, cycles per k tile of a
// workgroup that has its compute unit for itself and what each further one adds, PFLOP/s on a full chip.  The constants are a fit to
// 1050 timings of 113 shapes (20 - 4096 rows, K 768 - 14336, N 768 - 14336, 1 - 8 shares) of the kernels before the 256 x 256 tile had four
// waves (1355 cycles and 1.22 PFLOP/s are those of eight, which GELU still takes), before a last round went out in halves and before one
// share added itself: here it counts as a partial product that the norm reads.  Against every tile and share count of the present kernels
// over 235 shapes (the products of five model pairs at 20 - 4096 rows, partial products with the norm behind them) the pick is 2.3 %
// slower than the best in the mean and 10 - 29 % at 21 of them: QKV and GELU of 4800 - 6400 columns at 140 - 300 rows (6400 x 1600 at 140
// rows 15.2 for 11.8 us), O-proj of 768 columns in two shares for one (2032 rows 19.3 for 15.7).
struct TileCost { int tm, tn, per_cu; float start_us, cycles, shared, rate; };
static float tile_us(const TileCost& c, int epi, int rows, int N, int Kt, int sk) {
  const int mats = epi == EPI_SWIGLU ? 2 : 1, cols = c.tn / mats, slots = 256 * c.per_cu;
  const int wgs = (rows + c.tm - 1) / c.tm * ((N + cols - 1) / cols) * sk, full = wgs / slots, rest = wgs % slots;
  const float kt = (float)Kt / sk, part = epi == EPI_PART ? 4.f * rows * N * sk : 0.f;
  float cycles = full * (c.cycles + c.shared * (c.per_cu - 1)) * kt;
  if (rest) cycles += (c.cycles + c.shared * ((rest + 255) / 256 - 1)) * kt;
  const float product = 2.f * wgs * c.tm * c.tn * kt * 32 / c.rate * 1e-9f, memory = (64.f * N * Kt * mats + part) / 6.3e6f;
  // the norm reads the shares at 4.5 TB/s; more than 4 take its larger variant
  return c.start_us + std::max(cycles / 2400.f, std::max(product, memory)) + part / 4.5e6f + (epi == EPI_PART && sk > 4 ? 0.3f : 0.f);
}

template <typename T, int EPI>
static void launch_tile(const GemmArgs& a, int rows, int sk, hipStream_t s) {
  constexpr int tm = T::wm * T::mt * 16, cols = T::wn * T::nt * 16 / (EPI == EPI_SWIGLU ? 2 : 1);
  const int x_tiles = (int)(a.x_elems / ((size_t)a.Kt * 512)), gm = (rows + tm - 1) / tm, gn = (a.N + cols - 1) / cols;
  const int tiles = gm * gn, rest = T::pinned && sk == 1 ? tiles_in_halves(tiles) : 0, whole = tiles - rest;
  hipLaunchKernelGGL((k_gemm_tile<T, EPI>), dim3(whole + 2 * rest, sk), dim3(T::waves * 64), 0, s, a.W, a.X, EPI == EPI_SWIGLU ? a.W2 : (const void*)a.bias, a.Kt, a.N,
                     x_tiles, gm, gn, whole, a.n_rows, EPI == EPI_PART ? (void*)a.part : EPI == EPI_GELU || EPI == EPI_SWIGLU ? a.out_act : (void*)a.out_f32,
                     EPI == EPI_GELU || EPI == EPI_SWIGLU ? a.out_K : a.ldo, a.rows_live, 2 * rest, sk, a.part_stride, gemm_more<EPI>(a));
}

int gemm_tile_choice(int epi, int rows, int N, int K, int max_shares) {
  static const TileCost cost[5] = {{256, 256, 1, 8.0f, 1355.f, 0.f, 1.22f}, {128, 128, 2, 5.4f, 608.f, 465.f, 1.10f},
                                   {64, 128, 2, 4.2f, 478.f, 200.f, 0.83f}, {64, 64, 2, 3.7f, 327.f, 517.f, 0.64f},
                                   {32, 64, 3, 3.4f, 290.f, 293.f, 1.23f}};
  const int Kt = (K + 31) / 32;
  int best = 0, sk = 1;
  float best_us = 1e30f;
  for (int i = 0; i < 5; ++i)
    for (int k = 1; k <= max_shares && (k == 1 || Kt / k >= 3); ++k) {
      const float us = tile_us(cost[i], epi, rows, N, Kt, k);
      if (us < best_us) { best_us = us; best = i; sk = k; }
    }
  return best * 16 + sk;
}

template <int EPI>
static void launch_tile_epi(int tile, const GemmArgs& a, int rows, int sk, hipStream_t s) {
  switch (tile) {
    case 0: launch_tile<std::conditional_t<EPI == EPI_GELU || EPI == EPI_QKV, TileG, TileL>, EPI>(a, rows, sk, s); break;
    case 1: launch_tile<TileM, EPI>(a, rows, sk, s); break;
    case 2: launch_tile<TileS, EPI>(a, rows, sk, s); break;
    case 3: launch_tile<TileX, EPI>(a, rows, sk, s); break;
    default: launch_tile<TileN, EPI>(a, rows, sk, s); break;
  }
}

// 17 - 64 rows of an output that cannot be left in K shares: the K-split kernel of k_gemm.hip, whose 8 waves share a column tile
// (a pair of them), runs one workgroup per compute unit, so its time jumps where its 256 are exceeded - at 128 workgroups of this
// kernel's narrowest tile.  Up to there it is ahead at K from about 1000 on (8192 x 4096 at 20 / 40 / 64 rows 15.5 / 17.4 / 19.5
// against 19.3 / 19.3 / 19.5 us; 8192 x 1600 8.7 / 10.1 / 10.7 against 10.6; 2 x 4096 x 4096 14.7 / 16.4 / 19.0 against 19.5); from
// 132 on this one is, at any K (8448 x 4096 22.2 / 25.6 / 31.6 against 19.4 / 22.5 / 22.7; 8448 x 512 7.1 / 8.6 / 8.1 against 4.8 /
// 5.4 / 5.6; 2 x 4224 x 2048 12.7 / 15.0 / 17.7 against 11.3 / 12.4 / 12.5).  Partial products are ahead at any size:
// 4096 x 4096 12.2 -> 8.8 at 20 rows, 1600 x 6400 9.7 -> 6.9, 4096 x 14336 33.9 -> 24.7 at 64; and so is everything from 65 rows
// on, where that kernel takes two passes (4800 x 1600 at 80 rows 12.2 -> 9.0, 2 x 3072 x 768 9.1 -> 6.8; 12288 x 4096 36.9 / 37.4).
bool gemm_takes_tile(int epi, int N, int rows) {
  const int cols = epi == EPI_SWIGLU ? 32 : 64;
  return rows > 64 || (rows > 16 && (epi == EPI_PART || (N + cols - 1) / cols > 128));
}

// A product in one K share is added to the residual rows by its own epilogue, so that the norm that follows reads the rows alone.
// Product and norm together, us: 4096 x 4096 at 4096 rows 159 -> 148, 4096 x 14336 408 -> 389, 2048 x 2048 65.4 -> 60.4, 768 x 768 24.3 ->
// 22.8, 1500 rows of 512 x 512 11.4 -> 10.2; nowhere slower than the noise where the rule above picks one share: from 17 rows where K leaves no
// two shares of three k tiles (up to 160), from 18 - 90 at K 256 - 1600 and the widest outputs, else from a few hundred.
int launch_gemm_tile(int epi, const GemmArgs& a, int rows, int max_shares, hipStream_t s) {
  const int choice = gemm_tile_choice(epi, rows, a.N, a.K, epi == EPI_PART ? max_shares : 1), tile = choice / 16, sk = choice % 16;
  switch (epi) {
    case EPI_F32: launch_tile_epi<EPI_F32>(tile, a, rows, 1, s); return 1;
    case EPI_GELU: launch_tile_epi<EPI_GELU>(tile, a, rows, 1, s); return 1;
    case EPI_QKV: launch_tile_epi<EPI_QKV>(tile, a, rows, 1, s); return 1;
    case EPI_SWIGLU: launch_tile_epi<EPI_SWIGLU>(tile, a, rows, 1, s); return 1;
  }
  if (sk > 1) { launch_tile_epi<EPI_PART>(tile, a, rows, sk, s); return sk; }
  launch_tile_epi<EPI_RESID>(tile, a, rows, 1, s);
  return 0;
}

}  // namespace sprinter
