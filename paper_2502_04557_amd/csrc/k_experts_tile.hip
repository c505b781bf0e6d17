// HIP kernels of the experts' products for gfx950: many rows, in row blocks of one expert each.
#include "gemm_tile.h"
#include "experts.h"
#include <algorithm>

namespace sprinter {

// up: hidden[slot] = silu(Wg x) * (Wu x) of the gathered rows, float16 operand tiles; down: out[slot] = W2 hidden[slot], float32.  The
// tiles and the loop are those of the dense products (gemm_tile.h); a row block's weights are its expert's.  How many blocks there are
// is only known on the device, so the grid is the most there can be; the workgroups behind them end at once.
// What bounds them: 8192 pairs, 8 experts of 4096 x 14336: 1730 and 857 us, 1.11 and 1.12 PFLOP/s of useful work (a library product of
// 8192 x 8192 x 8192: 1.22); the matrix instructions are busy 58 % of the cycles, the clock is 1.9 GHz, 7 % of the products are padding of
// row blocks, and the last round is half empty.  14312 pairs, 64 experts of 2048 x 1024: 211 and 111 us for 537 and 268 MB of weights and 0.18
// TFLOP: neither HBM nor the products are at their rate, the first loads and the epilogue of a tile are a fifth of its 64 k tiles.
// Measured and dropped: rows gathered into operand tiles ahead (up 4 % faster, the gathering 22 - 31 us); a stage more in the ring (equal);
// columns dealt out to the XCDs in turn, long row blocks first (5 % slower: the short ones, which wait for weights, no longer run beside
// the long ones).
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
    if (b.rows <= 64) { expert_tile<TileQ, EPI>(a, t, b, bn, lds); return; }
    if (b.rows <= 128) { expert_tile<TileT, EPI>(a, t, b, bn, lds); return; }
  }
  if constexpr (std::is_same_v<T, TileM>)
    if (b.rows <= 64) { expert_tile<TileS, EPI>(a, t, b, bn, lds); return; }
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
  static const int rows[N_EXPERT_TILES] = {256, 128, 64, 32};
  return rows[tile];
}

void launch_expert_tiles(int tile, const ExpertTiles& a, hipStream_t s) {
  switch (tile) {
    case 0: launch_pair<TileL>(a, s); break;
    case 1: launch_pair<TileM>(a, s); break;
    case 2: launch_pair<TileS>(a, s); break;
    default: launch_pair<TileN>(a, s); break;
  }
}

// Which tile, by the rows r that an expert has in the mean.  Whole calls, us, 256 x 256 / 128 x 128 / 64 x 128 / 32 x 64:
//   8 experts of 4096 x 14336    r = 8: - / 497 / 477 / 489   24: - / 513 / 497 / 565     64: 695 / 698 / 658 / 838    96: 723 / 765 / 749 / -      1024: 2599 / 3437 / 4399 / -
//   64 of 2048 x 1024            r = 8: - / 151 / 148 / 149   24: - / 168 / 161 / 171     96: 237 / 226 / 234 / 307    192: 313 / 299 / 341 / -     224: 327 / 339 / 382 / -      512: 555 / 646 / 759 / -
//   16 of 1024 x 2816            r = 12: - / 70 / 64 / 57     32: - / 78 / 70 / 68        128: 138 / 101 / 116 / -     384: 194 / 176 / 217 / -     512: 220 / 226 / 266 / -
//   4 of 2048 x 8192             r = 16: - / 128 / 115 / 96   32: - / 131 / 115 / 106     192: 266 / 178 / 180 / -     512: 323 / 310 / 373 / -     768: 391 / 410 / 505 / -
//   32 of 512 x 1344             r = 8: - / 45 / 40 / 37      96: 84 / 55 / 51 / 63       256: 114 / 82 / 86 / -       1024: 271 / 240 / 281 / -
// The largest tile has one workgroup per compute unit, so it needs most of three rounds of them and a K that hides its first loads and
// its epilogue; the narrowest one is ahead while 64 x 128 leaves compute units empty.
// r counts ids without an expert too, since only the device knows them: where a row's experts mostly lie on other devices the mean is too high by
// the number of devices, and the tile that is taken for it the slower one (never a wrong one: row blocks follow the plan).
int expert_tile_choice(int E, long long pairs, int d, int ff) {
  const long long used = std::min<long long>(E, pairs), r = pairs / used, cols = (ff + 127) / 128;
  const long long large = std::max((pairs / 256 + (used + 1) / 2) * cols, used * cols);         // (an expert's last row block is half empty in the mean)
  if (r >= 80 && d >= 1024 && large >= (d >= 2048 ? 683 : 768)) return 0;
  if (r > 112) return 1;
  return r <= 12 || (r <= 32 && used * ((ff + 63) / 64) <= 512) ? 3 : 2;
}

}  // namespace sprinter
