// What the kernels of the experts' products (k_experts.hip, k_experts_tile.hip) share.
#pragma once
#include "ops.h"
#include "dev.h"

namespace sprinter {

// Every pair (t, j) with an expert gets a slot; an expert's slots lie together and begin at a multiple of 16, so that 16 slots are one
// row tile of the matrix instruction and belong to one expert.  Which of its expert's slots a pair takes is left to chance: a row's
// products do not depend on the rows beside it, and the sum over j runs in the order of j.
struct Block { int expert, slot, rows, first, count; };   // up to block_rows slots of one expert, whose blocks are [first, first + count)
struct Plan {
  int* n_blocks; Block* blocks; int* row_of; int* slot_of;             // row_of [slots], slot_of [T k]
};

// The products of the pairs in row blocks (bf16 mode).  x: float16 rows of round_up(d, 32), zeros behind d.
struct ExpertTiles {
  Plan plan; int max_blocks, slots;                    // slots: as many as the buffers have
  int E, d, ff;
  const void *wg, *wu, *w2, *x; long long row_bytes;
  void* hidden; float* out;                            // operand tiles [slots, ff]; [slots, d]
};
constexpr int N_EXPERT_TILES = 4;
int expert_tile_rows(int tile);
// 0 - 3: 256 x 256, 128 x 128, 64 x 128, 32 x 64.
int expert_tile_choice(int E, long long pairs, int d, int ff);
void launch_expert_tiles(int tile, const ExpertTiles& a, hipStream_t s);

}  // namespace sprinter
