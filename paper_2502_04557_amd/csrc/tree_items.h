// How a launch of the attention of drafted trees is cut into items, and the room that the host leaves for them (k_tree_attn.hip).  Plain C++: the host
// and every workgroup compute the same numbers.
#pragma once

namespace sprinter {

constexpr int STEP = 128;                          // slots of a step
constexpr int MOST_STEPS = 1 << 23;                // of any sequence, whose slots are fewer than 2^30: a share of as many is the only one

// Steps of a share, the same for all sequences: a little more than the quotient, so that the roundings of the sum cannot make more items than there is room for.
// work: steps over all blocks of rows.
constexpr int steps_of_share(bool split, float work, int target) {
  if (!split) return MOST_STEPS;
  const float q = work * (1.001f / (float)target);
  return (q < (float)(MOST_STEPS - 1) ? (int)q : MOST_STEPS - 1) + 1;
}
constexpr int shares(int steps, int share) { return (steps + share - 1) / share; }

// Items to aim for per KV head: workgroups that the chip holds at once.
constexpr int tree_target(int KVH, int workgroups) { return (workgroups + KVH - 1) / KVH; }

// The most blocks of rows there can be (rows: nodes x heads of a KV head; sequences: those with a node at most), and the most items.
constexpr long long most_blocks(long long rows, int QB, long long sequences) { return rows / QB + sequences; }
constexpr long long most_items(long long blocks, bool split, int target) { return blocks + (split ? target + 1 : 0); }
// The most items that leave sums to be merged, those of sequences of two shares or more: these have fewer than 2 steps / share each, and a share is more than a
// target-th of all steps.
constexpr long long most_sums(long long items, bool split, int target) { return !split ? 0 : items < 2ll * target ? items : 2ll * target; }

}  // namespace sprinter
