"""The items of a launch of the attention of drafted trees against the room that the host leaves for them, up to the limits of its arguments, on the CPU."""
import ctypes as C
import os
import subprocess
import pytest
from test_abi_cpu import lib  # noqa: F401

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_04557_amd", "csrc")

PROGRAM = r"""
#include "tree_items.h"
#include <cstdio>
#include <random>
#include <vector>
using namespace sprinter;
struct Seq { int nodes; long long slots; };

// as the kernels do: blocks and steps of each sequence, the work as a float32 sum
bool fits(const std::vector<Seq>& batch, int G, int QB, int KVH, int workgroups, bool split) {
  long long rows = 0, items = 0, sums = 0;
  float work = 0;
  auto blocks = [&](const Seq& s) { return (int)(((long long)s.nodes * G + QB - 1) / QB); };
  auto steps = [&](const Seq& s) { const long long n = (s.slots + STEP - 1) / STEP; return (int)(n > 1 ? n : 1); };
  for (const Seq& s : batch) {
    rows += (long long)s.nodes * G;
    work += (float)blocks(s) * (float)steps(s);
  }
  const int target = tree_target(KVH, workgroups), share = steps_of_share(split, work, target);
  for (const Seq& s : batch) {
    const int parts = shares(steps(s), share);
    items += (long long)blocks(s) * parts;
    sums += parts > 1 ? (long long)blocks(s) * parts : 0;
    if (!split && parts != 1) return std::printf("split: %lld slots\n", s.slots), false;
    // every step is in a share, none is empty, and no slot of a share passes 31 bits
    if ((long long)parts * share < steps(s) || (long long)(parts - 1) * share >= steps(s) || ((long long)(parts - 1) * share + share) * STEP >= 1ll << 31)
      return std::printf("shares: %lld slots, %d shares of %d steps\n", s.slots, parts, share), false;
  }
  const long long room = most_items(most_blocks(rows, QB, (long long)batch.size()), split, target);
  if (items > room)
    return std::printf("%zu sequences, first %d nodes, %lld slots, %d heads each of %d, blocks of %d: %lld items, room for %lld\n", batch.size(), batch[0].nodes, batch[0].slots, G,
                       KVH, QB, items, room), false;
  if (sums > most_sums(room, split, target)) return std::printf("%zu sequences: %lld sums, room for %lld\n", batch.size(), sums, most_sums(room, split, target)), false;
  return true;
}

int main() {
  const long long most = (1ll << 30) - 8;
  bool ok = true;
  ok &= fits({{320, most}}, 16, 256, 32, 256, true);                   // 20 blocks of rows of the longest sequence
  ok &= fits({{8192, (1ll << 29) + 1}}, 64, 256, 1, 256, true);
  ok &= fits({{1, most}}, 1, 16, 1, 512, true);
  ok &= fits({{1, most}, {512 * 1000, 1}}, 1, 16, 1, 1, true);        // a share one step short of the longest sequence
  ok &= fits({{1, most}, {1, most}, {1, most}}, 1, 16, 512, 512, true);
  ok &= fits(std::vector<Seq>(1 << 20, Seq{1, most}), 1, 16, 1, 512, true);
  ok &= fits(std::vector<Seq>(1 << 20, Seq{1, 0}), 1, 16, 1, 512, true);
  ok &= fits(std::vector<Seq>(1 << 20, Seq{1, 17 * STEP}), 8, 16, 1, 512, false);
  std::mt19937 g(1);
  auto upto = [&](double hi) { return std::exp2(std::uniform_real_distribution<double>(0, std::log2(hi))(g)); };
  for (int i = 0; i < 20000 && ok; ++i) {
    const int KVH = (int)upto(1024), G = (int)upto(64), n = (int)upto(300);
    const int shapes[5][2] = {{16, 512}, {32, 512}, {64, 512}, {128, 512}, {256, 256}}, *shape = shapes[g() % 5];
    const double nodes = upto((1 << 23) / (double)n / G / KVH + 1), slots = upto((double)most);
    std::vector<Seq> batch;
    for (int b = 0; b < n; ++b) batch.push_back({(int)(g() % 4 ? upto(nodes) : g() % 2), (long long)(g() % 4 ? upto(slots) : slots)});
    ok &= fits(batch, G, shape[0], KVH, shape[1], true);
  }
  return ok ? 0 : 1;
}
"""


def test_there_is_room_for_every_item(tmp_path):
    src = tmp_path / "items.cpp"
    src.write_text("#include <cmath>\n" + PROGRAM)
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(tmp_path / "items")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(tmp_path / "items")], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout


@pytest.mark.parametrize("dtype, H, KVH, dh, n_seq, slots, T, most", [
    (1, 32, 32, 128, 1024, 4096, 1024, 9 << 20),          # decode steps of a large batch
    (1, 32, 8, 128, 1, 1 << 17, 4096, 72 << 20),          # a piece of a prompt
    (1, 64, 8, 128, 1 << 17, 1 << 20, 1 << 17, 96 << 20), # the most rows
    (0, 1, 1, 128, 1 << 20, 1 << 20, 1 << 20, 96 << 20),
    (1, 32, 8, 128, 64, 2048, 4096, 0)])                  # sequences that are not split
def test_sums_of_split_sequences_alone_take_workspace(lib, dtype, H, KVH, dh, n_seq, slots, T, most):  # noqa: F811
    """Twice as many items as the launch aims for leave sums at most, however large the batch is: 2 x 512 x 256 rows x 130 x 4 bytes, and the list of items."""
    from paper_2502_04557_amd import operators as ops
    n = C.c_size_t(0)
    cfg = ops.CacheCfgC(dtype, 1, 1 << 20, 16, KVH, dh)
    assert lib.sprinter_cache_attend_bytes(C.byref(cfg), H, n_seq, slots // 16, T, C.byref(n)) == 0
    assert n.value <= most
