// HIP kernels of the attention of trees of drafted tokens over a cache in pages, for gfx950.
#include "ops.h"
#include "dev.h"
#include "tree_items.h"
#include <algorithm>
#include <cmath>
#include <type_traits>

namespace sprinter {

// A launch cuts the batch into items: a block of QB rows (node x head of one KV head) of a sequence against a share of its slots.  Lengths and trees are known
// on the device alone, so every workgroup works the cut out for itself from `lens` and `first` (more than 128 sequences: k_tree_plan does, once): `steps` of STEP slots
// over all blocks of rows, dealt out in shares of `share` steps so that about `target` items come out, however ragged the batch is.
struct TreeItem {
  int f0, n, len, b;                               // the sequence: rows f0 .. f0 + n - 1
  int block, part, parts, share;                   // block of rows, share of slots, how many of them, steps of each
  int sums;                                        // (parts > 1) which item it is among those of split sequences
};
struct TreePlan {
  int target, items;                               // shares to aim for; the most items there can be (per KV head)
  int split, sort, planned;                        // sequences may be split; the longest first; the items are listed before the launch
  TreeItem* list;                                  // [items] (split or planned) parts 0: there is none
  float* o;                                        // [most_sums][KVH][QB][DH] sums of split sequences, not divided, and
  float* ml;                                       // [most_sums][KVH][QB][2] the largest products q.k and the sums of weights
};

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

struct TreeSeq { int f0, n, len, blocks, steps; };
__device__ __forceinline__ TreeSeq tree_seq(const AttendArgs& a, int b, int QB, bool there) {
  TreeSeq s{0, 0, 0, 0, 0};
  if (there) {
    s.f0 = max(a.first[b], 0);
    s.n = max(min(a.first[b + 1], a.T) - s.f0, 0);
    s.len = max(a.lens[b], 0);
    s.blocks = (int)(((long long)s.n * (a.H / a.c.KVH) + QB - 1) / QB);
    s.steps = max(1, (int)((min((long long)s.len + s.n, (long long)a.c.n_table << a.c.shift) + STEP - 1) / STEP));
  }
  return s;
}

// Sums over the lanes up to this one (itself among them) of numbers from 0 to 2^30, where they stay; `all`: over the whole wave.
constexpr int MOST_ITEMS = 1 << 30;
__device__ __forceinline__ int scan_to_lane(int v, int& all) {
#define SPRINTER_SCAN_STEP(CTRL, ROWS) v = min(v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false), MOST_ITEMS)
  SPRINTER_SCAN_STEP(0x111, 0xF);   // row_shr:1, 2, 4, 8, then the last lanes of rows into the rows behind them
  SPRINTER_SCAN_STEP(0x112, 0xF);
  SPRINTER_SCAN_STEP(0x114, 0xF);
  SPRINTER_SCAN_STEP(0x118, 0xF);
  SPRINTER_SCAN_STEP(0x142, 0xA);
  SPRINTER_SCAN_STEP(0x143, 0xC);
#undef SPRINTER_SCAN_STEP
  all = __builtin_amdgcn_readlane(v, 63);
  return v;
}

__device__ __forceinline__ int tree_items(const TreeSeq& s, int parts) { return (int)min((long long)s.blocks * parts, (long long)MOST_ITEMS); }

// The item of index `item`, by one wave; false: there is none.
__device__ __forceinline__ bool find_item(const AttendArgs& a, const TreePlan& p, int QB, int item, TreeItem& out) {
  const int lane = threadIdx.x & 63, n = a.c.n_seq;
  TreeSeq s = tree_seq(a, lane, QB, lane < n);
  float work = (float)s.blocks * (float)s.steps;
  for (int b = lane + 64; b < n; b += 64) {
    const TreeSeq x = tree_seq(a, b, QB, true);
    work += (float)x.blocks * (float)x.steps;
  }
  work = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(wave_total(work)), 63));
  const int share = steps_of_share(p.split, work, p.target);
  // The longest sequences first, where workgroups wait for a place and one wave holds them all.
  int from = lane;                                 // the sequence that this lane stands for
  if (p.sort) {
    const int key = (s.blocks > 0 ? min(s.steps, 1 << 24) : 0) * 64 + 63 - lane;   // (no two alike)
    int rank = 0;
#pragma unroll
    for (int x = 0; x < 64; ++x) rank += __builtin_amdgcn_readlane(key, x) > key ? 1 : 0;
    auto to = [&](int v) { return __builtin_amdgcn_ds_permute(4 * rank, v); };
    s.f0 = to(s.f0); s.n = to(s.n); s.len = to(s.len); s.blocks = to(s.blocks); s.steps = to(s.steps);
    from = to(lane);
  }
  int base = 0, base_sums = 0;
  out.parts = 0;
  for (int b0 = 0; b0 < n; b0 += 64) {
    if (b0) s = tree_seq(a, b0 + lane, QB, b0 + lane < n);
    const int parts = shares(s.steps, share), mine = tree_items(s, parts);
    int all;
    const int before = base + scan_to_lane(mine, all) - mine, sums = parts > 1 ? mine : 0;
    int before_sums = base_sums, all_sums = 0;
    if (p.split) before_sums += scan_to_lane(sums, all_sums) - sums;
    const u64 hit = __ballot(item >= before && item < before + mine);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      out.b = b0 + __builtin_amdgcn_readlane(from, l);
      out.f0 = __builtin_amdgcn_readlane(s.f0, l);
      out.n = __builtin_amdgcn_readlane(s.n, l);
      out.len = __builtin_amdgcn_readlane(s.len, l);
      out.parts = __builtin_amdgcn_readlane(parts, l);
      out.share = uniform(share);
      const int i = item - __builtin_amdgcn_readlane(before, l);
      out.block = i / out.parts;
      out.part = i - out.block * out.parts;
      out.sums = __builtin_amdgcn_readlane(before_sums, l) + i;
      break;
    }
    base += all;
    base_sums += all_sums;
  }
  if (p.split && blockIdx.x % a.c.KVH == 0 && threadIdx.x == 0) p.list[item] = out;   // for k_tree_merge
  return out.parts > 0;
}
// The same by a workgroup: its first wave looks, the others get it through LDS.
__device__ __forceinline__ bool find_item_of_block(const AttendArgs& a, const TreePlan& p, int QB, TreeItem& out) {
  __shared__ TreeItem shared;
  if (p.planned) {
    out = p.list[blockIdx.x / a.c.KVH];
    return out.parts > 0;
  }
  if (wave_index() == 0) {
    find_item(a, p, QB, blockIdx.x / a.c.KVH, out);
    if (threadIdx.x == 0) shared = out;
  }
  __syncthreads();
  int v[9];
#pragma unroll
  for (int i = 0; i < 9; ++i) v[i] = uniform(reinterpret_cast<const int*>(&shared)[i]);
  out = TreeItem{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7], v[8]};
  return out.parts > 0;
}

// All items of a launch, by one workgroup: a list of as many entries as there is room for.
__global__ __launch_bounds__(1024) void k_tree_plan(AttendArgs a, TreePlan p, int QB) {
  __shared__ float wave_work[16];
  __shared__ int wave_items[16], wave_sums[16];
  const int tid = threadIdx.x, lane = tid & 63, w = wave_index(), n = a.c.n_seq;
  float work = 0.f;
  for (int b = tid; b < n; b += 1024) {
    const TreeSeq s = tree_seq(a, b, QB, true);
    work += (float)s.blocks * (float)s.steps;
  }
  work = wave_total(work);
  if (lane == 63) wave_work[w] = work;
  __syncthreads();
  work = 0.f;
  for (int x = 0; x < 16; ++x) work += wave_work[x];
  const int share = steps_of_share(p.split, work, p.target);
  int base = 0, base_sums = 0;
  for (int b0 = 0; b0 < n && base < p.items; b0 += 1024) {       // (the same for all threads)
    const TreeSeq s = tree_seq(a, b0 + tid, QB, b0 + tid < n);
    const int parts = shares(s.steps, share), mine = tree_items(s, parts), sums = parts > 1 ? mine : 0;
    int all, all_sums;
    const int upto = scan_to_lane(mine, all), upto_sums = scan_to_lane(sums, all_sums);
    if (lane == 0) { wave_items[w] = all; wave_sums[w] = all_sums; }
    __syncthreads();
    int before = base, total = base, before_sums = base_sums;
    for (int x = 0; x < 16; ++x) {
      if (x < w) before = min(before + wave_items[x], MOST_ITEMS);
      total = min(total + wave_items[x], MOST_ITEMS);
      if (x < w) before_sums += wave_sums[x];
      base_sums += wave_sums[x];
    }
    __syncthreads();
    base = total;
    before = min(before + (upto - mine), MOST_ITEMS);
    before_sums += upto_sums - sums;
    for (u64 some = __ballot(mine > 0 && before < p.items); some; some &= some - 1) {   // a sequence's items by the whole wave
      const int l = __builtin_ctzll(some), from = __builtin_amdgcn_readlane(before, l), count = min(__builtin_amdgcn_readlane(mine, l), p.items - from);
      TreeItem it{__builtin_amdgcn_readlane(s.f0, l), __builtin_amdgcn_readlane(s.n, l), __builtin_amdgcn_readlane(s.len, l), b0 + 64 * w + l, 0, 0,
                  __builtin_amdgcn_readlane(parts, l), share, 0};
      const int from_sums = __builtin_amdgcn_readlane(before_sums, l);
      for (int x = lane; x < count; x += 64) {
        it.block = x / it.parts;
        it.part = x - it.block * it.parts;
        it.sums = from_sums + x;
        p.list[from + x] = it;
      }
    }
  }
  for (int x = base + tid; x < p.items; x += 1024) p.list[x].parts = 0;
}

// bf16: 32 keys a block, of which a lane ends up with the scores of 8; float32: 16 and 4.
template <typename T> struct Tree {};
template <> struct Tree<bf16_t> { static constexpr int KB = 32, NK = 8, VEC = 8; };
template <> struct Tree<float> { static constexpr int KB = 16, NK = 4, VEC = 4; };

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// Which of a lane's NK keys a row sees: those from node j0 on (below 0: committed), of which `there` are there.  first: the row's first word of `visible`.
template <int NK>
__device__ __forceinline__ unsigned seen_keys(const AttendArgs& a, u64 first, long long row, int node, int j0, unsigned there) {
  unsigned see = (1u << NK) - 1;
  if (j0 + NK > 0) {
    if (a.visible) {
      const int j = max(j0, 0), word = j >> 6, sh = j & 63;
      const unsigned long long* v = a.visible + row * a.n_words;
      see = (unsigned)(first >> sh);
      if (word) see = word < a.n_words ? (unsigned)(v[word] >> sh) : 0u;
      if (sh > 64 - NK && word + 1 < a.n_words) see |= (unsigned)(v[word + 1] << (64 - sh));
      if (j0 < 0) see = see << -j0 | ((1u << -j0) - 1);
    } else {
      see = (1u << min(max(node - j0 + 1, 0), NK)) - 1;
    }
  }
  return see & there;
}

// The scores of a lane's NK keys (of one row, in p) become weights; m is their running maximum, l the lane's sum of weights.  A weight is a power of 2 with the exponent
// p c - m c, where m c stands for its rounding, as long as that is at most 2^24: the rounding is the same for all and at most 1.  Beyond (steep) it could be any
// power, and the exponent is (p - m) c, which is 0 for the largest and finite or -infinity for every finite score.  lacks: how much less than m c a weight's exponent is taken from;
// rescaling: what brings weights of the maximum `from` to those of `to`.
constexpr float LOW = -3.402823466e38f, STEEP = 16777216.f;
__device__ __forceinline__ float lacks(float m, float c) {
  const float x = m * c;
  return fabsf(x) > STEEP ? 0.f : fmaf(m, c, -x);
}
__device__ __forceinline__ float rescaling(float from, float to, float c) { return __builtin_amdgcn_exp2f((from - to) * c + (lacks(to, c) - lacks(from, c))); }

// The maximum moves only when a score passes it by more than 2^8 (uniform: any row of the wave), so that the common block needs no exchange between lanes: weights
// up to 2^8 cost float32 sums and bf16 pairs nothing.  masked: keys outside `bits` have weight 0.
template <int NK, int N>
__device__ __forceinline__ void softmax_step(float (&p)[NK], bool masked, unsigned bits, const Base2& sc, float& m, float& l, f32x4 (&O)[N]) {
  if (masked) {
#pragma unroll
    for (int e = 0; e < NK; ++e) p[e] = bits >> e & 1 ? p[e] : -INFINITY;
  }
  float mx = p[0];
#pragma unroll
  for (int e = 1; e < NK; ++e) mx = fmaxf(mx, p[e]);
  float c = sc.c, mc = m * c;
  if (__any(mx > m + sc.lag || fabsf(mc) > STEEP)) {
    const float mn = fmaxf(m, fmaxf(quarter_max(mx), LOW));   // (NaN: left out here, and in the weights below)
    const float corr = rescaling(m, mn, c);
    l *= corr;
#pragma unroll
    for (int i = 0; i < N; ++i) O[i] *= corr;
    m = mn;
    mc = m * c;
    const bool steep = fabsf(mc) > STEEP;
    if (__any(steep)) {
#pragma unroll
      for (int e = 0; e < NK; ++e) p[e] = steep ? (p[e] - m) * c : fmaf(p[e], c, -mc);
      c = 1.f;
      mc = 0.f;
    }
  }
#pragma unroll
  for (int e = 0; e < NK; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(p[e], c, -mc));
  if (masked) {                                    // (also where -infinity times a scale of 0 is NaN)
#pragma unroll
    for (int e = 0; e < NK; ++e) p[e] = bits >> e & 1 ? p[e] : 0.f;
  }
  float s[NK / 2];
#pragma unroll
  for (int e = 0; e < NK / 2; ++e) s[e] = p[2 * e] + p[2 * e + 1];
#pragma unroll
  for (int n = NK / 4; n > 0; n >>= 1)
#pragma unroll
    for (int e = 0; e < n; ++e) s[e] = s[2 * e] + s[2 * e + 1];
  l += s[0];
}

// An infinity among the committed values meets the two halves of a weight in bf16, the second of which may be 0 or negative: NaN, and so do sums of x[N], columns `col` of
// a row, whose sum of weights is l.  Where they are not finite (rare), what the row sees of infinities and NaN among the slots k0 .. end - 1 takes their place: weights are
// positive, so its plain sum has the value.  By a whole wave whose lanes with one lane / 16 have the same columns.
template <int N, typename Col>
__device__ __forceinline__ void take_infinities(const AttendArgs& a, const TreeItem& it, int kvh, int k0, int end, long long row, int node, float l, Col col, float (&x)[N]) {
  float z = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) z = fmaf(x[i], 0.f, z);
  if (!__any(z != z)) return;
  float sum[N] = {};
  auto add = [&](int s, bool sees) {
    const int page = a.c.table[(long long)it.b * a.c.ld_table + (s >> a.c.shift)];
    if (!sees || (unsigned)page >= (unsigned)a.c.n_page) return;
    const bf16_t* v = (const bf16_t*)a.c.values + ((((long long)page * a.c.KVH + kvh) << a.c.shift) + (s & ((1 << a.c.shift) - 1))) * a.c.dh;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float e = __uint_as_float((unsigned)v[col(i)] << 16);
      sum[i] += fabsf(e) < INFINITY ? 0.f : e;
    }
  };
  for (int s = k0 + (threadIdx.x & 15); s < min(it.len, end); s += 16) add(s, true);
#pragma unroll
  for (int i = 0; i < N; ++i)
    for (int d = 1; d < 16; d <<= 1) sum[i] += __shfl_xor(sum[i], d);
  for (int s = max(k0, it.len); s < end; ++s) {
    const int j = s - it.len;
    add(s, a.visible ? j < 64 * a.n_words && (a.visible[row * a.n_words + min(j >> 6, a.n_words - 1)] >> (j & 63) & 1) : j <= node);
  }
  if (l > 0.f && l < INFINITY) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = fabsf(sum[i]) < INFINITY ? x[i] : sum[i];
  }
}

// The attention of one item by NW waves, each with all QB = 16 QT rows and every NW-th block of the item's keys; one pass with running maxima and sums.
//   S^T = K Q^T: a lane holds the scores of one row (lane % 16).  bf16: row i of key tile t is key 8 (i / 4) + 4 t + i % 4, so that a lane's 8 scores are
//     those of the keys 8 (lane / 16) .. + 7, the operand layout of P.  float32: the 4 keys 4 (lane / 16) + r, one for each of four products.
//   O^T += V^T P^T: a lane fetches DH / 16 neighbouring columns of each of its keys, whole rows by 16 lanes; operand c takes column c of each
//     lane's, which for bf16 is one byte permutation per pair of keys.  The accumulators then hold DH / 4 neighbouring columns of a row.
// P enters as two bf16, 16 bits together: one alone would add an error as large as the result's own rounding (by its arithmetic 1.7e-3 ->
// 2.4e-3), for 10 % of the largest case's time.  For up to 32 rows of a sequence; a key costs the same for any of them.
// Bound by HBM where there is enough to read (128 sequences x 32 heads, 1 node, up to 1024 slots: 1.14 GB in 202 us = 5.6 TB/s; one sequence of 30000 slots: 26 us, its
// 123 MB take 20), else by a chain of 4 - 5 loads (lengths, table and queries, keys and values: 6 us).  Measured and dropped: registers for three workgroups on a
// compute unit (64 x 8 pairs, up to 2047 slots: 68 -> 75 us), 384 / 768 / 1024 / 1536 workgroups to split for instead of 512 (equal, or up to 15 % slower),
// 8 or 16 waves (one sequence of 500 / 1100 / 2000 slots unsplit: 4 waves 10.2 / 15.9 / 24.1 us, 8 waves 10.8 / 15.7 / 24.0: a compute unit fetches no faster).
template <typename T, int DH, int QT, int NW>
__global__ __launch_bounds__(NW * 64, 2) void k_tree_attn(AttendArgs a, TreePlan plan) {
  using P = Tree<T>;
  constexpr bool HALF = sizeof(T) == 2;
  constexpr int KB = P::KB, NK = P::NK, QB = 16 * QT, CPL = DH / 16, KF = DH / (HALF ? 32 : 16);   // columns of V per lane; 16-byte pieces of a key per lane and tile
  constexpr int KT = HALF ? 2 : 1;                 // key tiles
  constexpr int VW = CPL * sizeof(T) / 4;          // dwords of a key's columns
  __shared__ float merge[NW / 2][QB][DH];
  __shared__ float stats[NW][QB][2];
  TreeItem it;
  if (!find_item_of_block(a, plan, QB, it)) return;
  const int lane = threadIdx.x & 63, w = wave_index(), l16 = lane & 15, lq = lane >> 4, kvh = blockIdx.x % a.c.KVH, G = a.H / a.c.KVH;
  const int shift = a.c.shift, place_mask = (1 << shift) - 1;
  const int slots = (int)min((long long)it.len + it.n, (long long)a.c.n_table << shift);
  const int k0 = it.part * it.share * STEP, end = min(k0 + it.share * STEP, slots), sure = min(it.len, end);   // slots below `sure` are seen by every row
  const int* __restrict__ table = a.c.table + (long long)it.b * a.c.ld_table;

  // this lane's rows
  long long at_q[QT];
  int node[QT];
  bool row_there[QT];
  u64 first_word[QT];
  u32x4 q[QT][KF];
  const Base2 scale = a.scale;
  const unsigned flip = scale.flip ? (HALF ? 0x80008000u : 0x80000000u) : 0u;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const long long i = (long long)it.block * QB + 16 * t + l16;
    row_there[t] = i < (long long)it.n * G;
    const int g = (int)(i % G);
    node[t] = row_there[t] ? (int)(i / G) : 0;
    at_q[t] = (long long)(it.f0 + node[t]);
    first_word[t] = a.visible ? a.visible[at_q[t] * a.n_words] : 0;
    const T* src = (const T*)a.q + at_q[t] * a.ld_q + ((row_there[t] ? g : 0) + kvh * G) * DH;
#pragma unroll
    for (int f = 0; f < KF; ++f) {
      q[t][f] = *reinterpret_cast<const u32x4*>(src + f * (HALF ? 32 : 16) + lq * P::VEC);
      q[t][f] = row_there[t] ? q[t][f] ^ flip : (u32x4){0, 0, 0, 0};
    }
  }

  u32x4 K[KT][KF];
  u32x4 V[NK][(VW + 3) / 4];                       // (8 bytes of 64 columns of bf16: half a piece)
  int page_k = 0, page_v = 0, next_k = 0, next_v = 0;   // entries of the table for this block's pieces of 8 keys
  const int gk = HALF ? l16 >> 2 : l16 >> 3, gv = HALF ? lq : lq >> 1;
  const int last = max(a.c.n_table - 1, 0);
  auto fetch_pages = [&](int kb) {
    next_k = table[min((kb + 8 * gk) >> shift, last)];
    next_v = table[min((kb + 8 * gv) >> shift, last)];
  };
  auto ok = [&](int page) { return (unsigned)page < (unsigned)a.c.n_page; };
  auto base = [&](int page, int s) {               // the first element of a slot of this KV head (of page 0 where the page is not there: read, not used)
    return ((((long long)(ok(page) ? page : 0) * a.c.KVH + kvh) << shift) + (s & place_mask)) * DH;
  };
  auto fetch_k = [&](int kb) {
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      const T* src = (const T*)a.c.keys + base(page_k, kb + 8 * gk) + (HALF ? (l16 & 3) + 4 * t : l16 & 7) * DH + lq * P::VEC;
#pragma unroll
      for (int f = 0; f < KF; ++f) K[t][f] = *reinterpret_cast<const u32x4*>(src + f * (HALF ? 32 : 16));
    }
  };
  long long v_at = 0;
  auto fetch_v = [&](int kb) {
    v_at = base(page_v, kb + 8 * gv) + (HALF ? 0 : (4 * lq & 7)) * DH;
    const T* src = (const T*)a.c.values + v_at + l16 * CPL;
#pragma unroll
    for (int j = 0; j < NK; ++j) {
      if constexpr (VW == 2) {
        const u32x2 x = *reinterpret_cast<const u32x2*>(src + j * DH);
        V[j][0][0] = x[0]; V[j][0][1] = x[1];
      } else {
#pragma unroll
        for (int i = 0; i < VW / 4; ++i) V[j][i] = *reinterpret_cast<const u32x4*>(src + j * DH + i * P::VEC);
      }
    }
  };

  f32x4 O[QT][CPL];
  float m_run[QT], l_run[QT];                      // largest product q.k and this lane's sum of weights
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m_run[t] = LOW; l_run[t] = 0.f;
#pragma unroll
    for (int i = 0; i < CPL; ++i) O[t][i] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }
  int kb = k0 + w * KB;
  if (kb < end) {
    fetch_pages(kb);
    page_k = next_k; page_v = next_v;
    fetch_k(kb);
    fetch_v(kb);
    fetch_pages(kb + NW * KB);
  }
  // One block of KB keys, and the requests for the wave's next one.  plain: every key is there and seen by every row.
  auto attend = [&](auto is_plain) __attribute__((always_inline)) {
    constexpr bool plain = decltype(is_plain)::value;
    const bool v_ok = ok(page_v);
    f32x4 sc[QT][KT];
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int k = 0; k < KT; ++k) sc[t][k] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int f = 0; f < KF; ++f)
#pragma unroll
      for (int k = 0; k < KT; ++k)
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          if constexpr (HALF) {
            sc[t][k] = mfma_bf16(__builtin_bit_cast(uint4, K[k][f]), __builtin_bit_cast(uint4, q[t][f]), sc[t][k]);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[t][k] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(K[k][f][i]), __uint_as_float(q[t][f][i]), sc[t][k], 0, 0, 0);
          }
        }
    __builtin_amdgcn_sched_barrier(0);
    const long long v_here = v_at;
    page_k = next_k;
    const int page_v_next = next_v;
    if (kb + NW * KB < end) fetch_k(kb + NW * KB);
    __builtin_amdgcn_sched_barrier(0);

    float p[QT][NK];
    unsigned bits[QT];
    const int kl = kb + NK * lq;                   // this lane's first key
    const unsigned there = plain ? (1u << NK) - 1 : v_ok ? (1u << min(max(end - kl, 0), NK)) - 1 : 0u;
    uint4 ph[QT], pl[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
#pragma unroll
      for (int e = 0; e < NK; ++e) p[t][e] = sc[t][e >> 2][e & 3];
      bits[t] = plain ? there : seen_keys<NK>(a, first_word[t], at_q[t], node[t], kl - it.len, there);
      softmax_step(p[t], !plain, bits[t], scale, m_run[t], l_run[t], O[t]);
      if constexpr (HALF) {
        split2(p[t][0], p[t][1], ph[t].x, pl[t].x);
        split2(p[t][2], p[t][3], ph[t].y, pl[t].y);
        split2(p[t][4], p[t][5], ph[t].z, pl[t].z);
        split2(p[t][6], p[t][7], ph[t].w, pl[t].w);
      }
    }
    // What no row, or not every row, sees must not meet a weight of 0 as an infinity or NaN: slots that are not there are cleared, and elements of nodes
    // that are not finite are taken out here and added below to the rows that see them.
    unsigned bad = 0;                              // which of this lane's keys have an element that is not finite here
    if constexpr (!plain) {
      if (__any(there != (1u << NK) - 1)) {
#pragma unroll
        for (int j = 0; j < NK; ++j)
#pragma unroll
          for (int i = 0; i < VW; ++i) V[j][i / 4][i & 3] = there >> j & 1 ? V[j][i / 4][i & 3] : 0u;
      }
      if (kb + KB > it.len) {
        bool some = false;
        if constexpr (HALF) {
          u16x2 top = {0, 0};                      // the largest magnitudes, as integers: 0x7f80 and more are not finite
#pragma unroll
          for (int j = 0; j < NK; ++j)
#pragma unroll
            for (int i = 0; i < VW; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, V[j][i / 4][i & 3] & 0x7fff7fffu));
          some = top[0] >= 0x7f80 || top[1] >= 0x7f80;
        } else {
          unsigned top = 0;
#pragma unroll
          for (int j = 0; j < NK; ++j)
#pragma unroll
            for (int i = 0; i < VW; ++i) top = max(top, V[j][i / 4][i & 3] & 0x7fffffffu);
          some = top >= 0x7f800000u;
        }
        if (__any(some)) {
#pragma unroll
          for (int j = 0; j < NK; ++j)
#pragma unroll
            for (int i = 0; i < VW; ++i) {
              unsigned x = V[j][i / 4][i & 3];
              if constexpr (HALF) {
                const bool lo = kl + j >= it.len && (x & 0x7f80u) == 0x7f80u, hi = kl + j >= it.len && (x & 0x7f800000u) == 0x7f800000u;
                bad |= (lo || hi ? 1u : 0u) << j;
                x &= (lo ? 0xffff0000u : 0xffffffffu) & (hi ? 0x0000ffffu : 0xffffffffu);
              } else {
                const bool b = kl + j >= it.len && (x & 0x7f800000u) == 0x7f800000u;
                bad |= (b ? 1u : 0u) << j;
                x = b ? 0u : x;
              }
              V[j][i / 4][i & 3] = x;
            }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      if constexpr (HALF) {
        uint4 vf;
        const unsigned sel = i & 1 ? 0x07060302u : 0x05040100u;
        vf.x = __builtin_amdgcn_perm(V[1][i / 8][(i >> 1) & 3], V[0][i / 8][(i >> 1) & 3], sel);
        vf.y = __builtin_amdgcn_perm(V[3][i / 8][(i >> 1) & 3], V[2][i / 8][(i >> 1) & 3], sel);
        vf.z = __builtin_amdgcn_perm(V[5][i / 8][(i >> 1) & 3], V[4][i / 8][(i >> 1) & 3], sel);
        vf.w = __builtin_amdgcn_perm(V[7][i / 8][(i >> 1) & 3], V[6][i / 8][(i >> 1) & 3], sel);
#pragma unroll
        for (int t = 0; t < QT; ++t) O[t][i] = mfma_bf16(vf, ph[t], O[t][i]);
#pragma unroll
        for (int t = 0; t < QT; ++t) O[t][i] = mfma_bf16(vf, pl[t], O[t][i]);
      } else {
#pragma unroll
        for (int j = 0; j < NK; ++j)
#pragma unroll
          for (int t = 0; t < QT; ++t) O[t][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(V[j][i / 4][i & 3]), p[t][j], O[t][i], 0, 0, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    page_v = page_v_next;
    if (kb + NW * KB < end) {
      fetch_v(kb + NW * KB);
      fetch_pages(kb + 2 * NW * KB);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (!plain && __any(bad)) {                    // (rare)
      for (int key = 0; key < KB; ++key) {
        const int j = key % NK, g = key / NK;
        if (!(__ballot(bad >> j & 1) >> (16 * g) & 0xffff)) continue;
        const long long at = ((long long)__builtin_amdgcn_readlane((int)(v_here >> 32), 16 * g) << 32 | (unsigned)__builtin_amdgcn_readlane((int)v_here, 16 * g)) + j * DH;
        const T* src = (const T*)a.c.values + at + 4 * CPL * lq;
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          float pj = p[t][0];
#pragma unroll
          for (int e = 1; e < NK; ++e) pj = j == e ? p[t][e] : pj;
          pj = __shfl(pj, 16 * g + l16);
          const bool sees = __shfl((int)bits[t], 16 * g + l16) >> j & 1;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
#pragma unroll
            for (int i = 0; i < CPL; ++i) {
              float v;
              if constexpr (HALF) v = __uint_as_float((unsigned)src[CPL * r + i] << 16); else v = src[CPL * r + i];
              if (sees && !(fabsf(v) < INFINITY)) O[t][i][r] += pj * v;
            }
            asm volatile("" ::: "memory");         // (a few loads at a time: registers)
          }
        }
      }
    }
  };
  // First the blocks that every row sees and whose pages are there, up to the first that is none, then the others.
  for (; kb + KB <= sure && __all(ok(page_k)); kb += NW * KB) attend(std::true_type());
  for (; kb < end; kb += NW * KB) attend(std::false_type());

  // The waves' results, put together in pairs through LDS: every wave's in units of the largest maximum.
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    l_run[t] = quarter_sum(l_run[t]);
    if (lq == 0) { stats[w][16 * t + l16][0] = m_run[t]; stats[w][16 * t + l16][1] = l_run[t]; }
  }
  __syncthreads();
  float m_all[QT], l_all[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m_all[t] = LOW;
    for (int x = 0; x < NW; ++x) m_all[t] = fmaxf(m_all[t], stats[x][16 * t + l16][0]);
    l_all[t] = 0.f;
    for (int x = 0; x < NW; ++x) l_all[t] += stats[x][16 * t + l16][1] * rescaling(stats[x][16 * t + l16][0], m_all[t], scale.c);
    const float f = rescaling(m_run[t], m_all[t], scale.c);
#pragma unroll
    for (int i = 0; i < CPL; ++i) O[t][i] *= f;
  }
#pragma unroll
  for (int half = NW / 2; half > 0; half >>= 1) {
    if (w >= half && w < 2 * half) {
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int i = 0; i < CPL; ++i) *reinterpret_cast<f32x4*>(&merge[w - half][0][0] + (t * CPL + i) * 256 + lane * 4) = O[t][i];
    }
    __syncthreads();
    if (w < half) {
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int i = 0; i < CPL; ++i) O[t][i] += *reinterpret_cast<const f32x4*>(&merge[w][0][0] + (t * CPL + i) * 256 + lane * 4);
    }
    __syncthreads();
  }
  if (w) return;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    float x[4 * CPL];                              // columns 4 CPL lq .. of the row
    const float inv = it.parts > 1 ? 1.f : 1.f / l_all[t];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int i = 0; i < CPL; ++i) x[CPL * r + i] = l_all[t] == 0.f ? 0.f : O[t][i][r] * inv;
    if constexpr (HALF) take_infinities(a, it, kvh, k0, end, at_q[t], node[t], l_all[t], [&](int i) { return 4 * CPL * lq + i; }, x);
    if (!row_there[t]) continue;
    if (it.parts > 1) {
      const long long at = ((long long)it.sums * a.c.KVH + kvh) * QB + 16 * t + l16;
      float* dst = plan.o + at * DH + 4 * CPL * lq;
#pragma unroll
      for (int i = 0; i < 4 * CPL; i += 4) *reinterpret_cast<float4*>(dst + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
      if (lq == 0) *reinterpret_cast<float2*>(plan.ml + at * 2) = make_float2(m_all[t], l_all[t]);
    } else {
      const int g = (int)(((long long)it.block * QB + 16 * t + l16) % G);
      T* dst = (T*)a.y + at_q[t] * a.ld_y + (kvh * G + g) * DH + 4 * CPL * lq;
      if constexpr (HALF) {
#pragma unroll
        for (int i = 0; i < 4 * CPL; i += 8)
          *reinterpret_cast<uint4*>(dst + i) = make_uint4(pk_bf16(x[i], x[i + 1]), pk_bf16(x[i + 2], x[i + 3]), pk_bf16(x[i + 4], x[i + 5]), pk_bf16(x[i + 6], x[i + 7]));
      } else {
#pragma unroll
        for (int i = 0; i < 4 * CPL; i += 4) *reinterpret_cast<float4*>(dst + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
      }
    }
  }
}

// 16 bytes per lane from memory to LDS at `lds` + 16 x lane.  In asm, since the compiler waits for every such load of its builtin in front of the next read of
// LDS; the kernel's own waits count them.
__device__ __forceinline__ void piece_to_lds(u64 src, unsigned lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(src) : "memory", "m0");
}
__device__ __forceinline__ void piece_to_lds(u64 base, unsigned off, unsigned lds) {   // a scalar address and a lane's offset
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
}

// The same for many rows (bf16): the NW waves share the keys and values of the item through a ring of S stages of 32 keys in LDS and have 16 QT rows each.
// Half of the waves bring keys, half values, as whole rows of DH columns; the fragments of V^T are read with ds_read_b64_tr_b16, four keys of a column at a
// time.  The pieces of a row lie where an exclusive-or with its number puts them, so that no read meets a bank twice (SQ_LDS_BANK_CONFLICT 0).
// What bounds it: HBM up to 128 rows (4 sequences of 9000 - 40000 slots, 24 nodes x 4 heads: 493 MB in 103 us = 4.8 TB/s, and a merge of 10), above it matrix instructions next to the
// softmax's vector work at the clock that their power leaves (64 sequences of 64 - 2047 slots, 64 nodes x 4: 135 us, 1.3 us per block of 32 keys and 256 rows, of which the
// matrix instructions are 0.65 at 2.4 GHz; 60 launches in a row take 149 - 188 us each).  Measured there and dropped: a barrier for two blocks, the next block's scores under
// this one's softmax, weights of one row tile under the products of the other, wave priorities, the two waves of a SIMD half a block apart (all equal), 64 rows a
// wave (145 -> 177 us); without the low half of P 10 % faster, without memory traffic 9 %.  Eight waves with 256 rows against two blocks of 128: 150 -> 141 us.
template <int DH, int QT, int NW>
__global__ __launch_bounds__(NW * 64, 2) void k_tree_attn_shared(AttendArgs a, TreePlan plan) {
  constexpr int QB = 16 * QT * NW, KF = DH / 32, CT = DH / 16, F = 2 * CT, LPW = F / NW, S = 4, PPR = DH / 8;   // F pieces of 1 KiB a stage, LPW of them by a wave
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  __shared__ __align__(1024) u32x4 ring[S][F][64];
  TreeItem it;
  if (!find_item_of_block(a, plan, QB, it)) return;
  const int lane = threadIdx.x & 63, w = wave_index(), l16 = lane & 15, lq = lane >> 4, kvh = blockIdx.x % a.c.KVH, G = a.H / a.c.KVH;
  const int shift = a.c.shift, place_mask = (1 << shift) - 1;
  const int slots = (int)min((long long)it.len + it.n, (long long)a.c.n_table << shift);
  const int k0 = it.part * it.share * STEP, end = min(k0 + it.share * STEP, slots), sure = min(it.len, end);
  const int n_blk = max(0, (end - k0 + 31) >> 5);
  const int* __restrict__ table = a.c.table + (long long)it.b * a.c.ld_table;
  const int last = max(a.c.n_table - 1, 0);

  // Entries of the table, 64 at a time in the lanes (k0 is a multiple of 128, so that a block's never lie in two groups of 64): where a page's slots of this KV head
  // begin, in the keys or in the values as this wave brings them.
  const bool key_wave = w < NW / 2;
  const int first_piece = (key_wave ? w : w - NW / 2) * LPW;
  auto ok = [&](int page) { return (unsigned)page < (unsigned)a.c.n_page; };
  auto slots_of = [&](const void* array, int page) {   // (page 0 where the page is not there: read, not used)
    return (u64)array + (((u64)(ok(page) ? page : 0) * a.c.KVH + kvh) << shift) * (2 * DH);
  };
  int e0 = k0 >> shift, now = -1, then = -1;
  if (n_blk > 0) {                                 // (a table without columns is not read)
    now = table[min(e0 + lane, last)];
    then = table[min(e0 + 64 + lane, last)];
  }
  u64 at_now = 0, ok_now = 0, ok_before = 0;       // ok: which of these, and of the 64 before them, are pages
  // A lane's 16 bytes of each of its pieces: whole rows of DH columns, from group `lane_g` of 8 keys of the block on, and the offset if all of the block lay in
  // one page.  A row's 16-byte pieces (keys) or 32-byte ones (values) lie where an exclusive-or with its number puts them.
  auto swap_key = [&](int row) { return DH == 128 ? (row & 3) | (row >> 3 & 3) << 2 : (row >> 1 & 1) | (row >> 3 & 3) << 1; };
  auto swap_value = [&](int row) { return DH == 128 ? (row & 3) | (row >> 3 & 1) << 2 : (row >> 1 & 1) | (row >> 3 & 1) << 1; };
  int lane_g[LPW];
  unsigned lane_off[LPW];
#pragma unroll
  for (int j = 0; j < LPW; ++j) {
    const int row = (first_piece + j) * (64 / PPR) + lane / PPR;
    lane_g[j] = row >> 3;
    lane_off[j] = row * (2 * DH) + ((lane % PPR) ^ (key_wave ? swap_key(row) : swap_value(row) << 1)) * 16;
  }
  const unsigned my_ring = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)&ring[0][(key_wave ? 0 : CT) + first_piece][0];
  auto take_pages = [&]() {
    ok_now = __ballot(ok(now));
    at_now = slots_of(key_wave ? a.c.keys : a.c.values, now);
  };
  auto issue = [&](int i) {
    const int kb = k0 + 32 * min(i, n_blk - 1);
    int e = (kb >> shift) - e0;
    if (e >= 64) {
      e0 += 64;
      e -= 64;
      now = then;
      ok_before = ok_now;
      take_pages();
      then = table[min(e0 + 64 + lane, last)];
    }
    const unsigned dst = uniform(my_ring + (i % S) * (F * 1024));
    if (shift >= 5) {                              // (scalar) the block lies in one page
      const u64 base = ((u64)(unsigned)__builtin_amdgcn_readlane((int)(at_now >> 32), e) << 32 | (unsigned)__builtin_amdgcn_readlane((int)at_now, e)) +
                       (unsigned)((kb & place_mask) * (2 * DH));
#pragma unroll
      for (int j = 0; j < LPW; ++j) piece_to_lds(base, lane_off[j], dst + j * 1024);
    } else {
#pragma unroll
      for (int j = 0; j < LPW; ++j) {
        const int s = kb + 8 * lane_g[j], from = (s >> shift) - e0;
        const u64 page_at = (u64)(unsigned)__shfl((int)(at_now >> 32), from) << 32 | (unsigned)__shfl((int)at_now, from);
        piece_to_lds(page_at + (s & place_mask) * (2 * DH) + lane_off[j] - lane_g[j] * (16 * DH), dst + j * 1024);
      }
    }
  };
  // this lane's rows
  long long at_q[QT];
  int node[QT];
  bool row_there[QT];
  u64 first_word[QT];
  u32x4 q[QT][KF];
  const Base2 scale = a.scale;
  const unsigned flip = scale.flip ? 0x80008000u : 0u;
  const long long r0 = (long long)it.block * QB + 16 * QT * w;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const long long i = r0 + 16 * t + l16;
    row_there[t] = i < (long long)it.n * G;
    const int g = (int)(i % G);
    node[t] = row_there[t] ? (int)(i / G) : 0;
    at_q[t] = (long long)(it.f0 + node[t]);
    first_word[t] = a.visible ? a.visible[at_q[t] * a.n_words] : 0;
    const bf16_t* src = (const bf16_t*)a.q + at_q[t] * a.ld_q + ((row_there[t] ? g : 0) + kvh * G) * DH;
#pragma unroll
    for (int f = 0; f < KF; ++f) {
      q[t][f] = *reinterpret_cast<const u32x4*>(src + f * 32 + lq * 8);
    }
  }
  take_pages();
  if (n_blk > 0) {
#pragma unroll
    for (int i = 0; i < S - 1; ++i) issue(i);
  }

#pragma unroll
  for (int t = 0; t < QT; ++t)
#pragma unroll
    for (int f = 0; f < KF; ++f) q[t][f] = row_there[t] ? q[t][f] ^ flip : (u32x4){0, 0, 0, 0};
  // the slots that some row of this wave sees end here: none, a chain's last node, all
  const long long rows_left = (long long)it.n * G - r0;
  const int reach = rows_left <= 0 ? 0 : a.visible ? end : (int)min((long long)end, it.len + (r0 + min(rows_left, 16ll * QT) - 1) / G + 1);

  f32x4 O[QT][CT];
  float m_run[QT], l_run[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m_run[t] = LOW; l_run[t] = 0.f;
#pragma unroll
    for (int i = 0; i < CT; ++i) O[t][i] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }
  // Where this lane's fragments begin in a stage: its 8 columns of key 8 (l16 / 4) + l16 % 4 of tile 0 (4 keys on: tile 1), and its first column of V^T, 4
  // keys of tile 0, 8 lq + l16 / 4 (4 on: the others).  The pieces of the others are an exclusive-or away.
  const int k_row = 8 * (l16 >> 2) + (l16 & 3), v_row = 8 * lq + (l16 >> 2);
  const unsigned k_off = k_row * (2 * DH) + ((lq ^ swap_key(k_row)) << 4);
  const unsigned v_off = CT * 1024 + v_row * (2 * DH) + (swap_value(v_row) << 5) + (l16 & 3) * 8;
  // One block of 32 keys.  plain: every key is there and seen by every row.
  auto attend = [&](auto is_plain, int kb, const uint4 (&K)[2 * KF], const u32x4(*blk)[64], unsigned pages) __attribute__((always_inline)) {
    constexpr bool plain = decltype(is_plain)::value;
    f32x4 sc[QT][2];
#pragma unroll
    for (int t = 0; t < QT; ++t) sc[t][0] = sc[t][1] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int f = 0; f < KF; ++f)
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        sc[t][0] = mfma_bf16(K[f], __builtin_bit_cast(uint4, q[t][f]), sc[t][0]);
        sc[t][1] = mfma_bf16(K[KF + f], __builtin_bit_cast(uint4, q[t][f]), sc[t][1]);
      }
    uint4 V[CT];
    const unsigned v_at = (unsigned)(uintptr_t)(__attribute__((address_space(3))) const void*)blk + v_off;
#pragma unroll
    for (int x = 0; x < CT; ++x) {
      typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(v_at ^ (x << 5)));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)((v_at ^ (x << 5)) + 8 * DH));
      const uint2 l2 = __builtin_bit_cast(uint2, lo), h2 = __builtin_bit_cast(uint2, hi);
      V[x] = make_uint4(l2.x, l2.y, h2.x, h2.y);
    }
    const int kl = kb + 8 * lq;
    float p[QT][8];
    unsigned bits[QT];
    unsigned there = 0xff;
    if (!plain) there = pages >> ((kl >> shift) - (kb >> shift)) & 1 ? (1u << min(max(end - kl, 0), 8)) - 1 : 0u;
    uint4 ph[QT], pl[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
#pragma unroll
      for (int e = 0; e < 8; ++e) p[t][e] = sc[t][e >> 2][e & 3];
      bits[t] = plain ? there : seen_keys<8>(a, first_word[t], at_q[t], node[t], kl - it.len, there);
      softmax_step(p[t], !plain, bits[t], scale, m_run[t], l_run[t], O[t]);
      split2(p[t][0], p[t][1], ph[t].x, pl[t].x);
      split2(p[t][2], p[t][3], ph[t].y, pl[t].y);
      split2(p[t][4], p[t][5], ph[t].z, pl[t].z);
      split2(p[t][6], p[t][7], ph[t].w, pl[t].w);
    }
    unsigned bad = 0;                              // which of this lane's keys have an element that is not finite here
    if constexpr (!plain) {                        // (as above; a lane has one column of its 8 keys in each tile)
      if (__any(there != 0xff)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const unsigned keep = (there >> (2 * e) & 1 ? 0xffffu : 0u) | (there >> (2 * e + 1) & 1 ? 0xffff0000u : 0u);
#pragma unroll
          for (int x = 0; x < CT; ++x) reinterpret_cast<unsigned*>(&V[x])[e] &= keep;
        }
      }
      if (kb + 32 > it.len) {
        u16x2 top = {0, 0};                        // the largest magnitudes, as integers: 0x7f80 and more are not finite
#pragma unroll
        for (int x = 0; x < CT; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, reinterpret_cast<const unsigned*>(&V[x])[e] & 0x7fff7fffu));
        if (__any(top[0] >= 0x7f80 || top[1] >= 0x7f80)) {
#pragma unroll
          for (int x = 0; x < CT; ++x) {
            unsigned* v = reinterpret_cast<unsigned*>(&V[x]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const bool lo = kl + 2 * e >= it.len && (v[e] & 0x7f80u) == 0x7f80u, hi = kl + 2 * e + 1 >= it.len && (v[e] & 0x7f800000u) == 0x7f800000u;
              bad |= (lo ? 1u : 0u) << (2 * e) | (hi ? 2u : 0u) << (2 * e);
              v[e] &= (lo ? 0xffff0000u : 0xffffffffu) & (hi ? 0x0000ffffu : 0xffffffffu);
            }
          }
        }
      }
    }
#pragma unroll
    for (int x = 0; x < CT; ++x) {
#pragma unroll
      for (int t = 0; t < QT; ++t) O[t][x] = mfma_bf16(V[x], ph[t], O[t][x]);
#pragma unroll
      for (int t = 0; t < QT; ++t) O[t][x] = mfma_bf16(V[x], pl[t], O[t][x]);
    }
    if (!plain && __any(bad)) {                    // (rare)
      for (int key = 0; key < 32; ++key) {
        const int j = key & 7, g = key >> 3;
        if (!(__ballot(bad >> j & 1) >> (16 * g) & 0xffff)) continue;
        const int s = kb + key;
        const bf16_t* src = (const bf16_t*)slots_of(a.c.values, table[min(s >> shift, last)]) + (s & place_mask) * DH + 4 * lq;
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          float pj = p[t][0];
#pragma unroll
          for (int e = 1; e < 8; ++e) pj = j == e ? p[t][e] : pj;
          pj = __shfl(pj, 16 * g + l16);
          const bool sees = __shfl((int)bits[t], 16 * g + l16) >> j & 1;
#pragma unroll
          for (int x = 0; x < CT; ++x) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float v = __uint_as_float((unsigned)src[16 * x + r] << 16);
              if (sees && !(fabsf(v) < INFINITY)) O[t][x][r] += pj * v;
            }
            asm volatile("" ::: "memory");         // (one tile's loads at a time: registers)
          }
        }
      }
    }
  };
  auto landed = [&]() {   // this wave's part of the next block has, its reads of the last one are back; then the same of every wave
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((S - 2) * LPW) : "memory");
  };
  auto block = [&](auto is_plain, int i, unsigned pages) __attribute__((always_inline)) {
    const int kb = k0 + i * 32;
    const u32x4(*blk)[64] = ring[i % S];
    if (kb < reach) {                              // (scalar) something that a row of this wave sees
      uint4 K[2 * KF];
#pragma unroll
      for (int f = 0; f < KF; ++f) {
        typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;
        const unsigned at = (unsigned)(uintptr_t)(__attribute__((address_space(3))) const void*)blk + (k_off ^ (f << 6));
        K[f] = __builtin_bit_cast(uint4, *(lds_u32x4*)(uintptr_t)at);
        K[KF + f] = __builtin_bit_cast(uint4, *(lds_u32x4*)(uintptr_t)(at + 8 * DH));
      }
      issue(i + S - 1);                            // (next to the keys' way out of LDS)
      attend(is_plain, kb, K, blk, pages);
    } else {
      issue(i + S - 1);
    }
  };
  auto pages_of = [&](int i) {                     // (the registers may be a few blocks ahead)
    const int entry = ((k0 + i * 32) >> shift) - e0;
    return (unsigned)(entry < 0 ? ok_before >> (entry + 64) : ok_now >> entry);
  };
  // First the blocks that every row sees and whose pages are there, up to the first that is none, then the others.
  int i = 0;
  if (n_blk > 0) landed();
  for (; i < n_blk; ++i, landed()) {
    const int kb = k0 + i * 32;
    const unsigned all = (2u << (((kb + 31) >> shift) - (kb >> shift))) - 1;
    if (kb + 32 > sure || (pages_of(i) & all) != all) break;
    block(std::true_type(), i, all);
  }
  for (; i < n_blk; ++i, landed()) block(std::false_type(), i, pages_of(i));
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (the last stages' loads still write to LDS)
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const float l = quarter_sum(l_run[t]), inv = it.parts > 1 ? 1.f : 1.f / l;
    float y[4 * CT];                               // columns 16 x + 4 lq .. of the row
#pragma unroll
    for (int x = 0; x < CT; ++x)
#pragma unroll
      for (int r = 0; r < 4; ++r) y[4 * x + r] = l == 0.f ? 0.f : O[t][x][r] * inv;
    take_infinities(a, it, kvh, k0, end, at_q[t], node[t], l, [&](int i) { return 16 * (i >> 2) + 4 * lq + (i & 3); }, y);
    if (!row_there[t]) continue;
    const int i = (int)(16 * QT * w + 16 * t + l16);
    if (it.parts > 1) {
      const long long at = ((long long)it.sums * a.c.KVH + kvh) * QB + i;
#pragma unroll
      for (int x = 0; x < CT; ++x) *reinterpret_cast<float4*>(plan.o + at * DH + 16 * x + 4 * lq) = make_float4(y[4 * x], y[4 * x + 1], y[4 * x + 2], y[4 * x + 3]);
      if (lq == 0) *reinterpret_cast<float2*>(plan.ml + at * 2) = make_float2(m_run[t], l);
    } else {
      const int g = (int)((r0 + 16 * t + l16) % G);
      bf16_t* dst = (bf16_t*)a.y + at_q[t] * a.ld_y + (kvh * G + g) * DH + 4 * lq;
#pragma unroll
      for (int x = 0; x < CT; ++x) *reinterpret_cast<uint2*>(dst + 16 * x) = make_uint2(pk_bf16(y[4 * x], y[4 * x + 1]), pk_bf16(y[4 * x + 2], y[4 * x + 3]));
    }
  }
}

// The shares of split sequences put together, in their order: the workgroups of a block's shares take its rows in turn, a wave one at a time.
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_tree_merge(AttendArgs a, TreePlan plan, int QB) {
  constexpr int N = DH / 64;
  const int item = blockIdx.x / a.c.KVH;
  const TreeItem it = plan.list[item];
  if (it.parts < 2) return;
  const float c = a.scale.c;
  const int G = a.H / a.c.KVH, kvh = blockIdx.x - item * a.c.KVH, lane = threadIdx.x & 63, first = it.sums - it.part, parts = min(it.parts, plan.items - (item - it.part));
  const int rows = (int)min((long long)QB, (long long)it.n * G - (long long)it.block * QB);
  for (int r = it.part + it.parts * wave_index(); r < rows; r += it.parts * 4) {
    auto at = [&](int part) { return ((long long)(first + part) * a.c.KVH + kvh) * QB + r; };
    float2 ml = lane < parts ? *reinterpret_cast<const float2*>(plan.ml + at(lane) * 2) : make_float2(LOW, 0.f);
    constexpr int U = 16;                          // shares whose loads leave together, the first of them with their statistics'
    float v[U][N];
    auto fetch = [&](int x) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < N; ++e) v[u][e] = plan.o[at(min(x + u, parts - 1)) * DH + lane * N + e];
    };
    fetch(0);
    float m = ml.x, l = 0.f, o[N] = {};
    for (int x = lane + 64; x < parts; x += 64) m = fmaxf(m, plan.ml[at(x) * 2]);
    m = wave_max(m);
    for (int x0 = 0; x0 < parts; x0 += 64) {
      if (x0) ml = x0 + lane < parts ? *reinterpret_cast<const float2*>(plan.ml + at(x0 + lane) * 2) : make_float2(LOW, 0.f);
      const float f = x0 + lane < parts ? rescaling(ml.x, m, c) : 0.f;
      l += wave_sum(ml.y * f);
      for (int x = x0; x < min(parts, x0 + 64); x += U) {
        if (x) fetch(x);
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (x + u < parts)                       // (scalar)
#pragma unroll
            for (int e = 0; e < N; ++e) o[e] += v[u][e] * __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), (x + u) & 63));
      }
    }
    const long long i = (long long)it.block * QB + r;
    T* y = (T*)a.y + (it.f0 + i / G) * a.ld_y + (kvh * G + i % G) * DH + lane * N;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float v = l == 0.f ? 0.f : o[e] / l;
      if constexpr (sizeof(T) == 4) y[e] = v; else y[e] = f2bf(v);
    }
  }
}

// How the rows of an item are laid out: QT tiles of 16 rows a wave; NW waves that share the keys, or (1) waves that have the rows each and share the
// keys among them.  By the mean of rows (nodes x heads of a KV head) per sequence.
struct TreeShape { int QT, NW, QB; };
static TreeShape tree_shape(int type, int dh, int H, int KVH, int n_seq, int T) {
  const double rows = (double)T * (H / KVH) / std::max(1, std::min(n_seq, T));
  auto of = [](int QT, int NW) { return TreeShape{QT, NW, 16 * QT * NW}; };
  if (rows <= 16 || (type == X_F32 && dh == 128)) return of(1, 1);
  if (rows <= 32 || type == X_F32) return of(2, 1);
  return rows <= 64 ? of(1, 4) : rows <= 128 ? of(2, 4) : of(2, 8);
}

// Splitting a sequence's slots over workgroups costs the merge, its launch and the sums on their way (10 us to 5.7 where it is not needed at all), and is decided
// by what the table could hold, since only the device knows the lengths.  Measured, split / whole, us: 1 x 8 pairs of sequence and KV head, 250 slots 10.4 / 7.9, 500 10.4 / 10.2,
// 1000 10.2 / 15.1; 16 x 25 of 400 16.0 / 11.7; 16 x 8 pairs of 50 - 990 slots, 24 nodes 43.0 / 37.3, 64 nodes of 950 84 / 55, 10 nodes 28 / 31; 64 x 8 pairs of up to
// 2040 slots, 1 node 68 / 61, 9 89 / 77, 30 125 / 92; float32, 160 pairs of up to 1000 17.3 / 22.0, 24 of 132 10.5 / 7.5.
static bool tree_whole(int type, int KVH, int n_seq, int T, long long slots) {
  const long long pairs = (long long)std::min(n_seq, T) * KVH;
  const int steps = pairs >= 512 ? 17 : pairs >= 128 ? 8 : 4;
  return slots <= (long long)(type == X_F32 ? steps / 2 : steps) * STEP;
}

static TreePlan tree_plan(const TreeShape& shape, int type, int dh, int H, int KVH, int n_seq, int T, long long slots, size_t& bytes, void* ws) {
  TreePlan p{};
  p.target = tree_target(KVH, shape.NW == 8 ? 256 : 512);
  const bool whole = tree_whole(type, KVH, n_seq, T, slots);
  p.items = (int)most_items(most_blocks((long long)T * (H / KVH), shape.QB, std::min(n_seq, T)), !whole, p.target);
  p.split = !whole;
  p.sort = n_seq > 1 && n_seq <= 64 && (long long)p.items * KVH > 512;
  p.planned = n_seq > 128;
  const size_t rows = (size_t)most_sums(p.items, p.split, p.target) * KVH * shape.QB;
  bytes = rows * (dh + 2) * sizeof(float) + (whole && !p.planned ? 0 : p.items * sizeof(TreeItem));
  p.o = (float*)ws;
  p.ml = p.o + rows * dh;
  p.list = (TreeItem*)(p.ml + rows * 2);
  return p;
}

size_t attend_workspace(int type, int dh, int H, int KVH, int n_seq, int T, long long slots) {
  size_t bytes;
  if (n_seq < 1 || T < 1) return 0;
  tree_plan(tree_shape(type, dh, H, KVH, n_seq, T), type, dh, H, KVH, n_seq, T, slots, bytes, nullptr);
  return bytes;
}

Base2 base2(float scale) {
  const float c = fabsf(scale) * 1.4426950408889634f;
  return Base2{c, 8.f / c, scale < 0.f};           // (a scale of 0: the maximum never moves)
}

void launch_cache_attend(const AttendArgs& a, void* workspace, hipStream_t s) {
  size_t bytes;
  const TreeShape shape = tree_shape(a.type, a.c.dh, a.H, a.c.KVH, a.c.n_seq, a.T);
  const TreePlan p = tree_plan(shape, a.type, a.c.dh, a.H, a.c.KVH, a.c.n_seq, a.T, (long long)a.c.n_table << a.c.shift, bytes, workspace);
  const dim3 grid(a.c.KVH * p.items), block(256);
  if (p.planned) hipLaunchKernelGGL(k_tree_plan, dim3(1), dim3(1024), 0, s, a, p, shape.QB);
  auto go = [&](auto type, auto dh) {
    using T = decltype(type);
    constexpr int DH = decltype(dh)::value;
    if (shape.NW == 1 && shape.QT == 1) hipLaunchKernelGGL((k_tree_attn<T, DH, 1, 4>), grid, block, 0, s, a, p);
    if constexpr (sizeof(T) == 2 || DH == 64)
      if (shape.NW == 1 && shape.QT == 2) hipLaunchKernelGGL((k_tree_attn<T, DH, 2, 4>), grid, block, 0, s, a, p);
    if constexpr (sizeof(T) == 2) {
      if (shape.NW == 4 && shape.QT == 1) hipLaunchKernelGGL((k_tree_attn_shared<DH, 1, 4>), grid, block, 0, s, a, p);
      else if (shape.NW == 4) hipLaunchKernelGGL((k_tree_attn_shared<DH, 2, 4>), grid, block, 0, s, a, p);
      else if (shape.NW == 8) hipLaunchKernelGGL((k_tree_attn_shared<DH, 2, 8>), grid, dim3(512), 0, s, a, p);
    }
    if (p.split) hipLaunchKernelGGL((k_tree_merge<T, DH>), grid, block, 0, s, a, p, shape.QB);
  };
  auto typed = [&](auto dh) { if (a.type == X_F32) go(float(), dh); else go(bf16_t(), dh); };
  if (a.c.dh == 64) typed(std::integral_constant<int, 64>()); else typed(std::integral_constant<int, 128>());
}

}  // namespace sprinter
