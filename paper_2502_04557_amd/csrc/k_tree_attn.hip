// HIP kernels of the attention of trees of drafted tokens over a cache in pages, for gfx950.
#include "ops.h"
#include "dev.h"
#include <algorithm>
#include <type_traits>

namespace sprinter {

// A launch cuts the batch into items: a block of QB rows (node x head of one KV head) of a sequence against a share of its slots.  Lengths and trees are known
// on the device alone, so every workgroup works the cut out for itself from `lens` and `first`: `steps` of STEP slots over all blocks of rows,
// dealt out in shares of `share` steps so that about `target` items come out, however ragged the batch is.
struct TreePlan {
  int target, items;                               // shares to aim for; the most items there can be (per KV head)
  float* o;                                        // [items][KVH][QB][DH] sums of split sequences, not divided, and
  float* ml;                                       // [items][KVH][QB][2] their maxima (base-2 units) and sums of weights
};
constexpr int STEP = 128;

struct TreeItem {
  int b, f0, n, len, block, part, parts, share, base;   // rows f0 .. f0 + n - 1; block of rows, share of slots; base: the block's first item
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

// The item of index `item`, or (row >= 0) the first item of the block that holds this row's first head; false: there is none.  By a whole wave.
__device__ __forceinline__ bool find_item(const AttendArgs& a, const TreePlan& p, int QB, int item, int row, TreeItem& out) {
  const int lane = threadIdx.x & 63, n = a.c.n_seq;
  TreeSeq s = tree_seq(a, lane, QB, lane < n);
  float work = (float)s.blocks * (float)s.steps;
  for (int b = lane + 64; b < n; b += 64) {
    const TreeSeq x = tree_seq(a, b, QB, true);
    work += (float)x.blocks * (float)x.steps;
  }
  work = wave_sum(work);
  // (a little more than the quotient, so that the roundings of the sum cannot make more items than there is room for)
  const int share = (int)(work * (1.0001f / (float)p.target)) + 1;
  int base = 0;
  for (int b0 = 0; b0 < n; b0 += 64) {
    if (b0) s = tree_seq(a, b0 + lane, QB, b0 + lane < n);
    const int parts = (s.steps + share - 1) / share, mine = s.blocks * parts;
    int sum = mine;                                // items up to this sequence, itself among them
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(sum, o);
      if (lane >= o) sum += x;
    }
    const int before = base + sum - mine;
    const u64 hit = __ballot(row >= 0 ? s.blocks > 0 && row >= s.f0 && row < s.f0 + s.n : item >= before && item < before + mine);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      out.b = uniform(b0 + l);
      out.f0 = __builtin_amdgcn_readlane(s.f0, l);
      out.n = __builtin_amdgcn_readlane(s.n, l);
      out.len = __builtin_amdgcn_readlane(s.len, l);
      out.parts = __builtin_amdgcn_readlane(parts, l);
      out.share = uniform(share);
      const int first = __builtin_amdgcn_readlane(before, l);
      if (row >= 0) {
        out.block = 0; out.part = 0; out.base = first;
      } else {
        const int i = item - first;
        out.block = i / out.parts;
        out.part = i - out.block * out.parts;
        out.base = item - out.part;
      }
      return true;
    }
    base += __builtin_amdgcn_readlane(sum, 63);
  }
  return false;
}

// bf16: 32 keys a block, of which a lane ends up with the scores of 8; float32: 16 and 4.
template <typename T> struct Tree {};
template <> struct Tree<bf16_t> { static constexpr int KB = 32, NK = 8, VEC = 8; };
template <> struct Tree<float> { static constexpr int KB = 16, NK = 4, VEC = 4; };

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float quarters_max(float v) {   // over the lanes l, l + 16, l + 32, l + 48
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float quarters_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// The attention of one item by NW waves, each with all QB = 16 QT rows and every NW-th block of the item's keys; one pass with running maxima and sums.
//   S^T = K Q^T: a lane holds the scores of one row (lane % 16).  bf16: row i of key tile t is key 8 (i / 4) + 4 t + i % 4, so that a lane's 8 scores are
//     those of the keys 8 (lane / 16) .. + 7, the operand layout of P.  float32: the 4 keys 4 (lane / 16) + r, one for each of four products.
//   O^T += V^T P^T: a lane fetches DH / 16 neighbouring columns of each of its keys, whole rows by 16 lanes; operand c takes column c of each
//     lane's, which for bf16 is one byte permutation per pair of keys.  The accumulators then hold DH / 4 neighbouring columns of a row.
// P enters as two bf16 (16 bits, as the values of the plain bfloat16 path deserve: one alone would double the error of the result).
template <typename T, int DH, int QT, int NW>
__global__ __launch_bounds__(NW * 64, QT == 4 ? 1 : 2) void k_tree_attn(AttendArgs a, TreePlan plan) {
  using P = Tree<T>;
  constexpr bool HALF = sizeof(T) == 2;
  constexpr int KB = P::KB, NK = P::NK, QB = 16 * QT, CPL = DH / 16, KF = DH / (HALF ? 32 : 16);   // columns of V per lane; 16-byte pieces of a key per lane and tile
  constexpr int KT = HALF ? 2 : 1;                 // key tiles
  constexpr int VW = CPL * sizeof(T) / 4;          // dwords of a key's columns
  constexpr float LOW = -3.402823466e38f;
  __shared__ float merge[NW / 2][QB][DH];
  __shared__ float stats[NW][QB][2];
  TreeItem it;
  if (!find_item(a, plan, QB, blockIdx.x, -1, it)) return;
  const int lane = threadIdx.x & 63, w = wave_index(), l16 = lane & 15, lq = lane >> 4, kvh = blockIdx.y, G = a.H / a.c.KVH;
  const int shift = a.c.shift, place_mask = (1 << shift) - 1;
  const int slots = (int)min((long long)it.len + it.n, (long long)a.c.n_table << shift);
  const int k0 = it.part * it.share * STEP, end = min(k0 + it.share * STEP, slots), sure = min(it.len, end);   // slots below `sure` are seen by every row
  const int* __restrict__ table = a.c.table + (long long)it.b * a.c.ld_table;

  // this lane's rows
  long long at_q[QT];
  int node[QT];
  bool row_there[QT];
  u32x4 q[QT][KF];
  float c = a.scale * 1.4426950408889634f;
  const unsigned flip = c < 0.f ? (HALF ? 0x80008000u : 0x80000000u) : 0u;   // (a negative scale: the queries change their sign)
  c = fabsf(c);
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const long long i = (long long)it.block * QB + 16 * t + l16;
    row_there[t] = i < (long long)it.n * G;
    const int g = (int)(i % G);
    node[t] = row_there[t] ? (int)(i / G) : 0;
    at_q[t] = (long long)(it.f0 + node[t]);
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
  float m_run[QT], l_run[QT];                      // maximum (base-2 units) and this lane's sum of weights
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
  for (; kb < end; kb += NW * KB) {
    const bool plain = kb + KB <= sure && __all(ok(page_k));   // (uniform) every key is there and seen by every row
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
#pragma unroll
    for (int t = 0; t < QT; ++t) {
#pragma unroll
      for (int e = 0; e < NK; ++e) p[t][e] = sc[t][e >> 2][e & 3];
      bits[t] = (1u << NK) - 1;
    }
    const int kl = kb + NK * lq;                   // this lane's first key
    unsigned there = (1u << NK) - 1;
    if (!plain) {
      there = v_ok ? (1u << min(max(end - kl, 0), NK)) - 1 : 0u;
      const int j0 = kl - it.len;                  // as a node
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        unsigned see = (1u << NK) - 1;
        if (j0 + NK > 0) {
          if (a.visible) {
            const int j = max(j0, 0), word = j >> 6, sh = j & 63;
            const unsigned long long* v = a.visible + at_q[t] * a.n_words;
            see = word < a.n_words ? (unsigned)(v[word] >> sh) : 0u;
            if (sh > 64 - NK && word + 1 < a.n_words) see |= (unsigned)(v[word + 1] << (64 - sh));
            if (j0 < 0) see = see << -j0 | ((1u << -j0) - 1);
          } else {
            see = (1u << min(max(node[t] - j0 + 1, 0), NK)) - 1;
          }
        }
        bits[t] = see & there;
#pragma unroll
        for (int e = 0; e < NK; ++e) p[t][e] = bits[t] >> e & 1 ? p[t][e] : -INFINITY;
      }
    }
    uint4 ph[QT], pl[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float mx = p[t][0];
#pragma unroll
      for (int e = 1; e < NK; ++e) mx = fmaxf(mx, p[t][e]);
      const float mn = fmaxf(m_run[t], fmaxf(quarters_max(mx) * c, LOW));
      if (__any(mn > m_run[t])) {                  // (uniform) the maximum of some row moves
        const float corr = __builtin_amdgcn_exp2f(m_run[t] - mn);
        l_run[t] *= corr;
#pragma unroll
        for (int i = 0; i < CPL; ++i) O[t][i] *= corr;
        m_run[t] = mn;
      }
#pragma unroll
      for (int e = 0; e < NK; ++e) p[t][e] = __builtin_amdgcn_exp2f(fmaf(p[t][e], c, -mn));
      if (!plain) {                                // (also where -infinity times a scale of 0 is NaN)
#pragma unroll
        for (int e = 0; e < NK; ++e) p[t][e] = bits[t] >> e & 1 ? p[t][e] : 0.f;
      }
      if constexpr (HALF) {
        l_run[t] += ((p[t][0] + p[t][1]) + (p[t][2] + p[t][3])) + ((p[t][4] + p[t][5]) + (p[t][6] + p[t][7]));
        split2(p[t][0], p[t][1], ph[t].x, pl[t].x);
        split2(p[t][2], p[t][3], ph[t].y, pl[t].y);
        split2(p[t][4], p[t][5], ph[t].z, pl[t].z);
        split2(p[t][6], p[t][7], ph[t].w, pl[t].w);
      } else {
        l_run[t] += (p[t][0] + p[t][1]) + (p[t][2] + p[t][3]);
      }
    }
    // What no row, or not every row, sees must not meet a weight of 0 as an infinity or NaN: slots that are not there are cleared, and elements of nodes
    // that are not finite are taken out here and added below to the rows that see them.
    u64 sick[NK];
    bool any_sick = false;
    if (!plain) {
#pragma unroll
      for (int j = 0; j < NK; ++j) {
        bool bad = false;
#pragma unroll
        for (int i = 0; i < VW; ++i) {
          unsigned x = V[j][i / 4][i & 3];
          x = there >> j & 1 ? x : 0u;
          if (kl + j >= it.len) {
            if constexpr (HALF) {
              const bool lo = (x & 0x7f80u) == 0x7f80u, hi = (x & 0x7f800000u) == 0x7f800000u;
              bad |= lo || hi;
              x &= (lo ? 0xffff0000u : 0xffffffffu) & (hi ? 0x0000ffffu : 0xffffffffu);
            } else {
              const bool b = (x & 0x7f800000u) == 0x7f800000u;
              bad |= b;
              x = b ? 0u : x;
            }
          }
          V[j][i / 4][i & 3] = x;
        }
        sick[j] = __ballot(bad);
        any_sick |= sick[j] != 0;
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
    if (any_sick) {                                // (uniform, rare)
#pragma unroll
      for (int j = 0; j < NK; ++j)
        for (int g = 0; g < 4; ++g) {
          if (!(sick[j] >> (16 * g) & 0xffff)) continue;
          const long long at = ((long long)__builtin_amdgcn_readlane((int)(v_here >> 32), 16 * g) << 32 | (unsigned)__builtin_amdgcn_readlane((int)v_here, 16 * g)) + j * DH;
          const T* src = (const T*)a.c.values + at + 4 * CPL * lq;
#pragma unroll
          for (int t = 0; t < QT; ++t) {
            const float pj = __shfl(p[t][j], 16 * g + l16);
            const bool sees = __shfl((int)bits[t], 16 * g + l16) >> j & 1;
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
              for (int i = 0; i < CPL; ++i) {
                float v;
                if constexpr (HALF) v = __uint_as_float((unsigned)src[CPL * r + i] << 16); else v = src[CPL * r + i];
                if (sees && !(fabsf(v) < INFINITY)) O[t][i][r] += pj * v;
              }
          }
        }
    }
  }

  // The waves' results, put together in pairs through LDS: every wave's in units of the largest maximum.
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    l_run[t] = quarters_sum(l_run[t]);
    if (lq == 0) { stats[w][16 * t + l16][0] = m_run[t]; stats[w][16 * t + l16][1] = l_run[t]; }
  }
  __syncthreads();
  float m_all[QT], l_all[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m_all[t] = LOW;
    for (int x = 0; x < NW; ++x) m_all[t] = fmaxf(m_all[t], stats[x][16 * t + l16][0]);
    l_all[t] = 0.f;
    for (int x = 0; x < NW; ++x) l_all[t] += stats[x][16 * t + l16][1] * __builtin_amdgcn_exp2f(stats[x][16 * t + l16][0] - m_all[t]);
    const float f = __builtin_amdgcn_exp2f(m_run[t] - m_all[t]);
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
    if (!row_there[t]) continue;
    float x[4 * CPL];                              // columns 4 CPL lq .. of the row
    const float inv = it.parts > 1 ? 1.f : l_all[t] == 0.f ? 0.f : 1.f / l_all[t];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int i = 0; i < CPL; ++i) x[CPL * r + i] = l_all[t] == 0.f ? 0.f : O[t][i][r] * inv;
    if (it.parts > 1) {
      const long long at = (((long long)blockIdx.x * a.c.KVH + kvh) * QB + 16 * t + l16);
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

// The shares of a split sequence put together: a wave per row and head, the shares in their order.
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_tree_merge(AttendArgs a, TreePlan plan, int QB) {
  const int t = blockIdx.x, h = blockIdx.y * 4 + wave_index(), lane = threadIdx.x & 63;
  TreeItem it;
  if (h >= a.H || !find_item(a, plan, QB, 0, t, it) || it.parts < 2) return;
  const int G = a.H / a.c.KVH, kvh = h / G;
  const long long i = (long long)(t - it.f0) * G + h % G;
  const int block = (int)(i / QB), row = (int)(i % QB), item = it.base + block * it.parts;
  auto at = [&](int part) { return ((long long)(item + part) * a.c.KVH + kvh) * QB + row; };
  float m = -3.402823466e38f, l = 0.f;
  for (int x = lane; x < it.parts; x += 64) m = fmaxf(m, plan.ml[at(x) * 2]);
  m = wave_max(m);
  float o[DH / 64] = {};
  for (int x = 0; x < it.parts; ++x) {
    const float2 ml = *reinterpret_cast<const float2*>(plan.ml + at(x) * 2);
    const float f = __builtin_amdgcn_exp2f(ml.x - m);
    l += ml.y * f;
#pragma unroll
    for (int e = 0; e < DH / 64; ++e) o[e] += plan.o[at(x) * DH + lane * (DH / 64) + e] * f;
  }
  T* y = (T*)a.y + (long long)t * a.ld_y + h * DH + lane * (DH / 64);
#pragma unroll
  for (int e = 0; e < DH / 64; ++e) {
    const float r = l == 0.f ? 0.f : o[e] / l;
    if constexpr (sizeof(T) == 4) y[e] = r; else y[e] = f2bf(r);
  }
}

// Row tiles of a wave: as many as the rows of a sequence fill in the mean.
static int tree_tiles(int type, int H, int KVH, int n_seq, int T) {
  const double rows = (double)T * (H / KVH) / std::max(1, std::min(n_seq, T));
  return rows <= 16 ? 1 : rows <= 32 || type == X_F32 ? 2 : 4;
}

static TreePlan tree_plan(int type, int dh, int H, int KVH, int n_seq, int T, long long slots, size_t& bytes, void* ws) {
  const int QB = 16 * tree_tiles(type, H, KVH, n_seq, T);
  TreePlan p{};
  p.target = std::max(1, (512 + KVH - 1) / KVH);
  const long long blocks = (long long)T * (H / KVH) / QB + std::min(n_seq, T);   // at most
  const bool whole = slots <= STEP;                // one share each
  p.items = (int)(blocks + (whole ? 0 : p.target));
  bytes = 0;
  if (!whole) {
    const size_t rows = (size_t)p.items * KVH * QB;
    bytes = rows * (dh + 2) * sizeof(float);
    p.o = (float*)ws;
    p.ml = (float*)ws + rows * dh;
  }
  return p;
}

size_t attend_workspace(int type, int dh, int H, int KVH, int n_seq, int T, long long slots) {
  size_t bytes;
  if (n_seq < 1 || T < 1) return 0;
  tree_plan(type, dh, H, KVH, n_seq, T, slots, bytes, nullptr);
  return bytes;
}

void launch_cache_attend(const AttendArgs& a, void* workspace, hipStream_t s) {
  size_t bytes;
  const TreePlan p = tree_plan(a.type, a.c.dh, a.H, a.c.KVH, a.c.n_seq, a.T, (long long)a.c.n_table << a.c.shift, bytes, workspace);
  const int QT = tree_tiles(a.type, a.H, a.c.KVH, a.c.n_seq, a.T);
  const dim3 grid(p.items, a.c.KVH), block(256);
  auto go = [&](auto type, auto dh) {
    using T = decltype(type);
    constexpr int DH = decltype(dh)::value;
    if (QT == 1) hipLaunchKernelGGL((k_tree_attn<T, DH, 1, 4>), grid, block, 0, s, a, p);
    else if (QT == 2) hipLaunchKernelGGL((k_tree_attn<T, DH, 2, 4>), grid, block, 0, s, a, p);
    else if constexpr (sizeof(T) == 2) hipLaunchKernelGGL((k_tree_attn<T, DH, 4, 4>), grid, block, 0, s, a, p);
    if (bytes) hipLaunchKernelGGL((k_tree_merge<T, DH>), dim3(a.T, (a.H + 3) / 4), block, 0, s, a, p, 16 * QT);
  };
  auto typed = [&](auto dh) { if (a.type == X_F32) go(float(), dh); else go(bf16_t(), dh); };
  if (a.c.dh == 64) typed(std::integral_constant<int, 64>()); else typed(std::integral_constant<int, 128>());
}

}  // namespace sprinter
