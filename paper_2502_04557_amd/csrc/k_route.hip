// HIP kernel of routing to experts for gfx950: scores, selection and weights of every row in one launch.
#include "ops.h"
#include "dev.h"

namespace sprinter {

// Rows of E logits l.  p = softmax(l) or sigmoid(l); key = p + bias; of the groups of E / G experts only the top_group with the largest
// (max key | sum of the two best keys) stay; ids = the top_k largest keys in descending order, equal ones by index; w = p[ids], over
// their sum if renormalised, times scale.  -inf and NaN logits cannot be taken.  A +inf logit has its limit: it shares the softmax with
// the others like it.
// Scores and keys are float64: which expert is taken is decided by their order, and float32 scores next to each other would round onto
// one another (256 sigmoid scores of 16384 rows: one row in ten would tell).
struct RouteArgs {
  const float* logits; long long ld; const float* bias; int* ids; float* weights;
  int T, E, k, sigmoid, G, top_group, sum2, renorm, shared; float scale;
};

// Larger integer = larger key; no key (and nothing left of a lane): 0.
__device__ __forceinline__ u64 sortable(double v) {
  v += 0.0;                                            // -0 -> +0
  const u64 u = (u64)__double_as_longlong(v);
  return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned dpp_max(unsigned v) {
  const unsigned o = (unsigned)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, ROWS, 0xF, false);
  return v > o ? v : o;
}
__device__ __forceinline__ unsigned wave_umax(unsigned v) {
  v = dpp_max<0xB1, 0xF>(v); v = dpp_max<0x4E, 0xF>(v); v = dpp_max<0x141, 0xF>(v); v = dpp_max<0x140, 0xF>(v);
  v = dpp_max<0x142, 0xA>(v); v = dpp_max<0x143, 0xC>(v);
  return (unsigned)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ __forceinline__ double shfl_xor_f64(double v, int o) { return __longlong_as_double((long long)shfl_xor_u64((u64)__double_as_longlong(v), o)); }
__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v += shfl_xor_f64(v, o);
  return v;
}

// Keys of 32 bits of a float, larger integer = larger float; -inf and NaN: 0, never taken.
__device__ __forceinline__ unsigned sortable(float v) {
  if (!(v > -INFINITY)) return 0;
  const unsigned u = __float_as_uint(v + 0.0f);
  return (u >> 31) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float from_sortable(unsigned u) { return __uint_as_float((u >> 31) ? (u & 0x7fffffffu) : ~u); }

// Reductions over the 16 lanes of a row, the result in each of them
__device__ __forceinline__ unsigned max16(unsigned v) { return dpp_max<0x140, 0xF>(dpp_max<0x141, 0xF>(dpp_max<0x4E, 0xF>(dpp_max<0xB1, 0xF>(v)))); }
__device__ __forceinline__ u64 max16(u64 v) { return group_umax64_16(v); }
__device__ __forceinline__ double sum16(double v) {
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) v += shfl_xor_f64(v, o);
  return v;
}
// The taken keys of a row, one after the other: lane j of the row gets the j-th's value and expert (-1: there is none).
template <typename K, int N>
__device__ __forceinline__ void take16(K (&key)[N], int k, int lane, K& mine, int& id) {
  mine = 0; id = -1;
  for (int j = 0; j < k; ++j) {
    K best = key[0];
#pragma unroll
    for (int i = 1; i < N; ++i) best = best > key[i] ? best : key[i];
    best = max16(best);
    unsigned last = 0;                                 // ~ the lowest index of the largest key
#pragma unroll
    for (int i = N - 1; i >= 0; --i) last = key[i] == best ? ~(unsigned)(i * 16 + lane) : last;
    const unsigned e = ~max16(last);
#pragma unroll
    for (int i = 0; i < N; ++i) key[i] = (unsigned)(i * 16 + lane) == e ? 0 : key[i];
    if (lane == j && best) { mine = best; id = (int)e; }
  }
}

// Without bias and groups, up to 256 experts and 16 of them: four rows per wave, 16 lanes each; lane l of a row holds experts l, 16 + l, ...
// The scores rise with the logits, so the logits themselves are the keys, and only what is taken needs its exponential (and, unless the
// weights are renormalised, the sum of the softmax all of them).  Float64 scores of different logits can meet: by under- and overflow, and
// next to zero, where a float32 is finer than 1 + e^-l or l - max l in 64 bits.  There the wave takes the scores for keys, as the definition does.
// Elsewhere neither order can differ from the other, so that a row's ids depend neither on the rows beside it nor on which kernel takes
// it: logits are 0 or of magnitude 2^-20 and more, so differ by 2^-43 and more; l - max l (below 2^10) is then exact, and e^(l - max l) and
// 1 / (1 + e^-l) differ by 2^-44 of their value and more (p (1 - p) dl: 1 - p > 2^-24 below l = 16, where dl is 2^-20), roundings being a few 2^-53.
// What bounds it: the instructions of the selection rounds, about 45 for four rows (a row per wave: 50 for one).  16381 rows of 64 experts, 8
// taken: 6.8 us by itself, 5.9 in a row of launches (a row per wave 14.6; their 5 MB take 1.1 at the rate of a copy); one row 2.2.
template <int N>
__global__ __launch_bounds__(256) void k_route_plain(RouteArgs a) {
  const int lane = threadIdx.x & 15;
  const long long row = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
  const bool live = row < a.T;
  const float* __restrict__ l = a.logits + (live ? row : 0) * a.ld;
  float x[N];
  unsigned key[N], top = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = l[min(i * 16 + lane, a.E - 1)];
  float low = INFINITY;
  unsigned tiny = ~0u;                                 // least magnitude but 0, as bits, less 1
#pragma unroll
  for (int i = 0; i < N; ++i) {
    tiny = min(tiny, (__float_as_uint(x[i]) & 0x7fffffffu) - 1u);
    key[i] = i * 16 + lane < a.E ? sortable(x[i]) : 0;
    top = max(top, key[i]);
    low = key[i] ? fminf(low, x[i]) : low;
  }
  top = max16(top);
  const float most = from_sortable(top);               // (no expert at all: never used)
  auto score = [&](float v) { return a.sigmoid ? 1.0 / (1.0 + exp(-(double)v)) : v == most ? 1.0 : exp((double)v - (double)most); };
  float mine;
  int id;
  const bool meet = tiny < __float_as_uint(0x1p-20f) - 1u || (a.sigmoid ? most > 16.f || low < -700.f : !(most - low < 700.f));
  if (__ballot(top && meet)) {
    u64 wide[N], value;
    double p[N], part[4] = {0.0, 0.0, 0.0, 0.0}, sum = 1.0;
#pragma unroll
    for (int i = 0; i < N; ++i) { p[i] = key[i] ? score(x[i]) : 0.0; part[i & 3] += p[i]; }
    if (!a.sigmoid) {                                  // (in k_route's order: experts q 16 + lane + 64 i together)
#pragma unroll
      for (int q = 0; q < 4; ++q) part[q] = sum16(part[q]);
      sum = (part[0] + part[1]) + (part[2] + part[3]);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) wide[i] = key[i] ? sortable(p[i] / sum) : 0;
    take16(wide, a.k, lane, value, id);
    mine = l[max(id, 0)];
  } else {
    unsigned value, left[N];
#pragma unroll
    for (int i = 0; i < N; ++i) left[i] = key[i];
    take16(left, a.k, lane, value, id);
    mine = from_sortable(value);
  }
  double w = lane < a.k && id >= 0 ? score(mine) : 0.0;
  if (a.renorm) {
    const double total = sum16(w);
    w = total > 0.0 ? w / total : 0.0;
  } else if (!a.sigmoid) {
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < N; ++i) sum += key[i] ? score(x[i]) : 0.0;
    sum = sum16(sum);
    w = id >= 0 ? w / sum : 0.0;
  }
  w *= (double)a.scale;
  const int n_out = a.k + a.shared;
  if (lane >= a.k) { id = a.E + lane - a.k; w = 1.0; }
  if (live && lane < n_out) {
    a.ids[row * n_out + lane] = id;
    a.weights[row * n_out + lane] = (float)w;
  }
}

// Every other case: one wave per row; lane l holds experts l, 64 + l, ...  A selection round looks at the keys' upper words, and at the
// lower ones where more than one key has the largest upper word.  What bounds it: instructions, of which the exponentials and divisions in
// 64 bits are a third.  4096 rows of 256 sigmoid scores in 8 groups, 8 taken: 11.5 us by itself, 10.3 in a row of launches (groups one after the
// other: 17.5; 4.5 MB take 0.9).
template <int N>
__global__ __launch_bounds__(256) void k_route(RouteArgs a) {
  __shared__ u64 keys[4][N * 64];
  const int lane = threadIdx.x & 63, wave = wave_index();
  const long long row = (long long)blockIdx.x * 4 + wave;
  if (row >= a.T) return;                              // (scalar; no barrier below: a wave has its keys in LDS for itself)
  const float* __restrict__ l = a.logits + row * a.ld;
  float x[N];
  double p[N], bias[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int c = min(i * 64 + lane, a.E - 1);
    x[i] = l[c];
    bias[i] = a.bias ? (double)a.bias[c] : 0.0;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) if (i * 64 + lane >= a.E || !(x[i] > -INFINITY)) x[i] = -INFINITY;       // (NaN too)
  if (a.sigmoid) {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = 1.0 / (1.0 + exp(-(double)x[i]));
  } else {
    float top = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, x[i]);
    top = wave_max(top);
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      p[i] = x[i] == top ? 1.0 : exp((double)x[i] - (double)top);       // (equal infinities: 1)
      if (x[i] == -INFINITY) p[i] = 0.0;
      sum += p[i];
    }
    sum = wave_sum64(sum);
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = p[i] / sum;                      // (a row without experts: 0 / 0, never taken)
  }
  u64 key[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const double v = p[i] + bias[i];
    key[i] = x[i] > -INFINITY && v > -INFINITY ? sortable(v) : 0;
  }
  if (a.G > 1) {                                       // (uniform)
    // 64 / (G rounded up to a power of two) lanes per group find its two best keys
    const int per = a.E / a.G, wide = 1 << (32 - __clz(a.G - 1)), lanes = 64 / wide, g = lane / lanes, s = lane % lanes;
#pragma unroll
    for (int i = 0; i < N; ++i) keys[wave][i * 64 + lane] = key[i];
    __builtin_amdgcn_wave_barrier();                   // (LDS operations of one wave complete in order)
    u64 best = 0, second = 0;
    if (g < a.G)
      for (int c = s; c < per; c += lanes) {
        const u64 v = keys[wave][g * per + c];
        second = umax64(second, min(best, v));
        best = umax64(best, v);
      }
    for (int o = 1; o < lanes; o <<= 1) {
      const u64 ob = shfl_xor_u64(best, o), os = shfl_xor_u64(second, o);
      second = umax64(umax64(second, os), min(best, ob));
      best = umax64(best, ob);
    }
    auto back = [](u64 v) { return __longlong_as_double((long long)((v >> 63) ? (v & 0x7fffffffffffffffull) : ~v)); };
    u64 rank = best;
    if (a.sum2 && best && second) rank = sortable(back(best) + back(second));
    // a group is taken if fewer than top_group are ahead of it
    int ahead = 0;
    for (int q = 0; q < a.G; ++q) {
      const u64 other = ((u64)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)(rank >> 32), q * lanes) << 32) | (unsigned)__builtin_amdgcn_readlane((int)(unsigned)rank, q * lanes);
      ahead += other > rank || (other == rank && q < g);
    }
    const u64 taken = __ballot(g < a.G && ahead < a.top_group);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int mine = (i * 64 + lane) / per;
      if (!(taken >> (min(mine, a.G - 1) * lanes) & 1)) key[i] = 0;
    }
  }
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int i = 0; i < N; ++i) keys[wave][i * 64 + lane] = (u64)__double_as_longlong(p[i]);       // the scores, in the keys' place and type
  __builtin_amdgcn_wave_barrier();
  unsigned hi[N];
#pragma unroll
  for (int i = 0; i < N; ++i) hi[i] = (unsigned)(key[i] >> 32);
  int id = -1;                                         // lane j: the row's j-th
  for (int j = 0; j < a.k; ++j) {
    unsigned most = hi[0];
#pragma unroll
    for (int i = 1; i < N; ++i) most = max(most, hi[i]);
    most = wave_umax(most);
    if (most == 0) break;                              // (scalar)
    u64 at[N];
    int n = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) { at[i] = __ballot(hi[i] == most); n += __popcll(at[i]); }
    if (n > 1) {                                       // (scalar)
      unsigned lo = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) lo = hi[i] == most ? max(lo, (unsigned)key[i]) : lo;
      lo = wave_umax(lo);
#pragma unroll
      for (int i = 0; i < N; ++i) at[i] = __ballot(hi[i] == most && (unsigned)key[i] == lo);
    }
    int e = 0;
#pragma unroll
    for (int i = N - 1; i >= 0; --i) e = at[i] ? i * 64 + __builtin_ctzll(at[i]) : e;       // the lowest index of the largest (scalar)
#pragma unroll
    for (int i = 0; i < N; ++i) hi[i] = i * 64 + lane == e ? 0 : hi[i];
    if (lane == j) id = e;
  }
  double w = id >= 0 ? __longlong_as_double((long long)keys[wave][id]) : 0.0;
  if (a.renorm) {
    const double total = wave_sum64(w);
    w = total > 0.0 ? w / total : 0.0;
  }
  w *= (double)a.scale;
  const int n_out = a.k + a.shared;
  if (lane >= a.k) { id = a.E + lane - a.k; w = 1.0; }
  if (lane < n_out) {
    a.ids[row * n_out + lane] = id;
    a.weights[row * n_out + lane] = (float)w;
  }
}

const char* route_cfg_error(const sprinter_route_cfg& c) {
  if (c.n_expert < 1 || c.n_expert > MAX_EXPERTS) return "n_expert outside [1, 1024]";
  if (c.top_k < 1 || c.top_k > MAX_TOP_K - MAX_SHARED || c.top_k > c.n_expert) return "top_k outside [1, min(48, n_expert)]";
  if (c.score != SPRINTER_SCORE_SOFTMAX && c.score != SPRINTER_SCORE_SIGMOID) return "score is neither softmax nor sigmoid";
  if (c.n_group < 1 || c.n_group > MAX_GROUPS || c.n_expert % c.n_group) return "n_group is not a divisor of n_expert in [1, 64]";
  if (c.top_group < 1 || c.top_group > c.n_group) return "top_group outside [1, n_group]";
  if (c.top_k > c.n_expert / c.n_group * c.top_group) return "top_k experts do not fit in top_group groups";
  if (c.group_score != SPRINTER_GROUP_MAX && c.group_score != SPRINTER_GROUP_BEST_TWO) return "group_score is neither max nor the best two";
  if (c.n_shared < 0 || c.n_shared > MAX_SHARED) return "n_shared outside [0, 16]";
  if (!(c.scale > 0.f) || !(c.scale < INFINITY)) return "scale is not a positive number";
  return nullptr;
}

void launch_route(const sprinter_route_cfg& c, const float* logits, long long ld, const float* bias, int n_rows, int* ids, float* weights,
                  hipStream_t s) {
  const RouteArgs a{logits, ld, bias, ids, weights, n_rows, c.n_expert, c.top_k, c.score == SPRINTER_SCORE_SIGMOID, c.n_group, c.top_group,
                    c.group_score == SPRINTER_GROUP_BEST_TWO, c.renormalize != 0, c.n_shared, c.scale};
  if (!bias && c.n_group == 1 && c.n_expert <= 256 && c.top_k + c.n_shared <= 16) {
    const dim3 grid((n_rows + 15) / 16), block(256);
    if (c.n_expert <= 16) hipLaunchKernelGGL(k_route_plain<1>, grid, block, 0, s, a);
    else if (c.n_expert <= 64) hipLaunchKernelGGL(k_route_plain<4>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(k_route_plain<16>, grid, block, 0, s, a);
    return;
  }
  const dim3 grid((n_rows + 3) / 4), block(256);
  if (c.n_expert <= 64) hipLaunchKernelGGL(k_route<1>, grid, block, 0, s, a);
  else if (c.n_expert <= 128) hipLaunchKernelGGL(k_route<2>, grid, block, 0, s, a);
  else if (c.n_expert <= 256) hipLaunchKernelGGL(k_route<4>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(k_route<16>, grid, block, 0, s, a);
}

}  // namespace sprinter
