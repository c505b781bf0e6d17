// HIP kernel of routing to experts for gfx950: scores, selection and weights of every row in one launch.
#include "ops.h"
#include "dev.h"

namespace sprinter {

// Rows of E logits l.  p = softmax(l) or sigmoid(l); key = p + bias; of the groups of E / G experts only the top_group with the largest
// (max key | sum of the two best keys) stay; ids = the top_k largest keys in descending order, equal ones by index; w = p[ids], over
// their sum if renormalised, times scale.  -inf and NaN logits cannot be taken.  A +inf logit has its limit: it shares the softmax with
// the others like it.
// One wave per row; lane l holds experts l, 64 + l, ...  Scores and keys are float64: which expert is taken is decided by their order, and
// float32 scores next to each other would round onto one another (256 sigmoid scores of 16384 rows: one row in ten would tell).
// A selection round is a maximum over the lanes of the keys' upper words (six DPP steps of one v_max each), and of the lower words where
// more than one lane holds the upper one.
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
__device__ __forceinline__ u64 wave_umax64(u64 v) {
  const unsigned hi = wave_umax((unsigned)(v >> 32));
  const u64 at = __ballot((unsigned)(v >> 32) == hi);
  unsigned lo;
  if ((at & (at - 1)) == 0) lo = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)v, __builtin_ctzll(at));   // (scalar)
  else lo = wave_umax((unsigned)(v >> 32) == hi ? (unsigned)v : 0u);
  return ((u64)hi << 32) | lo;
}
__device__ __forceinline__ double read_lane(double v, int lane) {
  const u64 u = (u64)__double_as_longlong(v);
  const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)u, lane), hi = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)(u >> 32), lane);
  return __longlong_as_double((long long)(((u64)hi << 32) | lo));
}
__device__ __forceinline__ double shfl_xor_f64(double v, int o) { return __longlong_as_double((long long)shfl_xor_u64((u64)__double_as_longlong(v), o)); }
__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v += shfl_xor_f64(v, o);
  return v;
}

template <int N>                                       // experts per lane
__global__ __launch_bounds__(256) void k_route(RouteArgs a) {
  const int lane = threadIdx.x & 63;
  const long long row = (long long)blockIdx.x * 4 + wave_index();
  if (row >= a.T) return;                              // (scalar; no barrier below)
  const float* __restrict__ l = a.logits + row * a.ld;
  float x[N];
  double p[N], bias[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = i * 64 + lane, c = min(e, a.E - 1);
    x[i] = l[c];
    bias[i] = a.bias ? (double)a.bias[c] : 0.0;
    if (e >= a.E || !(x[i] > -INFINITY)) x[i] = -INFINITY;             // (NaN too)
  }
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
    // each group's rank in lane g, in sortable order; a group's experts lie in up to E / G lanes of up to N registers
    const int per = a.E / a.G;
    u64 rank = 0;
    for (int g = 0; g < a.G; ++g) {
      u64 best = 0, second = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const u64 v = (i * 64 + lane) / per == g ? key[i] : 0;
        second = umax64(second, min(best, v));
        best = umax64(best, v);
      }
      const u64 m = wave_umax64(best);
      u64 value = m;
      if (a.sum2 && m) {
        // one lane gives up its best; the rest keep theirs
        const u64 at = __ballot(best == m);
        const u64 s = wave_umax64(lane == __builtin_ctzll(at) ? second : best);
        auto back = [](u64 v) { return __longlong_as_double((long long)((v >> 63) ? (v & 0x7fffffffffffffffull) : ~v)); };
        value = sortable(back(m) + (s ? back(s) : 0.0));
      }
      if (lane == g) rank = value;
    }
    u64 taken = 0;                                     // a bit per group
    for (int j = 0; j < a.top_group; ++j) {
      const u64 m = wave_umax64(rank);
      if (m == 0) break;
      const int g = __builtin_ctzll(__ballot(rank == m));
      taken |= 1ull << g;
      if (lane == g) rank = 0;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (!(taken >> min((i * 64 + lane) / per, 63) & 1)) key[i] = 0;
  }
  const int n_out = a.k + a.shared;
  int id = lane < a.k ? -1 : a.E + lane - a.k;         // lane j: the row's j-th id and weight
  double w = lane < a.k ? 0.0 : 1.0, total = 0.0;
  for (int j = 0; j < a.k; ++j) {
    u64 best = key[0];
#pragma unroll
    for (int i = 1; i < N; ++i) best = umax64(best, key[i]);
    const u64 m = wave_umax64(best);
    if (m == 0) break;                                 // (scalar)
    int e = -1;
    double pe = 0.0;
#pragma unroll
    for (int i = N - 1; i >= 0; --i) {                 // the lowest index of the largest
      const u64 at = __ballot(key[i] == m);
      if (at) { const int at_lane = __builtin_ctzll(at); e = i * 64 + at_lane; pe = read_lane(p[i], at_lane); }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) if (i * 64 + lane == e) key[i] = 0;
    if (lane == j) { id = e; w = pe; }
    total += pe;
  }
  if (lane < a.k) {
    if (a.renorm) w = total > 0.0 ? w / total : 0.0;
    w *= (double)a.scale;
  }
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
  const dim3 grid((n_rows + 3) / 4), block(256);
  if (c.n_expert <= 64) hipLaunchKernelGGL(k_route<1>, grid, block, 0, s, a);
  else if (c.n_expert <= 128) hipLaunchKernelGGL(k_route<2>, grid, block, 0, s, a);
  else if (c.n_expert <= 256) hipLaunchKernelGGL(k_route<4>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(k_route<16>, grid, block, 0, s, a);
}

}  // namespace sprinter
