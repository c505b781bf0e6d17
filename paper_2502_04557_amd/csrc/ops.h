// Launchers of the operators of expert models and of norms around a block (k_route.hip, k_experts.hip, k_block_norm.hip), which the
// entry points of ops.cpp and the model path of abi.cpp share.  Arguments are valid: the callers check them.
#pragma once
#include "internal.h"
#include "../../include/sprinter.h"

namespace sprinter {

constexpr int MAX_EXPERTS = 1024, MAX_TOP_K = 64, MAX_SHARED = 16, MAX_GROUPS = 64;
constexpr int MAX_BLOCK_COLS = 16384;            // columns of launch_block_norm

// nullptr, or what is wrong with the configuration.
const char* route_cfg_error(const sprinter_route_cfg& c);
void launch_route(const sprinter_route_cfg& c, const float* logits, long long ld, const float* bias, int n_rows, int* ids, float* weights,
                  hipStream_t s);

// Packed form of a bf16 matrix [E][N][K]: each expert's operand tiles (float16), 16 rows and 32 k to a tile, zero padded.
inline size_t expert_elems(int N, int K) { return (size_t)round_up(N, 16) * round_up(K, 32); }
void launch_pack_experts(const void* w, void* out, int E, int N, int K, hipStream_t s);

enum { X_F32 = 0, X_BF16 = 1, X_F16 = 2 };       // element types of rows that come in (or go out)
struct ExpertsArgs {
  int dtype, E, d, ff;                           // dtype SPRINTER_BF16: packed weights; SPRINTER_F32: row-major float32
  const void *wg, *wu, *w2;
  const void* x; int x_type; long long ldx;      // rows of d, 16-byte aligned
  const int* ids; const float* weights;          // [T][k]; an id outside [0, E) adds nothing
  int T, k;
  void* y; int y_type; long long ldy;            // rows of d, 16-byte aligned
};
size_t experts_workspace(int dtype, int E, int d, int ff, long long T, int k);
void launch_experts(const ExpertsArgs& a, void* workspace, hipStream_t s);

// u = norm(y; post) or y;  h_out = h + scale gate u;  out = norm(h_out; gain).
struct BlockNormArgs {
  int kind, d, T;                                // kind 0: layer norm, 1: RMS norm (sprinter.h)
  float eps, scale;
  const float* h; long long ldh;
  const void* y; int y_type; long long ldy;
  const float *post_g, *post_b;                  // NULL: y itself; NULL: no offset
  const float* gate; long long gate_row, gate_col;   // NULL: 1
  const float *g, *b;
  float* h_out; long long ld_h_out;
  void* out; int out_type; long long ldo;        // rows, or NULL
  void* tiles;                                   // the same values as float16 operand tiles (or NULL)
  float* f32;                                    // the same values as float32 rows of d (or NULL)
};
void launch_block_norm(const BlockNormArgs& a, hipStream_t s);

int op_fail(int code, const char* fmt, ...);     // the thread's last error (abi.cpp)

}  // namespace sprinter
