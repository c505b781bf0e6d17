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

// A cache in pages, one layer of it (k_cache.hip, k_tree_attn.hip): keys and values [n_page][KVH][page][dh]; slot s of sequence b is place
// s % page of page table[b][s / page], and not there where that is no page.
struct PagedArgs {
  void *keys, *values;
  const int* table; long long ld_table;
  int n_seq, n_table, n_page, shift, KVH, dh;    // page size 1 << shift
};
struct AppendArgs {
  PagedArgs c;
  int cache_type, row_type, H, T, n_turned, pairs;   // pairs 0: columns (i, i + n / 2), 1: (2 i, 2 i + 1)
  const int *seq, *slot, *pos;                   // pos NULL: the slot
  const double* freq;                            // [n_turned / 2]
  const void *k, *v, *q; long long ld_k, ld_v, ld_q;   // q NULL: none
  void* q_out; long long ld_q_out;               // of the cache's type
};
void launch_cache_append(const AppendArgs& a, hipStream_t s);
struct KeepArgs {
  PagedArgs c;                                   // keys, values of layer 0
  int n_layer; long long layer_bytes;
  int element;                                   // bytes
  const int *lens, *first, *path, *n_keep; long long ld_path; int n_path;
};
void launch_cache_keep(const KeepArgs& a, hipStream_t s);
// The scale of scores as a base-2 exponent's, the difference of products q.k that is an exponent of 8, and whether the scale is negative.
struct Base2 { float c, lag; int flip; };
Base2 base2(float scale);
struct AttendArgs {
  PagedArgs c;
  int type, H, T, n_words;
  Base2 scale;
  const int *lens, *first;
  const unsigned long long* visible;             // [T][n_words], or NULL: the nodes up to the row's own
  const void* q; long long ld_q;
  void* y; long long ld_y;
};
size_t attend_workspace(int type, int dh, int H, int KVH, int n_seq, int T, long long slots);
void launch_cache_attend(const AttendArgs& a, void* workspace, hipStream_t s);

constexpr int MAX_HISTORY = 1 << 19, MAX_BIASES = 2047, MAX_NODE_WORDS = 16;
void launch_adjust_logits(const sprinter_logits& a, hipStream_t s);

int op_fail(int code, const char* fmt, ...);     // the thread's last error (abi.cpp)

}  // namespace sprinter
