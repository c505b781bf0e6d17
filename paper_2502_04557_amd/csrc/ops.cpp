// C-ABI layer of the operators: validation of their arguments, then the launchers of ops.h.
#include "ops.h"

using namespace sprinter;

namespace {

constexpr int MAX_EXPERT_PAIRS = 1 << 20, MAX_ROWS = 1 << 23;      // (a grid has fewer than 2^32 threads)

bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
size_t element(int dtype) { return dtype == SPRINTER_F32 ? 4 : 2; }

// Around a call's launches.  An error that other code of the thread has left is not this call's: it is dropped before them.
void launching() { (void)hipGetLastError(); }
int launched(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SPRINTER_OK : op_fail(SPRINTER_E_HIP, "%s: %s", what, hipGetErrorString(e));
}

int check_experts(const sprinter_experts_cfg* c, const char* who) {
  if (!c) return op_fail(SPRINTER_E_NULL, "%s: NULL configuration", who);
  if (c->dtype != SPRINTER_F32 && c->dtype != SPRINTER_BF16) return op_fail(SPRINTER_E_CONFIG, "%s: unknown dtype %d", who, c->dtype);
  if (c->n_expert < 1 || c->n_expert > MAX_EXPERTS) return op_fail(SPRINTER_E_CONFIG, "%s: n_expert %d outside [1, %d]", who, c->n_expert, MAX_EXPERTS);
  if (c->d_model < 8 || c->d_model > 8192 || c->d_model % 8)
    return op_fail(SPRINTER_E_CONFIG, "%s: d_model %d is not a multiple of 8 in [8, 8192]", who, c->d_model);
  if (c->d_ff < 8 || c->d_ff > 65536 || c->d_ff % 8) return op_fail(SPRINTER_E_CONFIG, "%s: d_ff %d is not a multiple of 8 in [8, 65536]", who, c->d_ff);
  return SPRINTER_OK;
}

int check_pairs(int n_rows, int top_k, const char* who) {
  if (n_rows < 0) return op_fail(SPRINTER_E_RANGE, "%s: %d rows", who, n_rows);
  if (top_k < 1 || top_k > MAX_TOP_K) return op_fail(SPRINTER_E_RANGE, "%s: top_k %d outside [1, %d]", who, top_k, MAX_TOP_K);
  if ((long long)n_rows * top_k > MAX_EXPERT_PAIRS)
    return op_fail(SPRINTER_E_RANGE, "%s: %d rows of %d ids are more than %d", who, n_rows, top_k, MAX_EXPERT_PAIRS);
  return SPRINTER_OK;
}

}  // namespace

extern "C" {

int sprinter_route(const sprinter_route_cfg* cfg, const float* dev_logits, int64_t ld_logits, const float* dev_bias, int n_rows,
                   int32_t* dev_ids, float* dev_weights, void* hip_stream) {
  if (!cfg) return op_fail(SPRINTER_E_NULL, "sprinter_route: NULL configuration");
  if (const char* e = route_cfg_error(*cfg)) return op_fail(SPRINTER_E_CONFIG, "sprinter_route: %s", e);
  if (n_rows < 0 || n_rows > MAX_ROWS) return op_fail(SPRINTER_E_RANGE, "sprinter_route: %d rows are not in [0, %d]", n_rows, MAX_ROWS);
  if (n_rows == 0) return SPRINTER_OK;
  if (!dev_logits || !dev_ids || !dev_weights) return op_fail(SPRINTER_E_NULL, "sprinter_route: NULL array");
  if (n_rows > 1 && ld_logits < cfg->n_expert)
    return op_fail(SPRINTER_E_RANGE, "sprinter_route: rows %lld apart hold no %d logits", (long long)ld_logits, cfg->n_expert);
  if (!aligned(dev_logits, 4) || !aligned(dev_bias, 4) || !aligned(dev_ids, 4) || !aligned(dev_weights, 4))
    return op_fail(SPRINTER_E_RANGE, "sprinter_route: an array is not aligned to its elements");
  launching();
  launch_route(*cfg, dev_logits, ld_logits, dev_bias, n_rows, dev_ids, dev_weights, (hipStream_t)hip_stream);
  return launched("sprinter_route");
}

int sprinter_experts_bytes(const sprinter_experts_cfg* cfg, int max_rows, int top_k, size_t* out_packed_up, size_t* out_packed_down,
                           size_t* out_workspace) {
  int rc = check_experts(cfg, "sprinter_experts_bytes");
  if (rc || (rc = check_pairs(max_rows, top_k, "sprinter_experts_bytes"))) return rc;
  const bool bf = cfg->dtype == SPRINTER_BF16;
  if (out_packed_up) *out_packed_up = bf ? expert_elems(cfg->d_ff, cfg->d_model) * cfg->n_expert * 2 : 0;
  if (out_packed_down) *out_packed_down = bf ? expert_elems(cfg->d_model, cfg->d_ff) * cfg->n_expert * 2 : 0;
  if (out_workspace) *out_workspace = experts_workspace(cfg->dtype, cfg->n_expert, cfg->d_model, cfg->d_ff, max_rows, top_k);
  return SPRINTER_OK;
}

int sprinter_experts_pack(const sprinter_experts_cfg* cfg, int down, const void* dev_weights, void* dev_packed, void* hip_stream) {
  const int rc = check_experts(cfg, "sprinter_experts_pack");
  if (rc) return rc;
  if (cfg->dtype != SPRINTER_BF16) return op_fail(SPRINTER_E_CONFIG, "sprinter_experts_pack: only bf16 weights are packed");
  if (!dev_weights || !dev_packed) return op_fail(SPRINTER_E_NULL, "sprinter_experts_pack: NULL array");
  if (!aligned(dev_weights, 16) || !aligned(dev_packed, 16))
    return op_fail(SPRINTER_E_RANGE, "sprinter_experts_pack: an array is not 16-byte aligned");
  launching();
  launch_pack_experts(dev_weights, dev_packed, cfg->n_expert, down ? cfg->d_model : cfg->d_ff, down ? cfg->d_ff : cfg->d_model,
                      (hipStream_t)hip_stream);
  return launched("sprinter_experts_pack");
}

int sprinter_experts(const sprinter_experts_cfg* cfg, const void* dev_gate, const void* dev_up, const void* dev_down, const void* dev_x,
                     int64_t ld_x, const int32_t* dev_ids, const float* dev_route_weights, int n_rows, int top_k, void* dev_y, int64_t ld_y,
                     void* dev_workspace, size_t workspace_bytes, void* hip_stream) {
  int rc = check_experts(cfg, "sprinter_experts");
  if (rc || (rc = check_pairs(n_rows, top_k, "sprinter_experts"))) return rc;
  if (n_rows == 0) return SPRINTER_OK;
  if (!dev_gate || !dev_up || !dev_down || !dev_x || !dev_ids || !dev_route_weights || !dev_y || !dev_workspace)
    return op_fail(SPRINTER_E_NULL, "sprinter_experts: NULL array");
  const size_t es = element(cfg->dtype);
  if (n_rows > 1 && (ld_x < cfg->d_model || ld_y < cfg->d_model))
    return op_fail(SPRINTER_E_RANGE, "sprinter_experts: rows %lld and %lld apart hold no %d columns", (long long)ld_x, (long long)ld_y, cfg->d_model);
  if (!aligned(dev_gate, 16) || !aligned(dev_up, 16) || !aligned(dev_down, 16) || !aligned(dev_x, 16) || !aligned(dev_y, 16) ||
      (n_rows > 1 && ((ld_x * es) % 16 || (ld_y * es) % 16)))
    return op_fail(SPRINTER_E_RANGE, "sprinter_experts: weights or rows are not 16-byte aligned");
  if (!aligned(dev_ids, 4) || !aligned(dev_route_weights, 4))
    return op_fail(SPRINTER_E_RANGE, "sprinter_experts: ids or weights are not aligned to their elements");
  const size_t need = experts_workspace(cfg->dtype, cfg->n_expert, cfg->d_model, cfg->d_ff, n_rows, top_k);
  if (!aligned(dev_workspace, 256)) return op_fail(SPRINTER_E_WORKSPACE, "sprinter_experts: workspace is not 256-byte aligned");
  if (workspace_bytes < need) return op_fail(SPRINTER_E_WORKSPACE, "sprinter_experts: workspace has %zu bytes, %zu needed", workspace_bytes, need);
  const int type = cfg->dtype == SPRINTER_F32 ? X_F32 : X_BF16;
  const ExpertsArgs a{cfg->dtype, cfg->n_expert, cfg->d_model, cfg->d_ff, dev_gate, dev_up, dev_down, dev_x, type, ld_x, dev_ids,
                      dev_route_weights, n_rows, top_k, dev_y, type, ld_y};
  launching();
  launch_experts(a, dev_workspace, (hipStream_t)hip_stream);
  return launched("sprinter_experts");
}

int sprinter_block_norm(const sprinter_block_norm_cfg* cfg, const float* dev_h, int64_t ld_h, const void* dev_y, int64_t ld_y,
                        const float* dev_post_gain, const float* dev_post_offset, const float* dev_gate, int64_t gate_row, int64_t gate_col,
                        const float* dev_gain, const float* dev_offset, int n_rows, float* dev_h_out, int64_t ld_h_out, void* dev_out,
                        int64_t ld_out, void* hip_stream) {
  if (!cfg) return op_fail(SPRINTER_E_NULL, "sprinter_block_norm: NULL configuration");
  if (cfg->dtype != SPRINTER_F32 && cfg->dtype != SPRINTER_BF16) return op_fail(SPRINTER_E_CONFIG, "sprinter_block_norm: unknown dtype %d", cfg->dtype);
  if (cfg->kind != SPRINTER_NORM_LAYER && cfg->kind != SPRINTER_NORM_RMS)
    return op_fail(SPRINTER_E_CONFIG, "sprinter_block_norm: kind %d is neither a layer norm nor an RMS norm", cfg->kind);
  if (cfg->d < 1 || cfg->d > MAX_BLOCK_COLS) return op_fail(SPRINTER_E_CONFIG, "sprinter_block_norm: d %d outside [1, %d]", cfg->d, MAX_BLOCK_COLS);
  if (!(cfg->eps >= 0.f) || !(cfg->scale == cfg->scale)) return op_fail(SPRINTER_E_CONFIG, "sprinter_block_norm: eps is negative or scale is NaN");
  if (n_rows < 0 || n_rows > MAX_ROWS) return op_fail(SPRINTER_E_RANGE, "sprinter_block_norm: %d rows are not in [0, %d]", n_rows, MAX_ROWS);
  if (n_rows == 0) return SPRINTER_OK;
  if (!dev_h || !dev_y || !dev_gain || !dev_h_out || !dev_out) return op_fail(SPRINTER_E_NULL, "sprinter_block_norm: NULL array");
  if (dev_post_offset && !dev_post_gain) return op_fail(SPRINTER_E_NULL, "sprinter_block_norm: post_offset without post_gain");
  if (n_rows > 1 && (ld_h < cfg->d || ld_y < cfg->d || ld_h_out < cfg->d || ld_out < cfg->d))
    return op_fail(SPRINTER_E_RANGE, "sprinter_block_norm: rows lie closer than their %d columns", cfg->d);
  if (gate_row < 0 || gate_col < 0) return op_fail(SPRINTER_E_RANGE, "sprinter_block_norm: negative stride of the gate");
  const size_t es = element(cfg->dtype);
  if (!aligned(dev_h, 4) || !aligned(dev_h_out, 4) || !aligned(dev_y, es) || !aligned(dev_out, es) || !aligned(dev_post_gain, 4) ||
      !aligned(dev_post_offset, 4) || !aligned(dev_gate, 4) || !aligned(dev_gain, 4) || !aligned(dev_offset, 4))
    return op_fail(SPRINTER_E_RANGE, "sprinter_block_norm: an array is not aligned to its elements");
  const int type = cfg->dtype == SPRINTER_F32 ? X_F32 : X_BF16;
  BlockNormArgs a{};
  a.kind = cfg->kind; a.d = cfg->d; a.T = n_rows; a.eps = cfg->eps; a.scale = cfg->scale;
  a.h = dev_h; a.ldh = ld_h; a.y = dev_y; a.y_type = type; a.ldy = ld_y; a.post_g = dev_post_gain; a.post_b = dev_post_offset;
  a.gate = dev_gate; a.gate_row = gate_row; a.gate_col = gate_col; a.g = dev_gain; a.b = dev_offset;
  a.h_out = dev_h_out; a.ld_h_out = ld_h_out; a.out = dev_out; a.out_type = type; a.ldo = ld_out;
  launching();
  launch_block_norm(a, (hipStream_t)hip_stream);
  return launched("sprinter_block_norm");
}

}  // extern "C"
