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

constexpr int MAX_TREE_ROWS = 1 << 20;
static_assert(sizeof(sprinter_append) == 160 && sizeof(sprinter_attend) == 136 && sizeof(sprinter_keep) == 88 && sizeof(sprinter_logits) == 200,
              "the layouts that bindings pack");

// What every call on a cache in pages has; fills *c for one layer's arrays.
int check_cache(const sprinter_cache_cfg* g, int layer, const void* keys, const void* values, const int32_t* table, int64_t ld_table, int n_seq,
                int n_table, const char* who, PagedArgs* c) {
  if (!g) return op_fail(SPRINTER_E_NULL, "%s: NULL configuration", who);
  if (g->dtype != SPRINTER_F32 && g->dtype != SPRINTER_BF16) return op_fail(SPRINTER_E_CONFIG, "%s: unknown dtype %d", who, g->dtype);
  if (g->n_layer < 1 || g->n_layer > 65535) return op_fail(SPRINTER_E_CONFIG, "%s: n_layer %d outside [1, 65535]", who, g->n_layer);
  if (g->n_page < 1) return op_fail(SPRINTER_E_CONFIG, "%s: n_page %d is not positive", who, g->n_page);
  if (g->page_size < 8 || g->page_size > 1024 || (g->page_size & (g->page_size - 1)))
    return op_fail(SPRINTER_E_CONFIG, "%s: page_size %d is no power of two in [8, 1024]", who, g->page_size);
  if (g->n_kv_head < 1 || g->n_kv_head > 1024) return op_fail(SPRINTER_E_CONFIG, "%s: n_kv_head %d outside [1, 1024]", who, g->n_kv_head);
  if (g->d_head != 64 && g->d_head != 128) return op_fail(SPRINTER_E_CONFIG, "%s: d_head %d is neither 64 nor 128", who, g->d_head);
  if (layer < 0 || layer >= g->n_layer) return op_fail(SPRINTER_E_RANGE, "%s: layer %d outside [0, %d)", who, layer, g->n_layer);
  if (n_seq < 0 || n_seq > MAX_TREE_ROWS) return op_fail(SPRINTER_E_RANGE, "%s: %d sequences are not in [0, %d]", who, n_seq, MAX_TREE_ROWS);
  if (n_table < 0 || (long long)n_table * g->page_size >= 1 << 30)
    return op_fail(SPRINTER_E_RANGE, "%s: %d pages of %d slots are not in [0, 2^30)", who, n_table, g->page_size);
  if (!keys || !values || (!table && n_table > 0 && n_seq > 0)) return op_fail(SPRINTER_E_NULL, "%s: NULL array", who);
  if (n_seq > 1 && ld_table < n_table) return op_fail(SPRINTER_E_RANGE, "%s: rows %lld apart hold no %d pages", who, (long long)ld_table, n_table);
  if (!aligned(keys, 16) || !aligned(values, 16)) return op_fail(SPRINTER_E_RANGE, "%s: keys or values are not 16-byte aligned", who);
  if (!aligned(table, 4)) return op_fail(SPRINTER_E_RANGE, "%s: table is not aligned to its elements", who);
  const long long off = (long long)layer * g->n_page * g->n_kv_head * g->page_size * g->d_head * element(g->dtype);
  int shift = 0;
  while (1 << shift < g->page_size) ++shift;
  *c = PagedArgs{(char*)keys + off, (char*)values + off, table, ld_table, n_seq, n_table, g->n_page, shift, g->n_kv_head, g->d_head};
  return SPRINTER_OK;
}

int check_heads(const sprinter_cache_cfg* g, int n_head, const char* who) {
  if (n_head < 1 || n_head > 4096 || n_head % g->n_kv_head)
    return op_fail(SPRINTER_E_RANGE, "%s: n_head %d is no multiple of n_kv_head %d up to 4096", who, n_head, g->n_kv_head);
  return SPRINTER_OK;
}

int check_tree_rows(int n_rows, const char* who) {
  if (n_rows < 0 || n_rows > MAX_TREE_ROWS) return op_fail(SPRINTER_E_RANGE, "%s: %d rows are not in [0, %d]", who, n_rows, MAX_TREE_ROWS);
  return SPRINTER_OK;
}

int check_attended(int n_rows, int n_head, const char* who) {
  const int rc = check_tree_rows(n_rows, who);
  if (rc) return rc;
  if ((long long)n_rows * n_head > 1 << 23) return op_fail(SPRINTER_E_RANGE, "%s: %d rows of %d heads are more than 2^23", who, n_rows, n_head);
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

int sprinter_cache_append(const sprinter_cache_cfg* cfg, const sprinter_append* args, void* hip_stream) {
  const char* who = "sprinter_cache_append";
  if (!args) return op_fail(SPRINTER_E_NULL, "%s: NULL arguments", who);
  const sprinter_append& x = *args;
  AppendArgs a{};
  int rc = check_cache(cfg, x.layer, x.keys, x.values, x.table, x.ld_table, x.n_seq, x.n_table, who, &a.c);
  if (rc || (rc = check_tree_rows(x.n_rows, who)) || (x.n_head != 0 && (rc = check_heads(cfg, x.n_head, who)))) return rc;
  if (x.n_turned < 0 || x.n_turned > cfg->d_head || x.n_turned % 2)
    return op_fail(SPRINTER_E_RANGE, "%s: n_turned %d is no even number up to d_head %d", who, x.n_turned, cfg->d_head);
  if (x.pairs != SPRINTER_PAIRS_HALVES && x.pairs != SPRINTER_PAIRS_NEIGHBOURS) return op_fail(SPRINTER_E_CONFIG, "%s: unknown pairs %d", who, x.pairs);
  if (x.rows_dtype != SPRINTER_F32 && x.rows_dtype != SPRINTER_BF16) return op_fail(SPRINTER_E_CONFIG, "%s: unknown rows_dtype %d", who, x.rows_dtype);
  if (x.n_rows == 0 || x.n_seq == 0) return SPRINTER_OK;
  if (!x.seq || !x.slot || !x.k || !x.v || (x.n_turned && !x.freq) || (x.n_head && (!x.q || !x.q_out)))
    return op_fail(SPRINTER_E_NULL, "%s: NULL array", who);
  const int w = cfg->n_kv_head * cfg->d_head, wq = x.n_head * cfg->d_head;
  if (x.n_rows > 1 && (x.ld_k < w || x.ld_v < w || (x.n_head && (x.ld_q < wq || x.ld_q_out < wq))))
    return op_fail(SPRINTER_E_RANGE, "%s: rows lie closer than their columns", who);
  const size_t in = element(x.rows_dtype), out = element(cfg->dtype);
  if (!aligned(x.seq, 4) || !aligned(x.slot, 4) || !aligned(x.pos, 4) || !aligned(x.freq, 8) || !aligned(x.k, in) || !aligned(x.v, in) ||
      (x.n_head && (!aligned(x.q, in) || !aligned(x.q_out, out))))
    return op_fail(SPRINTER_E_RANGE, "%s: an array is not aligned to its elements", who);
  a.cache_type = cfg->dtype == SPRINTER_F32 ? X_F32 : X_BF16;
  a.row_type = x.rows_dtype == SPRINTER_F32 ? X_F32 : X_BF16;
  a.H = x.n_head; a.T = x.n_rows; a.n_turned = x.n_turned; a.pairs = x.pairs;
  a.seq = x.seq; a.slot = x.slot; a.pos = x.pos; a.freq = x.freq;
  a.k = x.k; a.ld_k = x.ld_k; a.v = x.v; a.ld_v = x.ld_v; a.q = x.q; a.ld_q = x.ld_q; a.q_out = x.q_out; a.ld_q_out = x.ld_q_out;
  launching();
  launch_cache_append(a, (hipStream_t)hip_stream);
  return launched(who);
}

int sprinter_cache_attend_bytes(const sprinter_cache_cfg* cfg, int n_head, int n_seq, int n_table, int n_rows, size_t* out_workspace) {
  const char* who = "sprinter_cache_attend_bytes";
  PagedArgs c;
  const void* some = (const void*)256;                 // (only the sizes are looked at)
  int rc = check_cache(cfg, 0, some, some, (const int32_t*)some, n_table, n_seq, n_table, who, &c);
  if (rc || (rc = check_heads(cfg, n_head, who)) || (rc = check_attended(n_rows, n_head, who))) return rc;
  if (!out_workspace) return op_fail(SPRINTER_E_NULL, "%s: NULL result", who);
  *out_workspace = attend_workspace(cfg->dtype == SPRINTER_F32 ? X_F32 : X_BF16, cfg->d_head, n_head, cfg->n_kv_head, n_seq, n_rows,
                                    (long long)n_table * cfg->page_size);
  return SPRINTER_OK;
}

int sprinter_cache_attend(const sprinter_cache_cfg* cfg, const sprinter_attend* args, void* hip_stream) {
  const char* who = "sprinter_cache_attend";
  if (!args) return op_fail(SPRINTER_E_NULL, "%s: NULL arguments", who);
  const sprinter_attend& x = *args;
  AttendArgs a{};
  int rc = check_cache(cfg, x.layer, x.keys, x.values, x.table, x.ld_table, x.n_seq, x.n_table, who, &a.c);
  if (rc || (rc = check_heads(cfg, x.n_head, who)) || (rc = check_attended(x.n_rows, x.n_head, who))) return rc;
  if (x.visible && (x.n_words < 1 || x.n_words > MAX_NODE_WORDS))
    return op_fail(SPRINTER_E_RANGE, "%s: n_words %d outside [1, %d]", who, x.n_words, MAX_NODE_WORDS);
  if (!(x.scale * 2.f - x.scale * 2.f == 0.f)) return op_fail(SPRINTER_E_CONFIG, "%s: scale is not finite, or too large", who);
  if (x.n_rows == 0 || x.n_seq == 0) return SPRINTER_OK;
  if (!x.len || !x.first || !x.q || !x.y) return op_fail(SPRINTER_E_NULL, "%s: NULL array", who);
  const int w = x.n_head * cfg->d_head;
  const size_t es = element(cfg->dtype);
  if (x.n_rows > 1 && (x.ld_q < w || x.ld_y < w)) return op_fail(SPRINTER_E_RANGE, "%s: rows lie closer than their %d columns", who, w);
  if (!aligned(x.q, 16) || !aligned(x.y, 16) || (x.n_rows > 1 && ((x.ld_q * es) % 16 || (x.ld_y * es) % 16)))
    return op_fail(SPRINTER_E_RANGE, "%s: rows are not 16-byte aligned", who);
  if (!aligned(x.len, 4) || !aligned(x.first, 4) || !aligned(x.visible, 8))
    return op_fail(SPRINTER_E_RANGE, "%s: an array is not aligned to its elements", who);
  a.type = cfg->dtype == SPRINTER_F32 ? X_F32 : X_BF16;
  const size_t need = attend_workspace(a.type, cfg->d_head, x.n_head, cfg->n_kv_head, x.n_seq, x.n_rows, (long long)x.n_table * cfg->page_size);
  if (need && !x.workspace) return op_fail(SPRINTER_E_NULL, "%s: NULL workspace", who);
  if (!aligned(x.workspace, 256)) return op_fail(SPRINTER_E_WORKSPACE, "%s: workspace is not 256-byte aligned", who);
  if (x.workspace_bytes < need)
    return op_fail(SPRINTER_E_WORKSPACE, "%s: workspace has %zu bytes, %zu needed", who, (size_t)x.workspace_bytes, need);
  a.H = x.n_head; a.T = x.n_rows; a.n_words = x.n_words; a.scale = base2(x.scale); a.lens = x.len; a.first = x.first;
  a.visible = (const unsigned long long*)x.visible; a.q = x.q; a.ld_q = x.ld_q; a.y = x.y; a.ld_y = x.ld_y;
  launching();
  launch_cache_attend(a, x.workspace, (hipStream_t)hip_stream);
  return launched(who);
}

int sprinter_cache_keep(const sprinter_cache_cfg* cfg, const sprinter_keep* args, void* hip_stream) {
  const char* who = "sprinter_cache_keep";
  if (!args) return op_fail(SPRINTER_E_NULL, "%s: NULL arguments", who);
  const sprinter_keep& x = *args;
  KeepArgs a{};
  const int rc = check_cache(cfg, 0, x.keys, x.values, x.table, x.ld_table, x.n_seq, x.n_table, who, &a.c);
  if (rc) return rc;
  if (x.n_path < 0) return op_fail(SPRINTER_E_RANGE, "%s: a path of %d", who, x.n_path);
  if (x.n_seq == 0 || x.n_path == 0) return SPRINTER_OK;
  if (!x.len || !x.first || !x.path || !x.n_keep) return op_fail(SPRINTER_E_NULL, "%s: NULL array", who);
  if (x.n_seq > 1 && x.ld_path < x.n_path) return op_fail(SPRINTER_E_RANGE, "%s: rows %lld apart hold no path of %d", who, (long long)x.ld_path, x.n_path);
  if (!aligned(x.len, 4) || !aligned(x.first, 4) || !aligned(x.path, 4) || !aligned(x.n_keep, 4))
    return op_fail(SPRINTER_E_RANGE, "%s: an array is not aligned to its elements", who);
  a.n_layer = cfg->n_layer;
  a.element = (int)element(cfg->dtype);
  a.layer_bytes = (long long)cfg->n_page * cfg->n_kv_head * cfg->page_size * cfg->d_head * a.element;
  a.lens = x.len; a.first = x.first; a.path = x.path; a.ld_path = x.ld_path; a.n_path = x.n_path; a.n_keep = x.n_keep;
  launching();
  launch_cache_keep(a, (hipStream_t)hip_stream);
  return launched(who);
}

int sprinter_adjust_logits(const sprinter_logits* args, void* hip_stream) {
  const char* who = "sprinter_adjust_logits";
  if (!args) return op_fail(SPRINTER_E_NULL, "%s: NULL arguments", who);
  const sprinter_logits& a = *args;
  if (a.dtype != SPRINTER_F32 && a.dtype != SPRINTER_BF16) return op_fail(SPRINTER_E_CONFIG, "%s: unknown dtype %d", who, a.dtype);
  if (a.vocab < 1 || a.vocab > 1 << 24) return op_fail(SPRINTER_E_CONFIG, "%s: vocab %d outside [1, 2^24]", who, a.vocab);
  int rc = check_tree_rows(a.n_rows, who);
  if (rc) return rc;
  if (a.n_seq < 0 || a.n_seq > MAX_TREE_ROWS) return op_fail(SPRINTER_E_RANGE, "%s: %d sequences are not in [0, %d]", who, a.n_seq, MAX_TREE_ROWS);
  if (a.n_tokens < 0 || a.n_tokens > MAX_HISTORY) return op_fail(SPRINTER_E_RANGE, "%s: n_tokens %d outside [0, 2^19]", who, a.n_tokens);
  if (a.draft && a.n_rows > MAX_HISTORY) return op_fail(SPRINTER_E_RANGE, "%s: %d rows with draft are more than 2^19", who, a.n_rows);
  if (a.draft && a.n_rows == MAX_HISTORY && a.n_tokens == MAX_HISTORY)   // (a token's count is below 2^20)
    return op_fail(SPRINTER_E_RANGE, "%s: n_tokens and rows with draft are 2^20 together", who);
  if (a.visible && (a.n_words < 1 || a.n_words > MAX_NODE_WORDS))
    return op_fail(SPRINTER_E_RANGE, "%s: n_words %d outside [1, %d]", who, a.n_words, MAX_NODE_WORDS);
  if (a.n_bias < 0 || a.n_bias > MAX_BIASES) return op_fail(SPRINTER_E_RANGE, "%s: n_bias %d outside [0, %d]", who, a.n_bias, MAX_BIASES);
  if (a.n_mask < 0) return op_fail(SPRINTER_E_RANGE, "%s: %d masks", who, a.n_mask);
  if (a.n_rows == 0) return SPRINTER_OK;
  if (!a.logits || !a.out) return op_fail(SPRINTER_E_NULL, "%s: NULL logits or out", who);
  if (!a.bias != !a.bias_ids) return op_fail(SPRINTER_E_NULL, "%s: bias and bias_ids come together", who);
  if (!a.tokens && (a.n_token || a.n_prompt)) return op_fail(SPRINTER_E_NULL, "%s: n_token or n_prompt without tokens", who);
  if (!a.mask && a.mask_row) return op_fail(SPRINTER_E_NULL, "%s: mask_row without mask", who);
  const bool of_sequences = a.tokens || a.draft || a.bias || a.repetition || a.presence || a.frequency;
  if (!a.first && of_sequences && a.n_rows > a.n_seq)
    return op_fail(SPRINTER_E_RANGE, "%s: %d rows without first are more than %d sequences", who, a.n_rows, a.n_seq);
  if (a.mask && !a.mask_row && a.n_rows > a.n_mask)
    return op_fail(SPRINTER_E_RANGE, "%s: %d rows without mask_row are more than %d masks", who, a.n_rows, a.n_mask);
  const int words = (a.vocab + 31) / 32;
  if (a.n_rows > 1 && (a.ld_logits < a.vocab || a.ld_out < a.vocab)) return op_fail(SPRINTER_E_RANGE, "%s: rows lie closer than their %d columns", who, a.vocab);
  if ((a.tokens && a.n_seq > 1 && a.ld_tokens < a.n_tokens) || (a.bias && a.n_seq > 1 && (a.ld_bias < a.n_bias || a.ld_bias_ids < a.n_bias)) ||
      (a.mask && a.n_mask > 1 && a.ld_mask < words))
    return op_fail(SPRINTER_E_RANGE, "%s: rows of tokens, biases or masks lie closer than their columns", who);
  const size_t es = element(a.dtype);
  if (!aligned(a.logits, es) || !aligned(a.out, es) || !aligned(a.first, 4) || !aligned(a.tokens, 4) || !aligned(a.n_token, 4) || !aligned(a.n_prompt, 4) ||
      !aligned(a.repetition, 4) || !aligned(a.presence, 4) || !aligned(a.frequency, 4) || !aligned(a.draft, 4) || !aligned(a.visible, 8) ||
      !aligned(a.bias_ids, 4) || !aligned(a.bias, 4) || !aligned(a.mask, 4) || !aligned(a.mask_row, 4))
    return op_fail(SPRINTER_E_RANGE, "%s: an array is not aligned to its elements", who);
  launching();
  launch_adjust_logits(a, (hipStream_t)hip_stream);
  return launched(who);
}

}  // extern "C"
