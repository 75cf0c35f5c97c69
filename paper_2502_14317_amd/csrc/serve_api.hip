// C ABI of the serving operators over shared prefixes: argument validation and dispatch.  Every host-visible argument
// is checked before any GPU work is enqueued.
#include "serve.h"
#include <math.h>

static const int kMost = 1 << 20;

static int check_rope(const int32_t* pos, float base) {
  return pos && (!(base > 1.0f) || !isfinite(base)) ? PC_ERR_SHAPE : PC_OK;
}
static int check_heads(int n_q_heads, int n_kv_heads, int head_dim) {
  if (n_kv_heads < 1 || n_q_heads < 1 || n_q_heads > kMost || n_q_heads % n_kv_heads != 0) return PC_ERR_SHAPE;
  return head_dim == 64 || head_dim == 128 ? PC_OK : PC_ERR_SHAPE;
}

// Sizes of a shared-prefix call.  The kernels number workgroups, rows and (segment, head) pairs with 32-bit integers.
static int check_shared_sizes(const pc_row_cache* prefix, const pc_row_cache* tail, int batch, int n_prefix, int n_q,
                              int n_q_heads, int n_kv_heads, int head_dim, PcSharedCall& c, PcSharedPlan& plan) {
  if (batch < 1 || n_prefix < 1 || n_q < 1 || batch > kMost || n_q > kMost || batch % n_prefix != 0) return PC_ERR_SHAPE;
  const int rc = check_heads(n_q_heads, n_kv_heads, head_dim);
  if (rc != PC_OK) return rc;
  if ((long long)batch * n_q > (1LL << 25) || (long long)batch * n_q * n_q_heads >= (1LL << 25)) return PC_ERR_SHAPE;
  c = {};
  const pc_row_cache* rows[2] = {prefix, tail};
  for (int i = 0; i < 2; ++i) {
    const pc_row_cache* r = rows[i];
    if (!r) continue;
    if (r->n_seg < 0 || r->n_seg > (i ? 1 : kMost) || r->cap < 1 || r->cap > (1 << 24)) return PC_ERR_SHAPE;
    if (r->seg_len_per_head != 0 && r->seg_len_per_head != 1) return PC_ERR_SHAPE;
    if ((long long)(i ? batch : n_prefix) * r->n_seg * n_kv_heads > 0x7fffffffLL / 64) return PC_ERR_SHAPE;
    if (r->n_seg == 0) continue;         // nothing there: as if it were not given, its pointers are nobody's
    PcRows& to = i ? c.tail : c.prefix;
    to.k = r->k; to.v = r->v; to.k_scale = r->k_scale; to.v_scale = r->v_scale; to.len = r->seg_len;
    to.len_per_head = r->seg_len_per_head; to.n_seg = r->n_seg; to.cap = r->cap;
  }
  // 32-key blocks of a KV head's prefix, numbered with 32 bits
  if ((long long)c.prefix.n_seg * ((c.prefix.cap + 31) / 32) > 0x7fffffffLL) return PC_ERR_SHAPE;
  c.batch = batch; c.n_prefix = n_prefix; c.n_q = n_q; c.n_q_heads = n_q_heads; c.n_kv_heads = n_kv_heads;
  c.head_dim = head_dim;
  plan = pc_shared_plan(c);
  return pc_shared_fits(c, plan) ? PC_OK : PC_ERR_SHAPE;
}

extern "C" size_t pc_shared_attn_workspace_bytes(const pc_row_cache* prefix, const pc_row_cache* tail, int32_t batch,
                                                 int32_t n_prefix, int32_t n_q, int32_t n_q_heads, int32_t n_kv_heads,
                                                 int32_t head_dim) {
  PcSharedCall c;
  PcSharedPlan plan;
  if (check_shared_sizes(prefix, tail, batch, n_prefix, n_q, n_q_heads, n_kv_heads, head_dim, c, plan) != PC_OK) return 0;
  return pc_shared_ws_bytes(c, plan);
}

extern "C" int pc_shared_attn_plan(const pc_row_cache* prefix, const pc_row_cache* tail, int32_t batch, int32_t n_prefix,
                                   int32_t n_q, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                   pc_shared_attn_plan_info* plan_info) {
  PcSharedCall c;
  PcSharedPlan plan;
  const int rc = check_shared_sizes(prefix, tail, batch, n_prefix, n_q, n_q_heads, n_kv_heads, head_dim, c, plan);
  if (rc != PC_OK) return rc;
  if (!plan_info) return PC_ERR_NULL;
  pc_shared_plan_info(c, plan, *plan_info);
  return PC_OK;
}

extern "C" int pc_shared_attn(const void* q, const int32_t* q_pos, int32_t pos0, float rope_base, float softmax_scale,
                              const pc_row_cache* prefix, const pc_row_cache* tail, int32_t tail_own, int32_t batch,
                              int32_t n_prefix, int32_t n_q, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                              void* out, float* lse_out, void* ws, size_t ws_bytes, void* stream) {
  PcSharedCall c;
  PcSharedPlan plan;
  int rc = check_shared_sizes(prefix, tail, batch, n_prefix, n_q, n_q_heads, n_kv_heads, head_dim, c, plan);
  if (rc != PC_OK) return rc;
  if (!q || !out) return PC_ERR_NULL;
  for (const PcRows* r : {&c.prefix, &c.tail}) {
    if (r->n_seg == 0) continue;
    if (!r->k || !r->v || (r->k_scale == nullptr) != (r->v_scale == nullptr)) return PC_ERR_NULL;
    if (!pc_aligned(r->k, 16) || !pc_aligned(r->v, 16) || !pc_aligned(r->k_scale, 4) || !pc_aligned(r->v_scale, 4) ||
        !pc_aligned(r->len, 4))
      return PC_ERR_SHAPE;
  }
  if (c.prefix.n_seg + c.tail.n_seg == 0) return PC_ERR_SHAPE;
  if (tail_own != 0 && tail_own != 1) return PC_ERR_SHAPE;
  if (tail_own && c.tail.n_seg == 0) return PC_ERR_SHAPE;
  if (!(softmax_scale >= 0.0f) || !isfinite(softmax_scale)) return PC_ERR_SHAPE;
  if ((rc = check_rope(q_pos, rope_base)) != PC_OK) return rc;
  if (!pc_aligned(q, 16) || !pc_aligned(out, 16) || !pc_aligned(q_pos, 4) || !pc_aligned(lse_out, 4)) return PC_ERR_SHAPE;
  if (!ws || !pc_aligned(ws, 256) || ws_bytes < pc_shared_ws_bytes(c, plan)) return PC_ERR_WORKSPACE;
  c.q = q; c.q_pos = q_pos; c.pos0 = pos0; c.rope_base = rope_base;
  c.scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)head_dim);
  c.tail_own = tail_own; c.out = out; c.lse = lse_out;
  return pc_launch_shared_attn(c, plan, ws, (hipStream_t)stream);
}

static int check_row8(int batch, int cap, int n_kv_heads, int head_dim) {
  if (batch < 0 || cap < 1 || cap > (1 << 24) || n_kv_heads < 1) return PC_ERR_SHAPE;
  if (head_dim != 64 && head_dim != 128) return PC_ERR_SHAPE;
  return (long long)batch * n_kv_heads > 0x7fffffffLL ? PC_ERR_SHAPE : PC_OK;
}

extern "C" int pc_kv_append_row8(const void* k_new, const void* v_new, const int32_t* pos, int32_t pos0, float rope_base, int32_t batch,
                                 int32_t n_new, int32_t cap, int32_t n_kv_heads, int32_t head_dim, void* k8, void* v8,
                                 float* k_scale, float* v_scale, const int32_t* len_in, int32_t* len_out, void* stream) {
  int rc = check_row8(batch, cap, n_kv_heads, head_dim);
  if (rc != PC_OK) return rc;
  // rows are numbered with 31 bits (check_row8 has bounded the first product)
  if (n_new < 0 || (long long)batch * n_kv_heads * n_new > 0x7fffffffLL) return PC_ERR_SHAPE;
  if ((rc = check_rope(pos, rope_base)) != PC_OK) return rc;
  if (batch == 0) return PC_OK;
  if (n_new > 0 && (!k_new || !v_new || !k8 || !v8 || !k_scale || !v_scale)) return PC_ERR_NULL;
  if (len_in && len_in == len_out) return PC_ERR_SHAPE;
  if (!pc_aligned(k_new, 16) || !pc_aligned(v_new, 16) || !pc_aligned(k8, 16) || !pc_aligned(v8, 16) ||
      !pc_aligned(k_scale, 4) || !pc_aligned(v_scale, 4) || !pc_aligned(pos, 4) || !pc_aligned(len_in, 4) ||
      !pc_aligned(len_out, 4))
    return PC_ERR_SHAPE;
  if (n_new == 0 && !len_out) return PC_OK;
  return pc_launch_append_row8(k_new, v_new, pos, pos0, rope_base, batch, n_new, cap, n_kv_heads, head_dim, k8, v8, k_scale,
                               v_scale, len_in, len_out, (hipStream_t)stream);
}

extern "C" int pc_kv_read_row8(const void* k8, const void* v8, const float* k_scale, const float* v_scale,
                               const int32_t* seg_len, int32_t batch, int32_t cap, int32_t n_kv_heads, int32_t head_dim,
                               void* k, void* v, void* stream) {
  const int rc = check_row8(batch, cap, n_kv_heads, head_dim);
  if (rc != PC_OK) return rc;
  if ((long long)batch * n_kv_heads * cap > 0x7fffffffLL) return PC_ERR_SHAPE;
  if (batch == 0) return PC_OK;
  if (!k8 || !v8 || !k_scale || !v_scale || !k || !v) return PC_ERR_NULL;
  if (!pc_aligned(k8, 16) || !pc_aligned(v8, 16) || !pc_aligned(k, 16) || !pc_aligned(v, 16) || !pc_aligned(k_scale, 4) ||
      !pc_aligned(v_scale, 4) || !pc_aligned(seg_len, 4))
    return PC_ERR_SHAPE;
  return pc_launch_read_row8(k8, v8, k_scale, v_scale, seg_len, batch, cap, n_kv_heads, head_dim, k, v, (hipStream_t)stream);
}

static int check_verify(int batch, int n_draft, int vocab) {
  if (batch < 1 || n_draft < 0 || vocab < 1 || batch > kMost || n_draft > kMost || vocab > (1 << 24)) return PC_ERR_SHAPE;
  return (long long)batch * (n_draft + 1) > 0x7fffffffLL ? PC_ERR_SHAPE : PC_OK;
}

extern "C" size_t pc_verify_drafts_workspace_bytes(int32_t batch, int32_t n_draft, int32_t vocab) {
  return check_verify(batch, n_draft, vocab) == PC_OK ? pc_verify_ws_bytes(batch, vocab) : 0;
}

extern "C" int pc_verify_drafts(const int32_t* draft, const int32_t* draft_len, const float* draft_prob,
                                const float* target_prob, const float* u, const float* noise, int32_t batch,
                                int32_t n_draft, int32_t vocab, int32_t* tokens, int32_t* n_accepted,
                                const int32_t* len_in, int32_t* len_out, void* ws, size_t ws_bytes, void* stream) {
  const int rc = check_verify(batch, n_draft, vocab);
  if (rc != PC_OK) return rc;
  if (!target_prob || !noise || !tokens || !n_accepted || (n_draft > 0 && (!draft || !u))) return PC_ERR_NULL;
  if ((len_in == nullptr) != (len_out == nullptr)) return PC_ERR_NULL;
  for (const void* p : {(const void*)draft, (const void*)draft_len, (const void*)draft_prob, (const void*)target_prob,
                        (const void*)u, (const void*)noise, (const void*)tokens, (const void*)n_accepted,
                        (const void*)len_in, (const void*)len_out})
    if (!pc_aligned(p, 4)) return PC_ERR_SHAPE;
  if (!ws || !pc_aligned(ws, 256) || ws_bytes < pc_verify_ws_bytes(batch, vocab)) return PC_ERR_WORKSPACE;
  PcVerifyCall c;
  c.draft = draft; c.draft_prob = draft_prob; c.target_prob = target_prob; c.u = u; c.noise = noise;
  c.draft_len = draft_len; c.batch = batch; c.n_draft = n_draft; c.vocab = vocab; c.tokens = tokens; c.count = n_accepted;
  c.len_in = len_in; c.len_out = len_out;
  return pc_launch_verify(c, ws, (hipStream_t)stream);
}
