// C ABI of the drafted trees over a paged cache and of the tokens' log probabilities: argument validation and dispatch.
// Every host-visible argument is checked before any GPU work is enqueued.
#include "paged.h"

static const int kMost = 1 << 20;

static int check_heads(int n_q_heads, int n_kv_heads, int head_dim) {
  if (n_kv_heads < 1 || n_q_heads < 1 || n_q_heads > kMost || n_q_heads % n_kv_heads != 0) return PC_ERR_SHAPE;
  return head_dim == 64 || head_dim == 128 ? PC_OK : PC_ERR_SHAPE;
}
static int check_rope(const int32_t* pos, float base) {
  return pos && (!(base > 1.0f) || !isfinite(base)) ? PC_ERR_SHAPE : PC_OK;
}
// Do na 32-bit values at a and nb at b share memory?  (Every workgroup reads lengths and trees that one of them would write over.)
static bool overlap(const int32_t* a, long long na, const int32_t* b, long long nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return a && b && (x < y ? y - x < (uintptr_t)na * 4 : x - y < (uintptr_t)nb * 4);
}
// Strides in elements of rows of whole 16-byte pieces
static bool strides_fit(int64_t a, int64_t b, int64_t c) {
  const int64_t most = (int64_t)1 << 40;
  for (int64_t s : {a, b, c})
    if (s < 0 || s > most || s % 8 != 0) return false;
  return true;
}
static int check_page_sizes(const pc_page_cache* c, PcPages& p) {
  if (!c) return PC_ERR_NULL;
  if (c->page < 16 || c->page > 65536 || (c->page & (c->page - 1)) != 0) return PC_ERR_SHAPE;
  if (c->n_pages < 1 || c->max_pages < 1 || (long long)c->max_pages * c->page > (1LL << 30)) return PC_ERR_SHAPE;
  p.k = c->k; p.v = c->v; p.k_scale = c->k_scale; p.v_scale = c->v_scale; p.table = c->table;
  p.n_pages = c->n_pages; p.max_pages = c->max_pages; p.shift = 0;
  while ((1 << p.shift) < c->page) ++p.shift;
  return PC_OK;
}
static int check_page_memory(const PcPages& p, int n_kv_heads) {
  if (!p.k || !p.v || !p.table || (p.k_scale == nullptr) != (p.v_scale == nullptr)) return PC_ERR_NULL;
  if (!pc_aligned(p.k, 16) || !pc_aligned(p.v, 16) || !pc_aligned(p.k_scale, 4) || !pc_aligned(p.v_scale, 4) || !pc_aligned(p.table, 4))
    return PC_ERR_SHAPE;
  return n_kv_heads > 65536 ? PC_ERR_SHAPE : PC_OK;      // (rows of the pool, numbered with 63 bits)
}

extern "C" int pc_kv_append_paged(const void* k_new, const void* v_new, int64_t batch_stride, int64_t row_stride, int64_t head_stride,
                                  const int32_t* parent, const int32_t* n_rows, const int32_t* pos, int32_t pos0, float rope_base,
                                  int32_t batch, int32_t n_new, int32_t n_kv_heads, int32_t head_dim, const pc_page_cache* cache,
                                  const int32_t* len_in, int32_t* len_out, void* stream) {
  PcPagedAppend c;
  int rc = check_page_sizes(cache, c.pages);
  if (rc != PC_OK) return rc;
  if (batch < 0 || batch > kMost || n_new < 0 || (rc = check_heads(n_kv_heads, n_kv_heads, head_dim)) != PC_OK) return PC_ERR_SHAPE;
  if ((long long)batch * n_kv_heads > 0x7fffffffLL || (long long)batch * n_kv_heads * n_new > 0x7fffffffLL) return PC_ERR_SHAPE;
  if (parent && n_new > PC_TREE_NODES) return PC_ERR_SHAPE;
  if (!strides_fit(batch_stride, row_stride, head_stride)) return PC_ERR_SHAPE;
  if ((rc = check_rope(pos, rope_base)) != PC_OK) return rc;
  if (batch == 0) return PC_OK;
  if (n_new > 0) {
    if (!k_new || !v_new) return PC_ERR_NULL;
    if ((rc = check_page_memory(c.pages, n_kv_heads)) != PC_OK) return rc;
  }
  if (overlap(len_out, batch, len_in, batch)) return PC_ERR_SHAPE;
  if (n_new > 0 && (overlap(len_out, batch, n_rows, batch) || overlap(len_out, batch, pos, batch) ||
                    overlap(len_out, batch, parent, (long long)batch * n_new)))
    return PC_ERR_SHAPE;
  if (!pc_aligned(k_new, 16) || !pc_aligned(v_new, 16)) return PC_ERR_SHAPE;
  for (const void* p : {(const void*)parent, (const void*)n_rows, (const void*)pos, (const void*)len_in, (const void*)len_out})
    if (!pc_aligned(p, 4)) return PC_ERR_SHAPE;
  if (n_new == 0 && !len_out) return PC_OK;
  c.k_new = (const uint16_t*)k_new; c.v_new = (const uint16_t*)v_new;
  c.batch_stride = batch_stride; c.row_stride = row_stride; c.head_stride = head_stride;
  if (batch_stride == 0 && row_stride == 0 && head_stride == 0) {
    c.head_stride = head_dim; c.row_stride = (long long)n_kv_heads * head_dim; c.batch_stride = c.row_stride * n_new;
  }
  c.parent = parent; c.n_rows = n_rows; c.pos = pos; c.pos0 = pos0; c.rope_base = rope_base;
  c.batch = batch; c.n_new = n_new; c.n_kv_heads = n_kv_heads; c.head_dim = head_dim; c.len_in = len_in; c.len_out = len_out;
  return pc_launch_append_paged(c, (hipStream_t)stream);
}

// Sizes of a tree attention.  The kernels number workgroups and rows with 32-bit integers.
static int check_tree_sizes(const pc_page_cache* cache, int batch, int n, int n_q_heads, int n_kv_heads, int head_dim, PcTreeCall& c,
                            PcTreePlan& plan) {
  c = {};
  int rc = check_page_sizes(cache, c.pages);
  if (rc != PC_OK) return rc;
  if (batch < 1 || batch > kMost || n < 1 || n > PC_TREE_NODES) return PC_ERR_SHAPE;
  if ((rc = check_heads(n_q_heads, n_kv_heads, head_dim)) != PC_OK) return rc;
  if (n_kv_heads > 65536 || (long long)batch * n * n_q_heads >= (1LL << 25)) return PC_ERR_SHAPE;
  c.batch = batch; c.n = n; c.n_q_heads = n_q_heads; c.n_kv_heads = n_kv_heads; c.head_dim = head_dim;
  plan = pc_tree_plan(c);
  return pc_tree_fits(c, plan) ? PC_OK : PC_ERR_SHAPE;
}

extern "C" size_t pc_tree_attn_workspace_bytes(const pc_page_cache* cache, int32_t batch, int32_t n, int32_t n_q_heads,
                                               int32_t n_kv_heads, int32_t head_dim) {
  PcTreeCall c;
  PcTreePlan plan;
  if (check_tree_sizes(cache, batch, n, n_q_heads, n_kv_heads, head_dim, c, plan) != PC_OK) return 0;
  return pc_tree_ws_bytes(c, plan);
}

extern "C" int pc_tree_attn(const void* q, int64_t batch_stride, int64_t row_stride, const int32_t* parent, const int32_t* n_rows,
                            const int32_t* pos, int32_t pos0, float rope_base, float softmax_scale, const pc_page_cache* cache,
                            const int32_t* len, int32_t batch, int32_t n, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                            void* out, float* lse_out, void* ws, size_t ws_bytes, void* stream) {
  PcTreeCall c;
  PcTreePlan plan;
  int rc = check_tree_sizes(cache, batch, n, n_q_heads, n_kv_heads, head_dim, c, plan);
  if (rc != PC_OK) return rc;
  if (!q || !out || !len) return PC_ERR_NULL;
  if ((rc = check_page_memory(c.pages, n_kv_heads)) != PC_OK) return rc;
  if (!strides_fit(batch_stride, row_stride, 0)) return PC_ERR_SHAPE;
  if (!(softmax_scale >= 0.0f) || !isfinite(softmax_scale)) return PC_ERR_SHAPE;
  if ((rc = check_rope(pos, rope_base)) != PC_OK) return rc;
  if (!pc_aligned(q, 16) || !pc_aligned(out, 16)) return PC_ERR_SHAPE;
  for (const void* p : {(const void*)parent, (const void*)n_rows, (const void*)pos, (const void*)len, (const void*)lse_out})
    if (!pc_aligned(p, 4)) return PC_ERR_SHAPE;
  if (!ws || !pc_aligned(ws, 256) || ws_bytes < pc_tree_ws_bytes(c, plan)) return PC_ERR_WORKSPACE;
  c.q = (const uint16_t*)q; c.batch_stride = batch_stride; c.row_stride = row_stride;
  if (batch_stride == 0 && row_stride == 0) {
    c.row_stride = (long long)n_q_heads * head_dim; c.batch_stride = c.row_stride * n;
  }
  c.parent = parent; c.n_rows = n_rows; c.pos = pos; c.pos0 = pos0; c.rope_base = rope_base;
  c.scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)head_dim);
  c.len = len; c.out = (uint16_t*)out; c.lse = lse_out;
  return pc_launch_tree_attn(c, plan, ws, (hipStream_t)stream);
}

static int check_logprobs(int rows, int vocab, int n_top) {
  if (rows < 0 || rows > (1 << 21) || vocab < 1 || vocab > (1 << 24)) return PC_ERR_SHAPE;
  return n_top < 0 || n_top > PC_TOP_MOST || n_top > vocab ? PC_ERR_SHAPE : PC_OK;
}

extern "C" size_t pc_token_logprobs_workspace_bytes(int32_t rows, int32_t vocab, int32_t n_top) {
  return check_logprobs(rows, vocab, n_top) == PC_OK ? pc_logprobs_ws_bytes(rows, vocab, n_top) : 0;
}

extern "C" int pc_token_logprobs(const void* logits, int32_t logits_fp32, int64_t row_stride, const int32_t* tokens, int32_t n_tokens,
                                 int32_t n_top, int32_t rows, int32_t vocab, float* token_logprob, float* entropy, int32_t* top_idx,
                                 float* top_logprob, void* ws, size_t ws_bytes, void* stream) {
  const int rc = check_logprobs(rows, vocab, n_top);
  if (rc != PC_OK) return rc;
  if ((logits_fp32 != 0 && logits_fp32 != 1) || n_tokens < 0 || n_tokens > 65536) return PC_ERR_SHAPE;
  if (row_stride != 0 && (row_stride < vocab || row_stride > ((int64_t)1 << 40))) return PC_ERR_SHAPE;
  if (rows == 0) return PC_OK;
  if (!logits || (n_tokens > 0 && (!tokens || !token_logprob)) || (n_top > 0 && !top_idx)) return PC_ERR_NULL;
  if (n_tokens == 0 && n_top == 0 && !entropy) return PC_ERR_NULL;
  if (!pc_aligned(logits, logits_fp32 ? 4 : 2)) return PC_ERR_SHAPE;
  for (const void* p : {(const void*)tokens, (const void*)token_logprob, (const void*)entropy, (const void*)top_idx, (const void*)top_logprob})
    if (!pc_aligned(p, 4)) return PC_ERR_SHAPE;
  if (!ws || !pc_aligned(ws, 256) || ws_bytes < pc_logprobs_ws_bytes(rows, vocab, n_top)) return PC_ERR_WORKSPACE;
  PcLogprobs c;
  c.logits = logits; c.fp32 = logits_fp32; c.row_stride = row_stride ? row_stride : vocab;
  c.tokens = tokens; c.n_tokens = n_tokens; c.n_top = n_top; c.rows = rows; c.vocab = vocab;
  c.token_logprob = token_logprob; c.entropy = entropy; c.top_idx = top_idx; c.top_logprob = top_logprob;
  return pc_launch_logprobs(c, ws, (hipStream_t)stream);
}

extern "C" int pc_tree_accept(const int32_t* tokens, const int32_t* parent, const int32_t* choice, int32_t choice_stride,
                              const int32_t* n_rows, int32_t batch, int32_t n, const pc_page_cache* cache, int32_t n_kv_heads,
                              int32_t head_dim, const int32_t* len_in, int32_t* len_out, int32_t* pos, int32_t* path,
                              int32_t* n_kept, int32_t* next_token, void* stream) {
  if (batch < 0 || batch > kMost || n < 1 || n > PC_TREE_NODES || choice_stride < 1) return PC_ERR_SHAPE;
  PcTreeAccept c = {};
  if (cache) {
    int rc = check_page_sizes(cache, c.pages);
    if (rc != PC_OK || (rc = check_heads(n_kv_heads, n_kv_heads, head_dim)) != PC_OK) return rc;
    if ((long long)batch * (n_kv_heads + 1) > (1LL << 23)) return PC_ERR_SHAPE;       // (workgroups of 256 threads, two KV heads each)
  }
  if (batch == 0) return PC_OK;
  if (!tokens || !choice || !path || !n_kept || !next_token) return PC_ERR_NULL;
  if (cache) {
    const int rc = check_page_memory(c.pages, n_kv_heads);
    if (rc != PC_OK) return rc;
    if (!len_in) return PC_ERR_NULL;
    if (overlap(len_in, batch, len_out, batch) || overlap(len_in, batch, pos, batch) || overlap(len_out, batch, pos, batch)) return PC_ERR_SHAPE;
    if (n > 1) {                                             // (of one node nothing moves)
      const long long nodes = (long long)batch * n, choices = (nodes - 1) * choice_stride + 1;
      for (int32_t* out : {path, n_kept, next_token, len_out, pos}) {
        const long long m = out == path ? nodes : batch;
        if (overlap(out, m, tokens, nodes) || overlap(out, m, parent, nodes) || overlap(out, m, choice, choices) || overlap(out, m, n_rows, batch) ||
            overlap(out, m, len_in, batch))
          return PC_ERR_SHAPE;
      }
    }
    c.moves = 1; c.n_kv_heads = n_kv_heads; c.head_dim = head_dim; c.len_in = len_in; c.len_out = len_out;
  }
  for (const void* p : {(const void*)tokens, (const void*)parent, (const void*)choice, (const void*)n_rows, (const void*)len_in,
                        (const void*)len_out, (const void*)pos, (const void*)path, (const void*)n_kept, (const void*)next_token})
    if (!pc_aligned(p, 4)) return PC_ERR_SHAPE;
  c.tokens = tokens; c.parent = parent; c.choice = choice; c.choice_stride = choice_stride; c.n_rows = n_rows;
  c.batch = batch; c.n = n; c.pos = pos; c.path = path; c.n_kept = n_kept; c.next_token = next_token;
  return pc_launch_tree_accept(c, (hipStream_t)stream);
}
