// Entry points of the cache in 8 bits with block scales (see include/innerq.h): argument checks and dispatch.
#include "block.h"
#include "row_checks.h"

using namespace innerq;

namespace {

int check_config(const innerq_block_config_t* c) {
  if (!c) return INNERQ_E_NULL;
  if (c->batch < 1 || c->n_q_heads < 1 || c->n_kv_heads < 1 || c->head_dim < 1) return INNERQ_E_ARG;
  if (c->n_q_heads % c->n_kv_heads != 0) return INNERQ_E_ARG;
  if ((long long)c->batch * c->n_kv_heads > 65535) return INNERQ_E_ARG;
  if (c->type != INNERQ_INT8 && c->type != INNERQ_E4M3) return INNERQ_E_ARG;
  if (c->block < 1 || c->capacity_tokens < 1 || c->capacity_tokens % kPageTokens != 0) return INNERQ_E_ARG;
  if (c->page_pool_pages < 0 || c->page_pool_pages > 0x7fffffffLL) return INNERQ_E_ARG;
  if (c->head_dim != kHeadDim || (c->block != 32 && c->block != 64) || c->capacity_tokens > kBlockMostCapacity) return INNERQ_E_UNSUPPORTED;
  return INNERQ_OK;
}

// host_count: the call uses cache->n_tokens
int check_cache(const innerq_block_config_t& c, const innerq_block_cache_t* k, bool host_count) {
  if (!k) return INNERQ_E_NULL;
  for (const void* p : {k->k_codes, k->k_scales, k->k_open, k->v_codes, k->v_scales, k->v_open}) {
    if (!p) return INNERQ_E_NULL;
    if (misaligned(p)) return INNERQ_E_ALIGN;
  }
  if (host_count && (k->n_tokens < 0 || k->n_tokens > c.capacity_tokens)) return INNERQ_E_ARG;
  if (c.page_pool_pages > 0) {
    if (!k->page_table) return INNERQ_E_NULL;
    if (reinterpret_cast<uintptr_t>(k->page_table) & 3u) return INNERQ_E_ALIGN;
  }
  return INNERQ_OK;
}

// (either may be null where a call allows it)
int check_counts(const int32_t* a, const int32_t* b) {
  return ((reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b)) & 3u) ? INNERQ_E_ALIGN : INNERQ_OK;
}

int check_call(const innerq_block_config_t* cfg, const innerq_block_cache_t* cache, bool host_count, long long rows) {
  int st = check_config(cfg);
  if (st == INNERQ_OK) st = check_cache(*cfg, cache, host_count);
  if (st != INNERQ_OK) return st;
  return rows < 0 ? INNERQ_E_ARG : INNERQ_OK;
}

BlockStore store_of(const innerq_block_config_t& c, const innerq_block_cache_t& k, const int32_t* n_dev, const int32_t* t_dev, long long t_new) {
  BlockStore s;
  s.k = {static_cast<uint8_t*>(k.k_codes), static_cast<float*>(k.k_scales), static_cast<__half*>(k.k_open)};
  s.v = {static_cast<uint8_t*>(k.v_codes), static_cast<float*>(k.v_scales), static_cast<__half*>(k.v_open)};
  s.batch = c.batch; s.n_kv_heads = c.n_kv_heads; s.block = c.block;
  s.capacity = c.capacity_tokens;
  s.n_tokens = n_dev ? 0 : (int)k.n_tokens;
  s.n_dev = n_dev;
  s.t_dev = t_dev;
  s.t_new = (int)t_new;
  s.pages.table = c.page_pool_pages > 0 ? static_cast<const int*>(k.page_table) : nullptr;
  s.pages.tiles_per_seq = (int)(c.capacity_tokens / kPageTokens);
  s.pages.pool_pages = (int)c.page_pool_pages;
  return s;
}

int append(const innerq_block_config_t& c, const innerq_block_cache_t& k, int32_t* n_dev, const int32_t* t_dev, const void* k_new,
           const innerq_strides_t* k_strides, const void* v_new, const innerq_strides_t* v_strides, int64_t t_new, void* hip_stream) {
  int st = check_rows(k_new, k_strides);
  if (st == INNERQ_OK) st = check_rows(v_new, v_strides);
  if (st != INNERQ_OK) return st;
  BlockAppendArgs a;
  a.s = store_of(c, k, n_dev, t_dev, t_new);
  a.k = rows_of(k_new, *k_strides);
  a.v = rows_of(v_new, *v_strides);
  const long long waits = n_dev ? c.block - 1 : k.n_tokens % c.block, blocks = (waits + t_new) / c.block;
  a.units = (int)(blocks < 1 ? 1 : blocks);
  return launch_block_append(a, n_dev, c.type == INNERQ_E4M3, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? INNERQ_OK : INNERQ_E_HIP;
}

int read(const innerq_block_config_t& c, const innerq_block_cache_t& k, const int32_t* n_dev, const int32_t* first_dev, int64_t first, int64_t count,
         void* k_out, const innerq_strides_t* k_strides, void* v_out, const innerq_strides_t* v_strides, void* hip_stream) {
  if (!k_out && !v_out) return INNERQ_E_NULL;
  int st = k_out ? check_rows_out(k_out, k_strides, c.batch, c.n_kv_heads, count) : INNERQ_OK;
  if (st == INNERQ_OK && v_out) st = check_rows_out(v_out, v_strides, c.batch, c.n_kv_heads, count);
  if (st != INNERQ_OK) return st;
  BlockReadArgs a;
  a.s = store_of(c, k, n_dev, nullptr, count);
  a.k = static_cast<__half*>(k_out);
  a.v = static_cast<__half*>(v_out);
  const innerq_strides_t none = {0, 0, 0}, &ks = k_out ? *k_strides : none, &vs = v_out ? *v_strides : none;
  a.k_batch = ks.batch; a.k_head = ks.head; a.k_token = ks.token;
  a.v_batch = vs.batch; a.v_head = vs.head; a.v_token = vs.token;
  a.first = (int)first;
  a.first_dev = first_dev;
  return launch_block_read(a, c.type == INNERQ_E4M3, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? INNERQ_OK : INNERQ_E_HIP;
}

// Whether the rows of such a call can be counted in 31 bits.
bool rows_fit(const innerq_block_config_t& c, long long t_new) { return t_new <= kBlockMostCapacity && t_new * c.n_q_heads * c.batch < (1LL << 31); }

// tokens: the most that a query attends to.  k_new and v_new null: cross attention.
int attention(const innerq_block_config_t& c, const innerq_block_cache_t& k, const int32_t* n_dev, const int32_t* t_dev, long long tokens, const void* k_new,
              const innerq_strides_t* k_strides, const void* v_new, const innerq_strides_t* v_strides, bool causal, const void* q,
              const innerq_strides_t* q_strides, int64_t t_new, void* out, const innerq_strides_t* out_strides, int out_is_fp32, void* workspace,
              size_t workspace_bytes, void* hip_stream) {
  if (!rows_fit(c, t_new)) return INNERQ_E_UNSUPPORTED;
  int st = causal ? check_rows(k_new, k_strides) : INNERQ_OK;
  if (st == INNERQ_OK && causal) st = check_rows(v_new, v_strides);
  if (st == INNERQ_OK) st = check_rows(q, q_strides);
  if (st == INNERQ_OK) st = check_rows_out(out, out_strides, c.batch, c.n_q_heads, t_new, out_is_fp32 ? 4 : 8);
  if (st != INNERQ_OK) return st;
  if (!workspace) return INNERQ_E_NULL;
  if (misaligned(workspace)) return INNERQ_E_ALIGN;
  if (workspace_bytes < block_workspace_bytes(c, t_new)) return INNERQ_E_WORKSPACE;
  const long long heads = (long long)c.batch * c.n_kv_heads;
  BlockAttnArgs a;
  a.s = store_of(c, k, n_dev, t_dev, t_new);
  a.k = causal ? rows_of(k_new, *k_strides) : RowView{nullptr, 0, 0, 0};
  a.v = causal ? rows_of(v_new, *v_strides) : RowView{nullptr, 0, 0, 0};
  a.q = rows_of(q, *q_strides);
  a.out = out;
  a.out_batch = out_strides->batch; a.out_head = out_strides->head; a.out_token = out_strides->token;
  a.out_is_fp32 = out_is_fp32;
  a.heads_per_kv = c.n_q_heads / c.n_kv_heads;
  a.table = nullptr;
  a.list_few = a.list_many = 0;
  a.ws = a.ws_few = reinterpret_cast<float*>(static_cast<char*>(workspace) + kBlockTableBytes);
  a.slots = a.row_blocks = a.n_splits = 0;
  a.few_slots = a.few_rows = a.few_most = 0;
  const bool e4m3 = c.type == INNERQ_E4M3;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  auto launch = [&](const BlockForm& form) { return form.rows <= kBlockFewRows ? launch_block_attention(a, e4m3, form, stream) : launch_block_rows(a, e4m3, form, stream); };
  const BlockList list = n_dev ? block_list(c, t_new, tokens) : BlockList{};
  if (list.use) {
    a.table = static_cast<int*>(workspace);
    a.few_slots = a.slots = block_list_items(list.form);
    a.few_rows = list.form.rows;
    a.few_most = list.few_most;
    a.list_few = (int)list.few;
    a.list_many = (int)list.many;
    if (list.many) {
      a.ws = reinterpret_cast<float*>(reinterpret_cast<char*>(a.ws) + (size_t)a.few_slots * block_slot_bytes(list.form.rows));
      a.slots = block_list_items(kBlockMany.form);
    }
    hipError_t e = list.many ? launch_block_list(a, e4m3, stream) : launch(list.form);
    if (e == hipSuccess) e = launch_block_merge(a, kBlockMany.form, stream);
    return e == hipSuccess ? INNERQ_OK : INNERQ_E_HIP;
  }
  // (ragged: how many tokens the sequences have is not known here)
  const bool both = n_dev && block_both_kinds(c, t_new);
  const BlockPlan plan = both ? block_plan_both(c, t_new, tokens) : block_plan(c, t_new, tokens, causal && !n_dev ? 0.5f * (float)t_new : 0.f);
  a.row_blocks = (int)plan.row_blocks;
  a.n_splits = plan.n_splits;
  a.slots = heads * plan.row_blocks * plan.n_splits;
  if (both) {
    a.few_slots = a.slots;
    a.few_rows = plan.form.rows;
    a.few_most = kBlockFew.form.rows;
  }
  hipError_t e = both ? launch_block_list(a, e4m3, stream) : launch(plan.form);
  if (e == hipSuccess && a.n_splits > 1) e = launch_block_merge(a, plan.form, stream);
  return e == hipSuccess ? INNERQ_OK : INNERQ_E_HIP;
}

}  // namespace

extern "C" {

int innerq_block_validate_config(const innerq_block_config_t* cfg) { return check_config(cfg); }

size_t innerq_block_buffer_bytes(const innerq_block_config_t* cfg, int which) {
  if (check_config(cfg) != INNERQ_OK || which < 0 || which >= INNERQ_BLOCK_BUF_COUNT) return 0;
  const size_t heads = (size_t)cfg->batch * cfg->n_kv_heads;
  const size_t tokens = cfg->page_pool_pages > 0 ? (size_t)cfg->page_pool_pages * cfg->n_kv_heads * kPageTokens : heads * (size_t)cfg->capacity_tokens;
  switch (which % 3) {
    case INNERQ_BLOCK_K_CODES: return tokens * kHeadDim;
    case INNERQ_BLOCK_K_SCALES: return tokens / (size_t)cfg->block * sizeof(float);
    default: return heads * (size_t)cfg->block * kHeadDim * sizeof(__half);
  }
}

size_t innerq_block_workspace_bytes(const innerq_block_config_t* cfg, int64_t t_new) {
  if (check_config(cfg) != INNERQ_OK || t_new < 1 || !rows_fit(*cfg, t_new)) return 0;
  return block_workspace_bytes(*cfg, t_new);
}

int innerq_block_append(const innerq_block_config_t* cfg, innerq_block_cache_t* cache, const void* k_new, const innerq_strides_t* k_strides,
                        const void* v_new, const innerq_strides_t* v_strides, int64_t t_new, void* hip_stream) {
  int st = check_call(cfg, cache, true, t_new);
  if (st != INNERQ_OK || t_new == 0) return st;
  if (t_new > cfg->capacity_tokens - cache->n_tokens) return INNERQ_E_CAPACITY;
  st = append(*cfg, *cache, nullptr, nullptr, k_new, k_strides, v_new, v_strides, t_new, hip_stream);
  if (st == INNERQ_OK) cache->n_tokens += t_new;
  return st;
}

int innerq_block_append_ragged(const innerq_block_config_t* cfg, const innerq_block_cache_t* cache, int32_t* n_tokens_dev, const int32_t* t_new_dev,
                               const void* k_new, const innerq_strides_t* k_strides, const void* v_new, const innerq_strides_t* v_strides,
                               int64_t t_new, void* hip_stream) {
  int st = check_call(cfg, cache, false, t_new);
  if (st != INNERQ_OK) return st;
  if (!n_tokens_dev) return INNERQ_E_NULL;
  st = check_counts(n_tokens_dev, t_new_dev);
  if (st != INNERQ_OK || t_new == 0) return st;
  if (t_new > cfg->capacity_tokens) return INNERQ_E_CAPACITY;
  return append(*cfg, *cache, n_tokens_dev, t_new_dev, k_new, k_strides, v_new, v_strides, t_new, hip_stream);
}

int innerq_block_read(const innerq_block_config_t* cfg, const innerq_block_cache_t* cache, int64_t first, int64_t count, void* k_out,
                      const innerq_strides_t* k_strides, void* v_out, const innerq_strides_t* v_strides, void* hip_stream) {
  const int st = check_call(cfg, cache, true, count);
  if (st != INNERQ_OK) return st;
  if (first < 0 || first > cache->n_tokens || count > cache->n_tokens - first) return INNERQ_E_ARG;
  if (count == 0) return INNERQ_OK;
  return read(*cfg, *cache, nullptr, nullptr, first, count, k_out, k_strides, v_out, v_strides, hip_stream);
}

int innerq_block_read_ragged(const innerq_block_config_t* cfg, const innerq_block_cache_t* cache, const int32_t* n_tokens_dev, const int32_t* first_dev,
                             int64_t count, void* k_out, const innerq_strides_t* k_strides, void* v_out, const innerq_strides_t* v_strides,
                             void* hip_stream) {
  int st = check_call(cfg, cache, false, count);
  if (st != INNERQ_OK) return st;
  if (!n_tokens_dev) return INNERQ_E_NULL;
  st = check_counts(n_tokens_dev, first_dev);
  if (st != INNERQ_OK || count == 0) return st;
  if (count > cfg->capacity_tokens) return INNERQ_E_CAPACITY;
  return read(*cfg, *cache, n_tokens_dev, first_dev, 0, count, k_out, k_strides, v_out, v_strides, hip_stream);
}

int innerq_block_attention(const innerq_block_config_t* cfg, const innerq_block_cache_t* cache, const void* k_new, const innerq_strides_t* k_strides,
                           const void* v_new, const innerq_strides_t* v_strides, const void* q, const innerq_strides_t* q_strides, int64_t t_new,
                           void* out, const innerq_strides_t* out_strides, int out_is_fp32, void* workspace, size_t workspace_bytes,
                           void* hip_stream) {
  const int st = check_call(cfg, cache, true, t_new);
  if (st != INNERQ_OK || t_new == 0) return st;
  if (t_new > cfg->capacity_tokens - cache->n_tokens) return INNERQ_E_CAPACITY;
  return attention(*cfg, *cache, nullptr, nullptr, cache->n_tokens + t_new, k_new, k_strides, v_new, v_strides, true, q, q_strides, t_new, out,
                   out_strides, out_is_fp32, workspace, workspace_bytes, hip_stream);
}

int innerq_block_attention_ragged(const innerq_block_config_t* cfg, const innerq_block_cache_t* cache, const int32_t* n_tokens_dev,
                                  const int32_t* t_new_dev, int64_t max_tokens, const void* k_new, const innerq_strides_t* k_strides,
                                  const void* v_new, const innerq_strides_t* v_strides, const void* q, const innerq_strides_t* q_strides,
                                  int64_t t_new, void* out, const innerq_strides_t* out_strides, int out_is_fp32, void* workspace,
                                  size_t workspace_bytes, void* hip_stream) {
  int st = check_call(cfg, cache, false, t_new);
  if (st != INNERQ_OK) return st;
  if (!n_tokens_dev) return INNERQ_E_NULL;
  st = check_counts(n_tokens_dev, t_new_dev);
  if (st != INNERQ_OK) return st;
  if (max_tokens < 1) return INNERQ_E_ARG;
  if (t_new == 0) return INNERQ_OK;
  if (max_tokens > cfg->capacity_tokens || t_new > cfg->capacity_tokens) return INNERQ_E_CAPACITY;
  return attention(*cfg, *cache, n_tokens_dev, t_new_dev, max_tokens, k_new, k_strides, v_new, v_strides, true, q, q_strides, t_new, out, out_strides,
                   out_is_fp32, workspace, workspace_bytes, hip_stream);
}

int innerq_block_cross_attention(const innerq_block_config_t* cfg, const innerq_block_cache_t* cache, const void* q, const innerq_strides_t* q_strides,
                                 int64_t t_new, void* out, const innerq_strides_t* out_strides, int out_is_fp32, void* workspace,
                                 size_t workspace_bytes, void* hip_stream) {
  const int st = check_call(cfg, cache, true, t_new);
  if (st != INNERQ_OK || t_new == 0) return st;
  return attention(*cfg, *cache, nullptr, nullptr, cache->n_tokens, nullptr, nullptr, nullptr, nullptr, false, q, q_strides, t_new, out, out_strides,
                   out_is_fp32, workspace, workspace_bytes, hip_stream);
}

int innerq_block_cross_attention_ragged(const innerq_block_config_t* cfg, const innerq_block_cache_t* cache, const int32_t* n_tokens_dev,
                                        const int32_t* t_new_dev, int64_t max_tokens, const void* q, const innerq_strides_t* q_strides, int64_t t_new,
                                        void* out, const innerq_strides_t* out_strides, int out_is_fp32, void* workspace, size_t workspace_bytes,
                                        void* hip_stream) {
  int st = check_call(cfg, cache, false, t_new);
  if (st != INNERQ_OK) return st;
  if (!n_tokens_dev) return INNERQ_E_NULL;
  st = check_counts(n_tokens_dev, t_new_dev);
  if (st != INNERQ_OK) return st;
  if (max_tokens < 0) return INNERQ_E_ARG;
  if (t_new == 0) return INNERQ_OK;
  if (max_tokens > cfg->capacity_tokens) return INNERQ_E_CAPACITY;
  return attention(*cfg, *cache, n_tokens_dev, t_new_dev, max_tokens, nullptr, nullptr, nullptr, nullptr, false, q, q_strides, t_new, out, out_strides,
                   out_is_fp32, workspace, workspace_bytes, hip_stream);
}

}  // extern "C"
