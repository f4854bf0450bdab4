// C-ABI entry points of the operators around a verification (attention over the
// paged cache and of prompts, logits processing, growth and commit of the cache, the
// cache of 4 bits; declared in include/tv.h): argument validation on the host, then the launches on the
// caller's stream. Nothing here touches the GPU before the arguments are known
// to be valid.
#include <math.h>
#include <stdint.h>

#include "tv.h"
#include "tv_launch.h"

namespace {

uintptr_t bits(const void* p) { return reinterpret_cast<uintptr_t>(p); }

bool page_size_ok(int32_t page_size) {
  return page_size >= TV_MIN_PAGE && page_size <= TV_MAX_PAGE &&
         (page_size & (page_size - 1)) == 0;
}

constexpr int64_t kMaxBytes = int64_t{1} << 29;   // of a tree's nodes, and of a page
constexpr float kMaxScale = 0x1p127f;             // its product with log2(e) is finite

// Keys of a sequence: the kernels' tiles of 32 keys, rounded up and a few further ones of idle key
// groups, end below 2^31.
constexpr int32_t kMaxKeys = INT32_MAX - 1023;

// Query rows of a call: over a prefix they are one item's, whose last team of 32 workgroups of 192
// rows ends below 2^31.
constexpr int32_t kMaxRows = INT32_MAX - 16383;

// TV_OK if an attention call of these sizes is taken
int attention_sizes(int32_t batch, int32_t num_nodes, int32_t heads, int32_t kv_heads,
                    int32_t head_dim, int32_t prefix_len) {
  if (batch < 0 || num_nodes < 1 || heads < 1 || kv_heads < 1 || head_dim < 1 || prefix_len < 0)
    return TV_ERR_INVALID_ARG;
  if (heads % kv_heads) return TV_ERR_INVALID_ARG;
  if (batch > TV_MAX_BATCH || num_nodes > TV_MAX_NODES || head_dim > TV_MAX_HEAD_DIM ||
      head_dim % 8 || static_cast<int64_t>(heads) * head_dim > TV_MAX_HIDDEN ||
      static_cast<int64_t>(batch) * num_nodes * heads > kMaxRows)
    return TV_ERR_UNSUPPORTED;
  return TV_OK;
}

// Bytes of a head of a page of 4 bits; 0 for sizes that are not taken.
int64_t fp4_page_bytes(int32_t page_size, int32_t head_dim) {
  if (!page_size_ok(page_size) || head_dim < 1 || head_dim > TV_MAX_HEAD_DIM ||
      head_dim % TV_FP4_BLOCK)
    return 0;
  return static_cast<int64_t>(page_size) * (head_dim / TV_FP4_BLOCK) * TV_FP4_BLOCK_BYTES;
}

// fp4: the cache is of 4 bits, its page_stride in bytes.
int validate(const tv::AttentionArgs& a, void* workspace, size_t workspace_bytes,
             bool fp4 = false) {
  const int st =
      attention_sizes(a.batch, a.num_nodes, a.heads, a.kv_heads, a.head_dim, a.prefix_len);
  if (st != TV_OK) return st;
  if (a.dtype != TV_DTYPE_BF16 && a.dtype != TV_DTYPE_F16) return TV_ERR_INVALID_ARG;
  if (a.num_pages < 0 || a.page_size < 1 || a.table_width < 0) return TV_ERR_INVALID_ARG;
  if (!(a.scale > 0.0f) || !isfinite(a.scale)) return TV_ERR_INVALID_ARG;
  if (!page_size_ok(a.page_size) || a.scale > kMaxScale) return TV_ERR_UNSUPPORTED;
  if (a.prefix_len % a.page_size) return TV_ERR_INVALID_ARG;
  // (so that the first keys of a context's tiles of 32, rounded up, end below 2^31)
  if (a.table_width > kMaxKeys / a.page_size) return TV_ERR_UNSUPPORTED;
  const int64_t kv_row = static_cast<int64_t>(a.kv_heads) * a.head_dim;
  if (a.q_stride < static_cast<int64_t>(a.heads) * a.head_dim || a.kv_stride < kv_row)
    return TV_ERR_INVALID_ARG;
  const int64_t head = fp4 ? fp4_page_bytes(a.page_size, a.head_dim) : 0;
  if (fp4 && !head) return TV_ERR_UNSUPPORTED;
  if (a.num_pages > 0 && a.page_stride < (fp4 ? a.kv_heads * head : kv_row * a.page_size))
    return TV_ERR_INVALID_ARG;
  if (a.q_stride % 8 || a.kv_stride % 8 || a.page_stride % (fp4 ? 16 : 8)) return TV_ERR_UNSUPPORTED;
  if (a.q_stride > kMaxBytes / 2 / a.num_nodes || a.kv_stride > kMaxBytes / 2 / a.num_nodes ||
      a.page_stride > (fp4 ? kMaxBytes : kMaxBytes / 2))
    return TV_ERR_UNSUPPORTED;
  if (a.batch == 0) return TV_OK;
  if (!a.q || !a.k_new || !a.v_new || !a.ctx_len || !a.out || (a.num_nodes > 1 && !a.parents))
    return TV_ERR_INVALID_ARG;
  if (a.num_pages > 0 && (!a.k_cache || !a.v_cache)) return TV_ERR_INVALID_ARG;
  if ((a.table_width > 0 && !a.block_table) || (a.prefix_len > 0 && !a.prefix_pages))
    return TV_ERR_INVALID_ARG;
  for (const void* p : {a.q, a.k_new, a.v_new, a.k_cache, a.v_cache, (const void*)a.out})
    if (bits(p) % 16) return TV_ERR_INVALID_ARG;
  for (const int32_t* p : {a.parents, a.block_table, a.ctx_len, a.prefix_pages})
    if (bits(p) % 4) return TV_ERR_INVALID_ARG;
  if (!workspace || bits(workspace) % 256 ||
      workspace_bytes < tv::attention_workspace(a.batch, a.num_nodes, a.heads, a.kv_heads,
                                                a.head_dim, a.prefix_len))
    return TV_ERR_WORKSPACE;
  return TV_OK;
}

int validate(const tv::LogitsArgs& a, void* workspace, size_t workspace_bytes) {
  if (a.batch < 0 || a.num_nodes < 1 || a.vocab < 2 || a.first_node < 0 || a.num_rows < 0 ||
      a.max_history < 0 || a.max_bias < 0 || a.num_masks < 0)
    return TV_ERR_INVALID_ARG;
  if (a.dtype != TV_DTYPE_BF16 && a.dtype != TV_DTYPE_F32) return TV_ERR_INVALID_ARG;
  if (!(a.temperature > 0.0f) || !isfinite(a.temperature)) return TV_ERR_INVALID_ARG;
  if (a.temperature < TV_MIN_TEMPERATURE || a.temperature > TV_MAX_TEMPERATURE)
    return TV_ERR_UNSUPPORTED;
  if (a.batch > TV_MAX_BATCH || a.num_nodes > TV_MAX_NODES || a.vocab > TV_MAX_VOCAB ||
      (a.dtype == TV_DTYPE_F32 && a.vocab > TV_MAX_VOCAB_F32) || a.max_history > TV_MAX_HISTORY ||
      a.max_bias > TV_MAX_BIAS)
    return TV_ERR_UNSUPPORTED;
  if (a.first_node > a.num_nodes || a.num_rows > a.num_nodes - a.first_node)
    return TV_ERR_INVALID_ARG;
  if (a.batch == 0 || a.num_rows == 0) return TV_OK;
  if (!a.logits || !a.out || !a.parents != !a.tokens || !a.row_max != !a.row_sum)
    return TV_ERR_INVALID_ARG;
  if (a.history && !a.history_len) return TV_ERR_INVALID_ARG;
  if (!a.bias_tokens != !a.bias_values) return TV_ERR_INVALID_ARG;
  if (a.mask_index && a.num_masks > 0 && !a.masks) return TV_ERR_INVALID_ARG;
  const size_t esize = a.dtype == TV_DTYPE_BF16 ? 2 : 4;
  if (bits(a.logits) % esize || bits(a.out) % esize || bits(a.row_sum) % 8)
    return TV_ERR_INVALID_ARG;
  const void* words[] = {a.parents,   a.tokens,    a.history,     a.history_len, a.prompt_len,
                         a.repetition, a.presence, a.frequency,   a.bias_tokens, a.bias_values,
                         a.masks,     a.mask_index, a.row_max};
  for (const void* p : words)
    if (bits(p) % 4) return TV_ERR_INVALID_ARG;
  if (a.row_max && (!workspace || bits(workspace) % 256 ||
                    workspace_bytes <
                        tv::logits_layout(a.batch, a.num_nodes, a.vocab).bytes))
    return TV_ERR_WORKSPACE;
  return TV_OK;
}

// An empty batch whose count of free pages goes to another place.
bool count_alone(const tv::ExtendArgs& a) {
  return a.batch == 0 && a.free_count && a.new_free_count && a.free_count != a.new_free_count;
}

int validate(const tv::ExtendArgs& a) {
  if (a.batch < 0 || a.max_new < 0 || a.table_width < 0 || a.page_size < 1 || a.prefix_len < 0 ||
      a.num_pages < 0)
    return TV_ERR_INVALID_ARG;
  if (a.batch > TV_MAX_BATCH || a.max_new > TV_MAX_NEW || !page_size_ok(a.page_size))
    return TV_ERR_UNSUPPORTED;
  if (a.prefix_len % a.page_size) return TV_ERR_INVALID_ARG;
  if (a.num_pages > INT32_MAX / a.page_size || a.table_width > INT32_MAX / a.page_size)
    return TV_ERR_UNSUPPORTED;
  if (a.batch == 0)
    return count_alone(a) && (bits(a.free_count) | bits(a.new_free_count)) % 4 ? TV_ERR_INVALID_ARG
                                                                               : TV_OK;
  if (!a.new_len || !a.seq_len || !a.new_seq_len || !a.free_count || !a.new_free_count ||
      !a.status || (a.max_new > 0 && !a.slots) || (a.table_width > 0 && !a.block_table) ||
      (a.num_pages > 0 && !a.free_pages))
    return TV_ERR_INVALID_ARG;
  const void* words[] = {a.new_len,    a.seq_len,    a.new_seq_len, a.block_table, a.free_pages,
                         a.free_count, a.new_free_count, a.slots,   a.status};
  for (const void* p : words)
    if (bits(p) % 4) return TV_ERR_INVALID_ARG;
  return TV_OK;
}

using Wide = __int128;
Wide magnitude(int64_t x) { return x < 0 ? -static_cast<Wide>(x) : static_cast<Wide>(x); }

// Whether blocks of `size` that begin at multiples of `step` (no less) up to `last` share bytes with
// as many that begin `at` (0 or more) further on.
bool meets(Wide at, Wide step, Wide last, Wide size) {
  // the first one of those: behind a block's end, and before the next one's start
  const Wide block = at / step * step;
  return (block <= last && at - block < size) || (block + step <= last && block + step - at < size);
}

// Whether pages of two layers share bytes: layers begin cache_layer_stride apart, and a
// layer's pages of `size` bytes page_stride (no less).
template <class Args>
bool layers_overlap(const Args& a, int64_t size) {
  const Wide apart = magnitude(a.cache_layer_stride);
  const Wide step = a.page_stride, last = (a.num_pages - 1) * step;   // the last page
  if (a.layers < 2 || apart >= last + size) return false;
  for (int l = 1; l < a.layers; ++l)
    if (meets(l * apart, step, last, size)) return true;
  return false;
}

// The same of the rows that a read writes: of two layers, or of the keys and the values.
bool outputs_overlap(const tv::Fp4ReadArgs& a) {
  const Wide apart = magnitude(a.out_layer_stride) * 2, size = Wide{a.kv_heads} * a.head_dim * 2;
  const Wide step = Wide{a.row_stride} * 2, last = (a.num_rows - 1) * step;
  const bool one = a.layers < 2 || apart >= last + size;
  for (int l = 1; l < a.layers && !one; ++l)
    if (meets(l * apart, step, last, size)) return true;
  // (both of the same cache to the same rows: the same bytes)
  if (a.k_out == a.v_out) return a.k_cache != a.v_cache;
  const Wide from = static_cast<Wide>(bits(a.v_out)) - static_cast<Wide>(bits(a.k_out));
  if ((from < 0 ? -from : from) >= (a.layers - 1) * apart + last + size) return false;
  for (int l = 1 - a.layers; l < a.layers; ++l) {
    const Wide at = from + l * apart;
    if (meets(at < 0 ? -at : at, step, last, size)) return true;
  }
  return false;
}

int validate(const tv::CacheCommitArgs& a) {
  if (a.layers < 0 || a.batch < 0 || a.num_nodes < 1 || a.kv_heads < 1 || a.head_bytes < 1 ||
      a.num_pages < 0 || a.page_size < 1 || a.max_new < 0 || a.path_width < 0)
    return TV_ERR_INVALID_ARG;
  if (a.layers > TV_MAX_LAYERS || a.batch > TV_MAX_BATCH || a.head_bytes % 16 ||
      a.head_bytes > 4096 || a.max_new > TV_MAX_NEW || a.kv_heads > TV_MAX_HIDDEN || !page_size_ok(a.page_size) ||
      a.num_pages > INT32_MAX / a.page_size)
    return TV_ERR_UNSUPPORTED;
  const int64_t row = static_cast<int64_t>(a.kv_heads) * a.head_bytes;
  if (a.node_stride < row || (a.num_pages > 0 && a.page_stride < row * a.page_size))
    return TV_ERR_INVALID_ARG;
  if (a.num_pages > 0 && layers_overlap(a, row * a.page_size)) return TV_ERR_INVALID_ARG;
  if (a.new_layer_stride % 16 || a.node_stride % 16 || a.cache_layer_stride % 16 ||
      a.page_stride % 16)
    return TV_ERR_UNSUPPORTED;
  if (a.layers == 0 || a.batch == 0 || a.max_new == 0 || a.num_pages == 0) return TV_OK;
  if (!a.k_new || !a.v_new || !a.k_cache || !a.v_cache || !a.new_len || !a.slots)
    return TV_ERR_INVALID_ARG;
  for (const void* p : {a.k_new, a.v_new, (const void*)a.k_cache, (const void*)a.v_cache})
    if (bits(p) % 16) return TV_ERR_INVALID_ARG;
  for (const int32_t* p : {a.new_len, a.slots, a.path_nodes})
    if (bits(p) % 4) return TV_ERR_INVALID_ARG;
  return TV_OK;
}

// What a commit into a cache of 4 bits and a read from it have in common; the bytes of a head of
// a page in `head`.
template <class Args>
int fp4_sizes(const Args& a, int64_t* head) {
  if (a.layers < 0 || a.batch < 0 || a.kv_heads < 1 || a.head_dim < 1 || a.num_pages < 0 ||
      a.page_size < 1)
    return TV_ERR_INVALID_ARG;
  if (a.dtype != TV_DTYPE_BF16 && a.dtype != TV_DTYPE_F16) return TV_ERR_INVALID_ARG;
  *head = fp4_page_bytes(a.page_size, a.head_dim);
  if (!*head || a.layers > TV_MAX_LAYERS || a.batch > TV_MAX_BATCH ||
      static_cast<int64_t>(a.kv_heads) * a.head_dim > TV_MAX_HIDDEN ||
      a.num_pages > INT32_MAX / a.page_size)
    return TV_ERR_UNSUPPORTED;
  if (a.num_pages > 0 && a.page_stride < a.kv_heads * *head) return TV_ERR_INVALID_ARG;
  if (a.cache_layer_stride % 16 || a.page_stride % 16) return TV_ERR_UNSUPPORTED;
  return TV_OK;
}

int validate(const tv::Fp4CommitArgs& a) {
  if (a.num_nodes < 1 || a.max_new < 0 || a.path_width < 0) return TV_ERR_INVALID_ARG;
  int64_t head = 0;
  const int st = fp4_sizes(a, &head);
  if (st != TV_OK) return st;
  if (a.max_new > TV_MAX_NEW) return TV_ERR_UNSUPPORTED;
  if (a.node_stride < static_cast<int64_t>(a.kv_heads) * a.head_dim) return TV_ERR_INVALID_ARG;
  if (a.num_pages > 0 && layers_overlap(a, a.kv_heads * head)) return TV_ERR_INVALID_ARG;
  if (a.new_layer_stride % 8 || a.node_stride % 8) return TV_ERR_UNSUPPORTED;
  if (a.layers == 0 || a.batch == 0 || a.max_new == 0 || a.num_pages == 0) return TV_OK;
  if (!a.k_new || !a.v_new || !a.k_cache || !a.v_cache || !a.new_len || !a.slots)
    return TV_ERR_INVALID_ARG;
  for (const void* p : {a.k_new, a.v_new, (const void*)a.k_cache, (const void*)a.v_cache})
    if (bits(p) % 16) return TV_ERR_INVALID_ARG;
  for (const int32_t* p : {a.new_len, a.slots, a.path_nodes})
    if (bits(p) % 4) return TV_ERR_INVALID_ARG;
  // (of keys and values to the same places either could stay)
  return a.k_cache == a.v_cache && a.k_new != a.v_new ? TV_ERR_INVALID_ARG : TV_OK;
}

int validate(const tv::Fp4ReadArgs& a) {
  if (a.table_width < 0 || a.num_rows < 0) return TV_ERR_INVALID_ARG;
  int64_t head = 0;
  const int st = fp4_sizes(a, &head);
  if (st != TV_OK) return st;
  if (a.table_width > INT32_MAX / a.page_size) return TV_ERR_UNSUPPORTED;
  if (a.row_stride < static_cast<int64_t>(a.kv_heads) * a.head_dim) return TV_ERR_INVALID_ARG;
  if (a.out_layer_stride % 8 || a.row_stride % 8) return TV_ERR_UNSUPPORTED;
  if (a.layers == 0 || a.batch == 0 || a.num_rows == 0) return TV_OK;
  if (!a.length || !a.row_start || !a.k_out || !a.v_out || (a.table_width > 0 && !a.block_table) ||
      (a.num_pages > 0 && (!a.k_cache || !a.v_cache)))
    return TV_ERR_INVALID_ARG;
  for (const void* p : {a.k_cache, a.v_cache, (const void*)a.k_out, (const void*)a.v_out})
    if (bits(p) % 16) return TV_ERR_INVALID_ARG;
  for (const int32_t* p : {a.block_table, a.first, a.length, a.row_start})
    if (bits(p) % 4) return TV_ERR_INVALID_ARG;
  return outputs_overlap(a) ? TV_ERR_INVALID_ARG : TV_OK;
}

// TV_OK if a prompt attention of these sizes is taken
int prompt_sizes(int32_t batch, int32_t num_queries, int32_t num_keys, int32_t heads,
                 int32_t kv_heads, int32_t head_dim) {
  if (batch < 0 || num_queries < 0 || num_keys < 0 || heads < 1 || kv_heads < 1 || head_dim < 1)
    return TV_ERR_INVALID_ARG;
  if (heads % kv_heads) return TV_ERR_INVALID_ARG;
  if (batch > TV_MAX_BATCH || head_dim > TV_MAX_HEAD_DIM || head_dim % 8 || num_keys > kMaxKeys ||
      static_cast<int64_t>(heads) * head_dim > TV_MAX_HIDDEN ||
      static_cast<int64_t>(num_queries) * heads >= int64_t{1} << 29 ||
      static_cast<int64_t>(batch) * kv_heads >= int64_t{1} << 22)
    return TV_ERR_UNSUPPORTED;
  return TV_OK;
}

int validate(const tv::PromptArgs& a, void* workspace, size_t workspace_bytes) {
  const int st =
      prompt_sizes(a.batch, a.num_queries, a.num_keys, a.heads, a.kv_heads, a.head_dim);
  if (st != TV_OK) return st;
  if (a.dtype != TV_DTYPE_BF16 && a.dtype != TV_DTYPE_F16) return TV_ERR_INVALID_ARG;
  if (!(a.scale > 0.0f) || !isfinite(a.scale)) return TV_ERR_INVALID_ARG;
  if (a.scale > kMaxScale) return TV_ERR_UNSUPPORTED;
  if (a.q_stride < static_cast<int64_t>(a.heads) * a.head_dim ||
      a.kv_stride < static_cast<int64_t>(a.kv_heads) * a.head_dim)
    return TV_ERR_INVALID_ARG;
  if (a.q_stride % 8 || a.kv_stride % 8 || a.kv_stride > int64_t{1} << 24) return TV_ERR_UNSUPPORTED;
  if (a.batch == 0 || a.num_queries == 0) return TV_OK;
  if (!a.q || (a.num_keys > 0 && (!a.k || !a.v)) || !a.q_start || !a.out) return TV_ERR_INVALID_ARG;
  for (const void* p : {a.q, a.k, a.v, (const void*)a.out})
    if (bits(p) % 16) return TV_ERR_INVALID_ARG;
  for (const int32_t* p : {a.q_start, a.k_start})
    if (bits(p) % 4) return TV_ERR_INVALID_ARG;
  if (!workspace || bits(workspace) % 256 ||
      workspace_bytes < tv::prompt_workspace(a.batch, a.num_queries, a.num_keys, a.heads,
                                             a.kv_heads, a.head_dim))
    return TV_ERR_WORKSPACE;
  return TV_OK;
}

}  // namespace

extern "C" {

size_t tv_tree_attention_workspace_size(int32_t batch, int32_t num_nodes, int32_t heads,
                                        int32_t kv_heads, int32_t head_dim, int32_t prefix_len) {
  if (batch < 1 ||
      attention_sizes(batch, num_nodes, heads, kv_heads, head_dim, prefix_len) != TV_OK)
    return 0;
  return tv::attention_workspace(batch, num_nodes, heads, kv_heads, head_dim, prefix_len);
}

int tv_tree_attention(int32_t batch, int32_t num_nodes, int32_t heads, int32_t kv_heads,
                      int32_t head_dim, int32_t dtype, const int32_t* parents, const void* q,
                      int64_t q_stride, const void* k_new, const void* v_new, int64_t kv_stride,
                      const void* k_cache, const void* v_cache, int64_t page_stride,
                      int32_t num_pages, int32_t page_size, const int32_t* block_table,
                      int32_t table_width, const int32_t* ctx_len, const int32_t* prefix_pages,
                      int32_t prefix_len, float scale, void* out, void* workspace,
                      size_t workspace_bytes, hipStream_t stream) {
  const tv::AttentionArgs a{batch,     num_nodes,   heads,       kv_heads,  head_dim,
                            dtype,     parents,     q,           q_stride,  k_new,
                            v_new,     kv_stride,   k_cache,     v_cache,   page_stride,
                            num_pages, page_size,   block_table, table_width, ctx_len,
                            prefix_pages, prefix_len, scale,     out};
  const int st = validate(a, workspace, workspace_bytes);
  if (st != TV_OK || batch == 0) return st;
  return tv::launch_attention(a, workspace, stream);
}

size_t tv_process_logits_workspace_size(int32_t batch, int32_t num_nodes, int32_t vocab) {
  if (batch < 1 || batch > TV_MAX_BATCH || num_nodes < 1 || num_nodes > TV_MAX_NODES ||
      vocab < 2 || vocab > TV_MAX_VOCAB)
    return 0;
  return tv::logits_layout(batch, num_nodes, vocab).bytes;
}

int tv_process_logits(int32_t batch, int32_t num_nodes, int32_t vocab, int32_t first_node,
                      int32_t num_rows, const void* logits, int32_t dtype, float temperature,
                      const int32_t* parents, const int32_t* tokens, const int32_t* history,
                      int32_t max_history, const int32_t* history_len, const int32_t* prompt_len,
                      const float* repetition, const float* presence, const float* frequency,
                      const int32_t* bias_tokens, const float* bias_values, int32_t max_bias,
                      const uint32_t* masks, int32_t num_masks, const int32_t* mask_index,
                      void* out, float* row_max, double* row_sum, void* workspace,
                      size_t workspace_bytes, hipStream_t stream) {
  const tv::LogitsArgs a{batch,       num_nodes,   vocab,       first_node, num_rows,
                         logits,      dtype,       temperature, parents,    tokens,
                         history,     max_history, history_len, prompt_len, repetition,
                         presence,    frequency,   bias_tokens, bias_values, max_bias,
                         masks,       num_masks,   mask_index,  out,        row_max,
                         row_sum};
  const int st = validate(a, workspace, workspace_bytes);
  if (st != TV_OK || batch == 0 || num_rows == 0) return st;
  return tv::launch_logits(a, workspace, stream);
}

int tv_cache_extend(int32_t batch, const int32_t* new_len, int32_t max_new,
                    const int32_t* seq_len, int32_t* new_seq_len, int32_t* block_table,
                    int32_t table_width, int32_t page_size, int32_t prefix_len,
                    int32_t* free_pages, int32_t num_pages, const int32_t* free_count,
                    int32_t* new_free_count, int32_t* slots, int32_t* status,
                    hipStream_t stream) {
  const tv::ExtendArgs a{batch,      new_len,        max_new,    seq_len, new_seq_len,
                         block_table, table_width,   page_size,  prefix_len, free_pages,
                         num_pages,  free_count,     new_free_count, slots, status};
  const int st = validate(a);
  if (st != TV_OK || (batch == 0 && !count_alone(a))) return st;
  return tv::launch_extend(a, stream);
}

int tv_cache_commit(int32_t layers, int32_t batch, int32_t num_nodes, int32_t kv_heads,
                    int32_t head_bytes, const void* k_new, const void* v_new,
                    int64_t new_layer_stride, int64_t node_stride, void* k_cache, void* v_cache,
                    int64_t cache_layer_stride, int64_t page_stride, int32_t num_pages,
                    int32_t page_size, const int32_t* new_len, int32_t max_new,
                    const int32_t* slots, const int32_t* path_nodes, int32_t path_width,
                    hipStream_t stream) {
  const tv::CacheCommitArgs a{layers,      batch,    num_nodes, kv_heads,    head_bytes,
                              k_new,       v_new,    new_layer_stride, node_stride, k_cache,
                              v_cache,     cache_layer_stride, page_stride, num_pages, page_size,
                              new_len,     max_new,  slots,     path_nodes,  path_width};
  const int st = validate(a);
  if (st != TV_OK || layers == 0 || batch == 0 || max_new == 0 || num_pages == 0) return st;
  return tv::launch_cache_commit(a, stream);
}

size_t tv_prompt_attention_workspace_size(int32_t batch, int32_t num_queries, int32_t num_keys,
                                          int32_t heads, int32_t kv_heads, int32_t head_dim) {
  if (batch < 1 || num_queries < 1 ||
      prompt_sizes(batch, num_queries, num_keys, heads, kv_heads, head_dim) != TV_OK)
    return 0;
  return tv::prompt_workspace(batch, num_queries, num_keys, heads, kv_heads, head_dim);
}

int tv_prompt_attention(int32_t batch, int32_t num_queries, int32_t num_keys, int32_t heads,
                        int32_t kv_heads, int32_t head_dim, int32_t dtype, const void* q,
                        int64_t q_stride, const void* k, const void* v, int64_t kv_stride,
                        const int32_t* q_start, const int32_t* k_start, float scale, void* out,
                        void* workspace, size_t workspace_bytes, hipStream_t stream) {
  const tv::PromptArgs a{batch, num_queries, num_keys, heads,     kv_heads, head_dim,
                         dtype, q,           q_stride, k,         v,        kv_stride,
                         q_start, k_start,   scale,    out};
  const int st = validate(a, workspace, workspace_bytes);
  if (st != TV_OK || batch == 0 || num_queries == 0) return st;
  return tv::launch_prompt(a, workspace, stream);
}

size_t tv_fp4_page_bytes(int32_t page_size, int32_t head_dim) {
  return static_cast<size_t>(fp4_page_bytes(page_size, head_dim));
}

int tv_cache_commit_fp4(int32_t layers, int32_t batch, int32_t num_nodes, int32_t kv_heads,
                        int32_t head_dim, int32_t dtype, const void* k_new, const void* v_new,
                        int64_t new_layer_stride, int64_t node_stride, void* k_cache, void* v_cache,
                        int64_t cache_layer_stride, int64_t page_stride, int32_t num_pages,
                        int32_t page_size, const int32_t* new_len, int32_t max_new,
                        const int32_t* slots, const int32_t* path_nodes, int32_t path_width,
                        hipStream_t stream) {
  const tv::Fp4CommitArgs a{layers,  batch,   num_nodes, kv_heads,    head_dim,
                            dtype,   k_new,   v_new,     new_layer_stride, node_stride,
                            k_cache, v_cache, cache_layer_stride, page_stride, num_pages,
                            page_size, new_len, max_new, slots,       path_nodes,
                            path_width};
  const int st = validate(a);
  if (st != TV_OK || layers == 0 || batch == 0 || max_new == 0 || num_pages == 0) return st;
  return tv::launch_cache_commit_fp4(a, stream);
}

int tv_cache_read_fp4(int32_t layers, int32_t batch, int32_t kv_heads, int32_t head_dim, int32_t dtype,
                      const void* k_cache, const void* v_cache, int64_t cache_layer_stride,
                      int64_t page_stride, int32_t num_pages, int32_t page_size,
                      const int32_t* block_table, int32_t table_width, const int32_t* first,
                      const int32_t* length, const int32_t* row_start, int32_t num_rows, void* k_out,
                      void* v_out, int64_t out_layer_stride, int64_t row_stride, hipStream_t stream) {
  const tv::Fp4ReadArgs a{layers,    batch,     kv_heads, head_dim,    dtype,
                          k_cache,   v_cache,   cache_layer_stride, page_stride, num_pages,
                          page_size, block_table, table_width, first,  length,
                          row_start, num_rows,  k_out,    v_out,       out_layer_stride,
                          row_stride};
  const int st = validate(a);
  if (st != TV_OK || layers == 0 || batch == 0 || num_rows == 0) return st;
  return tv::launch_cache_read_fp4(a, stream);
}

int tv_tree_attention_fp4(int32_t batch, int32_t num_nodes, int32_t heads, int32_t kv_heads,
                          int32_t head_dim, int32_t dtype, const int32_t* parents, const void* q,
                          int64_t q_stride, const void* k_new, const void* v_new, int64_t kv_stride,
                          const void* k_cache, const void* v_cache, int64_t page_stride,
                          int32_t num_pages, int32_t page_size, const int32_t* block_table,
                          int32_t table_width, const int32_t* ctx_len, const int32_t* prefix_pages,
                          int32_t prefix_len, float scale, void* out, void* workspace,
                          size_t workspace_bytes, hipStream_t stream) {
  const tv::AttentionArgs a{batch,     num_nodes,   heads,       kv_heads,  head_dim,
                            dtype,     parents,     q,           q_stride,  k_new,
                            v_new,     kv_stride,   k_cache,     v_cache,   page_stride,
                            num_pages, page_size,   block_table, table_width, ctx_len,
                            prefix_pages, prefix_len, scale,     out};
  const int st = validate(a, workspace, workspace_bytes, true);
  if (st != TV_OK || batch == 0) return st;
  return tv::launch_attention_fp4(a, workspace, stream);
}

}  // extern "C"
