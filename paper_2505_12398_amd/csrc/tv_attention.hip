// Attention of tree nodes over a paged cache of 16-bit keys and values (tv_tree_attention).
#include "tv_tree_attention.h"

namespace tv {

size_t attention_workspace(int32_t batch, int32_t num_nodes, int32_t heads, int32_t kv_heads,
                           int32_t head_dim, int32_t prefix_len) {
  return layout(batch, num_nodes, heads, kv_heads, head_dim, prefix_len).bytes;
}

int launch_attention(const AttentionArgs& a, void* workspace, hipStream_t stream) {
  AttentionArgs in_bytes = a;
  in_bytes.page_stride *= 2;
  return ::launch<false>(in_bytes, workspace, stream);
}

}  // namespace tv
