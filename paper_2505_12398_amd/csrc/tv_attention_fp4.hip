// Attention of tree nodes over a paged cache of 4 bits (tv_tree_attention_fp4).
#include "tv_tree_attention.h"

namespace tv {

int launch_attention_fp4(const AttentionArgs& a, void* workspace, hipStream_t stream) {
  return ::launch<true>(a, workspace, stream);
}

}  // namespace tv
