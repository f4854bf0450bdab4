// Attention of tree nodes over a paged cache (tv_tree_attention): a workgroup per
// tree, node and query head, 256 keys at a time with the running maximum and sum
// of the softmax.
#include <hip/hip_runtime.h>
#include <math.h>

#include "tv.h"
#include "tv_launch.h"

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float value(__bf16 x) { return static_cast<float>(x); }
__device__ __forceinline__ float value(_Float16 x) { return static_cast<float>(x); }

template <class T>
__global__ void __launch_bounds__(kThreads) attention_kernel(tv::AttentionArgs a) {
  __shared__ float qs[TV_MAX_HEAD_DIM];
  __shared__ float ps[kThreads];
  __shared__ const T* vs[kThreads];
  __shared__ float red[kThreads / 64];
  __shared__ uint8_t on_path[TV_MAX_NODES];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int h = blockIdx.x, i = blockIdx.y, b = blockIdx.z;
  const int D = a.head_dim, n1 = a.num_nodes, kh = h / (a.heads / a.kv_heads);
  const int ctx = a.ctx_len[b];
  if (ctx < 0) return;
  const int shift = 31 - __builtin_clz(a.page_size);
  const bool shared = a.prefix_len > 0 && ctx >= a.prefix_len;
  const size_t node = static_cast<size_t>(b) * n1 + i;
  const T* q = static_cast<const T*>(a.q) + node * a.q_stride + h * D;
  for (int d = tid; d < D; d += kThreads) qs[d] = value(q[d]);
  for (int j = tid; j < n1; j += kThreads) on_path[j] = 0;
  __syncthreads();
  if (tid == 0) {
    int x = i;
    on_path[x] = 1;
    while (x > 0) {
      const int p = a.parents[static_cast<size_t>(b) * n1 + x];
      if (p < 0 || p >= x) break;
      x = p;
      on_path[x] = 1;
    }
  }
  __syncthreads();
  bool bad = ctx > static_cast<int64_t>(a.table_width) * a.page_size;
  const long long n = bad ? 0 : static_cast<long long>(ctx) + n1;
  float m = -INFINITY, l = 0.0f, o = 0.0f;
  for (long long t0 = 0; t0 < n; t0 += kThreads) {
    const long long x = t0 + tid;
    const T *k = nullptr, *v = nullptr;
    if (x < ctx) {
      const int at = static_cast<int>(x), j = at >> shift;
      const int page = shared && at < a.prefix_len
                           ? a.prefix_pages[j]
                           : a.block_table[static_cast<size_t>(b) * a.table_width + j];
      if (page < 0 || page >= a.num_pages) {
        bad = true;
      } else {
        const size_t e = page * a.page_stride +
                         (static_cast<size_t>(kh) * a.page_size + (at & (a.page_size - 1))) * D;
        k = static_cast<const T*>(a.k_cache) + e;
        v = static_cast<const T*>(a.v_cache) + e;
      }
    } else if (x < n && on_path[x - ctx]) {
      const size_t e = (static_cast<size_t>(b) * n1 + (x - ctx)) * a.kv_stride + kh * D;
      k = static_cast<const T*>(a.k_new) + e;
      v = static_cast<const T*>(a.v_new) + e;
    }
    float s = -INFINITY;
    if (k) {
      s = 0.0f;
      for (int d = 0; d < D; ++d) s = fmaf(qs[d], value(k[d]), s);
      s *= a.scale;
    }
    float top = s;
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    if (lane == 0) red[wave] = top;
    __syncthreads();
    top = m;
    for (int w = 0; w < kThreads / 64; ++w) top = fmaxf(top, red[w]);
    ps[tid] = k ? expf(s - top) : 0.0f;
    vs[tid] = v;
    __syncthreads();
    if (top > -INFINITY) {
      const float f = expf(m - top);
      l *= f;
      o *= f;
      m = top;
    }
    for (int j = 0; j < kThreads; ++j)
      if (vs[j]) {
        l += ps[j];
        if (tid < D) o = fmaf(ps[j], value(vs[j][tid]), o);
      }
    __syncthreads();
  }
  bad = __syncthreads_or(bad);
  if (tid < D)
    static_cast<T*>(a.out)[(node * a.heads + h) * D + tid] = static_cast<T>(bad ? NAN : o / l);
}

}  // namespace

namespace tv {

size_t attention_workspace(int32_t batch, int32_t num_nodes, int32_t heads, int32_t kv_heads,
                           int32_t head_dim, int32_t prefix_len) {
  return 256;
}

int launch_attention(const AttentionArgs& a, void* workspace, hipStream_t stream) {
  for (int b0 = 0; b0 < a.batch; b0 += 32768) {
    AttentionArgs c = a;
    c.batch = a.batch - b0 < 32768 ? a.batch - b0 : 32768;
    const size_t rows = static_cast<size_t>(b0) * a.num_nodes;
    c.parents = a.parents ? a.parents + rows : nullptr;
    c.q = static_cast<const uint16_t*>(a.q) + rows * a.q_stride;
    c.k_new = static_cast<const uint16_t*>(a.k_new) + rows * a.kv_stride;
    c.v_new = static_cast<const uint16_t*>(a.v_new) + rows * a.kv_stride;
    c.block_table = a.block_table + static_cast<size_t>(b0) * a.table_width;
    c.ctx_len = a.ctx_len + b0;
    c.out = static_cast<uint16_t*>(a.out) + rows * a.heads * a.head_dim;
    const dim3 grid(a.heads, a.num_nodes, c.batch);
    if (a.dtype == TV_DTYPE_BF16)
      hipLaunchKernelGGL((attention_kernel<__bf16>), grid, dim3(kThreads), 0, stream, c);
    else
      hipLaunchKernelGGL((attention_kernel<_Float16>), grid, dim3(kThreads), 0, stream, c);
  }
  return hipGetLastError() == hipSuccess ? TV_OK : TV_ERR_HIP;
}

}  // namespace tv
