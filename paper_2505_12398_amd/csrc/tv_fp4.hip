// The paged cache in 4 bits: committed nodes' keys and values into it
// (tv_cache_commit_fp4) and positions out of it again (tv_cache_read_fp4).
//
// Blocks of 32 elements of a head share a power of two 2^e, of which one byte holds e + 127;
// an element is a sign, and one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 (e2m1), which gfx950
// converts by itself in both directions. e is the least with amax <= 7 2^e: between 6 and 7
// elements are rounded to 6 as a grid that went on at 8 would round them. Root mean square
// errors of normal elements by that bound: 6 11.5%, 7 11.2%, 8 11.5% of theirs.
#include <hip/hip_runtime.h>

#include "tv.h"
#include "tv_attention_common.h"
#include "tv_launch.h"

namespace {

constexpr int kThreads = 256;
constexpr int kRows = 16;   // rows that a workgroup takes at a time

// Of eight elements as floats: the larger of their magnitudes' bits so far (those of NaN and
// infinity are above all others').
template <class T>
__device__ __forceinline__ uint32_t magnitudes(const u32x4& w, float (&x)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[i] = T::value(static_cast<uint16_t>(w[i >> 1] >> (16 * (i & 1))));
    top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  }
  return top;
}

// The exponent's byte of a block whose largest magnitude has these bits; 255 if it is not
// finite. (At most one whose elements the type holds: beyond 7 2^125, or 7 2^13 in fp16, they
// are rounded to 6 of that power.)
template <class T>
__device__ __forceinline__ int exponent_of(uint32_t top) {
  if (top >= 0x7f800000u) return 255;
  const int e = static_cast<int>(top >> 23) - 2 + ((top & 0x7fffffu) > 0x600000u);
  return min(max(e, 1), T::kExponent == 0x7c00 ? 127 + 13 : 127 + 125);
}

// Four lanes a block, eight elements a lane, so that reads are 16 bytes a lane and the four
// bytes that a lane writes follow each other.
template <class T>
__global__ void __launch_bounds__(kThreads) commit_kernel(tv::Fp4CommitArgs a) {
  const int b = blockIdx.x, layer = blockIdx.y, all = min(a.new_len[b], a.max_new);
  const int shift = 31 - __builtin_clz(a.page_size);
  const int per_head = a.head_dim / 8, per = per_head * a.kv_heads, row_bytes = a.head_dim / 2;
  const int blocks = a.head_dim / TV_FP4_BLOCK;
  const int64_t head_bytes = static_cast<int64_t>(a.page_size) * (row_bytes + blocks);
  const uint16_t* src[2] = {static_cast<const uint16_t*>(a.k_new), static_cast<const uint16_t*>(a.v_new)};
  uint8_t* dst[2] = {static_cast<uint8_t*>(a.k_cache), static_cast<uint8_t*>(a.v_cache)};
  const int64_t from = layer * a.new_layer_stride + static_cast<int64_t>(b) * a.num_nodes * a.node_stride;
  const int64_t to = layer * a.cache_layer_stride;
  for (int k0 = blockIdx.z * kRows; k0 < all; k0 += gridDim.z * kRows) {
    const int n = min(all - k0, kRows);
    // (whole blocks, so the four lanes of one are all there or none is)
    for (int i = threadIdx.x; i < n * per; i += kThreads) {
      const int r = i / per, w = i - r * per, head = w / per_head, piece = w - head * per_head;
      const int k = k0 + r;
      const int slot = a.slots[static_cast<size_t>(b) * a.max_new + k];
      int node = k;
      if (a.path_nodes && k > 0)
        node = k - 1 < a.path_width ? a.path_nodes[static_cast<size_t>(b) * a.path_width + k - 1] : -1;
      const int page = slot >> shift, row = slot & (a.page_size - 1);
      if (slot < 0 || page >= a.num_pages || node < 0 || node >= a.num_nodes) continue;
      const int64_t f = from + node * a.node_stride + static_cast<int64_t>(w) * 8;
      const int64_t t = to + page * a.page_stride + head * head_bytes;
      u32x4 in[2];
#pragma unroll
      for (int c = 0; c < 2; ++c) in[c] = *reinterpret_cast<const u32x4*>(src[c] + f);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float x[8];
        uint32_t top = magnitudes<T>(in[c], x);
        top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 1, 64)));
        top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 2, 64)));
        const int e = exponent_of<T>(top);
        const float s = __uint_as_float(static_cast<uint32_t>(e) << 23);
        uint32_t out = 0;
        out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, x[0], x[1], s, 0);
        out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, x[2], x[3], s, 1);
        out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, x[4], x[5], s, 2);
        out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, x[6], x[7], s, 3);
        *reinterpret_cast<uint32_t*>(dst[c] + t + row * row_bytes + 4 * piece) = e == 255 ? 0 : out;
        if (piece % 4 == 0)
          dst[c][t + static_cast<int64_t>(a.page_size) * row_bytes + row * blocks + piece / 4] =
              static_cast<uint8_t>(e);
      }
    }
  }
}

// Eight elements a lane: four bytes in, 16 out.
template <class T>
__global__ void __launch_bounds__(kThreads) read_kernel(tv::Fp4ReadArgs a) {
  const int b = blockIdx.x, layer = blockIdx.y, all = a.length[b];
  const int shift = 31 - __builtin_clz(a.page_size);
  const int per_head = a.head_dim / 8, per = per_head * a.kv_heads, row_bytes = a.head_dim / 2;
  const int blocks = a.head_dim / TV_FP4_BLOCK;
  const int64_t head_bytes = static_cast<int64_t>(a.page_size) * (row_bytes + blocks);
  const int first = a.first ? a.first[b] : 0, start = a.row_start[b];
  const uint8_t* src[2] = {static_cast<const uint8_t*>(a.k_cache), static_cast<const uint8_t*>(a.v_cache)};
  uint16_t* dst[2] = {static_cast<uint16_t*>(a.k_out), static_cast<uint16_t*>(a.v_out)};
  for (int64_t k0 = static_cast<int64_t>(blockIdx.z) * kRows; k0 < all;
       k0 += static_cast<int64_t>(gridDim.z) * kRows) {
    const int n = static_cast<int>(min<int64_t>(all - k0, kRows));
    for (int i = threadIdx.x; i < n * per; i += kThreads) {
      const int r = i / per, w = i - r * per, head = w / per_head, piece = w - head * per_head;
      const int64_t x = first + k0 + r, to_row = start + k0 + r;
      if (to_row < 0 || to_row >= a.num_rows) continue;
      const bool held = x >= 0 && x >> shift < a.table_width;
      const int page = held ? a.block_table[static_cast<size_t>(b) * a.table_width + (x >> shift)] : -1;
      const bool fine = page >= 0 && page < a.num_pages;
      const int row = static_cast<int>(x & (a.page_size - 1));
      const int64_t f = layer * a.cache_layer_stride + (fine ? page : 0) * a.page_stride + head * head_bytes;
      const int64_t t = layer * a.out_layer_stride + to_row * a.row_stride + static_cast<int64_t>(w) * 8;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint32_t q = 0;
        float s = NAN;
        if (fine) {
          q = *reinterpret_cast<const uint32_t*>(src[c] + f + row * row_bytes + 4 * piece);
          s = __uint_as_float(
              static_cast<uint32_t>(src[c][f + static_cast<int64_t>(a.page_size) * row_bytes +
                                           row * blocks + piece / 4]) << 23);
        }
        *reinterpret_cast<u32x4*>(dst[c] + t) =
            u32x4{T::template widen<0>(q, s), T::template widen<1>(q, s),
                  T::template widen<2>(q, s), T::template widen<3>(q, s)};
      }
    }
  }
}

// Workgroups of a request and layer for `rows` rows at most: enough to fill the device, the
// rest in steps.
unsigned parts(int64_t rows, int64_t items) {
  const int64_t all = (rows + kRows - 1) / kRows, room = (int64_t{1} << 16) / items;
  const int64_t n = all < room ? all : room;
  return static_cast<unsigned>(n < 1 ? 1 : n > 4096 ? 4096 : n);
}

}  // namespace

namespace tv {

int launch_cache_commit_fp4(const Fp4CommitArgs& a, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(a.batch), static_cast<unsigned>(a.layers),
                  parts(a.max_new, static_cast<int64_t>(a.batch) * a.layers));
  if (a.dtype == TV_DTYPE_BF16)
    hipLaunchKernelGGL((commit_kernel<Bf16>), grid, dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((commit_kernel<F16>), grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError() == hipSuccess ? TV_OK : TV_ERR_HIP;
}

int launch_cache_read_fp4(const Fp4ReadArgs& a, hipStream_t stream) {
  const int64_t rows = static_cast<int64_t>(a.table_width) * a.page_size;
  const dim3 grid(static_cast<unsigned>(a.batch), static_cast<unsigned>(a.layers),
                  parts(rows < a.num_rows ? rows : a.num_rows, static_cast<int64_t>(a.batch) * a.layers));
  if (a.dtype == TV_DTYPE_BF16)
    hipLaunchKernelGGL((read_kernel<Bf16>), grid, dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((read_kernel<F16>), grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError() == hipSuccess ? TV_OK : TV_ERR_HIP;
}

}  // namespace tv
