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
constexpr int kRows = 8;    // rows that a workgroup takes at a time

// The exponent's byte of a block whose largest magnitude is this float. 255 if it is not finite; at most
// one whose elements the type holds: beyond 7 2^125, or 7 2^13 in fp16, they are rounded to 6 of that
// power.
template <class T>
__device__ __forceinline__ int exponent_of(float top) {
  const uint32_t u = __float_as_uint(top);
  if (u >= 0x7f800000u) return 255;
  const int e = static_cast<int>(u >> 23) - 2 + ((u & 0x7fffffu) > 0x600000u);
  return min(max(e, 1), T::kExponent == 0x7c00 ? 127 + 13 : 127 + 125);
}

// Both halves' larger ones of two words.
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
  typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a),
                                                                __builtin_bit_cast(u16x2, b)));
}

// Pieces of eight elements, four lanes a block of 32, so that reads are 16 bytes a lane and the four
// bytes that a lane writes follow each other. A thread keeps its piece of the heads and goes over rows,
// of which a workgroup takes kRows at a time, their places from LDS: kAhead of a thread with their loads
// in flight. Bound by HBM, where writes beside reads are the slow ones: 16-bit elements go past the
// caches, in and out (64000 rows of 8 heads of 128 written and read back: 238 us through them, 195 with
// the writes past them, 177 with both; 75500 rows read back 125 and 83, 4.7 TB/s). kAhead and kRows, the
// same rows written and read back: 4 and 32 187, 4 and 16 176, 4 and 8 169, 2 and 16 160, 2 and 8 155, 1
// and 8 156.
constexpr int kAhead = 2;

struct Spread {                           // pieces w, w + w_step, .. of rows r, r + r_step, ..
  int w, w_step, r, r_step;
};
__device__ __forceinline__ Spread spread(int per) {
  const int tid = threadIdx.x;
  if (per >= kThreads) return {tid, kThreads, 0, 1};
  const int r = tid / per, rows = kThreads / per;
  return {tid - r * per, per, r < rows ? r : kRows, rows};
}

template <class T>
__global__ void __launch_bounds__(kThreads) commit_kernel(tv::Fp4CommitArgs a) {
  __shared__ int64_t froms[kRows], tos[kRows];   // a row's place in the new ones and its page's
  __shared__ int rows[kRows];                    // and which row of the page, -1 for none
  const int b = blockIdx.x, layer = blockIdx.y, all = min(a.new_len[b], a.max_new), tid = threadIdx.x;
  const int shift = 31 - __builtin_clz(a.page_size);
  const int per_head = a.head_dim / 8, per = per_head * a.kv_heads, row_bytes = a.head_dim / 2;
  const int blocks = a.head_dim / TV_FP4_BLOCK, exps = a.page_size * row_bytes;
  const int64_t head_bytes = exps + a.page_size * blocks;
  const uint16_t* src[2] = {static_cast<const uint16_t*>(a.k_new), static_cast<const uint16_t*>(a.v_new)};
  uint8_t* dst[2] = {static_cast<uint8_t*>(a.k_cache), static_cast<uint8_t*>(a.v_cache)};
  const int64_t from = layer * a.new_layer_stride + static_cast<int64_t>(b) * a.num_nodes * a.node_stride;
  const int64_t to = layer * a.cache_layer_stride;
  const Spread S = spread(per);
  for (int k0 = blockIdx.z * kRows; k0 < all; k0 += gridDim.z * kRows) {
    const int n = min(all - k0, kRows);
    __syncthreads();                      // (the rows before are written)
    if (tid < n) {
      const int k = k0 + tid;
      int node = k, slot = a.slots[static_cast<size_t>(b) * a.max_new + k];
      if (a.path_nodes && k > 0)
        node = k - 1 < a.path_width ? a.path_nodes[static_cast<size_t>(b) * a.path_width + k - 1] : -1;
      const bool fine = slot >= 0 && slot >> shift < a.num_pages && node >= 0 && node < a.num_nodes;
      froms[tid] = from + node * a.node_stride;
      tos[tid] = to + (slot >> shift) * a.page_stride;
      rows[tid] = fine ? slot & (a.page_size - 1) : -1;
    }
    __syncthreads();
    for (int w = S.w; w < per; w += S.w_step) {
      const int head = w / per_head, piece = w - head * per_head;
      const int64_t of_head = head * head_bytes;
      // (the four lanes of a block have the same rows)
      for (int r0 = S.r; r0 < n; r0 += kAhead * S.r_step) {
        u32x4 in[kAhead][2];
        int row[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          const int r = r0 + u * S.r_step;
          row[u] = r < n ? rows[r] : -1;
          if (row[u] < 0) continue;
#pragma unroll
          for (int c = 0; c < 2; ++c) in[u][c] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src[c] + froms[r] + w * 8));
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          if (row[u] < 0) continue;
          const int64_t t = tos[r0 + u * S.r_step] + of_head;
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const u32x4 x = in[u][c];
            uint32_t top = 0;             // magnitudes of 16 bits are in the order of their bits
#pragma unroll
            for (int i = 0; i < 4; ++i) top = larger(top, x[i] & 0x7fff7fffu);
            top = larger(top, top >> 16);
            top = larger(top, __builtin_amdgcn_mov_dpp(top, 0xb1, 0xf, 0xf, true));   // lanes 1 0 3 2
            top = larger(top, __builtin_amdgcn_mov_dpp(top, 0x4e, 0xf, 0xf, true));   // lanes 2 3 0 1
            const int e = exponent_of<T>(T::value(static_cast<uint16_t>(top)));
            const float s = __uint_as_float(static_cast<uint32_t>(e) << 23);
            uint32_t out = T::template narrow<0>(0, x[0], s);
            out = T::template narrow<1>(out, x[1], s);
            out = T::template narrow<2>(out, x[2], s);
            out = T::template narrow<3>(out, x[3], s);
            *reinterpret_cast<uint32_t*>(dst[c] + t + row[u] * row_bytes + 4 * piece) = e == 255 ? 0 : out;
            if (piece % 4 == 0) dst[c][t + exps + row[u] * blocks + piece / 4] = static_cast<uint8_t>(e);
          }
        }
      }
    }
  }
}

// The same the other way: four bytes in, 16 out.
template <class T>
__global__ void __launch_bounds__(kThreads) read_kernel(tv::Fp4ReadArgs a) {
  __shared__ int64_t froms[kRows];        // a row's page
  __shared__ int rows[kRows];             // and which row of it, -1 for none
  const int b = blockIdx.x, layer = blockIdx.y, tid = threadIdx.x;
  const int shift = 31 - __builtin_clz(a.page_size);
  const int per_head = a.head_dim / 8, per = per_head * a.kv_heads, row_bytes = a.head_dim / 2;
  const int blocks = a.head_dim / TV_FP4_BLOCK, exps = a.page_size * row_bytes;
  const int64_t head_bytes = exps + a.page_size * blocks;
  const int first = a.first ? a.first[b] : 0, start = a.row_start[b];
  // the positions whose rows the outputs have (a length may be far beyond them)
  const int64_t from = max(-static_cast<int64_t>(start), int64_t{0});
  const int64_t all = min(static_cast<int64_t>(a.length[b]), static_cast<int64_t>(a.num_rows) - start);
  const uint8_t* src[2] = {static_cast<const uint8_t*>(a.k_cache), static_cast<const uint8_t*>(a.v_cache)};
  uint16_t* dst[2] = {static_cast<uint16_t*>(a.k_out), static_cast<uint16_t*>(a.v_out)};
  const Spread S = spread(per);
  for (int64_t k0 = from + static_cast<int64_t>(blockIdx.z) * kRows; k0 < all;
       k0 += static_cast<int64_t>(gridDim.z) * kRows) {
    const int n = static_cast<int>(min<int64_t>(all - k0, kRows));
    __syncthreads();                      // (the rows before are written)
    if (tid < n) {
      const int64_t x = first + k0 + tid;
      int page = -1;
      if (x >= 0 && x >> shift < a.table_width)
        page = a.block_table[static_cast<size_t>(b) * a.table_width + (x >> shift)];
      froms[tid] = layer * a.cache_layer_stride + page * a.page_stride;
      rows[tid] = page < 0 || page >= a.num_pages ? -1 : static_cast<int>(x & (a.page_size - 1));
    }
    __syncthreads();
    for (int w = S.w; w < per; w += S.w_step) {
      const int head = w / per_head, piece = w - head * per_head;
      const int64_t of_head = head * head_bytes;
      const int64_t to = layer * a.out_layer_stride + (start + k0) * a.row_stride + w * 8;
      for (int r0 = S.r; r0 < n; r0 += kAhead * S.r_step) {
        uint32_t q[kAhead][2], e[kAhead][2];
        int row[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          const int r = r0 + u * S.r_step;
          row[u] = r < n ? rows[r] : -1;
          q[u][0] = q[u][1] = 0;
          e[u][0] = e[u][1] = 255;
          if (row[u] < 0) continue;
          const int64_t f = froms[r] + of_head;
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            q[u][c] = *reinterpret_cast<const uint32_t*>(src[c] + f + row[u] * row_bytes + 4 * piece);
            e[u][c] = src[c][f + exps + row[u] * blocks + piece / 4];
          }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          if (r0 + u * S.r_step >= n) continue;
          const int64_t t = to + (r0 + u * S.r_step) * a.row_stride;
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const float s = __uint_as_float(e[u][c] << 23);   // (255: NaN in every element)
            __builtin_nontemporal_store(
                u32x4{T::template widen<0>(q[u][c], s), T::template widen<1>(q[u][c], s),
                      T::template widen<2>(q[u][c], s), T::template widen<3>(q[u][c], s)},
                reinterpret_cast<u32x4*>(dst[c] + t));
          }
        }
      }
    }
  }
}

// Workgroups of a request and layer for `rows` rows at most: enough to fill the device, the rest in
// steps. (Most requests have fewer rows than they may: with eight times as many 256 requests of 32 layers
// took 10 us more.)
unsigned parts(int64_t rows, int64_t items) {
  const int64_t all = (rows + kRows - 1) / kRows, room = ((int64_t{1} << 13) + items - 1) / items;
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
