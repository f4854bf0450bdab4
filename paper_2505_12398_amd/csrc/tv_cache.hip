// The paged cache behind the trees: growth of the requests' block tables with
// the slots of the new positions (tv_cache_extend), and the write of committed
// nodes' keys and values into them (tv_cache_commit).
#include <hip/hip_runtime.h>

#include "tv.h"
#include "tv_launch.h"

namespace {

constexpr int kScanThreads = 1024, kScanWaves = kScanThreads / 64;

struct Request {
  int seq, add, held, need;   // positions, appended ones, pages held, pages to take
  int first, back;            // pages to give back: table entries first .. first + back - 1
  int status;
  bool ends;
};

__device__ __forceinline__ Request request(const tv::ExtendArgs& a, int b) {
  Request r{};
  const int ps = a.page_size, shift = 31 - __builtin_clz(ps), cap = a.table_width * ps;
  const int n = a.new_len[b];
  r.seq = a.seq_len[b];
  if (r.seq < 0 || r.seq > cap) {
    r.status = TV_CACHE_BAD_LENGTH;
    return r;
  }
  r.held = (r.seq >> shift) + ((r.seq & (ps - 1)) != 0);
  if (n == TV_CACHE_RELEASE) {
    r.first = r.seq >= a.prefix_len ? a.prefix_len >> shift : 0;
    r.back = r.held - r.first;
    r.ends = true;
    return r;
  }
  if (n > a.max_new || n > cap - r.seq) {
    r.status = TV_CACHE_OVERFLOW;
    return r;
  }
  r.add = n > 0 ? n : 0;
  const int seq = r.seq + r.add;
  r.need = (seq >> shift) + ((seq & (ps - 1)) != 0) - r.held;
  return r;
}

// The slot of a position on `page` (-1 on a page that is none).
__device__ __forceinline__ int slot_of(const tv::ExtendArgs& a, int page, int pos) {
  return page >= 0 && page < a.num_pages ? page * a.page_size + (pos & (a.page_size - 1)) : -1;
}

// Sum of x over the workgroup's lower threads; `total` that of all.
__device__ __forceinline__ long long scan(long long x, long long (&part)[kScanWaves],
                                          long long& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  long long s = x;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const long long o = __shfl_up(s, off, 64);
    if (lane >= off) s += o;
  }
  __syncthreads();
  if (lane == 63) part[wave] = s;
  __syncthreads();
  total = 0;
  long long before = 0;
#pragma unroll
  for (int w = 0; w < kScanWaves; ++w) {
    if (w < wave) before += part[w];
    total += part[w];
  }
  return before + s - x;
}

// One workgroup, 1024 requests at a time: pages given back are pushed first,
// then a scan over the needs says where in the stack each request's pages are.
// Bound by latency: a handful of dependent loads and three scans. kSlots: the
// slots are written here, from what the threads hold, else by slots_kernel.
template <bool kSlots>
__global__ void __launch_bounds__(kScanThreads) extend_kernel(tv::ExtendArgs a) {
  __shared__ long long part[kScanWaves];
  __shared__ int seqs[kScanThreads], adds[kScanThreads], helds[kScanThreads], tops[kScanThreads],
      needs[kScanThreads];
  const int tid = threadIdx.x, lane = tid & 63;
  const int shift = 31 - __builtin_clz(a.page_size);
  __shared__ int most;                 // pages taken
  if (tid == 0) most = 0;
  const int count = min(max(a.free_count[0], 0), a.num_pages);
  long long pushed = 0;
  Request r{};
  for (int b0 = 0; b0 < a.batch; b0 += kScanThreads) {
    const int b = b0 + tid;
    r = b < a.batch ? request(a, b) : Request{};
    if (!__syncthreads_or(r.back > 0)) continue;
    long long total;
    const long long at = count + pushed + scan(r.back, part, total);
    pushed += total;
    // a wavefront copies its requests' pages one request after the other
    for (uint64_t m = __ballot(r.back > 0); m; m &= m - 1) {
      const int l = __builtin_ctzll(m);
      const int n = __shfl(r.back, l, 64), first = __shfl(r.first, l, 64);
      const long long to = __shfl(at, l, 64);
      int32_t* row = a.block_table + static_cast<size_t>(b - lane + l) * a.table_width + first;
      for (int j = lane; j < n; j += 64) {
        if (to + j < a.num_pages) a.free_pages[to + j] = row[j];
        row[j] = -1;
      }
    }
  }
  __syncthreads();
  const int avail = static_cast<int>(min<long long>(count + pushed, a.num_pages));
  long long before = 0;
  for (int b0 = 0; b0 < a.batch; b0 += kScanThreads) {
    const int b = b0 + tid;
    if (a.batch > kScanThreads) r = b < a.batch ? request(a, b) : Request{};
    long long total;
    const long long at = before + scan(r.need, part, total);
    before += total;
    if (r.need > 0 && at + r.need > avail) {
      r.status = TV_CACHE_FULL;
      r.add = r.need = 0;
    }
    if (r.need > 0) atomicMax(&most, static_cast<int>(at) + r.need);
    // page j of the new ones is free_pages[top - j]
    const int top = avail - 1 - static_cast<int>(r.need > 0 ? at : 0);
    if (r.need > 0)
      a.block_table[static_cast<size_t>(b) * a.table_width + r.held] = a.free_pages[top];
    seqs[tid] = r.seq;
    adds[tid] = r.add;
    helds[tid] = r.held;
    tops[tid] = top;
    needs[tid] = r.need;
    if (b < a.batch) {
      a.status[b] = r.status;
      a.new_seq_len[b] = r.ends ? 0 : r.seq + r.add;
    }
    // a request's further pages by a wavefront, the requests by all wavefronts
    if (__syncthreads_or(r.need > 1)) {
      for (int q = tid >> 6; q < min(kScanThreads, a.batch - b0); q += kScanWaves) {
        const int n = needs[q], from = tops[q];
        const size_t to = static_cast<size_t>(b0 + q) * a.table_width + helds[q];
        for (int j = 1 + lane; j < n; j += 64) a.block_table[to + j] = a.free_pages[from - j];
      }
    }
    if constexpr (kSlots) {
      const int n = min(kScanThreads, a.batch - b0) * a.max_new;
      for (int i = tid; i < n; i += kScanThreads) {
        const int q = i / a.max_new, k = i - q * a.max_new;
        int slot = -1;
        if (k < adds[q]) {
          const int pos = seqs[q] + k, j = pos >> shift;
          const int page = j < helds[q]
                               ? a.block_table[static_cast<size_t>(b0 + q) * a.table_width + j]
                               : a.free_pages[tops[q] - (j - helds[q])];
          slot = slot_of(a, page, pos);
        }
        a.slots[static_cast<size_t>(b0) * a.max_new + i] = slot;
      }
    }
  }
  if (tid == 0) a.new_free_count[0] = avail - most;
}

constexpr int kCopyThreads = 256;

// The slots of many positions: a workgroup takes 256 of one request.
__global__ void __launch_bounds__(kCopyThreads) slots_kernel(tv::ExtendArgs a) {
  const int b = blockIdx.x;
  const int shift = 31 - __builtin_clz(a.page_size);
  const int add = a.status[b] == TV_CACHE_OK ? max(a.new_len[b], 0) : 0;
  const int seq = a.new_seq_len[b] - add;
  for (int k = blockIdx.y * kCopyThreads + threadIdx.x; k < a.max_new;
       k += gridDim.y * kCopyThreads) {
    int slot = -1;
    if (k < add) {
      const int pos = seq + k;
      slot = slot_of(a, a.block_table[static_cast<size_t>(b) * a.table_width + (pos >> shift)], pos);
    }
    a.slots[static_cast<size_t>(b) * a.max_new + k] = slot;
  }
}

// Up to how many slots the one workgroup writes them itself: 2560 of them 5.7 us, with
// a launch of their own 6.7; 16384 of them 16.2 and 12.4, 65536 of them 27 and 8.4.
constexpr int64_t kOwnSlots = 4096;

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
constexpr int kRows = 16;   // rows of a workgroup

// Workgroup (b, layer, z): every gridDim.z-th kRows rows' keys and values, 16 bytes a
// thread and step. Bound by HBM, in rows of a few hundred bytes to each head's page:
// 256 requests, 32 layers of 8 heads of 128, 4.9 rows each: 61 us, 5.4 TB/s read and
// written (within what the last-level cache holds of it).
__global__ void __launch_bounds__(kCopyThreads) cache_commit_kernel(tv::CacheCommitArgs a) {
  const int b = blockIdx.x, layer = blockIdx.y, all = min(a.new_len[b], a.max_new);
  const int shift = 31 - __builtin_clz(a.page_size), hp = a.head_bytes / 16;
  const int per = hp * a.kv_heads;
  const uint8_t* src[2] = {static_cast<const uint8_t*>(a.k_new), static_cast<const uint8_t*>(a.v_new)};
  uint8_t* dst[2] = {static_cast<uint8_t*>(a.k_cache), static_cast<uint8_t*>(a.v_cache)};
  const int64_t from = layer * a.new_layer_stride + static_cast<int64_t>(b) * a.num_nodes * a.node_stride;
  const int64_t to = layer * a.cache_layer_stride;
  for (int k0 = blockIdx.z * kRows; k0 < all; k0 += gridDim.z * kRows) {
    const int n = min(all - k0, kRows);
    for (int i = threadIdx.x; i < n * per; i += kCopyThreads) {
      const int r = i / per, w = i - r * per, head = w / hp, piece = w - head * hp;
      const int k = k0 + r;
      const int slot = a.slots[static_cast<size_t>(b) * a.max_new + k];
      int node = k;
      if (a.path_nodes && k > 0)
        node = k - 1 < a.path_width ? a.path_nodes[static_cast<size_t>(b) * a.path_width + k - 1] : -1;
      const int page = slot >> shift;
      if (slot < 0 || page >= a.num_pages || node < 0 || node >= a.num_nodes) continue;
      const int64_t f = from + node * a.node_stride + static_cast<int64_t>(w) * 16;
      const int64_t t = to + page * a.page_stride +
                        (static_cast<int64_t>(head) * a.page_size + (slot & (a.page_size - 1))) *
                            a.head_bytes + piece * 16;
#pragma unroll
      for (int c = 0; c < 2; ++c)
        *reinterpret_cast<u32x4*>(dst[c] + t) = *reinterpret_cast<const u32x4*>(src[c] + f);
    }
  }
}

}  // namespace

namespace tv {

int launch_extend(const ExtendArgs& a, hipStream_t stream) {
  if (static_cast<int64_t>(a.batch) * a.max_new <= kOwnSlots) {
    hipLaunchKernelGGL((extend_kernel<true>), dim3(1), dim3(kScanThreads), 0, stream, a);
  } else {
    hipLaunchKernelGGL((extend_kernel<false>), dim3(1), dim3(kScanThreads), 0, stream, a);
    if (hipGetLastError() != hipSuccess) return TV_ERR_HIP;
    const int64_t parts = (static_cast<int64_t>(a.max_new) + kCopyThreads - 1) / kCopyThreads;
    hipLaunchKernelGGL(slots_kernel,
                       dim3(static_cast<unsigned>(a.batch),
                            static_cast<unsigned>(parts < 1024 ? parts : 1024)),
                       dim3(kCopyThreads), 0, stream, a);
  }
  return hipGetLastError() == hipSuccess ? TV_OK : TV_ERR_HIP;
}

int launch_cache_commit(const CacheCommitArgs& a, hipStream_t stream) {
  const int64_t parts = (static_cast<int64_t>(a.max_new) + kRows - 1) / kRows;
  hipLaunchKernelGGL(cache_commit_kernel,
                     dim3(static_cast<unsigned>(a.batch), static_cast<unsigned>(a.layers),
                          static_cast<unsigned>(parts < 1024 ? parts : 1024)),
                     dim3(kCopyThreads), 0, stream, a);
  return hipGetLastError() == hipSuccess ? TV_OK : TV_ERR_HIP;
}

}  // namespace tv
