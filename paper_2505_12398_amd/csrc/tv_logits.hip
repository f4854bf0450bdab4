// Penalties, biases and masks on the logits of tree nodes, with the statistics
// of the resulting rows (tv_process_logits).
//
// A workgroup holds kLogitsChunk tokens of the vocabulary for one tree: it counts
// the history's tokens among them once, in LDS, and then streams its part of the
// tree's rows, so the history is read once for many rows and a row costs one read
// and one write. Every thread owns the same 32 tokens in every row: what the history
// and the biases take off their logits stays in its registers. The drafted tokens on
// a node's path change few logits: their owners compute those again.
//
// What bounds it is HBM: 256 trees of 65 nodes and 128256 tokens in bfloat16 take
// 1.80 ms, 4.75 TB/s read and written (a large copy: 4.74). One tree takes 25 us,
// bound by its launches and a set-up of reads that wait for each other (biases, tokens
// and links, history). (Accesses marked as used once: 1.78 ms of those 256 trees, but
// 250 us instead of 228 of 16 in float32, before biases were kept from the set-up.)
//
// The statistics are a maximum and a sum of 2^((z - max) k), k = log2(e)/T, per
// wavefront and row, in fp32 in the frame of the maximum; a second kernel merges
// them in fp64. The frame is the product -max k as rounded, which z k - max k (one
// instruction) is off by alike, unless that product is so large that its rounding
// moves the exponents themselves, as where all of a wavefront's tokens are masked with
// a large negative number: from 2^20 on the difference is taken first.
#include <hip/hip_runtime.h>
#include <math.h>

#include <type_traits>

#include "tv.h"
#include "tv_launch.h"

namespace {

constexpr int kWaves = tv::kLogitsWaves, kThreads = 64 * kWaves;
constexpr int kChunk = tv::kLogitsChunk;
constexpr int kGroups = kChunk / (8 * kThreads);   // groups of 8 consecutive tokens of a thread
constexpr int kOwn = 8 * kGroups;                  // tokens of a thread
static_assert(kOwn == 32, "a thread's tokens are the bits of a word");
static_assert(static_cast<int64_t>(TV_MAX_BIAS + 1) * kChunk <= INT32_MAX, "a place and a bias entry");
constexpr float kFrames = 0x1p20f;                 // below it the frame is the rounded product
constexpr uint32_t kTold = 0x80000000u;            // in the prompt; below it the count

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
// vectors of rows that need not start on 16 bytes
typedef u32x4 __attribute__((aligned(2))) u32x4_any2;
typedef u32x4 __attribute__((aligned(4))) u32x4_any4;

// eight logits as they are stored
template <class T> struct Raw;
template <> struct Raw<uint16_t> {
  u32x4 w;
  __device__ __forceinline__ void load(const uint16_t* p) {
    const auto* q = reinterpret_cast<const u32x4_any2*>(p);
    w = *q;
  }
  __device__ __forceinline__ float at(int i) const {
    const uint32_t u = w[i >> 1];
    return __uint_as_float(i & 1 ? u & 0xffff0000u : u << 16);
  }
};
template <> struct Raw<float> {
  u32x4 w[2];
  __device__ __forceinline__ void load(const float* p) {
    const auto* q = reinterpret_cast<const u32x4_any4*>(p);
    const auto* r = reinterpret_cast<const u32x4_any4*>(p + 4);
    w[0] = *q;
    w[1] = *r;
  }
  __device__ __forceinline__ float at(int i) const { return __uint_as_float(w[i >> 2][i & 3]); }
};

__device__ __forceinline__ float value(uint16_t x) { return __uint_as_float(uint32_t{x} << 16); }
__device__ __forceinline__ float value(float x) { return x; }
template <class T> __device__ __forceinline__ T stored(float x);
template <> __device__ __forceinline__ uint16_t stored<uint16_t>(float x) {
  return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));   // to nearest even
}
template <> __device__ __forceinline__ float stored<float>(float x) { return x; }

__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{v[2 * i], v[2 * i + 1]}, bf16x2));
  *reinterpret_cast<u32x4_any2*>(p) = w;
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(v[4 * h + i]);
    *reinterpret_cast<u32x4_any4*>(p + 4 * h) = w;
  }
}

// Reductions over a wavefront, in vector instructions alone: neighbours, pairs, the
// quads and halves of a row of 16, rows, halves.
template <class F>
__device__ __forceinline__ float over_wave(float x, F&& join) {
  auto other = [&](auto ctrl) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), ctrl.value, 0xf, 0xf, true));
  };
  x = join(x, other(std::integral_constant<int, 0xB1>{}));    // lanes 1 0 3 2
  x = join(x, other(std::integral_constant<int, 0x4E>{}));    // lanes 2 3 0 1
  x = join(x, other(std::integral_constant<int, 0x141>{}));   // half rows mirrored
  x = join(x, other(std::integral_constant<int, 0x140>{}));   // rows mirrored
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = join(__uint_as_float(r[0]), __uint_as_float(r[1]));
  const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return join(__uint_as_float(h[0]), __uint_as_float(h[1]));
}

// x where bit e of `bits` is set, else y
__device__ __forceinline__ float where_bit(uint32_t bits, int e, float x, float y) {
  const uint32_t m = static_cast<uint32_t>(static_cast<int32_t>(bits << (31 - e)) >> 31);
  return __uint_as_float((__float_as_uint(x) & m) | (__float_as_uint(y) & ~m));
}

struct Penalties {
  float rho, alpha, beta;
  float up, div, inv;   // a power of two, rho up, 1 / (rho up): rho may be any positive number
};
__device__ __forceinline__ Penalties penalties(float rho, float alpha, float beta) {
  const float up = rho < 0x1p-100f ? 0x1p64f : rho > 0x1p100f ? 0x1p-64f : 1.0f;
  auto uniform = [](float x) {
    return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(x)));
  };
  return {uniform(rho), uniform(alpha), uniform(beta),
          uniform(up),  uniform(rho * up), uniform(1.0f / (rho * up))};
}

// z / rho or z * rho. The quotient is the product with the reciprocal, at most the largest
// number, corrected by its own remainder: it rounds as the division does, to infinity too
// (but for the last bit of subnormal quotients).
__device__ __forceinline__ float repeated(float z, const Penalties& p) {
  const float n = z * p.up, q = fminf(n * p.inv, 0x1.fffffep127f);
  const float d = fmaf(fmaf(-q, p.div, n), p.inv, q);
  return z > 0.0f ? d : z * p.rho;
}

// what presence, frequency and bias take off (each operation rounded by itself)
__device__ __forceinline__ float taken(int n, float bias, const Penalties& p) {
#pragma clang fp contract(off)
  const float a = n > 0 ? p.alpha : 0.0f;
  const float b = p.beta * static_cast<float>(n);
  return (a + b) - bias;
}

struct Params {
  tv::LogitsArgs a;
  int chunks, slabs, rows;   // rows of a slab
  float* part_max;           // [batch][num_nodes][chunks][wavefront]
  float* part_sum;
  float k32;                 // log2(e) / T rounded to fp32
  long long first_row;       // of the launch that merges
};

// kMasks: nodes have masks.
template <class T, bool kMasks>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 4 : 3) logits_kernel(Params P) {
  const tv::LogitsArgs& a = P.a;
  __shared__ uint32_t words[kChunk];
  // Place in this chunk and the token's bias entry, counted from 1 (0: none), or -1. (64 trees
  // of 65 nodes with 16 / 10000 biases 491 / 502 us; with a search of the list for every
  // drafted token 610 / 49500.)
  __shared__ int32_t toks[TV_MAX_NODES];
  __shared__ int16_t ups[TV_MAX_NODES];    // nearest proper ancestor with a token in this chunk, or 0
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int chunk = blockIdx.x % P.chunks, rest = blockIdx.x / P.chunks;
  const int slab = rest % P.slabs, b = rest / P.slabs;
  const int V = a.vocab, n1 = a.num_nodes;
  const int base = chunk * kChunk, width = min(kChunk, V - base);
  const Penalties pen = penalties(a.repetition ? a.repetition[b] : 1.0f,
                                  a.presence ? a.presence[b] : 0.0f,
                                  a.frequency ? a.frequency[b] : 0.0f);
  auto clear = [&] {
    for (int i = tid; i < kChunk / 4; i += kThreads)
      *reinterpret_cast<u32x4*>(&words[4 * i]) = u32x4{0, 0, 0, 0};
  };
  // token e of this thread (e < 32): its place in the chunk
  auto place = [&](int e) { return ((e >> 3) * kThreads + tid) * 8 + (e & 7); };

  const T* const in = static_cast<const T*>(a.logits);
  T* const to = static_cast<T*>(a.out);
  const int mask_words = (V + 31) / 32;
  const int r0 = a.first_node + slab * P.rows;
  const int r1 = min(r0 + P.rows, a.first_node + a.num_rows);
  const T ninf = stored<T>(-INFINITY);
  auto row_of = [&](int i) { return static_cast<size_t>(b) * n1 + i; };
  auto load = [&](int i, Raw<T> (&raw)[kGroups]) {
    const T* p = in + row_of(i) * V + base;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int at = (g * kThreads + tid) * 8;
      if (at + 8 <= width) {
        raw[g].load(p + at);
      } else {
        // a row's last few tokens
        T x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = at + e < width ? p[at + e] : ninf;
        __builtin_memcpy(&raw[g], x, sizeof x);
      }
    }
  };
  Raw<T> next[kGroups];
  load(r0, next);             // (under way while the counts are formed)

  // biases: of several entries for a token the last one
  float off[kOwn];
#pragma unroll
  for (int e = 0; e < kOwn; ++e) off[e] = 0.0f;
  const float* bias = a.bias_values + static_cast<size_t>(b) * a.max_bias;
  const int32_t* bias_at = a.bias_tokens + static_cast<size_t>(b) * a.max_bias;
  const int nbias = a.bias_tokens ? a.max_bias : 0;
  // the tree's tokens that lie in this chunk, and the links between them
  auto tree = [&](bool biased) {
    if (a.parents)
      for (int i = tid; i < n1; i += kThreads) {
        const size_t at = static_cast<size_t>(b) * n1 + i;
        const unsigned t = static_cast<unsigned>(a.tokens[at]) - base;
        const bool here = i > 0 && t < static_cast<unsigned>(width);
        toks[i] = here ? static_cast<int>(t | (biased ? words[t] * kChunk : 0)) : -1;
        const int p = a.parents[at];
        ups[i] = static_cast<int16_t>(p > 0 && p < i ? p : 0);
      }
  };
  clear();
  if (nbias) {
    __syncthreads();
    for (int j = tid; j < nbias; j += kThreads) {
      const unsigned t = static_cast<unsigned>(bias_at[j]) - base;
      if (t < static_cast<unsigned>(width)) atomicMax(&words[t], static_cast<uint32_t>(j + 1));
    }
    __syncthreads();
    // (few threads have any)
    uint32_t any = 0;
#pragma unroll
    for (int e = 0; e < kOwn; ++e) any |= words[place(e)];
    if (any) {
#pragma unroll
      for (int e = 0; e < kOwn; ++e) {
        const uint32_t j = words[place(e)];
        if (j) off[e] = bias[j - 1];
      }
    }
    tree(true);
    __syncthreads();
    clear();
  } else {
    tree(false);
  }
  __syncthreads();
  if (a.history) {
    const int32_t* h = a.history + static_cast<size_t>(b) * a.max_history;
    const int n = min(max(a.history_len[b], 0), a.max_history);
    const int np = a.prompt_len ? min(max(a.prompt_len[b], 0), n) : 0;
    for (int j = tid; j < n; j += kThreads) {
      const unsigned t = static_cast<unsigned>(h[j]) - base;
      if (t < static_cast<unsigned>(width)) {
        if (j < np)
          atomicOr(&words[t], kTold);
        else
          atomicAdd(&words[t], 1u);
      }
    }
  }
  // Links skip nodes whose token is elsewhere: a few steps of every node's path at
  // first, which do for most trees, then by doubling (any ancestor read meanwhile is one).
  if (a.parents) {
    constexpr int kSteps = 8, kPer = TV_MAX_NODES / kThreads;
    int16_t up[kPer];
    bool more = false;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int i = tid + k * kThreads;
      if (i >= n1) break;
      int u = ups[i];
      for (int step = 0; step < kSteps && u > 0 && toks[u] < 0; ++step) u = ups[u];
      up[k] = static_cast<int16_t>(u);
      more |= u > 0 && toks[u] < 0;
    }
    more = __syncthreads_or(more);
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (tid + k * kThreads < n1) ups[tid + k * kThreads] = up[k];
    __syncthreads();
    while (more) {
      more = false;
      for (int i = tid; i < n1; i += kThreads) {
        const int u = ups[i];
        if (u > 0 && toks[u] < 0) {
          ups[i] = ups[u];
          more = true;
        }
      }
      more = __syncthreads_or(more);
    }
  } else {
    __syncthreads();
  }
  uint32_t seen = 0;
#pragma unroll
  for (int e = 0; e < kOwn; ++e) {
    const uint32_t w = words[place(e)];
    seen |= static_cast<uint32_t>(w != 0) << e;
    off[e] = taken(static_cast<int>(w & ~kTold), off[e], pen);
  }

  for (int i = r0; i < r1; ++i) {
    Raw<T> raw[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) raw[g] = next[g];
    if (i + 1 < r1) load(i + 1, next);
    const size_t row = row_of(i);
    asm volatile("" : "+v"(seen));     // 32 lane masks would not fit the scalar registers
    // this thread's tokens that are on the path
    uint32_t mine = 0;
    int first = 0;
    if (a.parents) {
      first = toks[i] >= 0 ? i : ups[i];
      for (int x = first; x > 0; x = ups[x]) {
        const int t = toks[x] & (kChunk - 1);
        if (((t >> 3) & (kThreads - 1)) == tid) mine |= 1u << (t / (8 * kThreads) * 8 + (t & 7));
      }
    }
    // this thread's allowed tokens
    uint32_t allowed = ~0u;
    if constexpr (kMasks) {
      const int m = a.mask_index[row];
      if (m >= a.num_masks) {
        allowed = 0;
      } else if (m >= 0) {
        const uint8_t* bytes = reinterpret_cast<const uint8_t*>(
            a.masks + static_cast<size_t>(m) * mask_words) + base / 8;
        allowed = 0;
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
          if ((g * kThreads + tid) * 8 < width)
            allowed |= uint32_t{bytes[g * kThreads + tid]} << (8 * g);
      }
    }
    float v[kGroups][8];
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float z = raw[g].at(e);
        const float x = where_bit(seen, 8 * g + e, repeated(z, pen), z) - off[8 * g + e];
        v[g][e] = kMasks ? where_bit(allowed, 8 * g + e, x, -INFINITY) : x;
      }
    for (uint32_t left = mine & allowed; left; left &= left - 1) {
      const int e = __builtin_ctz(left), t = place(e);
      int n = static_cast<int>(words[t] & ~kTold), entry = 0;
      for (int x = first; x > 0; x = ups[x]) {
        const int w = toks[x];
        if ((w & (kChunk - 1)) != t) continue;
        ++n;
        entry = w / kChunk;
      }
      const float add = entry ? bias[entry - 1] : 0.0f;
      const float x = repeated(value(in[row * V + base + t]), pen) - taken(n, add, pen);
#pragma unroll
      for (int g = 0; g < kGroups; ++g)
#pragma unroll
        for (int k = 0; k < 8; ++k) v[g][k] = 8 * g + k == e ? x : v[g][k];
    }
    T* q = to + row * V + base;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int at = (g * kThreads + tid) * 8;
      if (at + 8 <= width) {
        store8(q + at, v[g]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (at + e < width) q[at + e] = stored<T>(v[g][e]);
      }
    }
    if (!P.part_max) continue;
    float mx = -INFINITY;
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[g][e] = value(stored<T>(v[g][e]));   // (-inf past the vocabulary, as loaded)
        mx = fmaxf(mx, v[g][e]);
      }
    mx = over_wave(mx, [](float x, float y) { return fmaxf(x, y); });
    // a row with no finite value keeps the frame 0, so its terms are 0 as well
    const float f = mx > -INFINITY ? -mx * P.k32 : 0.0f;
    const bool near = fabsf(f) < kFrames;
    const float from = near ? 0.0f : mx, c = near ? f : 0.0f;
    float s = 0.0f;
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += __builtin_amdgcn_exp2f(fmaf(v[g][e] - from, P.k32, c));
    s = over_wave(s, [](float x, float y) { return x + y; });
    if (lane == 0) {
      const size_t part = (row * P.chunks + chunk) * kWaves + wave;
      P.part_max[part] = mx;
      P.part_sum[part] = s;
    }
  }
}

// The frame of a sum: the rounded product, or the exact one (see above).
__device__ __forceinline__ double frame_of(float m, float k) {
  const float c = -m * k;
  return fabsf(c) < kFrames ? static_cast<double>(c) : -static_cast<double>(m) * static_cast<double>(k);
}

// Merges a row's partials, a wavefront a row: each moves from its frame to that of the
// row's maximum.
__global__ void __launch_bounds__(kThreads) logits_merge_kernel(Params P) {
  const tv::LogitsArgs& a = P.a;
  const int lane = threadIdx.x & 63;
  const long long r = P.first_row + static_cast<long long>(blockIdx.x) * kWaves + (threadIdx.x >> 6);
  if (r >= static_cast<long long>(a.batch) * a.num_rows) return;
  const long long b = r / a.num_rows;
  const size_t row = static_cast<size_t>(b) * a.num_nodes + a.first_node + (r - b * a.num_rows);
  const int parts = P.chunks * kWaves;
  const float* pm = P.part_max + row * parts;
  const float* ps = P.part_sum + row * parts;
  float m = -INFINITY;
  for (int t = lane; t < parts; t += 64) m = fmaxf(m, pm[t]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  const double cm = frame_of(m, P.k32);
  double s = 0.0;
  for (int t = lane; t < parts; t += 64) {
    const float mt = pm[t];
    const double st = static_cast<double>(ps[t]);
    s += mt > -INFINITY ? st * exp2(cm - frame_of(mt, P.k32)) : st;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if (lane == 0) {
    a.row_max[row] = m;
    // from the rounded frame to the exact one of the maximum
    a.row_sum[row] = m > -INFINITY && isfinite(m)
                         ? s * exp2(-(cm + static_cast<double>(m) * static_cast<double>(P.k32)))
                         : s;
  }
}

template <class T>
hipError_t run(const Params& P, unsigned grid, hipStream_t stream) {
  if (P.a.mask_index)
    hipLaunchKernelGGL((logits_kernel<T, true>), dim3(grid), dim3(kThreads), 0, stream, P);
  else
    hipLaunchKernelGGL((logits_kernel<T, false>), dim3(grid), dim3(kThreads), 0, stream, P);
  return hipGetLastError();
}

// Workgroups that fill the device: four on a CU, or three of fp32 (their rows take more
// registers). Each counts its chunk's history anew, so more of them cost more than they
// gain: 16 trees of 41 nodes in float32 45.4 us, with twice as many 49.0, with half 49.4
// (one tree of 65 in bfloat16 within 3% by all three).
constexpr int kEnough = 1024, kEnoughF32 = 768;

// Workgroups of a launch: one has fewer than 2^32 threads.
constexpr int64_t kMostGroups = (int64_t{1} << 24) - 1;

}  // namespace

namespace tv {

int launch_logits(const LogitsArgs& a, void* workspace, hipStream_t stream) {
  const LogitsLayout L = logits_layout(a.batch, a.num_nodes, a.vocab);
  Params P{};
  P.a = a;
  P.chunks = L.chunks;
  if (a.row_max) {
    P.part_max = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + L.off_max);
    P.part_sum = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + L.off_sum);
  }
  P.k32 = static_cast<float>(1.4426950408889634 / static_cast<double>(a.temperature));
  const int64_t per = static_cast<int64_t>(a.batch) * P.chunks;
  const int64_t want = ((a.dtype == TV_DTYPE_BF16 ? kEnough : kEnoughF32) + per - 1) / per;
  P.slabs = static_cast<int>(want < a.num_rows ? want : a.num_rows);
  P.rows = (a.num_rows + P.slabs - 1) / P.slabs;
  P.slabs = (a.num_rows + P.rows - 1) / P.rows;
  if (per * P.slabs > kMostGroups) return TV_ERR_UNSUPPORTED;
  const unsigned grid = static_cast<unsigned>(per * P.slabs);
  const hipError_t e = a.dtype == TV_DTYPE_BF16 ? run<uint16_t>(P, grid, stream)
                                                : run<float>(P, grid, stream);
  if (e != hipSuccess) return TV_ERR_HIP;
  if (!a.row_max) return TV_OK;
  const int64_t rows = static_cast<int64_t>(a.batch) * a.num_rows;
  constexpr int64_t kMost = kMostGroups * kWaves;   // rows of a launch
  for (P.first_row = 0; P.first_row < rows; P.first_row += kMost) {
    const int64_t n = rows - P.first_row < kMost ? rows - P.first_row : kMost;
    hipLaunchKernelGGL(logits_merge_kernel, dim3(static_cast<unsigned>((n + kWaves - 1) / kWaves)),
                       dim3(kThreads), 0, stream, P);
    if (hipGetLastError() != hipSuccess) return TV_ERR_HIP;
  }
  return TV_OK;
}

}  // namespace tv
