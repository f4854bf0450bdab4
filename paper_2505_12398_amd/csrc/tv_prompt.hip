// Causal attention of packed prompts for gfx950 (tv_prompt_attention).
//
// The query rows of a sequence and key head, (position, head of the group) in that order, are
// the columns of a product with the keys: per 32 keys a wavefront forms S^T = K Q^T for its 64
// rows (32x32x16 products), takes 2^(s k - m k) with k = scale log2(e) in the frame of a running
// maximum m, and adds V^T P^T to its accumulators (out = sum p v / sum p). A lane holds four
// consecutive keys of one row at a time, which is how the second product wants its operand, the
// keys taken in the order in which the lanes hold them; values are read transposed from LDS.
// Frames and the rounding of weights are those of tv_tree_attention.
//
// A wavefront has its SIMD to itself, and so all its registers: queries and accumulators in those
// that the vector unit does not compute in, scores, weights and operands in the others. In step j
// it multiplies tile j + 1's keys, takes tile j's weights and adds tile j - 1's values, in one
// order of instructions in which the matrix unit always has a product to run beside the vector
// unit's work (16384 tokens: one after the other 4215 us, so 1905 on the same card). 36 products of 32
// cycles a step of 32 keys, row sums among them, as products with ones (dot products in the vector unit
// would hold up the matrix unit). Tiles come into LDS three steps ahead.
//
// What bounds it. One prompt of 16384 tokens, 32 heads over 8 of 128: 1855 us (in other runs, on other
// cards, up to 1980), 1185 TFLOP/s of the 1612 that a large product reaches: a step takes 1550 to 1650
// cycles of which the matrix unit is busy 1152 (the clock falls to 1.8 or 1.9 GHz meanwhile). An item
// costs 13 thousand cycles before its first step, nine of them the queries' loads, and 6 behind its
// last: 32 prompts of 20 to 3000 tokens 1056 us (to 1109), 795 TFLOP/s. Few items are bound by the
// longest: four pieces behind long contexts have 350 items for 256 CUs, 214 us (to 241), and a piece of
// 16 tokens behind 16000 has 8 that walk all keys, 178 us. One prompt of 100 tokens: 13 us, waits for
// queries, first keys and the other key group's part.
//
// The call of careful_item gives the kernel a stack, 264 to 652 bytes a lane that no other path touches;
// the runtime reserves them for all lanes of the device, 330 MB, at a hardware queue's first launch.
#include <hip/hip_runtime.h>
#include <math.h>

#include <mutex>

#include "tv.h"
#include "tv_attention_common.h"
#include "tv_launch.h"

namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16;

constexpr int kKeys = 32;                 // keys of a tile
constexpr int kWaveRows = 64, kWaves = 4, kThreads = 64 * kWaves;

struct Item {                             // rows tile * BM .. of a sequence's query rows
  int q0, nq, k0, nk, tile, pad[3];
};

struct Pass {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* out;
  int64_t q_stride, kv_stride;            // elements
  const int32_t* q_start;
  const int32_t* k_start;
  int batch, num_queries, num_keys, heads, kv_heads, head_dim, group;
  float k2;                               // scale log2(e)
  float slack;                            // how far a score may exceed its frame
  Item* items;                            // in the order in which they begin (NULL: one sequence)
  int* count;                             // of items
};

template <class T>
__device__ __forceinline__ f32x16 mfma32(s16x8 a, s16x8 b, f32x16 c) {
  if constexpr (std::is_same<T, Bf16>::value)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// The same onto an accumulator in the registers that the vector unit does not compute in, which
// leaves the others to scores and weights. (In assembly: the compiler has one kind of register for
// all products. It does not see that the result is late: settle() stands before the vector unit
// reads or writes accumulators; products among themselves wait for each other.)
template <class T>
__device__ __forceinline__ void accumulate(s16x8 a, s16x8 b, f32x16& c) {
  if constexpr (std::is_same<T, Bf16>::value)
    asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
  else
    asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}
// The sums: ones from a register that is theirs for good. (A constant is put into one right before
// the product, which reads it two instructions later at the earliest.)
template <class T>
__device__ __forceinline__ void accumulate_ones(s16x8 ones, s16x8 b, f32x16& c) {
  if constexpr (std::is_same<T, Bf16>::value)
    asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(c) : "a"(ones), "v"(b));
  else
    asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+a"(c) : "a"(ones), "v"(b));
}
template <int DB, int MT>
__device__ __forceinline__ void settle(f32x16 (&c)[DB][MT]) {
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) asm volatile("s_nop 7\n\ts_nop 3" : "+a"(c[db][mt]));
}

// RW row groups of 64 rows, KW key groups that take the tiles in turn and are merged at the end.
template <int DP_, int RW_>
struct Shape {
  static constexpr int DP = DP_, RW = RW_, KW = kWaves / RW_;
  static constexpr int BM = kWaveRows * RW;
  static constexpr int MT = 2;                       // blocks of 32 rows of a wavefront
  static constexpr int KK = DP / 16, DB = DP / 32;   // steps of the first product, blocks of the second
  static constexpr int CH = DP / 8, ROW = DP * 2;    // 16-byte chunks and bytes of a row
  static constexpr int MAT = kKeys * ROW, STAGE = 2 * MAT;
  static constexpr int LOADS = MAT / 1024 / RW;      // of a wavefront, for a tile's keys (or values)
  static constexpr int S = 4;                        // tiles in LDS per key group
  // Operands of a step: keys of the tile behind, values of the one before, each for MT products.
  static constexpr int NK = KK, NV = 2 * DB, OPS = NK + NV;
  static constexpr int AHEAD = 3;                    // operands read before they are multiplied
  // (the next step's first ones among them)
  static constexpr int WAIT = LOADS * (2 * (S - 3) + 1);
  static_assert(OPS % (AHEAD + 1) == 0, "places of operands are the same in every step");
  static constexpr int RING = KW * S * STAGE;
  static constexpr int ACC = (KW - 1) * RW * MT * DB * 4096;
  static constexpr int MERGE = ACC + (KW - 1) * RW * MT * 64 * 8;
  static constexpr int MAIN = RING > MERGE ? RING : MERGE;
  static constexpr int FLAGS = MAIN, MARKS = FLAGS + 4 * kWaves, BYTES = MARKS + kWaves * DP * 4;
  static constexpr int PER_CU = 1;        // workgroups
  static_assert(BYTES <= 160 * 1024, "LDS of a CU");
  static_assert(WAIT < 64, "the count of loads in flight");
};

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// A wavefront's part of a tile's keys, or values, into LDS: 1024 bytes at dst, and so on. (Without the
// wait states of load_to_lds: the scalars come from the scalar unit, which the generated code is
// tested for.)
template <int N>
__device__ __forceinline__ void load_tile(const i32x4& rs, const int (&voff)[N], int dst) {
#pragma unroll
  for (int i = 0; i < N; ++i)
    asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :: "s"(dst), "v"(voff[i]), "s"(rs), "n"(i * 1024) : "memory", "m0", "scc");
}
#pragma clang diagnostic pop

// Starts are kept within the tensors.
__device__ __forceinline__ int clamped(int x, int lo, int hi) { return min(max(x, lo), hi); }

// Swizzle of a tile's rows in LDS: a chunk of sixteen rows, and four chunks of four rows, touch all
// banks once.
template <int DP>
__device__ __forceinline__ int swizzle(int r) {
  return DP == 128 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 2 & 3);
}

// The end of an item: the key groups' parts merged by group 0, and its rows written. CAREFUL: the sums are
// without what is not finite of the values v (those of the item's first key and key head), which is added
// here, whatever its weight rounds to. odd: 1 if some key from `from` on, which not all rows of the
// wavefront see, has such values, 2 if one before it, whose sums are the marks in LDS.
template <class T, class SH, bool CAREFUL>
__device__ __forceinline__ void finish(lds_byte* lds, f32x16 (&acc)[SH::DB + 1][SH::MT], float (&m)[SH::MT],
                                       const int (&limit)[SH::MT], int odd, const uint16_t* v, int64_t kv_stride,
                                       uint16_t* out, int heads, int head_dim, int group, float k2, int kh, int q0,
                                       int rows, int rbase, int from) {
  constexpr int MT = SH::MT, RW = SH::RW, KW = SH::KW, DB = SH::DB;
  const int lane = threadIdx.x & 63, wave = uniform(static_cast<int>(threadIdx.x >> 6));
  const int rg = wave % RW, kg = wave / RW, n = lane & 31, h = lane >> 5;
  LDS(int)* const flags = (LDS(int)*)(lds + SH::FLAGS);
  LDS(float)* const marks = (LDS(float)*)(lds + SH::MARKS);
  float l[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) l[mt] = acc[DB][mt][0];
  if constexpr (KW > 1) {
    barrier();                            // (all have read the flags)
    if (CAREFUL && lane == 0) flags[wave] = odd;
    if (kg > 0) {
      const int w = (kg - 1) * RW + rg;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            *(LDS(f32x4)*)(lds + ((w * MT + mt) * DB + db) * 4096 + r * 1024 + lane * 16) =
                f32x4{acc[db][mt][4 * r], acc[db][mt][4 * r + 1], acc[db][mt][4 * r + 2], acc[db][mt][4 * r + 3]};
        *(LDS(f32x2)*)(lds + SH::ACC + (w * MT + mt) * 512 + lane * 8) = f32x2{m[mt], l[mt]};
      }
    }
    barrier();
    if (kg > 0) return;
#pragma unroll
    for (int j = 1; CAREFUL && j < KW; ++j) odd |= flags[j * RW + rg];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      f32x2 o[KW];
      float top = m[mt];
#pragma unroll
      for (int j = 1; j < KW; ++j) {
        o[j] = *(const LDS(f32x2)*)(lds + SH::ACC + (((j - 1) * RW + rg) * MT + mt) * 512 + lane * 8);
        top = fmaxf(top, o[j][0]);
      }
      const float f = to_frame<T>(m[mt], top, k2);
      l[mt] *= f;
#pragma unroll
      for (int db = 0; db < DB; ++db) acc[db][mt] *= f;
#pragma unroll
      for (int j = 1; j < KW; ++j) {
        const float fj = to_frame<T>(o[j][0], top, k2);
        l[mt] += o[j][1] * fj;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const f32x4 x = *(const LDS(f32x4)*)(
                lds + ((((j - 1) * RW + rg) * MT + mt) * DB + db) * 4096 + r * 1024 + lane * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[db][mt][4 * r + e] += fj * x[e];
          }
      }
    }
  }
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int r = rbase + 32 * mt + n;
    if (r >= rows) continue;
    const int x = r / group, g = r - x * group;
    uint16_t* const to = out + (static_cast<int64_t>(q0 + x) * heads + kh * group + g) * head_dim;
    const float inv = limit[mt] >= 0 ? 1.0f / l[mt] : 0.0f;   // (a row that sees nothing is 0)
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int d = 32 * db + 8 * i + 4 * h;
        if (d >= head_dim) continue;
        float o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = acc[db][mt][4 * i + e] * inv;
        if (CAREFUL && odd & 2) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x = 0.0f;
#pragma unroll
            for (int j = 0; j < KW; ++j) x += marks[(j * RW + rg) * SH::DP + d + e];
            if (x != 0.0f) o[e] += x;     // (-0 stays)
          }
        }
        if (CAREFUL && odd & 1) {
#pragma unroll 1
          for (int j = from; j <= limit[mt]; ++j) {
            const u32x2 w = *reinterpret_cast<const u32x2*>(v + static_cast<int64_t>(j) * kv_stride + d);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t u = w[e >> 1] >> (16 * (e & 1)) & 0xffffu;
              if ((u & T::kExponent) == T::kExponent) o[e] += T::value(static_cast<uint16_t>(u));
            }
          }
        }
        *reinterpret_cast<u32x2*>(to + d) = u32x2{T::pack(o[0], o[1]), T::pack(o[2], o[3])};
      }
  }
}

// An item whose keys or values hold what is not finite, a tile of each key group at a time: values are
// taken as 0 where they are not finite, and added to the rows that see them when these are written. (A
// weight that rounds to 0 would make NaN of an infinite one.) The same sums in the same order as in the
// kernel, so that the rows and the elements that see none of it keep their bits. Not inlined: the
// registers of the kernel are laid out for the other path.
template <class T, class SH>
__device__ __attribute__((noinline))
void careful_item(lds_byte* lds, const uint16_t* pq, const uint16_t* pk, const uint16_t* pv, uint16_t* out,
                  int64_t q_stride, int64_t kv_stride, int heads, int head_dim, int group, int kh, int q0, int nq,
                  int k0, int nk, int tile, float k2, float slack) {
  constexpr int MT = SH::MT, RW = SH::RW, KW = SH::KW, KK = SH::KK, DB = SH::DB;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int rg = wave % RW, kg = wave / RW, n = lane & 31, h = lane >> 5;
  const int rows = nq * group, r0 = tile * SH::BM, rbase = r0 + rg * kWaveRows, ctx = nk - nq;
  auto position = [&](int r) { return min(r, rows - 1) / group; };
  const int tiles = uniform((max(0, position(r0 + SH::BM - 1) + ctx + 1) + kKeys - 1) / kKeys);
  const int nfull = uniform(max(0, position(rbase) + ctx + 1) / kKeys);
  s16x8 q[MT][KK];
  int limit[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int r = min(rbase + 32 * mt + n, rows - 1), x = r / group, g = r - x * group;
    limit[mt] = x + ctx;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const int d = 16 * kk + 8 * h;
      q[mt][kk] = d < head_dim ? *reinterpret_cast<const s16x8*>(
                                     pq + static_cast<int64_t>(q0 + x) * q_stride + (kh * group + g) * head_dim + d)
                               : s16x8{};
    }
  }
  const int64_t first = static_cast<int64_t>(k0) * kv_stride + kh * head_dim;
  const int at0 = kg * SH::STAGE;         // of this key group's tile
  const int k_at = at0 + n * SH::ROW + (h ^ swizzle<SH::DP>(n & 15)) * 16;
  const int vrow = 4 * h + ((lane & 15) >> 2), vchunk = 2 * (lane >> 4 & 1) + ((lane & 3) >> 1);
  const s16x8 ones = T::ones();
  float m[MT], c[MT];
  f32x16 acc[DB + 1][MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    m[mt] = -INFINITY;
    c[mt] = 0.0f;
#pragma unroll
    for (int db = 0; db <= DB; ++db) acc[db][mt] = f32x16{};
  }
  int odd = 0;
  // sums of what the wavefront's tiles that all its rows see hold, an element of the head each
  LDS(float)* const marks = (LDS(float)*)(lds + SH::MARKS) + wave * SH::DP;
#pragma unroll
  for (int i = 0; i < SH::DP / 64; ++i) marks[64 * i + lane] = 0.0f;
#pragma unroll 1
  for (int t0 = 0; t0 < tiles; t0 += KW) {
    const int t = t0 + kg;
    __syncthreads();
    for (int i = rg * 64 + lane; i < 2 * kKeys * SH::CH; i += 64 * RW) {
      const int ch = i % SH::CH, r = i / SH::CH % kKeys, values = i / (SH::CH * kKeys), j = t * kKeys + r;
      u32x4 w = {0, 0, 0, 0};
      if (j < nk && 8 * ch < head_dim)
        w = *reinterpret_cast<const u32x4*>((values ? pv : pk) + first + static_cast<int64_t>(j) * kv_stride + 8 * ch);
      *(LDS(u32x4)*)(lds + at0 + values * SH::MAT + r * SH::ROW + (ch ^ swizzle<SH::DP>(r & 15)) * 16) = w;
    }
    __syncthreads();
    f32x16 s[MT] = {};
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const s16x8 a = *(const LDS(s16x8)*)(lds + (k_at ^ (32 * kk)));
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) s[mt] = mfma32<T>(a, q[mt][kk], s[mt]);
    }
    u32x4 p[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int last = limit[mt] - t * kKeys - 4 * h;
      float top = -INFINITY;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[mt][r] = 8 * (r >> 2) + (r & 3) <= last ? s[mt][r] : -INFINITY;
        top = __builtin_elementwise_maximum(top, s[mt][r]);
      }
      const float above = m[mt] + slack;
      float u = fmaxf(m[mt], top);
      u = fmaxf(u, __shfl_xor(u, 32, 64));
      u = u > above ? u : m[mt];
      const float f = to_frame<T>(m[mt], u, k2);
      if (u > m[mt]) {
#pragma unroll
        for (int db = 0; db <= DB; ++db) acc[db][mt] *= f;
      }
      m[mt] = u;
      c[mt] = frame<T>(u, k2);
#pragma unroll
      for (int r = 0; r < 16; r += 2)
        p[mt][r / 8][r % 8 / 2] = T::pack(__builtin_amdgcn_exp2f(fmaf(s[mt][r], k2, c[mt])),
                                          __builtin_amdgcn_exp2f(fmaf(s[mt][r + 1], k2, c[mt])));
    }
#pragma unroll
    for (int i = 0; i < SH::NV; ++i) {
      const int at = at0 + SH::MAT + (16 * (i & 1) + vrow) * SH::ROW + 8 * (lane & 1), ch = 4 * (i >> 1);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (LDS(s16x4)*)(lds + at + ((ch + vchunk) ^ swizzle<SH::DP>(vrow)) * 16));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (LDS(s16x4)*)(lds + at + 8 * SH::ROW + ((ch + vchunk) ^ swizzle<SH::DP>(vrow + 8)) * 16));
      u32x4 w = __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      bool some = false;
      float mark = 0.0f;                  // (this lane's eight values are of one element)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool a = (w[e] & T::kExponent) == T::kExponent, b = (w[e] >> 16 & T::kExponent) == T::kExponent;
        some |= a | b;
        mark += a ? T::value(static_cast<uint16_t>(w[e])) : 0.0f;
        mark += b ? T::value(static_cast<uint16_t>(w[e] >> 16)) : 0.0f;
        w[e] = (a ? 0 : w[e] & 0xffffu) | (b ? 0 : w[e] & 0xffff0000u);
      }
      if (__builtin_amdgcn_ballot_w64(some)) {
        odd |= t < nfull ? 2 : 1;
        mark += __shfl_xor(mark, 32, 64);
        if (t < nfull && h == 0) marks[32 * (i >> 1) + n] += mark;
      }
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        acc[i >> 1][mt] = mfma32<T>(__builtin_bit_cast(s16x8, w), __builtin_bit_cast(s16x8, p[mt][i & 1]), acc[i >> 1][mt]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        acc[DB][mt] = mfma32<T>(ones, __builtin_bit_cast(s16x8, p[mt][i]), acc[DB][mt]);
  }
  __syncthreads();
  finish<T, SH, true>(lds, acc, m, limit, odd, pv + first, kv_stride, out, heads, head_dim, group, k2, kh, q0, rows,
                rbase, nfull * kKeys);
}

template <class T, class SH>
__global__ void __launch_bounds__(kThreads, SH::PER_CU) prompt_kernel(Pass P) {
  constexpr int MT = SH::MT, RW = SH::RW, KW = SH::KW, KK = SH::KK, DB = SH::DB;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[SH::BYTES];
  lds_byte* const lds = (lds_byte*)smem;
  const int lds0 = static_cast<int>(reinterpret_cast<uintptr_t>(lds));
  const int lane = threadIdx.x & 63, wave = uniform(static_cast<int>(threadIdx.x >> 6));
  const int rg = wave % RW, kg = wave / RW;
  const int n = lane & 31, h = lane >> 5;

  // the item: consecutive workgroups, and so the XCDs in turn, take its key heads
  const int rank = blockIdx.x / P.kv_heads, kh = blockIdx.x - rank * P.kv_heads;
  Item I;
  // (read through the scalar cache: nothing of this launch writes them)
  if (P.items) {
    CONSTANT(Item)* const items = (CONSTANT(Item)*)P.items;
    if (rank >= *(CONSTANT(int)*)P.count) return;
    I.q0 = items[rank].q0;
    I.nq = items[rank].nq;
    I.k0 = items[rank].k0;
    I.nk = items[rank].nk;
    I.tile = items[rank].tile;
  } else {
    CONSTANT(int)* const qs = (CONSTANT(int)*)P.q_start;
    CONSTANT(int)* const ks = P.k_start ? (CONSTANT(int)*)P.k_start : qs;
    I.q0 = clamped(qs[0], 0, P.num_queries);
    I.nq = clamped(qs[1], I.q0, P.num_queries) - I.q0;
    I.k0 = clamped(ks[0], 0, P.num_keys);
    I.nk = clamped(ks[1], I.k0, P.num_keys) - I.k0;
    const int tiles = (I.nq * P.group + SH::BM - 1) / SH::BM;
    if (rank >= tiles) return;
    I.tile = tiles - 1 - rank;            // the one with the most keys first
  }
  const int rows = I.nq * P.group;        // (of all sequences below 2^30)
  const int r0 = I.tile * SH::BM, rbase = r0 + rg * kWaveRows;
  const int ctx = I.nk - I.nq;            // row position x sees keys up to x + ctx
  auto position = [&](int r) { return min(r, rows - 1) / P.group; };
  const int need = max(0, position(r0 + SH::BM - 1) + ctx + 1);
  const int tiles = (need + kKeys - 1) / kKeys;
  // tiles that all rows of this wavefront see whole
  const int nfull = max(0, uniform(position(rbase)) + ctx + 1) / kKeys;

  // Loads: instruction i fills 1024 bytes, this lane the chunk at position lane % CH of row
  // i * 1024 / ROW + lane / CH.
  const int stride = static_cast<int>(P.kv_stride) * 2;
  const uint64_t step_bytes = static_cast<uint64_t>(KW) * kKeys * stride;
  int kv_off[SH::LOADS];
#pragma unroll
  for (int i = 0; i < SH::LOADS; ++i) {
    const int r = (rg * SH::LOADS + i) * (1024 / SH::ROW) + lane / SH::CH;
    const int c = (lane % SH::CH) ^ swizzle<SH::DP>(r);
    kv_off[i] = 8 * c < P.head_dim ? r * stride + 16 * c : kPastRange;
  }
  const int lds_own = lds0 + kg * SH::S * SH::STAGE + rg * SH::LOADS * 1024;
  const int64_t first = static_cast<int64_t>(I.k0) * P.kv_stride + kh * P.head_dim;
  const uint64_t k_base = reinterpret_cast<uint64_t>(P.k + first), v_base = reinterpret_cast<uint64_t>(P.v + first);
  // The key group's next tile to load, of keys and of values: where it is, and how many rows it and
  // those behind it have.
  struct Next {
    uint64_t at;
    int left;
  };
  Next keys = {k_base + static_cast<uint64_t>(kg) * kKeys * stride, I.nk - kg * kKeys};
  Next values = {v_base + static_cast<uint64_t>(kg) * kKeys * stride, keys.left};
  // (rows behind the sequence's last key are zeros, and so are tiles that are none)
  auto issue = [&](Next& x, int place, bool values) {
    int some = min(x.left, kKeys);
    asm("" : "+s"(some));                 // (else one instruction of the vector unit)
    const int range = max(some, 0) * stride;
    load_tile<SH::LOADS>(i32x4{static_cast<int>(x.at), static_cast<int>(x.at >> 32), range, 0x00020000}, kv_off,
                         lds_own + place + (values ? SH::MAT : 0));
    x.at += step_bytes;
    x.left -= KW * kKeys;
  };
  // Step j of a key group, whose tiles are kg, kg + KW, ..: the weights of its tile j, the scores of
  // tile j + 1, and the values of tile j - 1 times theirs, so that the matrix units have products that
  // wait for nothing while the vector units form weights. Once all have passed step j's barrier, the
  // places of K_j and V_{j-2} are free: K_{j+S} and V_{j+S-2} go there. All but the WAIT newest loads
  // have landed by then, so K_{j+1} and V_{j-1} are there (and K_{j+2}, whose first operands the end
  // of the step reads).
  const int rounds = (tiles + KW - 1) / KW;   // (of all wavefronts; without a tile of its own, one masks all)
  const int whole = (nfull - kg + KW - 1) / KW;   // (0 or less: none)
  auto place = [](int j) { return (j & (SH::S - 1)) * SH::STAGE; };
  static_assert((SH::S & (SH::S - 1)) == 0, "places of tiles");
#pragma unroll
  for (int j = -SH::S; j < 0; ++j) {
    issue(keys, place(j), false);
    if (j == 1 - SH::S) {                 // (V_-1 is zeros)
      Next none = {v_base, 0};
      issue(none, place(-1), true);
    } else if (j > 1 - SH::S) {
      issue(values, place(j + SH::S - 2), true);
    }
  }

  // queries
  s16x8 q[MT][KK];
  int limit[MT];                          // the last key that a row sees
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int r = min(rbase + 32 * mt + n, rows - 1);
    const int x = r / P.group, g = r - x * P.group;
    limit[mt] = x + ctx;
    const uint16_t* const src = P.q + static_cast<int64_t>(I.q0 + x) * P.q_stride +
                                (kh * P.group + g) * P.head_dim;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const int d = 16 * kk + 8 * h;
      q[mt][kk] = d < P.head_dim ? *reinterpret_cast<const s16x8*>(src + d) : s16x8{};
    }
  }

  // Reads: keys, row n and chunk 2 kk + h; values, keys 4 h .. 4 h + 3 of 16 by sixteen of the
  // head, lane i of sixteen the eight bytes i % 4 at key i / 4, transposed by the read.
  const int k_at = n * SH::ROW + (h ^ swizzle<SH::DP>(n & 15)) * 16;
  const int vrow = 4 * h + ((lane & 15) >> 2);
  const int v_at = vrow * SH::ROW + ((2 * (lane >> 4 & 1) + ((lane & 3) >> 1)) ^ swizzle<SH::DP>(vrow)) * 16 +
                   (lane & 1) * 8;
  const int v_hi = (vrow + 8) * SH::ROW +
                   ((2 * (lane >> 4 & 1) + ((lane & 3) >> 1)) ^ swizzle<SH::DP>(vrow + 8)) * 16 + (lane & 1) * 8;

  float m[MT], c[MT], above[MT];          // above: what a score moves the frame from
  // The last block is that of the sums: the weights times ones. (The vector unit would take 64
  // instructions a step for them, of 250; a dot product of two weights waits for the matrix unit.)
  f32x16 acc[DB + 1][MT];

  const int ring = kg * SH::S * SH::STAGE;
  int k_from[KK], v_from[DB][2];          // where operands lie in a key group's first place
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) k_from[kk] = here(ring + (k_at ^ (32 * kk)));
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    v_from[db][0] = here(ring + SH::MAT + (v_at ^ (64 * db)));
    v_from[db][1] = here(ring + SH::MAT + (v_hi ^ (64 * db)));
  }
  // (the place is a constant in the steps that count, an offset in their reads)
  auto key_operand = [&](int place, int kk) {
    return *(const LDS(s16x8)*)(lds + k_from[kk] + place);
  };
  auto value_operand = [&](int place, int i) {
    const int at = place + 16 * (i & 1) * SH::ROW, db = i >> 1;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS(s16x4)*)(lds + v_from[db][0] + at));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS(s16x4)*)(lds + v_from[db][1] + at));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto scores = [&](int stage, f32x16 (&s)[MT]) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) s[mt] = f32x16{};
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const s16x8 a = key_operand(stage, kk);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) s[mt] = mfma32<T>(a, q[mt][kk], s[mt]);
    }
  };
  // Where some score exceeds its row's frame: the new frames; what the sums so far are multiplied
  // with (the accumulators once they hold all weights of the old frames).
  auto move = [&](const float (&top)[MT], float (&f)[MT]) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      float u = fmaxf(m[mt], top[mt]);
      u = fmaxf(u, __shfl_xor(u, 32, 64));
      u = u > above[mt] ? u : m[mt];
      f[mt] = to_frame<T>(m[mt], u, P.k2);
      m[mt] = u;
      above[mt] = u + P.slack;
      c[mt] = frame<T>(u, P.k2);
    }
  };
  auto rescale = [&](const float (&f)[MT]) {
    settle(acc);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int db = 0; db <= DB; ++db) acc[db][mt] *= f[mt];
    settle(acc);
  };
  auto weight = [&](const f32x16 (&s)[MT], int mt, int r) {
    return __builtin_amdgcn_exp2f(fmaf(s[mt][r], P.k2, c[mt]));
  };
  auto largest = [&](const f32x16& s, int i, float top) {   // of two more
    return i == 0 ? __builtin_elementwise_maximum(s[0], s[1]) : max3(top, s[2 * i], s[2 * i + 1]);
  };

  s16x8 ones8 = T::ones();
  asm volatile("" : "+a"(ones8));

  // (left to the compiler, the queries' wait would be one for all loads in flight)
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) asm volatile("" : "+a"(q[mt][kk]));

  f32x16 s0[MT], s1[MT];
  u32x4 p0[MT][2], p1[MT][2];             // weights, two of a row in a word
  s16x8 op[SH::AHEAD + 1];                // operand i at i % (AHEAD + 1)
  // Whether the frames moved for a tile's scores, and what the accumulators are multiplied with for
  // it once the weights before it are in them.
  bool moved = false;
  float f[MT];
  auto look = [&](const float (&top)[MT]) {
    bool moves = false;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) moves |= top[mt] > above[mt];
    moved = __builtin_amdgcn_ballot_w64(moves) != 0;
    if (moved) move(top, f);
  };
  auto look_all = [&](const f32x16 (&s)[MT]) {
    float top[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int i = 0; i < 8; ++i) top[mt] = largest(s[mt], i, top[mt]);
    look(top);
  };
  // Keys of tile j that a row does not see.
  auto mask = [&](int j, f32x16 (&s)[MT]) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int last = limit[mt] - (kg + j * KW) * kKeys - 4 * h;
#pragma unroll
      for (int r = 0; r < 16; ++r)
        s[mt][r] = 8 * (r >> 2) + (r & 3) <= last ? s[mt][r] : -INFINITY;
    }
  };

  // Step j, J = j modulo 4; the frames are those of tile j. One product a slot, the vector
  // instructions spread over the slots. masked: some row may not see tile j + 1 whole.
  auto step = [&](auto J, auto masked, int j, f32x16 (&s)[MT], f32x16 (&next)[MT], const u32x4 (&p)[MT][2],
                  u32x4 (&pn)[MT][2]) {
    wait_loads<SH::WAIT>();
    barrier();
    auto read = [&](auto ic) {
      constexpr int i = ic.value;
      if constexpr (i < SH::NK) op[i % (SH::AHEAD + 1)] = key_operand(place(J + 1), i);
      else if constexpr (i < SH::OPS) op[i % (SH::AHEAD + 1)] = value_operand(place(J - 1), i - SH::NK);
      else op[i % (SH::AHEAD + 1)] = key_operand(place(J + 2), i - SH::OPS);
    };
    auto product = [&](auto ic, auto mtc) {
      constexpr int i = ic.value, mt = mtc.value, v = i - SH::NK;
      const s16x8 a = op[i % (SH::AHEAD + 1)];
      if constexpr (i < SH::NK)
        next[mt] = mfma32<T>(a, q[mt][i], i == 0 ? f32x16{} : next[mt]);
      else
        accumulate<T>(a, __builtin_bit_cast(s16x8, p[mt][v & 1]), acc[v >> 1][mt]);
      if constexpr (i >= SH::OPS - 2)
        accumulate_ones<T>(ones8, __builtin_bit_cast(s16x8, p[mt][v & 1]), acc[DB][mt]);
    };
    // two weights in a word, a pair after they are formed (their result is late)
    float e[3], top[MT];
    auto pack_pair = [&](int x) {
      uint32_t w = T::pack(e[x % 3], e[(x + 1) % 3]);
      asm volatile("" : "+v"(w));         // (here, and not where it is used)
      pn[x / 16][x % 16 / 8][x % 8 / 2] = w;
    };
    unrolled<SH::OPS * MT>([&](auto uc) {
      constexpr int u = uc.value, i = u / MT, mt = u % MT, kAll = SH::OPS * MT;
      if constexpr (mt == 0) read(std::integral_constant<int, i + SH::AHEAD>{});
      product(std::integral_constant<int, i>{}, std::integral_constant<int, mt>{});
      if constexpr (u == 1) issue(keys, place(J), false);
      if constexpr (u == kAll / 4) issue(values, place(J + SH::S - 2), true);
      constexpr int kWeights = 16 * MT;
#pragma unroll
      for (int x = u * kWeights / kAll; x < (u + 1) * kWeights / kAll; ++x) {
        e[x % 3] = weight(s, x / 16, x % 16);
        if (x % 2 == 0 && x > 0) pack_pair(x - 2);
      }
      // the next tile's scores are there a few products after their last one
      constexpr int kFrom = SH::NK * MT + 4, kPairs = 8 * MT;
      if constexpr (masked.value && u == kFrom)
        if (j + 1 >= whole) mask(j + 1, next);
      if constexpr (u >= kFrom) {
#pragma unroll
        for (int x = (u - kFrom) * kPairs / (kAll - kFrom); x < (u + 1 - kFrom) * kPairs / (kAll - kFrom); ++x) {
          top[x / 8] = largest(next[x / 8], x % 8, top[x / 8]);
          asm volatile("" : "+v"(top[x / 8]));
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    pack_pair(16 * MT - 2);
    if (moved) rescale(f);
    look(top);
  };
  // The last tile's values.
  auto add_last = [&](int place, const u32x4 (&p)[MT][2]) {
#pragma unroll
    for (int i = 0; i < SH::NV; ++i) {
      const s16x8 v = value_operand(place, i);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        accumulate<T>(v, __builtin_bit_cast(s16x8, p[mt][i & 1]), acc[i >> 1][mt]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        accumulate_ones<T>(ones8, __builtin_bit_cast(s16x8, p[mt][i]), acc[DB][mt]);
  };
  constexpr std::integral_constant<int, 0> j0{};
  constexpr std::integral_constant<int, 1> j1{};
  constexpr std::integral_constant<int, 2> j2{};
  constexpr std::integral_constant<int, 3> j3{};
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    m[mt] = above[mt] = -INFINITY;
    c[mt] = f[mt] = 0.0f;
    p0[mt][0] = p0[mt][1] = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int db = 0; db <= DB; ++db) acc[db][mt] = f32x16{};
  }
  settle(acc);
  wait_loads<SH::WAIT>();
  barrier();
  scores(place(0), s0);
  unrolled<SH::AHEAD>([&](auto i) { op[i.value] = key_operand(place(1), i.value); });
  if (whole < 1) mask(0, s0);
  look_all(s0);
  int j = 0;
#pragma unroll 1
  for (; j + 4 < whole; j += 4) {
    step(j0, std::false_type{}, j, s0, s1, p0, p1);
    step(j1, std::false_type{}, j + 1, s1, s0, p1, p0);
    step(j2, std::false_type{}, j + 2, s0, s1, p0, p1);
    step(j3, std::false_type{}, j + 3, s1, s0, p1, p0);
  }
#pragma unroll 1
  for (; j < rounds; ++j) {
    step(j, std::true_type{}, j, s0, s1, p0, p1);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      s0[mt] = s1[mt];
      p0[mt][0] = p1[mt][0];
      p0[mt][1] = p1[mt][1];
    }
  }
  wait_loads<0>();                        // (zeros for tiles that are none)
  barrier();
  add_last(place(rounds - 1), p0);
  settle(acc);

  // Weight 0 times a value that is not finite is NaN, and a row must not see the values behind it:
  // an item with a sum that is not finite is computed again, a tile at a time.
  float zero = 0.0f;                      // NaN if some sum is not finite
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) zero = fmaf(acc[db][mt][r], 0.0f, zero);
  LDS(int)* const flags = (LDS(int)*)(lds + SH::FLAGS);
  const uint64_t bad = __builtin_amdgcn_ballot_w64(zero != zero);
  if (lane == 0) flags[wave] = bad != 0;
  barrier();                              // (all have read their last tile, too)
  int any = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) any |= flags[w];
  if (__builtin_expect(uniform(any), 0)) {
    careful_item<T, SH>(lds, P.q, P.k, P.v, P.out, P.q_stride, P.kv_stride, P.heads, P.head_dim, P.group,
                        kh, I.q0, I.nq, I.k0, I.nk, I.tile, P.k2, P.slack);
    return;
  }

  finish<T, SH, false>(lds, acc, m, limit, 0, nullptr, 0, P.out, P.heads, P.head_dim, P.group, P.k2, kh, I.q0, rows,
                rbase, 0);
}

// The items of all sequences, those with the most keys first, so that none begins late and
// long. One workgroup: it counts the items of 1024 classes of keys, and puts them behind those
// of the classes above. (The order within a class is that of its atomics: no result depends
// on it.)
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64, kClasses = 1024;

template <class F>
__device__ __forceinline__ int block_scan(int x, F&& join, int zero, LDS(int)* part, int& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int s = x;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int o = __shfl_up(s, off, 64);
    if (lane >= off) s = join(s, o);
  }
  __syncthreads();
  if (lane == 63) part[wave] = s;
  __syncthreads();
  int before = zero;
  all = zero;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    if (w < wave) before = join(before, part[w]);
    all = join(all, part[w]);
  }
  return join(before, s);                 // up to and with this thread's
}

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(Pass P, int bm) {
  __shared__ int part_[kPlanWaves], classes_[kClasses];
  __shared__ int upto_[kPlanThreads], q0_[kPlanThreads + 1], k0_[kPlanThreads + 1], most_;
  LDS(int)* const part = (LDS(int)*)part_;
  const int tid = threadIdx.x;
  const int32_t* const ks = P.k_start ? P.k_start : P.q_start;
  auto larger = [](int a, int b) { return a > b ? a : b; };
  auto plus = [](int a, int b) { return a + b; };
  classes_[tid] = 0;
  if (tid == 0) most_ = 1;
  __syncthreads();
  // the most keys of a sequence, which the classes divide
  int most = 0;
  for (int b = tid; b < P.batch; b += kPlanThreads)
    most = max(most, clamped(ks[b + 1], 0, P.num_keys) - clamped(ks[b], 0, P.num_keys));
  atomicMax(&most_, most);
  // Over all sequences: the items' classes are counted; each item's count before it is its place
  // in its class. Where a thread has one item at most it keeps that until the classes' places are
  // known, else all is gone over once more (32 prompts 11.0 us, and twice 15.6; four 9.7
  // and 12.5).
  int total = 0, cls = 0, at = 0, q_from, k_from;
  Item I{};
  // the starts of sequence b0 and on, and how many items they have up to each
  auto fetch = [&](int b0) {
    const int b = min(b0 + tid, P.batch);   // (start b; the last one's twice or more)
    int all;
    const int q = larger(q_from, block_scan(clamped(P.q_start[b], 0, P.num_queries), larger, 0, part, all));
    const int k = larger(k_from, block_scan(clamped(ks[b], 0, P.num_keys), larger, 0, part, all));
    __syncthreads();
    q0_[tid] = q;
    k0_[tid] = k;
    if (tid == kPlanThreads - 1) {
      const int e = min(b0 + kPlanThreads, P.batch);
      q0_[kPlanThreads] = larger(q, clamped(P.q_start[e], 0, P.num_queries));
      k0_[kPlanThreads] = larger(k, clamped(ks[e], 0, P.num_keys));
    }
    __syncthreads();
    q_from = q0_[kPlanThreads];
    k_from = k0_[kPlanThreads];
    const int rows = (q0_[tid + 1] - q) * P.group;
    const int mine = b0 + tid < P.batch ? (rows + bm - 1) / bm : 0;
    upto_[tid] = block_scan(mine, plus, 0, part, total);
    __syncthreads();
  };
  auto take = [&](int i) {
    int lo = 0, hi = kPlanThreads - 1;      // the sequence of item i: the first with upto > i
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (upto_[mid] > i) hi = mid;
      else lo = mid + 1;
    }
    I.q0 = q0_[lo];
    I.nq = q0_[lo + 1] - I.q0;
    I.k0 = k0_[lo];
    I.nk = k0_[lo + 1] - I.k0;
    I.tile = i - (lo ? upto_[lo - 1] : 0);
    const int last = min((I.tile + 1) * bm, I.nq * P.group) - 1;
    const int keys = clamped(last / P.group + 1 + I.nk - I.nq, 0, most_);
    cls = kClasses - 1 - static_cast<int>(static_cast<int64_t>(keys) * (kClasses - 1) / most_);
    at = atomicAdd(&classes_[cls], 1);
  };
  bool once = false;
  for (int pass = 0; pass < (once ? 1 : 2); ++pass) {
    q_from = k_from = 0;                    // starts that decrease count as the largest before them
    for (int b0 = 0; b0 < P.batch; b0 += kPlanThreads) {
      fetch(b0);
      once = P.batch <= kPlanThreads && total <= kPlanThreads;
      for (int i = tid; i < total; i += kPlanThreads) {
        take(i);
        if (pass) P.items[at] = I;
      }
      __syncthreads();
    }
    if (pass == 0) {
      int count;
      const int own = classes_[tid];
      const int upto = block_scan(own, plus, 0, part, count);
      __syncthreads();
      classes_[tid] = upto - own;
      if (tid == 0) *P.count = count;
      __syncthreads();
    }
  }
  if (once && tid < total) P.items[classes_[cls] + at] = I;
}

// Rows of a workgroup, of which a CU holds one: 256 of them where they give every CU one, else 128 (two
// key groups), and in heads of 64 (whose four key groups' tiles LDS holds) 64 where no CU has two. One
// prompt, 32 heads over 8 of 128, by 128 / 256 rows: 100 tokens 13.2 / 13.5 us, 700 21 / 28, 2000 (250
// workgroups of 256) 58 / 61, 3000 (375) 114 / 98, 6000 327 / 301. Heads of 64, by 64 / 128 rows: 100
// tokens 9.4 / 9.2, 500 (256 workgroups of 64) 12.5 / 13.2, 512 behind 7488 more 49 / 73, 1000 23.5 /
// 18.2, two of 512 behind 7488 more 105 / 95.
int64_t most_items(int64_t rows, int64_t batch, int bm) { return rows / bm + batch; }

int block_rows(int64_t rows, int64_t batch, int64_t kv_heads, int head_dim, int cus) {
  if (rows / 256 * kv_heads > cus) return 256;
  const int64_t narrow = (rows + kWaveRows - 1) / kWaveRows + batch - 1;
  return head_dim <= 64 && narrow * kv_heads <= cus ? 64 : 128;
}

int device_cus() {
  constexpr int kMaxDevices = 64;
  static int cus[kMaxDevices];
  static std::mutex mu;
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0) return 0;
  std::lock_guard<std::mutex> lock(mu);
  if (dev < kMaxDevices && cus[dev]) return cus[dev];
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) return 0;
  if (dev < kMaxDevices) cus[dev] = n;
  return n;
}

template <class T, int DP>
hipError_t run(const Pass& P, int bm, unsigned wgs, hipStream_t stream) {
  const dim3 grid(wgs), block(kThreads);
  if (bm == 256) hipLaunchKernelGGL((prompt_kernel<T, Shape<DP, 4>>), grid, block, 0, stream, P);
  else if constexpr (DP == 64) {
    if (bm == 64) hipLaunchKernelGGL((prompt_kernel<T, Shape<DP, 1>>), grid, block, 0, stream, P);
    else hipLaunchKernelGGL((prompt_kernel<T, Shape<DP, 2>>), grid, block, 0, stream, P);
  } else hipLaunchKernelGGL((prompt_kernel<T, Shape<DP, 2>>), grid, block, 0, stream, P);
  return hipGetLastError();
}

}  // namespace

namespace tv {

size_t prompt_workspace(int32_t batch, int32_t num_queries, int32_t num_keys, int32_t heads,
                        int32_t kv_heads, int32_t head_dim) {
  (void)num_keys;
  const int64_t rows = static_cast<int64_t>(num_queries) * (heads / kv_heads);
  return align256(256 + static_cast<size_t>(most_items(rows, batch, head_dim <= 64 ? 64 : 128)) * sizeof(Item));
}

int launch_prompt(const PromptArgs& a, void* workspace, hipStream_t stream) {
  const int cus = device_cus();
  if (!cus) return TV_ERR_HIP;
  Pass P{};
  P.q = static_cast<const uint16_t*>(a.q);
  P.k = static_cast<const uint16_t*>(a.k);
  P.v = static_cast<const uint16_t*>(a.v);
  P.out = static_cast<uint16_t*>(a.out);
  P.q_stride = a.q_stride;
  P.kv_stride = a.kv_stride;
  P.q_start = a.q_start;
  P.k_start = a.k_start;
  P.batch = a.batch;
  P.num_queries = a.num_queries;
  P.num_keys = a.num_keys;
  P.heads = a.heads;
  P.kv_heads = a.kv_heads;
  P.head_dim = a.head_dim;
  P.group = a.heads / a.kv_heads;
  P.k2 = static_cast<float>(static_cast<double>(a.scale) * 1.4426950408889634);
  const double slack = 8.0 / static_cast<double>(P.k2);
  P.slack = slack < 3.0e38 ? static_cast<float>(slack) : 3.0e38f;
  const int64_t rows = static_cast<int64_t>(a.num_queries) * P.group;
  const int bm = block_rows(rows, a.batch, a.kv_heads, a.head_dim, cus);
  const int64_t wgs = most_items(rows, a.batch, bm) * a.kv_heads;
  if (a.batch > 1) {
    P.count = static_cast<int*>(workspace);
    P.items = reinterpret_cast<Item*>(static_cast<uint8_t*>(workspace) + 256);
    hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, P, bm);
    if (hipGetLastError() != hipSuccess) return TV_ERR_HIP;
  }
  const unsigned grid = static_cast<unsigned>(wgs);
  hipError_t e;
  if (a.dtype == TV_DTYPE_BF16)
    e = a.head_dim <= 64 ? run<Bf16, 64>(P, bm, grid, stream) : run<Bf16, 128>(P, bm, grid, stream);
  else
    e = a.head_dim <= 64 ? run<F16, 64>(P, bm, grid, stream) : run<F16, 128>(P, bm, grid, stream);
  return e == hipSuccess ? TV_OK : TV_ERR_HIP;
}

}  // namespace tv
