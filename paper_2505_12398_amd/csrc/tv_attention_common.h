// Shared pieces of the attention kernels for gfx950: the two 16-bit types, loads that
// write LDS directly, and frames of running maxima.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>
#include <utility>

namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((address_space(3))) uint8_t lds_byte;
#define LDS(type) __attribute__((address_space(3))) type
// read through the scalar cache: nothing of the launch writes it
#define CONSTANT(type) const __attribute__((address_space(4))) type

struct Bf16 {
  static __device__ __forceinline__ f32x4 mfma(s16x8 a, s16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {   // to nearest even
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
  }
  // x plus both halves (off by less than two additions in turn: over 60000 weights of up
  // to 2^20 apart 3e-5 at worst where these have 7e-5)
  static __device__ __forceinline__ float plus(float x, uint32_t two) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two),
                                           __builtin_bit_cast(bf16x2, 0x3f803f80u), x, false);
  }
  // byte SEL of two 4-bit elements times f, a power of two (exact: e2m1 has two bits)
  template <int SEL>
  static __device__ __forceinline__ uint32_t widen(uint32_t x, float f) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, f, SEL));
  }
  // two elements divided by f, a power of two, as 4 bits each into byte SEL: to the nearest, ties to
  // even, beyond 6 to 6
  template <int SEL>
  static __device__ __forceinline__ uint32_t narrow(uint32_t old, uint32_t two, float f) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(bf16x2, two), f, SEL);
  }
  static __device__ __forceinline__ float value(uint16_t x) { return __uint_as_float(uint32_t{x} << 16); }
  static __device__ __forceinline__ s16x8 ones() {
    return s16x8{0x3f80, 0x3f80, 0x3f80, 0x3f80, 0x3f80, 0x3f80, 0x3f80, 0x3f80};
  }
  static constexpr uint32_t kExponent = 0x7f80;
  static constexpr float kLift = 0.0f;
};
struct F16 {
  static __device__ __forceinline__ f32x4 mfma(s16x8 a, s16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, f16x2));
  }
  static __device__ __forceinline__ float plus(float x, uint32_t two) {
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, two),
                                  __builtin_bit_cast(f16x2, 0x3c003c00u), x, false);
  }
  // (exact where fp16 holds the product, else to the nearest)
  template <int SEL>
  static __device__ __forceinline__ uint32_t widen(uint32_t x, float f) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x, f, SEL));
  }
  template <int SEL>
  static __device__ __forceinline__ uint32_t narrow(uint32_t old, uint32_t two, float f) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(old, __builtin_bit_cast(f16x2, two), f, SEL);
  }
  static __device__ __forceinline__ float value(uint16_t x) {
    return static_cast<float>(__builtin_bit_cast(_Float16, x));
  }
  static __device__ __forceinline__ s16x8 ones() {
    return s16x8{0x3c00, 0x3c00, 0x3c00, 0x3c00, 0x3c00, 0x3c00, 0x3c00, 0x3c00};
  }
  static constexpr uint32_t kExponent = 0x7c00;
  // Weights of up to 2^15 (the largest fp16 is below 2^16): those below 2^-21 of the largest
  // are rounded to multiples of 2^-31 of it. Without the lift these are 2^-14 and 2^-24, and
  // 30000 keys at e^-18 of one key's weight lost 51% of what they add.
  static constexpr float kLift = 7.0f;
};

constexpr int kPastRange = 0x40000000, kRange = 0x3fffffff;

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// N loads of 64 lanes' 16 bytes from the buffer at byte offsets voff into LDS, load i
// at dst + 1024 i + 16 lane; zeros for an offset past the range. (In assembly, so that
// the compiler does not wait for them at the next LDS read: the waits are written out
// below. The hazard recogniser does not look into it: the five wait states between a
// scalar that the vector unit wrote and a load, and the one behind m0, are here.)
template <int N>
__device__ __forceinline__ void load_to_lds(const i32x4& rs, const int (&voff)[N], int dst) {
  if constexpr (N == 1)
    asm volatile("s_nop 4\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :: "s"(dst), "v"(voff[0]), "s"(rs) : "memory", "m0");
  else if constexpr (N == 2)
    asm volatile("s_nop 4\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %3, 0 offen lds\n\t"
                 "s_add_u32 m0, %0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds"
                 :: "s"(dst), "v"(voff[0]), "v"(voff[1]), "s"(rs) : "memory", "m0", "scc");
  else
    asm volatile("s_nop 4\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %5, 0 offen lds\n\t"
                 "s_add_u32 m0, %0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %5, 0 offen lds\n\t"
                 "s_add_u32 m0, %0, 0x800\n\ts_nop 0\n\tbuffer_load_dwordx4 %3, %5, 0 offen lds\n\t"
                 "s_add_u32 m0, %0, 0xc00\n\ts_nop 0\n\tbuffer_load_dwordx4 %4, %5, 0 offen lds"
                 :: "s"(dst), "v"(voff[0]), "v"(voff[1]), "v"(voff[2]), "v"(voff[3]), "s"(rs)
                 : "memory", "m0", "scc");
}
#pragma clang diagnostic pop
// All but the newest N loads have landed, and this wavefront's LDS reads are done.
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(N) : "memory");
}
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// the largest of three, NaN if one is
__device__ __forceinline__ float max3(float a, float b, float c) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}

template <class F, int... I>
__device__ __forceinline__ void unrolled(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void unrolled(F&& f) {
  unrolled(f, std::make_integer_sequence<int, N>{});
}

// The frame of a maximum, -m k and the type's lift (0 where there is none), rounded by
// itself: sums are moved between frames by the differences of these.
template <class T>
__device__ __forceinline__ float frame(float m, float k) {
#pragma clang fp contract(off)
  return m > -INFINITY ? -m * k + T::kLift : 0.0f;
}
// What takes a sum from the frame of m to that of top >= m. (0 where nothing was
// seen; a sum that is NaN stays NaN.)
template <class T>
__device__ __forceinline__ float to_frame(float m, float top, float k) {
  return m > -INFINITY ? __builtin_amdgcn_exp2f(frame<T>(top, k) - frame<T>(m, k)) : 0.0f;
}

// A value that all lanes hold, known as such.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ long long uniform(long long x) {
  const uint32_t lo = static_cast<uint32_t>(uniform(static_cast<int>(x)));
  return static_cast<long long>(
      static_cast<uint64_t>(static_cast<uint32_t>(uniform(static_cast<int>(x >> 32)))) << 32 | lo);
}

// The same value, of which the compiler knows nothing: what is computed from it
// stays behind this point and out of the registers of the loop over the tiles.
__device__ __forceinline__ int here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

}  // namespace
