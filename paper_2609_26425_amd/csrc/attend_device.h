// Device helpers of the attention kernels: matrix-core fragments, conversions and the
// dequantisation of packed codes. Private to each translation unit.
#pragma once

#include "qwm_common.h"

#include <type_traits>

namespace qwm {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <typename T>
struct Mfma;
template <>
struct Mfma<bf16> {  // v_mfma_f32_32x32x16_bf16
  static constexpr int KPL = 8, KSTEP = 16;
  typedef bf16x8 V;
  static __device__ inline f32x16 run(V a, V b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Mfma<float> {  // v_mfma_f32_32x32x2_f32
  static constexpr int KPL = 1, KSTEP = 2;
  typedef float V;
  static __device__ inline f32x16 run(V a, V b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
  }
};

template <typename V, typename T>
__device__ inline void vset(V& v, int j, T x) {
  if constexpr (sizeof(V) == sizeof(T)) v = x;
  else v[j] = x;
}

// max(a, b, c): the compiler folds the pair into one v_max3_f32. This file is
// built without NaN semantics (the logits and running maxima are finite or
// -inf), so no input is first quieted with a v_max_f32 x, x. It is not inline
// asm on purpose: its inputs come straight from matrix-core results, and only
// the compiler inserts the wait states a VALU read of those needs.
__device__ inline float max3f(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }

template <typename V>
__device__ inline auto vget(const V& v, int j) {
  if constexpr (std::is_same_v<V, float>) return v;
  else return v[j];
}

// Row of the 32x32 accumulator held by accumulator slot i of a lane in half hf.
__device__ inline constexpr int acc_row(int i, int hf) { return (i / 4) * 8 + hf * 4 + (i % 4); }

template <typename T, int N>
__device__ inline void load_vals(const T* p, float (&out)[N]) {
  if constexpr (sizeof(T) == 2) {
    static_assert(N % 8 == 0 || N == 4, "bf16 loads of 8 or 4 values");
    if constexpr (N == 4) {
      const uint2 u = *reinterpret_cast<const uint2*>(p);
      out[0] = __uint_as_float(u.x << 16); out[1] = __uint_as_float(u.x & 0xffff0000u);
      out[2] = __uint_as_float(u.y << 16); out[3] = __uint_as_float(u.y & 0xffff0000u);
    } else {
#pragma unroll
      for (int i = 0; i < N / 8; ++i) {
        const uint4 u = reinterpret_cast<const uint4*>(p)[i];
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          out[8 * i + 2 * k] = __uint_as_float(w[k] << 16);
          out[8 * i + 2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = p[i];
  }
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Two floats -> two bf16 (round to nearest even) in one v_cvt_pk_bf16_f32.
__device__ inline uint32_t pack_bf16(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// N centroid components from LDS: BF16 (T), or with H16 the binary16 copy of
// the table (scaled by a power of two), which v_fma_mix_f32 converts to fp32 as
// an operand, so the dequant takes no separate unpack of a BF16 pair.
template <bool H16, typename T, int N>
__device__ inline void load_tab(const T* p, float (&out)[N]) {
  if constexpr (H16) {
    typedef _Float16 h8 __attribute__((ext_vector_type(8)));
    static_assert(N % 8 == 0, "binary16 table loads of 8 values");
#pragma unroll
    for (int i = 0; i < N / 8; ++i) {
      const h8 v = reinterpret_cast<const h8*>(p)[i];
#pragma unroll
      for (int k = 0; k < 8; ++k) out[8 * i + k] = (float)v[k];
    }
  } else {
    load_vals<T, N>(p, out);
  }
}

template <typename T, int N>
__device__ inline void store_vals(T* p, const float (&x)[N]) {
  if constexpr (sizeof(T) == 2) {
    static_assert(N % 8 == 0, "bf16 stores of 8 values");
#pragma unroll
    for (int i = 0; i < N / 8; ++i)
      reinterpret_cast<uint4*>(p)[i] = make_uint4(pack_bf16(x[8 * i], x[8 * i + 1]), pack_bf16(x[8 * i + 2], x[8 * i + 3]),
                                                  pack_bf16(x[8 * i + 4], x[8 * i + 5]), pack_bf16(x[8 * i + 6], x[8 * i + 7]));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = x[i];
  }
}

// Stores with 8-byte alignment only (rows whose stride is an odd multiple of 8 B).
template <typename T, int N>
__device__ inline void store_vals8(T* p, const float (&x)[N]) {
  if constexpr (sizeof(T) == 2) {
    static_assert(N % 4 == 0, "bf16 stores of 4 values");
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
      reinterpret_cast<uint2*>(p)[i] = make_uint2(pack_bf16(x[4 * i], x[4 * i + 1]), pack_bf16(x[4 * i + 2], x[4 * i + 3]));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = x[i];
  }
}

template <typename T>
__device__ inline void store_pair(T* p, float a, float b) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint32_t*>(p) = pack_bf16(a, b);
  } else {
    p[0] = a;
    p[1] = b;
  }
}

// max of x over lanes i and i ^ 32 (v_permlane32_swap: no LDS round trip)
__device__ inline float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// (x & m) | o in one v_and_or_b32; written as asm so that the compiler does not
// fold the mask into per-field extractions.
__device__ inline uint32_t and_or(uint32_t x, uint32_t m, uint32_t o) {
  uint32_t r;
  asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(r) : "v"(x), "v"(m), "v"(o));
  return r;
}

// x[c] = mu[c] + s (code_c - z) for the N consecutive channels of one code word
// (channel c in bits 2c). Each code is placed in a binary16 half as 1024 + code
// (exponent 10: one unit per ulp), so one packed f16 subtraction of 1024 + z
// yields two exact (code - z), and v_fma_mix_f32 takes them and the binary16
// scale as fp32 operands: one rounding, the same value as fma(s, code - z, mu).
// SI8 (App. D.1 8-bit group scales): the step is sigma * c with s = sigma and cm
// = (c, c); c (code - z) is an integer of magnitude <= 765, exact in binary16,
// so the fma still rounds once.
template <int N, bool SI8 = false, typename S>
__device__ inline void dequant_codes(uint32_t cw, S s, uint32_t zz, const float (&mu)[N], float (&x)[N],
                                     f16x2 cm = {}) {
  static_assert(N == 16 || N == 8, "16 or 8 channels per code word");
  const f16x2 zh = __builtin_bit_cast(f16x2, zz);
  // N == 8: channels 4..7 move to bits 16..23, so half k pairs channels k and k + N/2
  const uint32_t w = N == 16 ? cw : ((cw & 0xffu) | ((cw & 0xff00u) << 8));
#pragma unroll
  for (int k = 0; k < N / 2; ++k) {
    f16x2 d = __builtin_bit_cast(f16x2, and_or(w >> (2 * k), 0x00030003u, 0x64006400u)) - zh;
    if constexpr (SI8) d = d * cm;
    x[k] = __builtin_fmaf((float)s, (float)d.x, mu[k]);
    x[k + N / 2] = __builtin_fmaf((float)s, (float)d.y, mu[k + N / 2]);
  }
}

// Builds a bf16x8 MFMA operand from 8 floats with paired conversions.
template <typename V>
__device__ inline V pack_operand(const float* x) {
  if constexpr (sizeof(V) == 16) {
    const uint4 u = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    return __builtin_bit_cast(V, u);
  } else {
    return x[0];
  }
}

}  // namespace
}  // namespace qwm
