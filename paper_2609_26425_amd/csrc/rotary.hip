// Rotary positions on three axes (time, height, width) for the Queries and Keys of
// a chunk: pair p of a head's channels is turned by the angle a = x[axis(p)] f_p,
//     (u, v) -> (u cos a - v sin a, u sin a + v cos a).
// The angle depends on the token and the pair, not on the head: a workgroup takes
// a few whole tokens, computes their cosines and sines once into LDS, and turns
// every head of the Queries and the Keys with them. A far position's angle needs
// more than fp32: turns = x f / 2 pi is formed and reduced to [-1/2, 1/2] in fp64,
// and only the remainder goes to fp32. That is off by three roundings of the whole angle
// (2 pi, f / 2 pi and the product: at most 3 2^-53 of it) and by 2^-26 of a turn: some
// 1e-7 radians in all up to angles of 2^27, 8e-7 at position 2^31 with f = 1. Memory bound: every value is read once and written
// once. Queries and Keys of 4,680 tokens x 40 heads x 128: 192 MB in 31.5 us, 6.1 TB/s
// with its inputs in part in the caches (a copy of as many bytes: 5.2). A single token's
// launch is one workgroup: some 6 us from call to end, 2.2 of them the kernel.
#include "grid_rows.h"
#include "qwm_common.h"

namespace qwm {
namespace {

constexpr int kRotThreads = 256, kRotTokens = 8;  // of a workgroup, at most

template <typename T>
struct Vec16 {  // 16 bytes of T as floats
  static constexpr int N = 16 / int(sizeof(T));
  float x[N];
};

template <typename T>
__device__ inline Vec16<T> unpack(const uint4 u) {
  Vec16<T> r;
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      r.x[2 * i] = __uint_as_float(w[i] << 16);
      r.x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    } else {
      r.x[i] = __uint_as_float(w[i]);
    }
  }
  return r;
}

// The one rounding of the result (to nearest even in BF16).
template <typename T>
__device__ inline uint4 pack(const Vec16<T>& v) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
      typedef float f32x2 __attribute__((ext_vector_type(2)));
      const f32x2 p = {v.x[2 * i], v.x[2 * i + 1]};
      w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2));
    } else {
      w[i] = __float_as_uint(v.x[i]);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Stores past the caches: what is written once is not read here again, and the inputs, just
// written by a projection, stay in them. 4,680 tokens x 40 heads: 38.9 -> 31.5 us; between
// the copies that write its inputs and append and a read of q_out behind it, it adds 31.4
// us instead of 35.0 (with loads past the caches as well 29.3, but 34.8 by itself).
template <typename T>
__device__ inline void store16(T* p, const uint4 v) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  __builtin_nontemporal_store(u32x4{v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4*>(p));
}

// a.block_tokens tokens per workgroup. HALVES: pair p is channels (p, p + pairs), so a thread
// holds a vector of each half; otherwise it is channels (2 p, 2 p + 1) of one vector.
// Channels past the turned pairs (p >= pairs) are copied (a product with cos 1 and sin 0
// would lose the sign of a zero, and take a pair's second infinity into its first).
template <typename T, int D, bool HALVES>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(const RotaryArgs a) {
  constexpr int P = D / 2, N = Vec16<T>::N, UNIT = HALVES ? 2 * N : N, UNITS = D / UNIT;
  constexpr int VN = HALVES ? 2 : 1;  // vectors of a unit
  __shared__ __attribute__((aligned(16))) float2 cs[kRotTokens * P];
  const int64_t tok0 = (int64_t(blockIdx.y) * gridDim.x + blockIdx.x) * a.block_tokens;
  if (tok0 >= a.tokens) return;
  const int tokens = int(a.tokens - tok0 < a.block_tokens ? a.tokens - tok0 : a.block_tokens);
  const int row = a.heads * UNITS, total = tokens * row;
  const int64_t out_stride = int64_t(a.heads) * D;
  struct Unit {
    int64_t src, dst;  // first element of its first vector
    int second, pair;  // distance of its second vector; its first pair's angle
    int left;          // turned pairs from its first on
  };
  auto unit_of = [&](int i) __attribute__((always_inline)) {
    const int t = i / row, u = i % row, h = u / UNITS, c = u % UNITS;
    int first, second = 0, pair;
    if constexpr (HALVES) {
      const int turned = a.pairs / N;  // units of the turned channels
      pair = c * N;
      first = c < turned ? c * N : 2 * a.pairs + (c - turned) * 2 * N;
      second = c < turned ? a.pairs : N;
    } else {
      pair = c * (N / 2);
      first = c * N;
    }
    return Unit{(tok0 + t) * a.token_stride + h * D + first, (tok0 + t) * out_stride + h * D + first, second, t * P + pair,
                a.pairs - pair};
  };
  auto fetch = [&](const void* base, const Unit& u, uint4 (&to)[VN]) __attribute__((always_inline)) {
    const T* in = static_cast<const T*>(base) + u.src;
    to[0] = *reinterpret_cast<const uint4*>(in);
    if constexpr (HALVES) to[1] = *reinterpret_cast<const uint4*>(in + u.second);
  };
  auto turn = [&](void* base, const Unit& un, const uint4 (&from)[VN]) __attribute__((always_inline)) {
    T* out = static_cast<T*>(base) + un.dst;
    const float2* c = cs + un.pair;
    Vec16<T> u = unpack<T>(from[0]);
    if constexpr (HALVES) {
      Vec16<T> v = unpack<T>(from[1]);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float2 t = c[j];
        const float x = u.x[j], y = v.x[j];
        u.x[j] = un.left > 0 ? __builtin_fmaf(x, t.x, -y * t.y) : x;
        v.x[j] = un.left > 0 ? __builtin_fmaf(x, t.y, y * t.x) : y;
      }
      store16(out + un.second, pack<T>(v));
    } else {
#pragma unroll
      for (int j = 0; j < N / 2; ++j) {
        const float2 t = c[j];
        const float x = u.x[2 * j], y = u.x[2 * j + 1];
        u.x[2 * j] = j < un.left ? __builtin_fmaf(x, t.x, -y * t.y) : x;
        u.x[2 * j + 1] = j < un.left ? __builtin_fmaf(x, t.y, y * t.x) : y;
      }
    }
    store16(out, pack<T>(u));
  };
  // the first units are on their way while the angles are computed
  const int i0 = threadIdx.x;
  Unit u0{};
  uint4 q0[VN], k0[VN];
  if (i0 < total) {
    u0 = unit_of(i0);
    fetch(a.q, u0, q0);
    if (a.k) fetch(a.k, u0, k0);
  }
  __builtin_amdgcn_sched_barrier(0);
  for (int i = threadIdx.x; i < tokens * P; i += kRotThreads) {
    const int p = i % P;
    const int64_t tok = tok0 + i / P;
    float2 v = make_float2(1.0f, 0.0f);
    if (p < a.pairs) {
      const int axis = p < a.end_t ? 0 : (p < a.end_h ? 1 : 2);
      int64_t x;
      if (a.pos) {
        x = a.pos[tok * 3 + axis];
      } else {
        const int64_t at = a.pos0 + tok % a.n, area = int64_t(a.height) * a.width;
        const int64_t in = at % area;
        x = axis == 0 ? at / area : (axis == 1 ? in / a.width : in % a.width);
      }
      const double t = double(x) * a.turns[p];
      const float rest = float(t - rint(t));
      sincospif(2.0f * rest, &v.y, &v.x);
      v.y *= a.sign;
    }
    cs[i] = v;
  }
  __syncthreads();
  if (i0 < total) {
    turn(a.q_out, u0, q0);
    if (a.k) turn(a.k_out, u0, k0);
  }
  for (int i = i0 + kRotThreads; i < total; i += kRotThreads) {
    const Unit u = unit_of(i);
    uint4 qv[VN], kv[VN];
    fetch(a.q, u, qv);
    if (a.k) fetch(a.k, u, kv);
    turn(a.q_out, u, qv);
    if (a.k) turn(a.k_out, u, kv);
  }
}

template <typename T, int D, bool HALVES>
hipError_t launch_t(const RotaryArgs& a, hipStream_t s) {
  // A token a workgroup from half a unit a thread on: many small workgroups even out over
  // the CUs (d = 128, BF16, us with 1 / 2 / 4 tokens: 4 x 3,120 tokens of 30 heads 70 / 77 / 85,
  // 50,000 of 8 heads 70 / 73 / 77). Fewer heads take more, for their angles and their
  // workgroup's start (100,000 of 4 heads 94 / 72 / 74; 200,000 of 2 heads at d = 64 with 1 / 4
  // / 8 155 / 53 / 41).
  RotaryArgs b = a;
  const int units = a.heads * (D * int(sizeof(T)) / (HALVES ? 32 : 16)), fill = kRotThreads / 2 / units;
  b.block_tokens = fill < 1 ? 1 : (fill < kRotTokens ? fill : kRotTokens);
  const int64_t wgs = (a.tokens + b.block_tokens - 1) / b.block_tokens;
  hipLaunchKernelGGL((rotary_kernel<T, D, HALVES>), dim3(qwm_grid_x(wgs), qwm_grid_y(wgs)), dim3(kRotThreads), 0, s, b);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_d(const RotaryArgs& a, bool halves, hipStream_t s) {
  return halves ? launch_t<T, D, true>(a, s) : launch_t<T, D, false>(a, s);
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, int d, bool bf16_data, bool halves, hipStream_t s) {
  if (d == 64) return bf16_data ? launch_d<bf16, 64>(a, halves, s) : launch_d<float, 64>(a, halves, s);
  if (d == 128) return bf16_data ? launch_d<bf16, 128>(a, halves, s) : launch_d<float, 128>(a, halves, s);
  return hipErrorInvalidValue;
}

}  // namespace qwm
