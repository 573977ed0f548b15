// Attention of a few Queries (single tokens, a handful of rollouts) over the packed
// cache: Eq. 5 with Eq. 17 and an online base-2 softmax as in attend.hip, organised for
// launches that are bound by decoding the keys rather than by the products. There a
// workgroup's 256 Query rows would mostly be empty, and its four producer waves, one
// per SIMD, decode for eight consumers that have next to nothing to do. Here every
// wave decodes and multiplies its own runs of 32 keys, with no barrier between them,
// and uses the form of a packed Key,
//     q . khat_0 = q . mu_z + sum_g s_g q_g . (code - z)_g,
// so that no Key is rebuilt: with few Queries q . mu is a small table in LDS (one
// product per centroid and Query, made once), added to the logits after the fact. A
// lane holds a quarter of two keys' channels and turns their codes into binary16
// operands s (code - z) with packed arithmetic (the channel order of a contraction is
// free, so its codes are contiguous bytes); the Query is held as binary16 too, times the power
// of two that puts its largest magnitude in [2^14, 2^15), which keeps every BF16 value
// exact that is not 2^-29 times smaller. Values are decoded by key pairs to BF16 into a
// wave-private transposed tile (V^T rows of 32 keys), the A operand of O^T += V^T P^T.
// Packed fields are loaded a step ahead, each side's as soon as the last ones are used.
// Fewer than 32 bits have the operands of the products only: s (code - z) is rounded to
// binary16 (2^-11 of it), and Values, weights, coefficients and q U_r to BF16 (2^-8 of
// them), as in attend.hip; sums and softmax states are fp32. Outputs are 0.0018 to 0.0019 off,
// of which their own rounding to BF16 is 0.0017.
// A workgroup runs one part of one segment (an epoch's keys or the exact chunk), so its
// tables, scales and q U_r never change; its waves merge their softmax states through
// LDS, and the parts are merged by join_planes.
//
// Bound by vector issue and by latency at three waves a SIMD: some 530 vector instructions
// for 32 keys (d = 128, rank 16), against 18 matrix products. One Query of 40 heads over
// 15,600 keys of a cache of 32,760 (128 centroids): 34.6 us. 1,024 keys take 16 of that
// (the call, the staging of the tables, the merges), the rest is 1.3 ns a key of all
// heads, 3.2 TB/s of packed fields. 256-row workgroups of attend.hip: 75 us.
#include "attend_device.h"
#include "attend_shape.h"
#include "few_shape.h"

#include <atomic>

namespace qwm {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Waves of a workgroup. NQ: tiles of 16 Query rows; one leaves registers for three waves
// a SIMD, two for two. TAB: the Value table in LDS, for parts with at least as many keys
// as it has rows; shorter parts gather its rows and run in workgroups of four waves, of
// which a CU holds several (480 workgroups of 131 keys: one round instead of two).
constexpr int few_waves(int nq, bool tab) { return !tab ? 4 : (nq == 1 ? 12 : 8); }

// LDS: the products q . mu of every centroid and Query ([256][16 NQ] floats: an id is a
// byte, so none reads past it), the Value table (TAB, binary16) and a V^T tile per
// wave, in 32-bit words (key pairs): 64 channels, 16 of each quarter, of 16 pairs + 2
// words of padding, each quarter 8 words further. With 32 banks, the pair stores of 32
// lanes (8 pairs in four quarters) and the 8-byte operand reads of 16 lanes (as many rows)
// are then free of conflicts. The four lanes of a pair read their 16-byte pieces of one
// table row together, at a quarter row's distance: at d = 128 the pieces of the upper
// half are turned by two, so that these four too lie in banks of their own.
template <int D, int NQ>
struct FewLds {
  static constexpr int SMU = 256 * 16 * NQ, ROW = 18, QUARTER = 16 * ROW + 8, VW = 3 * QUARTER + 16 * ROW, TS = D + 8;
  static __device__ inline int at(int quarter) { return quarter * QUARTER; }  // its first row
  static __device__ inline int piece(int c) { return D == 128 ? (c & 8) | ((c + (c >> 3) * 2) & 7) : c; }
};

// Packed fields of one 32-key chunk in a lane between their load and their use: a quarter
// of the channels of two keys (l and 16 + l) and of two Values (a pair).
template <int D, int RP, bool SI8>
struct FewRegs {
  uint32_t k_c[2][D / 64], k_z[2], k_s[2], c_s[2], c_w[2][RP > 0 ? RP / 16 : 1];
  uint32_t k_id[2], k_sg[SI8 ? 4 : 1];  // of the keys of this lane's accumulator rows
  uint32_t v_c[2][D / 64], v_id, v_z[2], v_s[2], v_sg[2];
};

// x over the four lanes that hold one Query: i, i ^ 16, i ^ 32, i ^ 48
__device__ inline float max_quarters(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}

template <int D, int G, int RP, int NQ, bool TAB, bool SI8>
__global__ __launch_bounds__(64 * few_waves(NQ, TAB)) void attend_few_kernel(const AttendArgs a) {
  typedef bf16x8 V;
  typedef FewLds<D, NQ> LY;
  constexpr int NW = few_waves(NQ, TAB), CK = kFewChunk, HV = D / 4, W = D / 64, ST = D / 32, QC = 16 * NQ;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
  const int Kc = a.n_centroids, r = a.rank;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, l16 = lane % 16,
            kq = lane / 16;
  const FewPlace place = few_place(a, blockIdx.x, gridDim.x);
  const int part = place.part, h = place.h, b = place.b;
  const int64_t bh = place.bh, n_bh = place.n_bh;
  const int qa = place.block * a.block_rows, rows = min(a.block_rows, int(a.n_q) - qa);
  const int64_t nc = a.n_cache + a.n_act;
  const uint32_t F = uint32_t(a.frame_tokens);
  const FewReach reach = few_reach(a.q_start, F, nc, a.n_sink, a.window, a.windowed != 0, uint32_t(qa), uint32_t(qa + rows));
  int before = 0;
  const int seg = few_segment_at(a, reach, part, lane, before);
  const bool act = seg == a.n_epochs;
  FewSegment g{};
  if (!act || a.n_act > 0) g = few_segment_of(a, seg, reach);
  // chunks of this part; the wave's are t0 + wave, t0 + wave + NW, ...
  const int cpp = int(a.chunks_per_part), t0 = (part - before) * cpp, t1 = min(t0 + cpp, int(g.chunks));
  float* plane_ml = a.part_ml ? a.part_ml + 2 * ((int64_t(part) * n_bh + bh) * a.n_q + qa) : nullptr;
  if (t0 >= t1 && a.part_o) {  // this block of Queries has fewer parts than another: an empty plane
    if (int(threadIdx.x) < rows) {
      plane_ml[2 * threadIdx.x] = -__builtin_inff();
      plane_ml[2 * threadIdx.x + 1] = 0.0f;
    }
    return;
  }
  auto key_of = [&](int t) __attribute__((always_inline)) { return int(g.base) + (t >= int(g.cut) ? t + int(g.skip) : t) * CK; };

  const uint8_t* slab = a.calib + int64_t(act ? 0 : seg) * a.calib_stride + bh * a.slab;
  const bf16* gK = reinterpret_cast<const bf16*>(slab + a.o_mu_k);
  const bf16* gV = reinterpret_cast<const bf16*>(slab + a.o_mu_v16);  // binary16 bits
  float* smu = reinterpret_cast<float*>(smem_raw);
  bf16* tabV = reinterpret_cast<bf16*>(smu + LY::SMU);
  uint32_t* vt = reinterpret_cast<uint32_t*>(tabV + (TAB ? Kc * LY::TS : 0)) + wave * LY::VW;

  // ---- packed fields
  const CacheLayout& L = a.L;
  const int64_t slot0 = bh * L.slots;
  // zero-point bytes and scale bytes of a token, bytes of a scale
  constexpr uint32_t zpb = (D / G + 3) / 4, u8 = SI8 ? 1 : 2, ss = D / G * u8;
  auto field = [&](int64_t off, uint32_t bytes, int64_t end) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)(a.cache + off + slot0 * bytes), 0, int(uint32_t(end) * bytes), 0x00020000);
  };
  const auto r_kc = field(L.k_codes, D / 4, L.slots), r_ki = field(L.k_ids, 1, L.slots), r_kz = field(L.k_zp, zpb, L.slots),
             r_ks = field(L.k_scale, ss, L.slots), r_cc = field(L.k_coef, uint32_t(r), L.slots),
             r_cs = field(L.k_cscale, 2, L.slots), r_vc = field(L.v_codes, D / 4, L.slots),
             r_vi = field(L.v_ids, 1, L.slots), r_vz = field(L.v_zp, zpb, L.slots);
  // Value scales past the segment read as 0, so that its masked keys' Values are finite
  const auto r_vs = field(L.v_scale, ss, SI8 ? L.slots : g.hi), r_ksg = field(L.k_sigma, 2, L.slots),
             r_vsg = field(L.v_sigma, 2, g.hi);
  // key pair and channel quarter of a lane's Values: the lanes of a pair are neighbours,
  // so that lanes which read LDS together read few different rows of the Value table
  const int vp = lane / 4, vq = lane % 4;
  const int kg0 = kq * HV / G, vg0 = vq * HV / G;  // first group of the lane's channels
  constexpr int GN = HV / G > 1 ? HV / G : 1;      // their groups
  // their scale bytes. The loads hold no branch, here and below: at a join the compiler
  // could only wait for all of them.
  auto load_scales = [&](auto rsrc, int o, int so) __attribute__((always_inline)) {
    if constexpr (GN * u8 == 4) return uint32_t(__builtin_amdgcn_raw_buffer_load_b32(rsrc, o, so, 0));
    else if constexpr (GN * u8 == 2) return uint32_t(uint16_t(__builtin_amdgcn_raw_buffer_load_b16(rsrc, o, so, 0)));
    else return uint32_t(uint8_t(__builtin_amdgcn_raw_buffer_load_b8(rsrc, o, so, 0)));
  };
  auto load_codes = [&](auto rsrc, int o, int so, uint32_t (&to)[W]) __attribute__((always_inline)) {
    if constexpr (W == 2) {
      const auto c = __builtin_amdgcn_raw_buffer_load_b64(rsrc, o, so, 0);
      to[0] = c[0];
      to[1] = c[1];
    } else {
      to[0] = __builtin_amdgcn_raw_buffer_load_b32(rsrc, o, so, 0);
    }
  };
  typedef FewRegs<D, RP, SI8> Regs;
  auto load_key = [&](Regs& p, int t) __attribute__((always_inline)) {
    const int k0 = key_of(t);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int key = 16 * e + l16;
      load_codes(r_kc, key * (D / 4) + kq * (D / 16), k0 * (D / 4), p.k_c[e]);
      p.k_z[e] = uint8_t(__builtin_amdgcn_raw_buffer_load_b8(r_kz, key * int(zpb) + kg0 / 4, k0 * int(zpb), 0));
      p.k_s[e] = load_scales(r_ks, key * int(ss) + kg0 * int(u8), k0 * int(ss));
      p.k_id[e] = __builtin_amdgcn_raw_buffer_load_b32(r_ki, 16 * e + 4 * kq, k0, 0);
      if constexpr (SI8) {
        const auto v = __builtin_amdgcn_raw_buffer_load_b64(r_ksg, 2 * (16 * e + 4 * kq), 2 * k0, 0);
        p.k_sg[2 * e] = v[0];
        p.k_sg[2 * e + 1] = v[1];
      }
      if constexpr (RP > 0) {
        // ranks 16 i + 4 kq ... + 3: the rows that q U_r's fragment has (r is a multiple of
        // 4). Ranks past r read as 0, past the end of the resource.
        constexpr uint32_t kAbsent = 0xC0000000u;
        p.c_s[e] = uint16_t(__builtin_amdgcn_raw_buffer_load_b16(r_cs, 2 * key, 2 * k0, 0));
#pragma unroll
        for (int i = 0; i < RP / 16; ++i) {
          const int k = 16 * i + 4 * kq;
          p.c_w[e][i] = __builtin_amdgcn_raw_buffer_load_b32(r_cc, int(k < r ? uint32_t(key * r + k) : kAbsent), k0 * r, 0);
        }
      }
    }
  };
  auto load_value = [&](Regs& p, int t) __attribute__((always_inline)) {
    const int k0 = key_of(t);
    p.v_id = uint16_t(__builtin_amdgcn_raw_buffer_load_b16(r_vi, 2 * vp, k0, 0));
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int key = 2 * vp + e;
      load_codes(r_vc, key * (D / 4) + vq * (D / 16), k0 * (D / 4), p.v_c[e]);
      p.v_z[e] = uint8_t(__builtin_amdgcn_raw_buffer_load_b8(r_vz, key * int(zpb) + vg0 / 4, k0 * int(zpb), 0));
      p.v_s[e] = load_scales(r_vs, key * int(ss) + vg0 * int(u8), k0 * int(ss));
      if constexpr (SI8) p.v_sg[e] = uint16_t(__builtin_amdgcn_raw_buffer_load_b16(r_vsg, 2 * key, 2 * k0, 0));
    }
  };

  // ---- everything that a part starts with, in flight at once and in the order of its
  // use: the Queries, this wave's first rows of the Key table, U_r, the packed fields.
  // Step st of lane quarter kq holds channels kq D/4 + 8 st ... + 7.
  V qf[NQ][ST], ck[ST], cu[RP > 0 ? RP / 16 : 1][ST];
  auto load_row = [&](const bf16* row, V (&to)[ST]) __attribute__((always_inline)) {
#pragma unroll
    for (int st = 0; st < ST; ++st) to[st] = *reinterpret_cast<const V*>(row + st * 8);
  };
  auto centroids = [&](int z0) __attribute__((always_inline)) {
    load_row(gK + int64_t(min(z0 + l16, Kc - 1)) * D + kq * HV, ck);
  };
#pragma unroll
  for (int n = 0; n < NQ; ++n)
    load_row(reinterpret_cast<const bf16*>(a.q) +
                 ((int64_t(b) * a.n_q + qa + min(16 * n + l16, rows - 1)) * a.heads + h) * D + kq * HV, qf[n]);
  Regs P;
  int ek = 0, ev = 0;  // Values are decoded times 2^-e_v, the exponent of their binary16 table
  if (!act) {
    ek = reinterpret_cast<const int32_t*>(slab + a.o_e16)[0];
    ev = reinterpret_cast<const int32_t*>(slab + a.o_e16)[1];
    centroids(wave * 16);
    if constexpr (RP > 0) {
#pragma unroll
      for (int i = 0; i < RP / 16; ++i)
        load_row(reinterpret_cast<const bf16*>(slab + a.o_u_t) + min(16 * i + l16, r - 1) * D + kq * HV, cu[i]);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (t0 < t1) {
      load_key(P, min(t0 + wave, t1 - 1));
      load_value(P, min(t0 + wave, t1 - 1));
    }
    if constexpr (TAB) {
      constexpr int PER_ROW = D * 2 / 16;
      const uint4* sv = reinterpret_cast<const uint4*>(gV);
#pragma unroll 1
      for (int i = threadIdx.x; i < Kc * PER_ROW; i += 64 * NW)
        *reinterpret_cast<uint4*>(tabV + i / PER_ROW * LY::TS + LY::piece(i % PER_ROW) * 8) = sv[i];
    }
    __builtin_amdgcn_sched_barrier(0);
  }

  // ---- logits are in units of 2^qe of their Query: its binary16 copy holds q 2^-qe, with
  // its largest magnitude in [2^14, 2^15) unless the Key table's, below 2^(15 + e_k), is past
  // 2^104: q . mu, below 2^(23 + e_k) times the Query's, then stays below 2^126 in these units
  // (the residuals, at most 3 x 65,504 a channel, are lost in such a sum)
  float lscale[NQ], tau[NQ], unit[NQ];
  int qe[NQ], lim[NQ], wfrom[NQ];
  V qreg[NQ][ST], ureg[NQ];
  const float mscale = 1.4426950408889634f / sqrtf((float)D);  // as in attend.hip
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    float top = 0.0f;
#pragma unroll
    for (int st = 0; st < ST; ++st)
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(float(qf[n][st][j])));
    top = max_quarters(top);
    qe[n] = int((__float_as_uint(top) >> 23) & 255) - 127 + max(ek - 103, -14);
    qe[n] = min(max(qe[n], -100), 120);  // a zero Query: any unit
    unit[n] = __uint_as_float(uint32_t(127 - qe[n]) << 23);      // 2^-qe
    lscale[n] = ldexpf(mscale, qe[n]);
    tau[n] = 8.0f / lscale[n];
#pragma unroll
    for (int st = 0; st < ST; ++st) {
      // the channel order of the decoded operands: pairs (c, c + 8) of 16 channels; the
      // exact chunk's operands keep their own
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int c = st % 2 * 4 + j;
        w[j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(unit[n] * float(qf[n][st & ~1][c]),
                                                                       unit[n] * float(qf[n][st | 1][c])));
      }
      qreg[n][st] = act ? qf[n][st] : __builtin_bit_cast(V, make_uint4(w[0], w[1], w[2], w[3]));
    }
    if (act) unit[n] = 1.0f, lscale[n] = mscale, tau[n] = 8.0f / mscale, qe[n] = 0;
    const int qi = qa + 16 * n + l16;
    const int64_t l = a.q_start + int64_t(uint32_t(qi) / F + 1) * F, w = a.windowed ? l - a.window : 0;
    lim[n] = int(l < nc ? l : nc);
    wfrom[n] = int(w < 0 ? 0 : (w < nc ? w : nc));
  }
  if (!act) {
    // q . mu of every centroid: rows = centroids, columns = Queries
    for (int z0 = wave * 16; z0 < Kc; z0 += NW * 16) {
      f32x4 acc[NQ];
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        acc[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int st = 0; st < ST; ++st) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ck[st], qf[n][st], acc[n], 0, 0, 0);
      }
      if (z0 + NW * 16 < Kc) centroids(z0 + NW * 16);
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) smu[(z0 + 4 * kq + i) * QC + 16 * n + l16] = acc[n][i] * unit[n];
    }
    // q U_r (rows = ranks of U_r^T): slot (kq, j) of the fragment is rank 4 kq + j, and past
    // four 16 + 4 kq + j - 4. Ranks past r meet coefficients of 0.
    if constexpr (RP > 0) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        ureg[n] = V{};
#pragma unroll
        for (int i = 0; i < RP / 16; ++i) {
          f32x4 u = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int st = 0; st < ST; ++st) u = __builtin_amdgcn_mfma_f32_16x16x32_bf16(cu[i][st], qf[n][st], u, 0, 0, 0);
#pragma unroll
          for (int j = 0; j < 4; ++j) ureg[n][4 * i + j] = bf16(u[j] * unit[n]);
        }
      }
    }
  }
  ev = __builtin_amdgcn_readfirstlane(ev);
  const float scv = ldexpf(1.0f, -ev);
  __syncthreads();

  float m_run[NQ], l_run[NQ];
  f32x4 oacc[4 * W][NQ];  // [4 u + quarter]: channels quarter D/4 + 16 u + 4 kq + i
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    m_run[n] = -__builtin_inff();
    l_run[n] = 0.0f;
#pragma unroll
    for (int x = 0; x < 4 * W; ++x) oacc[x][n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  const int klo = int(g.lo), khi = int(g.hi), kclean = int(reach.kfull < g.hi ? reach.kfull : g.hi), sinks = int(reach.ns),
            wfull = int(reach.wfull);

  // binary16 scale (SI8: scale code) of word u of a lane's channels
  auto scale_of = [&](uint32_t w, int u) __attribute__((always_inline)) {
    if constexpr (SI8) return (_Float16)(int)((w >> (8 * (16 * u / G))) & 255);
    else return __builtin_bit_cast(_Float16, uint16_t(w >> (16 * (16 * u / G))));
  };
  auto zero_of = [&](uint32_t zb, int g0, int u) __attribute__((always_inline)) {
    return (0x6400u + ((zb >> (2 * (g0 % 4 + 16 * u / G))) & 3)) * 0x00010001u;
  };
  auto id_of = [&](uint32_t id) __attribute__((always_inline)) { return min(int(id), Kc - 1); };

  // masks the logits s of one chunk and turns them into BF16 weights, the B operands of
  // the Value product: slot (kq, j) is key 4 kq + j, and past four 16 + 4 kq + j - 4
  auto weigh = [&](f32x4 (&s)[2][NQ], int k0, V (&bv)[NQ]) __attribute__((always_inline)) {
    if (k0 < klo || k0 + CK > kclean || (k0 + CK > sinks && k0 < wfull)) {
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int key = k0 + 16 * (i / 4) + 4 * kq + i % 4;
          const bool hide = (key >= min(khi, lim[n])) | (key < klo) | ((key >= sinks) & (key < wfrom[n]));
          s[i / 4][n][i % 4] = hide ? -__builtin_inff() : s[i / 4][n][i % 4];
        }
    }
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      float mt = max3f(s[0][n][0], s[0][n][1], s[0][n][2]);
      mt = max3f(mt, s[0][n][3], s[1][n][0]);
      mt = max3f(mt, s[1][n][1], s[1][n][2]);
      mt = max_quarters(fmaxf(mt, s[1][n][3]));
      if (__any(mt > m_run[n] + tau[n])) {
        const float m_new = fmaxf(m_run[n], mt);
        const float alpha = m_new == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f((m_run[n] - m_new) * lscale[n]);
        l_run[n] *= alpha;
#pragma unroll
        for (int x = 0; x < 4 * W; ++x)
#pragma unroll
          for (int i = 0; i < 4; ++i) oacc[x][n][i] *= alpha;
        m_run[n] = m_new;
      }
      const float mc = m_run[n] == -__builtin_inff() ? 0.0f : -m_run[n] * lscale[n];
      float pv[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) pv[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 4][n][i % 4], lscale[n], mc));
      bv[n] = pack_operand<V>(pv);
      // the sum of the weights as rounded for the product
      const bf16x2 one = {bf16(1.0f), bf16(1.0f)};
      const uint4 pw = __builtin_bit_cast(uint4, bv[n]);
      const uint32_t w[4] = {pw.x, pw.y, pw.z, pw.w};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        l_run[n] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[j]), one, l_run[n], false);
    }
  };
  // A wave's stores to its tile, then its reads, then its next stores: LDS keeps a wave's
  // order, and these keep the compiler's
  auto in_order = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  // O^T += V^T P^T for the 64 channels in the tile, those of words u
  auto value_product = [&](const V (&bv)[NQ], int u) __attribute__((always_inline)) {
    in_order();
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const uint32_t* row = vt + LY::at(x) + l16 * LY::ROW + 2 * kq;
      const uint2 y = *reinterpret_cast<const uint2*>(row), z = *reinterpret_cast<const uint2*>(row + 8);
      const V av = __builtin_bit_cast(V, make_uint4(y.x, y.y, z.x, z.y));
#pragma unroll
      for (int n = 0; n < NQ; ++n)
        oacc[4 * u + x][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, bv[n], oacc[4 * u + x][n], 0, 0, 0);
    }
    in_order();
  };

  auto step = [&](Regs& p, int t) __attribute__((always_inline)) {
    // past the last chunk that one again: an unconditional load, so that the waits before
    // one side's use leave the other's loads in flight
    const int k0 = key_of(t), next = min(t + NW, t1 - 1);
    f32x4 s[2][NQ], mu[2][NQ];
    // q . mu of the keys of this lane's accumulator rows
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float* row = smu + ((p.k_id[e] >> (8 * i)) & 255) * QC + l16;
#pragma unroll
        for (int n = 0; n < NQ; ++n) mu[e][n][i] = row[16 * n];
      }
    // the residuals' products of one key, onto s; of its steps c, those that `pick` leaves
    auto residual = [&](int e, auto pick) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < W; ++u) {
        // s (code - z), or the integers c (code - z) (SI8), exact
        const _Float16 c = pick(scale_of(p.k_s[e], u));
        const f16x2 cc = {c, c}, zh = __builtin_bit_cast(f16x2, zero_of(p.k_z[e], kg0, u));
        uint32_t w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
          w[k] = __builtin_bit_cast(uint32_t, (__builtin_bit_cast(f16x2, and_or(p.k_c[e][u] >> (2 * k), 0x00030003u, 0x64006400u)) - zh) * cc);
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int n = 0; n < NQ; ++n)
            s[e][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                __builtin_bit_cast(f16x8, make_uint4(w[4 * x], w[4 * x + 1], w[4 * x + 2], w[4 * x + 3])),
                __builtin_bit_cast(f16x8, qreg[n][2 * u + x]), s[e][n], 0, 0, 0);
      }
    };
    auto coefficients = [&](int e) __attribute__((always_inline)) {
      if constexpr (SI8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const _Float16 sg = __builtin_bit_cast(_Float16, uint16_t(p.k_sg[2 * e + i / 2] >> (16 * (i % 2))));
#pragma unroll
          for (int n = 0; n < NQ; ++n) s[e][n][i] = __builtin_fmaf(s[e][n][i], (float)sg, mu[e][n][i]);
        }
      }
      if constexpr (RP > 0) {
        const float cs = (float)__builtin_bit_cast(_Float16, uint16_t(p.c_s[e]));
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < RP / 8; ++i) {
          const uint32_t c = p.c_w[e][i / 2];
          w[i] = pack_bf16((float)int8_t((c >> (16 * (i % 2))) & 255) * cs, (float)int8_t((c >> (16 * (i % 2) + 8)) & 255) * cs);
        }
        // with 16 ranks, half the depth is zeros: with a product of depth 16 onto the sums of
        // the deeper ones, right after them, results were wrong (the cause was not found)
#pragma unroll
        for (int n = 0; n < NQ; ++n)
          s[e][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(V, make_uint4(w[0], w[1], w[2], w[3])), ureg[n],
                                                            s[e][n], 0, 0, 0);
      }
    };
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) s[e][n] = SI8 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : mu[e][n];
      residual(e, [](_Float16 c) { return c; });
      coefficients(e);
    }
    if constexpr (!SI8) {
      // Steps of which three leave binary16's range (bits from 0x7555 on: the sum reaches a
      // half's top bit), in no Keys of usual size: the chunk again, with these steps a
      // quarter as large in products of their own. All the others stay as they are stored,
      // since a smaller one's lowest bits have no room below binary16's normal range.
      if (__any(((p.k_s[0] + 0x0aab0aabu) | (p.k_s[1] + 0x0aab0aabu)) & 0x80008000u)) {
        auto large = [](_Float16 c) { return __builtin_bit_cast(uint16_t, c) >= 0x7555; };
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
          for (int n = 0; n < NQ; ++n) s[e][n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
          residual(e, [&](_Float16 c) { return large(c) ? c * (_Float16)0.25f : (_Float16)0; });
#pragma unroll
          for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[e][n][i] = __builtin_fmaf(s[e][n][i], 4.0f, mu[e][n][i]);
          residual(e, [&](_Float16 c) { return large(c) ? (_Float16)0 : c; });
          coefficients(e);
        }
      }
    }
    load_key(p, next);
    // Values, 16 channels of each quarter at a time. Keys of the neighbouring epoch before
    // the segment's first take scale 0: finite, whatever they hold.
    const int id0 = id_of(p.v_id & 255), id1 = id_of(p.v_id >> 8);
    const bool in0 = k0 + 2 * vp >= klo, in1 = k0 + 2 * vp + 1 >= klo;
    auto values = [&](int u) __attribute__((always_inline)) {
      float m0[16], m1[16], x0[16], x1[16];
      const int c0 = vq * HV + 16 * u;
      // (a word's two pieces stay neighbours)
      const int at = TAB ? LY::piece(c0 / 8) * 8 : c0;
      load_tab<true, bf16, 16>((TAB ? tabV + id0 * LY::TS : gV + id0 * D) + at, m0);
      load_tab<true, bf16, 16>((TAB ? tabV + id1 * LY::TS : gV + id1 * D) + at, m1);
      const _Float16 y0 = scale_of(p.v_s[0], u), y1 = scale_of(p.v_s[1], u);
      const f16x2 cm0 = {y0, y0}, cm1 = {y1, y1};
      float s0 = SI8 ? (float)__builtin_bit_cast(_Float16, uint16_t(p.v_sg[0])) : (float)y0;
      float s1 = SI8 ? (float)__builtin_bit_cast(_Float16, uint16_t(p.v_sg[1])) : (float)y1;
      s0 = in0 ? s0 * scv : 0.0f;
      s1 = in1 ? s1 * scv : 0.0f;
      dequant_codes<16, SI8>(p.v_c[0][u], s0, zero_of(p.v_z[0], vg0, u), m0, x0, cm0);
      dequant_codes<16, SI8>(p.v_c[1][u], s1, zero_of(p.v_z[1], vg0, u), m1, x1, cm1);
#pragma unroll
      for (int c = 0; c < 16; ++c) vt[LY::at(vq) + c * LY::ROW + vp] = pack_bf16(x0[c], x1[c]);
    };
    V bv[NQ];
    values(0);
    weigh(s, k0, bv);
    value_product(bv, 0);
    if constexpr (W == 2) values(1);
    load_value(p, next);
    if constexpr (W == 2) value_product(bv, 1);
  };

  if (t0 + wave < t1) {
    if (!act) {
      for (int t = t0 + wave; t < t1; t += NW) step(P, t);
    } else {
      // exact rows: operands straight from memory, the last row again past the end
      const int last = int(a.n_act) - 1;
      auto row_of = [&](const void* base, int i) {
        return reinterpret_cast<const bf16*>(base) + ((int64_t(b) * a.n_act + min(i, last)) * a.heads + h) * D;
      };
      for (int t = t0 + wave; t < t1; t += NW) {
        const int k0 = key_of(t), r0 = k0 - int(a.n_cache);
        V kv[2][ST];
#pragma unroll
        for (int e = 0; e < 2; ++e) load_row(row_of(a.k_act, r0 + 16 * e + l16) + kq * HV, kv[e]);
        uint4 x0[HV / 8], x1[HV / 8];
#pragma unroll
        for (int i = 0; i < HV / 8; ++i) {
          x0[i] = reinterpret_cast<const uint4*>(row_of(a.v_act, r0 + 2 * vp) + vq * HV)[i];
          x1[i] = reinterpret_cast<const uint4*>(row_of(a.v_act, r0 + 2 * vp + 1) + vq * HV)[i];
        }
        f32x4 s[2][NQ];
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int n = 0; n < NQ; ++n) {
            s[e][n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int st = 0; st < ST; ++st)
              s[e][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kv[e][st], qreg[n][st], s[e][n], 0, 0, 0);
          }
        V bv[NQ];
        weigh(s, k0, bv);
#pragma unroll
        for (int u = 0; u < W; ++u) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint4 y = x0[2 * u + i], z = x1[2 * u + i];
            const uint32_t p0[4] = {y.x, y.y, y.z, y.w}, p1[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              uint32_t* to = vt + LY::at(vq) + (8 * i + 2 * j) * LY::ROW + vp;
              to[0] = __builtin_amdgcn_perm(p1[j], p0[j], 0x05040100u);
              to[LY::ROW] = __builtin_amdgcn_perm(p1[j], p0[j], 0x07060302u);
            }
          }
          value_product(bv, u);
        }
      }
    }
  }

  // ---- merge of the waves: every wave's O rows, running max and sum through LDS (the
  // tables and V^T tiles are done with)
  constexpr int OS = D + 4;
  float* mo = reinterpret_cast<float*>(smem_raw);  // [wave][row][OS]
  float* ml = mo + NW * rows * OS;                 // [wave][row][2]
  __syncthreads();
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int row = 16 * n + l16;
    float l = l_run[n] + __shfl_xor(l_run[n], 16);
    l += __shfl_xor(l, 32);
    if (row < rows) {
      float* to = mo + (wave * rows + row) * OS + 4 * kq;
#pragma unroll
      for (int x = 0; x < 4 * W; ++x) *reinterpret_cast<f32x4*>(to + x % 4 * HV + x / 4 * 16) = oacc[x][n];
      if (kq == 0) {
        ml[2 * (wave * rows + row)] = ldexpf(m_run[n], qe[n]);
        ml[2 * (wave * rows + row) + 1] = l;
      }
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < rows * D; i += 64 * NW) {
    const int q = i / D, c = i % D;
    float M = -__builtin_inff();
#pragma unroll
    for (int w = 0; w < NW; ++w) M = fmaxf(M, ml[2 * (w * rows + q)]);
    float o = 0.0f, l = 0.0f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float lw = ml[2 * (w * rows + q) + 1];
      const float e = lw > 0.0f ? __builtin_amdgcn_exp2f((ml[2 * (w * rows + q)] - M) * mscale) : 0.0f;
      l += e * lw;
      o += e * mo[(w * rows + q) * OS + c];
    }
    if (a.part_o) {
      a.part_o[((int64_t(part) * n_bh + bh) * a.n_q + qa + q) * D + c] = ldexpf(o, ev);
      if (c == 0) {
        plane_ml[2 * q] = M;
        plane_ml[2 * q + 1] = l;
      }
    } else {
      const float inv = l > 0.0f ? ldexpf(1.0f / l, ev) : 0.0f;
      reinterpret_cast<bf16*>(a.out)[((int64_t(b) * a.n_q + qa + q) * a.heads + h) * D + c] = bf16(o * inv);
      if (a.lse && c == 0)
        a.lse[bh * a.n_q + qa + q] = l > 0.0f ? M / sqrtf((float)D) + logf(l) : -__builtin_inff();
    }
  }
}

template <int D, int NQ>
size_t few_lds(int kc, int rows, bool tables) {
  const size_t loop = size_t(FewLds<D, NQ>::SMU) * 4 + (tables ? size_t(kc) * FewLds<D, NQ>::TS * 2 : 0) +
                      size_t(few_waves(NQ, tables)) * FewLds<D, NQ>::VW * 4;
  const size_t merge = size_t(few_waves(NQ, tables)) * rows * (D + 4 + 2) * 4;
  return loop > merge ? loop : merge;
}

template <int D, int G, int RP, int NQ, bool TAB, bool SI8>
hipError_t launch_k(const AttendArgs& a, int batch, hipStream_t s) {
  static std::atomic<uint64_t> raised{0};  // devices whose dynamic LDS limit is raised for this instance
  const size_t lds = few_lds<D, NQ>(a.n_centroids, a.block_rows, TAB);
  if (lds > kLdsLimit) return hipErrorInvalidValue;
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
  if (!bit || !(raised.load(std::memory_order_acquire) & bit)) {
    e = hipFuncSetAttribute((const void*)attend_few_kernel<D, G, RP, NQ, TAB, SI8>,
                            hipFuncAttributeMaxDynamicSharedMemorySize, int(kLdsLimit));
    if (e != hipSuccess) return e;
    raised.fetch_or(bit, std::memory_order_release);
  }
  const dim3 grid((unsigned)a.n_split * (unsigned)a.heads * (unsigned)(a.q_blocks * batch));
  hipLaunchKernelGGL((attend_few_kernel<D, G, RP, NQ, TAB, SI8>), grid, dim3(64 * few_waves(NQ, TAB)), lds, s, a);
  return hipGetLastError();
}

template <int D, int G, int RP, int NQ>
hipError_t launch_n(const AttendArgs& a, int batch, hipStream_t s) {
  if constexpr (NQ == 1) {
    // the Value table is worth its staging once a part has as many keys as it has rows
    // (launches of more than 16 Queries are taken with thousands of keys)
    if (a.chunks_per_part * kFewChunk < int64_t(a.n_centroids))
      return a.L.i8 ? launch_k<D, G, RP, 1, false, true>(a, batch, s) : launch_k<D, G, RP, 1, false, false>(a, batch, s);
  }
  return a.L.i8 ? launch_k<D, G, RP, NQ, true, true>(a, batch, s) : launch_k<D, G, RP, NQ, true, false>(a, batch, s);
}

template <int D, int G, int RP>
hipError_t launch_g(const AttendArgs& a, int batch, hipStream_t s) {
  return a.block_rows <= 16 ? launch_n<D, G, RP, 1>(a, batch, s) : launch_n<D, G, RP, 2>(a, batch, s);
}

}  // namespace

template <int D, int RP>
hipError_t launch_attend_few_rp(const AttendArgs& a, int batch, hipStream_t s) {
  const int g = D / a.L.ng;
  if (g == 16) return launch_g<D, 16, RP>(a, batch, s);
  if (g == 32) return launch_g<D, 32, RP>(a, batch, s);
  if (g == 64) return launch_g<D, 64, RP>(a, batch, s);
  return hipErrorInvalidValue;
}

template hipError_t launch_attend_few_rp<QWM_ATTEND_D, QWM_ATTEND_RP>(const AttendArgs&, int, hipStream_t);

}  // namespace qwm
