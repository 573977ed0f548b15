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
// lane holds half a key's channels and turns their codes into binary16 operands
// s (code - z) with packed arithmetic (the channel order of a contraction is free, so
// its codes are contiguous bytes); the Query is held as binary16 too, times the power
// of two that puts its largest magnitude in [2^14, 2^15), which keeps every BF16 value
// exact that is not 2^-29 times smaller. Values are decoded by key pairs to BF16 into a
// wave-private transposed tile (V^T rows of 32 keys), the A operand of O^T += V^T P^T.
// Packed fields are loaded two steps ahead.
// A workgroup runs one part of one segment (an epoch's keys or the exact chunk), so its
// tables, scales and q U_r never change; its waves merge their softmax states through
// LDS, and the parts are merged by the combine kernel.
#include "attend_device.h"
#include "attend_shape.h"
#include "few_shape.h"
#include "xcd_order.h"

#include <atomic>

namespace qwm {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// LDS: the products q . mu of every centroid and Query ([256][32] floats: an id is a
// byte, so none reads past it), the Value table (TAB, binary16) and a V^T tile per
// wave, in 32-bit words (key pairs): 64 channels of 16 pairs + 2 words of padding, the
// upper 32 channels 16 words further. The pair stores of a wave (four runs of 16 rows)
// and the 8-byte operand reads are then free of bank conflicts.
template <int D>
struct FewLds {
  static constexpr int SMU = 256 * kFewQ, ROW = 18, VW = 64 * ROW + 16, TS = D + 8;
  static __device__ inline int at(int row) { return row * ROW + row / 32 * 16; }
};

// Packed fields of one 32-key chunk in a lane between their load and their use.
template <int D, int RP, bool SI8>
struct FewRegs {
  uint32_t k_c[D / 32], k_z, k_s[2];       // half a Key's codes, zero-points and scales (codes)
  uint32_t k_id[4];                        // ids of the keys of this lane's accumulator rows, by four
  uint32_t k_sg[SI8 ? 8 : 1];              // their secondary scales, by two
  uint32_t c_w[RP > 0 ? RP / 8 : 1], c_s;  // ranks of this lane, by four
  uint32_t v_c[2][D / 64], v_id, v_z[2], v_s[2], v_sg[2];  // a quarter of two Values
};

// TAB: the Value table in LDS, for parts with at least as many keys as it has rows, with
// eight waves; shorter parts gather its rows and run in workgroups of four waves, of
// which a CU holds two (480 workgroups of 131 keys: one round instead of two).
constexpr int few_waves(bool tab) { return tab ? kFewWaves : kFewWaves / 2; }

template <int D, int G, int RP, bool TAB, bool SI8>
__global__ __launch_bounds__(64 * few_waves(TAB)) void attend_few_kernel(const AttendArgs a) {
  typedef Mfma<bf16> MF;
  typedef MF::V V;
  typedef FewLds<D> LY;
  constexpr int NW = few_waves(TAB), CK = kFewChunk, KW = D / 32, VWD = D / 64;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
  const int Kc = a.n_centroids;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, l32 = lane % 32,
            hf = lane / 32;
  uint32_t bx, by, bz;
  {
    const uint32_t gx = gridDim.x, gy = gridDim.y, n = gx * gy * gridDim.z;
    const uint32_t task = qwm_xcd_task(blockIdx.x + gx * (blockIdx.y + gy * blockIdx.z), n);
    bx = task % gx;
    by = (task / gx) % gy;
    bz = task / (gx * gy);
  }
  const int h = int(by), b = int(bz);
  const int64_t bh = int64_t(b) * a.heads + h;
  const int part = int(bx) % a.n_split;
  const int64_t qa = int64_t(bx / a.n_split) * kFewQ, qb = qa + kFewQ < a.n_q ? qa + kFewQ : a.n_q;
  const int rows = int(qb - qa);
  const int64_t nc = a.n_cache + a.n_act, F = a.frame_tokens;
  const FewReach reach = few_reach(a.q_start, F, nc, a.n_sink, a.window, a.windowed != 0, qa, qb);

  int64_t before = 0;
  const int seg = few_segment_at(a, reach, part, lane, before);
  const bool act = seg == a.n_epochs;
  FewSegment g{};
  if (!act || a.n_act > 0) g = few_segment_of(a, seg, reach);
  const int64_t cpp = a.chunks_per_part, t0 = (part - before) * cpp, t1 = t0 + cpp < g.chunks ? t0 + cpp : g.chunks;
  float* plane_ml = a.part_ml ? a.part_ml + 2 * ((int64_t(part) * a.heads * gridDim.z + bh) * a.n_q + qa) : nullptr;
  if (t0 >= t1 && a.part_o) {  // this block of Queries has fewer parts than another: an empty plane
    if (threadIdx.x < rows) {
      plane_ml[2 * threadIdx.x] = -__builtin_inff();
      plane_ml[2 * threadIdx.x + 1] = 0.0f;
    }
    return;
  }
  auto key_of = [&](int64_t t) __attribute__((always_inline)) { return g.base + (t >= g.cut ? t + g.skip : t) * CK; };

  const uint8_t* slab = a.calib + int64_t(act ? 0 : seg) * a.calib_stride + bh * a.slab;
  const bf16* gK = reinterpret_cast<const bf16*>(slab + a.o_mu_k);
  const bf16* gV = reinterpret_cast<const bf16*>(slab + a.o_mu_v16);  // binary16 bits
  float* smu = reinterpret_cast<float*>(smem_raw);
  bf16* tabV = reinterpret_cast<bf16*>(smu + LY::SMU);
  uint32_t* vt = reinterpret_cast<uint32_t*>(tabV + (TAB ? Kc * LY::TS : 0)) + wave * LY::VW;
  const int r = a.rank;
  const int qi = int(qa) + l32;
  const bool qvalid = l32 < rows;

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
  constexpr int HK = D / 2, HV = D / 4;     // channels of a lane: half a Key, a quarter of two Values
  // key pair and channel quarter: the lanes of a pair are neighbours, so that lanes
  // which read LDS together read few different rows of the Value table
  const int vp = lane / 4, vq = lane % 4;
  const int kg0 = hf * HK / G, vg0 = vq * HV / G;  // first group of the lane's channels
  constexpr int kgn = HK / G > 1 ? HK / G : 1, vgn = HV / G > 1 ? HV / G : 1;
  // scale bytes of n groups (a constant) at voffset o. The loads hold no branch, here
  // and below: at a join the compiler could only wait for all of them.
  auto load_scales = [&](auto rsrc, auto n, int o, int so, uint32_t& w0, uint32_t& w1) __attribute__((always_inline)) {
    constexpr uint32_t bytes = uint32_t(decltype(n)::value) * u8;
    if constexpr (bytes == 8) {
      const auto v = __builtin_amdgcn_raw_buffer_load_b64(rsrc, o, so, 0);
      w0 = v[0];
      w1 = v[1];
    } else if constexpr (bytes == 4) {
      w0 = __builtin_amdgcn_raw_buffer_load_b32(rsrc, o, so, 0);
    } else if constexpr (bytes == 2) {
      w0 = uint16_t(__builtin_amdgcn_raw_buffer_load_b16(rsrc, o, so, 0));
    } else {
      w0 = uint8_t(__builtin_amdgcn_raw_buffer_load_b8(rsrc, o, so, 0));
    }
  };
  typedef FewRegs<D, RP, SI8> Regs;
  auto load = [&](Regs& p, int64_t t) __attribute__((always_inline)) {
    const int k0 = int(key_of(t));
    if constexpr (KW == 4) {
      const auto c = __builtin_amdgcn_raw_buffer_load_b128(r_kc, l32 * (D / 4) + hf * (D / 8), k0 * (D / 4), 0);
#pragma unroll
      for (int u = 0; u < 4; ++u) p.k_c[u] = c[u];
    } else {
      const auto c = __builtin_amdgcn_raw_buffer_load_b64(r_kc, l32 * (D / 4) + hf * (D / 8), k0 * (D / 4), 0);
#pragma unroll
      for (int u = 0; u < 2; ++u) p.k_c[u] = c[u];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) p.k_id[i] = __builtin_amdgcn_raw_buffer_load_b32(r_ki, 8 * i + 4 * hf, k0, 0);
    p.k_z = uint8_t(__builtin_amdgcn_raw_buffer_load_b8(r_kz, l32 * int(zpb) + kg0 / 4, k0 * int(zpb), 0));
    load_scales(r_ks, std::integral_constant<int, kgn>{}, l32 * int(ss) + kg0 * int(u8), k0 * int(ss), p.k_s[0], p.k_s[1]);
    if constexpr (SI8) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const auto v = __builtin_amdgcn_raw_buffer_load_b64(r_ksg, 16 * i + 8 * hf, 2 * k0, 0);
        p.k_sg[2 * i] = v[0];
        p.k_sg[2 * i + 1] = v[1];
      }
    }
    if constexpr (RP > 0) {
      // ranks 8 i + 4 hf ... + 3 for i < RP / 8: the rows that q U_r's fragment has (r is
      // a multiple of 4). Ranks past r read as 0, past the end of the resource.
      constexpr uint32_t kAbsent = 0xC0000000u;
      p.c_s = uint16_t(__builtin_amdgcn_raw_buffer_load_b16(r_cs, 2 * l32, 2 * k0, 0));
#pragma unroll
      for (int i = 0; i < RP / 8; ++i) {
        const int k = 8 * i + 4 * hf;
        p.c_w[i] = __builtin_amdgcn_raw_buffer_load_b32(r_cc, int(k < r ? uint32_t(l32 * r + k) : kAbsent), k0 * r, 0);
      }
    }
    p.v_id = uint16_t(__builtin_amdgcn_raw_buffer_load_b16(r_vi, 2 * vp, k0, 0));
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int key = 2 * vp + e;
      if constexpr (VWD == 2) {
        const auto c = __builtin_amdgcn_raw_buffer_load_b64(r_vc, key * (D / 4) + vq * (D / 16), k0 * (D / 4), 0);
        p.v_c[e][0] = c[0];
        p.v_c[e][1] = c[1];
      } else {
        p.v_c[e][0] = __builtin_amdgcn_raw_buffer_load_b32(r_vc, key * (D / 4) + vq * (D / 16), k0 * (D / 4), 0);
      }
      p.v_z[e] = uint8_t(__builtin_amdgcn_raw_buffer_load_b8(r_vz, key * int(zpb) + vg0 / 4, k0 * int(zpb), 0));
      uint32_t none = 0;
      load_scales(r_vs, std::integral_constant<int, vgn>{}, key * int(ss) + vg0 * int(u8), k0 * int(ss), p.v_s[e], none);
      if constexpr (SI8) p.v_sg[e] = uint16_t(__builtin_amdgcn_raw_buffer_load_b16(r_vsg, 2 * key, 2 * k0, 0));
    }
  };

  // ---- everything that a part starts with, in flight at once and in the order of its
  // use: the Query, this wave's first rows of the Key table, U_r, the packed fields
  V qf[D / 16], ck[D / 16], cu[D / 16];
  const bf16* qrow = reinterpret_cast<const bf16*>(a.q) + ((int64_t(b) * a.n_q + (qvalid ? qi : qa)) * a.heads + h) * D + hf * HK;
  auto load_row = [&](const bf16* row, V (&to)[D / 16]) __attribute__((always_inline)) {
#pragma unroll
    for (int st = 0; st < D / 16; ++st) to[st] = *reinterpret_cast<const V*>(row + st * 8);
  };
  auto centroids = [&](int z0) __attribute__((always_inline)) {
    load_row(gK + int64_t(z0 + l32 < Kc ? z0 + l32 : Kc - 1) * D + hf * HK, ck);
  };
  Regs P0, P1;
  int ev = 0;  // Values are decoded times 2^-e_v, the exponent of their binary16 table
  load_row(qrow, qf);
  if (!act) {
    ev = reinterpret_cast<const int32_t*>(slab + a.o_e16)[1];
    centroids(wave * 32);
    if constexpr (RP > 0)
      load_row(reinterpret_cast<const bf16*>(slab + a.o_u_t) + int64_t(l32 < r ? l32 : 0) * D + hf * HK, cu);
    __builtin_amdgcn_sched_barrier(0);
    if (t0 < t1) {
      load(P0, t0 + wave < t1 ? t0 + wave : t1 - 1);
      load(P1, t0 + wave + NW < t1 ? t0 + wave + NW : t1 - 1);
    }
    if constexpr (TAB) {
      constexpr int PER_ROW = D * 2 / 16;
      const uint4* sv = reinterpret_cast<const uint4*>(gV);
      for (int i = threadIdx.x; i < Kc * PER_ROW; i += 64 * NW)
        *reinterpret_cast<uint4*>(tabV + i / PER_ROW * LY::TS + i % PER_ROW * 8) = sv[i];
    }
    __builtin_amdgcn_sched_barrier(0);
  }

  // ---- Query fragment: step st of lane half hf holds channels hf D/2 + 8 st ... + 7.
  // Everything that a Query multiplies is in units of 2^qe: the BF16 copy holds
  // q 2^-qe, the binary16 one q 2^(2 - qe), against Key residuals times 2^-2 (a step is a
  // binary16 value and three of them stay in its range).
  float qmax = 0.0f;
#pragma unroll
  for (int st = 0; st < D / 16; ++st)
#pragma unroll
    for (int j = 0; j < 8; ++j) qmax = fmaxf(qmax, fabsf(float(qf[st][j])));
  qmax = qvalid ? max_halves(qmax) : 0.0f;
  const int qe = qmax > 0.0f ? ilogbf(qmax) - 12 : 0;
#pragma unroll
  for (int st = 0; st < D / 16; ++st)
#pragma unroll
    for (int j = 0; j < 8; ++j) qf[st][j] = bf16(qvalid ? ldexpf(float(qf[st][j]), -qe) : 0.0f);

  V ureg[RP > 0 ? RP / 16 : 1];
  if (!act) {
    // q . mu of every centroid: rows = centroids, columns = Queries
    for (int z0 = wave * 32; z0 < Kc; z0 += NW * 32) {
      f32x16 acc;
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[i] = 0.0f;
#pragma unroll
      for (int st = 0; st < D / 16; ++st) acc = MF::run(ck[st], qf[st], acc);
      if (z0 + NW * 32 < Kc) centroids(z0 + NW * 32);
#pragma unroll
      for (int i = 0; i < 16; ++i) smu[(z0 + acc_row(i, hf)) * kFewQ + l32] = acc[i];
    }
    // q U_r (rows = ranks of U_r^T)
    if constexpr (RP > 0) {
      f32x16 u;
#pragma unroll
      for (int i = 0; i < 16; ++i) u[i] = 0.0f;
#pragma unroll
      for (int st = 0; st < D / 16; ++st) u = MF::run(l32 < r ? cu[st] : V{}, qf[st], u);
#pragma unroll
      for (int st = 0; st < RP / 16; ++st)
#pragma unroll
        for (int j = 0; j < 8; ++j) ureg[st][j] = bf16(u[st * 8 + j]);
    }
  }
  ev = __builtin_amdgcn_readfirstlane(ev);
  const float scv = ldexpf(1.0f, -ev);
  // the binary16 copy, in the channel order of the decoded operands: pairs (c, c + 8) of
  // 16 channels, the exact chunk's operands in their own order
  V qreg[D / 16];
#pragma unroll
  for (int st = 0; st < D / 16; ++st) {
    f16x8 x;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (_Float16)(4.0f * float(qf[(st & ~1) + j % 2][st % 2 * 4 + j / 2]));
    qreg[st] = act ? qf[st] : __builtin_bit_cast(V, x);
  }
  __syncthreads();

  float m_run = -__builtin_inff(), l_run = 0.0f;
  f32x16 oacc[D / 32];
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
    for (int i = 0; i < 16; ++i) oacc[cb][i] = 0.0f;
  int lim = int(nc), wfrom = 0;
  {
    const int64_t l = a.q_start + (qi / F + 1) * F, w = a.windowed ? l - a.window : 0;
    lim = int(l < nc ? l : nc);
    wfrom = int(w < 0 ? 0 : (w < nc ? w : nc));
  }
  // as in attend.hip; logits and their maxima are in units of the lane's 2^qe
  const float mscale = 1.4426950408889634f / sqrtf((float)D), lscale = ldexpf(mscale, qe), tau = 8.0f / lscale;

  // binary16 scale (SI8: scale code) of word u of a lane's channels
  auto scale_of = [&](const uint32_t (&w)[2], int u) __attribute__((always_inline)) {
    const int i = 16 * u / G;
    if constexpr (SI8) {
      return (_Float16)(int)((w[0] >> (8 * i)) & 255);
    } else {
      const uint32_t word = i < 2 ? w[0] : w[1];
      return __builtin_bit_cast(_Float16, uint16_t(word >> (16 * (i & 1))));
    }
  };
  auto zero_of = [&](uint32_t zb, int g0, int u) __attribute__((always_inline)) {
    return (0x6400u + ((zb >> (2 * (g0 % 4 + 16 * u / G))) & 3)) * 0x00010001u;
  };
  auto id_of = [&](uint32_t id) __attribute__((always_inline)) { return int(id) < Kc ? int(id) : Kc - 1; };

  // masks the logits s of one chunk and turns them into BF16 weights, the B operands of
  // the Value product
  auto weigh = [&](f32x16& s, int64_t k0, V (&bv)[2]) __attribute__((always_inline)) {
    if (k0 < g.lo || k0 + CK > (reach.kfull < g.hi ? reach.kfull : g.hi) ||
        (k0 + CK > reach.ns && k0 < reach.wfull)) {
      const int klo = int(g.lo), khi = int(g.hi) < lim ? int(g.hi) : lim;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = int(k0) + acc_row(i, hf);
        if (key >= khi || key < klo || (key >= int(reach.ns) && key < wfrom)) s[i] = -__builtin_inff();
      }
    }
    float mt = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < 8; ++i) mt = max3f(mt, s[2 * i], s[2 * i + 1]);
    mt = max_halves(mt);
    if (__any(mt > m_run + tau)) {
      const float m_new = fmaxf(m_run, mt);
      const float alpha = m_new == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f((m_run - m_new) * lscale);
      l_run *= alpha;
#pragma unroll
      for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
        for (int i = 0; i < 16; ++i) oacc[cb][i] *= alpha;
      m_run = m_new;
    }
    const float mc = m_run == -__builtin_inff() ? 0.0f : -m_run * lscale;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], lscale, mc));
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float pv[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) pv[j] = s[t * 8 + j];
      bv[t] = pack_operand<V>(pv);
      // the sum of the weights as rounded for the product
      const bf16x2 one = {bf16(1.0f), bf16(1.0f)};
      const uint4 pw = __builtin_bit_cast(uint4, bv[t]);
      const uint32_t w[4] = {pw.x, pw.y, pw.z, pw.w};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        l_run = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[j]), one, l_run, false);
    }
  };
  // A wave's stores to its tile, then its reads, then its next stores: LDS keeps a wave's
  // order, and these keep the compiler's
  auto in_order = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  // O^T += V^T P^T for the 64 channels in the tile (accumulators 2 u and 2 u + 1)
  auto value_product = [&](const V (&bv)[2], int u) __attribute__((always_inline)) {
    in_order();
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        // keys acc_row(8 t + j, hf): two runs of four
        const uint32_t* row = vt + LY::at(32 * x + l32) + 8 * t + 2 * hf;
        const uint2 y = *reinterpret_cast<const uint2*>(row), z = *reinterpret_cast<const uint2*>(row + 4);
        oacc[2 * u + x] = MF::run(__builtin_bit_cast(V, make_uint4(y.x, y.y, z.x, z.y)), bv[t], oacc[2 * u + x]);
      }
    in_order();
  };

  auto step = [&](Regs& p, int64_t t) __attribute__((always_inline)) {
    const int64_t k0 = key_of(t);
    f32x16 s;
    // q . mu of the keys of this lane's accumulator rows
    float mu[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) mu[i] = smu[((p.k_id[i / 4] >> (8 * (i % 4))) & 255) * kFewQ + l32];
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = SI8 ? 0.0f : mu[i];
#pragma unroll
    for (int u = 0; u < KW; ++u) {
      // SI8: the integers c (code - z), exact; else s 2^-2 (code - z)
      const _Float16 c = SI8 ? scale_of(p.k_s, u) : scale_of(p.k_s, u) * (_Float16)0.25f;
      const f16x2 cc = {c, c}, zh = __builtin_bit_cast(f16x2, zero_of(p.k_z, kg0, u));
      uint32_t w[8];
#pragma unroll
      for (int k = 0; k < 8; ++k)
        w[k] = __builtin_bit_cast(uint32_t, (__builtin_bit_cast(f16x2, and_or(p.k_c[u] >> (2 * k), 0x00030003u, 0x64006400u)) - zh) * cc);
#pragma unroll
      for (int x = 0; x < 2; ++x)
        s = __builtin_amdgcn_mfma_f32_32x32x16_f16(
            __builtin_bit_cast(f16x8, make_uint4(w[4 * x], w[4 * x + 1], w[4 * x + 2], w[4 * x + 3])),
            __builtin_bit_cast(f16x8, qreg[2 * u + x]), s, 0, 0, 0);
    }
    if constexpr (SI8) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const _Float16 sg = __builtin_bit_cast(_Float16, uint16_t(p.k_sg[i / 2] >> (16 * (i % 2))));
        s[i] = __builtin_fmaf(s[i], 0.25f * (float)sg, mu[i]);
      }
    }
    if constexpr (RP > 0) {
      const float cs = (float)__builtin_bit_cast(_Float16, uint16_t(p.c_s));
#pragma unroll
      for (int st = 0; st < RP / 16; ++st) {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = (float)int8_t((p.c_w[2 * st + j / 4] >> (8 * (j % 4))) & 255) * cs;
        s = MF::run(pack_operand<V>(x), ureg[st], s);
      }
    }
    // Values of 16 channels of each quarter at a time. Keys of the neighbouring epoch
    // before the segment's first take scale 0: finite, whatever they hold
    const int id0 = id_of(p.v_id & 255), id1 = id_of(p.v_id >> 8);
    const bool in0 = k0 + 2 * vp >= g.lo, in1 = k0 + 2 * vp + 1 >= g.lo;
    auto values = [&](int u) __attribute__((always_inline)) {
      float m0[16], m1[16], x0[16], x1[16];
      const int c0 = vq * HV + 16 * u;
      load_tab<true, bf16, 16>((TAB ? tabV + id0 * LY::TS : gV + id0 * D) + c0, m0);
      load_tab<true, bf16, 16>((TAB ? tabV + id1 * LY::TS : gV + id1 * D) + c0, m1);
      const uint32_t w0[2] = {p.v_s[0], 0}, w1[2] = {p.v_s[1], 0};
      const _Float16 y0 = scale_of(w0, u), y1 = scale_of(w1, u);
      const f16x2 cm0 = {y0, y0}, cm1 = {y1, y1};
      float s0 = SI8 ? (float)__builtin_bit_cast(_Float16, uint16_t(p.v_sg[0])) : (float)y0;
      float s1 = SI8 ? (float)__builtin_bit_cast(_Float16, uint16_t(p.v_sg[1])) : (float)y1;
      s0 = in0 ? s0 * scv : 0.0f;
      s1 = in1 ? s1 * scv : 0.0f;
      dequant_codes<16, SI8>(p.v_c[0][u], s0, zero_of(p.v_z[0], vg0, u), m0, x0, cm0);
      dequant_codes<16, SI8>(p.v_c[1][u], s1, zero_of(p.v_z[1], vg0, u), m1, x1, cm1);
#pragma unroll
      for (int c = 0; c < 16; ++c) vt[LY::at(16 * vq) + c * LY::ROW + vp] = pack_bf16(x0[c], x1[c]);
    };
    V bv[2];
    values(0);
    weigh(s, k0, bv);
    value_product(bv, 0);
    if constexpr (VWD == 2) {
      values(1);
      value_product(bv, 1);
    }
    // past the last chunk that one again: an unconditional load, so that the waits
    // before the other set's use leave these loads in flight
    load(p, t + 2 * NW < t1 ? t + 2 * NW : t1 - 1);
  };

  if (!act) {
    int64_t t = t0 + wave;
    for (; t + NW < t1; t += 2 * NW) {
      step(P0, t);
      step(P1, t + NW);
    }
    if (t < t1) step(P0, t);
  } else {
    // exact rows: operands straight from memory, the last row again past the end
    const bf16* ka = reinterpret_cast<const bf16*>(a.k_act);
    const bf16* va = reinterpret_cast<const bf16*>(a.v_act);
    const int64_t last = a.n_act - 1;
    auto row_of = [&](const bf16* base, int64_t i) { return base + ((int64_t(b) * a.n_act + (i < last ? i : last)) * a.heads + h) * D; };
    for (int64_t t = t0 + wave; t < t1; t += NW) {
      const int64_t k0 = key_of(t), r0 = k0 - a.n_cache;
      const bf16* krow = row_of(ka, r0 + l32) + hf * HK;
      V kv[D / 16];
#pragma unroll
      for (int st = 0; st < D / 16; ++st) kv[st] = *reinterpret_cast<const V*>(krow + st * 8);
      const uint4* v0 = reinterpret_cast<const uint4*>(row_of(va, r0 + 2 * vp) + vq * HV);
      const uint4* v1 = reinterpret_cast<const uint4*>(row_of(va, r0 + 2 * vp + 1) + vq * HV);
      uint4 x0[HV / 8], x1[HV / 8];
#pragma unroll
      for (int i = 0; i < HV / 8; ++i) {
        x0[i] = v0[i];
        x1[i] = v1[i];
      }
      f32x16 s;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
      for (int st = 0; st < D / 16; ++st) s = MF::run(kv[st], qreg[st], s);
      V bv[2];
      weigh(s, k0, bv);
#pragma unroll
      for (int u = 0; u < VWD; ++u) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint4 y = x0[2 * u + i], z = x1[2 * u + i];
          const uint32_t p0[4] = {y.x, y.y, y.z, y.w}, p1[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t* to = vt + LY::at(16 * vq) + (8 * i + 2 * j) * LY::ROW + vp;
            to[0] = __builtin_amdgcn_perm(p1[j], p0[j], 0x05040100u);
            to[LY::ROW] = __builtin_amdgcn_perm(p1[j], p0[j], 0x07060302u);
          }
        }
        value_product(bv, u);
      }
    }
  }

  // ---- merge of the waves: every wave's O rows, running max and sum through LDS (the
  // tables and V^T tiles are done with)
  constexpr int OS = D + 4;
  float* mo = reinterpret_cast<float*>(smem_raw);  // [wave][row][OS]
  float* ml = mo + NW * rows * OS;                 // [wave][row][2]
  const float l_tot = l_run + __shfl_xor(l_run, 32);
  __syncthreads();
  if (qvalid) {
    float* orow = mo + (wave * rows + l32) * OS;
#pragma unroll
    for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = 32 * (cb % 2) + acc_row(4 * i, hf);  // of the tile: 16 channels of each quarter
        *reinterpret_cast<float4*>(orow + row / 16 * HV + cb / 2 * 16 + row % 16) =
            make_float4(oacc[cb][4 * i], oacc[cb][4 * i + 1], oacc[cb][4 * i + 2], oacc[cb][4 * i + 3]);
      }
    if (hf == 0) {
      ml[2 * (wave * rows + l32)] = ldexpf(m_run, qe);
      ml[2 * (wave * rows + l32) + 1] = l_tot;
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
      a.part_o[((int64_t(part) * a.heads * gridDim.z + bh) * a.n_q + qa + q) * D + c] = ldexpf(o, ev);
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

template <int D>
size_t few_lds(int kc, int rows, bool tables) {
  const size_t loop = size_t(FewLds<D>::SMU) * 4 + (tables ? size_t(kc) * FewLds<D>::TS * 2 : 0) +
                      size_t(few_waves(tables)) * FewLds<D>::VW * 4;
  const size_t merge = size_t(few_waves(tables)) * rows * (D + 4 + 2) * 4;
  return loop > merge ? loop : merge;
}

template <int D, int G, int RP, bool TAB, bool SI8>
hipError_t launch_k(const AttendArgs& a, const dim3& grid, size_t lds, hipStream_t s) {
  static std::atomic<uint64_t> raised{0};  // devices whose dynamic LDS limit is raised for this instance
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
  if (!bit || !(raised.load(std::memory_order_acquire) & bit)) {
    e = hipFuncSetAttribute((const void*)attend_few_kernel<D, G, RP, TAB, SI8>, hipFuncAttributeMaxDynamicSharedMemorySize,
                            int(kLdsLimit));
    if (e != hipSuccess) return e;
    raised.fetch_or(bit, std::memory_order_release);
  }
  hipLaunchKernelGGL((attend_few_kernel<D, G, RP, TAB, SI8>), grid, dim3(64 * few_waves(TAB)), lds, s, a);
  return hipGetLastError();
}

template <int D, int G, int RP>
hipError_t launch_g(const AttendArgs& a, int batch, hipStream_t s) {
  const int rows = int(a.n_q < kFewQ ? a.n_q : kFewQ);
  const dim3 grid((unsigned)((a.n_q + kFewQ - 1) / kFewQ * a.n_split), (unsigned)a.heads, (unsigned)batch);
  // the Value table is worth its staging once a part has as many keys as it has rows
  const bool tab = few_lds<D>(a.n_centroids, rows, true) <= kLdsLimit &&
                   a.chunks_per_part * kFewChunk >= int64_t(a.n_centroids);
  const size_t lds = few_lds<D>(a.n_centroids, rows, tab);
  if (lds > kLdsLimit) return hipErrorInvalidValue;
  if (a.L.i8)
    return tab ? launch_k<D, G, RP, true, true>(a, grid, lds, s) : launch_k<D, G, RP, false, true>(a, grid, lds, s);
  return tab ? launch_k<D, G, RP, true, false>(a, grid, lds, s) : launch_k<D, G, RP, false, false>(a, grid, lds, s);
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
