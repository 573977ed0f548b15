// Attention of a few Queries (single tokens, a handful of rollouts) over the packed
// cache: the arithmetic of attend.hip (Eq. 5 with Eq. 17, BF16 operands, online base-2
// softmax), organised for launches that are bound by decoding the keys rather than by
// the products. There a workgroup's 256 Query rows would mostly be empty, and its four
// producer waves, one per SIMD, decode for eight consumers that have next to nothing
// to do. Here every wave decodes and multiplies its own runs of 32 keys, with no
// barrier between them:
//   - a lane holds half a key's channels (hf D/2 ...), decodes them straight into
//     matrix-core A operands (the channel order of the contraction is free, so a lane's
//     codes are contiguous bytes) and never writes a Key to LDS;
//   - Values are decoded by key pairs into a wave-private transposed tile (V^T rows of
//     32 keys), the A operand of O^T += V^T P^T;
//   - packed fields are loaded a step ahead.
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

constexpr int kFewThreads = 64 * kFewWaves;

// LDS of a wave's V^T tile, in 32-bit words (key pairs): rows of 16 pairs + 2 words of
// padding, each quarter of the channels 16 words further, which makes the pair stores
// of the four quarters and the 8-byte operand reads free of bank conflicts at d = 128.
template <int D>
struct FewLds {
  static constexpr int ROW = 18, VW = D * ROW + 3 * 16, TS = D + 8;
  static __device__ inline int at(int c) { return c * ROW + c / (D / 4) * 16; }
};

// Packed fields of one 32-key chunk in a lane between their load and their use.
template <int D, int RP>
struct FewRegs {
  uint32_t k_c[D / 32], k_id, k_z, k_s[2], k_sg;  // half a Key's codes, scales of its groups
  uint32_t c_w[RP > 0 ? RP / 8 : 1], c_s;         // ranks of this lane, by four
  uint32_t v_c[2][D / 64], v_id, v_z[2], v_s[2], v_sg[2];  // a quarter of two Values
};

template <int D, int RP, bool TAB, bool SI8>
__global__ __launch_bounds__(kFewThreads) void attend_few_kernel(const AttendArgs a) {
  typedef Mfma<bf16> MF;
  typedef MF::V V;
  typedef FewLds<D> LY;
  constexpr int NW = kFewWaves, CK = kFewChunk, KW = D / 32, VWD = D / 64;
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

  // ---- the segment of this part: a lane counts for each epoch
  const int64_t cpp = a.chunks_per_part;
  int seg = 0;
  int64_t before = 0;
  if (a.n_epochs == 1) {
    const int p0 = int((few_segment_of(a, 0, reach).chunks + cpp - 1) / cpp);
    if (part >= p0) {
      seg = 1;
      before = p0;
    }
  } else {
    static_assert(kMaxEpochs == 64, "a lane per epoch");
    int past = lane < a.n_epochs ? int((few_segment_of(a, lane, reach).chunks + cpp - 1) / cpp) : 0;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(past, o);
      past += lane >= o ? y : 0;
    }
    const uint64_t at = __ballot(past > part);
    seg = at ? __builtin_ctzll(at) : a.n_epochs;
    before = seg > 0 ? __builtin_amdgcn_readlane(past, seg - 1) : 0;
  }
  const bool act = seg == a.n_epochs;
  FewSegment g{};
  if (!act || a.n_act > 0) g = few_segment_of(a, seg, reach);
  const int64_t t0 = (part - before) * cpp, t1 = t0 + cpp < g.chunks ? t0 + cpp : g.chunks;
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
  const _Float16* gK = reinterpret_cast<const _Float16*>(slab + a.o_mu_k16);
  const _Float16* gV = reinterpret_cast<const _Float16*>(slab + a.o_mu_v16);
  bf16* tabK = reinterpret_cast<bf16*>(smem_raw);
  bf16* tabV = tabK + Kc * LY::TS;
  uint32_t* vt = reinterpret_cast<uint32_t*>(smem_raw + (TAB ? size_t(2) * Kc * LY::TS * 2 : 0)) + wave * LY::VW;
  int ek = 0, ev = 0;
  if (!act) {
    const int32_t* e16 = reinterpret_cast<const int32_t*>(slab + a.o_e16);
    ek = __builtin_amdgcn_readfirstlane(e16[0]);
    ev = __builtin_amdgcn_readfirstlane(e16[1]);
  }
  const float sck = ldexpf(1.0f, -ek), scv = ldexpf(1.0f, -ev);

  // ---- Query fragment: step st of lane half hf holds channels hf D/2 + 8 st ... + 7
  const int r = a.rank, G = D / a.L.ng;
  const int qi = int(qa) + l32;
  const bool qvalid = l32 < rows;
  V qreg[D / 16], ureg[RP > 0 ? RP / 16 : 1];
  const bf16* qrow = reinterpret_cast<const bf16*>(a.q) + ((int64_t(b) * a.n_q + (qvalid ? qi : qa)) * a.heads + h) * D + hf * (D / 2);
#pragma unroll
  for (int st = 0; st < D / 16; ++st) {
    qreg[st] = *reinterpret_cast<const V*>(qrow + st * 8);
    if (!qvalid) qreg[st] = V{};
  }

  // ---- packed fields
  const CacheLayout& L = a.L;
  const int64_t slot0 = bh * L.slots;
  const uint32_t zpb = L.zpb, ss = SI8 ? L.ng : 2 * L.ng, u8 = SI8 ? 1 : 2;
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
  constexpr int HK = D / 2, HV = D / 4;       // channels of a lane: half a Key, a quarter of two Values
  const int vp = lane % 16, vq = lane / 16;   // key pair and channel quarter
  const int kg0 = hf * HK / G, vg0 = vq * HV / G;  // first group of the lane's channels
  const int kgn = HK / G > 1 ? HK / G : 1, vgn = HV / G > 1 ? HV / G : 1;
  // scale bytes of n consecutive groups at voffset o: up to 8 bytes
  auto load_scales = [&](auto rsrc, int n, int o, int so, uint32_t& w0, uint32_t& w1) __attribute__((always_inline)) {
    const uint32_t bytes = uint32_t(n) * u8;
    if (bytes == 8) {
      const auto v = __builtin_amdgcn_raw_buffer_load_b64(rsrc, o, so, 0);
      w0 = v[0];
      w1 = v[1];
    } else if (bytes == 4) {
      w0 = __builtin_amdgcn_raw_buffer_load_b32(rsrc, o, so, 0);
    } else if (bytes == 2) {
      w0 = uint16_t(__builtin_amdgcn_raw_buffer_load_b16(rsrc, o, so, 0));
    } else {
      w0 = uint8_t(__builtin_amdgcn_raw_buffer_load_b8(rsrc, o, so, 0));
    }
  };
  typedef FewRegs<D, RP> Regs;
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
    p.k_id = uint8_t(__builtin_amdgcn_raw_buffer_load_b8(r_ki, l32, k0, 0));
    p.k_z = uint8_t(__builtin_amdgcn_raw_buffer_load_b8(r_kz, l32 * int(zpb) + kg0 / 4, k0 * int(zpb), 0));
    load_scales(r_ks, kgn, l32 * int(ss) + kg0 * int(u8), k0 * int(ss), p.k_s[0], p.k_s[1]);
    if constexpr (SI8) p.k_sg = uint16_t(__builtin_amdgcn_raw_buffer_load_b16(r_ksg, 2 * l32, 2 * k0, 0));
    if constexpr (RP > 0) {
      // ranks 8 i + 4 hf ... + 3 for i < RP / 8: the rows that q U_r's fragment has. Ranks
      // past r read as 0, past the end of the resource.
      constexpr uint32_t kAbsent = 0xC0000000u;
      p.c_s = uint16_t(__builtin_amdgcn_raw_buffer_load_b16(r_cs, 2 * l32, 2 * k0, 0));
#pragma unroll
      for (int i = 0; i < RP / 8; ++i) {
        const int k = 8 * i + 4 * hf;
        if (r % 4 == 0) {
          p.c_w[i] = __builtin_amdgcn_raw_buffer_load_b32(r_cc, int(k < r ? uint32_t(l32 * r + k) : kAbsent), k0 * r, 0);
        } else {
          p.c_w[i] = 0;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            p.c_w[i] |= uint32_t(uint8_t(__builtin_amdgcn_raw_buffer_load_b8(
                            r_cc, int(k + j < r ? uint32_t(l32 * r + k + j) : kAbsent), k0 * r, 0))) << (8 * j);
        }
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
      load_scales(r_vs, vgn, key * int(ss) + vg0 * int(u8), k0 * int(ss), p.v_s[e], none);
      if constexpr (SI8) p.v_sg[e] = uint16_t(__builtin_amdgcn_raw_buffer_load_b16(r_vsg, 2 * key, 2 * k0, 0));
    }
  };

  if constexpr (TAB) {
    if (!act) {
      constexpr int PER_ROW = D * 2 / 16;
      const uint4 *sk = reinterpret_cast<const uint4*>(gK), *sv = reinterpret_cast<const uint4*>(gV);
      for (int i = threadIdx.x; i < Kc * PER_ROW; i += kFewThreads) {
        const int row = i / PER_ROW, ch = i % PER_ROW;
        *reinterpret_cast<uint4*>(tabK + row * LY::TS + ch * 8) = sk[i];
        *reinterpret_cast<uint4*>(tabV + row * LY::TS + ch * 8) = sv[i];
      }
    }
    __syncthreads();
  }
  Regs P0, P1;
  if (!act) {
    if (t0 + wave < t1) load(P0, t0 + wave);
    if (t0 + wave + NW < t1) load(P1, t0 + wave + NW);
  }
  // q U_r on matrix cores (rows = ranks of U_r^T), then the Query times 2^e_k (exact in BF16)
  if constexpr (RP > 0) {
    if (act) {
#pragma unroll
      for (int st = 0; st < RP / 16; ++st) ureg[st] = V{};
    } else {
      const bf16* urow = reinterpret_cast<const bf16*>(slab + a.o_u_t) + int64_t(l32 < r ? l32 : 0) * D + hf * (D / 2);
      f32x16 u;
#pragma unroll
      for (int i = 0; i < 16; ++i) u[i] = 0.0f;
#pragma unroll
      for (int st = 0; st < D / 16; ++st) {
        V av = *reinterpret_cast<const V*>(urow + st * 8);
        if (l32 >= r) av = V{};
        u = MF::run(av, qreg[st], u);
      }
#pragma unroll
      for (int st = 0; st < RP / 16; ++st)
#pragma unroll
        for (int j = 0; j < 8; ++j) ureg[st][j] = bf16(u[st * 8 + j]);
    }
  }
#pragma unroll
  for (int st = 0; st < D / 16; ++st)
#pragma unroll
    for (int j = 0; j < 8; ++j) qreg[st][j] = bf16(ldexpf(float(qreg[st][j]), ek));

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
  const float mscale = 1.4426950408889634f / sqrtf((float)D), tau = 8.0f / mscale;  // as in attend.hip

  // the scale and the (1024 + z) pair of word u of a lane's channels
  auto scale_of = [&](const uint32_t (&w)[2], uint32_t sg, int u, float sc, f16x2& cm) __attribute__((always_inline)) {
    const int i = 16 * u / G;
    if constexpr (SI8) {
      const _Float16 c = (_Float16)(int)((w[0] >> (8 * i)) & 255);
      cm = f16x2{c, c};
      return (float)__builtin_bit_cast(_Float16, uint16_t(sg)) * sc;
    } else {
      const uint32_t word = i < 2 ? w[0] : w[1];
      return (float)__builtin_bit_cast(_Float16, uint16_t(word >> (16 * (i & 1)))) * sc;
    }
  };
  auto zero_of = [&](uint32_t zb, int g0, int u) __attribute__((always_inline)) {
    return (0x6400u + ((zb >> (2 * (g0 % 4 + 16 * u / G))) & 3)) * 0x00010001u;
  };
  auto id_of = [&](uint32_t id) __attribute__((always_inline)) { return int(id) < Kc ? int(id) : Kc - 1; };

  // softmax of the logits s of one chunk and O^T += V^T P^T, with V^T in this wave's tile
  auto finish = [&](f32x16& s, int64_t k0) __attribute__((always_inline)) {
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
      const float alpha = m_new == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f((m_run - m_new) * mscale);
      l_run *= alpha;
#pragma unroll
      for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
        for (int i = 0; i < 16; ++i) oacc[cb][i] *= alpha;
      m_run = m_new;
    }
    const float mc = m_run == -__builtin_inff() ? 0.0f : -m_run * mscale;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], mscale, mc));
    // the tile's stores are this wave's own: in order with its reads
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float pv[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) pv[j] = s[t * 8 + j];
      const V bv = pack_operand<V>(pv);
      const bf16x2 one = {bf16(1.0f), bf16(1.0f)};
      const uint4 pw = __builtin_bit_cast(uint4, bv);
      const uint32_t w[4] = {pw.x, pw.y, pw.z, pw.w};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        l_run = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[j]), one, l_run, false);
#pragma unroll
      for (int cb = 0; cb < D / 32; ++cb) {
        // keys acc_row(8 t + j, hf): two runs of four
        const uint32_t* row = vt + LY::at(cb * 32 + l32) + 8 * t + 2 * hf;
        const uint2 x = *reinterpret_cast<const uint2*>(row), y = *reinterpret_cast<const uint2*>(row + 4);
        oacc[cb] = MF::run(__builtin_bit_cast(V, make_uint4(x.x, x.y, y.x, y.y)), bv, oacc[cb]);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };

  auto step = [&](Regs& p, int64_t t) __attribute__((always_inline)) {
    const int64_t k0 = key_of(t);
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.0f;
    const int kid = id_of(p.k_id);
#pragma unroll
    for (int u = 0; u < KW; ++u) {
      float mu[16], x[16];
      if constexpr (TAB) load_tab<true, bf16, 16>(tabK + kid * LY::TS + hf * HK + 16 * u, mu);
      else load_tab<true, bf16, 16>(reinterpret_cast<const bf16*>(gK) + kid * D + hf * HK + 16 * u, mu);
      f16x2 cm = {};
      const float sc = scale_of(p.k_s, p.k_sg, u, sck, cm);
      dequant_codes<16, SI8>(p.k_c[u], sc, zero_of(p.k_z, kg0, u), mu, x, cm);
      s = MF::run(pack_operand<V>(x), qreg[2 * u], s);
      s = MF::run(pack_operand<V>(x + 8), qreg[2 * u + 1], s);
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
    {
      const int id0 = id_of(p.v_id & 255), id1 = id_of(p.v_id >> 8);
      // keys of the neighbouring epoch before the segment's first: scale 0, finite Values
      const bool in0 = k0 + 2 * vp >= g.lo, in1 = k0 + 2 * vp + 1 >= g.lo;
#pragma unroll
      for (int u = 0; u < VWD; ++u) {
        float m0[16], m1[16], x0[16], x1[16];
        const int c0 = vq * HV + 16 * u;
        if constexpr (TAB) {
          load_tab<true, bf16, 16>(tabV + id0 * LY::TS + c0, m0);
          load_tab<true, bf16, 16>(tabV + id1 * LY::TS + c0, m1);
        } else {
          load_tab<true, bf16, 16>(reinterpret_cast<const bf16*>(gV) + id0 * D + c0, m0);
          load_tab<true, bf16, 16>(reinterpret_cast<const bf16*>(gV) + id1 * D + c0, m1);
        }
        f16x2 cm0 = {}, cm1 = {};
        const uint32_t w0[2] = {p.v_s[0], 0}, w1[2] = {p.v_s[1], 0};
        const float v0 = scale_of(w0, p.v_sg[0], u, scv, cm0), v1 = scale_of(w1, p.v_sg[1], u, scv, cm1);
        const float s0 = in0 ? v0 : 0.0f, s1 = in1 ? v1 : 0.0f;
        dequant_codes<16, SI8>(p.v_c[0][u], s0, zero_of(p.v_z[0], vg0, u), m0, x0, cm0);
        dequant_codes<16, SI8>(p.v_c[1][u], s1, zero_of(p.v_z[1], vg0, u), m1, x1, cm1);
#pragma unroll
        for (int c = 0; c < 16; ++c) vt[LY::at(c0) + c * LY::ROW + vp] = pack_bf16(x0[c], x1[c]);
      }
    }
    if (t + 2 * NW < t1) load(p, t + 2 * NW);
    finish(s, k0);
  };

  if (!act) {
    for (int64_t t = t0 + wave; t < t1; t += 2 * NW) {
      step(P0, t);
      if (t + NW < t1) step(P1, t + NW);
    }
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
#pragma unroll
      for (int i = 0; i < HV / 8; ++i) {
        const uint32_t p0[4] = {x0[i].x, x0[i].y, x0[i].z, x0[i].w}, p1[4] = {x1[i].x, x1[i].y, x1[i].z, x1[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t* to = vt + LY::at(vq * HV) + (8 * i + 2 * j) * LY::ROW + vp;
          to[0] = __builtin_amdgcn_perm(p1[j], p0[j], 0x05040100u);
          to[LY::ROW] = __builtin_amdgcn_perm(p1[j], p0[j], 0x07060302u);
        }
      }
      finish(s, k0);
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
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(orow + cb * 32 + acc_row(4 * i, hf)) =
            make_float4(oacc[cb][4 * i], oacc[cb][4 * i + 1], oacc[cb][4 * i + 2], oacc[cb][4 * i + 3]);
    if (hf == 0) {
      ml[2 * (wave * rows + l32)] = m_run;
      ml[2 * (wave * rows + l32) + 1] = l_tot;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < rows * D; i += kFewThreads) {
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
  const size_t loop = (tables ? size_t(2) * kc * FewLds<D>::TS * 2 : 0) + size_t(kFewWaves) * FewLds<D>::VW * 4;
  const size_t merge = size_t(kFewWaves) * rows * (D + 4 + 2) * 4;
  return loop > merge ? loop : merge;
}

template <int D, int RP, bool TAB, bool SI8>
hipError_t launch_k(const AttendArgs& a, const dim3& grid, size_t lds, hipStream_t s) {
  static std::atomic<uint64_t> raised{0};  // devices whose dynamic LDS limit is raised for this instance
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
  if (!bit || !(raised.load(std::memory_order_acquire) & bit)) {
    e = hipFuncSetAttribute((const void*)attend_few_kernel<D, RP, TAB, SI8>, hipFuncAttributeMaxDynamicSharedMemorySize,
                            int(kLdsLimit));
    if (e != hipSuccess) return e;
    raised.fetch_or(bit, std::memory_order_release);
  }
  hipLaunchKernelGGL((attend_few_kernel<D, RP, TAB, SI8>), grid, dim3(kFewThreads), lds, s, a);
  return hipGetLastError();
}

}  // namespace

template <int D, int RP>
hipError_t launch_attend_few_rp(const AttendArgs& a, int batch, hipStream_t s) {
  const int rows = int(a.n_q < kFewQ ? a.n_q : kFewQ);
  const dim3 grid((unsigned)((a.n_q + kFewQ - 1) / kFewQ * a.n_split), (unsigned)a.heads, (unsigned)batch);
  // the tables are worth their staging once a part holds a few times their rows
  const bool tab = few_lds<D>(a.n_centroids, rows, true) <= kLdsLimit &&
                   a.chunks_per_part * kFewChunk >= int64_t(a.n_centroids);
  const size_t lds = few_lds<D>(a.n_centroids, rows, tab);
  if (lds > kLdsLimit) return hipErrorInvalidValue;
  if (a.L.i8) return tab ? launch_k<D, RP, true, true>(a, grid, lds, s) : launch_k<D, RP, false, true>(a, grid, lds, s);
  return tab ? launch_k<D, RP, true, false>(a, grid, lds, s) : launch_k<D, RP, false, false>(a, grid, lds, s);
}

template hipError_t launch_attend_few_rp<QWM_ATTEND_D, QWM_ATTEND_RP>(const AttendArgs&, int, hipStream_t);

}  // namespace qwm
