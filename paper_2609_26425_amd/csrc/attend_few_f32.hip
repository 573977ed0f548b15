// Attention over the packed cache in fp32 for launches that do not fill the GPU: the
// tiling of attend_few.hip (a wave decodes and multiplies its own runs of 32 keys for a
// block of 32 Queries, a workgroup runs one part of one segment, parts are merged by
// join_planes) with fp32 operands. The fp32 matrix cores take 16 times as long as
// the BF16 ones over a product (4,096 cycles for 32 Queries x 32 keys at d = 64), so
// decoding the keys again for every block of Queries costs little, and spreading the
// blocks and key runs over the SIMDs is what counts: with workgroups of 256 Query rows,
// 2 heads x 257 Queries give two row blocks a head, one of them with a single row.
// Keys are decoded into operands in registers (half a key's channels a lane), Values
// into a wave-private tile of 32 rows.
//
// Bound by its chain of loads, centroid gathers and products: with a chunk or two a wave
// there is nothing to hide them behind. 2 heads x 257 Queries with 305 to 361 keys in reach
// (d = 64, rank 4): 13 us and 4 for the merge, against 29 with 256-row workgroups.
#include "attend_device.h"
#include "attend_shape.h"
#include "few_shape.h"

#include <atomic>

namespace qwm {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kF32Waves = 4;

template <int D>
struct FewTile {  // fp32 Values of 32 keys; rows padded by 16 bytes
  static constexpr int ROW = D + 4, FLOATS = kFewChunk * ROW;
};

// Packed fields of one 32-key chunk in a lane: half of one key's channels, of which a
// word of codes holds 16, with each word's zero-point byte and scale.
template <int W, int RP>
struct F32Regs {
  uint32_t k_c[W], k_z[W], k_s[W], v_c[W], v_z[W], v_s[W];
  uint32_t k_id, v_id, k_sg, v_sg, c_s, c_b[RP > 0 ? RP / 2 : 1];
};

template <int D, int RP, bool SI8>
__device__ __forceinline__ void few_f32(const AttendArgs& a, uint32_t place_l, uint32_t place_n) {
  typedef Mfma<float> MF;
  constexpr int NW = kF32Waves, CK = kFewChunk, HK = D / 2, W = D / 32;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
  const int Kc = a.n_centroids, r = a.rank, G = D / a.L.ng;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, l32 = lane % 32,
            hf = lane / 32;
  const FewPlace place = few_place(a, place_l, place_n);
  const int part = place.part, h = place.h, b = place.b;
  const int64_t bh = place.bh, n_bh = place.n_bh;
  const int qa = place.block * kFewQ, rows = min(kFewQ, int(a.n_q) - qa);
  const int64_t nc = a.n_cache + a.n_act;
  const uint32_t F = uint32_t(a.frame_tokens);
  const FewReach reach = few_reach(a.q_start, F, nc, a.n_sink, a.window, a.windowed != 0, uint32_t(qa), uint32_t(qa + rows));
  int before = 0;
  const int seg = few_segment_at(a, reach, part, lane, before);
  const bool act = seg == a.n_epochs;
  FewSegment g{};
  if (!act || a.n_act > 0) g = few_segment_of(a, seg, reach);
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
  const float* gK = reinterpret_cast<const float*>(slab + a.o_mu_k) + hf * HK;
  const float* gV = reinterpret_cast<const float*>(slab + a.o_mu_v) + hf * HK;
  float* vt = reinterpret_cast<float*>(smem_raw) + wave * FewTile<D>::FLOATS;
  const int qi = qa + l32;
  const bool qvalid = l32 < rows;

  // ---- packed fields: the loads hold no branch (see attend_few.hip)
  const CacheLayout& L = a.L;
  const int64_t slot0 = bh * L.slots;
  const uint32_t zpb = L.zpb, ss = SI8 ? L.ng : 2 * L.ng;
  auto field = [&](int64_t off, uint32_t bytes, int64_t end) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)(a.cache + off + slot0 * bytes), 0, int(uint32_t(end) * bytes), 0x00020000);
  };
  const auto r_kc = field(L.k_codes, D / 4, L.slots), r_ki = field(L.k_ids, 1, L.slots), r_kz = field(L.k_zp, zpb, L.slots),
             r_ks = field(L.k_scale, ss, L.slots), r_cc = field(L.k_coef, uint32_t(r), L.slots),
             r_cs = field(L.k_cscale, 2, L.slots), r_vc = field(L.v_codes, D / 4, L.slots),
             r_vi = field(L.v_ids, 1, L.slots), r_vz = field(L.v_zp, zpb, L.slots), r_ksg = field(L.k_sigma, 2, L.slots);
  // Value scales past the segment read as 0, so that its masked keys' Values are finite
  const auto r_vs = field(L.v_scale, ss, SI8 ? L.slots : g.hi), r_vsg = field(L.v_sigma, 2, g.hi);
  int grp[W];  // group of each word of this lane's channels
#pragma unroll
  for (int u = 0; u < W; ++u) grp[u] = (hf * HK + 16 * u) / G;
  typedef F32Regs<W, RP> Regs;
  auto load = [&](Regs& p, int t) __attribute__((always_inline)) {
    const int k0 = key_of(t);
    auto codes = [&](auto rsrc, uint32_t (&to)[W]) __attribute__((always_inline)) {
      if constexpr (W == 4) {
        const auto c = __builtin_amdgcn_raw_buffer_load_b128(rsrc, l32 * (D / 4) + hf * (D / 8), k0 * (D / 4), 0);
#pragma unroll
        for (int u = 0; u < 4; ++u) to[u] = c[u];
      } else {
        const auto c = __builtin_amdgcn_raw_buffer_load_b64(rsrc, l32 * (D / 4) + hf * (D / 8), k0 * (D / 4), 0);
#pragma unroll
        for (int u = 0; u < 2; ++u) to[u] = c[u];
      }
    };
    auto side = [&](auto rz, auto rs, uint32_t (&z)[W], uint32_t (&s)[W]) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < W; ++u) {
        z[u] = uint8_t(__builtin_amdgcn_raw_buffer_load_b8(rz, l32 * int(zpb) + grp[u] / 4, k0 * int(zpb), 0));
        if constexpr (SI8) s[u] = uint8_t(__builtin_amdgcn_raw_buffer_load_b8(rs, l32 * int(ss) + grp[u], k0 * int(ss), 0));
        else s[u] = uint16_t(__builtin_amdgcn_raw_buffer_load_b16(rs, l32 * int(ss) + 2 * grp[u], k0 * int(ss), 0));
      }
    };
    p.k_id = uint8_t(__builtin_amdgcn_raw_buffer_load_b8(r_ki, l32, k0, 0));
    p.v_id = uint8_t(__builtin_amdgcn_raw_buffer_load_b8(r_vi, l32, k0, 0));
    codes(r_kc, p.k_c);
    side(r_kz, r_ks, p.k_z, p.k_s);
    if constexpr (RP > 0) {
      constexpr uint32_t kAbsent = 0xC0000000u;  // past the end of the resource: reads as 0
      p.c_s = uint16_t(__builtin_amdgcn_raw_buffer_load_b16(r_cs, 2 * l32, 2 * k0, 0));
#pragma unroll
      for (int i = 0; i < RP / 2; ++i) {
        const int k = acc_row(i, hf);
        p.c_b[i] = uint8_t(__builtin_amdgcn_raw_buffer_load_b8(r_cc, int(k < r ? uint32_t(l32 * r + k) : kAbsent), k0 * r, 0));
      }
    }
    codes(r_vc, p.v_c);
    side(r_vz, r_vs, p.v_z, p.v_s);
    if constexpr (SI8) {
      p.k_sg = uint16_t(__builtin_amdgcn_raw_buffer_load_b16(r_ksg, 2 * l32, 2 * k0, 0));
      p.v_sg = uint16_t(__builtin_amdgcn_raw_buffer_load_b16(r_vsg, 2 * l32, 2 * k0, 0));
    }
  };

  // ---- everything that a part starts with, in flight at once: the packed fields, the
  // Query (step st of lane half hf is channel hf D/2 + st) and U_r
  Regs P;
  if (!act && t0 < t1) load(P, t0 + wave < t1 ? t0 + wave : t1 - 1);
  float q[HK], ureg[RP > 0 ? RP / 2 : 1];
  float4 qv[HK / 4], uv[HK / 4];
  const float* qrow = reinterpret_cast<const float*>(a.q) + ((int64_t(b) * a.n_q + (qvalid ? qi : qa)) * a.heads + h) * D + hf * HK;
  const float* urow = reinterpret_cast<const float*>(slab + a.o_u_t) + int64_t(l32 < r ? l32 : 0) * D + hf * HK;
#pragma unroll
  for (int st = 0; st < HK / 4; ++st) qv[st] = reinterpret_cast<const float4*>(qrow)[st];
  if (RP > 0 && !act) {
#pragma unroll
    for (int st = 0; st < HK / 4; ++st) uv[st] = reinterpret_cast<const float4*>(urow)[st];
  }
  __builtin_amdgcn_sched_barrier(0);
  // both centroid rows of a chunk's keys are gathered before either is used (d = 64; the
  // registers of d = 128 hold one side at a time), the first ones while q U_r is made
  constexpr bool BOTH = W == 2;
  float muk[W][16], muv[W][16];
  auto gather = [&](const float* row, float (&mu)[W][16]) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < W; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 v = reinterpret_cast<const float4*>(row + 16 * u)[i];
        mu[u][4 * i] = v.x; mu[u][4 * i + 1] = v.y; mu[u][4 * i + 2] = v.z; mu[u][4 * i + 3] = v.w;
      }
  };
  auto gather_keys = [&]() __attribute__((always_inline)) { gather(gK + int64_t(int(P.k_id) < Kc ? int(P.k_id) : Kc - 1) * D, muk); };
  auto gather_first = [&]() __attribute__((always_inline)) {
    gather(gV + int64_t(int(P.v_id) < Kc ? int(P.v_id) : Kc - 1) * D, muv);
    if constexpr (BOTH) gather_keys();
    __builtin_amdgcn_sched_barrier(0);
  };
  if (!act && t0 < t1) gather_first();
#pragma unroll
  for (int st = 0; st < HK / 4; ++st) {
    q[4 * st] = qvalid ? qv[st].x : 0.0f;
    q[4 * st + 1] = qvalid ? qv[st].y : 0.0f;
    q[4 * st + 2] = qvalid ? qv[st].z : 0.0f;
    q[4 * st + 3] = qvalid ? qv[st].w : 0.0f;
  }
  if constexpr (RP > 0) {
#pragma unroll
    for (int i = 0; i < RP / 2; ++i) ureg[i] = 0.0f;
    if (!act) {  // q U_r (rows = ranks of U_r^T)
      f32x16 u;
#pragma unroll
      for (int i = 0; i < 16; ++i) u[i] = 0.0f;
#pragma unroll
      for (int st = 0; st < HK / 4; ++st) {
        u = MF::run(l32 < r ? uv[st].x : 0.0f, q[4 * st], u);
        u = MF::run(l32 < r ? uv[st].y : 0.0f, q[4 * st + 1], u);
        u = MF::run(l32 < r ? uv[st].z : 0.0f, q[4 * st + 2], u);
        u = MF::run(l32 < r ? uv[st].w : 0.0f, q[4 * st + 3], u);
      }
#pragma unroll
      for (int i = 0; i < RP / 2; ++i) ureg[i] = u[i];
    }
  }

  float m_run = -__builtin_inff(), l_run = 0.0f;
  f32x16 oacc[D / 32];
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
    for (int i = 0; i < 16; ++i) oacc[cb][i] = 0.0f;
  int lim = int(nc), wfrom = 0;
  {
    const int64_t l = a.q_start + int64_t(uint32_t(qi) / F + 1) * F, w = a.windowed ? l - a.window : 0;
    lim = int(l < nc ? l : nc);
    wfrom = int(w < 0 ? 0 : (w < nc ? w : nc));
  }
  const float mscale = 1.4426950408889634f / sqrtf((float)D), tau = 8.0f / mscale;  // as in attend.hip

  // softmax of the logits s of one chunk and O^T += V^T P^T, with the Values in the tile
  auto finish = [&](f32x16& s, int k0) __attribute__((always_inline)) {
    if (k0 < g.lo || k0 + CK > (reach.kfull < g.hi ? reach.kfull : g.hi) || (k0 + CK > reach.ns && k0 < reach.wfull)) {
      const int klo = int(g.lo), khi = int(g.hi) < lim ? int(g.hi) : lim;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = k0 + acc_row(i, hf);
        // a select: as a conditional store the compiler branched for each and copied all of s
        const bool hide = (key >= khi) | (key < klo) | ((key >= int(reach.ns)) & (key < wfrom));
        s[i] = hide ? -__builtin_inff() : s[i];
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
    float lp[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], mscale, mc));
      lp[i % 4] += s[i];
    }
    l_run += (lp[0] + lp[1]) + (lp[2] + lp[3]);
    // the tile's stores are this wave's own: LDS keeps their order, this the compiler's
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int cb = 0; cb < D / 32; ++cb)
        oacc[cb] = MF::run(vt[acc_row(i, hf) * FewTile<D>::ROW + cb * 32 + l32], s[i], oacc[cb]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };

  if (!act) {
    auto decode = [&](const float (&mu)[16], uint32_t code, uint32_t zb, uint32_t sb, uint32_t sg, int grp_u, float (&x)[16],
                      bool in) __attribute__((always_inline)) {
      const uint32_t z = (0x6400u + ((zb >> (2 * (grp_u % 4))) & 3)) * 0x00010001u;
      const _Float16 c = SI8 ? (_Float16)(int)sb : (_Float16)0;
      const float s = in ? (float)__builtin_bit_cast(_Float16, uint16_t(SI8 ? sg : sb)) : 0.0f;
      dequant_codes<16, SI8>(code, s, z, mu, x, f16x2{c, c});
    };
    for (int t = t0 + wave; t < t1; t += NW) {
      const int k0 = key_of(t);
      if (t > t0 + wave) gather_first();
      const bool in = k0 + l32 >= g.lo;  // not a key of the neighbouring epoch before the segment's first
#pragma unroll
      for (int u = 0; u < W; ++u) {
        float x[16];
        decode(muv[u], P.v_c[u], P.v_z[u], P.v_s[u], P.v_sg, grp[u], x, in);
        float4* row = reinterpret_cast<float4*>(vt + l32 * FewTile<D>::ROW + hf * HK + 16 * u);
#pragma unroll
        for (int i = 0; i < 4; ++i) row[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
      }
      if constexpr (!BOTH) gather_keys();
      f32x16 s;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
      for (int u = 0; u < W; ++u) {
        float x[16];
        decode(muk[u], P.k_c[u], P.k_z[u], P.k_s[u], P.k_sg, grp[u], x, true);
#pragma unroll
        for (int c = 0; c < 16; ++c) s = MF::run(x[c], q[16 * u + c], s);
      }
      if constexpr (RP > 0) {
        const float cs = (float)__builtin_bit_cast(_Float16, uint16_t(P.c_s));
#pragma unroll
        for (int i = 0; i < RP / 2; ++i) s = MF::run((float)int8_t(P.c_b[i]) * cs, ureg[i], s);
      }
      load(P, t + NW < t1 ? t + NW : t1 - 1);  // past the last chunk that one again
      finish(s, k0);
    }
  } else {
    // exact rows, the last one again past the end
    const int64_t last = a.n_act - 1;
    for (int t = t0 + wave; t < t1; t += NW) {
      const int k0 = key_of(t);
      const int64_t i0 = k0 - a.n_cache + l32;
      const int64_t at = ((int64_t(b) * a.n_act + (i0 < last ? i0 : last)) * a.heads + h) * D + hf * HK;
      const float4* kr = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.k_act) + at);
      const float4* vr = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.v_act) + at);
      float4* row = reinterpret_cast<float4*>(vt + l32 * FewTile<D>::ROW + hf * HK);
      float4 kv[HK / 4];
#pragma unroll
      for (int i = 0; i < HK / 4; ++i) kv[i] = kr[i];
#pragma unroll
      for (int i = 0; i < HK / 4; ++i) row[i] = vr[i];
      f32x16 s;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
      for (int i = 0; i < HK / 4; ++i) {
        s = MF::run(kv[i].x, q[4 * i], s);
        s = MF::run(kv[i].y, q[4 * i + 1], s);
        s = MF::run(kv[i].z, q[4 * i + 2], s);
        s = MF::run(kv[i].w, q[4 * i + 3], s);
      }
      finish(s, k0);
    }
  }

  // ---- merge of the waves through LDS (the tiles are done with)
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
  for (int i = threadIdx.x; i < rows * (D / 4); i += 64 * NW) {
    const int row = i / (D / 4), c = i % (D / 4) * 4;
    float M = -__builtin_inff();
#pragma unroll
    for (int w = 0; w < NW; ++w) M = fmaxf(M, ml[2 * (w * rows + row)]);
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    float l = 0.0f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float lw = ml[2 * (w * rows + row) + 1];
      const float e = lw > 0.0f ? __builtin_amdgcn_exp2f((ml[2 * (w * rows + row)] - M) * mscale) : 0.0f;
      const f32x4 ow = *reinterpret_cast<const f32x4*>(mo + (w * rows + row) * OS + c);
      l += e * lw;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] += e * ow[j];
    }
    if (a.part_o) {
      *reinterpret_cast<f32x4*>(a.part_o + ((int64_t(part) * n_bh + bh) * a.n_q + qa + row) * D + c) = o;
      if (c == 0) {
        plane_ml[2 * row] = M;
        plane_ml[2 * row + 1] = l;
      }
    } else {
      f32x4 r;
#pragma unroll
      for (int j = 0; j < 4; ++j) r[j] = l > 0.0f ? o[j] / l : 0.0f;
      *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(a.out) + ((int64_t(b) * a.n_q + qa + row) * a.heads + h) * D + c) = r;
      if (a.lse && c == 0)
        a.lse[bh * a.n_q + qa + row] = l > 0.0f ? M / sqrtf((float)D) + logf(l) : -__builtin_inff();
    }
  }
}

template <int D, int RP, bool SI8>
__global__ __launch_bounds__(64 * kF32Waves) void attend_few_f32_kernel(const AttendArgs a) {
  few_f32<D, RP, SI8>(a, blockIdx.x, gridDim.x);
}

// Both launches of a pair: a kernel of its own, since arguments at a computed address cost a
// single launch 1.4 us.
template <int D, int RP, bool SI8>
__global__ __launch_bounds__(64 * kF32Waves) void attend_few_f32_pair(const FewPair two) {
  const bool second = blockIdx.x >= two.n0;
  few_f32<D, RP, SI8>(two.a[second ? 1 : 0], blockIdx.x - (second ? two.n0 : 0), second ? gridDim.x - two.n0 : two.n0);
}

template <int D, int RP, bool SI8>
hipError_t launch_k(const AttendArgs& a, int batch, const AttendArgs* other, int other_batch, hipStream_t s) {
  // dynamic LDS: the tiles, and the merge in their place (32 rows of it are as large)
  constexpr size_t lds = size_t(kF32Waves) * (FewTile<D>::FLOATS + 2 * kFewQ) * 4;
  static_assert(lds <= kLdsLimit && FewTile<D>::FLOATS >= kFewQ * (D + 4), "the merge fits where the tiles were");
  static std::atomic<uint64_t> raised{0};  // devices whose dynamic LDS limit is raised for this instance
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
  if (!bit || !(raised.load(std::memory_order_acquire) & bit)) {
    for (const void* f : {(const void*)attend_few_f32_kernel<D, RP, SI8>, (const void*)attend_few_f32_pair<D, RP, SI8>}) {
      e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, int(kLdsLimit));
      if (e != hipSuccess) return e;
    }
    raised.fetch_or(bit, std::memory_order_release);
  }
  auto wgs = [](const AttendArgs& x, int n) { return uint32_t(x.n_split) * uint32_t(x.heads) * uint32_t(x.q_blocks * n); };
  const uint32_t n0 = wgs(a, batch);
  if (other)
    hipLaunchKernelGGL((attend_few_f32_pair<D, RP, SI8>), dim3(n0 + wgs(*other, other_batch)), dim3(64 * kF32Waves), lds, s,
                       FewPair{{a, *other}, n0});
  else
    hipLaunchKernelGGL((attend_few_f32_kernel<D, RP, SI8>), dim3(n0), dim3(64 * kF32Waves), lds, s, a);
  return hipGetLastError();
}

}  // namespace

template <int D, int RP>
hipError_t launch_attend_few_f32_rp(const AttendArgs& a, int batch, const AttendArgs* other, int other_batch, hipStream_t s) {
  return a.L.i8 ? launch_k<D, RP, true>(a, batch, other, other_batch, s) : launch_k<D, RP, false>(a, batch, other, other_batch, s);
}

template hipError_t launch_attend_few_f32_rp<QWM_ATTEND_D, QWM_ATTEND_RP>(const AttendArgs&, int, const AttendArgs*, int, hipStream_t);

}  // namespace qwm
