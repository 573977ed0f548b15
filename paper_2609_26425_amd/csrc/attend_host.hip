// Host side of the attention launches: key-split count, LDS sizes, dispatch
// to the kernel instances (one translation unit per element type, head_dim
// and PSAC rank padding) and the log-sum-exp merge of partial results.
#include "attend_shape.h"
#include "few_shape.h"
#include "grid_rows.h"

namespace qwm {
namespace {

// Merges the n_split partial results of every Query: with M the largest running
// max and w_s = 2^((m_s - M) log2(e) / sqrt(d)), O = sum w_s O_s / sum w_s l_s
// and lse = M / sqrt(d) + log(sum w_s l_s), the sums taken in split order. One
// wave per Query, D / 64 contiguous channels per lane. The planes are read four
// splits per trip so that their loads are in flight together (a split count
// known only at run time otherwise leaves one split's loads in flight at a time).
template <typename T, int D>
__global__ __launch_bounds__(256) void attend_combine(const AttendArgs a) {
  const int64_t qi = int64_t(blockIdx.x) * 4 + threadIdx.x / 64;
  const int lane = threadIdx.x % 64;
  const int h = blockIdx.y, b = blockIdx.z;
  if (qi >= a.n_q) return;
  const int64_t bh = int64_t(b) * a.heads + h;
  const int64_t plane = int64_t(a.heads) * gridDim.z * a.n_q;  // rows per split
  const float mscale = 1.4426950408889634f / sqrtf((float)D);
  constexpr int PL = D / 64;
  typedef float vecf __attribute__((ext_vector_type(PL)));
  const float2* ml = reinterpret_cast<const float2*>(a.part_ml);
  float M = -__builtin_inff();
  for (int sp = 0; sp < a.n_split; ++sp) M = fmaxf(M, ml[sp * plane + bh * a.n_q + qi].x);
  vecf o = {};
  float L = 0.0f;
  auto add = [&](const float2 p, const vecf v) __attribute__((always_inline)) {
    if (!(p.y > 0.0f)) return;  // this split saw no visible key of this Query
    const float w = __builtin_amdgcn_exp2f((p.x - M) * mscale);
    L += w * p.y;
#pragma unroll
    for (int j = 0; j < PL; ++j) o[j] += w * v[j];
  };
  auto row_of = [&](int sp) { return sp * plane + bh * a.n_q + qi; };
  auto vals = [&](int sp) { return *reinterpret_cast<const vecf*>(a.part_o + row_of(sp) * D + lane * PL); };
  int sp = 0;
  for (; sp + 4 <= a.n_split; sp += 4) {
    float2 p[4];
    vecf v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      p[u] = ml[row_of(sp + u)];
      v[u] = vals(sp + u);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) add(p[u], v[u]);
  }
  for (; sp < a.n_split; ++sp) add(ml[row_of(sp)], vals(sp));
  const float inv = L > 0.0f ? 1.0f / L : 0.0f;
  T* orow = reinterpret_cast<T*>(a.out) + ((int64_t(b) * a.n_q + qi) * a.heads + h) * D + lane * PL;
#pragma unroll
  for (int j = 0; j < PL; ++j) orow[j] = T(o[j] * inv);
  if (a.lse && lane == 0) a.lse[bh * a.n_q + qi] = L > 0.0f ? M / sqrtf((float)D) + logf(L) : -__builtin_inff();
}

// Log-sum-exp merge of partial planes for the windowed and shared-history forms: the
// planes of the shared prefix, whose rows are the rollouts' rows one after the other,
// and those of the own keys (the only ones of a windowed launch). Rows are taken in
// the order of the output. Two forms, by what bounds them:
//   - many planes of few rows: a wave per row, a lane per plane for the running maxima
//     and sums, so that the merge waits for memory twice however many planes there are
//     (25 planes of 480 rows: 4.1 us, with a loop over the planes 8.7);
//   - up to four planes of many rows: 16 lanes per row, so that a wave has four rows'
//     loads in flight (2 planes of 124,800 rows at d = 128: 25 us, the rate of a copy).
struct JoinRow {
  int64_t at1, at2;  // the row in a plane of the prefix, of the own keys
};
// (32-bit quotients: a 64-bit one is some 150 instructions)
__device__ inline JoinRow join_row(const JoinArgs& a, uint32_t row) {
  const uint32_t bi = row / uint32_t(a.heads), h = row % uint32_t(a.heads), b = bi / uint32_t(a.n_q), i = bi % uint32_t(a.n_q);
  return {int64_t(h) * (a.batch * a.n_q) + bi, (int64_t(b) * a.heads + h) * a.n_q + i};
}

template <typename T, int D>
__global__ __launch_bounds__(256) void join_planes(const JoinArgs a) {
  const int64_t rows = int64_t(a.batch) * a.n_q * a.heads;
  const uint32_t row = (blockIdx.y * gridDim.x + blockIdx.x) * 4 + threadIdx.x / 64;
  const int lane = threadIdx.x % 64, n = a.n_prefix + a.n_own;
  if (row >= rows) return;
  const JoinRow at = join_row(a, row);
  const float mscale = 1.4426950408889634f / sqrtf((float)D);
  constexpr int PL = D / 64;
  typedef float vecf __attribute__((ext_vector_type(PL)));
  auto ml_of = [&](int sp) {
    return sp < a.n_prefix ? reinterpret_cast<const float2*>(a.prefix_ml)[sp * rows + at.at1]
                           : reinterpret_cast<const float2*>(a.own_ml)[(sp - a.n_prefix) * rows + at.at2];
  };
  auto o_of = [&](int sp) {
    const float* o = sp < a.n_prefix ? a.prefix_o + (sp * rows + at.at1) * D : a.own_o + ((sp - a.n_prefix) * rows + at.at2) * D;
    return *reinterpret_cast<const vecf*>(o + lane * PL);
  };
  const float none = -__builtin_inff();
  // eight planes' O at a time, the first of them on their way with the maxima
  vecf v[8];
  auto load = [&](int sp) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = o_of(sp + u < n ? sp + u : n - 1);
  };
  float2 p = lane < n ? ml_of(lane) : make_float2(none, 0.0f);
  if (n > 0) load(0);
  float M = p.x;
  for (int s0 = 64; s0 < n; s0 += 64) M = fmaxf(M, s0 + lane < n ? ml_of(s0 + lane).x : none);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) M = fmaxf(M, __shfl_xor(M, o));
  vecf o = {};
  float L = 0.0f;
  for (int s0 = 0; s0 < n; s0 += 64) {
    if (s0 > 0) p = s0 + lane < n ? ml_of(s0 + lane) : make_float2(none, 0.0f);
    const float w = p.y > 0.0f ? __builtin_amdgcn_exp2f((p.x - M) * mscale) : 0.0f;  // 0: no visible key in that part
    L += w * p.y;
    const int m = n - s0 < 64 ? n - s0 : 64;
    for (int u0 = 0; u0 < m; u0 += 8) {
      if (s0 + u0 > 0) load(s0 + u0);
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        // (a part without a visible key leaves its O row unwritten)
        const float wu = u0 + u < m ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), u0 + u)) : 0.0f;
        if (wu > 0.0f) {
#pragma unroll
          for (int j = 0; j < PL; ++j) o[j] += wu * v[u][j];
        }
      }
    }
  }
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) L += __shfl_xor(L, s);
  const float inv = L > 0.0f ? 1.0f / L : 0.0f;
  T* orow = reinterpret_cast<T*>(a.out) + int64_t(row) * D + lane * PL;
#pragma unroll
  for (int j = 0; j < PL; ++j) orow[j] = T(o[j] * inv);
  if (a.lse && lane == 0) a.lse[at.at2] = L > 0.0f ? M / sqrtf((float)D) + logf(L) : none;
}

constexpr int kWidePlanes = 4;

template <typename T, int D>
__global__ __launch_bounds__(256) void join_rows(const JoinArgs a) {
  const int64_t rows = int64_t(a.batch) * a.n_q * a.heads;
  const uint32_t row = (blockIdx.y * gridDim.x + blockIdx.x) * 16 + threadIdx.x / 16;
  const int l16 = threadIdx.x % 16, n = a.n_prefix + a.n_own;
  if (row >= rows) return;
  const JoinRow at = join_row(a, row);
  const float mscale = 1.4426950408889634f / sqrtf((float)D);
  constexpr int PL = D / 16;
  typedef float vecf __attribute__((ext_vector_type(PL)));
  float2 p[kWidePlanes];
  vecf v[kWidePlanes];
#pragma unroll
  for (int sp = 0; sp < kWidePlanes; ++sp) {
    p[sp] = make_float2(-__builtin_inff(), 0.0f);
    if (sp < n) {
      const bool pre = sp < a.n_prefix;
      const int64_t r = pre ? sp * rows + at.at1 : (sp - a.n_prefix) * rows + at.at2;
      p[sp] = reinterpret_cast<const float2*>(pre ? a.prefix_ml : a.own_ml)[r];
      v[sp] = *reinterpret_cast<const vecf*>((pre ? a.prefix_o : a.own_o) + r * D + l16 * PL);
    }
  }
  float M = -__builtin_inff(), L = 0.0f;
#pragma unroll
  for (int sp = 0; sp < kWidePlanes; ++sp) M = fmaxf(M, p[sp].x);
  vecf o = {};
#pragma unroll
  for (int sp = 0; sp < kWidePlanes; ++sp) {
    if (p[sp].y > 0.0f) {
      const float w = __builtin_amdgcn_exp2f((p[sp].x - M) * mscale);
      L += w * p[sp].y;
#pragma unroll
      for (int j = 0; j < PL; ++j) o[j] += w * v[sp][j];
    }
  }
  const float inv = L > 0.0f ? 1.0f / L : 0.0f;
  typedef T vect __attribute__((ext_vector_type(PL)));
  vect r;
#pragma unroll
  for (int j = 0; j < PL; ++j) r[j] = T(o[j] * inv);
  *reinterpret_cast<vect*>(reinterpret_cast<T*>(a.out) + int64_t(row) * D + l16 * PL) = r;
  if (a.lse && l16 == 0) a.lse[at.at2] = L > 0.0f ? M / sqrtf((float)D) + logf(L) : -__builtin_inff();
}

template <typename T, int D>
hipError_t launch_join_d(const JoinArgs& a, hipStream_t s) {
  const int64_t rows = int64_t(a.batch) * a.n_q * a.heads;
  // 16 lanes a row from four rows for every SIMD on
  const bool wide = a.n_prefix + a.n_own <= kWidePlanes && rows >= 4096;
  const int64_t wgs = (rows + (wide ? 15 : 3)) / (wide ? 16 : 4);
  if (rows > kMaxJoinRows) return hipErrorInvalidValue;
  const dim3 grid(qwm_grid_x(wgs), qwm_grid_y(wgs));
  if (wide) hipLaunchKernelGGL((join_rows<T, D>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((join_planes<T, D>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

// The planes of one windowed launch.
template <typename T, int D>
hipError_t launch_join_own(const AttendArgs& a, int batch, hipStream_t s) {
  JoinArgs j{};
  j.own_o = a.part_o; j.own_ml = a.part_ml; j.n_own = a.n_split;
  j.n_q = a.n_q; j.heads = a.heads; j.batch = batch; j.out = a.out; j.lse = a.lse;
  return launch_join_d<T, D>(j, s);
}

template <typename T, int D>
hipError_t launch_d(const AttendArgs& a, int batch, bool logits, hipStream_t s) {
  hipError_t e;
  if (a.rank == 0) e = launch_attend_rp<T, D, 0>(a, batch, logits, s);
  else if (a.rank <= 16) e = launch_attend_rp<T, D, 16>(a, batch, logits, s);
  else e = launch_attend_rp<T, D, 32>(a, batch, logits, s);
  // planes without an output: the caller joins them with others
  if (e != hipSuccess || logits || a.n_split == 1 || !a.out) return e;
  if (a.windowed) return launch_join_own<T, D>(a, batch, s);
  hipLaunchKernelGGL((attend_combine<T, D>), dim3((unsigned)((a.n_q + 3) / 4), (unsigned)a.heads, (unsigned)batch),
                     dim3(256), 0, s, a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_few_f32_d(const AttendArgs& a, int batch, const AttendArgs* other, int other_batch, hipStream_t s) {
  hipError_t e;
  if (a.rank == 0) e = launch_attend_few_f32_rp<D, 0>(a, batch, other, other_batch, s);
  else if (a.rank <= 16) e = launch_attend_few_f32_rp<D, 16>(a, batch, other, other_batch, s);
  else e = launch_attend_few_f32_rp<D, 32>(a, batch, other, other_batch, s);
  if (e != hipSuccess || a.n_split == 1 || !a.out) return e;
  return launch_join_own<float, D>(a, batch, s);
}

template <int D>
hipError_t launch_few_d(const AttendArgs& a, int batch, hipStream_t s) {
  hipError_t e;
  if (a.rank == 0) e = launch_attend_few_rp<D, 0>(a, batch, s);
  else if (a.rank <= 16) e = launch_attend_few_rp<D, 16>(a, batch, s);
  else e = launch_attend_few_rp<D, 32>(a, batch, s);
  if (e != hipSuccess || a.n_split == 1 || !a.out) return e;
  return launch_join_own<bf16, D>(a, batch, s);
}

// Parts of a launch that gives each of them up to cpp chunks: the most that any Query
// block needs. *chunks: the most chunks of any block.
int few_parts(const AttendArgs& a, int64_t cpp, int64_t* chunks) {
  int64_t most = 0, total = 0;
  for (int64_t qa = 0; qa < a.n_q; qa += a.block_rows) {
    const int64_t qb = qa + a.block_rows < a.n_q ? qa + a.block_rows : a.n_q;
    const FewReach r = few_reach(a.q_start, uint32_t(a.frame_tokens), a.n_cache + a.n_act, a.n_sink, a.window,
                                 a.windowed != 0, uint32_t(qa), uint32_t(qb));
    int64_t parts = 0, sum = 0;
    for (int i = 0; i <= a.n_epochs; ++i) {
      if (i == a.n_epochs && a.n_act == 0) break;
      const int64_t c = few_segment_of(a, i, r).chunks;
      parts += (c + cpp - 1) / cpp;
      sum += c;
    }
    most = parts > most ? parts : most;
    total = sum > total ? sum : total;
  }
  if (chunks) *chunks = total;
  return int(most);
}

// Parts a launch asks for: one workgroup per CU, and at least a chunk for most waves
// (launches of one chunk a wave stay one part); fp32: two workgroups, of four waves, per
// CU, in which no wave has a chunk more than it must (attend_few_plan).
int64_t few_want(int64_t n_q, int heads, int batch, int64_t chunks, int cus, int elem) {
  const int64_t wgs = (n_q + kFewQ - 1) / kFewQ * heads * batch, parts = (elem == 4 ? 2 * cus : cus) / wgs,
                most = elem == 4 ? (chunks + 3) / 4 : (chunks <= 12 ? 1 : chunks / 8);
  const int64_t w = parts < most ? parts : most;
  return w > 1 ? w : 1;
}

}  // namespace

bool attend_few_takes(const quantwm_config& c, int64_t n_q, int64_t n_keys) {
  if (c.storage & QWM_STORE_SPARSE) return false;
  // (one grid dimension holds all parts: at most 65 of 768 threads for each head)
  if (int64_t(c.heads) * c.batch > 65536) return false;
  // BF16: one block of rows, with coefficient rows of whole words, over enough keys that
  // decoding them outweighs the merge of the waves' O rows (d = 128, 12 heads, us here /
  // tiled: 1 Query x 300 keys 13 / 15, x 30,000 33 / 55; 16 x 1,000 20 / 18, x 8,000 27 / 28, x
  // 30,000 37 / 56; 32 x 4,000 28 / 24, x 30,000 44 / 56; two blocks are never faster).
  if (c.dtype == QWM_BF16) return c.rank % 4 == 0 && n_q <= kFewQ && n_keys >= 384 * (n_q - 1);
  // fp32: up to nine products of 32 Queries x 32 keys a SIMD; beyond, blocks of 256 rows
  // decode less (us here / tiled, d = 64: 2 heads x 257 Queries x 362 keys 16 / 29; 8 x 257 x
  // 4,000 61 / 66; 8 x 512 x 4,000 83 / 70; d = 128: 23 / 48; 105 / 110; 150 / 114. The worst
  // below the limit, 30 x 128 x 1,500, 48 / 39 and 79 / 63).
  // (a launch without keys still has its blocks, a grid dimension)
  const double units = double((n_q + kFewQ - 1) / kFewQ) * c.heads * c.batch * double(n_keys / kFewChunk + 1);
  return n_q <= 4096 && units <= 9216;
}

int attend_few_planes(int64_t n_q, int heads, int batch, int64_t n_keys, int cus, int elem) {
  // a segment (epoch) may end in a part of its own: room for 16 of them. A launch with more
  // segments in reach than planes takes the tiles (one Query of 40 heads: more than 22)
  return int(few_want(n_q, heads, batch, n_keys / kFewChunk + 2, cus, elem)) + 16;
}

bool attend_few_plan(AttendArgs& a, int batch, int cus, int elem, int most) {
  a.block_rows = int(elem == 2 && a.n_q <= 16 ? a.n_q : (a.n_q < kFewQ ? a.n_q : kFewQ));
  a.q_blocks = int((a.n_q + a.block_rows - 1) / a.block_rows);
  int64_t chunks = 0;
  (void)few_parts(a, 1 << 30, &chunks);
  const int64_t want = few_want(a.n_q, a.heads, batch, chunks, cus, elem);
  int64_t cpp = (chunks + want - 1) / want;
  if (cpp < 1) cpp = 1;
  // fp32: whole rounds of the four waves, since a part takes as long as its first wave (14
  // chunks in parts of 4 instead of 5, whose first wave has a second one to do: 5 us less)
  if (elem == 4) cpp = (cpp + 3) / 4 * 4;
  int parts = few_parts(a, cpp, nullptr);
  while (parts > most && cpp < chunks) {
    cpp *= 2;
    parts = few_parts(a, cpp, nullptr);
  }
  if (parts > most && parts > 1) return false;
  a.chunks_per_part = cpp;
  a.n_split = parts > 1 ? parts : 1;
  return true;
}

// (BF16 launches fill the GPU by themselves, and differ in their waves.)
bool attend_few_pairs(const quantwm_config& a, const quantwm_config& b) {
  auto pad = [](int r) { return (r + 15) / 16; };
  return a.dtype == QWM_F32 && pad(a.rank) == pad(b.rank) && ((a.storage ^ b.storage) & QWM_STORE_SCALE_I8) == 0;
}

hipError_t launch_attend_few(const AttendArgs& a, int d, int elem, int batch, hipStream_t s, const AttendArgs* other,
                             int other_batch) {
  if (elem == 4) {
    if (d == 64) return launch_few_f32_d<64>(a, batch, other, other_batch, s);
    if (d == 128) return launch_few_f32_d<128>(a, batch, other, other_batch, s);
    return hipErrorInvalidValue;
  }
  if (other) return hipErrorInvalidValue;
  if (d == 64) return launch_few_d<64>(a, batch, s);
  if (d == 128) return launch_few_d<128>(a, batch, s);
  return hipErrorInvalidValue;
}

hipError_t launch_join(const JoinArgs& a, int d, bool bf16_out, hipStream_t s) {
  if (d == 64) return bf16_out ? launch_join_d<bf16, 64>(a, s) : launch_join_d<float, 64>(a, s);
  if (d == 128) return bf16_out ? launch_join_d<bf16, 128>(a, s) : launch_join_d<float, 128>(a, s);
  return hipErrorInvalidValue;
}

size_t attend_lds_bytes(int d, int elem, int rank, int n_centroids, bool tables) {
  if (elem == 2) return d == 64 ? attend_lds_bytes_t<bf16, 64>(rank, n_centroids, tables)
                                : attend_lds_bytes_t<bf16, 128>(rank, n_centroids, tables);
  return d == 64 ? attend_lds_bytes_t<float, 64>(rank, n_centroids, tables)
                 : attend_lds_bytes_t<float, 128>(rank, n_centroids, tables);
}
int attend_splits(int64_t n_q, int heads, int batch, int64_t n_cache, int cus, int elem, int most) {
  // Split the key range only when the launch gives fewer than two workgroups
  // per compute unit (one runs per CU). The split count minimises the rounds of
  // workgroups times each one's work: its share of the key tiles plus a fixed
  // cost of about 32 tiles (table staging, Query fragments, pipeline fill,
  // partial write). It goes up to `most`: 16, or what a smaller workspace holds
  // (with fewer parts than wanted no split may be the cheapest). A split has at
  // least 8 tiles; 4 while all the workgroups still run at once, where a split
  // only uses idle CUs (4 heads, 64 Queries, 704 keys at d = 128: 29 us in one
  // part, 20.5 us in two; 16 heads, 300 Queries, 2,000 keys: 53 us with 3 splits,
  // 35 us with 7, each with the faster start of the kernel). An fp32 tile (matrix
  // cores at 1/16 of the BF16 rate, scalar operand reads) takes 8.5 us for 256
  // Queries at d = 64 and 17 us at d = 128, and a workgroup 25 and 38 us besides:
  // the fixed cost is 2 tiles, and a split may be a single one (2 heads, 256
  // Queries, 1,024 keys, with 2, 8 and 16 splits: 92, 40 and 34 us at d = 64, 173,
  // 69 and 55 us at d = 128). Of the counts tried on each of 64 shapes from 2 x 64
  // Queries x 256 keys to 40 x 600 x 1,024 and 8 x 600 x 4,096 at both head
  // dimensions, the one picked here was the fastest every time.
  const int fixed = elem == 4 ? 2 : 32;
  const int64_t wgs = (n_q + BQ - 1) / BQ * heads * batch;
  if (wgs <= 0 || wgs >= 2 * int64_t(cus)) return 1;
  const int64_t tiles = (n_cache + KT - 1) / KT;
  int best = 1;
  int64_t best_cost = -1;
  for (int ns = 1; ns <= most; ++ns) {
    const int least = elem == 4 ? 1 : (wgs * ns <= cus ? 4 : 8);
    if (ns > 1 && tiles / ns < least) break;
    const int64_t rounds = (wgs * ns + cus - 1) / cus;
    const int64_t cost = rounds * ((tiles + ns - 1) / ns + fixed);
    if (best_cost < 0 || cost < best_cost) {
      best = ns;
      best_cost = cost;
    }
  }
  return best;
}

bool attend_tables_fit(int d, int elem, int rank, int n_centroids) {
  return attend_lds_bytes(d, elem, rank, n_centroids, true) <= kLdsLimit;
}

hipError_t launch_attend_f32(const AttendArgs& a, int d, int batch, bool logits, hipStream_t s) {
  if (d == 64) return launch_d<float, 64>(a, batch, logits, s);
  if (d == 128) return launch_d<float, 128>(a, batch, logits, s);
  return hipErrorInvalidValue;
}

hipError_t launch_attend_bf16(const AttendArgs& a, int d, int batch, bool logits, hipStream_t s) {
  if (d == 64) return launch_d<bf16, 64>(a, batch, logits, s);
  if (d == 128) return launch_d<bf16, 128>(a, batch, logits, s);
  return hipErrorInvalidValue;
}

}  // namespace qwm
