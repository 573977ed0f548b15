// Key ranges of the few-row attention kernel, as the host counts them for its grid and
// the kernel walks them: the 32-key chunks of one segment (an epoch's packed keys, or
// the exact chunk) that a block of Queries may see.
#pragma once

#include "qwm_common.h"
#include "xcd_order.h"

namespace qwm {

constexpr int kFewQ = 32;      // most Queries of a workgroup
constexpr int kFewChunk = 32;  // keys per wave and step

struct FewSegment {
  int64_t lo, hi, base, chunks;  // keys [lo, hi) in chunks from key `base`
  int64_t cut, skip;             // after `cut` chunks, `skip` chunks in nobody's reach are left out
};

// Keys of Queries [qa, qb) of a launch: [0, kend), of which [0, ns) and [wlo, kend) are
// in reach; below kfull and from wfull on every one of these Queries sees them.
struct FewReach {
  int64_t kend, kfull, ns, wlo, wfull;
};

inline __host__ __device__ FewReach few_reach(int64_t q_start, uint32_t F, int64_t nc, int64_t n_sink, int64_t window,
                                              bool windowed, uint32_t qa, uint32_t qb) {
  FewReach r;
  // (32-bit quotients: a 64-bit one is some 150 instructions on the device)
  const int64_t first = q_start + int64_t(qa / F + 1) * F, last = q_start + int64_t((qb - 1) / F + 1) * F;
  r.kfull = first < nc ? first : nc;
  r.kend = last < nc ? last : nc;
  r.ns = windowed ? n_sink : 0;
  const int64_t a = windowed ? first - window : 0, b = windowed ? last - window : 0;
  r.wlo = a < 0 ? 0 : (a < nc ? a : nc);
  r.wfull = b < 0 ? 0 : (b < nc ? b : nc);
  return r;
}

inline __host__ __device__ FewSegment few_segment(int64_t lo, int64_t end, bool act, const FewReach& r) {
  FewSegment s;
  s.lo = lo;
  s.hi = end < r.kend ? end : r.kend;
  s.base = act ? lo : lo / kFewChunk * kFewChunk;
  const int64_t all = s.hi > lo ? (s.hi - s.base + kFewChunk - 1) / kFewChunk : 0;
  const int64_t sink = r.ns > lo ? (r.ns - s.base + kFewChunk - 1) / kFewChunk : 0;
  s.cut = sink < all ? sink : all;
  const int64_t from = r.wlo >= s.hi ? all : (r.wlo > s.base ? (r.wlo - s.base) / kFewChunk : 0);
  s.skip = from > s.cut ? from - s.cut : 0;
  s.chunks = all - s.skip;
  return s;
}

// Segment i of a launch (n_epochs: the exact chunk).
inline __host__ __device__ FewSegment few_segment_of(const AttendArgs& a, int i, const FewReach& r) {
  const bool act = i == a.n_epochs;
  const int64_t lo = act ? a.n_cache : a.epoch_start[i];
  const int64_t end = act ? a.n_cache + a.n_act : (i + 1 < a.n_epochs ? a.epoch_start[i + 1] : a.n_cache);
  return few_segment(lo, end, act, r);
}

// Two launches of one kernel instance as one: workgroups [0, n0) run the first.
struct FewPair {
  AttendArgs a[2];
  uint32_t n0;
};

#ifdef __HIPCC__
// What workgroup L of n runs, in a launch of n_split parts of every unit (a Query block of
// a head). Two orders:
//   - few units, whose key range is cut: the parts of a unit on one XCD, so that its tables
//     come from one L2 (40 heads x 1 Query x 30,000 keys: 52.8 us, with the parts dealt
//     round the XCDs 53.9);
//   - units enough for every CU, so that a part is a whole segment: part by part, the
//     first segments of all units before the second. The exact chunk's parts, often a few
//     keys, then fill in behind the packed ones instead of standing between them (16
//     rollouts x 30 heads, 130 packed keys and one exact: 30 -> 22 us).
struct FewPlace {
  int part, h, b, block;
  int64_t bh, n_bh;
};
__device__ inline FewPlace few_place(const AttendArgs& a, uint32_t L, uint32_t n) {
  const uint32_t parts = uint32_t(a.n_split), units = n / parts, heads = uint32_t(a.heads);
  uint32_t part, u;
  if (units >= 256) {
    part = L / units;
    u = L % units;
  } else {
    const uint32_t t = qwm_xcd_task(L, n);
    u = t / parts;
    part = t % parts;
  }
  const uint32_t bb = u / heads, blocks = uint32_t(a.q_blocks);
  FewPlace p;
  p.part = int(part);
  p.h = int(u % heads);
  p.b = int(bb / blocks);
  p.block = int(bb % blocks);
  p.bh = int64_t(p.b) * heads + uint32_t(p.h);
  p.n_bh = units / blocks;
  return p;
}

// The segment of part `part`, and the parts before it: a lane counts for each epoch.
__device__ inline int few_segment_at(const AttendArgs& a, const FewReach& r, int part, int lane, int& before) {
  static_assert(kMaxEpochs == 64, "a lane per epoch");
  const uint32_t cpp = uint32_t(a.chunks_per_part);
  before = 0;
  if (a.n_epochs == 1) {
    const int p0 = int((uint32_t(few_segment_of(a, 0, r).chunks) + cpp - 1) / cpp);
    if (part < p0) return 0;
    before = p0;
    return 1;
  }
  int past = lane < a.n_epochs ? int((uint32_t(few_segment_of(a, lane, r).chunks) + cpp - 1) / cpp) : 0;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(past, o);
    past += lane >= o ? y : 0;
  }
  const uint64_t at = __ballot(past > part);
  const int seg = at ? __builtin_ctzll(at) : a.n_epochs;
  before = seg > 0 ? __builtin_amdgcn_readlane(past, seg - 1) : 0;
  return seg;
}
#endif

}  // namespace qwm
