// Evictions and insertion of a commit, for one unit and a group of threads (tree_commit.cu).
#pragma once

#include "multi.cuh"
#include "tree.cuh"

namespace roco {

constexpr int kCiMaxA = ROCO_TREE_MAX_PATH;
// Named barrier of the group.  Not kMqBarPolicy: lowest_r_block_victims synchronises its 128 threads on that one while the
// rest of a larger group already waits on this.
constexpr int kCiBar = 3;
static_assert(kCiBar != kMqBarPolicy, "the two groups differ in size");
constexpr int kCiShort = 256;  // candidates that are ranked one against the other

struct CiScratch {
  SelectScratch sel;
  int ctl[64];  // 20: counter; 24 .. 39: the chosen slots (the places that lowest_r_block_victims uses)
  int cand[kCiShort];
  unsigned long long cand_key[kCiShort];  // key, then position
  alignas(16) uint32_t best[512];
  uint32_t threshold;
  int list_pos[kCiMaxA];  // positions of the chosen slots
};

// Gathers the slots whose key is at or beyond sc.threshold; returns how many, -1 if they are too many to rank (many equal
// keys).  Every thread of the group of NT calls it.
template <int NT, bool kLow>
__device__ __forceinline__ int gather_candidates(const uint32_t *key, const int *pos, int live, CiScratch &sc) {
  const int lane = threadIdx.x & 31;
  int *cnt = sc.ctl + 20;
  const uint32_t T = sc.threshold;
  for (int j0 = threadIdx.x - lane; j0 < live; j0 += NT) {  // (the warp stays together)
    const int j = j0 + lane;
    const uint32_t k = j < live ? key[j] : 0u;
    const bool take = j < live && (kLow ? k <= T && k < 0x7f800000u : k >= T);
    const uint32_t who = __ballot_sync(0xffffffffu, take);
    if (who) {
      int at = 0;
      if (lane == 0) at = atomicAdd(cnt, __popc(who));
      at = __shfl_sync(0xffffffffu, at, 0) + __popc(who & ((1u << lane) - 1u));
      if (take && at < kCiShort) sc.cand[at] = j;
    }
  }
  named_bar_sync(kCiBar, NT);
  const int n = *cnt;
  if (n > kCiShort) return -1;
  for (int c = threadIdx.x; c < n; c += NT) {  // (the positions, in global memory, all at once)
    const int j = sc.cand[c];
    sc.cand_key[c] = (unsigned long long)key[j] << 32 | (uint32_t)pos[j];
  }
  named_bar_sync(kCiBar, NT);
  return n;
}

// How many of the n gathered come before (kLow) or behind this one in (key, position) order.
template <bool kLow>
__device__ __forceinline__ int rank_candidate(const CiScratch &sc, int n, unsigned long long mine) {
  int rank = 0;
#pragma unroll 8
  for (int i = 0; i < n; ++i) rank += kLow ? sc.cand_key[i] < mine : sc.cand_key[i] > mine;
  return rank;
}

// The kn (<= 16) slots first in (key, position) order over keys that are bit patterns of non-negative floats below
// infinity, to sc.ctl[24 ..] and their positions to sc.list_pos.  The threads form 16 groups: at least kn keys lie at or
// below the kn-th smallest of the groups' minima, and few more, so those are gathered and ranked one against the other.
// Returns how many were gathered: fewer than kn if there are no more, -1 if too many to rank.
template <int NT>
__device__ __forceinline__ int lowest_slots(const uint32_t *key, const int *pos, int live, int kn, CiScratch &sc) {
  const int tid = threadIdx.x;
  uint32_t low = 0xffffffffu;
#pragma unroll 4
  for (int j = tid; j < live; j += NT) low = min(low, key[j]);
#pragma unroll
  for (int o = NT / 32; o > 0; o >>= 1) low = min(low, __shfl_xor_sync(0xffffffffu, low, o));  // NT / 16 neighbours
  if (tid % (NT / 16) == 0) sc.best[tid / (NT / 16)] = low;
  if (tid == 0) sc.ctl[20] = 0;
  named_bar_sync(kCiBar, NT);
  if (tid < 16) {
    int rank = 0;
    const uint32_t mine = sc.best[tid];
#pragma unroll
    for (int i = 0; i < 16; ++i) rank += (sc.best[i] < mine) | ((sc.best[i] == mine) & (i < tid));
    if (rank == kn - 1) sc.threshold = mine;
  }
  named_bar_sync(kCiBar, NT);
  const int n = gather_candidates<NT, true>(key, pos, live, sc);
  for (int c = tid; c < n; c += NT) {
    const int rank = rank_candidate<true>(sc, n, sc.cand_key[c]);
    if (rank < kn) { sc.ctl[24 + rank] = sc.cand[c]; sc.list_pos[rank] = (int)(uint32_t)sc.cand_key[c]; }
  }
  named_bar_sync(kCiBar, NT);
  return n;
}

// Takes the x slots last in (variance, position) order out of the scope (their means become infinite); false if it could
// not.  The same idea the other way round, with 128 groups for x <= 64 and a group per thread up to x = NT / 2.
template <int NT>
__device__ __forceinline__ bool exclude_highest(const uint32_t *vkey, float *mkey, const int *pos, int live, int x, CiScratch &sc) {
  const int tid = threadIdx.x;
  uint32_t high = 0u;
#pragma unroll 4
  for (int j = tid; j < live; j += NT) high = max(high, vkey[j]);
  const int groups = x <= 64 ? 128 : NT;
  if (groups < NT) {
#pragma unroll
    for (int o = NT / 256; o > 0; o >>= 1) high = max(high, __shfl_xor_sync(0xffffffffu, high, o));  // NT / 128 neighbours
    if (tid % (NT / 128) == 0) sc.best[tid / (NT / 128)] = high;
  } else {
    sc.best[tid] = high;
  }
  if (tid == 0) sc.ctl[20] = 0;
  named_bar_sync(kCiBar, NT);
  if (tid < groups) {  // the x-th largest of them: fewer than x are above it, x or more not below
    const uint32_t mine = sc.best[tid];
    int above = 0, below = 0;
#pragma unroll 8
    for (int i = 0; i < groups; i += 4) {
      const uint4 v = *reinterpret_cast<const uint4 *>(&sc.best[i]);
      above += (v.x > mine) + (v.y > mine) + (v.z > mine) + (v.w > mine);
      below += (v.x < mine) + (v.y < mine) + (v.z < mine) + (v.w < mine);
    }
    if (above < x && groups - below >= x) sc.threshold = mine;
  }
  named_bar_sync(kCiBar, NT);
  const int n = gather_candidates<NT, false>(vkey, pos, live, sc);
  for (int c = tid; c < n; c += NT)
    if (rank_candidate<false>(sc, n, sc.cand_key[c]) < x) mkey[sc.cand[c]] = INFINITY;
  named_bar_sync(kCiBar, NT);
  return n >= 0;
}

// The kn slots of lowest_slots by a radix select on the keys, whatever the ties; unordered, to sc.ctl[24 ..] and sc.list_pos;
// false if there are fewer.
template <int NT>
__device__ __forceinline__ bool lowest_by_radix(const uint32_t *key, const int *pos, int live, int kn, CiScratch &sc) {
  const int tid = threadIdx.x;
  int *list = sc.ctl + 24, *cnt = sc.ctl + 20;
  uint32_t k_and = 0xffffffffu, k_or = 0u, rank, ties;
  for (int j = tid; j < live; j += NT) { k_and &= key[j]; k_or |= key[j]; }
  group_and_or(k_and, k_or, sc.sel, tid, NT, kCiBar);
  const uint32_t R = radix_select<uint32_t>([&](int j) { return key[j]; }, [&](int) { return true; }, live, (uint32_t)(kn - 1),
                                            sc.sel, tid, NT, kCiBar, &rank, &ties, k_and, k_or);
  int P = 0x7fffffff;
  if (ties != rank + 1) {  // only some of the slots tied at the threshold: lowest positions
    uint32_t r2, t2;
    P = (int)radix_select<uint32_t>([&](int j) { return (uint32_t)pos[j]; }, [&](int j) { return key[j] == R; }, live, rank,
                                    sc.sel, tid, NT, kCiBar, &r2, &t2);
  }
  if (tid == 0) *cnt = 0;
  named_bar_sync(kCiBar, NT);
  for (int j = tid; j < live; j += NT) {
    const uint32_t k = key[j];
    if (k < 0x7f800000u && (k < R || (k == R && (P == 0x7fffffff || pos[j] <= P)))) {
      const int at = atomicAdd(cnt, 1);
      if (at < kCiMaxA) { list[at] = j; sc.list_pos[at] = pos[j]; }
    }
  }
  named_bar_sync(kCiBar, NT);
  return *cnt == kn;
}

// What a unit's accepted tokens start with: pbar[i][m], the mean over the heads of accepted query i's probability of accepted
// token m <= i, from the accepted keys in shared memory.  A warp per query head at a time, the next one's row on its way;
// the heads' shares are added up in the order of the heads by the warp that owns the query.
template <typename T, int D>
__device__ __forceinline__ void commit_new_probabilities(const CommitParams &p, int u, int a, const int *path, const T *keys,
                                                         int warp, int warps, int lane, float (*pbar)[kCiMaxA]) {
  constexpr int kN = D / 32;
  const float zscale = p.scale * kLog2e, share = 1.f / (float)p.group;
  const T *Qu = reinterpret_cast<const T *>(p.Q) + (size_t)u * p.T * p.group * D + lane;
  const float *lse = p.lse + (size_t)u * p.T * p.group;
  for (int i = a - 1 - warp; i >= 0; i -= warps) {  // the longest first
    const size_t row0 = (size_t)path[i] * p.group;
    float next[kN], nl = lse[row0];
#pragma unroll
    for (int c = 0; c < kN; ++c) next[c] = Elem<T>::load(Qu + row0 * D + c * 32);
    float acc = 0.f;  // lane m: token m
    for (int g = 0; g < p.group; ++g) {
      float q[kN];
      const float l = -nl * kLog2e;
#pragma unroll
      for (int c = 0; c < kN; ++c) q[c] = next[c];
      if (g + 1 < p.group) {
        nl = lse[row0 + g + 1];
#pragma unroll
        for (int c = 0; c < kN; ++c) next[c] = Elem<T>::load(Qu + (row0 + g + 1) * D + c * 32);
      }
      float mine = 0.f;
#pragma unroll 4
      for (int m = 0; m <= i; ++m) {
        float x = 0.f;
#pragma unroll
        for (int c = 0; c < kN; ++c) x = fmaf(q[c], Elem<T>::load(keys + m * D + c * 32 + lane), x);
        x = warp_sum(x);
        if (lane == m) mine = x;
      }
      if (lane <= i) acc += exp2f(fmaf(mine, zscale, l));
    }
    if (lane <= i) pbar[i][lane] = acc * share;
  }
}

// Keys of a token: mean s / n and variance (q n - s^2) / n^2, formed in 64 bits and rounded to fp32 once, at the end.  Equal means
// are equal keys whatever the counts: with 1 / n to 2^-53 (two of Newton's steps) the quotient is off by less than 2^-51, and one
// of a 24-bit by a 24-bit number lies at least 2^-49 from the middle between two floats, so it comes out as the correctly rounded
// quotient, as in the decode step.  (A product with an fp32 reciprocal does not: s = c n at different n came out different.)
// The decode step's divisions instead cost more, having a branch each: 8192 units x 1024 430 us, 24 units x 4093 x 4 heads 21.1;
// with these 421 and 18.9.
__device__ __forceinline__ void commit_key(float s, float q, int n, uint32_t &vkey, float &mkey) {
  const double nd = (double)n, sd = (double)s;
  double r = (double)__fdividef(1.f, (float)n);
  r = fma(r, fma(-nd, r, 1.0), r);
  r = fma(r, fma(-nd, r, 1.0), r);
  const double num = fmax(fma((double)q, nd, -(sd * sd)), 0.0);  // (exact products; NaN -> 0)
  vkey = __float_as_uint((float)(num * (r * r)));
  mkey = (float)(sd * r);
}

// Variance and mean keys of a unit's slots (keys: 8 bytes per slot of shared memory) from its statistics as they stand.
template <int NT>
__device__ __forceinline__ void commit_keys(const CommitParams &p, int u, int live, char *keys, uint32_t &k_and, uint32_t &k_or) {
  const size_t st = (size_t)u * p.B;
  uint32_t *vkey = reinterpret_cast<uint32_t *>(keys);
  float *mkey = reinterpret_cast<float *>(vkey + p.B);
#pragma unroll 4
  for (int j = threadIdx.x; j < live; j += NT) {
    const float s = p.s[st + j], q = p.q[st + j];
    const int n = p.n[st + j];
    uint32_t v;
    commit_key(s, q, n, v, mkey[j]);
    vkey[j] = v;
    k_and &= v;
    k_or |= v;
  }
}

// The slots that the a > 0 accepted tokens take, ascending, to tgt[0 .. a); the first `need` of them are evicted, their
// positions to tgt_pos.  Called by the NT threads 0 .. NT - 1 of a CTA, which synchronise on kCiBar, with the keys in
// place.  Each pass is over shared memory.
template <int NT>
__device__ __forceinline__ void commit_slots(const CommitParams &p, int u, int a, int live, int need, char *keys, uint32_t k_and,
                                             uint32_t k_or, CiScratch &sc, int *tgt, int *tgt_pos) {
  const int tid = threadIdx.x, B = p.B;
  const size_t st = (size_t)u * B;
  uint32_t *vkey = reinterpret_cast<uint32_t *>(keys);
  float *mkey = reinterpret_cast<float *>(vkey + B);
  uint32_t *mbits = reinterpret_cast<uint32_t *>(mkey);
  const int *opos = p.pos + st;
  int *list = sc.ctl + 24;
  if (need > 0) {
    named_bar_sync(kCiBar, NT);  // the keys are complete
    const int m = scope_size(live, p.r, p.scope_mode);
    bool ok = true;
    if (need > 1 && p.scope_mode == ROCO_SCOPE_LOWEST_R && m < live) {
      group_and_or(k_and, k_or, sc.sel, tid, NT, kCiBar);
      if (tid < kMqPolicyThreads)
        lowest_r_block_victims(vkey, mkey, &sc.sel, sc.ctl, opos, p.status, p.r, live, need, m, k_and, k_or, tid);
      if (tid < need) sc.list_pos[tid] = opos[list[tid]];
    } else {
      // Frozen statistics: the m first in (variance, position) order stay the scope, and the `need` of them first in
      // (mean, position) order leave.  The radix selects take a few hundred cycles per digit and barrier; they are left for
      // a scope that leaves out many tokens and for many equal keys.
      if (m < live && !(live - m <= NT / 2 && exclude_highest<NT>(vkey, mkey, opos, live, live - m, sc))) {
        uint32_t rank, ties;
        group_and_or(k_and, k_or, sc.sel, tid, NT, kCiBar);
        const uint32_t Tv = radix_select<uint32_t>([&](int j) { return vkey[j]; }, [&](int) { return true; }, live,
                                                   (uint32_t)(m - 1), sc.sel, tid, NT, kCiBar, &rank, &ties, k_and, k_or);
        int Pv = 0x7fffffff;
        if (ties != rank + 1) {
          uint32_t r2, t2;
          Pv = (int)radix_select<uint32_t>([&](int j) { return (uint32_t)opos[j]; }, [&](int j) { return vkey[j] == Tv; },
                                           live, rank, sc.sel, tid, NT, kCiBar, &r2, &t2);
        }
        for (int j = tid; j < live; j += NT) {
          const uint32_t v = vkey[j];
          if (!(v < Tv || (v == Tv && (Pv == 0x7fffffff || opos[j] <= Pv)))) mkey[j] = INFINITY;
        }
        named_bar_sync(kCiBar, NT);
      }
      const int n = lowest_slots<NT>(mbits, opos, live, need, sc);
      ok = n >= need || (n < 0 && lowest_by_radix<NT>(mbits, opos, live, need, sc));
    }
    if (!ok && tid == 0) {  // only after corrupt statistics: distinct slots all the same
      atomicOr(p.status, ROCO_DEV_BAD_VICTIM);
      for (int e = 0; e < need; ++e) { list[e] = e; sc.list_pos[e] = opos[e]; }
    }
    named_bar_sync(kCiBar, NT);
    if (tid < need) {  // freed slots in increasing order
      int at = 0;
      for (int x = 0; x < need; ++x) at += list[x] < list[tid] || (list[x] == list[tid] && x < tid);
      tgt[at] = list[tid];
      tgt_pos[at] = sc.list_pos[tid];
    }
  }
  if (tid >= need && tid < a) tgt[tid] = live + tid - need;
}

}  // namespace roco
