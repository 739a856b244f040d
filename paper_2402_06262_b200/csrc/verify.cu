// Verification of drafted trees against the target's probabilities.
//
// A cluster of CTAs (one to eight) per sequence.  Everything about a node is two numbers, p(x) and q(x) behind its parent, fetched for
// all nodes at once; the walk over them is a few instructions per child.  A row is only touched where a child was rejected (to sum
// what is left of p) and at the end (to pick the next token): what is left of p after any number of rejections is
// max(p - C q, 0) for one C, because rejecting once more takes (R / M) q from what is still positive and leaves zero at zero.  Without
// draft probabilities what is left is the row less single tokens, so the sums over all of it stand while the walk stays at a node.
// A row is cut into one run per warp of the cluster.  Every warp sends its run's sum to every rank by an asynchronous store that also
// signals (no barrier of the cluster, no reduction in the CTA before it); the sums are the upper level of a prefix sum, which the pick
// descends: run, chunk of 16 bytes, element.
// Bound by a chain of latencies (one tree x 32000 tokens: 7 us in a graph, of which launch 0.7, the nodes' numbers 1.4, the walk 0.8, a
// pass over the row 1.4, the sums' way 0.3, the pick about 1), and with many sequences by the walks with most rejections: 64 sequences x
// 128000 tokens take 31.3 us: the first row ends at 11 to 13, every further pass takes 3 to 4 (with three CTAs per SM a quarter of the
// clusters found no room at first and started when others ended).
// Sums and products are in 64 bits: an index is the answer, and an error of 2^-24 in a sum over 10^5 tokens moves it about once in a
// thousand calls.
#include "decoding.cuh"

namespace roco {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
template <typename T>
constexpr int kResident = sizeof(T) == 4 ? 4 : 3;  // CTAs per SM: as many as their registers allow
constexpr int kDepth = 4, kRingBytes = kDepth * 2 * kThreads * 16;  // chunks of a thread under way
constexpr int kWarpShift = 3, kMaxRanks = 8, kRuns = kMaxRanks * kWarps, kPer = kRuns / 32;
constexpr int kLast = kThreads;  // chunks that are searched at once
static_assert(kWarps == 1 << kWarpShift, "runs are divided by shifts");
// Of a sum less some of its terms at least this much has to be left, or it is formed again without them: no more than ten bits are lost.
constexpr double kLeast = 1.0 / 1024;
// Where drafts are drawn without replacement and less than this is left of the draft, its mass is summed.  One less the rejected is off
// by as much as the row's sum is off one (up to 2^-8 in bf16), which is all that matters once little is left.  Exact distributions of the
// first token over bf16 rows of five and six tokens, two and three siblings, from flat drafts to a token of 0.999: at most 0.003 in
// total variation from the target's (never summed 0.19, from 1/8 on 0.008, from 1/4 on 0.0028, always 0.0024, which is what the rows' sums
// cost in the first test).
constexpr double kLittle = 3.0 / 16;
constexpr int kNodes = ROCO_TREE_MAX_NODES;
static_assert(kNodes == 64, "a node's children are the bits of one 64-bit word");

template <bool kDistinct>
struct Smem {
  float p[kNodes], q[kNodes], u[kNodes];
  unsigned long long children[kNodes + 1];  // of the prefix, then of every node
  double sums[2][kRuns];                    // of every warp of every rank; one set while the other may still be read
  double masses[2][kDistinct ? kRuns : 1];  // the same of the draft's tokens that are not rejected, where that is wanted
  double part[kWarps];
  uint64_t bar[2];                          // completes when a set is here
  unsigned first[2];                        // bits of the nodes that are accepted where no sibling was rejected before
  int token[kNodes];
  int gone[kNodes];                         // tokens rejected behind the node the walk stands on, each once
  float gone_p[kNodes];                     // their probabilities
  int path[ROCO_TREE_MAX_PATH];
  // where the walk stands: node, nodes on the path, children of it that are not tried yet, tokens in gone
  int tip, len, n_gone;
  unsigned long long untried;
  double C, R, M;
  double number;                            // sample_u
  int more;                                 // R is to be summed before the walk goes on
  int weigh;                                // and M, from the draft's row
  int abort_flag;
};

__device__ __forceinline__ double warp_sum64(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// A row of probabilities of the target and, where the draft counts, one of the draft, cut into chunks of 16 bytes from the last such
// boundary at or before the target's first element.
template <typename T>
struct Rows {
  static constexpr int E = Elem<T>::kPerChunk;
  const T *p, *q;   // q: nullptr without draft probabilities
  int lead, V, chunks;
  bool q_like_p;    // the draft's row has the same alignment

  __device__ Rows() {}
  __device__ Rows(const char *target, const char *draft, int v) : p(reinterpret_cast<const T *>(target)), q(reinterpret_cast<const T *>(draft)), V(v) {
    lead = (int)((reinterpret_cast<uintptr_t>(target) & 15u) / sizeof(T));
    chunks = (int)(((long long)V + lead + E - 1) / E);
    q_like_p = ((reinterpret_cast<uintptr_t>(target) ^ reinterpret_cast<uintptr_t>(draft)) & 15u) == 0;
  }

  // The draft's probabilities in chunk i but for the tokens in gone; 0 outside the row.
  __device__ __forceinline__ double mass(int i, const int *gone, int n_gone) const {
    const int first = i * E - lead;
    float f[E];
    if (q_like_p && first >= 0 && first + E <= V) Elem<T>::unpack(__ldg(reinterpret_cast<const uint4 *>(q + first)), f);
    else some(q, first, f);
    double sum = 0.0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      for (int g = 0; g < n_gone; ++g)
        if (gone[g] == first + e) f[e] = 0.f;
      sum += f[e] <= 0.f ? 0.0 : (double)f[e];
    }
    return sum;
  }

  __device__ __forceinline__ void some(const T *row, int first, float (&f)[E]) const {
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = first + e >= 0 && first + e < V ? Elem<T>::load(row + first + e) : 0.f;
  }

  // What is left of p in chunk i; 0 outside the row.  A NaN stays one.
  __device__ __forceinline__ void left(int i, double C, const int *gone, int n_gone, double (&r)[E]) const {
    const int first = i * E - lead;
    const bool whole = first >= 0 && first + E <= V;
    float fp[E], fq[E];
    if (whole) Elem<T>::unpack(__ldg(reinterpret_cast<const uint4 *>(p + first)), fp);
    else some(p, first, fp);
    if (q) {
      if (whole && q_like_p) Elem<T>::unpack(__ldg(reinterpret_cast<const uint4 *>(q + first)), fq);
      else some(q, first, fq);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const double x = q ? fma(-C, (double)fq[e], (double)fp[e]) : (double)fp[e];
      r[e] = x <= 0.0 ? 0.0 : x;
    }
    for (int g = 0; g < n_gone; ++g) {
      const int e = gone[g] - first;
      if (e >= 0 && e < E) {
#pragma unroll
        for (int k = 0; k < E; ++k)
          if (k == e) r[k] = 0.0;
      }
    }
  }
};

// Conversions and comparisons in 64 bits are issued at an eighth to a quarter of the rate of its sums and products (16 and 21 of 62
// per cycle and SM, measured), so where all numbers are positive and normal conversions are done on the bits, and max(x, 0) is half
// of x + |x|.
constexpr uint32_t kLeastNormal = 0x00800000u, kInfinity = 0x7f800000u;
__device__ __forceinline__ double widen(float x) {
  const uint32_t bits = __float_as_uint(x);
  return __hiloint2double((int)((bits >> 3) + ((1023u - 127u) << 20)), (int)(bits << 29));
}

// A lane's part of the sum of what is left of p over whole chunks i, i + 32, ... before `end`.  A row is read at the pace of loads in
// flight, so the thread keeps kDepth of them under way into places of its own in shared memory (`ring`: the address of its first; through
// registers, four at a time, 34.1 us where this took 32.8, and fewer CTAs per SM).  One chunk is worked on at a time: two cost more
// registers than they hide (37 us).
template <typename T, bool kDraft, bool kMass>
__device__ __forceinline__ double sum_whole(const Rows<T> &rows, int i, int end, double C, const uint4 *ring, double &mass) {
  constexpr int E = Rows<T>::E;
  const uint4 *p = reinterpret_cast<const uint4 *>(rows.p - rows.lead) + i, *q = reinterpret_cast<const uint4 *>(rows.q - rows.lead) + i;
  const uint32_t at = smem_u32(ring);
  auto fetch = [&](int slot, int ahead) {
    if (i + ahead < end) {
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at + slot * (2 * kThreads * 16)), "l"(p + ahead) : "memory");
      if (kDraft)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at + slot * (2 * kThreads * 16) + kThreads * 16), "l"(q + ahead) : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  double twice = 0.0;
#pragma unroll
  for (int s = 0; s < kDepth; ++s) fetch(s, 32 * s);
  for (int n = 0; i < end; n = (n + 1) % kDepth) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
    const uint4 a = ring[n * (2 * kThreads)];
    const uint4 b = kDraft ? ring[n * (2 * kThreads) + kThreads] : a;
    fetch(n, 32 * kDepth);
    i += 32;
    p += 32;
    q += 32;
    float fp[E], fq[E];
    Elem<T>::unpack(a, fp);
    if (kDraft) Elem<T>::unpack(b, fq);
    uint32_t least = __float_as_uint(fp[0]), most = least;
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      least = __vimin3_u32(least, __float_as_uint(fp[e]), __float_as_uint(fp[e + 1]));
      most = __vimax3_u32(most, __float_as_uint(fp[e]), __float_as_uint(fp[e + 1]));
      if (kDraft) {
        least = __vimin3_u32(least, __float_as_uint(fq[e]), __float_as_uint(fq[e + 1]));
        most = __vimax3_u32(most, __float_as_uint(fq[e]), __float_as_uint(fq[e + 1]));
      }
    }
    if (least >= kLeastNormal && most < kInfinity) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const double x = kDraft ? fma(-C, widen(fq[e]), widen(fp[e])) : widen(fp[e]);
        twice += kDraft ? x + fabs(x) : x;
        if (kMass) mass += widen(fq[e]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const double x = kDraft ? fma(-C, (double)fq[e], (double)fp[e]) : (double)fp[e];
        twice += x <= 0.0 ? 0.0 : kDraft ? x + x : x;
        if (kMass) mass += fq[e] <= 0.f ? 0.0 : (double)fq[e];
      }
    }
  }
  return (kDraft ? 0.5 : 1.0) * twice;
}

// What is left of p over chunks lo .. hi - 1 of a warp; where it is wanted, the draft's mass there as well.
template <typename T>
__device__ __forceinline__ double sum_run(const Rows<T> &rows, int lo, int hi, double C, const int *gone, int n_gone, const uint4 *ring,
                                          bool weigh, double &mass) {
  constexpr int E = Rows<T>::E;
  const int lane = threadIdx.x & 31, full = (rows.V + rows.lead) / E;
  int i = lo + lane;
  double sum = 0.0, held = 0.0;
  const bool plain = n_gone == 0 && (!rows.q || rows.q_like_p);
  // the row's first and last chunk may reach beyond it
  const bool head = plain && rows.lead && lo == 0 && hi > 0, tail = plain && full < rows.chunks && full >= lo && full < hi && (full > 0 || !head);
  if (head && lane == 0) i += 32;
  if (plain) {
    if (weigh) sum = sum_whole<T, true, true>(rows, i, min(hi, full), C, ring, held);
    else if (rows.q) sum = sum_whole<T, true, false>(rows, i, min(hi, full), C, ring, held);
    else sum = sum_whole<T, false, false>(rows, i, min(hi, full), C, ring, held);
  }
  // what is left for one chunk at a time
  int from = plain ? hi : lo + lane, step = 32;
  if (lane == 0 && (head || tail)) {
    from = head ? 0 : full;
    step = head && tail ? full : hi;
  }
  for (; from < hi; from += step) {
    double r[E];
    rows.left(from, C, gone, n_gone, r);
#pragma unroll
    for (int e = 0; e < E; ++e) sum += r[e];
    if (weigh) held += rows.mass(from, gone, 0);
  }
  if (weigh) mass = warp_sum64(held);
  return warp_sum64(sum);
}

// The draft's mass over chunks lo .. hi - 1 of a warp without the rejected tokens, from `all` of it there.
template <typename T>
__device__ __forceinline__ double mass_left(const Rows<T> &rows, int lo, int hi, double all, const int *gone, int n_gone) {
  constexpr int E = Rows<T>::E;
  double less = 0.0;
  bool here = false;
  for (int g = 0; g < n_gone; ++g) {
    const int at = gone[g] + rows.lead;
    if (at < lo * E || at >= hi * E) continue;
    here = true;
    less += fmaxf(Elem<T>::load(rows.q + gone[g]), 0.f);
  }
  if (!here || all - less > kLeast * all) return all - less;
  double sum = 0.0;
  for (int i = lo + (threadIdx.x & 31); i < hi; i += 32) sum += rows.mass(i, gone, n_gone);
  return warp_sum64(sum);
}

// A number into another CTA's shared memory (or the own), and the signal that it is there.
__device__ __forceinline__ void send(uint32_t to, double x, uint32_t bar) {
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.b64 [%0], %1, [%2];" ::"r"(to), "l"(__double_as_longlong(x)),
               "r"(bar)
               : "memory");
}

__device__ __forceinline__ double warp_scan64(double v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const double y = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += y;
  }
  return v;
}

// Which of n <= 32 runs (one per lane: its sum, from 0 on, and the sum up to its end) holds the place `target` of the running sum that
// starts at `base`; the last one with any mass where roundings leave the place behind the end.  base becomes the sum before it; -1
// where nothing has mass.
__device__ __forceinline__ int pick_run(double sum, double upto, double target, double &base) {
  const unsigned over = __ballot_sync(0xffffffffu, sum > 0.0 && base + upto > target);
  const unsigned some = __ballot_sync(0xffffffffu, sum > 0.0);
  if (!some) return -1;
  const int at = over ? __ffs((int)over) - 1 : 31 - __clz((int)some);
  const double before = __shfl_sync(0xffffffffu, upto, at > 0 ? at - 1 : 0);
  if (at > 0) base += before;
  return at;
}
__device__ __forceinline__ int pick_run(double sum, double target, double &base) { return pick_run(sum, warp_scan64(sum), target, base); }

// kDistinct: there is a draft, drawn from without replacement.
template <typename T, bool kDistinct>
__global__ void __launch_bounds__(kThreads, kResident<T>) tree_verify_kernel(const VerifyParams p) {
  constexpr int E = Elem<T>::kPerChunk;
  // kDepth times a chunk of p and one of q for every thread (16 bytes off a 32-byte boundary a batch takes 8 % longer)
  extern __shared__ __align__(128) uint4 ring[];
  __shared__ Smem<kDistinct> sm;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int ranks = p.ranks, b = blockIdx.x >> p.rank_shift, rank = blockIdx.x & (ranks - 1);
  const bool rooted = p.target_prefix == nullptr;
  const char *target = p.target + b * p.target_seq;
  const char *draft = p.draft ? p.draft + b * p.draft_seq : nullptr;
  const char *target_prefix = rooted ? nullptr : p.target_prefix + b * p.target_prefix_seq;
  const char *draft_prefix = rooted || !draft ? nullptr : p.draft_prefix + b * p.draft_prefix_seq;

  int nodes = p.nodes ? p.nodes[b] : p.T, up = -1, x = 0;
  float u = 0.f;
  if (tid < p.T) {
    up = p.parent[b * p.T + tid];
    x = p.tokens[b * p.T + tid];
    u = p.accept_u[b * p.T + tid];
  }
  const float number = tid == 0 ? p.sample_u[b] : 0.f;
  if (nodes < 0 || nodes > p.T) {
    if (tid == 0 && rank == 0) atomicOr(p.status, ROCO_DEV_BAD_TREE);
    nodes = 0;
  }
  if (tid <= kNodes) sm.children[tid] = 0;
  if (tid == 0) {
    sm.abort_flag = 0;
    mbar_init(&sm.bar[0], 1);
    mbar_init(&sm.bar[1], 1);
    mbar_init_fence();
  }
  __syncthreads();
  if (tid < kNodes) {
    bool first = false;  // accepted if none of its siblings was rejected before it
    if (tid < nodes) {
      const bool given = rooted && tid == 0;  // the token sampled last: nothing is looked up for it
      const bool ok = up >= -1 && up < tid && (given || (x >= 0 && x < p.V));
      if (!ok && rank == 0) atomicOr(p.status, ROCO_DEV_BAD_TREE);
      if (ok && (given || up >= 0 || !rooted)) {
        if (!given) {
          const char *row = up < 0 ? target_prefix : target + up * p.target_row;
          const float px = Elem<T>::load(reinterpret_cast<const T *>(row) + x);
          float qx = 1.f;
          if (draft) {
            row = up < 0 ? draft_prefix : draft + up * p.draft_row;
            qx = Elem<T>::load(reinterpret_cast<const T *>(row) + x);
          }
          sm.p[tid] = px;
          sm.q[tid] = qx;
          sm.u[tid] = u;
          first = (double)u * qx < px;
        }
        sm.token[tid] = x;
        atomicOr(&sm.children[up + 1], 1ull << tid);
      }
    }
    const unsigned accepted = __ballot_sync(0xffffffffu, first);
    if (lane == 0) sm.first[warp] = accepted;
  }
  __syncthreads();

  // The walk is thread 0's (every rank's on its own, with the same numbers).
  if (rooted && !(sm.children[0] & 1)) {  // no root: nothing to verify, nothing to draw from (before any exchange)
    if (rank == 0) {
      if (tid < p.A) p.path[b * p.A + tid] = -1;
      if (tid == 0) {
        p.path_len[b] = 0;
        p.next_token[b] = -1;
      }
    }
    return;
  }
  if (tid == 0) {
    sm.path[0] = 0;
    sm.tip = rooted ? 0 : -1;
    sm.len = rooted ? 1 : 0;
    sm.untried = sm.children[rooted ? 1 : 0];
    sm.n_gone = 0;
    sm.C = 0.0; sm.R = 1.0; sm.M = 1.0;
    sm.number = number;
    sm.more = 0;
    sm.weigh = 0;
  }
  // (a peer's shared memory may be written once the peer runs and its barriers are ready; an aligned barrier wants the whole warp)
  __syncwarp();
  if (ranks > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  bool anew = false;   // nothing was left of p after the rejections: once more with p itself
  double total = 0.0, base = 0.0, mine[kPer];
  int pass = 0, out = 0, run = 0;   // out: tokens that are out of p
  int all_of = -2;             // the node behind which `all` is this warp's sum over all of p
  double c = 0.0, all = 0.0;
  Rows<T> rows;
  int first = 0, end = 0;      // the chunks that hold the next token, once the sums are known
  double place = 0.0;
  while (true) {
    if (tid == 0 && !anew && end == 0) {
      const unsigned long long firsts = sm.first[0] | (unsigned long long)sm.first[1] << 32;
      unsigned long long untried = sm.untried;
      int tip = sm.tip, len = sm.len, n_gone = sm.n_gone;
      double C = sm.C, R = sm.R, M = sm.M;
      bool more = false, summed = sm.more;   // R has been summed behind this node
      const double least = kLeast * R;
      while (!more && len < p.A && untried) {
        const int i = __ffsll((long long)untried) - 1, x = sm.token[i];
        untried &= untried - 1;
        bool again = false;   // rejected already
        for (int g = 0; g < n_gone; ++g) again |= sm.gone[g] == x;
        bool yes;
        double q = 0.0;
        if (n_gone == 0) {
          yes = firsts >> i & 1;
          q = sm.q[i];
        } else if (kDistinct || draft) {
          q = again && kDistinct ? 0.0 : sm.q[i];
          const double left = sm.p[i] - C * sm.q[i];
          yes = sm.u[i] * q * R < (left <= 0.0 ? 0.0 : left) * M;
        } else {
          yes = sm.u[i] * R < (again ? 0.0 : sm.p[i]);
        }
        if (yes) {
          sm.path[len++] = i;
          tip = i;
          untried = sm.children[i + 1];
          C = 0.0; R = 1.0; M = 1.0;
          n_gone = 0;
          summed = false;
        } else {
          if (!again) {
            sm.gone_p[n_gone] = sm.p[i] > 0.0 ? sm.p[i] : 0.0;
            sm.gone[n_gone++] = x;
          }
          if (kDistinct || draft) {
            if (M > 0.0) C += M == 1.0 ? R : R / M;
            if (kDistinct) M -= q;
            more = untried != 0;
          } else if (!summed) {
            more = untried != 0;
          } else if (!again) {
            R -= sm.gone_p[n_gone - 1];
            more = untried != 0 && R < least;
          }
        }
      }
      sm.untried = untried;
      sm.tip = tip;
      sm.len = len;
      sm.n_gone = n_gone;
      sm.C = C;
      sm.R = R;
      sm.M = M;
      sm.more = more;
      if (kDistinct) sm.weigh = more && M < kLittle;
    }
    __syncthreads();
    int lo, hi;
    const bool weigh = kDistinct && end == 0 && !anew && sm.weigh;
    if (end == 0) {
      const int on = sm.tip;
      c = anew ? 0.0 : sm.C;
      out = kDistinct || draft || anew ? 0 : sm.n_gone;
      rows = Rows<T>(on < 0 ? target_prefix : target + on * p.target_row,
                     !draft || (c == 0.0 && !weigh) ? nullptr : on < 0 ? draft_prefix : draft + on * p.draft_row, p.V);
      // runs of chunks: of this rank, of this warp in it
      run = (rows.chunks + (kWarps << p.rank_shift) - 1) >> (kWarpShift + p.rank_shift);
      lo = min((rank * kWarps + warp) * run, rows.chunks);
      hi = min(lo + run, rows.chunks);
    } else {  // a long run is cut among the warps once more
      run = (end - first + kWarps - 1) >> kWarpShift;
      lo = min(first + warp * run, end);
      hi = min(lo + run, end);
    }
    // Tokens that are out are taken off a sum over all of p, which stands while the walk stays at its node; where too little would be
    // left of it, the sum is formed without them.
    const bool from_all = !kDistinct && !draft && end == 0 && !anew;
    int here = 0;
    double less = 0.0;
    if (from_all) {
      for (int g = 0; g < out; ++g) {
        const int at = sm.gone[g] + rows.lead;
        if (at >= lo * E && at < hi * E) {
          ++here;
          less += sm.gone_p[g];
        }
      }
    }
    const bool known = from_all && all_of == sm.tip;
    double sum = known ? all : 0.0, mass = 0.0;
    for (int exact = from_all ? 0 : 1; exact < 2; ++exact) {
      if (exact || !known) sum = sum_run(rows, lo, hi, c, sm.gone, exact ? out : 0, ring + tid, weigh, mass);
      if (exact) break;
      all = sum;
      all_of = sm.tip;
      sum -= less;
      if (!here || sum > kLeast * all) break;
    }
    if (weigh) mass = mass_left(rows, lo, hi, mass, sm.gone, sm.n_gone);
    if (end != 0) {
      if (lane == 0) sm.part[warp] = sum;
      __syncthreads();
      const int at = pick_run(lane < kWarps ? sm.part[lane] : 0.0, place, base);
      first = min(first + at * run, end);
      end = min(first + run, end);
      if (end - first <= kLast) break;
      continue;
    }
    double *sums = sm.sums[pass & 1], *masses = sm.masses[pass & 1];
    if (ranks > 1) {
      // every warp sends its sum to every rank; the store and the signal that it is there travel together
      __syncwarp();
      if (pass == 0) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
      uint64_t *bar = &sm.bar[pass & 1];
      if (tid == 0) mbar_expect_tx(bar, ranks * kWarps * (weigh ? 16 : 8));
      if (lane < ranks) {
        send(map_to_rank(&sums[rank * kWarps + warp], lane), sum, map_to_rank(bar, lane));
        if (weigh) send(map_to_rank(&masses[rank * kWarps + warp], lane), mass, map_to_rank(bar, lane));
      }
      mbar_wait_compact(bar, (pass >> 1) & 1, &sm.abort_flag, p.status);
    } else {
      if (lane == 0) {
        sums[warp] = sum;
        if (kDistinct) masses[warp] = mass;
      }
      __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k) mine[k] = kPer * lane + k < ranks * kWarps ? sums[kPer * lane + k] : 0.0;
    double some = mine[0];
#pragma unroll
    for (int k = 1; k < kPer; ++k) some += mine[k];
    const double upto = warp_scan64(some);
    total = __shfl_sync(0xffffffffu, upto, 31);
    if (tid == 0) sm.R = total;
    if (weigh && warp == 0) {
      double m = 0.0;
#pragma unroll
      for (int k = 0; k < kPer; ++k) m += kPer * lane + k < ranks * kWarps ? masses[kPer * lane + k] : 0.0;
      m = warp_sum64(m);
      if (lane == 0 && isfinite(m)) sm.M = m;
    }
    ++pass;
    // on with the walk, or once more where nothing is left
    const bool more = sm.more;
    if (!anew && !more && total == 0.0 && (sm.C != 0.0 || sm.n_gone > 0)) anew = true;
    else if (anew || !more) {
      // the last exchange; nobody leaves before everybody has it
      __syncwarp();
      if (ranks > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
      if (rank == 0) {
        if (tid < p.A) p.path[b * p.A + tid] = tid < sm.len ? sm.path[tid] : -1;
        if (tid == 0) p.path_len[b] = sm.len;
      }
      if (!(total > 0.0) || isinf(total)) {   // no distribution to draw from
        if (rank == 0 && tid == 0) {
          p.next_token[b] = -1;
          atomicOr(p.status, ROCO_DEV_BAD_PROBS);
        }
        __syncwarp();
        if (ranks > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        return;
      }
      // the pick descends the sums: a few warps, one of them, chunks of its run, one chunk, one element
      place = sm.number * total;
      const int lane_at = pick_run(some, upto, place, base);
      int k_at = 0;   // (the lane's first run with mass that reaches the place, else its last with mass)
      double before = 0.0, sofar = 0.0;
      bool found = false;
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        if (!found && mine[k] > 0.0) {
          k_at = k;
          before = sofar;
          found = base + (sofar + mine[k]) > place;
        }
        sofar += mine[k];
      }
      const int at = __shfl_sync(0xffffffffu, kPer * lane + k_at, lane_at);
      base += __shfl_sync(0xffffffffu, before, lane_at);
      if (at / kWarps != rank) {
        if (ranks > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        return;
      }
      first = min(at * run, rows.chunks);
      end = min(first + run, rows.chunks);
      if (end - first <= kLast) break;
    }
    __syncthreads();   // (what is written next has been read)
  }
  // a chunk per thread
  double r[E], own = 0.0;
#pragma unroll
  for (int e = 0; e < E; ++e) r[e] = 0.0;
  if (first + tid < end) rows.left(first + tid, c, sm.gone, out, r);
#pragma unroll
  for (int e = 0; e < E; ++e) own += r[e];
  const double upto = warp_scan64(own);
  __syncthreads();   // (part has been read)
  if (lane == 31) sm.part[warp] = upto;
  __syncwarp();
  if (ranks > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  __syncthreads();
  if (pick_run(lane < kWarps ? sm.part[lane] : 0.0, place, base) != warp) return;
  if (pick_run(own, upto, place, base) != lane) return;
  int token = 0;   // the first element with mass that reaches the place, else the last with mass
  bool found = false;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (!found && r[e] > 0.0) {
      token = (first + tid) * E - rows.lead + e;
      found = base + r[e] > place;
      base += r[e];
    }
  }
  p.next_token[b] = token;
}

template <typename T, bool kDistinct>
roco_status launch_t(VerifyParams p, int S, int sms, cudaStream_t stream) {
  // CTAs per sequence, a power of two: doubled while they fill less than three quarters of the GPU, so up to half as many again as
  // reside together, because the walks with most rejections end last and every rejection costs a pass over a row by its own CTAs
  // alone (64 sequences x 128000 tokens, fp32: eight 31.3 us; with three CTAs per SM eight took 34, six, which reside together, 37, four 53).
  // None with fewer 16-byte chunks of a row than threads.
  int shift = 0;
  const long long chunks = (p.V + Elem<T>::kPerChunk - 1) / Elem<T>::kPerChunk;
  while ((1 << shift) < kMaxRanks && ((4LL * S) << shift) < 3LL * kResident<T> * sms && chunks >= (2LL * kThreads) << shift) ++shift;
  p.rank_shift = shift;
  p.ranks = 1 << shift;
  const int ranks = p.ranks;
  static SmemLimit limit;
  const auto kernel = tree_verify_kernel<T, kDistinct>;
  if (!limit((const void *)kernel, kRingBytes)) return ROCO_ERR_CUDA;
  const bool ok = launch_cluster(kernel, (unsigned)S * (unsigned)ranks, (unsigned)ranks, kThreads, kRingBytes, stream, p);
  return ok ? ROCO_OK : ROCO_ERR_CUDA;
}

}  // namespace

roco_status launch_tree_verify(const VerifyParams &p, int dtype, int S, int sms, cudaStream_t stream) {
  if (p.draft && p.distinct)
    return dtype == ROCO_BF16 ? launch_t<__nv_bfloat16, true>(p, S, sms, stream) : launch_t<float, true>(p, S, sms, stream);
  return dtype == ROCO_BF16 ? launch_t<__nv_bfloat16, false>(p, S, sms, stream) : launch_t<float, false>(p, S, sms, stream);
}

}  // namespace roco
