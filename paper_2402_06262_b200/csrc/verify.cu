// Verification of drafted trees against the target's probabilities.
//
// A cluster of CTAs (one to eight) per sequence.  Everything about a node is two numbers, p(x) and q(x) behind its parent, fetched for
// all nodes at once; the walk over them is a few instructions per child.  A row is only touched where a child was rejected (to sum
// what is left of p) and at the end (to pick the next token): what is left of p after any number of rejections is
// max(p - C q, 0) for one C, because rejecting once more takes (R / M) q from what is still positive and leaves zero at zero.  A row is
// cut into one run per CTA and that into one per warp, so the sums that a pass leaves behind are a prefix sum's upper levels, and the
// pick descends them: CTA, warp, the chunk of 32 lanes, the lane.
// Bound by the latencies of a chain (two loads of the nodes' numbers, the row, the sums' way through the cluster), for many
// sequences by the rows' bytes.  Sums and products are in 64 bits: an index is the answer, and an error of 2^-24 in a sum over
// 10^5 tokens moves it about once in a thousand calls.
#include "heads.cuh"

namespace roco {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxRanks = 8;
constexpr int kNodes = ROCO_TREE_MAX_NODES;
static_assert(kNodes == 64, "a node's children are the bits of one 64-bit word");

struct Smem {
  double p[kNodes], q[kNodes], u[kNodes];
  unsigned long long children[kNodes + 1];  // of the prefix, then of every node
  double warp_sum[kWarps];
  double rank_sum[2][kMaxRanks];            // written by all ranks, one set while the other may still be read
  int token[kNodes];
  int gone[kNodes];                         // tokens rejected behind the node the walk stands on
  int n_gone, path_len, path[ROCO_TREE_MAX_PATH];
  int tip, more;                            // what the next pass is for
  double C;
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

  __device__ Rows(const char *target, const char *draft, int v) : p(reinterpret_cast<const T *>(target)), q(reinterpret_cast<const T *>(draft)), V(v) {
    lead = (int)((reinterpret_cast<uintptr_t>(target) & 15u) / sizeof(T));
    chunks = (int)(((long long)V + lead + E - 1) / E);
    q_like_p = ((reinterpret_cast<uintptr_t>(target) ^ reinterpret_cast<uintptr_t>(draft)) & 15u) == 0;
  }

  __device__ __forceinline__ void some(const T *row, int first, float (&f)[E]) const {
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = first + e >= 0 && first + e < V ? Elem<T>::load(row + first + e) : 0.f;
  }

  // The probabilities of chunk i; elements outside the row are 0.
  __device__ __forceinline__ void load(int i, float (&fp)[E], float (&fq)[E]) const {
    const int first = i * E - lead;
    const bool whole = first >= 0 && first + E <= V;
    if (whole) Elem<T>::unpack(__ldg(reinterpret_cast<const uint4 *>(p + first)), fp);
    else some(p, first, fp);
    if (q) {
      if (whole && q_like_p) Elem<T>::unpack(__ldg(reinterpret_cast<const uint4 *>(q + first)), fq);
      else some(q, first, fq);
    }
  }

  // What is left of p in them.  A NaN stays one.
  __device__ __forceinline__ void left(int i, const float (&fp)[E], const float (&fq)[E], double C, const int *gone, int n_gone,
                                       double (&r)[E]) const {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const double x = q ? (double)fp[e] - C * (double)fq[e] : (double)fp[e];
      r[e] = x <= 0.0 ? 0.0 : x;
    }
    const int first = i * E - lead;
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

// Which of n runs holds the place `target` of the running sum that starts at `base`; the last one with any mass where roundings
// leave the place behind the end.  base becomes the sum before the run; -1 where nothing has mass.
__device__ __forceinline__ int pick_run(const double *sums, int n, double target, double &base) {
  int at = -1;
  double before = base, sum = base;
  for (int i = 0; i < n; ++i) {
    if (sums[i] > 0.0) {
      at = i;
      before = sum;
      if (sum + sums[i] > target) break;
    }
    sum += sums[i];
  }
  base = before;
  return at;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) tree_verify_kernel(const VerifyParams p) {
  constexpr int E = Elem<T>::kPerChunk;
  __shared__ Smem sm;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int ranks = p.ranks, b = blockIdx.x / ranks, rank = blockIdx.x - b * ranks;
  const bool rooted = p.target_prefix == nullptr;
  const char *target = p.target + b * p.target_seq;
  const char *draft = p.draft ? p.draft + b * p.draft_seq : nullptr;
  const char *target_prefix = rooted ? nullptr : p.target_prefix + b * p.target_prefix_seq;
  const char *draft_prefix = rooted || !draft ? nullptr : p.draft_prefix + b * p.draft_prefix_seq;

  int nodes = p.nodes ? p.nodes[b] : p.T;
  if (nodes < 0 || nodes > p.T) {
    if (tid == 0 && rank == 0) atomicOr(p.status, ROCO_DEV_BAD_TREE);
    nodes = 0;
  }
  if (tid <= kNodes) sm.children[tid] = 0;
  __syncthreads();
  if (tid < nodes) {
    const int up = p.parent[b * p.T + tid], x = p.tokens[b * p.T + tid];
    const bool given = rooted && tid == 0;  // the token sampled last: nothing is looked up for it
    const bool ok = up >= -1 && up < tid && (given || (x >= 0 && x < p.V));
    if (!ok && rank == 0) atomicOr(p.status, ROCO_DEV_BAD_TREE);
    if (ok && (given || up >= 0 || !rooted)) {
      if (!given) {
        const char *row = up < 0 ? target_prefix : target + up * p.target_row;
        sm.p[tid] = Elem<T>::load(reinterpret_cast<const T *>(row) + x);
        if (draft) {
          row = up < 0 ? draft_prefix : draft + up * p.draft_row;
          sm.q[tid] = Elem<T>::load(reinterpret_cast<const T *>(row) + x);
        }
        sm.u[tid] = p.accept_u[b * p.T + tid];
      }
      sm.token[tid] = x;
      atomicOr(&sm.children[up + 1], 1ull << tid);
    }
  }
  __syncthreads();

  // The walk; thread 0 keeps it (every rank on its own, with the same numbers).
  int tip = -1, len = 0, n_gone = 0;
  double C = 0.0, R = 1.0, M = 1.0;
  unsigned long long untried = sm.children[0];
  if (rooted) {
    if (!(untried & 1)) {  // no root: nothing to verify, nothing to draw from.  (Uniform, and before any exchange.)
      if (rank == 0) {
        if (tid < p.A) p.path[b * p.A + tid] = -1;
        if (tid == 0) {
          p.path_len[b] = 0;
          p.next_token[b] = -1;
        }
      }
      return;
    }
    if (tid == 0) sm.path[0] = 0;
    tip = 0;
    len = 1;
    untried = sm.children[1];
  }
  // (a peer's shared memory may be written once the peer runs)
  if (ranks > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  bool met = ranks == 1;
  bool anew = false;   // nothing was left of p after the rejections: once more with p itself
  double total = 0.0, base = 0.0;
  int parity = 0;
  while (true) {
    if (tid == 0 && !anew) {
      bool rejected = false;
      while (!rejected && len < p.A && untried) {
        const int i = __ffsll((long long)untried) - 1, x = sm.token[i];
        untried &= untried - 1;
        const double u = sm.u[i];
        bool again = false;   // rejected already
        for (int g = 0; g < n_gone; ++g) again |= sm.gone[g] == x;
        bool yes;
        double q = 0.0;
        if (draft) {
          q = again && p.distinct ? 0.0 : sm.q[i];
          const double x_left = sm.p[i] - C * sm.q[i];
          yes = u * q * R < (x_left <= 0.0 ? 0.0 : x_left) * M;
        } else {
          yes = u * R < (again ? 0.0 : sm.p[i]);
        }
        if (yes) {
          sm.path[len++] = i;
          tip = i;
          untried = sm.children[i + 1];
          C = 0.0; R = 1.0; M = 1.0;
          n_gone = 0;
        } else {
          rejected = true;
          sm.gone[n_gone++] = x;
          if (draft && M > 0.0) C += R / M;
          if (p.distinct) M -= q;
        }
      }
      sm.tip = tip;
      sm.C = C;
      sm.n_gone = n_gone;
      sm.path_len = len;
      sm.more = rejected && len < p.A && untried;   // a sibling is left to try
    }
    __syncthreads();
    const int at = sm.tip;
    const double c = anew ? 0.0 : sm.C;
    const int out = draft || anew ? 0 : sm.n_gone;
    const Rows<T> rows(at < 0 ? target_prefix : target + at * p.target_row,
                       c == 0.0 || !draft ? nullptr : at < 0 ? draft_prefix : draft + at * p.draft_row, p.V);
    // runs of chunks: of this rank, of this warp in it
    const int run = (rows.chunks + ranks * kWarps - 1) / (ranks * kWarps);
    const int lo = min((rank * kWarps + warp) * run, rows.chunks), hi = min(lo + run, rows.chunks);
    double sum = 0.0;
#pragma unroll 4
    for (int i = lo + lane; i < hi; i += 32) {
      float fp[E], fq[E];
      double r[E];
      rows.load(i, fp, fq);
      rows.left(i, fp, fq, c, sm.gone, out, r);
#pragma unroll
      for (int e = 0; e < E; ++e) sum += r[e];
    }
    sum = warp_sum64(sum);
    if (lane == 0) sm.warp_sum[warp] = sum;
    __syncthreads();
    double mine = 0.0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) mine += sm.warp_sum[w];
    if (!met) {
      asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
      met = true;
    }
    if (ranks > 1) {
      if (tid < ranks) {
        const uint32_t dst = map_to_rank(&sm.rank_sum[parity][rank], tid);
        asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(dst), "d"(mine) : "memory");
      }
      cluster_sync_all();
    } else {
      if (tid == 0) sm.rank_sum[parity][0] = mine;
      __syncthreads();
    }
    total = 0.0;
    for (int k = 0; k < ranks; ++k) total += sm.rank_sum[parity][k];
    R = total;
    if (!anew && sm.more) {
      parity ^= 1;
      __syncthreads();   // (what thread 0 writes next has been read)
      continue;
    }
    // the last pass, unless nothing is left
    if (!(total > 0.0) && total == 0.0 && !anew && (sm.C != 0.0 || sm.n_gone > 0)) {
      anew = true;
      parity ^= 1;
      __syncthreads();
      continue;
    }
    if (rank == 0) {
      if (tid < p.A) p.path[b * p.A + tid] = tid < sm.path_len ? sm.path[tid] : -1;
      if (tid == 0) p.path_len[b] = sm.path_len;
    }
    if (!(total > 0.0) || isinf(total)) {   // no distribution to draw from
      if (rank == 0 && tid == 0) {
        p.next_token[b] = -1;
        atomicOr(p.status, ROCO_DEV_BAD_PROBS);
      }
      return;
    }
    // the pick: rank, then warp, then chunk by chunk with one warp
    const double place = (double)p.sample_u[b] * total;
    base = 0.0;
    if (pick_run(sm.rank_sum[parity], ranks, place, base) != rank) return;
    const int w = pick_run(sm.warp_sum, kWarps, place, base);
    int first = min((rank * kWarps + w) * run, rows.chunks), end = min(first + run, rows.chunks);
    __syncthreads();   // (warp_sum has been read)
    // A run of more than eight times 32 chunks is cut among the warps once more.
    while (end - first > 256) {
      const int sub = (end - first + kWarps - 1) / kWarps;
      const int l = min(first + warp * sub, end), h = min(l + sub, end);
      sum = 0.0;
      for (int i = l + lane; i < h; i += 32) {
        float fp[E], fq[E];
        double r[E];
        rows.load(i, fp, fq);
        rows.left(i, fp, fq, c, sm.gone, out, r);
#pragma unroll
        for (int e = 0; e < E; ++e) sum += r[e];
      }
      sum = warp_sum64(sum);
      if (lane == 0) sm.warp_sum[warp] = sum;
      __syncthreads();
      const int k = pick_run(sm.warp_sum, kWarps, place, base);
      first = min(first + k * sub, end);
      end = min(first + sub, end);
      __syncthreads();
    }
    if (warp != 0) return;
    int answer = -1;
    for (int i0 = first; i0 < end; i0 += 32) {
      const int i = i0 + lane;
      float fp[E], fq[E];
      double r[E], own = 0.0;
#pragma unroll
      for (int e = 0; e < E; ++e) r[e] = 0.0;
      if (i < end) {
        rows.load(i, fp, fq);
        rows.left(i, fp, fq, c, sm.gone, out, r);
      }
#pragma unroll
      for (int e = 0; e < E; ++e) own += r[e];
      double upto = own;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const double y = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += y;
      }
      const unsigned over = __ballot_sync(0xffffffffu, own > 0.0 && base + upto > place);
      const unsigned some = __ballot_sync(0xffffffffu, own > 0.0);
      const int who = over ? __ffs(over) - 1 : some ? 31 - __clz(some) : -1;
      if (lane == who) {
        double sums = base + (upto - own);
        for (int e = 0; e < E; ++e) {
          if (r[e] > 0.0) {
            answer = i * E - rows.lead + e;
            if (sums + r[e] > place) break;
          }
          sums += r[e];
        }
      }
      const int found = __shfl_sync(0xffffffffu, answer, who < 0 ? 0 : who);
      if (who >= 0) answer = found;
      if (over) break;
      base += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (lane == 0) p.next_token[b] = answer;
    return;
  }
}

template <typename T>
roco_status launch_t(VerifyParams p, int S, int sms, cudaStream_t stream) {
  // CTAs per sequence: as many as are resident together (two per SM), none with fewer than a chunk for every thread.
  int ranks = 1;
  const long long chunks = (p.V + Elem<T>::kPerChunk - 1) / Elem<T>::kPerChunk;
  while (ranks < kMaxRanks && 2LL * S * ranks <= 2LL * sms && chunks >= 2LL * ranks * kThreads) ranks *= 2;
  p.ranks = ranks;
  const bool ok = launch_cluster(tree_verify_kernel<T>, (unsigned)S * (unsigned)ranks, (unsigned)ranks, kThreads, 0, stream, p);
  return ok ? ROCO_OK : ROCO_ERR_CUDA;
}

}  // namespace

roco_status launch_tree_verify(const VerifyParams &p, int dtype, int S, int sms, cudaStream_t stream) {
  return dtype == ROCO_BF16 ? launch_t<__nv_bfloat16>(p, S, sms, stream) : launch_t<float>(p, S, sms, stream);
}

}  // namespace roco
