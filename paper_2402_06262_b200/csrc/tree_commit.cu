// Commit of the accepted path of a draft tree: the statistics of Sec. 4.3 for the accepted queries over the cached
// tokens (CUDA-core kernel; tensor-core kernel in tree_commit_tc.cu), then per unit the evictions on the updated
// statistics and the insertion of the accepted tokens.
#include "multi.cuh"
#include "tree.cuh"

namespace roco {

// ---------------------------------------------------------------- statistics, CUDA cores

constexpr int kCsThreads = 256;
constexpr int kCsKeys = kCsThreads / 4;  // keys in flight per CTA
constexpr int kCsRows = 16;              // query rows staged at a time (whole tokens: a multiple of the group)

// Four threads share a key: each keeps a quarter of it in registers and the queries pass by in shared memory, so a key
// is read once whatever the number of accepted queries.  p_ij = 2^(x_ij - lse_i) needs no maximum and no sum: the
// log-sum-exp is known.
template <typename T, int D>
__global__ void __launch_bounds__(kCsThreads) commit_stats_simt_kernel(const CommitParams p, int keys_per_cta, int key_blocks) {
  constexpr int kQ = D / 4;        // elements of a quarter
  constexpr int kPitch = kQ + 4;   // the four quarters of a query row lie in different banks
  constexpr int kEPC = Elem<T>::kPerChunk;
  __shared__ __align__(16) float sq[kCsRows][4 * kPitch];
  __shared__ float slse[kCsRows];
  __shared__ int sh_a, sh_node[32];
  const int tid = threadIdx.x, u = blockIdx.x / key_blocks, kb = blockIdx.x % key_blocks, b = u / p.G;
  if (tid < 32) {
    int node;
    const int a = commit_path(p, b, tid, node, kb == 0);
    sh_node[tid] = node;
    if (tid == 0) sh_a = a;
  }
  __syncthreads();
  const int a = sh_a;
  if (a == 0) return;
  const int live = tree_live(p.live, u, p.B, p.status, tid == 0 && kb == 0);
  const int key0 = kb * keys_per_cta, key1 = key0 + keys_per_cta < live ? key0 + keys_per_cta : live;
  if (key0 >= live) return;
  const int key = tid >> 2, quarter = tid & 3;
  const float zscale = p.scale * kLog2e, inv_group = 1.f / (float)p.group;
  const T *Qu = reinterpret_cast<const T *>(p.Q) + (size_t)u * p.T * p.group * D;
  const T *Ku = reinterpret_cast<const T *>(p.K) + (size_t)u * p.B * D;
  const int per = kCsRows / p.group;  // accepted tokens per pass over the queries
  // One pass over the queries serves all keys of the CTA when they fit (the usual case); a key's sums over several
  // passes are carried in its statistics.
  for (int i0 = 0; i0 < a; i0 += per) {
    const int nt = a - i0 < per ? a - i0 : per, rows = nt * p.group;
    __syncthreads();
    for (int w = tid; w < rows * D / kEPC; w += kCsThreads) {
      const int rr = w / (D / kEPC), c = w % (D / kEPC) * kEPC;
      float f[kEPC];
      Elem<T>::unpack(*reinterpret_cast<const uint4 *>(Qu + ((size_t)sh_node[i0 + rr / p.group] * p.group + rr % p.group) * D + c), f);
#pragma unroll
      for (int e = 0; e < kEPC; ++e) sq[rr][(c + e) / kQ * kPitch + (c + e) % kQ] = f[e];
    }
    if (tid < rows)
      slse[tid] = p.lse[((size_t)u * p.T + sh_node[i0 + tid / p.group]) * p.group + tid % p.group] * kLog2e;
    __syncthreads();
    for (int j0 = key0; j0 < key1; j0 += kCsKeys) {
      const int j = j0 + key;
      const bool valid = j < key1;
      float k[kQ];
#pragma unroll
      for (int c = 0; c < kQ; c += kEPC) {
        uint4 x = make_uint4(0u, 0u, 0u, 0u);
        if (valid) x = *reinterpret_cast<const uint4 *>(Ku + (size_t)j * D + quarter * kQ + c);
        float f[kEPC];
        Elem<T>::unpack(x, f);
#pragma unroll
        for (int e = 0; e < kEPC; ++e) k[c + e] = f[e];
      }
      float ds = 0.f, dq = 0.f;
      for (int t = 0; t < nt; ++t) {
        float pbar = 0.f;
        for (int g = 0; g < p.group; ++g) {
          const float *qr = &sq[t * p.group + g][quarter * kPitch];
          float x = 0.f;
#pragma unroll
          for (int c = 0; c < kQ; c += 4) {
            const float4 qv = *reinterpret_cast<const float4 *>(qr + c);
            x = fmaf(qv.x, k[c], fmaf(qv.y, k[c + 1], fmaf(qv.z, k[c + 2], fmaf(qv.w, k[c + 3], x))));
          }
          x += __shfl_xor_sync(0xffffffffu, x, 1);
          x += __shfl_xor_sync(0xffffffffu, x, 2);
          pbar += exp2f(fmaf(x, zscale, -slse[t * p.group + g]));
        }
        pbar *= inv_group;
        ds += pbar;
        dq = fmaf(pbar, pbar, dq);
      }
      if (valid) {
        const size_t at = (size_t)u * p.B + j;
        if (quarter == 0) p.s[at] += ds;
        if (quarter == 1) p.q[at] += dq;
        if (quarter == 2 && i0 == 0) p.n[at] += a;
      }
    }
  }
}

// ---------------------------------------------------------------- evictions and insertion, one CTA per unit

constexpr int kCiMaxA = ROCO_TREE_MAX_PATH;
constexpr int kCiShort = 64;  // candidates that are ranked one against the other

struct CiScratch {
  SelectScratch sel;
  int ctl[64];  // 20: counter; 24 .. 39: the chosen slots (the places that lowest_r_block_victims uses)
  int cand[kCiShort];
  uint32_t group_min[16], threshold;
};

// The kn (<= 16) slots first in (key, position) order over keys that are bit patterns of non-negative floats below
// infinity, in that order to sc.ctl[24 ..]; false if there are fewer.  The threads form 16 groups: at least kn keys lie
// at or below the kn-th smallest of the groups' minima, and few more, so those are gathered and ranked one against the
// other.  Only where many keys are equal do they not fit; then a radix select finds the threshold and the lowest
// positions at it.  Every thread of the CTA calls it.
template <int NT>
__device__ __forceinline__ bool lowest_slots(const uint32_t *key, const int *pos, int live, int kn, CiScratch &sc) {
  const int tid = threadIdx.x;
  int *list = sc.ctl + 24, *cnt = sc.ctl + 20;
  constexpr uint32_t kInf = 0x7f800000u;
  uint32_t low = 0xffffffffu;
  for (int j = tid; j < live; j += NT) low = min(low, key[j]);
#pragma unroll
  for (int o = NT / 32; o > 0; o >>= 1) low = min(low, __shfl_xor_sync(0xffffffffu, low, o));  // NT / 16 neighbours
  if (tid % (NT / 16) == 0) sc.group_min[tid / (NT / 16)] = low;
  if (tid == 0) *cnt = 0;
  __syncthreads();
  if (tid < 16) {
    int rank = 0;
    const uint32_t mine = sc.group_min[tid];
#pragma unroll
    for (int i = 0; i < 16; ++i) rank += sc.group_min[i] < mine || (sc.group_min[i] == mine && i < tid);
    if (rank == kn - 1) sc.threshold = mine;
  }
  __syncthreads();
  const uint32_t T = sc.threshold;
  for (int j = tid; j < live; j += NT) {
    const uint32_t k = key[j];
    if (k <= T && k < kInf) {
      const int at = atomicAdd(cnt, 1);
      if (at < kCiShort) sc.cand[at] = j;
    }
  }
  __syncthreads();
  const int n = *cnt;
  __syncthreads();
  if (n <= kCiShort) {
    if (tid < n) {
      const int j = sc.cand[tid];
      const uint32_t k = key[j];
      const int ps = pos[j];
      int rank = 0;
      for (int i = 0; i < n; ++i) {
        const int c = sc.cand[i];
        const uint32_t kc = key[c];
        rank += kc < k || (kc == k && pos[c] < ps);
      }
      if (rank < kn) list[rank] = j;
    }
    __syncthreads();
    return n >= kn;
  }
  uint32_t k_and = 0xffffffffu, k_or = 0u, rank, ties;
  for (int j = tid; j < live; j += NT) { k_and &= key[j]; k_or |= key[j]; }
  group_and_or(k_and, k_or, sc.sel, tid, NT, kMqBarPolicy);
  const uint32_t R = radix_select<uint32_t>([&](int j) { return key[j]; }, [&](int) { return true; }, live, (uint32_t)(kn - 1),
                                            sc.sel, tid, NT, kMqBarPolicy, &rank, &ties, k_and, k_or);
  int P = 0x7fffffff;
  if (ties != rank + 1) {  // only some of the slots tied at the threshold: lowest positions
    uint32_t r2, t2;
    P = (int)radix_select<uint32_t>([&](int j) { return (uint32_t)pos[j]; }, [&](int j) { return key[j] == R; }, live, rank,
                                    sc.sel, tid, NT, kMqBarPolicy, &r2, &t2);
  }
  if (tid == 0) *cnt = 0;
  __syncthreads();
  for (int j = tid; j < live; j += NT) {
    const uint32_t k = key[j];
    if (k < kInf && (k < R || (k == R && (P == 0x7fffffff || pos[j] <= P)))) {
      const int at = atomicAdd(cnt, 1);
      if (at < kCiMaxA) list[at] = j;
    }
  }
  __syncthreads();
  return *cnt == kn;
}

// NT threads: the keys of a unit are formed, scanned for the lowest means and counted for the scope, each pass over shared
// memory; what bounds it is the chain of these passes and of the first loads, so the loads of the statistics do not wait
// for the check of the path.
template <typename T, int D, int NT>
__global__ void __launch_bounds__(NT) commit_insert_kernel(const CommitParams p) {
  extern __shared__ char ci_smem[];
  __shared__ CiScratch sc;
  __shared__ int tgt[kCiMaxA], sh_node[32], sh_a;
  __shared__ float pbar[kCiMaxA][kCiMaxA];  // [query][accepted token]
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, u = blockIdx.x, b = u / p.G, A = p.A, B = p.B;
  const size_t st = (size_t)u * B;
  uint32_t *vkey = reinterpret_cast<uint32_t *>(ci_smem);
  float *mkey = reinterpret_cast<float *>(vkey + B);
  uint32_t *mbits = reinterpret_cast<uint32_t *>(mkey);
  const int *opos = p.pos + st;
  const int live = tree_live(p.live, u, B, p.status, false), t_new = p.t_next[u];
  if (warp == 0) {
    int node;
    const int a = commit_path(p, b, lane, node, false);
    sh_node[lane] = node;
    if (lane == 0) sh_a = a;
  }
  uint32_t k_and = 0xffffffffu, k_or = 0u;
  if (live + A > B) {  // (some path could evict)
#pragma unroll 4
    for (int j = tid; j < live; j += NT) {
      const float s = p.s[st + j], q = p.q[st + j];
      const int n = p.n[st + j];
      const uint32_t v = variance_key_fast(s, q, n);
      vkey[j] = v;
      mkey[j] = mean_fast(s, n);
      k_and &= v;
      k_or |= v;
    }
  }
  __syncthreads();
  const int a = sh_a;
  if (a == 0) {
    if (tid < A) {
      p.ev_slot[(size_t)u * A + tid] = -1;
      if (p.ev_pos) p.ev_pos[(size_t)u * A + tid] = -1;
    }
    return;
  }
  const int need = live + a - B > 0 ? live + a - B : 0;
  int *list = sc.ctl + 24;

  // the accepted queries against the accepted tokens, a warp per (query, token) at a time
  {
    constexpr int kN = D / 32;
    const float zscale = p.scale * kLog2e;
    const T *Qu = reinterpret_cast<const T *>(p.Q) + (size_t)u * p.T * p.group * D;
    const T *Ku = reinterpret_cast<const T *>(p.k_new) + (size_t)u * p.T * D;
    for (int w = warp; w < a * (a + 1) / 2; w += NT / 32) {
      int i = 0;
      while ((i + 1) * (i + 2) / 2 <= w) ++i;
      const int m = w - i * (i + 1) / 2;  // m <= i
      float k[kN], sum = 0.f;
#pragma unroll
      for (int c = 0; c < kN; ++c) k[c] = Elem<T>::load(Ku + (size_t)sh_node[m] * D + c * 32 + lane);
#pragma unroll 4
      for (int g = 0; g < p.group; ++g) {
        const size_t row = (size_t)sh_node[i] * p.group + g;
        float x = 0.f;
#pragma unroll
        for (int c = 0; c < kN; ++c) x = fmaf(Elem<T>::load(Qu + row * D + c * 32 + lane), k[c], x);
        x = warp_sum(x);
        sum += exp2f(fmaf(x, zscale, -p.lse[(size_t)u * p.T * p.group + row] * kLog2e));
      }
      if (lane == 0) pbar[i][m] = sum / (float)p.group;
    }
  }

  if (need > 0) {
    const int m = scope_size(live, p.r, p.scope_mode);
    bool ok = true;
    if (need > 1 && p.scope_mode == ROCO_SCOPE_LOWEST_R && m < live) {
      group_and_or(k_and, k_or, sc.sel, tid, NT, kMqBarPolicy);
      if (tid < kMqPolicyThreads)
        lowest_r_block_victims(vkey, mkey, &sc.sel, sc.ctl, opos, p.status, p.r, live, need, m, k_and, k_or, tid);
    } else {
      // Frozen statistics: the m first in (variance, position) order stay the scope, and the `need` of them first in
      // (mean, position) order leave.  Those are looked for among all cached tokens first: they are all in scope if the
      // one of them last in (variance, position) order is, which one count decides; a scope that leaves out few tokens
      // nearly always contains them, and the search for its threshold is saved.
      bool done = m == live;
      ok = lowest_slots<NT>(mbits, opos, live, need, sc);
      if (!done && ok) {
        uint32_t cv = 0u;
        int cp = -1;
        for (int e = 0; e < need; ++e) {
          const uint32_t v = vkey[list[e]];
          const int ps = opos[list[e]];
          if (v > cv || (v == cv && ps > cp)) { cv = v; cp = ps; }
        }
        uint32_t before = 0;
        for (int j = tid; j < live; j += NT) {
          const uint32_t v = vkey[j];
          before += (v < cv || (v == cv && opos[j] < cp)) ? 1u : 0u;
        }
        before = __reduce_add_sync(0xffffffffu, before);
        if (lane == 0) sc.sel.hist[warp] = before;
        __syncthreads();
        before = 0;
#pragma unroll
        for (int w = 0; w < NT / 32; ++w) before += sc.sel.hist[w];
        done = before < (uint32_t)m;
        __syncthreads();
      }
      if (!done) {
        uint32_t rank, ties;
        group_and_or(k_and, k_or, sc.sel, tid, NT, kMqBarPolicy);
        const uint32_t Tv = radix_select<uint32_t>([&](int j) { return vkey[j]; }, [&](int) { return true; }, live,
                                                   (uint32_t)(m - 1), sc.sel, tid, NT, kMqBarPolicy, &rank, &ties, k_and, k_or);
        int Pv = 0x7fffffff;
        if (ties != rank + 1) {
          uint32_t r2, t2;
          Pv = (int)radix_select<uint32_t>([&](int j) { return (uint32_t)opos[j]; }, [&](int j) { return vkey[j] == Tv; },
                                           live, rank, sc.sel, tid, NT, kMqBarPolicy, &r2, &t2);
        }
        for (int j = tid; j < live; j += NT) {
          const uint32_t v = vkey[j];
          if (!(v < Tv || (v == Tv && (Pv == 0x7fffffff || opos[j] <= Pv)))) mkey[j] = INFINITY;
        }
        __syncthreads();
        ok = lowest_slots<NT>(mbits, opos, live, need, sc);
      }
    }
    if (!ok && tid == 0) {  // only after corrupt statistics: distinct slots all the same
      atomicOr(p.status, ROCO_DEV_BAD_VICTIM);
      for (int e = 0; e < need; ++e) list[e] = e;
    }
    __syncthreads();
    if (tid < need) {  // freed slots in increasing order
      int at = 0;
      for (int x = 0; x < need; ++x) at += list[x] < list[tid] || (list[x] == list[tid] && x < tid);
      tgt[at] = list[tid];
    }
  }
  if (tid >= need && tid < a) tgt[tid] = live + tid - need;
  __syncthreads();
  if (tid < A) {
    const bool freed = tid < need;
    p.ev_slot[(size_t)u * A + tid] = freed ? tgt[tid] : -1;
    if (p.ev_pos) p.ev_pos[(size_t)u * A + tid] = freed ? opos[tgt[tid]] : -1;
  }
  if (tid < a) {  // the thread that reads a freed slot's position is the one that writes the new one
    const size_t at = st + tgt[tid];
    float s = 0.f, q = 0.f;
    for (int i = tid; i < a; ++i) {
      s += pbar[i][tid];
      q = fmaf(pbar[i][tid], pbar[i][tid], q);
    }
    p.s[at] = s;
    p.q[at] = q;
    p.n[at] = a - tid;
    p.pos[at] = t_new + tid;
  }
  if (tid == 0) {
    p.live[u] = live - need + a;
    p.t_next[u] = t_new + a;
  }
  constexpr int kRow = D * (int)sizeof(T) / 16;
  for (int w = tid; w < a * 2 * kRow; w += NT) {
    const int i = w / (2 * kRow), c = w % (2 * kRow);
    const bool isv = c >= kRow;
    const int cc = isv ? c - kRow : c;
    const uint4 x = reinterpret_cast<const uint4 *>(isv ? p.v_new : p.k_new)[((size_t)u * p.T + sh_node[i]) * kRow + cc];
    reinterpret_cast<uint4 *>(isv ? p.V : p.K)[(st + tgt[i]) * kRow + cc] = x;
  }
}

template <typename T, int D, int NT>
roco_status commit_insert_nt(const CommitParams &p, int U, cudaStream_t stream) {
  static SmemLimit limit;
  auto kernel = commit_insert_kernel<T, D, NT>;
  if (!limit((const void *)kernel, 8192 * 8)) return ROCO_ERR_CUDA;
  kernel<<<U, NT, (size_t)p.B * 8, stream>>>(p);
  return cudaGetLastError() == cudaSuccess ? ROCO_OK : ROCO_ERR_CUDA;
}

template <typename T, int D>
roco_status commit_insert_t(const CommitParams &p, int U, cudaStream_t stream) {
  return p.B <= 2048 ? commit_insert_nt<T, D, 256>(p, U, stream) : commit_insert_nt<T, D, 512>(p, U, stream);
}

template <typename T, int D>
roco_status commit_stats_t(const CommitParams &p, int U, int sms, cudaStream_t stream) {
  // keys per CTA: the queries are staged once per CTA, so many keys where the units fill the GPU, few where they do not
  int per = 512;
  while (per > kCsKeys && (long long)U * ((p.B + per - 1) / per) < 8LL * sms) per >>= 1;
  const int blocks = (p.B + per - 1) / per;
  commit_stats_simt_kernel<T, D><<<(unsigned)U * (unsigned)blocks, kCsThreads, 0, stream>>>(p, per, blocks);
  return cudaGetLastError() == cudaSuccess ? ROCO_OK : ROCO_ERR_CUDA;
}

roco_status launch_tree_commit(const CommitParams &p, int kv_dtype, int d, int U, int sms, cudaStream_t stream) {
  roco_status st;
  if (kv_dtype == ROCO_BF16)
    st = launch_commit_stats_tc(p, d, U, sms, stream);
  else
    st = d == 128 ? commit_stats_t<float, 128>(p, U, sms, stream) : commit_stats_t<float, 64>(p, U, sms, stream);
  if (st != ROCO_OK) return st;
  if (kv_dtype == ROCO_BF16)
    return d == 128 ? commit_insert_t<__nv_bfloat16, 128>(p, U, stream) : commit_insert_t<__nv_bfloat16, 64>(p, U, stream);
  return d == 128 ? commit_insert_t<float, 128>(p, U, stream) : commit_insert_t<float, 64>(p, U, stream);
}

}  // namespace roco
