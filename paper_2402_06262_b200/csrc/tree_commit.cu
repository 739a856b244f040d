// Commit of the accepted path of a draft tree: the statistics of Sec. 4.3 for the accepted queries over the cached
// tokens (CUDA-core kernel; tensor-core kernel in tree_commit_tc.cu), then per unit the evictions on the updated
// statistics and the insertion of the accepted tokens.
#include "tree_insert.cuh"

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
  launch_dependents();
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

// What bounds a unit is its chain of dependent loads and of passes over shared memory.  The launch starts while the
// statistics are still being formed, and what does not need them comes first: the path, the accepted rows, what the accepted
// tokens start with.
template <typename T, int D, int NT>
__global__ void __launch_bounds__(NT) commit_insert_kernel(const CommitParams p) {
  extern __shared__ __align__(16) char ci_smem[];  // keys and values of the accepted tokens [2][A][D], then the slots' keys
  __shared__ CiScratch sc;
  __shared__ int tgt[kCiMaxA], tgt_pos[kCiMaxA], sh_node[32], sh_a;
  __shared__ float pbar[kCiMaxA][kCiMaxA];
  constexpr int kRow = D * (int)sizeof(T) / 16;
  const int tid = threadIdx.x, u = blockIdx.x, b = u / p.G, A = p.A, B = p.B;
  const int live = tree_live(p.live, u, B, p.status, false), t_new = p.t_next[u];
  if (tid < 32) {
    int node;
    const int a = commit_path(p, b, tid, node, false);
    sh_node[tid] = node;
    if (tid == 0) sh_a = a;
  }
  __syncthreads();
  const int a = sh_a;
  uint4 *rows = reinterpret_cast<uint4 *>(ci_smem);
  for (int w = tid; w < a * 2 * kRow; w += NT) {
    const int isv = w >= a * kRow, x = w - isv * a * kRow;
    rows[isv * A * kRow + x] =
        reinterpret_cast<const uint4 *>(isv ? p.v_new : p.k_new)[((size_t)u * p.T + sh_node[x / kRow]) * kRow + x % kRow];
  }
  __syncthreads();
  commit_new_probabilities<T, D>(p, u, a, sh_node, reinterpret_cast<const T *>(ci_smem), tid >> 5, NT / 32, tid & 31, pbar);
  wait_for_launch_before();
  if (a == 0) {
    if (tid < A) {
      p.ev_slot[(size_t)u * A + tid] = -1;
      if (p.ev_pos) p.ev_pos[(size_t)u * A + tid] = -1;
    }
    return;
  }
  const int need = live + a - B > 0 ? live + a - B : 0;
  char *keys = ci_smem + (size_t)2 * A * kRow * 16;
  uint32_t k_and = 0xffffffffu, k_or = 0u;
  if (need > 0) commit_keys<NT>(p, u, live, keys, k_and, k_or);
  commit_slots<NT>(p, u, a, live, need, keys, k_and, k_or, sc, tgt, tgt_pos);
  __syncthreads();
  if (tid < A) {
    p.ev_slot[(size_t)u * A + tid] = tid < need ? tgt[tid] : -1;
    if (p.ev_pos) p.ev_pos[(size_t)u * A + tid] = tid < need ? tgt_pos[tid] : -1;
  }
  const size_t st = (size_t)u * B;
  if (tid < a) {
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
  for (int w = tid; w < a * 2 * kRow; w += NT) {
    const int isv = w >= a * kRow, x = w - isv * a * kRow;
    reinterpret_cast<uint4 *>(isv ? p.V : p.K)[(st + tgt[x / kRow]) * kRow + x % kRow] = rows[isv * A * kRow + x];
  }
}

template <typename T, int D, int NT>
roco_status commit_insert_nt(const CommitParams &p, int U, cudaStream_t stream) {
  static SmemLimit limit;
  auto kernel = commit_insert_kernel<T, D, NT>;
  if (!limit((const void *)kernel, 8192 * 8 + 2 * kCiMaxA * D * sizeof(T))) return ROCO_ERR_CUDA;
  const size_t smem = (size_t)p.B * 8 + (size_t)2 * p.A * D * sizeof(T);
  return launch_overlapped(kernel, U, NT, smem, stream, p) ? ROCO_OK : ROCO_ERR_CUDA;
}

// A unit is a chain of passes and loads: with few units more threads shorten the passes, with many it is the number of
// units in flight that counts.  Whole commits with 128, 256 and 512 threads: 8192 units x 1024 tokens 470, 499, 642 us (every unit
// evicts five); 1184 units 80, 83, 101; 600 units 52, 47, 60; 300 units x 4096 80, 75, 80; 148 units x 1024 20.6, 18.6, 16.7; 32 units
// x 512 12.5, 11.8, 11.3, x 1024 15.8, 14.1, 13.5, x 8192 41, 30, 23; and x 256 tokens, d = 64, with 256 and 512 11.3, 11.9.
template <typename T, int D>
roco_status commit_insert_t(const CommitParams &p, int U, int sms, cudaStream_t stream) {
  if (U >= 8 * sms) return commit_insert_nt<T, D, 128>(p, U, stream);
  return U > sms || p.B < 512 ? commit_insert_nt<T, D, 256>(p, U, stream) : commit_insert_nt<T, D, 512>(p, U, stream);
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
    return d == 128 ? commit_insert_t<__nv_bfloat16, 128>(p, U, sms, stream) : commit_insert_t<__nv_bfloat16, 64>(p, U, sms, stream);
  return d == 128 ? commit_insert_t<float, 128>(p, U, sms, stream) : commit_insert_t<float, 64>(p, U, sms, stream);
}

}  // namespace roco
