// Statistics of the accepted queries over the cached tokens on the fifth-generation tensor cores (bf16).
//
// S^T[128 keys x N rows] = K_tile Q^T with the key index on the accumulator's lanes: a thread finds all accepted queries'
// scores of its key side by side, so p_ij = 2^(x_ij - lse_i), the mean over a token's heads and the two sums over the
// tokens stay inside the thread; no maximum, no reduction.  Bound by the stream of the keys (each read once, 256 bytes
// at d = 128, beside 24 bytes of statistics): 8192 units x 1024 tokens 322 us, 0.98 of the measured copy rate.
#include <cuda.h>

#include "tc.cuh"
#include "tree.cuh"

namespace roco {

constexpr int kCtTile = 128;
constexpr int kCtThreads = 192;  // four warps of keys, one of loads, one of products
constexpr int kCtTmaWarp = 4, kCtMmaWarp = 5;

template <int D, int N>
struct CtShape {
  static constexpr int kTile = kCtTile * D * 2, kBlock = kCtTile * 128, kQ = N * D * 2;
  // three CTAs per SM while the queries are few, else two (one for the widest)
  static constexpr int kCtas = N * D <= 16 * 128 ? 3 : (N <= 128 ? 2 : 1);
  static constexpr int kRoom = 227 * 1024 / kCtas - 2048 - kQ - N * 4 - 1024;
  static constexpr int kStages = kRoom / kTile > 6 ? 6 : kRoom / kTile;
  static constexpr int kTmemCols = 2 * N < 32 ? 32 : 2 * N;
  static constexpr size_t kSmem = 1024 + (size_t)kStages * kTile + kQ + N * 4 + (2 * kStages + 4) * 8 + 64 * 4 + 32;
  static_assert(kStages >= 2, "shared memory");
};

template <int D, int N>
__global__ void __launch_bounds__(kCtThreads, (CtShape<D, N>::kCtas))
    commit_stats_tc_kernel(const __grid_constant__ CUtensorMap mapK, const CommitParams p, int tiles_per_cta, int key_blocks) {
  using Sh = CtShape<D, N>;
  constexpr int kTile = Sh::kTile, kBlock = Sh::kBlock, kStages = Sh::kStages;
  constexpr uint32_t kIdesc = (1u << 4) | (1u << 7) | (1u << 10) | (8u << 24) | (((uint32_t)N >> 3) << 17);
  extern __shared__ char ct_raw[];
  launch_dependents();
  char *at = smem_align(ct_raw, 1024);
  char *ring = at; at += kStages * kTile;
  char *qop = at; at += Sh::kQ;
  float *nlse = reinterpret_cast<float *>(at); at += N * 4;     // minus the log-sum-exp of a row, log2 domain
  uint32_t *ends = reinterpret_cast<uint32_t *>(at); at += 32 * 4;  // per 16 columns: those that are a token's last head
  int *sh_node = reinterpret_cast<int *>(at); at += 32 * 4;
  uint64_t *full = reinterpret_cast<uint64_t *>(at), *empty = full + kStages, *s_full = empty + kStages, *s_free = s_full + 2;
  at += (2 * kStages + 4) * 8;
  uint32_t *tmem_base = reinterpret_cast<uint32_t *>(at);
  int *abort_ptr = reinterpret_cast<int *>(at + 8);
  volatile int *abort_flag = abort_ptr;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int u = blockIdx.x / key_blocks, kb = blockIdx.x % key_blocks, b = u / p.G;
  int node;
  const int a = __shfl_sync(0xffffffffu, commit_path(p, b, lane, node, kb == 0 && warp == 0), 0);
  if (a == 0) return;
  const int live = __shfl_sync(0xffffffffu, tree_live(p.live, u, p.B, p.status, tid == 0 && kb == 0), 0);
  const int tiles = (live + kCtTile - 1) / kCtTile, t0 = kb * tiles_per_cta;
  const int nt = tiles - t0 < tiles_per_cta ? tiles - t0 : tiles_per_cta;
  if (nt <= 0) return;
  const int rows = a * p.group;

  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&s_full[i], 1); mbar_init(&s_free[i], 4); }
    *abort_ptr = 0;
    mbar_init_fence();
  }
  if (warp == 0) {
    tmem_alloc(tmem_base, Sh::kTmemCols);
    tmem_relinquish();
    sh_node[lane] = node;
  }
  __syncthreads();
  // the accepted queries, gathered along the path, as the K-major operand; rows that do not exist are zero
  const uint4 *Qu = reinterpret_cast<const uint4 *>(p.Q) + (size_t)u * p.T * p.group * (D / 8);
  for (int w = tid; w < N * D / 8; w += kCtThreads) {
    const int i = w / (D / 8), c = w % (D / 8);
    uint4 x = make_uint4(0u, 0u, 0u, 0u);
    if (i < rows) x = Qu[(size_t)(sh_node[i / p.group] * p.group + i % p.group) * (D / 8) + c];
    *reinterpret_cast<uint4 *>(qop + (c >> 3) * (N * 128) + i * 128 + (((c & 7) ^ (i & 7)) << 4)) = x;
  }
  fence_async_smem();
  for (int i = tid; i < N; i += kCtThreads)
    nlse[i] = i < rows ? -p.lse[((size_t)u * p.T + sh_node[i / p.group]) * p.group + i % p.group] * kLog2e : -INFINITY;
  if (tid < N / 16) {
    uint32_t m = 0;
    for (int i = 0; i < 16; ++i)
      if ((16 * tid + i + 1) % p.group == 0) m |= 1u << i;
    ends[tid] = m;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_base, 0);

  if (warp == kCtTmaWarp) {
    if (lane == 0) {
      for (int t = 0; t < nt; ++t) {
        const int st = t % kStages;
        if (t >= kStages) mbar_wait_compact(&empty[st], (t / kStages - 1) & 1, abort_flag, p.status);
        mbar_expect_tx(&full[st], kTile);
#pragma unroll
        for (int h = 0; h < D / 64; ++h)
          tma_load_3d(ring + st * kTile + h * kBlock, &mapK, 64 * h, (t0 + t) * kCtTile, u, &full[st]);
      }
    }
  } else if (warp == kCtMmaWarp) {
    for (int t = 0; t < nt; ++t) {
      const int st = t % kStages;
      if (t >= 2) mbar_wait_compact(&s_free[t & 1], ((t >> 1) - 1) & 1, abort_flag, p.status);
      mbar_wait_compact(&full[st], (t / kStages) & 1, abort_flag, p.status);
      tc_fence_after();
      const char *k = ring + st * kTile;
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
        umma_bf16_w(tmem + (t & 1) * N, smem_desc_sw128(k + (kk / 4) * kBlock + (kk % 4) * 32),
                    smem_desc_sw128(qop + (kk / 4) * (N * 128) + (kk % 4) * 32), kIdesc, kk > 0 ? 1u : 0u);
      umma_commit_w(&s_full[t & 1]);
      umma_commit_w(&empty[st]);
    }
  } else {
    const float zs = p.scale * kLog2e, inv_group = 1.f / (float)p.group;
    const uint32_t tl = tmem + ((uint32_t)(warp * 32) << 16);
#pragma unroll 1
    for (int t = 0; t < nt; ++t) {
      const int j = (t0 + t) * kCtTile + tid;
      const size_t at_j = (size_t)u * p.B + j;
      float s = 0.f, q = 0.f;
      int n = 0;
      if (j < live) { s = p.s[at_j]; q = p.q[at_j]; n = p.n[at_j]; }  // on their way while the scores are formed
      mbar_wait_compact(&s_full[t & 1], (t >> 1) & 1, abort_flag, p.status);
      tc_fence_after();
      float ds = 0.f, dq = 0.f, pb = 0.f;
#pragma unroll 1
      for (int x = 0; x < rows; x += 16) {
        uint32_t r[16];
        tmem_ld16(tl + (t & 1) * N + x, r);
        const uint32_t m = ends[x >> 4];
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const float4 n4 = *reinterpret_cast<const float4 *>(nlse + x + i);  // (-inf, probability 0, behind the last row)
          const float e[4] = {n4.x, n4.y, n4.z, n4.w};
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            pb += ex2_approx(fmaf(__uint_as_float(r[i + h]), zs, e[h]));
            if ((m >> (i + h)) & 1u) {  // the token's heads are together
              pb *= inv_group;
              ds += pb;
              dq = fmaf(pb, pb, dq);
              pb = 0.f;
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s_free[t & 1]);
      if (j < live) {
        p.s[at_j] = s + ds;
        p.q[at_j] = q + dq;
        p.n[at_j] = n + a;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, Sh::kTmemCols);
}

template <int D, int N>
roco_status commit_stats_tc_t(const CommitParams &p, int U, int sms, cudaStream_t stream) {
  CUtensorMap mk;
  if (!make_tensor_map_units_bf16(&mk, p.K, U, p.B, D, kCtTile)) return ROCO_ERR_CUDA;
  constexpr size_t smem = CtShape<D, N>::kSmem;
  // a unit's keys in one CTA (the queries are gathered once) unless that leaves SMs without work
  const int tiles = (p.B + kCtTile - 1) / kCtTile;
  const long long slots = (long long)CtShape<D, N>::kCtas * sms;
  int blocks = (int)(slots / U);
  blocks = blocks < 1 ? 1 : (blocks > tiles ? tiles : blocks);
  const int per = (tiles + blocks - 1) / blocks;
  blocks = (tiles + per - 1) / per;
  auto kernel = commit_stats_tc_kernel<D, N>;
  static SmemLimit limit;
  if (!limit((const void *)kernel, smem)) return ROCO_ERR_CUDA;
  kernel<<<(unsigned)U * (unsigned)blocks, kCtThreads, smem, stream>>>(mk, p, per, blocks);
  return cudaGetLastError() == cudaSuccess ? ROCO_OK : ROCO_ERR_CUDA;
}

template <int D>
roco_status commit_stats_tc_d(const CommitParams &p, int U, int sms, cudaStream_t stream) {
  const int rows = p.A * p.group;
  if (rows <= 16) return commit_stats_tc_t<D, 16>(p, U, sms, stream);
  if (rows <= 32) return commit_stats_tc_t<D, 32>(p, U, sms, stream);
  if (rows <= 64) return commit_stats_tc_t<D, 64>(p, U, sms, stream);
  if (rows <= 128) return commit_stats_tc_t<D, 128>(p, U, sms, stream);
  return commit_stats_tc_t<D, 256>(p, U, sms, stream);
}

roco_status launch_commit_stats_tc(const CommitParams &p, int d, int U, int sms, cudaStream_t stream) {
  return d == 128 ? commit_stats_tc_d<128>(p, U, sms, stream) : commit_stats_tc_d<64>(p, U, sms, stream);
}

}  // namespace roco
