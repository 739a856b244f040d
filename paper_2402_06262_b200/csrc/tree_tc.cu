// Attention of a tree of drafted tokens over the cache on the fifth-generation tensor cores (bf16, positive scale).
//
// The query rows of a unit (heads x nodes, a few dozen) cannot fill the 128 rows of a tensor-core tile, the cached keys
// can: the key index lies on the accumulator's lanes and the N = 16, 32 or 64 query rows of a CTA are its columns.
//     S^T[128 keys x N] = K_tile Q^T          O^T[d x N] += V_tile^T P^T
// One pass over the cache.  A thread owns one key of a tile: it forms p = 2^(z - m) for its N scores, keeps N partial sums
// of its own in registers (joined over the lanes once, at the end) and writes the N probabilities as bf16, the second
// product's operand.  The reference m of a row is the maximum of its first tile and moves only when a score comes out
// more than 2^8 above it (one vote per tile instead of a maximum over the lanes; up to there fp32 sums and bf16
// probabilities lose nothing): then the row's column of O^T and its sums are rescaled.
// The drafted tokens are the last tile's keys, masked by the rows' ancestor sets; their values are added on the CUDA cores
// with fp32 probabilities, node by node where a row sees the node, so that what lies on other branches cannot reach it.
//
// What bounds it: the cache is read once; 64 KiB per tile of 128 tokens at d = 128 against about 700 cycles of
// exponentials for N = 64.  Two CTAs per SM, so that one's prologue and epilogue run under the other's stream.
#include <cuda.h>

#include "tc.cuh"
#include "tree.cuh"

namespace roco {

constexpr int kTtTile = 128;  // keys of a tile
constexpr int kTtConsumers = 128;
constexpr int kTtTmaWarp = 4, kTtMmaWarp = 5;
constexpr int kTtThreads = 192;
constexpr int kTtBar = 1;                // named barrier of the consumers
constexpr float kTtMoveReference = 8.f;  // binary orders

template <int D, int N>
struct TtShape {
  static constexpr int kTile = kTtTile * D * 2, kBlock = kTtTile * 128;
  static constexpr int kQ = N * D * 2;
  static constexpr int kP = N * kTtTile * 2;         // P^T of a tile: 128-byte rows of 64 / N keys each
  static constexpr int kPRows = kP / 128;
  static constexpr int kPBufs = N == 64 ? 1 : 2;
  // what two CTAs can have beside each other on an SM
  static constexpr int kRoom = 113 * 1024 - 1024 - kQ - kP * kPBufs - 4096 - N * 16;
  static constexpr int kStages = kRoom / kTile > 6 ? 6 : kRoom / kTile;
  static constexpr int kTmemCols = 4 * N < 32 ? 32 : 4 * N;  // S^T twice, O^T; a power of two
  static constexpr size_t kSmem = 1024 + (size_t)kStages * kTile + kQ + kP * kPBufs + 4 * N * 4 /* red */ + 2 * N * 4 /* mref, alpha */ +
                                  kTreeMaxNodes * 12 + N * 8 + (2 * kStages + 8) * 8 + 32;
  static_assert(kStages >= 2 && kSmem <= 113 * 1024, "two CTAs per SM");
  // the drafted tokens' probabilities [nodes][N] lie in the ring once the stream is over
  static_assert(kTreeMaxNodes * N * 4 <= kTile, "draft probabilities");
};

// v[i] reduced over the 32 lanes; lane l gets column l >> 1.  The exchange halves the live values at every step.
template <bool kMax>
__device__ __forceinline__ float tt_lanes_reduce(float (&v)[16], int lane) {
#pragma unroll
  for (int step = 0; step < 4; ++step) {
    const int w = 8 >> step, o = 16 >> step;
    const bool up = (lane & o) != 0;
#pragma unroll
    for (int k = 0; k < w; ++k) {
      const float send = up ? v[k] : v[k + w], keep = up ? v[k + w] : v[k];
      const float got = __shfl_xor_sync(0xffffffffu, send, o);
      v[k] = kMax ? fmaxf(keep, got) : keep + got;
    }
  }
  const float got = __shfl_xor_sync(0xffffffffu, v[0], 1);
  return kMax ? fmaxf(v[0], got) : v[0] + got;
}

__device__ __forceinline__ bool tt_any(bool x) {  // over the consumer threads
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"((uint32_t)x), "n"(kTtBar), "n"(kTtConsumers)
      : "memory");
  return r != 0;
}

__device__ __forceinline__ uint32_t tt_pack(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t *>(&v);
}

template <int D, int N>
__global__ void __launch_bounds__(kTtThreads, 2)
    tree_tc_kernel(const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV,
                   const __grid_constant__ CUtensorMap mapKn, const TreeParams p) {
  using Sh = TtShape<D, N>;
  constexpr int kTile = Sh::kTile, kBlock = Sh::kBlock, kStages = Sh::kStages;
  constexpr uint32_t kIdescS = (1u << 4) | (1u << 7) | (1u << 10) | (8u << 24) | (((uint32_t)N >> 3) << 17);
  constexpr uint32_t kIdescO = kIdescS | (1u << 15) | (1u << 16);  // both operands with the M / N index contiguous
  extern __shared__ char tt_raw[];
  launch_dependents();
  char *at = smem_align(tt_raw, 1024);
  char *ring = at; at += kStages * kTile;
  char *pbuf = at; at += Sh::kP * Sh::kPBufs;
  char *qop = at; at += Sh::kQ;
  float *red = reinterpret_cast<float *>(at); at += 4 * N * 4;
  float *nref = reinterpret_cast<float *>(at); at += N * 4;   // minus the reference of a row, log2 domain
  float *alpha = reinterpret_cast<float *>(at); at += N * 4;
  unsigned long long *anc = reinterpret_cast<unsigned long long *>(at); at += kTreeMaxNodes * 8;
  unsigned long long *sees = reinterpret_cast<unsigned long long *>(at); at += N * 8;  // per query row: the nodes it sees
  int *up = reinterpret_cast<int *>(at); at += kTreeMaxNodes * 4;
  uint64_t *full = reinterpret_cast<uint64_t *>(at), *empty = full + kStages, *s_full = empty + kStages, *p_ready = s_full + 2;
  uint64_t *pv_done = p_ready + 2;
  at += (2 * kStages + 8) * 8;
  uint32_t *tmem_base = reinterpret_cast<uint32_t *>(at);
  int *abort_ptr = reinterpret_cast<int *>(at + 8);
  volatile int *abort_flag = abort_ptr;
  float *pd = reinterpret_cast<float *>(ring);  // [node][N], after the stream

  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int row_blocks = (p.rows + N - 1) / N;
  const int rb = blockIdx.x % row_blocks, split = blockIdx.x / row_blocks % p.splits, u = blockIdx.x / (row_blocks * p.splits);
  const int b = u / p.G, row0 = rb * N;
  const bool report = tid == 0 && rb == 0 && split == 0;
  const int n_nodes = __shfl_sync(0xffffffffu, tree_nodes(p, b, report), 0);
  if (row0 >= n_nodes * p.group) return;
  const int live = __shfl_sync(0xffffffffu, tree_live(p.live, u, p.B, p.status, report), 0);
  const int tiles = (live + kTtTile - 1) / kTtTile;
  const int t0 = (int)((long long)tiles * split / p.splits);
  const int nt = (int)((long long)tiles * (split + 1) / p.splits) - t0;  // cached tiles of this CTA
  const bool drafts = split == p.splits - 1;
  const int ns = nt + (drafts ? 1 : 0);  // score tiles

  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&s_full[i], 1); mbar_init(&p_ready[i], 4); mbar_init(&pv_done[i], 1); }
    *abort_ptr = 0;
    mbar_init_fence();
  }
  if (warp == 0) {
    tmem_alloc(tmem_base, Sh::kTmemCols);
    tmem_relinquish();
  }
  if (tid < kTtConsumers) {  // the queries as the K-major operand; rows that do not exist are zero
    const uint4 *Qu = reinterpret_cast<const uint4 *>(p.Q) + ((size_t)u * p.rows + row0) * (D / 8);
#pragma unroll
    for (int w = tid; w < N * D / 8; w += kTtConsumers) {
      const int i = w / (D / 8), c = w % (D / 8);
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if (row0 + i < n_nodes * p.group) x = Qu[w];
      *reinterpret_cast<uint4 *>(qop + (c >> 3) * (N * 128) + i * 128 + (((c & 7) ^ (i & 7)) << 4)) = x;
    }
    fence_async_smem();
  }
  tc_fence_before();
  if (drafts) {
    tree_ancestors(p, b, n_nodes, anc, up, rb == 0);  // (synchronises)
    if (tid < N) sees[tid] = row0 + tid < n_nodes * p.group ? anc[(row0 + tid) / p.group] : 0ull;
  }
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_base, 0);
  const uint32_t tmem_o = tmem + 2 * N;

  if (warp == kTtTmaWarp) {
    if (lane == 0) {
      const int items = 2 * nt + (drafts ? 1 : 0);  // K, V, K, V, ..., the drafted keys
      for (int g = 0; g < items; ++g) {
        const int st = g % kStages;
        if (g >= kStages) mbar_wait_compact(&empty[st], (g / kStages - 1) & 1, abort_flag, p.status);
        const CUtensorMap *map = g == 2 * nt ? &mapKn : ((g & 1) ? &mapV : &mapK);
        const int row = g == 2 * nt ? 0 : (t0 + (g >> 1)) * kTtTile;
        mbar_expect_tx(&full[st], kTile);
#pragma unroll
        for (int h = 0; h < D / 64; ++h) tma_load_3d(ring + st * kTile + h * kBlock, map, 64 * h, row, u, &full[st]);
      }
    }
  } else if (warp == kTtMmaWarp) {
    for (int t = 0; t <= ns; ++t) {
      if (t < ns) {  // scores of tile t; what its accumulator held was read before p_ready of two tiles ago
        const int g = 2 * t, st = g % kStages;
        mbar_wait_compact(&full[st], (g / kStages) & 1, abort_flag, p.status);
        tc_fence_after();
        const char *k = ring + st * kTile;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          umma_bf16_w(tmem + (t & 1) * N, smem_desc_sw128(k + (kk / 4) * kBlock + (kk % 4) * 32),
                      smem_desc_sw128(qop + (kk / 4) * (N * 128) + (kk % 4) * 32), kIdescS, kk > 0 ? 1u : 0u);
        umma_commit_w(&s_full[t & 1]);
        umma_commit_w(&empty[st]);
      }
      if (t >= 1 && t <= nt) {  // output of tile t - 1
        const int g = 2 * t - 1, st = g % kStages, tv = t - 1;
        mbar_wait_compact(&p_ready[tv & 1], (tv >> 1) & 1, abort_flag, p.status);
        mbar_wait_compact(&full[st], (g / kStages) & 1, abort_flag, p.status);
        char *v = ring + st * kTile;
        const int first_bad = live - (t0 + tv) * kTtTile;
        if (first_bad < kTtTile) {  // slots behind the last token may hold anything (0 x NaN)
          for (int w = lane; w < (kTtTile - first_bad) * 8; w += 32) {
#pragma unroll
            for (int h = 0; h < D / 64; ++h)
              *reinterpret_cast<uint4 *>(v + h * kBlock + first_bad * 128 + w * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
          fence_async_smem();
          __syncwarp();
        }
        tc_fence_after();
        const char *pb = pbuf + (tv % Sh::kPBufs) * Sh::kP;
#pragma unroll
        for (int kk = 0; kk < 8; ++kk)  // (d = 64: the upper 64 accumulator lanes repeat the lower, unread)
          umma_bf16_w(tmem_o, smem_desc_sw128_mn(v + kk * 2048, D == 128 ? kBlock : 0),
                      smem_desc_sw128_mn(pb + (16 * kk % Sh::kPRows) * 128 + (16 * kk / Sh::kPRows) * (N * 2), 16), kIdescO,
                      (tv > 0 || kk > 0) ? 1u : 0u);
        umma_commit_w(&pv_done[tv & 1]);
        umma_commit_w(&empty[st]);
      }
    }
  } else {
    // ---------------------------------------------------------------- consumers: a key per lane
    const float zs = p.scale * kLog2e;
    const uint32_t tl = tmem + ((uint32_t)(warp * 32) << 16);
    const int prow = tid % Sh::kPRows, pc0 = tid / Sh::kPRows * (N / 8);
    float l[N];
#pragma unroll
    for (int i = 0; i < N; ++i) l[i] = 0.f;
    // The output product of tile t is complete.  One barrier per tile parity: this thread is never two phases of either
    // behind, since the product of tile t + 2 waits for its own probabilities of that tile.
    auto wait_pv = [&](int t) {
      if (t >= 0) mbar_wait_compact(&pv_done[t & 1], (t >> 1) & 1, abort_flag, p.status);
    };
#pragma unroll 1
    for (int t = 0; t < ns; ++t) {
      const bool is_draft = t == nt;
      const bool held = is_draft ? tid < n_nodes : (t0 + t) * kTtTile + tid < live;
      const uint32_t ts = tl + (t & 1) * N;
      mbar_wait_compact(&s_full[t & 1], (t >> 1) & 1, abort_flag, p.status);
      tc_fence_after();
      // which of the columns x .. x + 15 this key takes part in
      auto seen = [&](int x) -> uint32_t {
        if (!held) return 0u;
        if (!is_draft) return 0xffffu;
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          if ((sees[x + i] >> tid) & 1ull) m |= 1u << i;
        }
        return m;
      };
      bool move = t == 0;
      if (t > 0) {
        float top = -INFINITY;
#pragma unroll
        for (int x = 0; x < N; x += 16) {
          uint32_t r[16];
          tmem_ld16(ts + x, r);
          const uint32_t m = seen(x);
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            const float4 n4 = *reinterpret_cast<const float4 *>(nref + x + i);
            const float d0 = fmaf(__uint_as_float(r[i]), zs, n4.x), d1 = fmaf(__uint_as_float(r[i + 1]), zs, n4.y);
            const float d2 = fmaf(__uint_as_float(r[i + 2]), zs, n4.z), d3 = fmaf(__uint_as_float(r[i + 3]), zs, n4.w);
            if (is_draft) {
              top = fmaxf(top, fmaxf(fmaxf((m >> i) & 1u ? d0 : -INFINITY, (m >> (i + 1)) & 1u ? d1 : -INFINITY),
                                     fmaxf((m >> (i + 2)) & 1u ? d2 : -INFINITY, (m >> (i + 3)) & 1u ? d3 : -INFINITY)));
            } else {
              top = max3(max3(top, d0, d1), d2, d3);
            }
          }
        }
        move = held && top > kTtMoveReference;
      }
      if (tt_any(move)) {
        // new references: the tile's maxima where they are larger
#pragma unroll 1
        for (int x = 0; x < N; x += 16) {
          uint32_t r[16];
          float v[16];
          tmem_ld16(ts + x, r);
          const uint32_t m = seen(x);
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = (m >> i) & 1u ? __uint_as_float(r[i]) * zs : -INFINITY;
          const float top = tt_lanes_reduce<true>(v, lane);
          if ((lane & 1) == 0) red[warp * N + x + (lane >> 1)] = top;
        }
        named_bar_sync(kTtBar, kTtConsumers);
        if (tid < N) {
          const float top = fmaxf(fmaxf(red[tid], red[N + tid]), fmaxf(red[2 * N + tid], red[3 * N + tid]));
          const float old = t == 0 ? -INFINITY : -nref[tid];
          float ref = fmaxf(old, top);
          if (ref == -INFINITY) ref = 0.f;  // a row that does not exist sees nothing
          alpha[tid] = t == 0 ? 0.f : exp2f(old - ref);
          nref[tid] = -ref;
        }
        wait_pv(t - 1);  // nothing adds to O^T now
        tc_fence_after();
        named_bar_sync(kTtBar, kTtConsumers);
#pragma unroll
        for (int x = 0; x < N; x += 16) {
          uint32_t r[16];
          if (t > 0) tmem_ld16(tl + 2 * N + x, r);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float f = alpha[x + i];
            l[x + i] *= f;
            r[i] = __float_as_uint(__uint_as_float(r[i]) * f);
          }
          if (t > 0) tmem_st16(tl + 2 * N + x, r);
        }
        tmem_st_wait();
      }
      if (is_draft) {
        // (every product of the stream has been issued by now, and the ring is free once they are done)
        wait_pv(nt - 1);
      } else {
        wait_pv(t - Sh::kPBufs);  // the operand's place is free
      }
      char *prow_p = pbuf + (t % Sh::kPBufs) * Sh::kP + prow * 128;
#pragma unroll
      for (int x = 0; x < N; x += 16) {
        uint32_t r[16];
        tmem_ld16(ts + x, r);
        const uint32_t m = is_draft ? seen(x) : 0u;
        float e[16];
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const float4 n4 = *reinterpret_cast<const float4 *>(nref + x + i);
          e[i] = ex2_approx(fmaf(__uint_as_float(r[i]), zs, n4.x));
          e[i + 1] = ex2_approx(fmaf(__uint_as_float(r[i + 1]), zs, n4.y));
          e[i + 2] = ex2_approx(fmaf(__uint_as_float(r[i + 2]), zs, n4.z));
          e[i + 3] = ex2_approx(fmaf(__uint_as_float(r[i + 3]), zs, n4.w));
        }
        if (is_draft) {
#pragma unroll
          for (int i = 0; i < 16; ++i) e[i] = (m >> i) & 1u ? e[i] : 0.f;
          if (tid < kTreeMaxNodes) {
#pragma unroll
            for (int i = 0; i < 16; i += 4)
              *reinterpret_cast<float4 *>(pd + tid * N + x + i) = make_float4(e[i], e[i + 1], e[i + 2], e[i + 3]);
          }
        } else {
          if (!held) {
#pragma unroll
            for (int i = 0; i < 16; ++i) e[i] = 0.f;
          }
#pragma unroll
          for (int h = 0; h < 2; ++h)
            *reinterpret_cast<uint4 *>(prow_p + (((pc0 + x / 8 + h) ^ (prow & 7)) << 4)) =
                make_uint4(tt_pack(e[8 * h], e[8 * h + 1]), tt_pack(e[8 * h + 2], e[8 * h + 3]),
                           tt_pack(e[8 * h + 4], e[8 * h + 5]), tt_pack(e[8 * h + 6], e[8 * h + 7]));
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) l[x + i] += e[i];
      }
      if (!is_draft) {
        fence_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_ready[t & 1]);
      }
    }
    // ---------------------------------------------------------------- the sums over the lanes, then a dimension per lane
    wait_pv(nt - 1);
    tc_fence_after();
    named_bar_sync(kTtBar, kTtConsumers);  // red is free, pd complete
#pragma unroll
    for (int x = 0; x < N; x += 16) {
      float v[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = l[x + i];
      const float sum = tt_lanes_reduce<false>(v, lane);
      if ((lane & 1) == 0) red[warp * N + x + (lane >> 1)] = sum;
    }
    named_bar_sync(kTtBar, kTtConsumers);
    const int rows = n_nodes * p.group - row0 < N ? n_nodes * p.group - row0 : N;
    if (tid < N) {
      const float sum = (red[tid] + red[N + tid]) + (red[2 * N + tid] + red[3 * N + tid]);
      alpha[tid] = p.splits > 1 ? 1.f : 1.f / sum;
      if (tid < rows) {
        const float ref = ns > 0 ? -nref[tid] : -INFINITY;
        if (p.splits > 1) {
          const size_t pt = ((size_t)u * p.splits + split) * p.rows + row0 + tid;
          *reinterpret_cast<float2 *>(p.part_ml + 2 * pt) = make_float2(ref, sum);
        } else if (p.lse) {
          p.lse[(size_t)u * p.rows + row0 + tid] = (ref + log2f(sum)) * kLn2;
        }
      }
    }
    named_bar_sync(kTtBar, kTtConsumers);
    if (warp * 32 < D) {
      const __nv_bfloat16 *vn = reinterpret_cast<const __nv_bfloat16 *>(p.v_new) + (size_t)u * p.T * D + tid;
#pragma unroll 1
      for (int x = 0; x < rows; x += 16) {
        float o[16];
        if (nt > 0) {
          uint32_t r[16];
          tmem_ld16(tl + 2 * N + x, r);
#pragma unroll
          for (int i = 0; i < 16; ++i) o[i] = __uint_as_float(r[i]);
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) o[i] = 0.f;
        }
        if (drafts) {
#pragma unroll 4
          for (int j = 0; j < n_nodes; ++j) {
            const float v = __bfloat162float(vn[(size_t)j * D]);
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
              const float4 e = *reinterpret_cast<const float4 *>(pd + j * N + x + i);
              if (e.x != 0.f) o[i] = fmaf(e.x, v, o[i]);
              if (e.y != 0.f) o[i + 1] = fmaf(e.y, v, o[i + 1]);
              if (e.z != 0.f) o[i + 2] = fmaf(e.z, v, o[i + 2]);
              if (e.w != 0.f) o[i + 3] = fmaf(e.w, v, o[i + 3]);
            }
          }
        }
        if (p.splits > 1) {
          float *dst = p.part_o + (((size_t)u * p.splits + split) * p.rows + row0 + x) * D + tid;
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (x + i < rows) dst[(size_t)i * D] = o[i];
        } else {
          __nv_bfloat16 *dst = reinterpret_cast<__nv_bfloat16 *>(p.out) + ((size_t)u * p.rows + row0 + x) * D + tid;
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (x + i < rows) dst[(size_t)i * D] = __float2bfloat16_rn(o[i] * alpha[x + i]);
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, Sh::kTmemCols);
}

// Query rows of a CTA: the smallest width that takes a unit's rows, 64 at most (the rest goes to further CTAs, which find
// the cache in L2).
int tree_tc_width(int rows) { return rows <= 16 ? 16 : (rows <= 32 ? 32 : 64); }

template <int D, int N>
roco_status tree_tc_t(const TreeParams &p, int U, cudaStream_t stream) {
  CUtensorMap mk, mv, mn;
  if (!make_tensor_map_units_bf16(&mk, p.K, U, p.B, D, kTtTile) || !make_tensor_map_units_bf16(&mv, p.V, U, p.B, D, kTtTile) ||
      !make_tensor_map_units_bf16(&mn, p.k_new, U, p.T, D, kTtTile))
    return ROCO_ERR_CUDA;
  auto kernel = tree_tc_kernel<D, N>;
  constexpr size_t smem = TtShape<D, N>::kSmem;
  static SmemLimit limit;
  if (!limit((const void *)kernel, smem)) return ROCO_ERR_CUDA;
  kernel<<<(unsigned)U * (unsigned)((p.rows + N - 1) / N) * (unsigned)p.splits, kTtThreads, smem, stream>>>(mk, mv, mn, p);
  if (cudaGetLastError() != cudaSuccess) return ROCO_ERR_CUDA;
  return p.splits > 1 ? launch_tree_join(p, ROCO_BF16, D, U, stream) : ROCO_OK;
}

roco_status launch_tree_attend_tc(const TreeParams &p, int d, int U, cudaStream_t stream) {
  const int n = tree_tc_width(p.rows);
  if (d == 128)
    return n == 16 ? tree_tc_t<128, 16>(p, U, stream) : n == 32 ? tree_tc_t<128, 32>(p, U, stream) : tree_tc_t<128, 64>(p, U, stream);
  return n == 16 ? tree_tc_t<64, 16>(p, U, stream) : n == 32 ? tree_tc_t<64, 32>(p, U, stream) : tree_tc_t<64, 64>(p, U, stream);
}

}  // namespace roco
