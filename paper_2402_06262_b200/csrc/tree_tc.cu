// Attention of a tree of drafted tokens over the cache on the fifth-generation tensor cores (bf16, positive scale).
//
// The query rows of a unit (heads x nodes, a few dozen) cannot fill the 128 rows of a tensor-core tile, the cached keys
// can: the key index lies on the accumulator's lanes and the N = 16, 32 or 64 query rows of a CTA are its columns.
//     S^T[128 keys x N] = K_tile Q^T          O^T[d x N] += V_tile^T P^T
// One pass over the cache.  A thread owns one key of a tile: it forms p = 2^(z - m) for its N scores, keeps N partial sums
// of its own in registers (joined over the lanes once, at the end) and writes the N probabilities as bf16, the second
// product's operand.  The reference m of a row need not be its maximum: any score that the row's sum contains will do, so
// it is that of the first cached key, and moves only when a score comes out more than 32 binary orders above it (fp32 and bf16
// share their exponents, so probabilities and sums above 1 lose nothing; the sum holds a 1).  The sum of a row's up to 8256 terms
// p v is then below 2^(32 + 13.02) max |v|, inside fp32 for values up to 2^82.  (At 16 orders that would be 2^98, and the moves of
// rows with a few dominant keys show: 24 units x 8192 x 96 rows 33.6 us instead of 32.0.)  It costs one vote per tile instead of
// a maximum over the lanes.  When it moves, to the tile's maximum, the row's column of O^T and its sums are rescaled.
// The drafted tokens are the last tile, masked by the rows' ancestor sets.  A product with zero keeps no NaN or infinity
// out, so if one of their values is not finite their part of the output is formed on the CUDA cores instead, node by node
// where a row sees the node: what lies on other branches cannot reach a row.
//
// Few units: their tokens are divided among CTAs, which join their results as a cluster (tree_cluster_join), or in a second
// launch where a cluster would not do.
//
// What bounds it.  The cache is read once.  Up to 32 rows two CTAs per SM, so that one's prologue and epilogue run under the
// other's stream: 8192 units x 1024 tokens x 16 rows 676 us in a replayed
// graph, 6.5 TB/s, the measured copy rate (687 us in single calls).  64 and 128 rows, one CTA: a
// tile of 128 tokens at 128 rows costs its two groups about 3000 cycles (1050 of products, 1020 of the exponential unit, the
// rest instructions and what 8 warps cannot hide of their latencies; 16 warps came out the same) where its 64 KiB take 2850: 24
// units x 8192 x 96 rows (worked on as 128) 32.2 us, of which 6 are the first tile's way here and 5 the join.  Small calls are latency: 32 units x
// 1024 x 8 rows 8.7 us, of which about 2 are the launch, 2.5 the first tile's way, 2 the draft and 1.5 the join.
#include <cuda.h>

#include <cfloat>
#include <type_traits>

#include "tc.cuh"
#include "tree.cuh"

namespace roco {

constexpr int kTtTile = 128;  // keys of a tile
constexpr int kTtGroup = 128;            // threads of a consumer group
constexpr int kTtBar = 1;     // named barriers of the consumer groups (kTtBar + group)
constexpr int kTtBarQ = 3;    // and of all of them with the warp of the products
constexpr float kTtMoveReference = 32.f;  // binary orders above the reference at which a row moves to a new one

// W groups of four consumer warps, N query rows each, share the tiles of a CTA and the products over them, N W columns wide
// (a product reads its 4 KiB of keys or values per 16-step once, however many columns it has); C CTAs per SM.
template <int D, int N, int W, int C>
struct TtShape {
  static constexpr int kThreads = W * kTtGroup + 64;
  static constexpr int kTile = kTtTile * D * 2, kBlock = kTtTile * 128;
  static constexpr int kCols = N * W;
  static constexpr int kQ = kCols * D * 2;
  // P^T of a tile: blocks of up to 64 columns, in 128-byte rows of 64 / columns keys each
  static constexpr int kPCols = kCols < 64 ? kCols : 64, kPRows = kPCols * 2, kPBlock = kPRows * 128;
  static constexpr int kP = kCols / kPCols * kPBlock;
  static constexpr int kPBufs = kCols == 128 ? 1 : 2;
  static constexpr int kGroupFloats = 4 * N /* red */ + 2 * N /* nref, alpha */;
  static constexpr int kFixed = 1024 + kQ + kP * kPBufs + W * kGroupFloats * 4 + kTreeMaxNodes * 12 + 256;
  static constexpr int kRoom = (227 / C) * 1024 - 1024 - kFixed;
  static constexpr int kStages = kRoom / kTile > 6 ? 6 : kRoom / kTile;
  static constexpr int kTmemCols = 4 * kCols;  // S^T twice, O^T; a power of two
  static constexpr size_t kSmem = (size_t)kFixed + (size_t)kStages * kTile;
  static_assert(kStages >= 2 && kTmemCols * C <= 512, "shared and tensor memory");
  // a cluster's results [columns][D] take the place of the operands P^T and Q
  static_assert(kCols * D * 4 <= kP * kPBufs + kQ, "results of a cluster");
  static_assert((2 * kStages + 6) * 8 + 16 <= 256, "barriers");
  // the drafted tokens' probabilities [nodes][N] of a group lie in a place of the ring once the stream is over
  static_assert(kTreeMaxNodes * N * 4 <= kTile && kStages >= W + 1, "draft probabilities");
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

__device__ __forceinline__ bool tt_any(bool x, int bar) {  // over the threads of a consumer group
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"((uint32_t)x), "r"(bar), "n"(kTtGroup)
      : "memory");
  return r != 0;
}

__device__ __forceinline__ void prefetch_tensor_map(const CUtensorMap *map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

__device__ __forceinline__ uint32_t tt_pack(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t *>(&v);
}

template <int D, int N, int W, int C>
__global__ void __launch_bounds__((TtShape<D, N, W, C>::kThreads), C)
    tree_tc_kernel(const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV,
                   const __grid_constant__ CUtensorMap mapKn, const __grid_constant__ CUtensorMap mapVn, const TreeParams p) {
  using Sh = TtShape<D, N, W, C>;
  constexpr int kTile = Sh::kTile, kBlock = Sh::kBlock, kStages = Sh::kStages, kCols = Sh::kCols;
  constexpr uint32_t kIdescS = (1u << 4) | (1u << 7) | (1u << 10) | (8u << 24) | (((uint32_t)kCols >> 3) << 17);
  constexpr uint32_t kIdescO = kIdescS | (1u << 15) | (1u << 16);  // both operands with the M / N index contiguous
  extern __shared__ char tt_raw[];
  launch_dependents();
  char *at = smem_align(tt_raw, 1024);
  char *ring = at; at += kStages * kTile;
  char *pbuf = at; at += Sh::kP * Sh::kPBufs;
  char *qop = at; at += Sh::kQ;
  float *floats = reinterpret_cast<float *>(at); at += W * Sh::kGroupFloats * 4;
  unsigned long long *anc = reinterpret_cast<unsigned long long *>(at); at += kTreeMaxNodes * 8;
  int *up = reinterpret_cast<int *>(at); at += kTreeMaxNodes * 4;
  uint64_t *full = reinterpret_cast<uint64_t *>(at), *empty = full + kStages;
  uint64_t *s_full = empty + kStages, *p_ready = s_full + 2, *pv_done = p_ready + 2;  // by tile parity
  uint32_t *tmem_base = reinterpret_cast<uint32_t *>(pv_done + 2);
  int *abort_ptr = reinterpret_cast<int *>(tmem_base + 2);
  int *odd = reinterpret_cast<int *>(tmem_base + 1);  // the drafted values are not all finite
  volatile int *abort_flag = abort_ptr;

  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int row_blocks = (p.rows + N * W - 1) / (N * W);
  const int split = blockIdx.x % p.splits, rb = blockIdx.x / p.splits % row_blocks, u = blockIdx.x / (row_blocks * p.splits);
  const int b = u / p.G, cta_row0 = rb * N * W;
  const bool report = tid == 0 && rb == 0 && split == 0;
  if (tid == 0) {  // on their way before the first load asks for them
    prefetch_tensor_map(&mapK);
    prefetch_tensor_map(&mapV);
  }
  const int n_nodes_ = tree_nodes(p, b, report), live_ = tree_live(p.live, u, p.B, p.status, report);
  const int n_nodes = __shfl_sync(0xffffffffu, n_nodes_, 0), live = __shfl_sync(0xffffffffu, live_, 0);
  if (cta_row0 >= n_nodes * p.group) return;
  const int tiles = (live + kTtTile - 1) / kTtTile;
  // the drafted tokens are one more tile, the last one's
  const int t0 = (int)((long long)(tiles + 1) * split / p.splits);
  const int ns = (int)((long long)(tiles + 1) * (split + 1) / p.splits) - t0;  // score tiles
  const bool drafts = split == p.splits - 1;
  const int nt = ns - (drafts ? 1 : 0);  // cached tiles of this CTA

  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&s_full[i], 1); mbar_init(&p_ready[i], 4 * W); mbar_init(&pv_done[i], 1); }
    *abort_ptr = 0;
    mbar_init_fence();
  }
  if (warp == 0) {
    tmem_alloc(tmem_base, Sh::kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_base, 0);

  if (warp == 4 * W) {
    if (lane == 0) {
      const int items = 2 * nt + (drafts ? 2 : 0);  // K, V, K, V, ..., the drafted tokens' keys and values
      for (int g = 0; g < items; ++g) {
        const int st = g % kStages;
        if (g >= kStages) mbar_wait_compact(&empty[st], (g / kStages - 1) & 1, abort_flag, p.status);
        const CUtensorMap *map = g >= 2 * nt ? ((g & 1) ? &mapVn : &mapKn) : ((g & 1) ? &mapV : &mapK);
        const int row = g >= 2 * nt ? 0 : (t0 + (g >> 1)) * kTtTile;
        mbar_expect_tx(&full[st], kTile);
#pragma unroll
        for (int h = 0; h < D / 64; ++h) tma_load_3d(ring + st * kTile + h * kBlock, map, 64 * h, row, u, &full[st]);
      }
    }
  } else if (warp == 4 * W + 1) {
    if (drafts) tree_ancestors_warp(p, b, n_nodes, anc, up, rb == 0);  // while the queries and the first tile are on their way
    named_bar_sync(kTtBarQ, W * kTtGroup + 32);                        // the queries are in place
    for (int t = 0; t <= ns; ++t) {
      if (t < ns) {  // scores of tile t; what its accumulator held was read before p_ready of two tiles ago
        const int g = 2 * t, st = g % kStages;
        mbar_wait_compact(&full[st], (g / kStages) & 1, abort_flag, p.status);
        tc_fence_after();
        const char *k = ring + st * kTile;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          umma_bf16_w(tmem + (t & 1) * kCols, smem_desc_sw128(k + (kk / 4) * kBlock + (kk % 4) * 32),
                      smem_desc_sw128(qop + (kk / 4) * (kCols * 128) + (kk % 4) * 32), kIdescS, kk > 0 ? 1u : 0u);
        umma_commit_w(&s_full[t & 1]);
        umma_commit_w(&empty[st]);
      }
      if (t >= 1) {  // output of tile t - 1
        const int g = 2 * t - 1, st = g % kStages, tv = t - 1;
        mbar_wait_compact(&full[st], (g / kStages) & 1, abort_flag, p.status);
        char *v = ring + st * kTile;
        const int keys = tv == nt ? n_nodes : live - (t0 + tv) * kTtTile;
        const int steps = keys < kTtTile ? (keys + 15) / 16 : 8;  // of 16 keys
        if (keys < 16 * steps) {  // what lies behind the last key may be anything (0 x NaN)
          for (int w = lane; w < (16 * steps - keys) * 8; w += 32) {
#pragma unroll
            for (int h = 0; h < D / 64; ++h)
              *reinterpret_cast<uint4 *>(v + h * kBlock + keys * 128 + w * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
          fence_async_smem();
          __syncwarp();
        }
        mbar_wait_compact(&p_ready[tv & 1], (tv >> 1) & 1, abort_flag, p.status);
        tc_fence_after();
        const char *pb = pbuf + tv % Sh::kPBufs * Sh::kP;
        const bool skip = tv == nt && __shfl_sync(0xffffffffu, *odd, 0);
        if (!skip) {
#pragma unroll
          for (int kk = 0; kk < 8; ++kk)  // (d = 64: the upper 64 accumulator lanes repeat the lower, unread)
            if (kk < steps)
              umma_bf16_w(tmem + 2 * kCols, smem_desc_sw128_mn(v + kk * 2048, D == 128 ? kBlock : 0),
                          smem_desc_sw128_mn(pb + (16 * kk % Sh::kPRows) * 128 + (16 * kk / Sh::kPRows) * (Sh::kPCols * 2), Sh::kPBlock),
                          kIdescO, (tv > 0 || kk > 0) ? 1u : 0u);
        }
        umma_commit_w(&pv_done[tv & 1]);
        umma_commit_w(&empty[st]);
      }
    }
  } else {
    // ---------------------------------------------------------------- consumers: a key per lane
    const int grp = W == 1 ? 0 : warp >> 2, bar = kTtBar + grp, row0 = cta_row0 + grp * N;
    const int gt = tid - grp * kTtGroup, gw = warp - 4 * grp;
    float *red = floats + grp * Sh::kGroupFloats, *nref = red + 4 * N, *alpha = nref + N;  // nref: minus a row's reference, log2
    // the drafted tokens' probabilities [node][N], after the stream: group 0's where their keys were, group 1's in the place
    // behind their values
    float *pd = reinterpret_cast<float *>(ring + (2 * nt + 2 * grp) % kStages * kTile);
    auto drafted_value = [&](int j) -> uint32_t {  // dimension gt of node j's value, as its 16 bits
      const char *vn = ring + (2 * nt + 1) % kStages * kTile + (gt >> 6) * kBlock + j * 128;
      return *reinterpret_cast<const uint16_t *>(vn + ((((gt & 63) >> 3) ^ (j & 7)) << 4) + (gt & 7) * 2);
    };
    {  // the queries as a K-major operand; rows that do not exist are zero
      const uint4 *Qu = reinterpret_cast<const uint4 *>(p.Q) + ((size_t)u * p.rows + cta_row0) * (D / 8);
      constexpr int kPieces = N * D / 8 / kTtGroup;  // 16-byte pieces per thread, all loaded before the first is stored
      uint4 x[kPieces];
#pragma unroll
      for (int k = 0; k < kPieces; ++k) {
        const int w = tid + k * W * kTtGroup;
        x[k] = make_uint4(0u, 0u, 0u, 0u);
        if (cta_row0 + w / (D / 8) < n_nodes * p.group) x[k] = Qu[w];
      }
#pragma unroll
      for (int k = 0; k < kPieces; ++k) {
        const int w = tid + k * W * kTtGroup, i = w / (D / 8), c = w % (D / 8);
        *reinterpret_cast<uint4 *>(qop + (c >> 3) * (kCols * 128) + i * 128 + (((c & 7) ^ (i & 7)) << 4)) = x[k];
      }
      fence_async_smem();
    }
    named_bar_sync(kTtBarQ, W * kTtGroup + 32);
    const float zs = p.scale * kLog2e;
    const f32x2 zs2 = pack2(zs, zs);
    const uint32_t tl = tmem + grp * N + ((uint32_t)(gw * 32) << 16);
    // this thread's key and the group's columns in P^T
    const int prow = gt % Sh::kPRows, pc0 = gt / Sh::kPRows * (Sh::kPCols / 8) + grp * N % Sh::kPCols / 8;
    char *pgrp = pbuf + grp * N / Sh::kPCols * Sh::kPBlock + prow * 128;
    f32x2 l[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) l[i] = pack2(0.f, 0.f);
    // The output product of tile t is complete.  One barrier per tile parity: this thread is never two phases of either
    // behind, since the product of tile t + 2 waits for its own probabilities of that tile.
    auto wait_pv = [&](int t) {
      if (t >= 0) mbar_wait_compact(&pv_done[t & 1], (t >> 1) & 1, abort_flag, p.status);
    };
    // The rows (bits) of the group that see drafted token gt: its descendants and itself, each `group` rows long.  Found while
    // the first tile is on its way, if there are registers to keep it.
    auto rows_that_see = [&]() {
      unsigned long long sees = 0ull;
      if (gt < n_nodes) {
        const uint32_t *set = reinterpret_cast<const uint32_t *>(anc) + (gt >> 5);
        const int node0 = row0 / p.group, nodes = min((row0 + N + p.group - 1) / p.group, n_nodes) - node0;
        const int before = row0 - node0 * p.group;  // rows of the first node that belong to the group of columns before
        const unsigned long long run = (1ull << p.group) - 1ull;
#pragma unroll 4
        for (int k = 0; k < nodes; ++k) {
          if ((set[2 * (node0 + k)] >> (gt & 31)) & 1u) sees |= k ? run << (k * p.group - before) : run >> before;
        }
      }
      return sees;
    };
    const uint32_t early = N <= 32 && drafts ? (uint32_t)rows_that_see() : 0u;
    if (gt < N) nref[gt] = 0.f;
    named_bar_sync(bar, kTtGroup);
    bool by_hand = false;

#pragma unroll 1
    for (int t = 0; t < ns; ++t) {
      const bool is_draft = t == nt;
      const int keys = is_draft ? n_nodes : live - (t0 + t) * kTtTile;  // of this tile (more: a full one)
      unsigned long long mine = gt < keys ? ~0ull : 0ull;               // the rows (bits) that see this thread's key
      if (is_draft) mine = N <= 32 ? (unsigned long long)early : rows_that_see();
      const uint32_t ts = tl + (t & 1) * kCols;
      mbar_wait_compact(&s_full[t & 1], (t >> 1) & 1, abort_flag, p.status);
      tc_fence_after();
      f32x2 d[N / 2];  // z - m, log2
      auto scores = [&]() {
        if constexpr (N == 16) {
          uint32_t r[16];
          tmem_ld16(ts, r);
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            const float4 n4 = *reinterpret_cast<const float4 *>(nref + i);
            d[i / 2] = fma2(pack2u(r[i], r[i + 1]), zs2, pack2(n4.x, n4.y));
            d[i / 2 + 1] = fma2(pack2u(r[i + 2], r[i + 3]), zs2, pack2(n4.z, n4.w));
          }
        } else {
#pragma unroll
          for (int x = 0; x < N; x += 32) {
            uint32_t r[32];
            tmem_ld32_issue(ts + x, r);
            tmem_ld_wait(r);
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
              const float4 n4 = *reinterpret_cast<const float4 *>(nref + x + i);
              d[(x + i) / 2] = fma2(pack2u(r[i], r[i + 1]), zs2, pack2(n4.x, n4.y));
              d[(x + i) / 2 + 1] = fma2(pack2u(r[i + 2], r[i + 3]), zs2, pack2(n4.z, n4.w));
            }
          }
        }
      };
      auto masked_scores = [&]() {
        scores();
        if (keys < kTtTile) {
#pragma unroll
          for (int i = 0; i < N / 2; ++i) {
            float lo, hi;
            unpack2(d[i], lo, hi);
            d[i] = pack2((mine >> (2 * i)) & 1ull ? lo : -INFINITY, (mine >> (2 * i + 1)) & 1ull ? hi : -INFINITY);
          }
        }
      };
      bool move = false;
      if (t == 0) {
        if (is_draft) {
          move = true;  // no key that every row sees
        } else {
          if (gw == 0) {
#pragma unroll 1
            for (int x = 0; x < N; x += 16) {
              uint32_t r[16];
              tmem_ld16(ts + x, r);
              if (lane == 0) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                  const float z = __uint_as_float(r[i]) * zs;
                  nref[x + i] = -z;
                  move |= !(fabsf(z) < INFINITY);
                }
              }
            }
          }
          named_bar_sync(bar, kTtGroup);
        }
      }
      masked_scores();
      {
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
          float lo, hi;
          unpack2(d[i], lo, hi);
          top = max3(top, lo, hi);
        }
        move |= top > kTtMoveReference;
      }
      if (tt_any(move, bar)) {
        // new references: the tile's maxima where they are larger
#pragma unroll 1
        for (int x = 0; x < N; x += 16) {
          uint32_t r[16];
          float v[16];
          tmem_ld16(ts + x, r);
          const uint32_t m = (uint32_t)(mine >> x);
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = (m >> i) & 1u ? __uint_as_float(r[i]) * zs : -INFINITY;
          const float top = tt_lanes_reduce<true>(v, lane);
          if ((lane & 1) == 0) red[gw * N + x + (lane >> 1)] = top;
        }
        named_bar_sync(bar, kTtGroup);
        if (gt < N) {
          const float top = fmaxf(fmaxf(red[gt], red[N + gt]), fmaxf(red[2 * N + gt], red[3 * N + gt]));
          const float old = t == 0 ? -INFINITY : -nref[gt];
          float ref = fmaxf(old, top);
          // nothing seen so far (every score is minus infinity, or the row does not exist): the first finite score moves it
          if (ref == -INFINITY) ref = -FLT_MAX;
          alpha[gt] = t == 0 ? 0.f : exp2f(old - ref);
          nref[gt] = -ref;
        }
        wait_pv(t - 1);  // nothing adds to O^T now
        tc_fence_after();
        named_bar_sync(bar, kTtGroup);
        if (t > 0) {
#pragma unroll
          for (int x = 0; x < N; x += 16) {
            uint32_t r[16];
            tmem_ld16(tl + 2 * kCols + x, r);
#pragma unroll
            for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * alpha[x + i]);
            tmem_st16(tl + 2 * kCols + x, r);
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
              float lo, hi;
              unpack2(l[(x + i) / 2], lo, hi);
              l[(x + i) / 2] = pack2(lo * alpha[x + i], hi * alpha[x + i + 1]);
            }
          }
          tmem_st_wait();
        }
        masked_scores();
      }
      wait_pv(t - Sh::kPBufs);  // the operand's place is free
      if (is_draft) {
        // are the drafted values finite?  (0 x: NaN if not)
        mbar_wait_compact(&full[(2 * nt + 1) % kStages], ((2 * nt + 1) / kStages) & 1, abort_flag, p.status);
        __nv_bfloat162 zero = __float2bfloat162_rn(0.f), nil = zero;
#pragma unroll 1
        for (int w = gt; w < n_nodes * 8; w += kTtGroup) {
#pragma unroll
          for (int h = 0; h < D / 64; ++h) {
            const uint4 x = *reinterpret_cast<const uint4 *>(ring + (2 * nt + 1) % kStages * kTile + h * kBlock + w * 16);
            nil = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&x.x), zero, nil);
            nil = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&x.y), zero, nil);
            nil = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&x.z), zero, nil);
            nil = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&x.w), zero, nil);
          }
        }
        by_hand = tt_any(!(__low2float(nil) == 0.f && __high2float(nil) == 0.f), bar);
        if (gt == 0) *odd = by_hand;
        if (by_hand) {
          // the places of the ring where the probabilities go are free once the products have read them (the scores of this
          // tile, which are here, and the output of the last)
          wait_pv(nt - 1);
        }
      }
      char *prow_p = pgrp + t % Sh::kPBufs * Sh::kP;
#pragma unroll
      for (int x = 0; x < N; x += 8) {
        float f[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // (every one by the exponential unit, which keeps NaN and is good to 2^-22; a quarter by a polynomial on the FMA pipe
          // was slower too: 1024 units x 1024 x 128 rows 158 us, now 153)
          const f32x2 e = exp2_mufu2(d[x / 2 + i]);
          l[x / 2 + i] = add2(l[x / 2 + i], e);
          unpack2(e, f[2 * i], f[2 * i + 1]);
        }
        if (is_draft && by_hand && gt < kTreeMaxNodes) {
#pragma unroll
          for (int i = 0; i < 8; ++i) pd[gt * N + x + i] = f[i];
        }
        *reinterpret_cast<uint4 *>(prow_p + (((pc0 + x / 8) ^ (prow & 7)) << 4)) =
            make_uint4(tt_pack(f[0], f[1]), tt_pack(f[2], f[3]), tt_pack(f[4], f[5]), tt_pack(f[6], f[7]));
      }
      fence_async_smem();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&p_ready[t & 1]);
    }

    // ---------------------------------------------------------------- the sums over the lanes, then a dimension per lane
    wait_pv(ns - 1);
    tc_fence_after();
    named_bar_sync(bar, kTtGroup);  // red is free, pd complete
#pragma unroll
    for (int x = 0; x < N; x += 16) {
      float v[16];
#pragma unroll
      for (int i = 0; i < 16; i += 2) unpack2(l[(x + i) / 2], v[i], v[i + 1]);
      const float sum = tt_lanes_reduce<false>(v, lane);
      if ((lane & 1) == 0) red[gw * N + x + (lane >> 1)] = sum;
    }
    named_bar_sync(bar, kTtGroup);
    const int rows = max(0, min(N, n_nodes * p.group - row0));
    if (gt < N) {
      const float sum = (red[gt] + red[N + gt]) + (red[2 * N + gt] + red[3 * N + gt]);
      const float ref = ns > 0 ? -nref[gt] : -INFINITY;
      alpha[gt] = p.splits > 1 ? sum : 1.f / sum;
      if (p.cluster) {
        nref[gt] = ref;
      } else if (gt < rows) {
        if (p.splits > 1) {
          const size_t pt = ((size_t)u * p.splits + split) * p.rows + row0 + gt;
          *reinterpret_cast<float2 *>(p.part_ml + 2 * pt) = make_float2(ref, sum);
        } else if (p.lse) {
          p.lse[(size_t)u * p.rows + row0 + gt] = (ref + log2f(sum)) * kLn2;
        }
      }
    }
    named_bar_sync(bar, kTtGroup);
    if (gw * 32 < D) {
#pragma unroll 1
      for (int x = 0; x < rows; x += 16) {
        float o[16];
        if (nt > 0 || (drafts && !by_hand)) {
          uint32_t r[16];
          tmem_ld16(tl + 2 * kCols + x, r);
#pragma unroll
          for (int i = 0; i < 16; ++i) o[i] = __uint_as_float(r[i]);
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) o[i] = 0.f;
        }
        if (by_hand) {
#pragma unroll 1
          for (int j = 0; j < n_nodes; ++j) {
            const float v = __uint_as_float(drafted_value(j) << 16);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float e = pd[j * N + x + i];
              if (e != 0.f) o[i] = fmaf(e, v, o[i]);
            }
          }
        }
        if (p.splits > 1) {
          float *dst = p.cluster ? reinterpret_cast<float *>(pbuf) + (grp * N + x) * D + gt
                                 : p.part_o + (((size_t)u * p.splits + split) * p.rows + row0 + x) * D + gt;
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (x + i < rows) dst[(size_t)i * D] = o[i];
        } else {
          __nv_bfloat16 *dst = reinterpret_cast<__nv_bfloat16 *>(p.out) + ((size_t)u * p.rows + row0 + x) * D + gt;
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
  if (p.cluster) {
    auto row_ref = [&](int row) { return floats + row / N * Sh::kGroupFloats + 4 * N + row % N; };
    tree_cluster_join<__nv_bfloat16, D>(p, u, cta_row0, min(kCols, n_nodes * p.group - cta_row0), split, warp, Sh::kThreads / 32,
                                        lane, reinterpret_cast<const float *>(pbuf), row_ref, N);
  }
}

// How the query rows of a unit are laid out: N columns a group, W groups of a CTA that share its tiles, C CTAs per SM.  Rows
// beyond 128 go to further CTAs, which find the cache in L2.
struct TtPlan {
  int n, w, c;
};
TtPlan tree_tc_plan(int rows) {
  if (rows <= 16) return {16, 1, 2};
  if (rows <= 32) return {32, 1, 2};
  if (rows <= 64) return {32, 2, 1};
  return {64, 2, 1};
}
int tree_tc_rows(int rows) { const TtPlan t = tree_tc_plan(rows); return t.n * t.w; }
int tree_tc_ctas(int rows) { return tree_tc_plan(rows).c; }

template <int D, int N, int W, int C>
roco_status tree_tc_t(const TreeParams &p, int U, cudaStream_t stream) {
  CUtensorMap mk, mv, mn, mw;
  if (!make_tensor_map_units_bf16(&mk, p.K, U, p.B, D, kTtTile) || !make_tensor_map_units_bf16(&mv, p.V, U, p.B, D, kTtTile) ||
      !make_tensor_map_units_bf16(&mn, p.k_new, U, p.T, D, kTtTile) || !make_tensor_map_units_bf16(&mw, p.v_new, U, p.T, D, kTtTile))
    return ROCO_ERR_CUDA;
  using Sh = TtShape<D, N, W, C>;
  auto kernel = tree_tc_kernel<D, N, W, C>;
  static SmemLimit limit;
  if (!limit((const void *)kernel, Sh::kSmem)) return ROCO_ERR_CUDA;
  const unsigned blocks = (unsigned)U * (unsigned)((p.rows + N * W - 1) / (N * W)) * (unsigned)p.splits;
  if (p.cluster) {
    const bool ok = launch_cluster(kernel, blocks, (unsigned)p.splits, Sh::kThreads, Sh::kSmem, stream, mk, mv, mn, mw, p);
    return ok ? ROCO_OK : ROCO_ERR_CUDA;
  }
  kernel<<<blocks, Sh::kThreads, Sh::kSmem, stream>>>(mk, mv, mn, mw, p);
  if (cudaGetLastError() != cudaSuccess) return ROCO_ERR_CUDA;
  return p.splits > 1 ? launch_tree_join_bf16(p, D, U, stream) : ROCO_OK;
}

template <int D>
roco_status tree_tc_d(const TreeParams &p, int U, int sms, cudaStream_t stream) {
  const TtPlan t = tree_tc_plan(p.rows);
  // Few CTAs: one per SM, with a ring that holds three tiles (8 units x 8192 x 32 rows: 21.1 -> 16.5 us); not where clusters
  // of more than four would not pack (16 of eight: 11.0 -> 16.1 us).
  const long long ctas = (long long)U * p.splits;
  const bool few = ctas <= sms && (!p.cluster || p.splits <= 4 || 2 * ctas <= sms);
  if (t.n == 16) return few ? tree_tc_t<D, 16, 1, 1>(p, U, stream) : tree_tc_t<D, 16, 1, 2>(p, U, stream);
  if (t.n == 32 && t.w == 1) return few ? tree_tc_t<D, 32, 1, 1>(p, U, stream) : tree_tc_t<D, 32, 1, 2>(p, U, stream);
  if (t.n == 32) return tree_tc_t<D, 32, 2, 1>(p, U, stream);
  return tree_tc_t<D, 64, 2, 1>(p, U, stream);
}

roco_status launch_tree_attend_tc(const TreeParams &p, int d, int U, int sms, cudaStream_t stream) {
  return d == 128 ? tree_tc_d<128>(p, U, sms, stream) : tree_tc_d<64>(p, U, sms, stream);
}

}  // namespace roco
