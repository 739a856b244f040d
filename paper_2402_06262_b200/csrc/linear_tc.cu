// Linear attention with a decay for each head over a prompt on the fifth-generation tensor cores (bf16).
//
// In chunks of C = 128 tokens, with i, j counted inside the chunk and S the fp32 state before it:
//     out_i = scale * ( g^(i+1) q_i S + sum_{j <= i} g^(i-j) (q_i.k_j) v_j )
//     S    <- g^C S + sum_j (g^(C-1-j) k_j)^T v_j
// which is four products per chunk, issued by one thread, accumulators in tensor memory:
//     S1 = Q K^T                                   both operands as TMA wrote them
//     O  = Q bf16(S)          then, by the A warps, row i times g^(i+1)
//     O += P V                P = S1 with the decays as bf16, from tensor memory
//     DS = KH^T V + KL^T V    KH + KL = g^(C-1-j) k_j as the sum of two bf16, from tensor memory
// Every power of the decay is at most 1, so nothing overflows however fast a head forgets.  The state itself stays in the
// registers of the B warps in fp32 from the first chunk to the last: a thread keeps half a row, adds DS (which the
// split keys make exact to 2^-16 of each term) and writes the row as the next chunk's operand.  Rounded to bf16 are the
// operands P and S of the output, which is bf16 itself.
//
// Warps: 0-7 (A) a token per tensor-memory lane, half of the columns each: P, the scaling of O, the output.  8-15 (B) a
// row of the state per lane: DS, the state, KH and KL.  16 TMA loads and stores (the output of a chunk is staged where its
// queries were), 17 the products.
//
// What bounds it: 128 KiB cross HBM per chunk at d = 128, 3.0 us at one SM's share of the measured copy rate, against
// 2560 tensor cycles (1.4 us); the chain DS -> state -> KH -> DS and the one S1 -> P -> O -> output run side by side.
#include <cuda.h>

#include "linear.cuh"
#include "tc.cuh"

namespace roco {

constexpr int kLtChunk = 128;
constexpr int kLtAWarps = 8, kLtBWarps = 8;
constexpr int kLtTmaWarp = kLtAWarps + kLtBWarps, kLtMmaWarp = kLtTmaWarp + 1;
constexpr int kLtThreads = (kLtMmaWarp + 1) * 32;
constexpr uint32_t kLtColS = 0, kLtColO = 128, kLtColDS = 256, kLtColKH = 384, kLtColKL = 448, kLtTmemCols = 512;

template <int D>
struct LtSmem {
  static constexpr int kTile = kLtChunk * D * 2;
  static constexpr int kSop = D * D * 2;
  static constexpr int kBars = 24;
  static constexpr size_t bytes(bool states) {
    return 1024 + (size_t)kTile * (states ? 4 : 6) + (states ? 0 : kSop) + 260 * 4 + kBars * 8 + 16;
  }
};

__device__ __forceinline__ void umma_bf16_tmem_a(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc,
                                                 uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap *map, const void *src, int c0, int c1, int c2) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
               ::"l"(map), "r"(smem_u32(src)), "r"(c0), "r"(c1), "r"(c2)
               : "memory");
}
__device__ __forceinline__ uint32_t lt_pack(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t *>(&v);
}

template <int D, bool kStates>
__global__ void __launch_bounds__(kLtThreads, 1)
    linear_prefill_tc_kernel(const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapK,
                             const __grid_constant__ CUtensorMap mapV, const __grid_constant__ CUtensorMap mapO,
                             const LinearParams p) {
  constexpr int kTile = LtSmem<D>::kTile, kBlock = kLtChunk * 128;  // a 64-column block of a tile: 128 rows of 128 bytes
  constexpr int kHalfCols = D / 2;                                  // columns of the state or output a thread works on
  constexpr uint32_t kIdesc = (1u << 4) | (1u << 7) | (1u << 10) | (8u << 24);       // bf16, fp32 accumulator, M = 128
  constexpr uint32_t kIdescS = kIdesc | ((128u >> 3) << 17);                         // N = 128, both K-major
  constexpr uint32_t kIdescV = kIdesc | (((uint32_t)D >> 3) << 17) | (1u << 16);     // N = D, B with N contiguous
  extern __shared__ char lt_raw[];
  char *at = smem_align(lt_raw, 1024);
  char *kt = at; at += 2 * kTile;
  char *vt = at; at += 2 * kTile;
  char *qt = at; if (!kStates) at += 2 * kTile;
  char *sop = at; if (!kStates) at += LtSmem<D>::kSop;
  float *tbl = reinterpret_cast<float *>(at); at += 260 * 4;  // tbl[128 + n] = g^n for 0 <= n <= 128, 0 for n < 0
  uint64_t *bars = reinterpret_cast<uint64_t *>(at); at += LtSmem<D>::kBars * 8;
  uint64_t *k_full = bars, *k_empty = bars + 2, *v_full = bars + 4, *v_empty = bars + 6, *q_full = bars + 8;
  uint64_t *s1_full = bars + 12, *p_ready = bars + 13, *o1_full = bars + 14, *o_scaled = bars + 15, *o_full = bars + 16;
  uint64_t *o_free = bars + 17, *sop_ready = bars + 18, *ds_full = bars + 19, *kp_ready = bars + 20, *staged = bars + 21;
  uint32_t *tmem_base = reinterpret_cast<uint32_t *>(at);
  int *abort_ptr = reinterpret_cast<int *>(at + 8);
  volatile int *abort_flag = abort_ptr;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int segs = kStates ? p.segments - 1 : p.segments, seg = blockIdx.x % segs, u = blockIdx.x / segs;
  const int len = linear_len(p, u / p.G, tid == 0 && seg == 0 && (kStates || p.segments == 1));
  if (len == 0) return;
  const int n_chunks = (len + kLtChunk - 1) / kLtChunk;
  const int first = linear_segment(n_chunks, p.segments, seg), last = linear_segment(n_chunks, p.segments, seg + 1);
  const int n = last - first;
  const int tail = last == n_chunks ? len - (n_chunks - 1) * kLtChunk : kLtChunk;  // tokens of this segment's last chunk
  const double logd = (double)p.log_decay[u % p.G];

  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&k_full[i], 1); mbar_init(&k_empty[i], 1);
      mbar_init(&v_full[i], 1); mbar_init(&v_empty[i], 1);
      mbar_init(&q_full[i], 1);
    }
    mbar_init(s1_full, 1); mbar_init(p_ready, kLtAWarps); mbar_init(o1_full, 1); mbar_init(o_scaled, kLtAWarps);
    mbar_init(o_full, 1); mbar_init(o_free, kLtAWarps); mbar_init(sop_ready, kLtBWarps); mbar_init(ds_full, 1);
    mbar_init(kp_ready, kLtBWarps); mbar_init(staged, kLtAWarps);
    *abort_ptr = 0;
    mbar_init_fence();
  }
  if (tid < 257) tbl[tid] = tid < 128 ? 0.f : (float)decay_pow(logd, tid - 128);
  if (warp == 0) {
    tmem_alloc(tmem_base, kLtTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_base;

  if (warp == kLtTmaWarp) {
    if (lane == 0) {
      for (int c = 0; c < n + 2; ++c) {
        const int sl = c & 1, row = (first + c) * kLtChunk;
        auto load = [&](char *tiles, const CUtensorMap *map, uint64_t *full) {
          mbar_expect_tx(&full[sl], kTile);
#pragma unroll
          for (int h = 0; h < D / 64; ++h) tma_load_3d(tiles + sl * kTile + h * kBlock, map, 64 * h, row, u, &full[sl]);
        };
        if (c < n) {
          if (c >= 2) mbar_wait(&k_empty[sl], ((c >> 1) - 1) & 1, abort_flag, p.status);
          load(kt, &mapK, k_full);
          if (c >= 2) mbar_wait(&v_empty[sl], ((c >> 1) - 1) & 1, abort_flag, p.status);
          load(vt, &mapV, v_full);
        }
        if (!kStates) {
          // the output of the chunk before the last leaves its slot, which then takes the queries of this one (a partial
          // chunk is the segment's last and is written by the A warps)
          if (c >= 2 && !(c - 2 == n - 1 && tail < kLtChunk)) {
            mbar_wait(staged, c & 1, abort_flag, p.status);
#pragma unroll
            for (int h = 0; h < D / 64; ++h) tma_store_3d(&mapO, qt + sl * kTile + h * kBlock, 64 * h, row - 2 * kLtChunk, u);
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
          }
          if (c < n) load(qt, &mapQ, q_full);
        }
      }
      if (!kStates) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
  } else if (warp == kLtMmaWarp) {
    for (int c = 0; c < n; ++c) {
      const int sl = c & 1;
      const uint32_t full = (c >> 1) & 1, par = c & 1;
      char *k = kt + sl * kTile, *v = vt + sl * kTile, *q = qt + sl * kTile;
      mbar_wait(&k_full[sl], full, abort_flag, p.status);
      if (c == n - 1 && tail < kLtChunk) {
        // rows behind the prompt may hold anything: their scores are multiplied by zero, and so are their values
        mbar_wait(&v_full[sl], full, abort_flag, p.status);
        for (int w = lane; w < (kLtChunk - tail) * 8; w += 32) {
#pragma unroll
          for (int h = 0; h < D / 64; ++h) {
            if (!kStates) *reinterpret_cast<uint4 *>(k + h * kBlock + tail * 128 + w * 16) = make_uint4(0u, 0u, 0u, 0u);
            *reinterpret_cast<uint4 *>(v + h * kBlock + tail * 128 + w * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
        }
        fence_async_smem();
        __syncwarp();
      }
      if (!kStates) {
        mbar_wait(&q_full[sl], full, abort_flag, p.status);
        tc_fence_after();
        if (lane == 0) {  // S1 (the product that read P from these columns was issued before it)
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            const int off = (kk / 4) * kBlock + (kk % 4) * 32;
            umma_bf16(tmem + kLtColS, smem_desc_sw128(q + off), smem_desc_sw128(k + off), kIdescS, kk > 0 ? 1u : 0u);
          }
          umma_commit(s1_full);
        }
        __syncwarp();
        mbar_wait(sop_ready, par, abort_flag, p.status);
        if (c > 0) mbar_wait(o_free, (c - 1) & 1, abort_flag, p.status);
        tc_fence_after();
        if (lane == 0) {  // O = Q S
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)
            umma_bf16(tmem + kLtColO, smem_desc_sw128(q + (kk / 4) * kBlock + (kk % 4) * 32),
                      smem_desc_sw128_mn(sop + kk * 2048, D * 128), kIdescV, kk > 0 ? 1u : 0u);
          umma_commit(o1_full);
        }
        __syncwarp();
      }
      mbar_wait(kp_ready, par, abort_flag, p.status);
      mbar_wait(&v_full[sl], full, abort_flag, p.status);
      tc_fence_after();
      if (lane == 0) {  // DS
#pragma unroll
        for (int kk = 0; kk < 16; ++kk)
          umma_bf16_tmem_a(tmem + kLtColDS, tmem + (kk < 8 ? kLtColKH : kLtColKL) + (uint32_t)(8 * (kk & 7)),
                           smem_desc_sw128_mn(v + (kk & 7) * 2048, kBlock), kIdescV, kk > 0 ? 1u : 0u);
        umma_commit(ds_full);
        umma_commit(&k_empty[sl]);
        if (kStates) umma_commit(&v_empty[sl]);
      }
      __syncwarp();
      if (!kStates) {
        mbar_wait(p_ready, par, abort_flag, p.status);
        mbar_wait(o_scaled, par, abort_flag, p.status);
        tc_fence_after();
        if (lane == 0) {  // O += P V
#pragma unroll
          for (int kk = 0; kk < 8; ++kk)
            umma_bf16_tmem_a(tmem + kLtColO, tmem + kLtColS + (uint32_t)((kk >> 2) * 64 + (kk & 3) * 8),
                             smem_desc_sw128_mn(v + kk * 2048, kBlock), kIdescV, 1u);
          umma_commit(o_full);
          umma_commit(&v_empty[sl]);
        }
        __syncwarp();
      }
    }
  } else if (warp < kLtAWarps) {
    // ---------------------------------------------------------------- A: scores and output, a token per lane
    if (!kStates) {
      const int wq = warp & 3, half = warp >> 2, i = wq * 32 + lane;
      const uint32_t tl = tmem + ((uint32_t)(wq * 32) << 16);
      const float inter = tbl[128 + i + 1];
      for (int c = 0; c < n; ++c) {
        const uint32_t par = c & 1;
        mbar_wait(s1_full, par, abort_flag, p.status);
        tc_fence_after();
#pragma unroll
        for (int cc = 0; cc < 2; ++cc) {
          const int j0 = half * 64 + cc * 32;
          uint32_t pk[16];
          if (wq * 32 + 31 < j0) {  // the whole block lies behind the diagonal
#pragma unroll
            for (int e = 0; e < 16; ++e) pk[e] = 0u;
          } else {
            uint32_t r[32];
            tmem_ld32_issue(tl + kLtColS + (uint32_t)j0, r);
            const float *w = tbl + 128 + i - j0;
            tmem_ld_wait(r);
#pragma unroll
            for (int e = 0; e < 32; e += 2)
              pk[e >> 1] = lt_pack(__uint_as_float(r[e]) * w[-e], __uint_as_float(r[e + 1]) * w[-e - 1]);
          }
          tmem_st16(tl + kLtColS + (uint32_t)(half * 64 + cc * 16), pk);
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_ready);
        mbar_wait(o1_full, par, abort_flag, p.status);
        tc_fence_after();
        const uint32_t to = tl + kLtColO + (uint32_t)(half * kHalfCols);
#pragma unroll
        for (int x = 0; x < kHalfCols; x += 32) {
          uint32_t r[32];
          tmem_ld32_issue(to + (uint32_t)x, r);
          tmem_ld_wait(r);
          uint32_t a[16], b[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            a[e] = __float_as_uint(__uint_as_float(r[e]) * inter);
            b[e] = __float_as_uint(__uint_as_float(r[e + 16]) * inter);
          }
          tmem_st16(to + (uint32_t)x, a);
          tmem_st16(to + (uint32_t)x + 16u, b);
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(o_scaled);
        mbar_wait(o_full, par, abort_flag, p.status);
        tc_fence_after();
        const bool partial = c == n - 1 && tail < kLtChunk;
        char *stage = qt + (c & 1) * kTile;  // the products that read the queries are complete
        char *orow = p.out + (((size_t)u * p.Lmax + (size_t)(first + c) * kLtChunk + i) * D) * 2;
#pragma unroll
        for (int x = 0; x < kHalfCols; x += 32) {
          uint32_t r[32];
          tmem_ld32_issue(to + (uint32_t)x, r);
          tmem_ld_wait(r);
          if (x + 32 >= kHalfCols) {  // the accumulator may take the next chunk's product
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(o_free);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint4 o;
            o.x = lt_pack(__uint_as_float(r[8 * e]) * p.scale, __uint_as_float(r[8 * e + 1]) * p.scale);
            o.y = lt_pack(__uint_as_float(r[8 * e + 2]) * p.scale, __uint_as_float(r[8 * e + 3]) * p.scale);
            o.z = lt_pack(__uint_as_float(r[8 * e + 4]) * p.scale, __uint_as_float(r[8 * e + 5]) * p.scale);
            o.w = lt_pack(__uint_as_float(r[8 * e + 6]) * p.scale, __uint_as_float(r[8 * e + 7]) * p.scale);
            const int col = half * kHalfCols + x + 8 * e, ch = (col & 63) >> 3;
            if (!partial) *reinterpret_cast<uint4 *>(stage + (col >> 6) * kBlock + i * 128 + ((ch ^ (i & 7)) << 4)) = o;
            else if (i < tail) *reinterpret_cast<uint4 *>(orow + col * 2) = o;
          }
        }
        if (!partial) {
          fence_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(staged);
        }
      }
    }
  } else {
    // ---------------------------------------------------------------- B: the state, a row per lane
    const int wq = warp & 3, half = (warp >> 2) & 1, r0 = wq * 32 + lane;
    const bool mine = wq * 32 < D;  // d = 64: the upper two lane quarters hold no rows
    const uint32_t tl = tmem + ((uint32_t)(wq * 32) << 16);
    float *S = p.state + ((size_t)u * D + r0) * D + half * kHalfCols;
    float *part = p.parts + ((size_t)u * p.segments * D + r0) * D + half * kHalfCols;
    float s[kHalfCols];
#pragma unroll
    for (int x = 0; x < kHalfCols; ++x) s[x] = 0.f;
    if (mine) {
      if (seg == 0) {
        const float *src = (kStates || p.segments == 1) ? S : part;
#pragma unroll
        for (int x = 0; x < kHalfCols; x += 4) {
          const float4 f = *reinterpret_cast<const float4 *>(src + x);
          s[x] = f.x; s[x + 1] = f.y; s[x + 2] = f.z; s[x + 3] = f.w;
          if (kStates) *reinterpret_cast<float4 *>(part + x) = f;  // the second launch starts from this copy
        }
      } else if (!kStates) {
        for (int m = 1; m <= seg; ++m) {
          const float w = (float)decay_pow(logd, (double)(first - linear_segment(n_chunks, p.segments, m)) * kLtChunk);
          const float *src = part + (size_t)m * D * D;
#pragma unroll
          for (int x = 0; x < kHalfCols; x += 4) {
            const float4 f = *reinterpret_cast<const float4 *>(src + x);
            s[x] = fmaf(w, f.x, s[x]); s[x + 1] = fmaf(w, f.y, s[x + 1]);
            s[x + 2] = fmaf(w, f.z, s[x + 2]); s[x + 3] = fmaf(w, f.w, s[x + 3]);
          }
        }
      }
    }
    const Decay2 g_chunk(decay_pow(logd, kLtChunk));
    auto add_ds = [&](int c, const Decay2 &g) {  // the state behind chunk c
      mbar_wait(ds_full, c & 1, abort_flag, p.status);
      tc_fence_after();
      if (mine) {
#pragma unroll
        for (int x = 0; x < kHalfCols; x += 16) {
          uint32_t r[16];
          tmem_ld16(tl + kLtColDS + (uint32_t)(half * kHalfCols + x), r);
#pragma unroll
          for (int e = 0; e < 16; ++e) s[x + e] = g.madd(s[x + e], __uint_as_float(r[e]));
        }
      }
    };
    for (int c = 0; c < n; ++c) {
      const int sl = c & 1;
      if (c > 0) add_ds(c - 1, g_chunk);
      if (!kStates) {
        if (c > 0) mbar_wait(o1_full, (c - 1) & 1, abort_flag, p.status);  // the operand of the chunk before is used up
        if (mine) {
          // row r0 of the operand: 64 columns to a block of D rows of 128 bytes
          char *row = sop + r0 * 128;
#pragma unroll
          for (int x = 0; x < kHalfCols; x += 8) {
            const int col = half * kHalfCols + x, ch = (col & 63) >> 3;
            *reinterpret_cast<uint4 *>(row + (col >> 6) * (D * 128) + ((ch ^ (r0 & 7)) << 4)) =
                make_uint4(lt_pack(s[x], s[x + 1]), lt_pack(s[x + 2], s[x + 3]), lt_pack(s[x + 4], s[x + 5]),
                           lt_pack(s[x + 6], s[x + 7]));
          }
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(sop_ready);
      }
      mbar_wait(&k_full[sl], (c >> 1) & 1, abort_flag, p.status);
      if (mine) {
        // component r0 of 64 keys, times what is left of each at the end of the chunk, as a sum of two bf16
        const int nt = c == n - 1 ? tail : kLtChunk;
        const char *kcol = kt + sl * kTile + (r0 >> 6) * kBlock + (r0 & 7) * 2;
        const int ch = (r0 & 63) >> 3;
#pragma unroll 1
        for (int tt = half * 64; tt < half * 64 + 64; tt += 16) {
          uint32_t hi[8], lo[8];
          const float *w = tbl + 128 + nt - 1 - tt;
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            const uint32_t ka = *reinterpret_cast<const uint16_t *>(kcol + (tt + e) * 128 + ((ch ^ (e & 7)) << 4));
            const uint32_t kb = *reinterpret_cast<const uint16_t *>(kcol + (tt + e + 1) * 128 + ((ch ^ ((e + 1) & 7)) << 4));
            const float fa = tt + e < nt ? __uint_as_float(ka << 16) * w[-e] : 0.f;
            const float fb = tt + e + 1 < nt ? __uint_as_float(kb << 16) * w[-e - 1] : 0.f;
            const uint32_t h = lt_pack(fa, fb);
            hi[e >> 1] = h;
            lo[e >> 1] = lt_pack(fa - __uint_as_float(h << 16), fb - __uint_as_float(h & 0xffff0000u));
          }
          tmem_st8(tl + kLtColKH + (uint32_t)(tt >> 1), hi);
          tmem_st8(tl + kLtColKL + (uint32_t)(tt >> 1), lo);
        }
        tmem_st_wait();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(kp_ready);
    }
    if (n > 0) add_ds(n - 1, Decay2(decay_pow(logd, tail)));
    if (mine && (kStates || seg == p.segments - 1)) {
      float *dst = kStates ? part + (size_t)(seg + 1) * D * D : S;
#pragma unroll
      for (int x = 0; x < kHalfCols; x += 4)
        *reinterpret_cast<float4 *>(dst + x) = make_float4(s[x], s[x + 1], s[x + 2], s[x + 3]);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, kLtTmemCols);
}

template <int D>
roco_status linear_prefill_tc_t(const LinearParams &p, int U, cudaStream_t stream) {
  CUtensorMap mq, mk, mv, mo;
  if (!make_tensor_map_units_bf16(&mq, p.Q, U, p.Lmax, D, kLtChunk) || !make_tensor_map_units_bf16(&mk, p.K, U, p.Lmax, D, kLtChunk) ||
      !make_tensor_map_units_bf16(&mv, p.V, U, p.Lmax, D, kLtChunk) || !make_tensor_map_units_bf16(&mo, p.out, U, p.Lmax, D, kLtChunk))
    return ROCO_ERR_CUDA;
  auto states = linear_prefill_tc_kernel<D, true>;
  auto whole = linear_prefill_tc_kernel<D, false>;
  constexpr size_t kB1 = LtSmem<D>::bytes(true), kB0 = LtSmem<D>::bytes(false);
  if (cudaFuncSetAttribute(states, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kB1) != cudaSuccess ||
      cudaFuncSetAttribute(whole, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kB0) != cudaSuccess)
    return ROCO_ERR_CUDA;
  if (p.segments > 1) states<<<(unsigned)U * (unsigned)(p.segments - 1), kLtThreads, kB1, stream>>>(mq, mk, mv, mo, p);
  whole<<<(unsigned)U * (unsigned)p.segments, kLtThreads, kB0, stream>>>(mq, mk, mv, mo, p);
  return cudaGetLastError() == cudaSuccess ? ROCO_OK : ROCO_ERR_CUDA;
}

int linear_tc_segments(int U, int Lmax, int sms) {
  const int most = Lmax / (4 * kLtChunk);
  int n = sms / U;
  if (n > most) n = most;
  if (n > 64) n = 64;
  return n < 2 ? 1 : n;
}

roco_status launch_linear_prefill_tc(const LinearParams &p, int d, int U, cudaStream_t stream) {
  return d == 128 ? linear_prefill_tc_t<128>(p, U, stream) : linear_prefill_tc_t<64>(p, U, stream);
}

}  // namespace roco
