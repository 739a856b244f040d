// Linear attention with a decay for each head over a prompt on the fifth-generation tensor cores (bf16).
//
// In chunks of C = 128 tokens, with i, j counted inside the chunk and S the fp32 state before it:
//     out_i = scale * ( g^(i+1) q_i S + sum_{j <= i} g^(i-j) (q_i.k_j) v_j )
//     S    <- g^C S + sum_j (g^(C-1-j) k_j)^T v_j
// which is four products per chunk, issued by one elected lane of a converged warp, accumulators in tensor memory:
//     S1 = Q K^T              both operands as TMA wrote them
//     O  = Q bf16(S)          then, by the A warps, row i times scale g^(i+1)
//     O += P V                P = S1 with the decays and the scale as bf16, from tensor memory
//     DS = (K1 + K2 + K3)^T V K1 + K2 + K3 = g^(C-1-j) k_j as the sum of three bf16, from tensor memory
// Every power of the decay is at most 1, so nothing overflows however fast a head forgets.  The state itself stays in the
// registers of the B warps in fp32 from the first chunk to the last: a thread keeps half a row, adds DS and writes the row
// as the next chunk's operand.  Three bf16 carry the 24 bits of an fp32 key, so the state is as exact as one formed in
// fp32 (with two, 2.4e-6 of it were lost; with one, as much as bf16 loses).  Rounded to bf16 are the operands P and S of
// the output, which is bf16 itself.
//
// Warps: 0-7 (A) a token per tensor-memory lane, half of the columns each: P, the scaling of O, the output.  8-15 (B) a
// row of the state per lane: DS, the state.  Both split keys, 32 tokens at a time through two buffers: A the first half of
// the next chunk's while its product P V runs, B the other half behind its operand, so that the tensor cores never wait
// for keys.  16 TMA loads and stores (the output of a chunk is staged where its queries were), 17 the products.
//
// What bounds it.  A chunk at d = 128 moves 128 KiB through HBM (3.0 us at one SM's share of the measured copy rate) and
// takes 48 products of 128 x 128 x 16, 3200 cycles at the tensor cores' rate (67 a product).  They follow one another without
// a gap, at 127 cycles each: operands from shared memory (two per product for S1 and O, 8 KiB per 64 cycles, one for the
// others) share its ports with the tiles that arrive and leave, and the chip is at its power limit (1.97 GHz falls to 1.4
// within milliseconds, 1.0 kW).  1024 units x 8192 tokens: 2.07 ms, 800 Tflop/s and 4.2 TB/s at the same time, 0.65 of the
// copy rate (1.78 ms before the clock falls).  Two terms per key instead of three would be 8 percent faster at five times
// the error of the state (2.4e-6).
#include <cuda.h>

#include <type_traits>

#include "linear.cuh"
#include "tc.cuh"

namespace roco {

constexpr int kLtChunk = 128;
constexpr int kLtAWarps = 8, kLtBWarps = 8;
constexpr int kLtTmaWarp = kLtAWarps + kLtBWarps, kLtMmaWarp = kLtTmaWarp + 1;
constexpr int kLtThreads = (kLtMmaWarp + 1) * 32;
constexpr int kLtSplits = 3;          // bf16 terms of a decayed key
constexpr int kLtPiece = 32;          // tokens whose keys are split at a time
constexpr int kLtPieceCols = kLtSplits * kLtPiece / 2;
constexpr uint32_t kLtColS = 0, kLtColO = 128, kLtTmemCols = 512;

// What a launch that only forms states has room for besides: a buffer per piece of a chunk and two accumulators DS, so that
// no group waits for a product of the chunk it works on, and three slots of tiles.
template <bool kStates>
struct LtPlan {
  static constexpr int kSlots = kStates ? 3 : 2, kPieceBufs = kStates ? 4 : 2;
  static constexpr uint32_t kColK = kStates ? 256 : 384;
  __device__ static constexpr uint32_t col_ds(int c) { return kStates ? (uint32_t)(c & 1) * 128 : 256; }
  static_assert(kColK + kPieceBufs * kLtPieceCols <= kLtTmemCols, "tensor memory");
};

template <int D>
struct LtSmem {
  static constexpr int kTile = kLtChunk * D * 2;
  static constexpr int kSop = D * D * 2;
  static constexpr int kBars = 32;
  static constexpr int kTables = 256 + 128 + 32;
  static constexpr size_t bytes(bool states) {
    return 1024 + (size_t)kTile * 6 + (states ? 0 : kSop) + kTables * 4 + kBars * 8 + 16;
  }
};

__device__ __forceinline__ void tma_store_3d(const CUtensorMap *map, const void *src, int c0, int c1, int c2) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
               ::"l"(map), "r"(smem_u32(src)), "r"(c0), "r"(c1), "r"(c2)
               : "memory");
}
__device__ __forceinline__ uint32_t lt_pack(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t *>(&v);
}

__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint32_t lt_pack2(f32x2 v) {
  float a, b;
  unpack2(v, a, b);
  return lt_pack(a, b);
}
// Four 8 x 8 blocks of 16-bit elements, transposed: lane t gets of block m the elements (rows 2 (t & 3) and the next,
// column t >> 2), rows being what the addresses of lanes 8 m .. 8 m + 7 point to.
__device__ __forceinline__ void lt_ldsm_t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// 16 tensor-memory lanes x 8 columns: lane t writes row t >> 2 (r[0], r[2]) and 8 + (t >> 2) (r[1], r[3]), columns
// t & 3 (r[0], r[1]) and 4 + (t & 3).
__device__ __forceinline__ void lt_st_16x8(uint32_t taddr, const uint32_t (&r)[4]) {
  asm volatile("tcgen05.st.sync.aligned.16x128b.x2.b32 [%0], {%1, %2, %3, %4};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}

template <int D, bool kStates>
__global__ void __launch_bounds__(kLtThreads, 1)
    linear_prefill_tc_kernel(const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapK,
                             const __grid_constant__ CUtensorMap mapV, const __grid_constant__ CUtensorMap mapO,
                             const LinearParams p) {
  constexpr int kTile = LtSmem<D>::kTile, kBlock = kLtChunk * 128;  // a 64-column block of a tile: 128 rows of 128 bytes
  using Plan = LtPlan<kStates>;
  constexpr int kSlots = Plan::kSlots, kPieceBufs = Plan::kPieceBufs;
  constexpr int kHalfCols = D / 2;                                  // columns of the state or output a thread works on
  constexpr uint32_t kIdesc = (1u << 4) | (1u << 7) | (1u << 10) | (8u << 24);       // bf16, fp32 accumulator, M = 128
  constexpr uint32_t kIdescS = kIdesc | ((128u >> 3) << 17);                         // N = 128, both K-major
  constexpr uint32_t kIdescV = kIdesc | (((uint32_t)D >> 3) << 17) | (1u << 16);     // N = D, B with N contiguous
  extern __shared__ char lt_raw[];
  char *at = smem_align(lt_raw, 1024);
  char *kt = at; at += kSlots * kTile;
  char *vt = at; at += kSlots * kTile;
  char *qt = at; if (!kStates) at += 2 * kTile;
  char *sop = at; if (!kStates) at += LtSmem<D>::kSop;
  float *ptab = reinterpret_cast<float *>(at);  // ptab[128 + n] = scale g^n, 0 for n < 0
  float *ktab = ptab + 256;                     // ktab[x] = g^(127 - x)
  float *ctab = ktab + 128;                     // ctab[e] = g^(31 - e)
  at += LtSmem<D>::kTables * 4;
  uint64_t *bars = reinterpret_cast<uint64_t *>(at); at += LtSmem<D>::kBars * 8;
  uint64_t *full = bars, *kv_empty = bars + 3, *q_full = bars + 6;  // per slot: keys and values landed, used up; queries
  uint64_t *kp_ready = bars + 8, *kp_free = bars + 12;              // per piece buffer; per piece of a chunk
  uint64_t *ds_full = bars + 16, *ds_free = bars + 18;              // per chunk parity
  uint64_t *s1_full = bars + 20, *o1_full = bars + 21, *o_scaled = bars + 22, *o_full = bars + 23;
  uint64_t *o_free = bars + 24, *sop_ready = bars + 25, *staged = bars + 26;
  uint32_t *tmem_base = reinterpret_cast<uint32_t *>(at);
  int *abort_ptr = reinterpret_cast<int *>(at + 8);
  volatile int *abort_flag = abort_ptr;

  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);  // uniform for the compiler too, and so is what follows
  const int segs = kStates ? p.segments - 1 : p.segments, seg = blockIdx.x % segs, u = blockIdx.x / segs;
  const int len = __shfl_sync(0xffffffffu, linear_len(p, u / p.G, tid == 0 && seg == 0 && (kStates || p.segments == 1)), 0);
  if (len == 0) {
    if (!kStates) wait_for_launch_before();
    return;
  }
  const int n_chunks = (len + kLtChunk - 1) / kLtChunk;
  const int first = linear_segment(n_chunks, p.segments, seg), last = linear_segment(n_chunks, p.segments, seg + 1);
  const int n = last - first;
  const int tail = last == n_chunks ? len - (n_chunks - 1) * kLtChunk : kLtChunk;  // tokens of this segment's last chunk
  const double logd = (double)p.log_decay[u % p.G];

  if (tid == 0) {
    for (int i = 0; i < kSlots; ++i) { mbar_init(&full[i], 2); mbar_init(&kv_empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&q_full[i], 1); mbar_init(&ds_full[i], 1); mbar_init(&ds_free[i], kLtBWarps); }
    for (int i = 0; i < 4; ++i) { mbar_init(&kp_ready[i], kLtBWarps); mbar_init(&kp_free[i], 1); }
    mbar_init(s1_full, 1); mbar_init(o1_full, 1); mbar_init(o_scaled, kLtAWarps); mbar_init(o_full, 1);
    mbar_init(o_free, kLtAWarps); mbar_init(sop_ready, kLtBWarps); mbar_init(staged, kLtAWarps);
    *abort_ptr = 0;
    mbar_init_fence();
  }
  if (tid < 256) ptab[tid] = tid < 128 ? 0.f : (float)(decay_pow(logd, tid - 128) * (double)p.scale);
  else if (tid < 384) ktab[tid - 256] = (float)decay_pow(logd, 127 - (tid - 256));
  else if (tid < 416) ctab[tid - 384] = (float)decay_pow(logd, 31 - (tid - 384));
  if (warp == 0) {
    tmem_alloc(tmem_base, kLtTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_base;
  // Not before this CTA has its tensor memory: the second launch's CTAs take all of an SM's too, and wait for this launch
  // while they hold it.  One that came first would wait for a CTA that waits for its columns.  (At d = 64 the shared memory
  // of both fits an SM.)
  if (kStates) launch_dependents();

  // Keys of a piece of 32 tokens, times what is left of each token at the end of the chunk, as the sum of three bf16; by
  // eight warps: a lane quarter's 32 components each, 16 tokens each.  A register holds two neighbouring tokens.
  // (ldmatrix: lanes 8 m .. 8 m + 7 point to eight tokens' 16 bytes of 8 components; blocks 0 and 1 are 16 components of
  // the first eight tokens, 2 and 3 of the next eight.)
  const int lm_tok = ((lane >> 4) & 1) * 8 + (lane & 7), lm_ch = (lane >> 3) & 1;
  auto split_keys = [&](int c, int q) {
    const int wq = warp & 3, half = (warp >> 2) & 1, bf = q % kPieceBufs, nt = c == n - 1 ? tail : kLtChunk;
    const char *ktile = kt + c % kSlots * kTile + (wq >> 1) * kBlock;
    // the buffer's last piece is used up (one barrier per piece of a chunk, so that whoever waits on one waits for each of
    // its phases in turn)
    if (kPieceBufs == 4) {
      if (c > 0) mbar_wait_compact(&kp_free[q], (c - 1) & 1, abort_flag, p.status);
    } else if (c > 0 || q >= 2) {
      mbar_wait_compact(&kp_free[q ^ 2], (q >= 2 ? c : c - 1) & 1, abort_flag, p.status);
    }
    if (wq * 32 < D) {  // d = 64: the upper two lane quarters hold no rows
      const int t0 = q * kLtPiece + half * 16, tok = t0 + 2 * (lane & 3), tr = t0 + lm_tok;
      uint32_t r[2][4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int ch = (wq & 1) * 4 + 2 * h + lm_ch;
        lt_ldsm_t(smem_u32(ktile + tr * 128 + ((ch ^ (tr & 7)) << 4)), r[h]);
      }
      f32x2 w2[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int at = tok + 8 * x + kLtChunk - nt;
        w2[x] = pack2(ktab[min(at, kLtChunk - 1)], ktab[min(at + 1, kLtChunk - 1)]);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t k1[4], k2[4], k3[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const int x = m & 2;  // (blocks 2 and 3 are eight tokens further)
          if (nt < kLtChunk) {  // tokens behind the last may hold anything
            if (tok + 4 * x >= nt) r[h][m] &= 0xffff0000u;
            if (tok + 4 * x + 1 >= nt) r[h][m] &= 0x0000ffffu;
          }
          // cut, not rounded: the upper halves of an fp32, of what they leave, and of what those leave are all its 24 bits
          const f32x2 minus = pack2(-1.f, -1.f);
          f32x2 f = mul2(pack2u(r[h][m] << 16, r[h][m] & 0xffff0000u), w2[m >> 1]);
          float a, b;
          unpack2(f, a, b);
          k1[m] = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
          f = fma2(pack2u(__float_as_uint(a) & 0xffff0000u, __float_as_uint(b) & 0xffff0000u), minus, f);
          unpack2(f, a, b);
          k2[m] = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
          f = fma2(pack2u(__float_as_uint(a) & 0xffff0000u, __float_as_uint(b) & 0xffff0000u), minus, f);
          unpack2(f, a, b);
          k3[m] = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
        }
        const uint32_t to = tmem + ((uint32_t)(wq * 32 + 16 * h) << 16) + Plan::kColK + (uint32_t)(bf * kLtPieceCols + half * 8);
        lt_st_16x8(to, k1);
        lt_st_16x8(to + kLtPiece / 2, k2);
        lt_st_16x8(to + kLtPiece, k3);
      }
      tmem_st_wait();
    }
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(&kp_ready[bf]);
  };

  if (warp == kLtTmaWarp) {
    if (lane == 0) {
      for (int c = 0; c < n + 2; ++c) {
        const int sl = c % kSlots, row = (first + c) * kLtChunk;
        auto load = [&](char *tiles, int sl, const CUtensorMap *map, uint64_t *bar) {
          mbar_expect_tx(bar, kTile);
#pragma unroll
          for (int h = 0; h < D / 64; ++h) tma_load_3d(tiles + sl * kTile + h * kBlock, map, 64 * h, row, u, bar);
        };
        if (c < n) {
          if (c >= kSlots) mbar_wait_compact(&kv_empty[sl], (c / kSlots - 1) & 1, abort_flag, p.status);
          load(kt, sl, &mapK, &full[sl]);
          load(vt, sl, &mapV, &full[sl]);
        }
        if (!kStates) {
          // the output of the chunk before the last leaves its slot, which then takes the queries of this one (a partial
          // chunk is the segment's last and is written by the A warps)
          if (c >= 2 && !(c - 2 == n - 1 && tail < kLtChunk)) {
            mbar_wait_compact(staged, c & 1, abort_flag, p.status);
#pragma unroll
            for (int h = 0; h < D / 64; ++h) tma_store_3d(&mapO, qt + (c & 1) * kTile + h * kBlock, 64 * h, row - 2 * kLtChunk, u);
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
          }
          if (c < n) load(qt, c & 1, &mapQ, &q_full[c & 1]);
        }
      }
      if (!kStates) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
  } else if (warp == kLtMmaWarp) {
    // (The accumulators sit at fixed columns: the allocation is all of tensor memory.  The pieces are kept as a loop: the
    // roles' code together has to stay in the instruction cache.)
    auto tile = [&](char *tiles, int c) { return tiles + c % kSlots * kTile; };
    auto scores = [&](int c) {  // S1 (the product that read P from these columns was issued before it)
      const char *k = tile(kt, c), *q = qt + (c & 1) * kTile;
      mbar_wait_compact(&full[c % kSlots], (c / kSlots) & 1, abort_flag, p.status);
      if (c == n - 1 && tail < kLtChunk) {
        // rows behind the prompt may hold anything: their scores are multiplied by zero, and so are their values
        for (int w = lane; w < (kLtChunk - tail) * 8; w += 32) {
#pragma unroll
          for (int h = 0; h < D / 64; ++h) {
            if (!kStates) *reinterpret_cast<uint4 *>(tile(kt, c) + h * kBlock + tail * 128 + w * 16) = make_uint4(0u, 0u, 0u, 0u);
            *reinterpret_cast<uint4 *>(tile(vt, c) + h * kBlock + tail * 128 + w * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
        }
        fence_async_smem();
        __syncwarp();
      }
      if (!kStates) {
        mbar_wait_compact(&q_full[c & 1], (c >> 1) & 1, abort_flag, p.status);
        tc_fence_after();
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          const int off = (kk / 4) * kBlock + (kk % 4) * 32;
          umma_bf16_w(kLtColS, smem_desc_sw128(q + off), smem_desc_sw128(k + off), kIdescS, kk > 0 ? 1u : 0u);
        }
        umma_commit_w(s1_full);
      }
    };
    if (n > 0) scores(0);
    for (int c = 0; c < n; ++c) {
      const uint32_t par = c & 1;
      const char *v = tile(vt, c);
      // the accumulator's last sum has been read
      if (kStates ? c > 1 : c > 0) {
        const int cb = kStates ? c - 2 : c - 1;
        mbar_wait_compact(&ds_free[cb & 1], (cb >> 1) & 1, abort_flag, p.status);
      }
#pragma unroll 1
      for (int q4 = 0; q4 < 4; ++q4) {
        if (!kStates && q4 == 2) {
          mbar_wait_compact(sop_ready, par, abort_flag, p.status);
          if (c > 0) mbar_wait_compact(o_free, (c - 1) & 1, abort_flag, p.status);
          tc_fence_after();
          const char *q = qt + (c & 1) * kTile;
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)  // O = Q S
            umma_bf16_w(kLtColO, smem_desc_sw128(q + (kk / 4) * kBlock + (kk % 4) * 32),
                        smem_desc_sw128_mn(sop + kk * 2048, D * 128), kIdescV, kk > 0 ? 1u : 0u);
          umma_commit_w(o1_full);
        }
        // DS, a piece of 32 tokens
        mbar_wait_compact(&kp_ready[q4 % kPieceBufs], kPieceBufs == 4 ? c & 1 : (2 * c + (q4 >> 1)) & 1, abort_flag, p.status);
        tc_fence_after();
#pragma unroll
        for (int x = 0; x < 2 * kLtSplits; ++x)  // term x >> 1, tokens 16 (x & 1) .. of the piece
          umma_bf16_ts_w(Plan::col_ds(c), Plan::kColK + (uint32_t)(q4 % kPieceBufs * kLtPieceCols + 8 * x),
                         smem_desc_sw128_mn(v + (2 * q4 + (x & 1)) * 2048, kBlock), kIdescV, (q4 > 0 || x > 0) ? 1u : 0u);
        umma_commit_w(&kp_free[q4]);
      }
      umma_commit_w(&ds_full[c & 1]);
      if (!kStates) {
        mbar_wait_compact(o_scaled, par, abort_flag, p.status);  // and P, which the same warps wrote before
        tc_fence_after();
#pragma unroll
        for (int kk = 0; kk < 8; ++kk)  // O += P V
          umma_bf16_ts_w(kLtColO, kLtColS + (uint32_t)((kk >> 2) * 64 + (kk & 3) * 8),
                         smem_desc_sw128_mn(v + kk * 2048, kBlock), kIdescV, 1u);
        umma_commit_w(o_full);
      }
      umma_commit_w(&kv_empty[c % kSlots]);
      if (c + 1 < n) scores(c + 1);
    }
  } else if (warp < kLtAWarps) {
    // ---------------------------------------------------------------- A: scores and output, a token per lane
    if (kStates) {
      for (int c = 0; c < n; ++c) {
        mbar_wait_compact(&full[c % kSlots], (c / kSlots) & 1, abort_flag, p.status);
#pragma unroll 1
        for (int q = 2; q < 4; ++q) split_keys(c, q);
      }
    } else {
      const int wq = warp & 3, half = warp >> 2, i = wq * 32 + lane;
      const uint32_t tl = tmem + ((uint32_t)(wq * 32) << 16);
      const float inter = (float)(decay_pow(logd, i + 1) * (double)p.scale);
      const f32x2 inter2 = pack2(inter, inter);
#pragma unroll 1
      for (int c = -1; c < n; ++c) {
        if (c >= 0) {
          const uint32_t par = c & 1;
          mbar_wait_compact(s1_full, par, abort_flag, p.status);
          tc_fence_after();
#pragma unroll 1
          for (int cc = 0; cc < 2; ++cc) {
            const int j0 = half * 64 + cc * 32;
            uint32_t pk[16];
            if (wq * 32 + 31 < j0) {  // the whole block lies behind the diagonal
#pragma unroll
              for (int e = 0; e < 16; ++e) pk[e] = 0u;
            } else {
              uint32_t r[32];
              tmem_ld32_issue(tl + kLtColS + (uint32_t)j0, r);
              const float *w = ptab + 128 + i - j0;  // w[-e]: column j0 + e
              if (wq * 32 > j0) {  // wholly below the diagonal: one power per row times 32 that all rows share
                const float base = w[-31];
                const f32x2 b2 = pack2(base, base);
                tmem_ld_wait(r);
#pragma unroll
                for (int e = 0; e < 32; e += 4) {
                  const float4 c4 = *reinterpret_cast<const float4 *>(ctab + e);
                  pk[e >> 1] = lt_pack2(mul2(mul2(pack2(c4.x, c4.y), b2), pack2u(r[e], r[e + 1])));
                  pk[(e >> 1) + 1] = lt_pack2(mul2(mul2(pack2(c4.z, c4.w), b2), pack2u(r[e + 2], r[e + 3])));
                }
              } else {  // on it: a later token's score is left out, not multiplied by zero (it may have left fp32's range)
                tmem_ld_wait(r);
                auto weighted = [&](int e) { return j0 + e <= i ? __uint_as_float(r[e]) * w[-e] : 0.f; };
#pragma unroll
                for (int e = 0; e < 32; e += 2) pk[e >> 1] = lt_pack(weighted(e), weighted(e + 1));
              }
            }
            tmem_st16(tl + kLtColS + (uint32_t)(half * 64 + cc * 16), pk);
          }
          tmem_st_wait();
          mbar_wait_compact(o1_full, par, abort_flag, p.status);
          tc_fence_after();
          const uint32_t to = tl + kLtColO + (uint32_t)(half * kHalfCols);
#pragma unroll 1
          for (int x = 0; x < kHalfCols; x += 32) {
            uint32_t r[32];
            tmem_ld32_issue(to + (uint32_t)x, r);
            tmem_ld_wait(r);
            uint32_t a[16], b[16];
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
              float f0, f1;
              unpack2(mul2(pack2u(r[e], r[e + 1]), inter2), f0, f1);
              a[e] = __float_as_uint(f0); a[e + 1] = __float_as_uint(f1);
              unpack2(mul2(pack2u(r[e + 16], r[e + 17]), inter2), f0, f1);
              b[e] = __float_as_uint(f0); b[e + 1] = __float_as_uint(f1);
            }
            tmem_st16(to + (uint32_t)x, a);
            tmem_st16(to + (uint32_t)x + 16u, b);
          }
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(o_scaled);
        }
        if (c + 1 < n) {  // while the product P V runs: half of the next chunk's keys
          mbar_wait_compact(&full[(c + 1) % kSlots], ((c + 1) / kSlots) & 1, abort_flag, p.status);
#pragma unroll 1
          for (int q = 0; q < 2; ++q) split_keys(c + 1, q);
        }
        if (c >= 0) {
          const uint32_t par = c & 1;
          const uint32_t to = tl + kLtColO + (uint32_t)(half * kHalfCols);
          mbar_wait_compact(o_full, par, abort_flag, p.status);
          tc_fence_after();
          const bool partial = c == n - 1 && tail < kLtChunk;
          char *stage = qt + (c & 1) * kTile;  // the products that read the queries are complete
          char *orow = p.out + (((size_t)u * p.Lmax + (size_t)(first + c) * kLtChunk + i) * D) * 2;
#pragma unroll 1
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
              o.x = lt_pack(__uint_as_float(r[8 * e]), __uint_as_float(r[8 * e + 1]));
              o.y = lt_pack(__uint_as_float(r[8 * e + 2]), __uint_as_float(r[8 * e + 3]));
              o.z = lt_pack(__uint_as_float(r[8 * e + 4]), __uint_as_float(r[8 * e + 5]));
              o.w = lt_pack(__uint_as_float(r[8 * e + 6]), __uint_as_float(r[8 * e + 7]));
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
    }
  } else {
    // ---------------------------------------------------------------- B: the state, a row per lane
    const int wq = warp & 3, half = (warp >> 2) & 1, r0 = wq * 32 + lane;
    const bool mine = wq * 32 < D;
    const uint32_t tl = tmem + ((uint32_t)(wq * 32) << 16);
    float *S = p.state + ((size_t)u * D + r0) * D + half * kHalfCols;
    float *part = p.parts + ((size_t)u * p.segments * D + r0) * D + half * kHalfCols;
    f32x2 s[kHalfCols / 2];
#pragma unroll
    for (int x = 0; x < kHalfCols / 2; ++x) s[x] = pack2(0.f, 0.f);
    if (!kStates) wait_for_launch_before();  // the segments' states
    if (mine) {
      if (seg == 0) {
        const float *src = (kStates || p.segments == 1) ? S : part;
#pragma unroll
        for (int x = 0; x < kHalfCols; x += 4) {
          const float4 f = *reinterpret_cast<const float4 *>(src + x);
          s[x / 2] = pack2(f.x, f.y);
          s[x / 2 + 1] = pack2(f.z, f.w);
          if (kStates) *reinterpret_cast<float4 *>(part + x) = f;  // the second launch starts from this copy
        }
      } else if (!kStates) {
        for (int m = 1; m <= seg; ++m) {
          const float w = (float)decay_pow(logd, (double)(first - linear_segment(n_chunks, p.segments, m)) * kLtChunk);
          const float *src = part + (size_t)m * D * D;
#pragma unroll
          for (int x = 0; x < kHalfCols; x += 4) {
            const float4 f = *reinterpret_cast<const float4 *>(src + x);
            s[x / 2] = fma2(pack2(w, w), pack2(f.x, f.y), s[x / 2]);
            s[x / 2 + 1] = fma2(pack2(w, w), pack2(f.z, f.w), s[x / 2 + 1]);
          }
        }
      }
    }
    const Decay2 g_chunk(decay_pow(logd, kLtChunk)), g_tail(decay_pow(logd, tail));
    for (int c = 0; c <= n; ++c) {
      if (c < n) {
        mbar_wait_compact(&full[c % kSlots], (c / kSlots) & 1, abort_flag, p.status);
        if (kStates) {
#pragma unroll 1
          for (int q = 0; q < 2; ++q) split_keys(c, q);
        }
      }
      if (c > 0) {  // the state behind the chunk before
        mbar_wait_compact(&ds_full[(c - 1) & 1], ((c - 1) >> 1) & 1, abort_flag, p.status);
        tc_fence_after();
        if (mine) {
          const Decay2 &g = c == n ? g_tail : g_chunk;
          const f32x2 hi = pack2(g.hi, g.hi), lo = pack2(g.lo, g.lo);
#pragma unroll
          for (int x = 0; x < kHalfCols; x += 16) {
            uint32_t r[16];
            tmem_ld16(tl + Plan::col_ds(c - 1) + (uint32_t)(half * kHalfCols + x), r);
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
              f32x2 &v = s[(x + e) / 2];
              v = fma2(hi, v, fma2(lo, v, pack2u(r[e], r[e + 1])));
            }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0 && c < n) mbar_arrive(&ds_free[(c - 1) & 1]);
      }
      if (!kStates && c < n) {
        if (c > 0) mbar_wait_compact(o1_full, (c - 1) & 1, abort_flag, p.status);  // the operand before is used up
        if (mine) {
          // row r0 of the operand: 64 columns to a block of D rows of 128 bytes
          char *row = sop + r0 * 128;
#pragma unroll
          for (int x = 0; x < kHalfCols; x += 8) {
            const int col = half * kHalfCols + x, ch = (col & 63) >> 3;
            *reinterpret_cast<uint4 *>(row + (col >> 6) * (D * 128) + ((ch ^ (r0 & 7)) << 4)) =
                make_uint4(lt_pack2(s[x / 2]), lt_pack2(s[x / 2 + 1]), lt_pack2(s[x / 2 + 2]), lt_pack2(s[x / 2 + 3]));
          }
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(sop_ready);
#pragma unroll 1
        for (int q = 2; q < 4; ++q) split_keys(c, q);
      }
    }
    if (mine && (kStates || seg == p.segments - 1)) {
      float *dst = kStates ? part + (size_t)(seg + 1) * D * D : S;
#pragma unroll
      for (int x = 0; x < kHalfCols; x += 4) {
        float4 f;
        unpack2(s[x / 2], f.x, f.y);
        unpack2(s[x / 2 + 1], f.z, f.w);
        *reinterpret_cast<float4 *>(dst + x) = f;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, kLtTmemCols);
}

static_assert(LtSmem<128>::bytes(false) <= 227 * 1024, "shared memory");

template <int D>
roco_status linear_prefill_tc_t(const LinearParams &p, int U, cudaStream_t stream) {
  CUtensorMap mq, mk, mv, mo;
  if (!make_tensor_map_units_bf16(&mq, p.Q, U, p.Lmax, D, kLtChunk) || !make_tensor_map_units_bf16(&mk, p.K, U, p.Lmax, D, kLtChunk) ||
      !make_tensor_map_units_bf16(&mv, p.V, U, p.Lmax, D, kLtChunk) || !make_tensor_map_units_bf16(&mo, p.out, U, p.Lmax, D, kLtChunk))
    return ROCO_ERR_CUDA;
  auto states = linear_prefill_tc_kernel<D, true>;
  auto whole = linear_prefill_tc_kernel<D, false>;
  constexpr size_t kB1 = LtSmem<D>::bytes(true), kB0 = LtSmem<D>::bytes(false);
  static SmemLimit limit_states, limit_whole;
  if (!limit_states((const void *)states, kB1) || !limit_whole((const void *)whole, kB0)) return ROCO_ERR_CUDA;
  if (p.segments > 1) states<<<(unsigned)U * (unsigned)(p.segments - 1), kLtThreads, kB1, stream>>>(mq, mk, mv, mo, p);
  if (cudaGetLastError() != cudaSuccess) return ROCO_ERR_CUDA;
  const unsigned blocks = (unsigned)U * (unsigned)p.segments;
  if (p.segments > 1) return launch_overlapped(whole, blocks, kLtThreads, kB0, stream, mq, mk, mv, mo, p) ? ROCO_OK : ROCO_ERR_CUDA;
  whole<<<blocks, kLtThreads, kB0, stream>>>(mq, mk, mv, mo, p);
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
