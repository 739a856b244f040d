// Attention of a tree of drafted tokens over the cache on the CUDA cores (any supported dtype, head dimension and
// scale), and the kernel that joins the parts of a unit that several CTAs worked on.
#include "tree.cuh"

namespace roco {

constexpr int kTsKeys = 64;  // keys of a tile; the drafted nodes are one more tile

// R query rows a thread, sixteen threads a row: each forms four of the tile's 64 scores of its rows, then owns D / 16 of
// their output dimensions.
template <int D, int R>
struct TsShape {
  static constexpr int kThreads = R == 1 ? 256 : 128, kRows = kThreads / 16 * R;
  static constexpr int kPitch = D + 4;  // float4 reads of 16 different rows hit different banks
  static constexpr int kPPitch = kTsKeys + 4;
  static constexpr size_t kSmem = (size_t)(kRows * kPitch + kTsKeys * kPitch + kRows * kPPitch) * 4;
};

// One CTA: kRows query rows of a unit against one range of its cached tokens (the last range also against the drafted nodes), one
// pass with a running maximum and sum per row.  A key that a row does not see has probability zero; a drafted one is left out of
// the sums too, so what lies in its value does not matter.
// What bounds it: one row a thread, the latency of two or three tiles where the cache is short (16 units x 1001 tokens x 64, 5
// rows: 10.3 us); it reads 5 values from shared memory for 4 products, so its ports in long ones.  Four rows a thread: 8 for 16.
template <typename T, int D, int R>
__global__ void __launch_bounds__((TsShape<D, R>::kThreads)) tree_simt_kernel(const TreeParams p) {
  using Sh = TsShape<D, R>;
  constexpr int kThreads = Sh::kThreads, kRows = Sh::kRows, kPitch = Sh::kPitch, kPPitch = Sh::kPPitch;
  constexpr int kEPC = Elem<T>::kPerChunk;
  constexpr int kVec = D / 64;   // float4 pieces of the output per row and thread
  extern __shared__ __align__(16) float ts_smem[];
  float *sq = ts_smem, *skv = sq + kRows * kPitch, *sp = skv + kTsKeys * kPitch;
  __shared__ unsigned long long anc[kTreeMaxNodes];
  __shared__ int up[kTreeMaxNodes];
  launch_dependents();
  const int tid = threadIdx.x, row = (tid >> 4) * R, part = tid & 15;
  const int row_blocks = (p.rows + kRows - 1) / kRows;
  const int split = blockIdx.x % p.splits, rb = blockIdx.x / p.splits % row_blocks;
  const int u = blockIdx.x / (row_blocks * p.splits), b = u / p.G;
  const bool report = tid == 0 && rb == 0 && split == 0;
  const int n_nodes = tree_nodes(p, b, report);
  const int row0 = rb * kRows, n_rows = n_nodes * p.group - row0;
  if (n_rows <= 0) return;
  const int live = tree_live(p.live, u, p.B, p.status, report);
  const bool drafts = split == p.splits - 1;
  if (drafts && tid < 32) tree_ancestors_warp(p, b, n_nodes, anc, up, rb == 0);
  const bool busy = (tid >> 5) * 2 * R < n_rows;  // a row of this warp exists
  const T *Qu = reinterpret_cast<const T *>(p.Q) + ((size_t)u * p.rows + row0) * D;
  for (int w = tid; w < kRows * D / kEPC; w += kThreads) {
    const int rr = w / (D / kEPC), c = w % (D / kEPC);
    float f[kEPC];
    uint4 x = make_uint4(0u, 0u, 0u, 0u);
    if (rr < n_rows) x = reinterpret_cast<const uint4 *>(Qu + (size_t)rr * D)[c];
    Elem<T>::unpack(x, f);
#pragma unroll
    for (int e = 0; e < kEPC; ++e) sq[rr * kPitch + c * kEPC + e] = f[e];
  }
  const int tiles = (live + kTsKeys - 1) / kTsKeys;
  // the drafted tokens are one more tile, the last one's
  const int t0 = (int)((long long)(tiles + 1) * split / p.splits), t_end = (int)((long long)(tiles + 1) * (split + 1) / p.splits);
  const float zscale = p.scale * kLog2e;
  float m[R], l[R];
  float4 acc[R][kVec];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < kVec; ++c) acc[i][c] = make_float4(0.f, 0.f, 0.f, 0.f);
  }

  // rows [0, count) of a key or value tile, the others zero; to shared memory as fp32
  constexpr int kPieces = kTsKeys * D / kEPC / kThreads, kBatch = kPieces < 8 ? kPieces : 8;
  auto fetch = [&](const T *src, int count, int i0, uint4 (&x)[kBatch]) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int w = tid + (i0 + i) * kThreads, j = w / (D / kEPC), c = w % (D / kEPC);
      x[i] = make_uint4(0u, 0u, 0u, 0u);
      if (j < count) x[i] = reinterpret_cast<const uint4 *>(src + (size_t)j * D)[c];
    }
  };
  auto stage = [&](int i0, const uint4 (&x)[kBatch]) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int w = tid + (i0 + i) * kThreads, j = w / (D / kEPC), c = w % (D / kEPC);
      float f[kEPC];
      Elem<T>::unpack(x[i], f);
#pragma unroll
      for (int e = 0; e < kEPC; e += 4)
        *reinterpret_cast<float4 *>(&skv[j * kPitch + c * kEPC + e]) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
    }
  };

#pragma unroll 1
  for (int t = t0; t < t_end; ++t) {
    const bool is_draft = t == tiles;
    const int count = is_draft ? n_nodes : (live - t * kTsKeys < kTsKeys ? live - t * kTsKeys : kTsKeys);
    const T *ks = is_draft ? reinterpret_cast<const T *>(p.k_new) + (size_t)u * p.T * D
                           : reinterpret_cast<const T *>(p.K) + ((size_t)u * p.B + (size_t)t * kTsKeys) * D;
    const T *vs = is_draft ? reinterpret_cast<const T *>(p.v_new) + (size_t)u * p.T * D
                           : reinterpret_cast<const T *>(p.V) + ((size_t)u * p.B + (size_t)t * kTsKeys) * D;
    // The first batch of the keys before the tile before is used up, the values' during the scores.
    uint4 x[kBatch], v[kBatch];
    fetch(ks, count, 0, x);
    if (R == 1) fetch(vs, count, 0, v);
    __syncthreads();  // (the first time: queries and ancestor sets are in place)
    stage(0, x);
#pragma unroll
    for (int i0 = kBatch; i0 < kPieces; i0 += kBatch) {
      fetch(ks, count, i0, x);
      stage(i0, x);
    }
    if (R > 1) fetch(vs, count, 0, v);
    __syncthreads();
    unsigned long long sees[R];
    float alpha[R];
    if (busy) {
      float z[R][4];
#pragma unroll
      for (int i = 0; i < R; ++i) {
        sees[i] = is_draft && row + i < n_rows ? anc[(row0 + row + i) / p.group] : 0ull;
#pragma unroll
        for (int k = 0; k < 4; ++k) z[i][k] = 0.f;
      }
#pragma unroll(R == 1 ? 4 : 2)
      for (int c = 0; c < D; c += 4) {
        float4 qv[R];
#pragma unroll
        for (int i = 0; i < R; ++i) qv[i] = *reinterpret_cast<const float4 *>(&sq[(row + i) * kPitch + c]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float4 kv = *reinterpret_cast<const float4 *>(&skv[(part + 16 * k) * kPitch + c]);
#pragma unroll
          for (int i = 0; i < R; ++i)
            z[i][k] = fmaf(qv[i].x, kv.x, fmaf(qv[i].y, kv.y, fmaf(qv[i].z, kv.z, fmaf(qv[i].w, kv.w, z[i][k]))));
        }
      }
#pragma unroll
      for (int i = 0; i < R; ++i) {
        float top = -INFINITY;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int j = part + 16 * k;
          const bool seen = j < count && (!is_draft || ((sees[i] >> j) & 1ull));
          z[i][k] = seen ? z[i][k] * zscale : -INFINITY;
          top = fmaxf(top, z[i][k]);
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const float m_new = fmaxf(m[i], top);
        const float ref = m_new == -INFINITY ? 0.f : m_new;
        alpha[i] = exp2f(m[i] - ref);  // 0 before the first seen key
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float e = exp2f(z[i][k] - ref);
          sp[(row + i) * kPPitch + part + 16 * k] = e;
          sum += e;
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        l[i] = fmaf(l[i], alpha[i], sum);
        m[i] = m_new;
      }
    }
    __syncthreads();  // the keys are used up, the probabilities in place
    stage(0, v);
#pragma unroll
    for (int i0 = kBatch; i0 < kPieces; i0 += kBatch) {
      fetch(vs, count, i0, v);
      stage(i0, v);
    }
    __syncthreads();
    if (!busy) continue;
#pragma unroll
    for (int i = 0; i < R; ++i) {
#pragma unroll
      for (int c = 0; c < kVec; ++c) {
        acc[i][c].x *= alpha[i]; acc[i][c].y *= alpha[i]; acc[i][c].z *= alpha[i]; acc[i][c].w *= alpha[i];
      }
    }
    auto add = [&](float4 &o, float w, const float4 &x4) {
      o = make_float4(fmaf(w, x4.x, o.x), fmaf(w, x4.y, o.y), fmaf(w, x4.z, o.z), fmaf(w, x4.w, o.w));
    };
    if (is_draft) {  // what a row does not see may be infinite or NaN
#pragma unroll 1
      for (int j = 0; j < count; ++j) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
          if ((sees[i] >> j) & 1ull) {
            const float pj = sp[(row + i) * kPPitch + j];
#pragma unroll
            for (int c = 0; c < kVec; ++c)
              add(acc[i][c], pj, *reinterpret_cast<const float4 *>(&skv[j * kPitch + c * 64 + part * 4]));
          }
        }
      }
    } else {
#pragma unroll(R == 1 ? 4 : 2)
      for (int j = 0; j < kTsKeys; j += 4) {  // (rows behind the last are zero)
        float pj[R][4];
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const float4 p4 = *reinterpret_cast<const float4 *>(&sp[(row + i) * kPPitch + j]);
          pj[i][0] = p4.x; pj[i][1] = p4.y; pj[i][2] = p4.z; pj[i][3] = p4.w;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
#pragma unroll
          for (int c = 0; c < kVec; ++c) {
            const float4 w = *reinterpret_cast<const float4 *>(&skv[(j + k) * kPitch + c * 64 + part * 4]);
#pragma unroll
            for (int i = 0; i < R; ++i) add(acc[i][c], pj[i][k], w);
          }
        }
      }
    }
  }
  if (p.cluster) {
    __syncthreads();  // the last values are used up
#pragma unroll
    for (int i = 0; i < R; ++i) {
#pragma unroll
      for (int c = 0; c < kVec; ++c) *reinterpret_cast<float4 *>(&skv[(row + i) * D + c * 64 + part * 4]) = acc[i][c];
      if (part == 0) {
        sp[(row + i) * kPPitch] = m[i];
        sp[(row + i) * kPPitch + 1] = l[i];
      }
    }
    tree_cluster_join<T, D>(p, u, row0, min(kRows, n_rows), split, tid >> 5, kThreads / 32, tid & 31, skv,
                            [&](int r) { return sp + r * kPPitch; }, 1);
    return;
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int grow = row0 + row + i;
    if (row + i >= n_rows) return;
    if (p.splits > 1) {
      const size_t at = ((size_t)u * p.splits + split) * p.rows + grow;
      if (part == 0) { p.part_ml[2 * at] = m[i]; p.part_ml[2 * at + 1] = l[i]; }
#pragma unroll
      for (int c = 0; c < kVec; ++c) *reinterpret_cast<float4 *>(p.part_o + at * D + c * 64 + part * 4) = acc[i][c];
      continue;
    }
    const size_t at = (size_t)u * p.rows + grow;
    const float inv = 1.f / l[i];  // a node sees itself: l > 0
    T *o = reinterpret_cast<T *>(p.out) + at * D;
#pragma unroll
    for (int c = 0; c < kVec; ++c) {
      const int d0 = c * 64 + part * 4;
      Elem<T>::store(o + d0, acc[i][c].x * inv);
      Elem<T>::store(o + d0 + 1, acc[i][c].y * inv);
      Elem<T>::store(o + d0 + 2, acc[i][c].z * inv);
      Elem<T>::store(o + d0 + 3, acc[i][c].w * inv);
    }
    if (p.lse && part == 0) p.lse[at] = (m[i] + log2f(l[i])) * kLn2;
  }
}

// Joins the parts of every row: with m the largest of the parts' maxima, o = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s.
// One warp per row; the parts of a row are few and still in L2.
constexpr int kTreeJoinWarps = 4;
template <typename T, int D>
__global__ void __launch_bounds__(kTreeJoinWarps * 32) tree_join_kernel(const TreeParams p, int U) {
  const long long w = (long long)blockIdx.x * kTreeJoinWarps + (threadIdx.x >> 5);
  wait_for_launch_before();
  if (w >= (long long)U * p.rows) return;
  const int lane = threadIdx.x & 31, u = (int)(w / p.rows), row = (int)(w % p.rows);
  if (row >= tree_nodes(p, u / p.G, false) * p.group) return;
  constexpr int kN = D / 32;
  float m = -INFINITY;
  const size_t first = (size_t)u * p.splits * p.rows + row;
  for (int s = lane; s < p.splits; s += 32) m = fmaxf(m, p.part_ml[2 * (first + (size_t)s * p.rows)]);
  m = warp_max(m);
  float l = 0.f, acc[kN];
#pragma unroll
  for (int c = 0; c < kN; ++c) acc[c] = 0.f;
#pragma unroll 4
  for (int s = 0; s < p.splits; ++s) {
    const size_t at = first + (size_t)s * p.rows;
    const float f = exp2f(p.part_ml[2 * at] - m);  // an empty part has maximum -inf and contributes nothing
    l = fmaf(f, p.part_ml[2 * at + 1], l);
    const float *o = p.part_o + at * D + lane * kN;
#pragma unroll
    for (int c = 0; c < kN; ++c) acc[c] = fmaf(f, o[c], acc[c]);
  }
  const float inv = 1.f / l;
  T *o = reinterpret_cast<T *>(p.out) + ((size_t)u * p.rows + row) * D + lane * kN;
#pragma unroll
  for (int c = 0; c < kN; ++c) Elem<T>::store(o + c, acc[c] * inv);
  if (p.lse && lane == 0) p.lse[(size_t)u * p.rows + row] = (m + log2f(l)) * kLn2;
}

template <typename T, int D>
roco_status tree_join_t(const TreeParams &p, int U, cudaStream_t stream) {
  const long long blocks = ((long long)U * p.rows + kTreeJoinWarps - 1) / kTreeJoinWarps;
  return launch_overlapped(tree_join_kernel<T, D>, (unsigned)blocks, kTreeJoinWarps * 32, 0, stream, p, U) ? ROCO_OK
                                                                                                           : ROCO_ERR_CUDA;
}

roco_status launch_tree_join_bf16(const TreeParams &p, int d, int U, cudaStream_t stream) {
  return d == 128 ? tree_join_t<__nv_bfloat16, 128>(p, U, stream) : tree_join_t<__nv_bfloat16, 64>(p, U, stream);
}

// One row a thread up to sixteen rows (64 units x 2048 tokens x 16 rows 114 us, with four rows a thread 134; 8 rows 76 and 110), else
// four (64 units x 8192 x 24 rows 453 us, with one 666; 4 units x 8192 x 512 rows 444 and 754).
int tree_simt_row_blocks(int rows) {
  constexpr int kRows = TsShape<64, 4>::kRows;
  return rows <= TsShape<64, 1>::kRows ? 1 : (rows + kRows - 1) / kRows;
}

template <typename T, int D, int R>
roco_status tree_simt_r(const TreeParams &p, int U, cudaStream_t stream) {
  using Sh = TsShape<D, R>;
  auto kernel = tree_simt_kernel<T, D, R>;
  static SmemLimit limit;
  if (!limit((const void *)kernel, Sh::kSmem)) return ROCO_ERR_CUDA;
  const unsigned grid = (unsigned)U * (unsigned)tree_simt_row_blocks(p.rows) * (unsigned)p.splits;
  if (p.cluster)
    return launch_cluster(kernel, grid, (unsigned)p.splits, Sh::kThreads, Sh::kSmem, stream, p) ? ROCO_OK : ROCO_ERR_CUDA;
  kernel<<<grid, Sh::kThreads, Sh::kSmem, stream>>>(p);
  if (cudaGetLastError() != cudaSuccess) return ROCO_ERR_CUDA;
  return p.splits > 1 ? tree_join_t<T, D>(p, U, stream) : ROCO_OK;
}

template <typename T, int D>
roco_status tree_simt_t(const TreeParams &p, int U, cudaStream_t stream) {
  return p.rows <= TsShape<D, 1>::kRows ? tree_simt_r<T, D, 1>(p, U, stream) : tree_simt_r<T, D, 4>(p, U, stream);
}

roco_status launch_tree_attend_simt(const TreeParams &p, int kv_dtype, int d, int U, cudaStream_t stream) {
  if (kv_dtype == ROCO_BF16)
    return d == 128 ? tree_simt_t<__nv_bfloat16, 128>(p, U, stream) : tree_simt_t<__nv_bfloat16, 64>(p, U, stream);
  return d == 128 ? tree_simt_t<float, 128>(p, U, stream) : tree_simt_t<float, 64>(p, U, stream);
}

}  // namespace roco
