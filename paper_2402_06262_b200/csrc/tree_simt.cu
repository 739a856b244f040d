// Attention of a tree of drafted tokens over the cache on the CUDA cores (any supported dtype, head dimension and
// scale), and the kernel that joins the parts of a unit that several CTAs worked on.
#include "tree.cuh"

namespace roco {

constexpr int kTsThreads = 256;
constexpr int kTsRows = 16;  // query rows of a CTA
constexpr int kTsKeys = 64;  // keys of a tile; the drafted nodes are one more tile

// One CTA: kTsRows query rows of a unit against one range of its cached tokens (the last range also against the
// drafted nodes), one pass with a running maximum and sum per row.  Sixteen threads share a row: each forms four of the
// tile's 64 scores, then owns D / 16 of the row's output dimensions.  A key that a row does not see has probability
// zero; a drafted one is left out of the sums too, so what lies in its value does not matter.
// Bound by the latency of its two or three tiles where the cache is short (16 units x 1001 tokens x 64, 5 rows: 10.3 us), by
// shared memory's ports in long ones (5 reads of 16 bytes for 16 products).
template <typename T, int D>
__global__ void __launch_bounds__(kTsThreads) tree_simt_kernel(const TreeParams p) {
  constexpr int kPitch = D + 4;  // float4 reads of 16 different rows hit different banks
  constexpr int kEPC = Elem<T>::kPerChunk;
  constexpr int kVec = D / 64;   // float4 pieces of the output per thread
  __shared__ __align__(16) float sq[kTsRows * kPitch];
  __shared__ __align__(16) float skv[kTsKeys * kPitch];
  __shared__ __align__(16) float sp[kTsRows][kTsKeys + 4];
  __shared__ unsigned long long anc[kTreeMaxNodes];
  __shared__ int up[kTreeMaxNodes];
  launch_dependents();
  const int tid = threadIdx.x, row = tid >> 4, part = tid & 15;
  const int row_blocks = (p.rows + kTsRows - 1) / kTsRows;
  const int split = blockIdx.x % p.splits, rb = blockIdx.x / p.splits % row_blocks;
  const int u = blockIdx.x / (row_blocks * p.splits), b = u / p.G;
  const bool report = tid == 0 && rb == 0 && split == 0;
  const int n_nodes = tree_nodes(p, b, report);
  const int row0 = rb * kTsRows;
  if (row0 >= n_nodes * p.group) return;
  const int live = tree_live(p.live, u, p.B, p.status, report);
  const bool drafts = split == p.splits - 1;
  if (drafts && tid < 32) tree_ancestors_warp(p, b, n_nodes, anc, up, rb == 0);
  const int grow = row0 + row;
  const bool valid = grow < n_nodes * p.group;
  const bool busy = grow - (row & 1) < n_nodes * p.group;  // a row of this warp exists
  const T *Qu = reinterpret_cast<const T *>(p.Q) + (size_t)u * p.rows * D;
  for (int w = tid; w < kTsRows * D / kEPC; w += kTsThreads) {
    const int rr = w / (D / kEPC), c = w % (D / kEPC);
    float f[kEPC];
    uint4 x = make_uint4(0u, 0u, 0u, 0u);
    if (row0 + rr < n_nodes * p.group) x = reinterpret_cast<const uint4 *>(Qu + (size_t)(row0 + rr) * D)[c];
    Elem<T>::unpack(x, f);
#pragma unroll
    for (int e = 0; e < kEPC; ++e) sq[rr * kPitch + c * kEPC + e] = f[e];
  }
  const int tiles = (live + kTsKeys - 1) / kTsKeys;
  // the drafted tokens are one more tile, the last one's
  const int t0 = (int)((long long)(tiles + 1) * split / p.splits), t_end = (int)((long long)(tiles + 1) * (split + 1) / p.splits);
  const float zscale = p.scale * kLog2e;
  float m = -INFINITY, l = 0.f;
  float4 acc[kVec];
#pragma unroll
  for (int c = 0; c < kVec; ++c) acc[c] = make_float4(0.f, 0.f, 0.f, 0.f);

  // rows [0, count) of a key or value tile, the others zero; to shared memory as fp32
  constexpr int kPieces = kTsKeys * D / kEPC / kTsThreads;
  auto fetch = [&](const T *src, int count, uint4 (&x)[kPieces]) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int w = tid + i * kTsThreads, j = w / (D / kEPC), c = w % (D / kEPC);
      x[i] = make_uint4(0u, 0u, 0u, 0u);
      if (j < count) x[i] = reinterpret_cast<const uint4 *>(src + (size_t)j * D)[c];
    }
  };
  auto stage = [&](const uint4 (&x)[kPieces]) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int w = tid + i * kTsThreads, j = w / (D / kEPC), c = w % (D / kEPC);
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
    uint4 x[kPieces], v[kPieces];
    fetch(ks, count, x);
    fetch(vs, count, v);  // on their way during the scores
    __syncthreads();      // the tile before is used up (and, the first time, queries and ancestor sets are in place)
    stage(x);
    __syncthreads();
    unsigned long long sees = 0ull;
    float alpha = 1.f;
    if (busy) {
      if (is_draft && valid) sees = anc[grow / p.group];
      float z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
      for (int c = 0; c < D; c += 4) {
        const float4 qv = *reinterpret_cast<const float4 *>(&sq[row * kPitch + c]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float4 kv = *reinterpret_cast<const float4 *>(&skv[(part + 16 * k) * kPitch + c]);
          z[k] = fmaf(qv.x, kv.x, fmaf(qv.y, kv.y, fmaf(qv.z, kv.z, fmaf(qv.w, kv.w, z[k]))));
        }
      }
      float top = -INFINITY;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int j = part + 16 * k;
        const bool seen = j < count && (!is_draft || ((sees >> j) & 1ull));
        z[k] = seen ? z[k] * zscale : -INFINITY;
        top = fmaxf(top, z[k]);
      }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      const float m_new = fmaxf(m, top);
      const float ref = m_new == -INFINITY ? 0.f : m_new;
      alpha = exp2f(m - ref);  // 0 before the first seen key
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float e = exp2f(z[k] - ref);
        sp[row][part + 16 * k] = e;
        sum += e;
      }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      l = fmaf(l, alpha, sum);
      m = m_new;
    }
    __syncthreads();  // the keys are used up, the probabilities in place
    stage(v);
    __syncthreads();
    if (!busy) continue;
#pragma unroll
    for (int c = 0; c < kVec; ++c) { acc[c].x *= alpha; acc[c].y *= alpha; acc[c].z *= alpha; acc[c].w *= alpha; }
    if (is_draft) {  // what a row does not see may be infinite or NaN
#pragma unroll 2
      for (int j = 0; j < count; ++j) {
        if ((sees >> j) & 1ull) {
          const float pj = sp[row][j];
#pragma unroll
          for (int c = 0; c < kVec; ++c) {
            const float4 w = *reinterpret_cast<const float4 *>(&skv[j * kPitch + c * 64 + part * 4]);
            acc[c] = make_float4(fmaf(pj, w.x, acc[c].x), fmaf(pj, w.y, acc[c].y), fmaf(pj, w.z, acc[c].z), fmaf(pj, w.w, acc[c].w));
          }
        }
      }
    } else {
#pragma unroll 4
      for (int j = 0; j < kTsKeys; j += 4) {  // (rows behind the last are zero)
        const float4 p4 = *reinterpret_cast<const float4 *>(&sp[row][j]);
        const float pj[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
#pragma unroll
          for (int c = 0; c < kVec; ++c) {
            const float4 w = *reinterpret_cast<const float4 *>(&skv[(j + k) * kPitch + c * 64 + part * 4]);
            acc[c] = make_float4(fmaf(pj[k], w.x, acc[c].x), fmaf(pj[k], w.y, acc[c].y), fmaf(pj[k], w.z, acc[c].z),
                                 fmaf(pj[k], w.w, acc[c].w));
          }
        }
      }
    }
  }
  if (p.cluster) {
    __syncthreads();  // the last values are used up
#pragma unroll
    for (int c = 0; c < kVec; ++c) *reinterpret_cast<float4 *>(&skv[row * D + c * 64 + part * 4]) = acc[c];
    if (part == 0) { sp[row][0] = m; sp[row][1] = l; }
    tree_cluster_join<T, D>(p, u, row0, min(kTsRows, n_nodes * p.group - row0), split, tid >> 5, kTsThreads / 32, tid & 31, skv,
                            [&](int r) { return &sp[r][0]; }, 1);
    return;
  }
  if (!valid) return;
  if (p.splits > 1) {
    const size_t at = ((size_t)u * p.splits + split) * p.rows + grow;
    if (part == 0) { p.part_ml[2 * at] = m; p.part_ml[2 * at + 1] = l; }
#pragma unroll
    for (int c = 0; c < kVec; ++c) *reinterpret_cast<float4 *>(p.part_o + at * D + c * 64 + part * 4) = acc[c];
    return;
  }
  const size_t at = (size_t)u * p.rows + grow;
  const float inv = 1.f / l;  // a node sees itself: l > 0
  T *o = reinterpret_cast<T *>(p.out) + at * D;
#pragma unroll
  for (int c = 0; c < kVec; ++c) {
    const int d0 = c * 64 + part * 4;
    Elem<T>::store(o + d0, acc[c].x * inv);
    Elem<T>::store(o + d0 + 1, acc[c].y * inv);
    Elem<T>::store(o + d0 + 2, acc[c].z * inv);
    Elem<T>::store(o + d0 + 3, acc[c].w * inv);
  }
  if (p.lse && part == 0) p.lse[at] = (m + log2f(l)) * kLn2;
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

roco_status launch_tree_join(const TreeParams &p, int kv_dtype, int d, int U, cudaStream_t stream) {
  if (kv_dtype == ROCO_BF16)
    return d == 128 ? tree_join_t<__nv_bfloat16, 128>(p, U, stream) : tree_join_t<__nv_bfloat16, 64>(p, U, stream);
  return d == 128 ? tree_join_t<float, 128>(p, U, stream) : tree_join_t<float, 64>(p, U, stream);
}

int tree_simt_row_blocks(int rows) { return (rows + kTsRows - 1) / kTsRows; }

template <typename T, int D>
roco_status tree_simt_t(const TreeParams &p, int U, cudaStream_t stream) {
  const unsigned grid = (unsigned)U * (unsigned)tree_simt_row_blocks(p.rows) * (unsigned)p.splits;
  if (p.cluster)
    return launch_cluster(tree_simt_kernel<T, D>, grid, (unsigned)p.splits, kTsThreads, 0, stream, p) ? ROCO_OK : ROCO_ERR_CUDA;
  tree_simt_kernel<T, D><<<grid, kTsThreads, 0, stream>>>(p);
  if (cudaGetLastError() != cudaSuccess) return ROCO_ERR_CUDA;
  return p.splits > 1 ? tree_join_t<T, D>(p, U, stream) : ROCO_OK;
}

roco_status launch_tree_attend_simt(const TreeParams &p, int kv_dtype, int d, int U, cudaStream_t stream) {
  if (kv_dtype == ROCO_BF16)
    return d == 128 ? tree_simt_t<__nv_bfloat16, 128>(p, U, stream) : tree_simt_t<__nv_bfloat16, 64>(p, U, stream);
  return d == 128 ? tree_simt_t<float, 128>(p, U, stream) : tree_simt_t<float, 64>(p, U, stream);
}

}  // namespace roco
