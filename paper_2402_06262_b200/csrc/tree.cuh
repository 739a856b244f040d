// Shared by the kernels of speculative decoding over the cache (attention of a tree of drafted tokens, commit of the
// accepted path): launch parameters, the tree's ancestor sets, the check of an accepted path.
#pragma once

#include "common.cuh"
#include "launch.h"

namespace roco {

struct TreeParams {
  const char *K, *V;
  const int *live;
  int *status;
  const char *Q, *k_new, *v_new;
  const int *parent, *nodes;
  char *out;
  float *lse;
  float *part_o, *part_ml;  // splits > 1, no cluster: [U][splits][rows][d] unnormalised outputs, [U][splits][rows][2] (max, sum)
  int B, T, group, G;
  int rows;    // T * group query rows of a unit; row i is head i % group of node i / group
  int splits;  // CTAs that share a unit's cached tokens
  int cluster;  // they are a cluster and join their results themselves
  float scale;
};

constexpr int kTreeMaxNodes = ROCO_TREE_MAX_NODES;

// Nodes of sequence b; a count outside [0, T] is none.
template <typename Params>
__device__ __forceinline__ int tree_nodes(const Params &p, int b, bool report) {
  const int n = p.nodes ? p.nodes[b] : p.T;
  if (n >= 0 && n <= p.T) return n;
  if (report) atomicOr(p.status, ROCO_DEV_BAD_TREE);
  return 0;
}

// Occupied slots of unit u, clipped to [0, B].
__device__ __forceinline__ int tree_live(const int *live, int u, int B, int *status, bool report) {
  const int n = live[u];
  if (n >= 0 && n <= B) return n;
  if (report) atomicOr(status, ROCO_DEV_BAD_LIVE);
  return n < 0 ? 0 : B;
}

// anc[i] = bit set of node i's ancestors and itself, by pointer doubling (six rounds for 64 nodes).  up: scratch.  Called by
// one warp, two nodes a lane; the others synchronise with it before they use the result.
__device__ __forceinline__ void tree_ancestors_warp(const TreeParams &p, int b, int n_nodes, unsigned long long *anc, int *up,
                                                    bool report) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = lane + 32 * h;
    int par = -1;
    if (i < n_nodes) {
      par = p.parent[(size_t)b * p.T + i];
      if (par < -1 || par >= i) {
        if (report) atomicOr(p.status, ROCO_DEV_BAD_TREE);
        par = -1;
      }
    }
    up[i] = par;
    anc[i] = i < n_nodes ? 1ull << i : 0ull;
  }
  __syncwarp();
#pragma unroll 1
  for (int round = 0; round < 6; ++round) {
    unsigned long long a[2];
    int to[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      a[h] = anc[lane + 32 * h];
      to[h] = up[lane + 32 * h];
      if (to[h] >= 0) {
        a[h] |= anc[to[h]];
        to[h] = up[to[h]];
      }
    }
    __syncwarp();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      anc[lane + 32 * h] = a[h];
      up[lane + 32 * h] = to[h];
    }
    __syncwarp();
  }
}

constexpr int kTreeMaxCluster = 8;  // CTAs of a cluster

__device__ __forceinline__ float ld_cluster_f32(uint32_t at) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void ld_cluster_vec(uint32_t at, float (&v)[2]) {
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v[0]), "=f"(v[1]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ld_cluster_vec(uint32_t at, float (&v)[4]) {
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(at) : "memory");
}

// The CTAs of a cluster join what each has found over its range of the cached tokens, for `rows` rows from row0 on: CTA `split`
// those of index split, split + splits, ..., a warp a row.  With m the largest reference of the parts,
//     o = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s.
// In the shared memory of each: o[row][D], at(row) a row's reference and l `to_sum` floats behind it.  Called by all threads of
// all CTAs.
template <typename T, int D, typename At>
__device__ __forceinline__ void tree_cluster_join(const TreeParams &p, int u, int row0, int rows, int split, int warp, int warps,
                                                  int lane, const float *o, At at, int to_sum) {
  cluster_sync_all();
  constexpr int kN = D / 32;
  for (int row = split + p.splits * warp; row < rows; row += p.splits * warps) {
    const float *mine = at(row);
    float ref = -INFINITY, sum = 0.f;
    if (lane < p.splits) {
      ref = ld_cluster_f32(map_to_rank(mine, lane));
      sum = ld_cluster_f32(map_to_rank(mine + to_sum, lane));
    }
    float v[kTreeMaxCluster][kN], acc[kN];
#pragma unroll
    for (int r = 0; r < kTreeMaxCluster; ++r) {
#pragma unroll
      for (int i = 0; i < kN; ++i) v[r][i] = 0.f;
      if (r < p.splits) ld_cluster_vec(map_to_rank(o + row * D + lane * kN, r), v[r]);
    }
    const float m = warp_max(ref), f = exp2f(ref - m);  // (an empty part: 0)
    const float l = warp_sum(f * sum), inv = 1.f / l;
#pragma unroll
    for (int i = 0; i < kN; ++i) acc[i] = 0.f;
#pragma unroll
    for (int r = 0; r < kTreeMaxCluster; ++r) {
      const float w = __shfl_sync(0xffffffffu, f, r);
#pragma unroll
      for (int i = 0; i < kN; ++i) acc[i] = fmaf(w, v[r][i], acc[i]);
    }
    const size_t to = (size_t)u * p.rows + row0 + row;
    T *out = reinterpret_cast<T *>(p.out) + to * D + lane * kN;
#pragma unroll
    for (int i = 0; i < kN; i += 2) {
      const float a = acc[i] * inv, b = acc[i + 1] * inv;
      if constexpr (sizeof(T) == 2) *reinterpret_cast<__nv_bfloat162 *>(out + i) = __floats2bfloat162_rn(a, b);
      else *reinterpret_cast<float2 *>(out + i) = make_float2(a, b);
    }
    if (lane == 0 && p.lse) p.lse[to] = (m + log2f(l)) * kLn2;
  }
  cluster_sync_all();  // the others have read this CTA's results
}

struct CommitParams {
  char *K, *V;
  float *s, *q;
  int *n, *pos, *live, *t_next, *status;
  const char *Q, *k_new, *v_new;
  const float *lse;
  const int *parent, *nodes, *path, *path_len;  // nodes: NULL where every sequence has T
  int *ev_slot, *ev_pos;
  int B, T, group, G, A, r, scope_mode;
  float scale;
};

// Length of sequence b's accepted path: 0 unless its nodes exist, path[0] hangs on the cached prefix and every next node on the
// one before, which has to be an earlier one (any other parent hung on the prefix when the tree was attended).  Called by one
// whole warp; every lane gets the length and lane m < a the node path[m].
__device__ __forceinline__ int commit_path(const CommitParams &p, int b, int lane, int &node, bool report) {
  int a = p.path_len[b];
  const int n_nodes = tree_nodes(p, b, report && lane == 0);
  bool ok = a >= 0 && a <= p.A;
  if (!ok) a = 0;
  node = lane < a ? p.path[(size_t)b * p.A + lane] : -1;
  const int before = __shfl_up_sync(0xffffffffu, node, 1);
  bool chain = true;
  if (lane < a) {
    const int from = lane ? before : -1;
    chain = node > from && node < n_nodes && p.parent[(size_t)b * p.T + node] == from;
  }
  ok = __all_sync(0xffffffffu, chain) && ok;
  if (!ok) {
    if (report && lane == 0) atomicOr(p.status, ROCO_DEV_BAD_TREE);
    a = 0;
  }
  return a;
}

}  // namespace roco
