// Linear attention with a decay for each head on the CUDA cores: the single-token step (any dtype) and the prompt pass in
// single precision (bf16: linear_tc.cu).
//
//     state_t = g state_{t-1} + k_t v_t^T,     out_t = scale * q_t state_t
//
// Column c of the state meets only component c of v and of the output, so a unit can be cut into slabs of columns that
// know nothing of one another.
#include "linear.cuh"

namespace roco {

constexpr int kLsThreads = 128;
constexpr int kLsCols = 32;  // columns of the state per CTA: 128-byte rows

// One CTA: 32 columns of a unit's state, eight threads (16 bytes each) across, sixteen rows at a time; every thread has
// all of its D / 16 loads in flight before it uses the first.  Reads and writes the state once: bound by that traffic (8192
// units x 128 x 128: 143 us, 6.6 TB/s; 32 units: 2.8 us, less than their launch).
template <typename T, int D>
__global__ void __launch_bounds__(kLsThreads) linear_step_kernel(const LinearParams p, const int *active) {
  constexpr int kSlabs = D / kLsCols, kRows = D / 16;
  __shared__ __align__(16) float red[kLsThreads / 32][kLsCols];
  const int u = blockIdx.x / kSlabs, c0 = (blockIdx.x % kSlabs) * kLsCols;
  if (active && active[u / p.G] == 0) return;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, col = (tid & 7) * 4, r0 = tid >> 3;
  float *S = p.state + (size_t)u * D * D + c0 + col;
  float4 s[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) s[i] = *reinterpret_cast<const float4 *>(S + (size_t)(r0 + 16 * i) * D);
  const T *q = reinterpret_cast<const T *>(p.Q) + (size_t)u * D, *k = reinterpret_cast<const T *>(p.K) + (size_t)u * D;
  const T *v = reinterpret_cast<const T *>(p.V) + (size_t)u * D + c0 + col;
  float kr[kRows], qr[kRows], vc[4];
#pragma unroll
  for (int i = 0; i < kRows; ++i) { kr[i] = Elem<T>::load(k + r0 + 16 * i); qr[i] = Elem<T>::load(q + r0 + 16 * i); }
#pragma unroll
  for (int e = 0; e < 4; ++e) vc[e] = Elem<T>::load(v + e);
  // The decay to 48 bits, as in the prompt pass: rounded to fp32 it would be off in one direction at every token, by
  // n 2^-25 of the state after n of them.
  const Decay2 g(decay_pow((double)p.log_decay[u % p.G], 1.0));
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    s[i].x = fmaf(g.hi, s[i].x, fmaf(kr[i], vc[0], g.lo * s[i].x));
    s[i].y = fmaf(g.hi, s[i].y, fmaf(kr[i], vc[1], g.lo * s[i].y));
    s[i].z = fmaf(g.hi, s[i].z, fmaf(kr[i], vc[2], g.lo * s[i].z));
    s[i].w = fmaf(g.hi, s[i].w, fmaf(kr[i], vc[3], g.lo * s[i].w));
    *reinterpret_cast<float4 *>(S + (size_t)(r0 + 16 * i) * D) = s[i];
    o.x = fmaf(qr[i], s[i].x, o.x);
    o.y = fmaf(qr[i], s[i].y, o.y);
    o.z = fmaf(qr[i], s[i].z, o.z);
    o.w = fmaf(qr[i], s[i].w, o.w);
  }
#pragma unroll
  for (int d = 8; d < 32; d <<= 1) {  // lanes 8, 16, 24 apart hold other rows of the same columns
    o.x += __shfl_xor_sync(0xffffffffu, o.x, d);
    o.y += __shfl_xor_sync(0xffffffffu, o.y, d);
    o.z += __shfl_xor_sync(0xffffffffu, o.z, d);
    o.w += __shfl_xor_sync(0xffffffffu, o.w, d);
  }
  if (lane < 8) *reinterpret_cast<float4 *>(&red[warp][col]) = o;
  __syncthreads();
  if (tid < kLsCols) {
    float x = 0.f;
#pragma unroll
    for (int w = 0; w < kLsThreads / 32; ++w) x += red[w][tid];
    Elem<T>::store(reinterpret_cast<T *>(p.out) + (size_t)u * D + c0 + tid, x * p.scale);
  }
}

roco_status launch_linear_step(const LinearParams &p, const int *active, int dtype, int d, int U, cudaStream_t stream) {
  const unsigned grid = (unsigned)U * (unsigned)(d / kLsCols);
  if (dtype == ROCO_BF16) {
    if (d == 128) linear_step_kernel<__nv_bfloat16, 128><<<grid, kLsThreads, 0, stream>>>(p, active);
    else linear_step_kernel<__nv_bfloat16, 64><<<grid, kLsThreads, 0, stream>>>(p, active);
  } else {
    if (d == 128) linear_step_kernel<float, 128><<<grid, kLsThreads, 0, stream>>>(p, active);
    else linear_step_kernel<float, 64><<<grid, kLsThreads, 0, stream>>>(p, active);
  }
  return cudaGetLastError() == cudaSuccess ? ROCO_OK : ROCO_ERR_CUDA;
}

// ---------------------------------------------------------------- prompt pass

constexpr int kLpThreads = 128;
constexpr int kLpChunk = 32;  // tokens of a chunk
constexpr int kLpCols = 64;   // columns of the state per CTA
constexpr int kLpSegments = 64;

__device__ __forceinline__ void madd4(float4 &o, float w, const float4 &x) {
  o.x = fmaf(w, x.x, o.x); o.y = fmaf(w, x.y, o.y); o.z = fmaf(w, x.z, o.z); o.w = fmaf(w, x.w, o.w);
}

template <int D>
struct LpSmem {
  float q[kLpChunk][D + 4], k[kLpChunk][D + 4];  // pitch: eight rows read at once lie in different banks
  float v[kLpChunk][kLpCols], s[D][kLpCols];
  float p[kLpChunk][kLpChunk + 4];
  float pw[kLpChunk + 1];                        // g^n
  float seg_w[kLpSegments];                      // what is left of the state behind segment m - 1 at this one's start
};

// In chunks of 32 tokens, with i, j counted inside the chunk and S the state before it:
//     out_i  = g^(i+1) q_i S + sum_{j <= i} g^(i-j) (q_i.k_j) v_j
//     S     <- g^32 S + sum_j g^(31-j) k_j^T v_j
// Three small matrix products per chunk in place of 32 dependent updates of the state.  A CTA has 64 columns of one
// unit's state (registers; a copy in shared memory is the operand of the first product) and one segment of the prompt.
// All powers are at most 1: nothing overflows however fast the head forgets.  A thread forms four tokens by four columns, eight
// products per value read: shared memory's ports bound it (24 units x 777 tokens x 64: 28.7 us; one token by eight columns 40).
//
// Segments (few units): a first launch (kStates) runs every segment but the last and leaves its state in `parts`:
// segment 0's (which starts from the unit's state) in slot 1, the others', started from zero, in the slot behind their
// index; slot 0 takes a copy of the unit's state, which the second launch overwrites at a time of its own.  The second
// launch starts segment i > 0 from  g^(t_i - t_1) slot_1 + sum_{m=1}^{i-1} g^(t_i - t_{m+1}) slot_{m+1}.
template <int D, bool kStates>
__global__ void __launch_bounds__(kLpThreads) linear_prefill_simt_kernel(const LinearParams p) {
  constexpr int kSlabs = D / kLpCols, kRows = D * 16 / kLpThreads;
  constexpr int kEPC = 4;  // elements of a 16-byte piece
  extern __shared__ __align__(16) char lp_raw[];
  LpSmem<D> &sm = *reinterpret_cast<LpSmem<D> *>(lp_raw);
  const int tid = threadIdx.x;
  const int slab = blockIdx.x % kSlabs, segs = kStates ? p.segments - 1 : p.segments;
  const int seg = blockIdx.x / kSlabs % segs, u = blockIdx.x / (kSlabs * segs), c0 = slab * kLpCols;
  if (kStates) launch_dependents();
  const int len = linear_len(p, u / p.G, tid == 0 && slab == 0 && seg == 0 && (kStates || p.segments == 1));
  if (len == 0) {
    if (!kStates) wait_for_launch_before();
    return;
  }
  const int n_chunks = (len + kLpChunk - 1) / kLpChunk;
  const int first = linear_segment(n_chunks, p.segments, seg), last = linear_segment(n_chunks, p.segments, seg + 1);
  const double logd = (double)p.log_decay[u % p.G];
  if (tid <= kLpChunk) sm.pw[tid] = (float)decay_pow(logd, tid);
  else if (!kStates && tid >= 64 && tid - 64 <= seg)
    sm.seg_w[tid - 64] = (float)decay_pow(logd, (double)(first - linear_segment(n_chunks, p.segments, tid - 64)) * kLpChunk);
  const int sr0 = (tid >> 4) * kRows, sc = (tid & 15) * 4;  // this thread's rows and columns of the state
  float *S = p.state + (size_t)u * D * D + (size_t)sr0 * D + c0 + sc;
  float *part = p.parts + (size_t)u * p.segments * D * D + (size_t)sr0 * D + c0 + sc;
  float4 s[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) s[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  if (!kStates) {
    __syncthreads();
    wait_for_launch_before();  // the segments' states
  }
  if (seg == 0) {
    const float *src = (p.segments == 1 || kStates) ? S : part;
#pragma unroll
    for (int i = 0; i < kRows; ++i) s[i] = *reinterpret_cast<const float4 *>(src + (size_t)i * D);
    if (kStates) {
#pragma unroll
      for (int i = 0; i < kRows; ++i) *reinterpret_cast<float4 *>(part + (size_t)i * D) = s[i];
    }
  } else if (!kStates) {
#pragma unroll 4
    for (int m = 1; m <= seg; ++m) {
      const float w = sm.seg_w[m];
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const float4 x = *reinterpret_cast<const float4 *>(part + (size_t)m * D * D + (size_t)i * D);
        s[i].x = fmaf(w, x.x, s[i].x); s[i].y = fmaf(w, x.y, s[i].y);
        s[i].z = fmaf(w, x.z, s[i].z); s[i].w = fmaf(w, x.w, s[i].w);
      }
    }
  }
  const float *Q = reinterpret_cast<const float *>(p.Q) + (size_t)u * p.Lmax * D;
  const float *K = reinterpret_cast<const float *>(p.K) + (size_t)u * p.Lmax * D;
  const float *V = reinterpret_cast<const float *>(p.V) + (size_t)u * p.Lmax * D + c0;
  float *O = reinterpret_cast<float *>(p.out) + (size_t)u * p.Lmax * D + c0;
  const int row0 = (tid >> 4) * 4, col = sc;  // this thread's four tokens and four columns of the output
  const Decay2 g_chunk(decay_pow(logd, kLpChunk)), g_tail(decay_pow(logd, len - (n_chunks - 1) * kLpChunk));
  // A chunk's loads are issued while the one before is worked on.  Tokens behind the last are zeros: they add nothing to
  // the sums, and their own rows are not written.
  constexpr int kPieces = kLpChunk * D / kEPC / kLpThreads, kVPieces = kLpChunk * kLpCols / kEPC / kLpThreads;
  static_assert(kPieces >= 1 && kVPieces >= 1, "a piece of 16 bytes per thread");
  float4 qv[kPieces], kv[kPieces], vv[kVPieces];
  auto load = [&](int c) {
    const int t0 = c * kLpChunk;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int w = tid + i * kLpThreads, t = t0 + w / (D / kEPC), x = w % (D / kEPC) * kEPC;
      qv[i] = kv[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (t < len) {
        if (!kStates) qv[i] = *reinterpret_cast<const float4 *>(Q + (size_t)t * D + x);
        kv[i] = *reinterpret_cast<const float4 *>(K + (size_t)t * D + x);
      }
    }
#pragma unroll
    for (int i = 0; i < kVPieces; ++i) {
      const int w = tid + i * kLpThreads, t = t0 + w / (kLpCols / kEPC), x = w % (kLpCols / kEPC) * kEPC;
      vv[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (t < len) vv[i] = *reinterpret_cast<const float4 *>(V + (size_t)t * D + x);
    }
  };
  if (first < last) load(first);
#pragma unroll 1
  for (int c = first; c < last; ++c) {
    const int t0 = c * kLpChunk, nt = len - t0 < kLpChunk ? len - t0 : kLpChunk;
    __syncthreads();  // the chunk before is used up
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int w = tid + i * kLpThreads, t = w / (D / kEPC), x = w % (D / kEPC) * kEPC;
      if (!kStates) *reinterpret_cast<float4 *>(&sm.q[t][x]) = qv[i];
      *reinterpret_cast<float4 *>(&sm.k[t][x]) = kv[i];
    }
#pragma unroll
    for (int i = 0; i < kVPieces; ++i) {
      const int w = tid + i * kLpThreads;
      *reinterpret_cast<float4 *>(&sm.v[w / (kLpCols / kEPC)][w % (kLpCols / kEPC) * kEPC]) = vv[i];
    }
    if (c + 1 < last) load(c + 1);
    if (!kStates) {
#pragma unroll
      for (int i = 0; i < kRows; ++i) *reinterpret_cast<float4 *>(&sm.s[sr0 + i][sc]) = s[i];
    }
    __syncthreads();
    if (!kStates) {
      // four tokens, four columns; and of the scores the four tokens' with keys tid & 15 and 16 further
      float z[4][2];
      float4 o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        z[i][0] = z[i][1] = 0.f;
        o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll 2
      for (int x = 0; x < D; x += 4) {
        float4 q4[4], s4[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          q4[i] = *reinterpret_cast<const float4 *>(&sm.q[row0 + i][x]);
          s4[i] = *reinterpret_cast<const float4 *>(&sm.s[x + i][col]);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float4 k4 = *reinterpret_cast<const float4 *>(&sm.k[(tid & 15) + 16 * h][x]);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            z[i][h] = fmaf(q4[i].x, k4.x, fmaf(q4[i].y, k4.y, fmaf(q4[i].z, k4.z, fmaf(q4[i].w, k4.w, z[i][h]))));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          madd4(o[i], q4[i].x, s4[0]);
          madd4(o[i], q4[i].y, s4[1]);
          madd4(o[i], q4[i].z, s4[2]);
          madd4(o[i], q4[i].w, s4[3]);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int j = (tid & 15) + 16 * h, row = row0 + i;
          sm.p[row][j] = j <= row ? z[i][h] * sm.pw[row - j] : 0.f;
        }
        const float w = sm.pw[row0 + i + 1];
        o[i].x *= w; o[i].y *= w; o[i].z *= w; o[i].w *= w;
      }
      __syncwarp();  // a row's scores come from sixteen lanes of the same warp
#pragma unroll 1
      for (int j = 0; j <= row0; j += 4) {
        float4 v4[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v4[e] = *reinterpret_cast<const float4 *>(&sm.v[j + e][col]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 p4 = *reinterpret_cast<const float4 *>(&sm.p[row0 + i][j]);
          madd4(o[i], p4.x, v4[0]);
          madd4(o[i], p4.y, v4[1]);
          madd4(o[i], p4.z, v4[2]);
          madd4(o[i], p4.w, v4[3]);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (row0 + i < nt) {
          *reinterpret_cast<float4 *>(O + (size_t)(t0 + row0 + i) * D + col) =
              make_float4(o[i].x * p.scale, o[i].y * p.scale, o[i].z * p.scale, o[i].w * p.scale);
        }
      }
    }
    float4 add[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) add[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int t = 0; t < nt; ++t) {
      const float w = sm.pw[nt - 1 - t];
      float4 v4 = *reinterpret_cast<const float4 *>(&sm.v[t][sc]);
      v4.x *= w; v4.y *= w; v4.z *= w; v4.w *= w;
#pragma unroll
      for (int i = 0; i < kRows; i += 4) {
        const float4 k4 = *reinterpret_cast<const float4 *>(&sm.k[t][sr0 + i]);
        const float ks[4] = {k4.x, k4.y, k4.z, k4.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          add[i + e].x = fmaf(ks[e], v4.x, add[i + e].x); add[i + e].y = fmaf(ks[e], v4.y, add[i + e].y);
          add[i + e].z = fmaf(ks[e], v4.z, add[i + e].z); add[i + e].w = fmaf(ks[e], v4.w, add[i + e].w);
        }
      }
    }
    const Decay2 &g = nt == kLpChunk ? g_chunk : g_tail;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      s[i].x = g.madd(s[i].x, add[i].x); s[i].y = g.madd(s[i].y, add[i].y);
      s[i].z = g.madd(s[i].z, add[i].z); s[i].w = g.madd(s[i].w, add[i].w);
    }
  }
  if (kStates) part += (size_t)(seg + 1) * D * D;
  float *dst = kStates ? part : S;
  if (!kStates && seg != p.segments - 1) return;
#pragma unroll
  for (int i = 0; i < kRows; ++i) *reinterpret_cast<float4 *>(dst + (size_t)i * D) = s[i];
}

template <int D>
roco_status linear_prefill_simt_t(const LinearParams &p, int U, cudaStream_t stream) {
  constexpr int kSmem = (int)sizeof(LpSmem<D>);
  const unsigned slabs = (unsigned)U * (unsigned)(D / kLpCols);
  auto states = linear_prefill_simt_kernel<D, true>;
  auto whole = linear_prefill_simt_kernel<D, false>;
  static SmemLimit limit_states, limit_whole;
  if (!limit_states((const void *)states, kSmem) || !limit_whole((const void *)whole, kSmem)) return ROCO_ERR_CUDA;
  if (p.segments > 1) states<<<slabs * (unsigned)(p.segments - 1), kLpThreads, kSmem, stream>>>(p);
  if (cudaGetLastError() != cudaSuccess) return ROCO_ERR_CUDA;
  if (p.segments > 1)
    return launch_overlapped(whole, slabs * (unsigned)p.segments, kLpThreads, kSmem, stream, p) ? ROCO_OK : ROCO_ERR_CUDA;
  whole<<<slabs, kLpThreads, kSmem, stream>>>(p);
  return cudaGetLastError() == cudaSuccess ? ROCO_OK : ROCO_ERR_CUDA;
}

// Segments that fill the GPU with two CTAs per SM, none shorter than two chunks: a prompt that is divided is read
// twice (its keys and values), which pays only while SMs would be idle.
int linear_simt_segments(int U, int d, int Lmax, int sms) {
  const long long ctas = (long long)U * (d / kLpCols);
  long long n = 2LL * sms / ctas;
  const int most = Lmax / (2 * kLpChunk);
  if (n > most) n = most;
  if (n > kLpSegments) n = kLpSegments;
  return n < 2 ? 1 : (int)n;
}

roco_status launch_linear_prefill_simt(const LinearParams &p, int d, int U, cudaStream_t stream) {
  return d == 128 ? linear_prefill_simt_t<128>(p, U, stream) : linear_prefill_simt_t<64>(p, U, stream);
}

}  // namespace roco
