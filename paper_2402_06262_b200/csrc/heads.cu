// Queries, keys and values of a layer out of its projections: norm of each head, rotation by position, layout by unit.
//
// A stream: every element is read once and written once, 2 d e bytes per head of a token, and that bounds it: 32768 tokens x 96 heads,
// bf16, d 128, take 239 us (6.1 TB/s, 0.94 of the measured copy rate; a plain copy of these bytes takes 229).
//
// A row (the head of one token) is held by d e / 32 lanes with two 16-byte pieces each.  For pairs (i, i + rot/2) the two pieces are
// the two halves of the same pairs, so the rotation needs no exchange between lanes, and the norm a butterfly over 4 to 16 lanes.  A
// thread keeps its place in the row and its token and goes through a range of heads: sines and cosines are formed once for all
// of them, and four rows are fetched together (two 279 us, three 251, six 277, eight 263; fetching two while two are worked on 288).
// Neighbouring rows of a CTA are neighbouring tokens, which follow one another in the unit layout: what is read as rows of the
// projections leaves as blocks of 8 to 32 tokens per head.  128 threads (64: 262 us, 256: 299), five CTAs per SM by their registers.
// A small call is a chain of latencies (8 tokens x 96 heads 3.5 us in a graph): positions, frequencies, weights and the first rows are
// all under way before any of them is needed.
#include "decoding.cuh"

namespace roco {
namespace {

constexpr int kThreads = 128;
constexpr int kFlight = 4;  // rows of a thread that are fetched together

// Cosine and sine of position * freq, formed in turns and without its whole turns in 64 bits: off by 2^-52 of itself, which for a
// position of 2^32 and a radian per step is less than 2e-7 of a turn.
__device__ __forceinline__ void angle(double position, float freq, float &c, float &s) {
  const double turns = position * ((double)freq * 0.15915494309189533577);
  sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
}

__device__ __forceinline__ void rotate(float &a, float &b, float c, float s) {
  const float x = a * c - b * s;
  b = b * c + a * s;
  a = x;
}

__device__ __forceinline__ uint4 pack(const float (&f)[4]) {
  return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 x = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&x);
}
__device__ __forceinline__ uint4 pack(const float (&f)[8]) {
  return make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
}

// Heads h .. end - 1 of one kind (queries, keys, values) in a CTA's range.
struct Run {
  int kind, first, end;  // first: number of the kind's first head
};
__device__ __forceinline__ Run run_from(const HeadsParams &p, int h, int last) {
  const int q_heads = p.G * p.group;
  Run r;
  r.kind = h < q_heads ? 0 : h < q_heads + p.G ? 1 : 2;
  r.first = r.kind == 0 ? 0 : r.kind == 1 ? q_heads : q_heads + p.G;
  r.end = min(last, r.kind == 0 ? q_heads : r.first + p.G);
  return r;
}

template <typename T, int D, bool kAdjacent>
__global__ void __launch_bounds__(kThreads) norm_rotate_kernel(const HeadsParams p) {
  constexpr int E = Elem<T>::kPerChunk, kLanes = D / E / 2, kRows = kThreads / kLanes;
  constexpr int kRowBytes = D * (int)sizeof(T);
  const int lane = threadIdx.x % kLanes;
  const unsigned token = blockIdx.x * kRows + threadIdx.x / kLanes;  // (there are fewer than 2^31)
  int b = 0, n = 0, len = 0;
  const bool real = token < (unsigned)p.S * (unsigned)p.N;
  if (real) {
    b = (int)(token / (unsigned)p.N);
    n = (int)(token - (unsigned)b * (unsigned)p.N);
    len = p.lens ? p.lens[b] : p.N;
  }
  // where the two pieces lie in the row, and what turns their pairs
  const int half = p.rot / 2 / E;  // pieces in half of the rotated elements
  int at[2];
  bool turn[2];
  if (kAdjacent) {
    at[0] = lane;
    at[1] = lane + kLanes;
    turn[0] = at[0] * E < p.rot;
    turn[1] = at[1] * E < p.rot;
  } else {
    turn[0] = turn[1] = lane < half;
    at[0] = lane < half ? lane : 2 * half + 2 * (lane - half);
    at[1] = lane < half ? lane + half : at[0] + 1;
  }
  float c[E], s[E];  // the frequencies at first
  int steps[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int piece = kAdjacent ? 2 * e / E : 0;
    const int pair = kAdjacent ? at[piece] * (E / 2) + e % (E / 2) : at[0] * E + e;
    c[e] = real && turn[piece] ? p.freq[pair] : 0.f;
    int axis = real && turn[piece] && p.axis ? p.axis[pair] : 0;
    if (axis < 0 || axis >= p.axes) {
      if (token == 0 && blockIdx.y == 0) atomicOr(p.status, ROCO_DEV_BAD_MAP);
      axis = 0;
    }
    steps[e] = !real ? 0 : p.positions ? p.positions[(long long)token * p.axes + axis] : n;
  }
  const double start = real && p.start ? (double)p.start[(long long)b * p.start_stride] : 0.0;

  const int last = min((int)(blockIdx.y + 1) * p.heads, p.G * (p.group + 2));
  int h = blockIdx.y * p.heads;
  Run run = run_from(p, h, last);
  uint4 raw[kFlight][2];
  auto fetch = [&](bool on) {
    const char *in = p.in[run.kind] + b * p.seq[run.kind] + n * p.row[run.kind] + (long long)(h - run.first) * kRowBytes;
    on = on && p.in[run.kind];
#pragma unroll
    for (int r = 0; r < kFlight; ++r)
      if (on && h + r < run.end) {
        const uint4 *src = reinterpret_cast<const uint4 *>(in + r * kRowBytes);
        raw[r][0] = __ldg(src + at[0]);
        raw[r][1] = __ldg(src + at[1]);
      }
  };
  // Of a call that is a chain of latencies the first rows are under way before the length is here.
  if (p.ahead) fetch(real);
  float w[2][E];
  auto fetch_weight = [&]() {
    const float *weight = run.kind < 2 ? p.weight[run.kind] : nullptr;
    if (weight) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) w[i][e] = __ldg(weight + at[i] * E + e);
    }
    return weight != nullptr;
  };
  bool normed = fetch_weight();
  if (len < 0 || len > p.N) {
    if (n == 0 && lane == 0 && blockIdx.y == 0) atomicOr(p.status, ROCO_DEV_BAD_LENS);
    len = 0;
  }
  const bool on = n < len;
  if (!__syncthreads_or(on)) return;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    s[e] = 0.f;
    if (turn[kAdjacent ? 2 * e / E : 0]) angle(start + (double)steps[e], c[e], c[e], s[e]);
  }

  bool here = p.ahead;
  while (true) {
    if (!here) fetch(on);
    here = false;
    const int per = run.kind == 0 ? p.group : 1;
    char *out = p.out[run.kind] + (((long long)b * p.G * p.N + n) * per) * kRowBytes;
    if (p.in[run.kind]) {
#pragma unroll
      for (int r = 0; r < kFlight; ++r) {
        if (h + r >= run.end) break;
        if (run.kind < 2) {
          float x[2][E];
          Elem<T>::unpack(raw[r][0], x[0]);
          Elem<T>::unpack(raw[r][1], x[1]);
          if (normed) {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) sum = fmaf(x[0][e], x[0][e], fmaf(x[1][e], x[1][e], sum));
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            const float norm = rsqrtf(sum * (1.f / D) + p.eps);
#pragma unroll
            for (int e = 0; e < E; ++e) {
              x[0][e] = x[0][e] * norm * w[0][e];
              x[1][e] = x[1][e] * norm * w[1][e];
            }
          }
          if (kAdjacent) {
#pragma unroll
            for (int e = 0; e < E; e += 2) {
              if (turn[0]) rotate(x[0][e], x[0][e + 1], c[e / 2], s[e / 2]);
              if (turn[1]) rotate(x[1][e], x[1][e + 1], c[E / 2 + e / 2], s[E / 2 + e / 2]);
            }
          } else if (turn[0]) {
#pragma unroll
            for (int e = 0; e < E; ++e) rotate(x[0][e], x[1][e], c[e], s[e]);
          }
          raw[r][0] = pack(x[0]);
          raw[r][1] = pack(x[1]);
        }
        if (on) {
          const int head = h + r - run.first, g = head / per, j = head - g * per;
          uint4 *dst = reinterpret_cast<uint4 *>(out + ((long long)g * p.N * per + j) * kRowBytes);
          dst[at[0]] = raw[r][0];
          dst[at[1]] = raw[r][1];
        }
      }
    }
    h = min(h + kFlight, run.end);
    if (h >= last) break;
    if (h == run.end) {
      run = run_from(p, h, last);
      normed = fetch_weight();
    }
  }
}

template <typename T, int D>
roco_status launch_t(HeadsParams p, int pairing, int sms, cudaStream_t stream) {
  constexpr int kRows = kThreads / (D / Elem<T>::kPerChunk / 2);
  const long long tokens = (long long)p.S * p.N;
  const long long tiles = (tokens + kRows - 1) / kRows;
  const int all = p.G * (p.group + 2);
  // CTAs that share a tile of tokens: a head each where all of them reside together.  Else, as each forms the tile's sines and cosines
  // anew, which costs as much as kSetup heads, and of more than one wave the last is half full on average, the time is about
  // (waves + 1/2) (heads per CTA + kSetup) (1180 tokens x 400 heads: ten CTAs, one wave, 44 us; 6, 13 and 30 take 56, 54 and 47; 32768 tokens
  // x 96 heads: three 239 us, one and six 246; 6002 x 40 heads, fp32, d 64: two 20.5 us, one and seven 26.5 and 22).
  // (CTAs per SM by their registers: five in bf16, six in single precision; adjacent pairs there would allow seven, which is not told apart)
  constexpr double kSetup = 3.0, kResident = sizeof(T) == 2 ? 5.0 : 6.0;
  const double slots = kResident * sms;
  int parts = all;
  if ((double)tiles * all > slots) {
    double best = 0.0;
    for (int n = 1; n <= all && n <= 128; ++n) {
      const double waves = (double)tiles * n / slots;
      const double cost = (waves > 1.0 ? waves + 0.5 : 1.0) * ((all + n - 1) / n + kSetup);
      if (n == 1 || cost < best) {
        best = cost;
        parts = n;
      }
    }
  }
  p.heads = (all + parts - 1) / parts;
  p.ahead = p.heads <= kFlight;
  parts = (all + p.heads - 1) / p.heads;
  if (tokens > 0x7fffffffLL - kRows) return ROCO_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)tiles, (unsigned)parts);
  if (pairing == ROCO_PAIR_ADJACENT) norm_rotate_kernel<T, D, true><<<grid, kThreads, 0, stream>>>(p);
  else norm_rotate_kernel<T, D, false><<<grid, kThreads, 0, stream>>>(p);
  return cudaGetLastError() == cudaSuccess ? ROCO_OK : ROCO_ERR_CUDA;
}

}  // namespace

roco_status launch_norm_rotate(const HeadsParams &p, int dtype, int d, int pairing, int sms, cudaStream_t stream) {
  if (dtype == ROCO_BF16)
    return d == 128 ? launch_t<__nv_bfloat16, 128>(p, pairing, sms, stream) : launch_t<__nv_bfloat16, 64>(p, pairing, sms, stream);
  return d == 128 ? launch_t<float, 128>(p, pairing, sms, stream) : launch_t<float, 64>(p, pairing, sms, stream);
}

}  // namespace roco
