// Shared by the kernels of linear attention with a decay for each head.
#pragma once

#include "common.cuh"
#include "launch.h"

namespace roco {

struct LinearParams {
  float *state;            // [U][d][d]
  const float *log_decay;  // [G]
  int *status;
  const char *Q, *K, *V;
  char *out;
  const int *lens;  // prompt pass only
  float *parts;     // segments > 1: [U][segments][d][d] states of the segments (see linear_segment)
  int G, Lmax;
  int segments;     // CTAs (times slabs) that share a unit's prompt
  float scale;
};

// g^n for n >= 0 in 64 bits: in fp32 the rounding of g alone would be off by n 2^-24 after n tokens.
// (Out of line: the exponential in 64 bits is long.)
static __device__ __noinline__ double decay_pow(double log_decay, double n) { return n == 0.0 ? 1.0 : exp(log_decay * n); }

// A factor as the sum of two floats, so that applying it thousands of times in a row does not drift.
struct Decay2 {
  float hi, lo;
  __device__ explicit Decay2(double x) : hi((float)x), lo((float)(x - (double)(float)x)) {}
  // *this * s + a
  __device__ __forceinline__ float madd(float s, float a) const { return fmaf(hi, s, fmaf(lo, s, a)); }
};

// Where a prompt is divided, its segments are whole chunks: segment i of a prompt of n chunks starts at this one.
__device__ __forceinline__ int linear_segment(int n_chunks, int segments, int i) {
  return (int)((long long)n_chunks * i / segments);
}

// Prompt length of sequence b; one outside [0, Lmax] is none.
__device__ __forceinline__ int linear_len(const LinearParams &p, int b, bool report) {
  const int n = p.lens[b];
  if (n >= 0 && n <= p.Lmax) return n;
  if (report) atomicOr(p.status, ROCO_DEV_BAD_LENS);
  return 0;
}

}  // namespace roco
