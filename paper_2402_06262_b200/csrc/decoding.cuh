// Parameters of the norm and rotation of a layer's heads, of the verification of drafted trees and of the reordering of
// sequences.
#pragma once

#include "common.cuh"
#include "launch.h"

namespace roco {

struct HeadsParams {
  const char *in[3];              // q, k, v; nullptr: left out
  long long seq[3], row[3];       // strides in bytes: from a sequence to the next, from a token to the next
  char *out[3];                   // Q, K, V
  const int *lens, *start, *positions;
  int start_stride;
  const float *freq, *weight[2];  // weight: of queries, of keys
  const int *axis;
  int *status;
  int S, N, G, group, rot, axes;
  int heads;                      // heads per CTA
  bool ahead;                     // rows are fetched before the lengths are known
  float eps;
};

struct VerifyParams {
  const char *target, *draft, *target_prefix, *draft_prefix;
  long long target_seq, target_row, draft_seq, draft_row, target_prefix_seq, draft_prefix_seq;  // strides in bytes
  const int *tokens, *parent, *nodes;
  const float *accept_u, *sample_u;
  int *path, *path_len, *next_token, *status;
  int T, V, A, distinct, ranks, rank_shift;  // ranks = 1 << rank_shift: CTAs that share a sequence
};

struct ReorderParams {
  const char *src[2];             // arrays of rows that move: K and V, or the states
  char *dst[2];
  long long src_unit, dst_unit;   // bytes of a unit's rows in them
  const float *src_s, *src_q;     // the cache's arrays; unused for states
  const int *src_n, *src_pos, *src_live, *src_t_next;
  float *dst_s, *dst_q;
  int *dst_n, *dst_pos, *dst_live, *dst_t_next;
  const int *map;
  int *status;
  int S_src, S_dst, G, B_src, B_dst;
  int row_shift;                  // 16-byte chunks of a row: 1 << row_shift
  int arrays;                     // 2: a cache, 1: states
  bool in_place;
  int parts, room;                // CTAs that share a unit; 16-byte chunks that a thread has room for
};

}  // namespace roco
