// Launch interfaces of the operators on the paged cache: rotary append,
// attention with modified scores and masks, eviction.
#pragma once
#include "eb_internal.h"
#include "op_plan.h"

namespace eb {

// A request table: the host's words, and the place in the workspace that a
// table too long for the kernels' arguments is written to.
struct Table {
  const int32_t *words;
  size_t n;
  int32_t *dev;
};

struct RotaryCall {
  uint16_t *qkv;
  KV kv;  // k null: no cache
  const int32_t *positions;
  const uint16_t *gq, *gk;
  int32_t T, S, R, interleaved, uniform_n;
  float magnitude;
  double turn[64];
  Table table;
};
hipError_t launch_rotary_append(const Shape &s, const RotaryCall &c, hipStream_t st);

struct AttendCall {
  const uint16_t *qkv;
  uint16_t *out;
  float *lse;        // [T, nq], null where the caller wants none and no weights are kept
  float *weights;    // paged [num_pages, n_kv, 16], or null
  const int32_t *first_key;
  const float *slopes;
  KV kv;
  int32_t window, weight_rows;
  float scale, softcap;
  const AttendPlan *plan;
  char *ws;
};
hipError_t launch_attend(const Shape &s, const AttendCall &c, hipStream_t st);

struct EvictCall {
  KV src, dst;
  const float *weights;
  float *dst_weights;
  int32_t *kept;
  int32_t sink, recent, kept_stride;
  const EvictPlan *plan;
  char *ws;
};
hipError_t launch_evict(const Shape &s, const EvictCall &c, hipStream_t st);

}  // namespace eb
