// Request tables of the cache operators (rotary append, modified attention,
// eviction): a few int32 arrays, one entry per request, that every kernel of
// the call reads.  Tables of up to kInlineInts words travel inside the
// kernels' own arguments, so a small call costs no copy and no launch for
// them; larger ones are written into the workspace by k_put_words, again from
// kernel arguments.  Neither way leaves anything on the host that a captured
// call would read when it is replayed.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace eb {

// Kernel arguments stay below 4 KiB: these words, 64 doubles (rotary) and a
// few dozen words more.
constexpr int kInlineInts = 768;

template <int N>
struct WordsOf {
  static constexpr size_t kMost = N;
  int32_t w[N];
};
using Words = WordsOf<kInlineInts>;

// Enqueue the write of n words to dev (device memory).
hipError_t put_words(const int32_t *words, size_t n, int32_t *dev, hipStream_t st);

// A table as a kernel reads it: read-only while the kernel runs, so entries at
// uniform places come by scalar loads.
typedef const __attribute__((address_space(4))) int32_t *meta_t;

// The tables of a kernel whose only parameter is a struct A with members
// `const int32_t *meta` (null: the words follow in the arguments) and
// `Words inl` (or another WordsOf).
template <class A>
__device__ __forceinline__ meta_t meta_words(const A &a) {
  typedef const __attribute__((address_space(4))) char *karg_t;
  // the struct is the kernel's first and only parameter: offset 0
  const karg_t p = (karg_t)__builtin_amdgcn_kernarg_segment_ptr();
  const meta_t in = (meta_t)(p + offsetof(A, inl));
  return a.meta ? (meta_t)a.meta : in;
}

// Index of the last entry of the ascending array first[0 .. n) that is <= v
// (first[0] <= v); called by whole wavefronts with a uniform v.  Each round
// probes 64 evenly spaced entries, one per lane.
__device__ __forceinline__ int last_at_or_below(meta_t first, int n, int v) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  while (n > 1) {
    const int step = (n + 63) >> 6;
    const int idx = lane * step;
    const bool ok = idx < n && first[lo + idx] <= v;
    const int last = __builtin_popcountll(__builtin_amdgcn_ballot_w64(ok)) - 1;
    n = min(step, n - last * step);
    lo += last * step;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

}  // namespace eb
