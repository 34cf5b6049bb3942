// Writes request tables from kernel arguments into device memory.
#include "op_meta.h"

#include <string.h>

namespace eb {

namespace {
struct PutArgs {
  int32_t *dst;
  int32_t n;
  Words inl;
};

__global__ __launch_bounds__(256) void k_put_words(PutArgs a) {
  typedef const __attribute__((address_space(4))) char *karg_t;
  const karg_t p = (karg_t)__builtin_amdgcn_kernarg_segment_ptr();
  const int32_t *in = (const int32_t *)(p + offsetof(PutArgs, inl));
  for (int i = threadIdx.x; i < a.n; i += 256) a.dst[i] = in[i];
}
}  // namespace

hipError_t put_words(const int32_t *words, size_t n, int32_t *dev, hipStream_t st) {
  for (size_t at = 0; at < n; at += kInlineInts) {
    PutArgs a;
    a.dst = dev + at;
    a.n = (int32_t)(n - at < (size_t)kInlineInts ? n - at : (size_t)kInlineInts);
    memcpy(a.inl.w, words + at, (size_t)a.n * sizeof(int32_t));
    memset(a.inl.w + a.n, 0, (size_t)(kInlineInts - a.n) * sizeof(int32_t));
    hipLaunchKernelGGL(k_put_words, dim3(1), dim3(256), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace eb
