// What the C entry points share: errors, argument checks and the view of a
// handle that operators outside the layer step need.
#pragma once
#include <hip/hip_runtime.h>

#include <string>

#include "../../include/eb_layer.h"
#include "eb_internal.h"

namespace eb {

struct HandleView {
  const eb_layer_config *cfg;
  const Shape *shape;
  int32_t max_seqs;
  int device;
  bool debug_validate;
};
HandleView api_view(const eb_handle *h);

// Each sets the calling thread's error message when it does not return EB_OK.
eb_status api_fail(eb_status s, const std::string &msg);
eb_status api_hip_fail(hipError_t e, const char *what);
eb_status api_check_kv(const eb_kv_cache *kv);
eb_status api_check_ws(void *ws, size_t ws_bytes, size_t need);
eb_status api_check_batch(const eb_handle *h, const eb_batch *b, int32_t max_pages);
eb_status api_debug_tables(const eb_handle *h, const eb_batch *b, const eb_kv_cache *kv, hipStream_t st);
KV api_kv(const eb_kv_cache *kv);

}  // namespace eb
