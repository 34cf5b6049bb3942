// C entry points of the operators on the paged cache: rotary append, modified
// attention, eviction.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "api_internal.h"
#include "host_plan.h"
#include "op_meta.h"
#include "ops.h"

using namespace eb;

namespace {

constexpr size_t kAlign = 256;
size_t round_up(size_t n) { return (n + kAlign - 1) / kAlign * kAlign; }

// Runs f; nothing thrown inside crosses the C boundary.
template <class F>
eb_status guarded(F f) {
  try {
    return f();
  } catch (const std::bad_alloc &) {
    return api_fail(EB_ERR_LIMITS, "out of host memory");
  } catch (...) {
    return api_fail(EB_ERR_LIMITS, "internal error while planning the call");
  }
}
template <class F>
size_t guarded_bytes(F f) {
  try {
    return f();
  } catch (...) {
    return 0;
  }
}

eb_status check_device(const HandleView &v) {
  int dev = -1;
  const hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return api_hip_fail(e, "hipGetDevice");
  if (dev != v.device)
    return api_fail(EB_ERR_CONFIG, "the handle belongs to device " + std::to_string(v.device) +
                                       ", the current device is " + std::to_string(dev));
  return EB_OK;
}

eb_status check_aligned(const void *p, const char *what, size_t a = 16) {
  if (reinterpret_cast<uintptr_t>(p) % a)
    return api_fail(EB_ERR_CONFIG, std::string(what) + " must be " + std::to_string(a) + "-byte aligned");
  return EB_OK;
}

eb_status check_cache(const eb_kv_cache *kv, const char *what) {
  eb_status s = api_check_kv(kv);
  if (s == EB_OK) s = check_aligned(kv->k_cache, what);
  if (s == EB_OK) s = check_aligned(kv->v_cache, what);
  if (s == EB_OK) s = check_aligned(kv->block_tables, "block_tables", 4);
  return s;
}

// Host copy of a cache's block tables, for debug validation.
eb_status table_copy(const eb_kv_cache *kv, int32_t S, hipStream_t st, std::vector<int32_t> &bt) {
  bt.resize((size_t)S * kv->max_pages_per_seq);
  hipError_t e = hipMemcpyAsync(bt.data(), kv->block_tables, bt.size() * 4, hipMemcpyDeviceToHost, st);
  if (e == hipSuccess) e = hipStreamSynchronize(st);
  return e == hipSuccess ? EB_OK : api_hip_fail(e, "debug validation copy");
}

// ---------------------------------------------------------------- rotary
constexpr double kTwoPi = 6.283185307179586476925286766559;

eb_status rotary_turns(const Shape &sh, const eb_rotary &r, RotaryCall &c) {
  const int R = r.rotary_dim == 0 ? sh.hd : r.rotary_dim;
  if (R < 0 || R % 16 || R > sh.hd)
    return api_fail(EB_ERR_CONFIG, "rotary_dim must be a multiple of 16 and at most head_dim");
  if (r.layout != EB_ROTARY_HALF && r.layout != EB_ROTARY_INTERLEAVED)
    return api_fail(EB_ERR_CONFIG, "unknown rotary layout");
  if (r.scaling < EB_ROTARY_PLAIN || r.scaling > EB_ROTARY_YARN)
    return api_fail(EB_ERR_CONFIG, "unknown rotary scaling");
  if (!(std::isfinite(r.theta) && r.theta > 1.f)) return api_fail(EB_ERR_CONFIG, "theta must be finite and above 1");
  if (!std::isfinite(r.magnitude) || r.magnitude < 0.f)
    return api_fail(EB_ERR_CONFIG, "magnitude must be finite and not negative");
  if (r.scaling != EB_ROTARY_PLAIN && !(std::isfinite(r.factor) && r.factor >= 1.f))
    return api_fail(EB_ERR_CONFIG, "factor must be finite and at least 1");
  const bool banded = r.scaling == EB_ROTARY_WAVELENGTH || r.scaling == EB_ROTARY_YARN;
  double low = r.low, high = r.high;
  if (banded) {
    if (r.original_len < 1) return api_fail(EB_ERR_CONFIG, "original_len must be at least 1");
    if (low == 0. && high == 0.) {
      low = 1.;
      high = r.scaling == EB_ROTARY_YARN ? 32. : 4.;
    }
    if (!(std::isfinite(low) && std::isfinite(high) && low > 0. && high > low))
      return api_fail(EB_ERR_CONFIG, "low and high must be finite with 0 < low < high");
  }
  const double f = r.factor, len = r.original_len;
  double theta = r.theta;
  if (r.scaling == EB_ROTARY_NTK) theta *= std::pow(f, (double)R / (R - 2));
  // the ramp of YARN over the pair index
  double a = 0., b = 1.;
  if (r.scaling == EB_ROTARY_YARN) {
    const auto index = [&](double turns) { return R * std::log(len / (kTwoPi * turns)) / (2. * std::log(theta)); };
    a = std::max(std::floor(index(high)), 0.);
    b = std::min(std::ceil(index(low)), (double)R - 1.);
    b = std::max(b, a + 1e-3);
  }
  double w[64];
  rotary_frequencies(R, theta, w);
  for (int t = 0; t < R / 2; ++t) {
    double v = w[t];
    if (r.scaling == EB_ROTARY_LINEAR) v /= f;
    if (r.scaling == EB_ROTARY_WAVELENGTH) {
      const double turns = len * v / kTwoPi, mix = std::min(std::max((turns - low) / (high - low), 0.), 1.);
      v = v * mix + v / f * (1. - mix);
    }
    if (r.scaling == EB_ROTARY_YARN) {
      const double g = std::min(std::max((t - a) / (b - a), 0.), 1.);
      v = v * (1. - g) + v / f * g;
    }
    c.turn[t] = v / kTwoPi;
  }
  c.R = R;
  c.interleaved = r.layout == EB_ROTARY_INTERLEAVED;
  c.magnitude = r.magnitude != 0.f                       ? r.magnitude
                : r.scaling == EB_ROTARY_YARN && f > 1. ? (float)(0.1 * std::log(f) + 1.)
                                                         : 1.f;
  return EB_OK;
}

size_t rotary_words(int32_t S) { return (size_t)2 * S; }

// ---------------------------------------------------------------- attention
eb_status check_mod(const eb_score_mod *m, const eb_batch *b) {
  if (!m) return EB_OK;
  if (!(m->scale == 0.f || (std::isfinite(m->scale) && m->scale > 0.f)))
    return api_fail(EB_ERR_CONFIG, "scale must be 0 or finite and positive");
  if (!(m->softcap >= 0.f && m->softcap <= 1000.f))
    return api_fail(EB_ERR_CONFIG, "softcap must be 0 (none) or at most 1000");
  if (m->window < 0) return api_fail(EB_ERR_CONFIG, "window must not be negative");
  if (m->prefix_lens_host)
    for (int i = 0; i < b->num_seqs; ++i) {
      const int32_t p = m->prefix_lens_host[i];
      if (p < 0 || p > b->context_lens_host[i] + b->chunk_lens_host[i])
        return api_fail(EB_ERR_BATCH, "request " + std::to_string(i) + ": prefix outside [0, context + chunk]");
    }
  return EB_OK;
}

// ---------------------------------------------------------------- eviction
eb_status check_evict(int32_t n_kv, int32_t S, const int32_t *lens, const int32_t *keep, EvictPlan &p) {
  if (S < 0) return api_fail(EB_ERR_BATCH, "negative num_seqs");
  if (S > 0 && (!lens || !keep)) return api_fail(EB_ERR_NULL, "lens_host or keep_lens_host is NULL");
  for (int i = 0; i < S; ++i) {
    if (lens[i] < 0 || keep[i] < 0)
      return api_fail(EB_ERR_BATCH, "request " + std::to_string(i) + ": negative length");
    if (lens[i] > 0x3FFFFFFF) return api_fail(EB_ERR_BATCH, "request " + std::to_string(i) + ": length overflows");
  }
  if (!plan_evict(n_kv, S, lens, keep, p)) return api_fail(EB_ERR_LIMITS, "more keys than a launch holds");
  return EB_OK;
}

}  // namespace

extern "C" {

size_t eb_op_rotary_kv_append_workspace_bytes(const eb_handle *h, const eb_batch *batch) {
  return guarded_bytes([&]() -> size_t {
    if (!h || api_check_batch(h, batch, -1) != EB_OK) return 0;
    return round_up(rotary_words(batch->num_seqs) * 4);
  });
}

eb_status eb_op_rotary_kv_append(eb_handle *h, const eb_rotary *rot, void *qkv, const eb_kv_cache *kv,
                                 const eb_batch *batch, const int32_t *positions, void *ws, size_t ws_bytes,
                                 void *stream) {
  return guarded([&]() -> eb_status {
    if (!h) return api_fail(EB_ERR_NULL, "handle is NULL");
    if (!rot) return api_fail(EB_ERR_NULL, "rot is NULL");
    const HandleView v = api_view(h);
    RotaryCall c{};
    eb_status s = rotary_turns(*v.shape, *rot, c);
    if (s == EB_OK && kv) s = check_cache(kv, "the cache");
    if (s == EB_OK) s = api_check_batch(h, batch, kv ? kv->max_pages_per_seq : -1);
    if (s != EB_OK) return s;
    if (batch->num_tokens == 0) return EB_OK;
    if (!qkv) return api_fail(EB_ERR_NULL, "qkv is NULL");
    s = check_aligned(qkv, "qkv");
    if (s == EB_OK && positions) s = check_aligned(positions, "positions", 4);
    if (s != EB_OK) return s;
    if (v.shape->qkn) {
      if (!rot->q_norm || !rot->k_norm) return api_fail(EB_ERR_NULL, "q_norm or k_norm is NULL");
      s = check_aligned(rot->q_norm, "q_norm");
      if (s == EB_OK) s = check_aligned(rot->k_norm, "k_norm");
      if (s != EB_OK) return s;
    }
    const int S = batch->num_seqs;
    s = api_check_ws(ws, ws_bytes, round_up(rotary_words(S) * 4));
    if (s == EB_OK) s = check_device(v);
    if (s != EB_OK) return s;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (kv) {
      s = api_debug_tables(h, batch, kv, st);
      if (s != EB_OK) return s;
    }
    std::vector<int32_t> words(rotary_words(S));
    int32_t row = 0, uniform = batch->chunk_lens_host[0];
    for (int i = 0; i < S; ++i) {
      words[i] = batch->context_lens_host[i];
      words[S + i] = row;
      row += batch->chunk_lens_host[i];
      if (batch->chunk_lens_host[i] != uniform) uniform = 0;
    }
    c.qkv = static_cast<uint16_t *>(qkv);
    if (kv) c.kv = api_kv(kv);
    c.positions = positions;
    c.gq = static_cast<const uint16_t *>(rot->q_norm);
    c.gk = static_cast<const uint16_t *>(rot->k_norm);
    c.T = batch->num_tokens;
    c.S = S;
    c.uniform_n = uniform;
    // rows of equal length need the contexts alone
    c.table = Table{words.data(), uniform > 0 ? (size_t)S : words.size(), static_cast<int32_t *>(ws)};
    const hipError_t e = launch_rotary_append(*v.shape, c, st);
    return e == hipSuccess ? EB_OK : api_hip_fail(e, "rotary append");
  });
}

size_t eb_op_attention_mod_workspace_bytes(const eb_handle *h, const eb_batch *batch, const eb_score_mod *mod,
                                           int32_t want_weights) {
  return guarded_bytes([&]() -> size_t {
    if (!h || api_check_batch(h, batch, -1) != EB_OK || check_mod(mod, batch) != EB_OK) return 0;
    AttendPlan p;
    return plan_attend(*api_view(h).cfg, *batch, mod ? mod->window : 0, mod ? mod->prefix_lens_host : nullptr,
                       want_weights != 0, 0, p)
               ? p.total
               : 0;
  });
}

eb_status eb_op_attention_mod(eb_handle *h, const void *qkv, const eb_kv_cache *kv, const eb_batch *batch,
                              const eb_score_mod *mod, void *out, float *lse, float *kv_weights,
                              int32_t weight_rows, void *ws, size_t ws_bytes, void *stream) {
  return guarded([&]() -> eb_status {
    if (!h) return api_fail(EB_ERR_NULL, "handle is NULL");
    const HandleView v = api_view(h);
    eb_status s = check_cache(kv, "the cache");
    if (s == EB_OK) s = api_check_batch(h, batch, kv->max_pages_per_seq);
    if (s == EB_OK) s = check_mod(mod, batch);
    if (s != EB_OK) return s;
    if (weight_rows < 0) return api_fail(EB_ERR_CONFIG, "weight_rows must not be negative");
    if (batch->num_tokens == 0) return EB_OK;
    if (!qkv || !out) return api_fail(EB_ERR_NULL, "qkv or out is NULL");
    s = check_aligned(qkv, "qkv");
    if (s == EB_OK) s = check_aligned(out, "out");
    if (s == EB_OK) s = check_aligned(lse, "lse", 4);
    if (s == EB_OK) s = check_aligned(kv_weights, "kv_weights");
    if (s == EB_OK && mod) s = check_aligned(mod->slopes, "slopes", 4);
    if (s == EB_OK && mod) s = check_aligned(mod->first_key, "first_key", 4);
    if (s != EB_OK) return s;
    AttendPlan p;
    if (!plan_attend(*v.cfg, *batch, mod ? mod->window : 0, mod ? mod->prefix_lens_host : nullptr,
                     kv_weights != nullptr, weight_rows, p))
      return api_fail(EB_ERR_LIMITS, "more keys than a launch holds");
    s = api_check_ws(ws, ws_bytes, p.total);
    if (s == EB_OK) s = check_device(v);
    if (s != EB_OK) return s;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    s = api_debug_tables(h, batch, kv, st);
    if (s != EB_OK) return s;
    AttendCall c{};
    c.qkv = static_cast<const uint16_t *>(qkv);
    c.out = static_cast<uint16_t *>(out);
    c.lse = lse;
    c.weights = kv_weights;
    c.kv = api_kv(kv);
    c.weight_rows = weight_rows;
    c.scale = 1.0f / std::sqrt((float)v.shape->hd);
    if (mod) {
      if (mod->scale > 0.f) c.scale = mod->scale;
      c.softcap = mod->softcap;
      c.slopes = mod->slopes;
      c.first_key = mod->first_key;
      c.window = mod->window;
    }
    const double by = (double)c.scale * c.kv.ks, unit = by / (c.softcap > 0.f ? c.softcap : 1.0);
    if (!(std::min(by, unit) > 1e-37 && std::max(by, unit) < 5e37))
      return api_fail(EB_ERR_CONFIG, "scale (with the cache's scale, over softcap) leaves fp32");
    c.plan = &p;
    c.ws = static_cast<char *>(ws);
    const hipError_t e = launch_attend(*v.shape, c, st);
    return e == hipSuccess ? EB_OK : api_hip_fail(e, "modified attention");
  });
}

size_t eb_op_kv_evict_workspace_bytes(const eb_handle *h, int32_t num_seqs, const int32_t *lens_host,
                                      const int32_t *keep_lens_host) {
  return guarded_bytes([&]() -> size_t {
    EvictPlan p;
    if (!h || check_evict(api_view(h).shape->nkv, num_seqs, lens_host, keep_lens_host, p) != EB_OK) return 0;
    return p.total;
  });
}

eb_status eb_op_kv_evict(eb_handle *h, const eb_kv_cache *src, const float *kv_weights, int32_t num_seqs,
                         const int32_t *lens_host, const int32_t *keep_lens_host, int32_t sink, int32_t recent,
                         const eb_kv_cache *dst, float *dst_weights, int32_t *kept, int32_t kept_stride, void *ws,
                         size_t ws_bytes, void *stream) {
  return guarded([&]() -> eb_status {
    if (!h) return api_fail(EB_ERR_NULL, "handle is NULL");
    const HandleView v = api_view(h);
    eb_status s = check_cache(src, "the source cache");
    if (s == EB_OK) s = check_cache(dst, "the destination cache");
    if (s != EB_OK) return s;
    if (src->kv_dtype != dst->kv_dtype ||
        (src->kv_dtype == EB_KV_FP8_E4M3 && (src->k_scale != dst->k_scale || src->v_scale != dst->v_scale)))
      return api_fail(EB_ERR_CONFIG, "source and destination must have the same element type and scales");
    EvictPlan p;
    s = check_evict(v.shape->nkv, num_seqs, lens_host, keep_lens_host, p);
    if (s != EB_OK) return s;
    if (num_seqs > v.max_seqs) return api_fail(EB_ERR_LIMITS, "batch larger than the handle's max_seqs");
    if (sink < 0 || recent < 0) return api_fail(EB_ERR_CONFIG, "sink and recent must not be negative");
    for (int i = 0; i < num_seqs; ++i) {
      const int64_t must = std::min<int64_t>(lens_host[i], (int64_t)sink + recent);
      if (must > keep_lens_host[i])
        return api_fail(EB_ERR_BATCH, "request " + std::to_string(i) + ": sink + recent exceeds the keys to keep");
      if (lens_host[i] > (int64_t)src->max_pages_per_seq * kPageSize)
        return api_fail(EB_ERR_PAGES, "request " + std::to_string(i) + ": length exceeds the source's pages");
      if (std::min(lens_host[i], keep_lens_host[i]) > (int64_t)dst->max_pages_per_seq * kPageSize)
        return api_fail(EB_ERR_PAGES, "request " + std::to_string(i) + ": kept keys exceed the destination's pages");
    }
    if (p.max_keep == 0) return EB_OK;
    if (!kv_weights) return api_fail(EB_ERR_NULL, "kv_weights is NULL");
    s = check_aligned(kv_weights, "kv_weights");
    if (s == EB_OK) s = check_aligned(dst_weights, "dst_weights", 4);
    if (s == EB_OK) s = check_aligned(kept, "kept", 4);
    if (s != EB_OK) return s;
    if (kept && kept_stride < p.max_keep)
      return api_fail(EB_ERR_CONFIG, "kept_stride is smaller than the largest number of kept keys");
    s = api_check_ws(ws, ws_bytes, p.total);
    if (s == EB_OK) s = check_device(v);
    if (s != EB_OK) return s;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (v.debug_validate) {
      // every needed page inside its pool; no destination page used twice, or
      // by a source where both are one pool
      std::vector<int32_t> bt[2];
      std::vector<char> seen((size_t)dst->num_pages, 0);
      for (int d = 0; d < 2; ++d) {
        const eb_kv_cache *kv = d ? dst : src;
        s = table_copy(kv, num_seqs, st, bt[d]);
        if (s != EB_OK) return s;
        for (int i = 0; i < num_seqs; ++i) {
          const int32_t len = d ? std::min(lens_host[i], keep_lens_host[i]) : lens_host[i];
          for (int64_t j = 0; j < ((int64_t)len + kPageSize - 1) / kPageSize; ++j) {
            const int32_t id = bt[d][(size_t)i * kv->max_pages_per_seq + j];
            if (id < 0 || id >= kv->num_pages)
              return api_fail(EB_ERR_PAGES, "request " + std::to_string(i) + ": page id outside [0, num_pages)");
            if (!d && src->k_cache == dst->k_cache && id < dst->num_pages) seen[id] = 1;
            if (d && seen[id]++)
              return api_fail(EB_ERR_PAGES, "request " + std::to_string(i) + ": destination page is in use");
          }
        }
      }
    }
    EvictCall c{};
    c.src = api_kv(src);
    c.dst = api_kv(dst);
    c.weights = kv_weights;
    c.dst_weights = dst_weights;
    c.ws = static_cast<char *>(ws);
    c.kept = kept ? kept : reinterpret_cast<int32_t *>(c.ws + p.o_kept);
    c.kept_stride = kept ? kept_stride : p.max_keep;
    c.sink = sink;
    c.recent = recent;
    c.plan = &p;
    const hipError_t e = launch_evict(*v.shape, c, st);
    return e == hipSuccess ? EB_OK : api_hip_fail(e, "eviction");
  });
}

}  // extern "C"
