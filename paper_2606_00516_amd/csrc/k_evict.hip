// Eviction by accumulated weight: which keys of each (request, kv head) stay,
// and their copy, in order, into other pages.
//
// A key stays if it is among the first `sink` or the last `recent` of its
// request, or among the heaviest of the rest (equal weights: the lower key).
// Reads 4 bytes of weight per (key, kv head) and moves 4 hd elements (K and V,
// in and out) per kept one: the copy is bound by HBM, the choice by the
// latency of one block's passes over its head's weights.
//
// k_evict_select, one block of 1024 threads per (request, kv head), takes the
// weights as ordered integers into registers (64 per thread hold 65536 keys;
// longer requests are read again from the caches in each pass) and finds
// the threshold by counting: three passes of a 2048-bin histogram over 11, 11
// and 10 bits of those that still agree with it, starting at the highest
// bit in which the candidates differ.  Every key then knows from two counts,
// of the heavier and of the equal ones before it, whether it stays and where
// it goes.  k_evict_copy moves the kept rows.
#include <string.h>

#include "device_common.h"
#include "eb_internal.h"
#include "op_meta.h"
#include "ops.h"

namespace eb {

namespace {

struct EvictArgs {
  KV src, dst;
  const float *weights;
  float *dst_weights;
  int32_t *kept;
  int32_t S, nkv, sink, recent, kept_stride;
  const int32_t *meta;  // [S] lengths, [S] kept, [S + 1] first destination page group
  Words inl;
};
static_assert(sizeof(EvictArgs) < 4096, "kernel arguments");

constexpr int kThreads = 1024, kBins = 2048;
constexpr int kPagesPerGroup = 4;  // destination pages per copy block

// fp32 in an unsigned order: larger numbers are larger integers, NaN above
// all, both zeros the same.
EB_DEV uint32_t ordered(float f) {
  const uint32_t u = __float_as_uint(f + 0.0f);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// Sum over the block in every thread; two barriers.
EB_DEV int block_sum(int v, int *part) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  int s = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) s += part[w];
  return s;
}

// NR: weights per thread in registers, in runs of four consecutive keys; run
// j of thread t starts at key 4 (1024 j + t).  AGAIN: the request may be longer,
// the keys past NR x 1024 are read anew in every pass.
template <int NR, bool AGAIN>
__global__ __launch_bounds__(kThreads) void k_evict_select(EvictArgs a) {
  constexpr int RUNS = NR / 4;
  __shared__ int hist[kBins];
  __shared__ int part[64];
  __shared__ uint32_t lim[2];
  __shared__ int cnt[2][2][kThreads / 64];
  const int32_t *m = meta_words(a);
  const int seq = blockIdx.x / a.nkv, kh = blockIdx.x - seq * a.nkv;
  const int c = m[seq], keep = m[a.S + seq];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int32_t *kept = a.kept + ((size_t)seq * a.nkv + kh) * a.kept_stride;
  if (keep >= c) {  // nothing leaves
    for (int t = tid; t < c; t += kThreads) kept[t] = t;
    return;
  }
  const int32_t *bt = a.src.bt + (size_t)seq * a.src.max_pages;
  const int s0 = min(a.sink, c), s1 = max(s0, c - a.recent);  // candidates: [s0, s1)
  const int want = keep - (s0 + c - s1);                      // of them to keep (>= 0, < s1 - s0)
  auto run_at = [&](int t) -> u32x4_t {  // the four ordered weights from key t on
    u32x4_t v = {0u, 0u, 0u, 0u};
    if (t < c) {
      const int page = bt[t / kPageSize];
      if ((unsigned)page < (unsigned)a.src.num_pages) {
        const f32x4_t f =
            *reinterpret_cast<const f32x4_t *>(a.weights + ((size_t)page * a.nkv + kh) * kPageSize + t % kPageSize);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = ordered(f[e]);
      }
    }
    return v;
  };
  u32x4_t reg[RUNS];
#pragma unroll
  for (int j = 0; j < RUNS; ++j) reg[j] = run_at(4 * (kThreads * j + tid));
  const int nruns = (c + 4 * kThreads - 1) / (4 * kThreads);
  // every (first key, four weights) of this thread
  auto each = [&](auto f) {
#pragma unroll
    for (int j = 0; j < RUNS; ++j)
      if (j < nruns) f(4 * (kThreads * j + tid), reg[j]);
    if constexpr (AGAIN)
      for (int j = RUNS; j < nruns; ++j) {
        const int t = 4 * (kThreads * j + tid);
        f(t, run_at(t));
      }
  };
  // the smallest and largest candidate: bits above the highest in which they
  // differ are common to all
  uint32_t mn = 0xFFFFFFFFu, mx = 0u;
  each([&](int t, const u32x4_t &v) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (t + e >= s0 && t + e < s1) {
        mn = min(mn, v[e]);
        mx = max(mx, v[e]);
      }
  });
  if (tid == 0) {
    lim[0] = 0xFFFFFFFFu;
    lim[1] = 0u;
  }
  __syncthreads();
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    mn = min(mn, (uint32_t)__shfl_xor((int)mn, o, 64));
    mx = max(mx, (uint32_t)__shfl_xor((int)mx, o, 64));
  }
  if (lane == 0) {
    atomicMin(&lim[0], mn);
    atomicMax(&lim[1], mx);
  }
  __syncthreads();
  mn = lim[0];
  mx = lim[1];
  // The want-th largest candidate: known bits `pre` above position `top`.
  int left = want;          // to take among those that agree with pre
  int top = mn == mx ? 0 : 32 - __builtin_clz(mn ^ mx);
  uint32_t pre = top < 32 ? (mx >> top) << top : 0u;
  if (want == 0) {
    pre = 0xFFFFFFFFu;  // nothing is taken: no candidate counts as heavier, none as equal
    top = 0;
  }
  while (top > 0) {
    const int bits = min(top, 11), sh = top - bits;
    for (int i = tid; i < kBins; i += kThreads) hist[i] = 0;
    __syncthreads();
    const uint32_t mask = (1u << bits) - 1u;
    each([&](int t, const u32x4_t &v) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool in = t + e >= s0 && t + e < s1 && (top == 32 || (v[e] >> top) == (pre >> top));
        const uint64_t live = __builtin_amdgcn_ballot_w64(in);
        if (live == 0) continue;
        const int bin = (int)((v[e] >> sh) & mask);
        // many equal weights (keys that never received any) would meet on one
        // counter lane by lane
        const int first = __builtin_amdgcn_readlane(bin, __builtin_ctzll(live));
        if (__builtin_amdgcn_ballot_w64(in && bin != first) == 0) {
          if (lane == 0) atomicAdd(&hist[first], __builtin_popcountll(live));
        } else if (in) {
          atomicAdd(&hist[bin], 1);
        }
      }
    });
    __syncthreads();
    // the bin from above in which the left-th falls: each thread sums two bins
    // from the top, a scan over the block gives the counts above them
    const int b0 = kBins - 1 - 2 * tid;
    const int h0 = hist[b0], h1 = hist[b0 - 1];
    int sum = h0 + h1;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(sum, o, 64);
      if (lane >= o) sum += v;
    }
    if (lane == 63) part[wave] = sum;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < wave; ++w) before += part[w];
    const int upto = before + sum, above = upto - h0 - h1;  // with and without this thread's bins
    if (above < left && left <= upto) {
      const int b = left <= above + h0 ? b0 : b0 - 1;
      part[32] = b;
      part[33] = left - (b == b0 ? above : above + h0);
    }
    __syncthreads();
    pre |= (uint32_t)part[32] << sh;
    left = part[33];
    top = sh;
    __syncthreads();
  }
  // pre is the threshold, left the number of keys equal to it that stay, the
  // lowest first.  Counts before each key: over the runs of 4096 keys in turn,
  // over the wavefronts of a run through LDS, over the lanes by ballots.
  int g_before = 0, e_before = 0;  // heavier (or always kept) and equal keys before the run
  int j = 0;
  auto place = [&](int t, const u32x4_t &v) {
    bool gt[4], eq[4];
    int ng = 0, ne = 0, gl = 0, el = 0;
    const uint64_t below = lane == 0 ? 0ull : (~0ull >> (64 - lane));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int k = t + e;
      const bool cand = k >= s0 && k < s1;
      gt[e] = k < c && (!cand || (want > 0 && v[e] > pre));
      eq[e] = cand && want > 0 && v[e] == pre;
      const uint64_t bg = __builtin_amdgcn_ballot_w64(gt[e]), be = __builtin_amdgcn_ballot_w64(eq[e]);
      ng += __builtin_popcountll(bg);
      ne += __builtin_popcountll(be);
      gl += __builtin_popcountll(bg & below);
      el += __builtin_popcountll(be & below);
    }
    int(&cg)[2][kThreads / 64] = cnt[j & 1];
    if (lane == 0) {
      cg[0][wave] = ng;
      cg[1][wave] = ne;
    }
    __syncthreads();  // (the other half of cnt is rewritten only after the next barrier)
    int pg = g_before + gl, pe = e_before + el;
    for (int w = 0; w < kThreads / 64; ++w) {
      const int x = cg[0][w], y = cg[1][w];
      if (w < wave) {
        pg += x;
        pe += y;
      }
      g_before += x;
      e_before += y;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (gt[e] || (eq[e] && pe < left)) kept[pg + min(pe, left)] = t + e;
      pg += gt[e];
      pe += eq[e];
    }
    ++j;
  };
  each(place);
}

// Copies the kept rows: one block per (group of four destination pages, kv
// head), 16 bytes per thread and step; K and V loads of all steps are issued
// before the first store.
template <int RB>  // bytes of a key's K (or V) row
__global__ __launch_bounds__(256) void k_evict_copy(EvictArgs a) {
  constexpr int LPR = RB / 16;                                      // threads per row
  constexpr int STEPS = kPagesPerGroup * kPageSize * LPR / 256;     // 1 .. 4
  const int32_t *m = meta_words(a);
  const int grp = blockIdx.x / a.nkv, kh = blockIdx.x - grp * a.nkv;
  const int32_t *first = m + 2 * a.S;
  const int seq = last_at_or_below(first, a.S, grp);
  const int k = min(m[seq], m[a.S + seq]);
  const int j0 = (grp - first[seq]) * kPagesPerGroup * kPageSize;
  const int32_t *kept = a.kept + ((size_t)seq * a.nkv + kh) * a.kept_stride;
  const int32_t *sbt = a.src.bt + (size_t)seq * a.src.max_pages;
  const int32_t *dbt = a.dst.bt + (size_t)seq * a.dst.max_pages;
  const uint8_t *sk = reinterpret_cast<const uint8_t *>(a.src.k), *sv = reinterpret_cast<const uint8_t *>(a.src.v);
  uint8_t *dk = reinterpret_cast<uint8_t *>(a.dst.k), *dv = reinterpret_cast<uint8_t *>(a.dst.v);
  u32x4_t kx[STEPS], vx[STEPS];
  size_t to[STEPS];
  bool ok[STEPS];
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    const int u = s * 256 + threadIdx.x, j = j0 + u / LPR, ch = u % LPR;
    ok[s] = j < k;
    kx[s] = vx[s] = u32x4_t{0u, 0u, 0u, 0u};
    to[s] = 0;
    if (ok[s]) {
      const int t = kept[j], page = sbt[t / kPageSize], dpage = dbt[j / kPageSize];
      ok[s] = (unsigned)dpage < (unsigned)a.dst.num_pages;
      to[s] = (((size_t)dpage * a.nkv + kh) * kPageSize + j % kPageSize) * RB + ch * 16;
      if ((unsigned)page < (unsigned)a.src.num_pages) {  // (a bad id reads as zeros)
        const size_t from = (((size_t)page * a.nkv + kh) * kPageSize + t % kPageSize) * RB + ch * 16;
        kx[s] = ld_stream_u32x4(sk + from);
        vx[s] = ld_stream_u32x4(sv + from);
      }
    }
  }
#pragma unroll
  for (int s = 0; s < STEPS; ++s)
    if (ok[s]) {
      st_u32x4(dk + to[s], kx[s]);
      st_u32x4(dv + to[s], vx[s]);
    }
  if (a.dst_weights && threadIdx.x < kPagesPerGroup * kPageSize) {
    const int j = j0 + threadIdx.x;
    if (j < k) {
      const int t = kept[j], page = sbt[t / kPageSize], dpage = dbt[j / kPageSize];
      if ((unsigned)dpage < (unsigned)a.dst.num_pages)
        a.dst_weights[((size_t)dpage * a.nkv + kh) * kPageSize + j % kPageSize] =
            (unsigned)page < (unsigned)a.src.num_pages
                ? a.weights[((size_t)page * a.nkv + kh) * kPageSize + t % kPageSize]
                : 0.f;
    }
  }
}

}  // namespace

hipError_t launch_evict(const Shape &s, const EvictCall &c, hipStream_t st) {
  EvictArgs a;
  memset(&a, 0, sizeof a);
  a.src = c.src;
  a.dst = c.dst;
  a.weights = c.weights;
  a.dst_weights = c.dst_weights;
  a.kept = c.kept;
  a.S = c.S;
  a.nkv = s.nkv;
  a.sink = c.sink;
  a.recent = c.recent;
  a.kept_stride = c.kept_stride;
  if (c.table.n <= (size_t)kInlineInts) {
    memcpy(a.inl.w, c.table.words, c.table.n * sizeof(int32_t));
  } else {
    a.meta = c.table.dev;
    const hipError_t e = put_words(c.table.words, c.table.n, c.table.dev, st);
    if (e != hipSuccess) return e;
  }
  const dim3 grid(c.S * s.nkv), block(kThreads);
  if (c.max_len <= 4 * kThreads)
    hipLaunchKernelGGL((k_evict_select<4, false>), grid, block, 0, st, a);
  else if (c.max_len <= 16 * kThreads)
    hipLaunchKernelGGL((k_evict_select<16, false>), grid, block, 0, st, a);
  else if (c.max_len <= 64 * kThreads)
    hipLaunchKernelGGL((k_evict_select<64, false>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((k_evict_select<64, true>), grid, block, 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || c.groups == 0) return e;
  const dim3 cg((unsigned)(c.groups * s.nkv));
  const int rb = s.hd * (c.src.f8 ? 1 : 2);
  if (rb == 256)
    hipLaunchKernelGGL(k_evict_copy<256>, cg, dim3(256), 0, st, a);
  else if (rb == 128)
    hipLaunchKernelGGL(k_evict_copy<128>, cg, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL(k_evict_copy<64>, cg, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace eb
