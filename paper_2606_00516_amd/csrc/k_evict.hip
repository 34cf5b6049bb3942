// Eviction by accumulated weight: which keys of each (request, kv head) stay,
// and their copy, in order, into other pages.
//
// A key stays if it is among the first `sink` or the last `recent` of its
// request, or among the heaviest of the rest (equal weights: the lower key).
// Reads 4 bytes of weight per (key, kv head) and moves 4 hd elements (K and V,
// in and out) per kept one: the copy is bound by HBM, the choice by latency.
// Weights are compared as ordered integers; a threshold and the number of keys
// equal to it that stay say everything, and every key then knows from two
// counts, of the heavier and of the equal ones before it, whether it stays and
// where it goes.  Three forms, by the longest request of the call:
//  - to 512 keys (k_evict_few): one wavefront per (request, kv head) finds the
//    threshold bit by bit with ballots, without a barrier, and its block copies
//    (three requests of 250 to 330 keys: 8.9 us; the next form's two launches
//    16.5).
//  - to 16384 keys (k_evict_select, k_evict_copy): a block holds a head's
//    weights in registers and finds the bin of the threshold by a histogram of
//    the 11 bits from the highest in which the candidates differ, then the
//    threshold among the bin's few keys (32 requests of 4350 keys and 8 heads:
//    12 us, and 109 for the copy of 4000 keys each, 4.9 TB/s).
//  - longer (k_evict_hist, _list, _solve, _place): the same over segments of
//    4096 keys, as many blocks as there are segments; the histogram and the
//    list of the bin's keys are in the workspace (16000 keys, 8 heads, this form
//    and the one before: one request 23.9 and 22.9 us, 32 requests 61 and 50;
//    four requests of 40000 to 66000 keys: 24 us to choose, one block per head
//    99; the copy 38 with its counting).
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
  // long requests: [S nkv][2048] counts, then [S nkv] list lengths; the lists
  // (values, keys); per segment and head the heavier and equal keys before it;
  // per head the threshold and the number of equal keys that stay
  int32_t *hist, *list_n, *list_t, *seg_heavier, *seg_equal, *solved;
  uint32_t *list_v;
  const int32_t *meta;  // EvictField arrays of S (+ 1) words
  Words inl;
};
static_assert(sizeof(EvictArgs) < 4096, "kernel arguments");

constexpr int kThreads = 512, kWaves = kThreads / 64, kBins = 2048;
constexpr int kRun = 4 * kThreads;  // keys of one run over the block
constexpr int kListMost = 512;      // keys that one wavefront finds a threshold among
constexpr int kPagesPerGroup = 4;   // destination pages per copy block
static_assert(kEvictGroupKeys == kPagesPerGroup * kPageSize && kEvictFew == kListMost, "plan");

// A (request, kv head) of a call.
struct Head {
  int seq, kh, c, keep, s0, want;
  unsigned span;  // candidates: [s0, s0 + span)
  const int32_t *bt;
};
__device__ __forceinline__ Head head_of(const EvictArgs &a, meta_t m, int seq, int kh) {
  Head h;
  h.seq = seq;
  h.kh = kh;
  h.c = __builtin_amdgcn_readfirstlane(m[EV_LEN * a.S + seq]);
  h.keep = __builtin_amdgcn_readfirstlane(m[EV_KEEP * a.S + seq]);
  h.s0 = min(a.sink, h.c);
  const int s1 = max(h.s0, h.c - a.recent);
  h.span = (unsigned)(s1 - h.s0);
  // candidates that stay; all of them where nothing leaves
  h.want = h.keep >= h.c ? (int)h.span : h.keep - (h.s0 + h.c - s1);
  h.bt = a.src.bt + (size_t)seq * a.src.max_pages;
  return h;
}

// fp32 in an unsigned order: larger numbers are larger integers, every NaN
// above all and like the others, both zeros the same.
constexpr uint32_t kZeroWeight = 0x80000000u, kNanWeight = 0xFFC00000u;
EB_DEV uint32_t ordered(float f) {
  const uint32_t u = __float_as_uint(f + 0.0f);
  return f != f ? kNanWeight : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// N runs of four keys per thread from key t0 on, run j from t0 + 2048 j + 4 tid.
// No branch between the loads, so that all are in flight together: keys past
// the request read its last page, ids outside the pool page 0 (weight 0).
template <int N>
EB_DEV void load_runs(const EvictArgs &a, const Head &h, int t0, u32x4_t (&v)[N]) {
  int page[N];
  f32x4_t f[N];
#pragma unroll
  for (int j = 0; j < N; ++j) page[j] = h.bt[min(t0 + kRun * j + 4 * (int)threadIdx.x, h.c - 1) / kPageSize];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int p = (unsigned)page[j] < (unsigned)a.src.num_pages ? page[j] : 0;
    f[j] = *reinterpret_cast<const f32x4_t *>(a.weights + ((size_t)p * a.nkv + h.kh) * kPageSize +
                                              (t0 + kRun * j + 4 * (int)threadIdx.x) % kPageSize);
  }
#pragma unroll
  for (int j = 0; j < N; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) v[j][e] = (unsigned)page[j] < (unsigned)a.src.num_pages ? ordered(f[j][e]) : kZeroWeight;
}

// Inclusive sum over the wavefront's lanes, without LDS: within rows of 16
// lanes, then each row's total to the next.
EB_DEV int wave_scan(int x) {
#define EB_SCAN(CTRL, ROWS) x += __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xF, false)
  EB_SCAN(0x111, 0xF);  // row_shr 1, 2, 4, 8
  EB_SCAN(0x112, 0xF);
  EB_SCAN(0x114, 0xF);
  EB_SCAN(0x118, 0xF);
  EB_SCAN(0x142, 0xA);  // lane 15 of a row to the next row (rows 1 and 3)
  EB_SCAN(0x143, 0xC);  // lane 31 to rows 2 and 3
#undef EB_SCAN
  return x;
}

// The bin from above in which the left-th key falls, from this thread's four
// bins kBins - 1 - 4 tid - i; left becomes its rank inside the bin.  Two
// barriers; the counts may be overwritten after the call.
struct BinScratch {
  int part[kWaves], found[3];
};
EB_DEV void find_bin(const int (&h)[4], int &left, int &bin, int &in_bin, BinScratch &x) {
  static_assert(kBins == 4 * kThreads, "four bins per thread");
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int own = h[0] + h[1] + h[2] + h[3], sum = wave_scan(own);
  if (lane == 63) x.part[wave] = sum;
  __syncthreads();
  int above = sum - own;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) above += w < wave ? x.part[w] : 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (above < left && left <= above + h[i]) {
      x.found[0] = kBins - 1 - 4 * (int)threadIdx.x - i;
      x.found[1] = left - above;
      x.found[2] = h[i];
    }
    above += h[i];
  }
  __syncthreads();
  bin = x.found[0];
  left = x.found[1];
  in_bin = x.found[2];
}

// The left-th largest of a wavefront's values (8 per lane, 0 where there is
// none), all of which agree with pre above bit top: bit by bit with ballots.
// Returns the threshold; left becomes the number of values equal to it that
// count.  (Where exactly left values reach a trial, the value below it serves:
// all of those are heavier, and none equal to it counts.)
template <int N>
EB_DEV uint32_t wave_threshold(const uint32_t (&v)[N], int n, uint32_t pre, int top, int &left) {
  for (int b = top - 1; b >= 0; --b) {
    const uint32_t trial = pre | 1u << b;
    int reach = 0;
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (64 * j < n) reach += __builtin_popcountll(__builtin_amdgcn_ballot_w64(v[j] >= trial));
    if (reach >= left) pre = trial;
    if (reach == left) {
      left = 0;
      return pre - 1u;
    }
  }
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (64 * j < n) left -= __builtin_popcountll(__builtin_amdgcn_ballot_w64(v[j] > pre));
  return pre;
}

EB_DEV bool heavier(const Head &h, int t, uint32_t v, uint32_t pre) {
  return (unsigned)(t - h.s0) < h.span ? v > pre : t < h.c;
}
EB_DEV bool equal(const Head &h, int t, uint32_t v, uint32_t pre) {
  return (unsigned)(t - h.s0) < h.span && v == pre;
}

// ---------------------------------------------------------------------------
// to 16384 keys: RUNS x 2048 weights in registers
// ---------------------------------------------------------------------------
template <int RUNS>
__global__ __launch_bounds__(kThreads) void k_evict_select(EvictArgs a) {
  __shared__ int hist[kBins];
  __shared__ uint32_t list[kListMost], lim[2];
  __shared__ BinScratch bs;
  __shared__ int n_list, cnt[RUNS * kWaves];  // heavier and (upper half) equal keys of a run's wavefront
  const meta_t m = meta_words(a);
  const int seq = blockIdx.x / a.nkv;
  const Head h = head_of(a, m, seq, blockIdx.x - seq * a.nkv);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int32_t *kept = a.kept + ((size_t)seq * a.nkv + h.kh) * a.kept_stride;
  if (h.keep >= h.c) {  // nothing leaves
    for (int t = tid; t < h.c; t += kThreads) kept[t] = t;
    return;
  }
  u32x4_t reg[RUNS];
  load_runs<RUNS>(a, h, 0, reg);
  if (tid == 0) {
    lim[0] = 0xFFFFFFFFu;
    lim[1] = 0u;
    n_list = 0;
  }
  for (int i = tid; i < kBins; i += kThreads) hist[i] = 0;
  auto each = [&](auto f) {  // every candidate of this thread
#pragma unroll
    for (int j = 0; j < RUNS; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if ((unsigned)(kRun * j + 4 * tid + e - h.s0) < h.span) f(reg[j][e]);
  };
  // the smallest and largest candidate: bits above the highest in which they
  // differ are common to all
  uint32_t mn = 0xFFFFFFFFu, mx = 0u;
  each([&](uint32_t v) {
    mn = min(mn, v);
    mx = max(mx, v);
  });
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    mn = min(mn, (uint32_t)__shfl_xor((int)mn, o, 64));
    mx = max(mx, (uint32_t)__shfl_xor((int)mx, o, 64));
  }
  __syncthreads();
  if (lane == 0) {
    atomicMin(&lim[0], mn);
    atomicMax(&lim[1], mx);
  }
  __syncthreads();
  mn = lim[0];
  mx = lim[1];
  // the want-th largest candidate: known bits `pre` above position `top`
  int left = h.want, top = mn == mx ? 0 : 32 - __builtin_clz(mn ^ mx);
  uint32_t pre = top < 32 ? (mx >> top) << top : 0u;
  if (h.want == 0) {
    pre = 0xFFFFFFFFu;  // no candidate is heavier, and none of the equal ones stays
    top = 0;
  }
  while (top > 0) {
    const int bits = min(top, 11), sh = top - bits;
    const uint32_t mask = (1u << bits) - 1u;
    // (keys of the smallest weight, such as those that never received any,
    // would meet on one counter: they are counted in a register)
    int least = 0;
    each([&](uint32_t v) {
      if (top == 32 || (v >> top) == (pre >> top)) {
        if (v == mn)
          ++least;
        else
          atomicAdd(&hist[(v >> sh) & mask], 1);
      }
    });
    least = wave_scan(least);
    if (lane == 63 && least > 0) atomicAdd(&hist[(mn >> sh) & mask], least);
    __syncthreads();
    int own[4], bin, in_bin;
#pragma unroll
    for (int i = 0; i < 4; ++i) own[i] = hist[kBins - 1 - 4 * tid - i];
    find_bin(own, left, bin, in_bin, bs);
    pre |= (uint32_t)bin << sh;
    top = sh;
    if (top == 0) break;
    if (in_bin <= kListMost) {
      each([&](uint32_t v) {
        if ((v >> top) == (pre >> top)) list[atomicAdd(&n_list, 1)] = v;
      });
      __syncthreads();
      uint32_t v[kListMost / 64];  // every wavefront for itself
#pragma unroll
      for (int j = 0; j < kListMost / 64; ++j) v[j] = 64 * j + lane < in_bin ? list[64 * j + lane] : 0u;
      pre = wave_threshold(v, in_bin, pre, top, left);
      break;
    }
    for (int i = tid; i < kBins; i += kThreads) hist[i] = 0;
    __syncthreads();
  }
  // Before each key: over the lanes by a scan of both counts in one word (at
  // most 256 each), over the wavefronts and runs through LDS.
  int before[RUNS];
#pragma unroll
  for (int j = 0; j < RUNS; ++j) {
    const int t = kRun * j + 4 * tid;
    int x = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      x += (heavier(h, t + e, reg[j][e], pre) ? 1 : 0) + (equal(h, t + e, reg[j][e], pre) ? 1 << 16 : 0);
    const int upto = wave_scan(x);
    before[j] = upto - x;
    if (lane == 63) cnt[j * kWaves + wave] = upto;
  }
  __syncthreads();
  static_assert(RUNS * kWaves <= 64, "entries of one wavefront's scan");
  const int x = lane < RUNS * kWaves ? cnt[lane] : 0;
  const int g_incl = wave_scan(x & 0xFFFF), e_incl = wave_scan(x >> 16);
  const int g_excl = g_incl - (x & 0xFFFF), e_excl = e_incl - (x >> 16);
#pragma unroll
  for (int j = 0; j < RUNS; ++j) {
    const int t = kRun * j + 4 * tid;
    int pg = __shfl(g_excl, j * kWaves + wave, 64) + (before[j] & 0xFFFF);
    int pe = __shfl(e_excl, j * kWaves + wave, 64) + (before[j] >> 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool gt = heavier(h, t + e, reg[j][e], pre), eq = equal(h, t + e, reg[j][e], pre);
      if (gt || (eq && pe < left)) kept[pg + min(pe, left)] = t + e;
      pg += gt;
      pe += eq;
    }
  }
}

// Copies the kept rows: one block per (group of four destination pages, kv
// head), 16 bytes per thread and step; K and V loads of all steps are issued
// before the first store.
template <int RB>  // bytes of a key's K (or V) row
__global__ __launch_bounds__(256) void k_evict_copy(EvictArgs a) {
  constexpr int LPR = RB / 16;                                      // threads per row
  constexpr int STEPS = kPagesPerGroup * kPageSize * LPR / 256;     // 1 .. 4
  const meta_t m = meta_words(a);
  const int grp = blockIdx.x / a.nkv, kh = blockIdx.x - grp * a.nkv;
  const meta_t first = m + EV_GROUP0 * a.S;
  const int seq = last_at_or_below(first, a.S, grp);
  const int k = min(m[EV_LEN * a.S + seq], m[EV_KEEP * a.S + seq]);
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

// Copies n rows of a head by the block: row i is key at[i], which goes to slot
// j0 + i.
template <int RB, int NT>
EB_DEV void copy_rows(const EvictArgs &a, const Head &h, const int *at, int n, int j0) {
  constexpr int LPR = RB / 16, ROWS = NT / LPR, UN = 4;
  const int32_t *dbt = a.dst.bt + (size_t)h.seq * a.dst.max_pages;
  const uint8_t *sk = reinterpret_cast<const uint8_t *>(a.src.k), *sv = reinterpret_cast<const uint8_t *>(a.src.v);
  uint8_t *dk = reinterpret_cast<uint8_t *>(a.dst.k), *dv = reinterpret_cast<uint8_t *>(a.dst.v);
  const int tid = threadIdx.x, ch = tid % LPR * 16;
  for (int i0 = tid / LPR; i0 < n; i0 += UN * ROWS) {
    u32x4_t kx[UN], vx[UN];
    int page[UN], dpage[UN];
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int i = min(i0 + u * ROWS, n - 1);
      page[u] = h.bt[at[i] / kPageSize];
      dpage[u] = dbt[(j0 + i) / kPageSize];
    }
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int i = min(i0 + u * ROWS, n - 1), p = (unsigned)page[u] < (unsigned)a.src.num_pages ? page[u] : 0;
      const size_t from = (((size_t)p * a.nkv + h.kh) * kPageSize + at[i] % kPageSize) * RB + ch;
      kx[u] = ld_stream_u32x4(sk + from);
      vx[u] = ld_stream_u32x4(sv + from);
    }
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int i = i0 + u * ROWS, j = j0 + i;
      if (i < n && (unsigned)dpage[u] < (unsigned)a.dst.num_pages) {
        const bool ok = (unsigned)page[u] < (unsigned)a.src.num_pages;  // (a bad id reads as zeros)
        const size_t to = (((size_t)dpage[u] * a.nkv + h.kh) * kPageSize + j % kPageSize) * RB + ch;
        st_u32x4(dk + to, ok ? kx[u] : u32x4_t{0u, 0u, 0u, 0u});
        st_u32x4(dv + to, ok ? vx[u] : u32x4_t{0u, 0u, 0u, 0u});
      }
    }
  }
  if (a.dst_weights)
    for (int i = tid; i < n; i += NT) {
      const int t = at[i], page = h.bt[t / kPageSize], j = j0 + i, dpage = dbt[j / kPageSize];
      if ((unsigned)dpage < (unsigned)a.dst.num_pages)
        a.dst_weights[((size_t)dpage * a.nkv + h.kh) * kPageSize + j % kPageSize] =
            (unsigned)page < (unsigned)a.src.num_pages
                ? a.weights[((size_t)page * a.nkv + h.kh) * kPageSize + t % kPageSize]
                : 0.f;
    }
}

// ---------------------------------------------------------------------------
// to 512 keys: the first wavefront holds eight keys per lane (key 64 j + lane)
// ---------------------------------------------------------------------------
template <int RB>
__global__ __launch_bounds__(256) void k_evict_few(EvictArgs a) {
  constexpr int NJ = kEvictFew / 64;
  __shared__ int at[kEvictFew];
  const meta_t m = meta_words(a);
  const int seq = blockIdx.x / a.nkv;
  const Head h = head_of(a, m, seq, blockIdx.x - seq * a.nkv);
  const int k = min(h.c, h.keep), lane = threadIdx.x & 63;
  if (k == 0) return;
  if (threadIdx.x < 64) {
    int page[NJ];
    uint32_t v[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) page[j] = h.bt[min(64 * j + lane, h.c - 1) / kPageSize];
    float f[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int p = (unsigned)page[j] < (unsigned)a.src.num_pages ? page[j] : 0;
      f[j] = a.weights[((size_t)p * a.nkv + h.kh) * kPageSize + (64 * j + lane) % kPageSize];
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const uint32_t w = (unsigned)page[j] < (unsigned)a.src.num_pages ? ordered(f[j]) : kZeroWeight;
      v[j] = (unsigned)(64 * j + lane - h.s0) < h.span ? w : 0u;  // (others stay whatever they weigh)
    }
    int left = h.want;
    const uint32_t pre = left > 0 ? wave_threshold(v, h.c, 0u, 32, left) : 0xFFFFFFFFu;
    int32_t *kept = a.kept + ((size_t)seq * a.nkv + h.kh) * a.kept_stride;
    int pg = 0, pe = 0;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int t = 64 * j + lane;
      const bool gt = heavier(h, t, v[j], pre), eq = equal(h, t, v[j], pre);
      const uint64_t bg = __builtin_amdgcn_ballot_w64(gt), be = __builtin_amdgcn_ballot_w64(eq);
      const auto below = [](uint64_t b) {
        return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(b >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)b, 0u));
      };
      const int g = pg + below(bg), q = pe + below(be);
      if (gt || (eq && q < left)) {
        at[g + min(q, left)] = t;
        kept[g + min(q, left)] = t;
      }
      pg += __builtin_popcountll(bg);
      pe += __builtin_popcountll(be);
    }
  }
  __syncthreads();
  copy_rows<RB, 256>(a, h, at, k, 0);
}

// ---------------------------------------------------------------------------
// longer requests: segments of kEvictSegment keys or a multiple
// ---------------------------------------------------------------------------
struct Segment {
  Head h;
  int head;      // seq nkv + kh
  int seg, at;   // segment of the request, its place in the per-segment arrays
  int t0, t1;    // keys
};
__device__ __forceinline__ Segment segment_of(const EvictArgs &a, meta_t m, int block) {
  Segment s;
  const int g = block / a.nkv, kh = block - g * a.nkv;
  const meta_t first = m + EV_SEG0 * a.S;
  const int seq = last_at_or_below(first, a.S, g);
  s.h = head_of(a, m, seq, kh);
  s.head = seq * a.nkv + kh;
  s.seg = __builtin_amdgcn_readfirstlane(g - first[seq]);
  s.at = block;
  const int len = evict_segment(s.h.c);
  s.t0 = s.seg * len;
  s.t1 = min(s.h.c, s.t0 + len);
  return s;
}
__device__ __forceinline__ int64_t list_at(const EvictArgs &a, meta_t m, const Head &h) {
  return ((int64_t)m[EV_LIST0 * a.S + h.seq] * a.nkv + (int64_t)h.kh * ((h.c + 15) / 16)) * 16;
}
constexpr int kTopShift = 21;  // the first 11 bits

__global__ __launch_bounds__(256) void k_evict_zero(EvictArgs a, int n) {
  for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) a.hist[i] = 0;
}

__global__ __launch_bounds__(kThreads) void k_evict_hist(EvictArgs a) {
  __shared__ int hist[kBins];
  const Segment s = segment_of(a, meta_words(a), blockIdx.x);
  const Head &h = s.h;
  if (h.keep >= h.c || h.want == 0) return;
  const int tid = threadIdx.x, lane = tid & 63;
  for (int i = tid; i < kBins; i += kThreads) hist[i] = 0;
  __syncthreads();
  int least = 0;  // keys that never received any weight, counted apart
  for (int t0 = s.t0; t0 < s.t1; t0 += 2 * kRun) {
    u32x4_t v[2];
    load_runs<2>(a, h, t0, v);
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int t = t0 + kRun * j + 4 * tid + e;
        if (t < s.t1 && (unsigned)(t - h.s0) < h.span) {
          if (v[j][e] == kZeroWeight)
            ++least;
          else
            atomicAdd(&hist[v[j][e] >> kTopShift], 1);
        }
      }
  }
  least = wave_scan(least);
  if (lane == 63 && least > 0) atomicAdd(&hist[kZeroWeight >> kTopShift], least);
  __syncthreads();
  for (int i = tid; i < kBins; i += kThreads)
    if (hist[i]) atomicAdd(&a.hist[(size_t)s.head * kBins + i], hist[i]);
}

// The bin of the threshold from the head's histogram.
EB_DEV void head_bin(const EvictArgs &a, int head, int &left, int &bin, int &in_bin, BinScratch &bs) {
  int own[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) own[i] = a.hist[(size_t)head * kBins + kBins - 1 - 4 * (int)threadIdx.x - i];
  find_bin(own, left, bin, in_bin, bs);
}

// Lists the keys of the threshold's bin and counts the segment's heavier ones
// (the keys that always stay are left out: their number is known).
__global__ __launch_bounds__(kThreads) void k_evict_list(EvictArgs a) {
  __shared__ BinScratch bs;
  __shared__ uint32_t lv[2 * kRun];
  __shared__ int lt[2 * kRun];
  __shared__ int n_here, base, total;
  const meta_t m = meta_words(a);
  const Segment s = segment_of(a, m, blockIdx.x);
  const Head &h = s.h;
  const int tid = threadIdx.x, lane = tid & 63;
  if (h.keep >= h.c || h.want == 0) return;
  int left = h.want, bin, in_bin;
  if (tid == 0) total = n_here = 0;
  head_bin(a, s.head, left, bin, in_bin, bs);
  const int64_t at = list_at(a, m, h);
  int more = 0;
  for (int t0 = s.t0; t0 < s.t1; t0 += 2 * kRun) {
    u32x4_t v[2];
    load_runs<2>(a, h, t0, v);
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int t = t0 + kRun * j + 4 * tid + e;
        if (t < s.t1 && (unsigned)(t - h.s0) < h.span) {
          const int b = (int)(v[j][e] >> kTopShift);
          more += b > bin;
          if (b == bin) {
            const int i = atomicAdd(&n_here, 1);
            lv[i] = v[j][e];
            lt[i] = t;
          }
        }
      }
    __syncthreads();
    if (tid == 0) base = atomicAdd(&a.list_n[s.head], n_here);
    __syncthreads();
    for (int i = tid; i < n_here; i += kThreads) {
      a.list_v[at + base + i] = lv[i];
      a.list_t[at + base + i] = lt[i];
    }
    __syncthreads();
    if (tid == 0) n_here = 0;
    __syncthreads();
  }
  more = wave_scan(more);
  if (lane == 63) atomicAdd(&total, more);
  __syncthreads();
  if (tid == 0) a.seg_heavier[s.at] = total;
}

// One block per (request, kv head): the threshold among the listed keys, and
// the heavier and equal keys before each segment.
__global__ __launch_bounds__(kThreads) void k_evict_solve(EvictArgs a) {
  __shared__ BinScratch bs;
  __shared__ int hist[kBins];
  __shared__ int seg_g[kEvictSegments], seg_e[kEvictSegments], part_g[kWaves], part_e[kWaves];
  const meta_t m = meta_words(a);
  const int seq = blockIdx.x / a.nkv;
  const Head h = head_of(a, m, seq, blockIdx.x - seq * a.nkv);
  const int head = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int len = evict_segment(h.c), first = m[EV_SEG0 * a.S + seq], nseg = (h.c + len - 1) / len;
  const bool plain = h.keep >= h.c || h.want == 0;
  uint32_t pre = h.keep >= h.c ? 0u : 0xFFFFFFFFu;
  int left = 0;
  seg_g[tid] = seg_e[tid] = 0;
  static_assert(kEvictSegments == kThreads, "a segment per thread");
  if (!plain) {
    left = h.want;
    int bin, in_bin;
    head_bin(a, head, left, bin, in_bin, bs);
    const int64_t at = list_at(a, m, h);
    const uint32_t *lv = a.list_v + at;
    const int32_t *lt = a.list_t + at;
    const int n = in_bin;
    pre = (uint32_t)bin << kTopShift;
    if (n <= kListMost) {
      uint32_t v[kListMost / 64];  // every wavefront for itself
#pragma unroll
      for (int j = 0; j < kListMost / 64; ++j) v[j] = 64 * j + lane < n ? lv[64 * j + lane] : 0u;
      pre = wave_threshold(v, n, pre, kTopShift, left);
    } else {
      for (int top = kTopShift; top > 0;) {
        const int bits = min(top, 11), sh = top - bits;
        for (int i = tid; i < kBins; i += kThreads) hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += kThreads) {
          const uint32_t v = lv[i];
          if ((v >> top) == (pre >> top)) {
            // (equal weights meet on one counter: once for those of a wavefront)
            const int b = (int)((v >> sh) & ((1u << bits) - 1u));
            const uint64_t live = __builtin_amdgcn_ballot_w64(true);
            const int one = __builtin_amdgcn_readfirstlane(b);
            if (__builtin_amdgcn_ballot_w64(b != one) == 0) {
              if (lane == __builtin_ctzll(live)) atomicAdd(&hist[one], __builtin_popcountll(live));
            } else {
              atomicAdd(&hist[b], 1);
            }
          }
        }
        __syncthreads();
        int own[4], in;
#pragma unroll
        for (int i = 0; i < 4; ++i) own[i] = hist[kBins - 1 - 4 * tid - i];
        find_bin(own, left, bin, in, bs);
        pre |= (uint32_t)bin << sh;
        top = sh;
      }
    }
    __syncthreads();
    for (int i = tid; i < n; i += kThreads) {
      const uint32_t v = lv[i];
      if (v > pre) atomicAdd(&seg_g[lt[i] / len], 1);
      if (v == pre) atomicAdd(&seg_e[lt[i] / len], 1);
    }
  }
  __syncthreads();
  const int mine = (first + tid) * a.nkv + h.kh;
  const int g = tid < nseg && !plain ? seg_g[tid] + a.seg_heavier[mine] : 0, e = seg_e[tid];
  const int gi = wave_scan(g), ei = wave_scan(e);
  if (lane == 63) {
    part_g[wave] = gi;
    part_e[wave] = ei;
  }
  __syncthreads();
  int gb = gi - g, eb = ei - e;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    gb += w < wave ? part_g[w] : 0;
    eb += w < wave ? part_e[w] : 0;
  }
  if (tid < nseg) {
    a.seg_heavier[mine] = gb;
    a.seg_equal[mine] = eb;
  }
  if (tid == 0) {
    a.solved[2 * head] = (int32_t)pre;
    a.solved[2 * head + 1] = left;
  }
}

// The segment's kept keys and their copy.
template <int RB>
__global__ __launch_bounds__(kThreads) void k_evict_place(EvictArgs a) {
  __shared__ int cnt[2 * kWaves], at[2 * kRun];
  const meta_t m = meta_words(a);
  const Segment s = segment_of(a, m, blockIdx.x);
  const Head &h = s.h;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t pre = (uint32_t)a.solved[2 * s.head];
  const int left = a.solved[2 * s.head + 1];
  int32_t *kept = a.kept + ((size_t)h.seq * a.nkv + h.kh) * a.kept_stride;
  // heavier (or always kept) and equal keys before the keys at hand
  int g0 = a.seg_heavier[s.at], e0 = a.seg_equal[s.at];
  g0 += min(s.t0, h.s0) + max(0, s.t0 - (h.s0 + (int)h.span));
  if (h.keep >= h.c) g0 = s.t0;
  for (int t0 = s.t0; t0 < s.t1; t0 += 2 * kRun) {
    u32x4_t v[2];
    load_runs<2>(a, h, t0, v);
    int before[2];
    auto gt_at = [&](int j, int e) {
      const int t = t0 + kRun * j + 4 * tid + e;
      return t < s.t1 && (h.keep >= h.c || heavier(h, t, v[j][e], pre));
    };
    auto eq_at = [&](int j, int e) {
      const int t = t0 + kRun * j + 4 * tid + e;
      return t < s.t1 && h.keep < h.c && equal(h, t, v[j][e], pre);
    };
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      int x = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) x += (gt_at(j, e) ? 1 : 0) + (eq_at(j, e) ? 1 << 16 : 0);
      const int upto = wave_scan(x);
      before[j] = upto - x;
      if (lane == 63) cnt[j * kWaves + wave] = upto;
    }
    __syncthreads();
    const int x = lane < 2 * kWaves ? cnt[lane] : 0;
    const int gi = wave_scan(x & 0xFFFF), ei = wave_scan(x >> 16);
    const int gx = gi - (x & 0xFFFF), ex = ei - (x >> 16);
    const int j0 = g0 + min(e0, left);  // the first kept key's slot
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      int pg = g0 + __shfl(gx, j * kWaves + wave, 64) + (before[j] & 0xFFFF);
      int pe = e0 + __shfl(ex, j * kWaves + wave, 64) + (before[j] >> 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool gt = gt_at(j, e), eq = eq_at(j, e);
        if (gt || (eq && pe < left)) {
          const int to = pg + min(pe, left), t = t0 + kRun * j + 4 * tid + e;
          kept[to] = t;
          at[to - j0] = t;
        }
        pg += gt;
        pe += eq;
      }
    }
    g0 += __builtin_amdgcn_readlane(gi, 63);
    e0 += __builtin_amdgcn_readlane(ei, 63);
    const int n = g0 + min(e0, left) - j0;
    __syncthreads();
    if (n > 0) copy_rows<RB, kThreads>(a, h, at, n, j0);
    __syncthreads();
  }
}

}  // namespace

hipError_t launch_evict(const Shape &s, const EvictCall &c, hipStream_t st) {
  const EvictPlan &p = *c.plan;
  EvictArgs a;
  memset(&a, 0, sizeof a);
  a.src = c.src;
  a.dst = c.dst;
  a.weights = c.weights;
  a.dst_weights = c.dst_weights;
  a.kept = c.kept;
  a.S = p.S;
  a.nkv = s.nkv;
  a.sink = c.sink;
  a.recent = c.recent;
  a.kept_stride = c.kept_stride;
  hipError_t e = hipSuccess;
  if (p.words.size() <= (size_t)kInlineInts) {
    memcpy(a.inl.w, p.words.data(), p.words.size() * sizeof(int32_t));
  } else {
    int32_t *place = reinterpret_cast<int32_t *>(c.ws + p.o_words);
    a.meta = place;
    if ((e = put_words(p.words.data(), p.words.size(), place, st)) != hipSuccess) return e;
  }
  const int heads = p.S * s.nkv, rb = s.hd * (c.src.f8 ? 1 : 2);
#define EB_BY_ROW(KERNEL_, GRID_, BLOCK_)                                      \
  do {                                                                         \
    if (rb == 256)                                                             \
      hipLaunchKernelGGL(KERNEL_<256>, dim3(GRID_), dim3(BLOCK_), 0, st, a);   \
    else if (rb == 128)                                                        \
      hipLaunchKernelGGL(KERNEL_<128>, dim3(GRID_), dim3(BLOCK_), 0, st, a);   \
    else                                                                       \
      hipLaunchKernelGGL(KERNEL_<64>, dim3(GRID_), dim3(BLOCK_), 0, st, a);    \
  } while (0)
  if (p.max_len <= kEvictFew) {
    EB_BY_ROW(k_evict_few, heads, 256);
    return hipGetLastError();
  }
  if (p.max_len <= kEvictBlock) {
    if (p.max_len <= 2 * kRun)
      hipLaunchKernelGGL(k_evict_select<2>, dim3(heads), dim3(kThreads), 0, st, a);
    else if (p.max_len <= 4 * kRun)
      hipLaunchKernelGGL(k_evict_select<4>, dim3(heads), dim3(kThreads), 0, st, a);
    else
      hipLaunchKernelGGL(k_evict_select<8>, dim3(heads), dim3(kThreads), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess || p.groups == 0) return e;
    EB_BY_ROW(k_evict_copy, (unsigned)(p.groups * s.nkv), 256);
    return hipGetLastError();
  }
  a.hist = reinterpret_cast<int32_t *>(c.ws + p.o_hist);
  a.list_n = a.hist + (size_t)heads * kBins;
  a.list_v = reinterpret_cast<uint32_t *>(c.ws + p.o_list_v);
  a.list_t = reinterpret_cast<int32_t *>(c.ws + p.o_list_t);
  a.seg_heavier = reinterpret_cast<int32_t *>(c.ws + p.o_seg);
  a.seg_equal = a.seg_heavier + (size_t)p.segments * s.nkv;
  a.solved = reinterpret_cast<int32_t *>(c.ws + p.o_solved);
  const unsigned blocks = (unsigned)(p.segments * s.nkv);
  const int words = heads * (kBins + 1);
  hipLaunchKernelGGL(k_evict_zero, dim3((words + 2047) / 2048 < 512 ? (words + 2047) / 2048 : 512), dim3(256), 0, st, a,
                     words);
  hipLaunchKernelGGL(k_evict_hist, dim3(blocks), dim3(kThreads), 0, st, a);
  hipLaunchKernelGGL(k_evict_list, dim3(blocks), dim3(kThreads), 0, st, a);
  hipLaunchKernelGGL(k_evict_solve, dim3(heads), dim3(kThreads), 0, st, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  EB_BY_ROW(k_evict_place, blocks, kThreads);
#undef EB_BY_ROW
  return hipGetLastError();
}

}  // namespace eb
