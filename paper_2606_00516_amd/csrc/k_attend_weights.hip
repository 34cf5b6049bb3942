// The weights that the cached keys receive from the rows of chunk requests:
//   weights[t] += sum over rows r and heads h of 2^(s_rht - lse_rh),
// with the rows' log-sum-exp from the attention that ran before.
//
// The same scores again, key by key instead of row by row, so that each
// weight is one lane's register sum and no atomics are needed.  A block takes
// 64 keys of a (request, kv head), held by each of its four wavefronts as two
// 32-key A operands; the wavefronts take every fourth run of 32 rows (32 / G
// positions x G heads; with few blocks the runs are split into parts, which
// k_attend_weights_join adds in their order; with many blocks and few runs each
// wavefront has 64 keys of its own, by the plan's rule), loaded straight into
// registers one run ahead: no LDS
// and no barrier on the walk, whose length is that of the block whose keys
// the most rows see (six prompts of about 1800 rows in documents of 300, hd 64:
// 96 us through LDS tiles that the block shared, 56 so).  Per 32 x 64 scores 2 hd / 16 products of 32
// cycles stand against 32 exponentials, multiply-adds and sums per lane
// (about 26 cycles each, 70 with the cap): bound by the vector unit.
#include <string.h>

#include <cmath>

#include "attend_device.h"

namespace eb {

namespace {

constexpr int kWaves = kWeightWaves;

// A block's request, place in it and keys.
struct WBlock {
  int k, seq, row0, c, n, prefix, parts, at, part, j0, k0, keys;  // at: block of keys in the request
};
__device__ __forceinline__ WBlock weight_block(const AttendArgs &a, meta_t m, int blk, bool join) {
  WBlock b;
  b.k = last_at_or_below(m + (join ? PRE_WJOIN0 : PRE_WBLOCK0) * a.n, a.n, blk);
  const auto field = [&](int f) { return __builtin_amdgcn_readfirstlane(m[f * a.n + b.k]); };
  b.seq = field(PRE_SEQ);
  b.row0 = field(PRE_ROW);
  b.c = field(PRE_CTX);
  b.n = field(PRE_LEN);
  b.prefix = field(PRE_PREFIX);
  b.parts = field(PRE_WPARTS);
  const int local = blk - field(join ? PRE_WJOIN0 : PRE_WBLOCK0), parts = join ? 1 : max(b.parts, 1);
  b.at = local / parts;
  b.part = local - b.at * parts;
  b.j0 = a.weight_rows > 0 ? max(0, b.n - a.weight_rows) : 0;
  b.keys = b.parts == 0 ? kWeightKeys * kWaves : kWeightKeys;
  b.k0 = (min(b.c, attend_first(b.c + b.j0, a.window)) / b.keys + b.at) * b.keys;
  return b;
}
// The new weight of a key from what this call gives it.
__device__ __forceinline__ void add_weight(const AttendArgs &a, const WBlock &b, int kh, int key, float got) {
  if (key >= b.c + b.n) return;
  const int phys = a.kv.bt[(size_t)b.seq * a.kv.max_pages + key / kPageSize];
  if ((unsigned)phys >= (unsigned)a.kv.num_pages) return;
  float *dst = a.weights + ((size_t)phys * a.nkv + kh) * kPageSize + key % kPageSize;
  *dst = key < b.c ? *dst + got : got;  // a new key starts at what this call gives it
}

template <int HD, bool F8, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void k_attend_weights(AttendArgs a) {
  constexpr int NKS = HD / 16, KG = kWeightKeys / 32;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lq = lane & 31, lh = lane >> 5;
  const meta_t m = meta_words(a);
  const int blk = blockIdx.x / a.nkv, kh = blockIdx.x - blk * a.nkv;
  const WBlock b = weight_block(a, m, blk, false);
  const int seq = b.seq, row0 = b.row0, c = b.c, n = b.n, prefix = b.prefix, j0 = b.j0;
  const int klen = c + n, G = a.group, PB = 32 / G;  // positions per run
  const bool apart = b.parts == 0;                   // each wavefront has keys of its own
  const int kb = b.k0, kend = kb + b.keys;           // the block's keys
  const int k0 = kb + (apart ? wave * kWeightKeys : 0);
  const int cols = (a.nq + 2 * a.nkv) * HD;

  // rows that may see the block's keys: from the first position at or past
  // its first key (all of them below a prefix), up to the window's reach
  int ja = kb < prefix ? j0 : max(j0, kb - c);
  int jb = n;
  const int reach = kend - 1 - c;  // (compared before the window is added: any int32 is a window)
  if (a.window > 0 && reach < n - a.window) jb = max(0, reach + a.window);
  if (a.first_key) {
    // documents: only rows from the first to the last that sees one of the
    // block's keys are worth their products
    __shared__ int span[2];
    if (tid < 2) span[tid] = tid ? 0 : 0x7fffffff;
    __syncthreads();
    int mn = 0x7fffffff, mx = 0;
    for (int j = ja + tid; j < jb; j += 8 * 256) {
      int f[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) f[u] = a.first_key[row0 + min(j + 256 * u, n - 1)];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int ju = j + 256 * u;
        if (ju < jb && f[u] < min(kend, max(c + ju + 1, prefix))) {
          mn = min(mn, ju);
          mx = max(mx, ju + 1);
        }
      }
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
      mn = min(mn, __shfl_xor(mn, o, 64));
      mx = max(mx, __shfl_xor(mx, o, 64));
    }
    if (lane == 0) {
      atomicMin(&span[0], mn);
      atomicMax(&span[1], mx);
    }
    __syncthreads();
    ja = max(ja, __builtin_amdgcn_readfirstlane(span[0]));
    jb = min(jb, __builtin_amdgcn_readfirstlane(span[1]));
  }
  int runs = ja < jb ? (jb - ja + PB - 1) / PB : 0;
  if (b.parts > 1) {  // this part's runs
    const int lo = (int)((int64_t)runs * b.part / b.parts), hi = (int)((int64_t)runs * (b.part + 1) / b.parts);
    jb = min(jb, ja + hi * PB);
    ja += lo * PB;
    runs = hi - lo;
  }
  const int t0 = apart ? 0 : wave, step = apart ? 1 : kWaves;  // this wavefront's runs

  float acc[KG][16];
#pragma unroll
  for (int g = 0; g < KG; ++g)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[g][i] = 0.f;
  if (t0 < runs) {
    // K of the block's keys: lane (lq, lh) holds dims 16 ks + 8 lh .. of key 32 g + lq
    u32x4_t kf[KG][NKS];
#pragma unroll
    for (int g = 0; g < KG; ++g) {
      const int key = min(k0 + 32 * g + lq, klen - 1);
      const int phys = a.kv.bt[(size_t)seq * a.kv.max_pages + key / kPageSize];
      const bool ok = (unsigned)phys < (unsigned)a.kv.num_pages && k0 + 32 * g + lq < klen;
      const size_t e0 = (((size_t)(ok ? phys : 0) * a.nkv + kh) * kPageSize + key % kPageSize) * HD + 8 * lh;
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) {
        u32x4_t v;
        if constexpr (F8)
          v = e4m3x8_to_bf16x8(*reinterpret_cast<const u32x2_t *>(a.kv.k8() + e0 + ks * 16));
        else
          v = ld_u32x4(a.kv.k + e0 + ks * 16);
        kf[g][ks] = ok ? v : u32x4_t{0u, 0u, 0u, 0u};
      }
    }
    // Row lq of a run is position lq / G, head lq % G: its q as the B operand,
    // its visible keys [lo, lo + span) and its log-sum-exp in log2 units.
    // Runs past the end read the last row and see nothing.
    const int jr = lq / G, head = kh * G + lq - jr * G;
    const uint16_t *const qh = a.qkv + (size_t)row0 * cols + (size_t)head * HD + 8 * lh;
    float slope = 0.f;
    if constexpr (BIAS) slope = a.slopes[head] * kLog2e;
    struct Run {
      u32x4_t q[NKS];
      float lse;
      int first;
    };
    auto load = [&](int t, Run &r) {
      const int j = min(ja + t * PB + jr, n - 1);
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) r.q[ks] = ld_u32x4(qh + (size_t)j * cols + ks * 16);
      r.lse = a.lse[(size_t)(row0 + j) * a.nq + head];
      r.first = a.first_key ? a.first_key[row0 + j] : 0;
    };
    auto add = [&](int t, const Run &r) {
      const int j = ja + t * PB + jr, pos = c + j;
      const bool ok = j < jb;
      int lo = max(r.first, 0);
      if (a.window > 0) lo = max(lo, pos - a.window + 1);
      const int span = ok ? max(max(pos + 1, prefix) - lo, 0) : 0;
      const int d = k0 - lo;  // the block's first key from the row's
      // nothing of the block's keys visible to any of the 32 rows
      if (__builtin_amdgcn_ballot_w64(span > 0 && d + kWeightKeys > 0 && d < span) == 0) return;
      const bool masked = __builtin_amdgcn_ballot_w64(d < 0 || d + kWeightKeys > span) != 0;
      const float z = r.lse * kLog2e;
      const int dl = d + 4 * lh;
      const float d0 = BIAS ? (float)(pos - k0 - 4 * lh) : 0.f;
#pragma unroll
      for (int g = 0; g < KG; ++g) {
        f32x16_t one[1];
        f32x16_t &s = one[0];
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) s = mfma32x32x16(kf[g][ks], r.q[ks], s);
        if constexpr (CAP) {
          if (none(largest<1>(one) > a.small_raw)) {
            asm volatile("");  // (a branch: not both forms and a select)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = small_score(s[i], a);
          } else {
            asm volatile("");
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = capped_score(s[i], a);
          }
        }
        if constexpr (CAP || BIAS) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float v = CAP ? s[i] : s[i] * a.qscale;
            if constexpr (BIAS) v = fmaf(-slope, fabsf(d0 - (float)(32 * g + 8 * (i >> 2) + (i & 3))), v);
            s[i] = v - z;
          }
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = fmaf(s[i], a.qscale, -z);
        }
        if (masked) {
          asm volatile("");  // (a branch, not 16 selects in every run)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            s[i] = (unsigned)(dl + 32 * g + 8 * (i >> 2) + (i & 3)) < (unsigned)span ? s[i] : kNoScore;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = fast_exp2(s[i]);
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[g][i] += s[i];
      }
    };
    Run x, y;
    load(t0, x);
    for (int t = t0; t < runs; t += 2 * step) {
      load(t + step, y);
      add(t, x);
      load(t + 2 * step, x);
      add(t + step, y);
    }
  }
  // Over the 32 rows' lanes by halves: in each exchange a lane keeps the half
  // of its values that its own bit names and adds the partner's of that half
  // (31 exchanges instead of 5 for each of 32 values); lane lq ends with value
  // lq.  Then over the wavefronts in their order.
  __shared__ float part[kWaves][kWeightKeys];
  float v[16 * KG];
#pragma unroll
  for (int i = 0; i < 16 * KG; ++i) v[i] = acc[i / 16][i % 16];
  static_assert(KG == 2, "as many values as lanes of a half wavefront");
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) {
    const bool up = (lq & o) != 0;
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const float give = up ? v[i] : v[i + o], keep = up ? v[i + o] : v[i];
      v[i] = keep + shfl_xor_f32(give, o);
    }
  }
  part[wave][32 * (lq >> 4) + 8 * ((lq >> 2) & 3) + 4 * lh + (lq & 3)] = v[0];
  __syncthreads();
  if (apart) {
    add_weight(a, b, kh, kb + tid, part[wave][lane]);
  } else if (tid < kWeightKeys) {
    float got = part[0][tid];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) got += part[w][tid];
    if (b.parts > 1)
      a.wparts[((size_t)(m[PRE_WPART0 * a.n + b.k] + b.at * b.parts + b.part) * a.nkv + kh) * kWeightKeys + tid] = got;
    else
      add_weight(a, b, kh, kb + tid, got);
  }
}

// Joins the parts of the rows, in their order.
__global__ __launch_bounds__(kWeightKeys) void k_attend_weights_join(AttendArgs a) {
  const meta_t m = meta_words(a);
  const int blk = blockIdx.x / a.nkv, kh = blockIdx.x - blk * a.nkv, tid = threadIdx.x;
  const WBlock b = weight_block(a, m, blk, true);
  const float *src =
      a.wparts + ((size_t)(m[PRE_WPART0 * a.n + b.k] + b.at * b.parts) * a.nkv + kh) * kWeightKeys + tid;
  float got = 0.f;
  for (int p = 0; p < b.parts; ++p) got += src[(size_t)p * a.nkv * kWeightKeys];
  add_weight(a, b, kh, b.k0 + tid, got);
}

}  // namespace

hipError_t launch_attend_weights(const Shape &s, const AttendCall &c, const AttendArgs &a, hipStream_t st) {
  const dim3 grid(c.plan->pre_wblocks * s.nkv);
#define EB_WTS(HD_, F8_)                                                                                       \
  do {                                                                                                         \
    if (c.softcap > 0.f && c.slopes)                                                                           \
      hipLaunchKernelGGL((k_attend_weights<HD_, F8_, true, true>), grid, dim3(256), 0, st, a);                 \
    else if (c.softcap > 0.f)                                                                                  \
      hipLaunchKernelGGL((k_attend_weights<HD_, F8_, true, false>), grid, dim3(256), 0, st, a);                \
    else if (c.slopes)                                                                                         \
      hipLaunchKernelGGL((k_attend_weights<HD_, F8_, false, true>), grid, dim3(256), 0, st, a);                \
    else                                                                                                       \
      hipLaunchKernelGGL((k_attend_weights<HD_, F8_, false, false>), grid, dim3(256), 0, st, a);               \
  } while (0)
  if (s.hd == 128) {
    if (a.kv.f8)
      EB_WTS(128, true);
    else
      EB_WTS(128, false);
  } else {
    if (a.kv.f8)
      EB_WTS(64, true);
    else
      EB_WTS(64, false);
  }
#undef EB_WTS
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || c.plan->pre_wjoins == 0) return e;
  hipLaunchKernelGGL(k_attend_weights_join, dim3((unsigned)(c.plan->pre_wjoins * s.nkv)), dim3(kWeightKeys), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_attend_decode(const Shape &s, const AttendCall &c, const AttendArgs &a, hipStream_t st);
hipError_t launch_attend_chunk(const Shape &s, const AttendCall &c, const AttendArgs &a, hipStream_t st);

namespace {
hipError_t with_table(AttendArgs &a, const std::vector<int32_t> &t, int32_t n, char *place, hipStream_t st) {
  a.n = n;
  a.meta = nullptr;
  if (t.size() <= (size_t)kInlineInts) {
    memcpy(a.inl.w, t.data(), t.size() * sizeof(int32_t));
    return hipSuccess;
  }
  a.meta = reinterpret_cast<const int32_t *>(place);
  return put_words(t.data(), t.size(), reinterpret_cast<int32_t *>(place), st);
}
}  // namespace

hipError_t launch_attend(const Shape &s, const AttendCall &c, hipStream_t st) {
  const AttendPlan &p = *c.plan;
  AttendArgs a;
  memset(&a, 0, sizeof a);
  a.qkv = c.qkv;
  a.out = c.out;
  a.lse = c.lse ? c.lse : c.weights ? reinterpret_cast<float *>(c.ws + p.o_lse) : nullptr;
  a.weights = c.weights;
  a.part_o = reinterpret_cast<float *>(c.ws + p.o_part_o);
  a.part_ml = reinterpret_cast<float *>(c.ws + p.o_part_ml);
  a.scores = c.weights ? reinterpret_cast<float *>(c.ws + p.o_scores) : nullptr;
  a.wparts = reinterpret_cast<float *>(c.ws + p.o_wparts);
  a.first_key = c.first_key;
  a.slopes = c.slopes;
  a.kv = c.kv;
  a.nq = s.nq;
  a.nkv = s.nkv;
  a.group = s.group();
  a.window = c.window;
  a.weight_rows = c.weight_rows;
  const float scale = c.scale * (c.kv.f8 ? c.kv.ks : 1.f);
  a.qscale = c.softcap > 0.f ? 2.f * kLog2e * (scale / c.softcap) : kLog2e * scale;
  a.cap2 = c.softcap * kLog2e;
  a.ratio = c.softcap > 0.f ? scale / c.softcap : 0.f;
  if (c.softcap > 0.f) {
    const double y = (double)scale / c.softcap;
    double f = (double)c.softcap * 1.4426950408889634 * y;
    bool ok = true;
    for (int i = 0; i < 5; ++i, f *= y * y) {
      a.tanh_c[i] = (float)(f * kTanhP[i]);
      ok = ok && std::fabs(a.tanh_c[i]) > 1e-36f && std::fabs(a.tanh_c[i]) < 1e36f;
    }
    a.small_raw = ok ? (float)(kTanhSmall / y) : -1.f;  // (below every score: never)
    a.even_raw = std::fmin(a.small_raw, (float)(kCappedSlack / (1.4426950408889634 * scale)));
  }
  hipError_t e = hipSuccess;
  if (p.n_dec > 0) {
    e = with_table(a, p.dec, p.n_dec, c.ws + p.o_dec, st);
    // A split's scores wait in LDS for its end, if two blocks still share a CU.
    const size_t slots = (size_t)256 * s.hd * (c.kv.f8 ? 1 : 2), stash = (size_t)p.dec_most * a.group * sizeof(float);
    a.stash = c.weights && slots + stash <= 80 * 1024 ? (int32_t)stash : 0;
    if (e == hipSuccess) e = launch_attend_decode(s, c, a, st);
  }
  if (e == hipSuccess && p.n_pre > 0) {
    e = with_table(a, p.pre, p.n_pre, c.ws + p.o_pre, st);
    if (e == hipSuccess) e = launch_attend_chunk(s, c, a, st);
    if (e == hipSuccess && c.weights) e = launch_attend_weights(s, c, a, st);
  }
  return e;
}

}  // namespace eb
