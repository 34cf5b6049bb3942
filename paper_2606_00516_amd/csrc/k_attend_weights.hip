// The weights that the cached keys receive from the rows of chunk requests:
//   weights[t] += sum over rows r and heads h of 2^(s_rht - lse_rh),
// with the rows' log-sum-exp from the attention that ran before.
//
// The same scores again, key by key instead of row by row, so that each
// weight is one lane's register sum and no atomics are needed: a block takes
// 128 keys of a (request, kv head), each of its four wavefronts holds 32 keys'
// K in registers as the A operand, and the rows stream by in tiles of 64
// (64 / G positions) through two LDS buffers.  Per 32 x 32 scores 8 products of
// 32 cycles stand against 16 exponentials, multiply-adds and sums per lane
// (about 28 cycles each, 70 with the cap): bound by the vector unit.
#include <string.h>

#include "attend_device.h"

namespace eb {

namespace {

constexpr int kWaves = 4, kRT = 64;  // rows per tile

template <int HD, bool F8, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void k_attend_weights(AttendArgs a) {
  constexpr int ROW = HD * 2, CPR = ROW / 16, TILE = kRT * ROW;
  constexpr int NKS = HD / 16;
  constexpr int RPI = 1024 / ROW, NI = kRT / (RPI * kWaves);  // rows per load instruction, instructions per wave
  __shared__ __attribute__((aligned(16))) uint8_t buf[2 * TILE];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lq = lane & 31, lh = lane >> 5;
  const int32_t *m = meta_words(a);
  const int blk = blockIdx.x / a.nkv, kh = blockIdx.x - blk * a.nkv;
  const int k = last_at_or_below(m + PRE_WBLOCK0 * a.n, a.n, blk);
  const auto field = [&](int f) { return __builtin_amdgcn_readfirstlane(m[f * a.n + k]); };
  const int seq = field(PRE_SEQ), row0 = field(PRE_ROW), c = field(PRE_CTX), n = field(PRE_LEN),
            prefix = field(PRE_PREFIX);
  const int klen = c + n, G = a.group, PB = kRT / G;  // positions per tile
  const int j0 = a.weight_rows > 0 ? max(0, n - a.weight_rows) : 0;
  const int first = min(c, attend_first(c + j0, a.window)) / kWeightKeys;
  const int kb0 = (first + blk - field(PRE_WBLOCK0)) * kWeightKeys;  // the block's first key
  const int k0 = kb0 + wave * 32;                                         // this wavefront's
  const int cols = (a.nq + 2 * a.nkv) * HD;

  // K of the wavefront's 32 keys: lane (lq, lh) holds dims 16 ks + 8 lh .. of key lq
  u32x4_t kf[NKS];
  {
    const int key = min(k0 + lq, klen - 1);
    const int phys = a.kv.bt[(size_t)seq * a.kv.max_pages + key / kPageSize];
    const bool ok = (unsigned)phys < (unsigned)a.kv.num_pages && k0 + lq < klen;
    const size_t e0 = (((size_t)(ok ? phys : 0) * a.nkv + kh) * kPageSize + key % kPageSize) * HD + 8 * lh;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {
      u32x4_t v;
      if constexpr (F8)
        v = e4m3x8_to_bf16x8(*reinterpret_cast<const u32x2_t *>(a.kv.k8() + e0 + ks * 16));
      else
        v = ld_u32x4(a.kv.k + e0 + ks * 16);
      kf[ks] = ok ? v : u32x4_t{0u, 0u, 0u, 0u};
    }
  }
  // rows that may see the block's keys: from the first position at or past
  // its first key (all of them below a prefix), up to the window's reach
  int ja = kb0 < prefix ? j0 : max(j0, kb0 - c);
  int jb = n;
  if (a.window > 0) jb = min(n, max(0, kb0 + kWeightKeys - 1 + a.window - c));
  ja = ja / PB * PB;
  const int ntiles = ja < jb ? (jb - ja + PB - 1) / PB : 0;

  // row rr of a tile is position rr / G, head rr % G; load instruction i of
  // wave w fills rows RPI (i 4 + w) .. + RPI - 1, chunk ch of row rr at ch ^ (rr & 7)
  auto dma = [&](int t, uint8_t *dst) {
    const int pos = ja + t * PB;  // uniform
    const int left = n - pos;     // positions that exist
    const uint16_t *base = a.qkv + (size_t)(row0 + pos) * cols + (size_t)kh * G * HD;
    // (the range ends with the last row's last head of the group)
    const int bytes =
        __builtin_amdgcn_readfirstlane(left > 0 ? ((min(left, PB) - 1) * cols + G * HD) * 2 : 0);
    const buf_rsrc_t rs = make_rsrc(base, bytes);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int rr0 = RPI * (i * kWaves + wave), rr = rr0 + lane / CPR, ch = (lane % CPR) ^ (rr & 7);
      lds_dma16(rs, dst + rr0 * ROW, (uint32_t)(((rr / G) * cols + (rr % G) * HD) * 2 + 16 * ch));
    }
  };
  float acc[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = 0.f;
  int qaddr[4];
#pragma unroll
  for (int k4 = 0; k4 < 4; ++k4) qaddr[k4] = lq * ROW + 16 * ((2 * k4 + lh) ^ (lq & 7));
  // bounds and log-sum-exp (log2 units) of this lane's row in each half of a tile
  auto row_of = [&](int t, int half, int &rlo, int &rhi, int &pos, float &z, float &slope) {
    const int rr = half * 32 + lq, j = ja + t * PB + rr / G, h = kh * G + rr % G;
    const bool ok = j >= j0 && j < jb;
    const int row = row0 + (ok ? j : 0);
    pos = c + j;
    rlo = ok ? row_first(a, row, pos) : 0;
    rhi = ok ? max(pos + 1, prefix) : 0;
    z = ok ? a.lse[(size_t)row * a.nq + h] * kLog2e : 0.f;
    if constexpr (BIAS) slope = a.slopes[h] * kLog2e;
  };
  if (ntiles > 0) dma(0, buf);
  wait_loads<0>();
  __syncthreads();
  for (int t = 0; t < ntiles; ++t) {
    uint8_t *const cur = buf + (t & 1) * TILE;
    if (t + 1 < ntiles) dma(t + 1, buf + ((t + 1) & 1) * TILE);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      int rlo, rhi, pos;
      float z, slope = 0.f;
      row_of(t, half, rlo, rhi, pos, z, slope);
      // nothing of the wavefront's keys visible to any of the 32 rows
      if (__builtin_amdgcn_ballot_w64(rlo < k0 + 32 && rhi > k0 && rlo < rhi) == 0) continue;
      f32x16_t s;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) {
        const u32x4_t q = *reinterpret_cast<const u32x4_t *>(cur + half * 32 * ROW + qaddr[ks & 3] + 128 * (ks >> 2));
        s = mfma32x32x16(kf[ks], q, s);
      }
      const bool masked = __builtin_amdgcn_ballot_w64(rlo > k0 || rhi < k0 + 32) != 0;
      const float d0 = (float)(pos - k0 - 4 * lh);
      const int d = k0 + 4 * lh - rlo;
      const unsigned span = (unsigned)max(rhi - rlo, 0);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int at = 8 * (i >> 2) + (i & 3);
        float p;
        if constexpr (CAP || BIAS) {
          float v = mod_score<CAP>(s[i], a.qscale, a.cap2);
          if constexpr (BIAS) v = fmaf(-slope, fabsf(d0 - (float)at), v);
          p = fast_exp2(v - z);
        } else {
          p = fast_exp2(fmaf(s[i], a.qscale, -z));
        }
        if (masked) p = (unsigned)(d + at) < span ? p : 0.f;
        acc[i] += p;
      }
    }
    wait_loads<0>();
    __syncthreads();
  }
  // over the 32 rows' lanes; lane lq keeps value lq % 16
  float mine = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float v = acc[i];
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) v += shfl_xor_f32(v, o);
    mine = (lq & 15) == i ? v : mine;
  }
  if (lq < 16) {
    const int key = k0 + 8 * (lq >> 2) + 4 * lh + (lq & 3);
    if (key < klen) {
      const int phys = a.kv.bt[(size_t)seq * a.kv.max_pages + key / kPageSize];
      if ((unsigned)phys < (unsigned)a.kv.num_pages) {
        float *dst = a.weights + ((size_t)phys * a.nkv + kh) * kPageSize + key % kPageSize;
        *dst = key < c ? *dst + mine : mine;  // a new key starts at what this call gives it
      }
    }
  }
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
  hipError_t e = hipSuccess;
  if (p.n_dec > 0) {
    e = with_table(a, p.dec, p.n_dec, c.ws + p.o_dec, st);
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
