// Rotary positions with the cache append: half or neighbouring pairs, the
// leading part of each head, positions apart from the cache slots, and the
// frequencies the caller scaled.
//
// Pair t (t < R / 2) of a head at position p turns by p f_t:
//   (x, y) -> m (x cos - y sin, x sin + y cos).
// The turn p f_t / 2 pi is formed and reduced to [-1/2, 1/2] in fp64 (p and
// the context can be long), its sine and cosine are taken in fp32 of the
// reduced angle, the products are fp32 and each result is rounded once.
//
// The work is 3 R operations per head against 4 R + bytes moved: memory bound,
// and at a few rows bound by one launch's latency (7000 rows of 48 heads of 128:
// 32.7 us, 5.2 TB/s; one row 2.9 us).  So every block issues
// all of its loads, forms the angles of its rows while they are in flight
// (once per row, shared by all heads through LDS) and then stores.
#include <string.h>

#include "device_common.h"
#include "eb_internal.h"
#include "op_meta.h"
#include "ops.h"

namespace eb {

namespace {

// Fewer words than other kernels carry: the host writes every call's arguments
// out, and one row's call is bound by that (768 words 7.7 us, 256 words 6.8).
constexpr size_t kRotWords = 256;

struct RotArgs {
  uint16_t *qkv;
  uint8_t *kc, *vc;  // null: no cache, k is rotated in place
  const int32_t *bt, *positions;
  const uint16_t *gq, *gk;
  int32_t num_pages, max_pages, T, S, nq, nkv, R, rows_per_block, uniform_n;
  float ks, vs, eps, mag;
  const int32_t *meta;  // [S] contexts, then [S] first rows (unless uniform_n)
  double turn[64];      // f_t / 2 pi
  WordsOf<kRotWords> inl;
};
static_assert(sizeof(RotArgs) < 4096, "kernel arguments");

// Request and cache slot of row r.
__device__ __forceinline__ void row_place(const RotArgs &a, meta_t m, int r, int &seq, int &slot) {
  if (a.uniform_n > 0) {
    seq = r / a.uniform_n;
    slot = m[seq] + r - seq * a.uniform_n;
    return;
  }
  const meta_t first = m + a.S;
  int lo = 0, hi = a.S - 1;
  while (lo < hi) {  // last request whose first row is <= r
    const int mid = (lo + hi + 1) >> 1;
    if (first[mid] <= r)
      lo = mid;
    else
      hi = mid - 1;
  }
  seq = lo;
  slot = m[lo] + r - first[lo];
}

// A head is the work of HD / 16 adjacent threads with two 16-byte chunks each:
// half pairs, chunks 8 t and R / 2 + 8 t of the rotated part; neighbouring
// pairs, chunks 16 t and 16 t + 8; past the rotated part, two chunks of the
// rest.  Block x takes rows_per_block rows, block y one part of NI x 256
// (head, thread) units of them.
constexpr int kMaxRows = 16;

template <int HD, bool F8, bool QKN, bool INTER, int NI>
__global__ __launch_bounds__(256) void k_rotary_append(RotArgs a) {
  constexpr int TPH = HD / 16;
  __shared__ float cs[kMaxRows * HD / 2], sn[kMaxRows * HD / 2];
  const meta_t m = meta_words(a);
  const int nh = a.nq + 2 * a.nkv, U = nh * TPH, cols = nh * HD;
  const int r0 = blockIdx.x * a.rows_per_block;
  const int nrows = min(a.rows_per_block, a.T - r0);
  const int half = a.R >> 1, rt = a.R >> 4;  // pairs, threads of a head that rotate
  const bool cache = a.kc != nullptr;

  u32x4_t x0[NI], x1[NI];
  int row[NI], head[NI], c0[NI], c1[NI], kind[NI];  // kind: -1 nothing, 0 q, 1 k, 2 v
#pragma unroll
  for (int j = 0; j < NI; ++j) {
    const int i = (blockIdx.y * NI + j) * 256 + threadIdx.x;
    const int rr = i / U, u = i - rr * U;
    head[j] = u / TPH;
    const int t = u - head[j] * TPH;
    row[j] = rr;
    kind[j] = head[j] < a.nq ? 0 : head[j] < a.nq + a.nkv ? 1 : 2;
    const bool turns = t < rt;
    if (INTER) {
      c0[j] = 16 * t;
      c1[j] = 16 * t + 8;
    } else {
      c0[j] = turns ? 8 * t : 16 * t;
      c1[j] = turns ? half + 8 * t : 16 * t + 8;
    }
    // nothing to do: past the block's rows, v or the plain end of a q (or uncached k) head
    if (rr >= nrows || (kind[j] == 2 && !cache) || (!turns && !QKN && (kind[j] == 0 || (kind[j] == 1 && !cache))))
      kind[j] = -1;
    const uint16_t *src = a.qkv + (size_t)(r0 + (kind[j] < 0 ? 0 : rr)) * cols + (kind[j] < 0 ? 0 : head[j]) * HD;
    x0[j] = x1[j] = u32x4_t{0u, 0u, 0u, 0u};
    if (kind[j] >= 0) {
      x0[j] = ld_u32x4(src + c0[j]);
      x1[j] = ld_u32x4(src + c1[j]);
    }
  }
  for (int i = threadIdx.x; i < nrows * half; i += 256) {
    const int rr = i / half, t = i - rr * half;
    int pos;
    if (a.positions) {
      pos = a.positions[r0 + rr];
    } else {
      int seq;
      row_place(a, m, r0 + rr, seq, pos);
    }
    typedef const __attribute__((address_space(4))) char *karg_t;
    const double *turn =
        (const double *)((karg_t)__builtin_amdgcn_kernarg_segment_ptr() + offsetof(RotArgs, turn));
    const double rev = (double)pos * turn[t];
    const double red = rev - rint(rev);
    float s, c;
    sincosf((float)(red * 6.283185307179586476925286766559), &s, &c);
    cs[i] = c * a.mag;
    sn[i] = s * a.mag;
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < NI; ++j) {
    if (kind[j] < 0) continue;  // (whole heads: the threads of one head go together)
    const int t = INTER ? c0[j] >> 4 : (c0[j] < half ? c0[j] >> 3 : c0[j] >> 4);
    const bool turns = t < rt && kind[j] < 2;
    u32x4_t y0 = x0[j], y1 = x1[j];
    if (kind[j] < 2 && (turns || QKN)) {
      float f0[8], f1[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f0[2 * e] = bf16_lo(x0[j][e]);
        f0[2 * e + 1] = bf16_hi(x0[j][e]);
        f1[2 * e] = bf16_lo(x1[j][e]);
        f1[2 * e + 1] = bf16_hi(x1[j][e]);
      }
      if constexpr (QKN) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss += f0[e] * f0[e] + f1[e] * f1[e];
        for (int o = 1; o < TPH; o <<= 1) ss += __shfl_xor(ss, o, 64);
        const float rs = 1.f / sqrtf(ss / (float)HD + a.eps);
        const uint16_t *gain = kind[j] == 0 ? a.gq : a.gk;
        const u32x4_t g0 = ld_u32x4(gain + c0[j]), g1 = ld_u32x4(gain + c1[j]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          f0[2 * e] *= rs * bf16_lo(g0[e]);
          f0[2 * e + 1] *= rs * bf16_hi(g0[e]);
          f1[2 * e] *= rs * bf16_lo(g1[e]);
          f1[2 * e + 1] *= rs * bf16_hi(g1[e]);
        }
      }
      if (turns) {
        const float *c = cs + row[j] * half + 8 * t, *s = sn + row[j] * half + 8 * t;
        float n0[8], n1[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          // pair e of the thread: half pairs (f0[e], f1[e]); neighbours (f[2e], f[2e + 1])
          const float x = INTER ? (e < 4 ? f0[2 * (e & 3)] : f1[2 * (e & 3)]) : f0[e];
          const float y = INTER ? (e < 4 ? f0[2 * (e & 3) + 1] : f1[2 * (e & 3) + 1]) : f1[e];
          const float u = x * c[e] - y * s[e], w = x * s[e] + y * c[e];
          if (INTER) {
            (e < 4 ? n0 : n1)[2 * (e & 3)] = u;
            (e < 4 ? n0 : n1)[2 * (e & 3) + 1] = w;
          } else {
            n0[e] = u;
            n1[e] = w;
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          f0[e] = n0[e];
          f1[e] = n1[e];
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        y0[e] = pack_bf16x2(f0[2 * e], f0[2 * e + 1]);
        y1[e] = pack_bf16x2(f1[2 * e], f1[2 * e + 1]);
      }
    }
    if (kind[j] == 0 || !cache) {
      uint16_t *dst = a.qkv + (size_t)(r0 + row[j]) * cols + head[j] * HD;
      st_u32x4(dst + c0[j], y0);
      st_u32x4(dst + c1[j], y1);
      continue;
    }
    int seq, slot;
    row_place(a, m, r0 + row[j], seq, slot);
    const int page = a.bt[(size_t)seq * a.max_pages + slot / kPageSize];
    if ((unsigned)page >= (unsigned)a.num_pages) continue;
    const int kh = head[j] - a.nq - (kind[j] == 2 ? a.nkv : 0);
    const size_t e0 = (((size_t)page * a.nkv + kh) * kPageSize + slot % kPageSize) * HD;
    uint8_t *base = kind[j] == 1 ? a.kc : a.vc;
    if constexpr (F8) {
      const float sc = kind[j] == 1 ? a.ks : a.vs;
      *reinterpret_cast<u32x2_t *>(base + e0 + c0[j]) = e4m3x8_of_bf16x8(y0, sc);
      *reinterpret_cast<u32x2_t *>(base + e0 + c1[j]) = e4m3x8_of_bf16x8(y1, sc);
    } else {
      st_u32x4(base + 2 * (e0 + c0[j]), y0);
      st_u32x4(base + 2 * (e0 + c1[j]), y1);
    }
  }
}

}  // namespace

hipError_t launch_rotary_append(const Shape &s, const RotaryCall &c, hipStream_t st) {
  RotArgs a{};
  a.qkv = c.qkv;
  a.kc = reinterpret_cast<uint8_t *>(c.kv.k);
  a.vc = reinterpret_cast<uint8_t *>(c.kv.v);
  a.bt = c.kv.bt;
  a.positions = c.positions;
  a.gq = c.gq;
  a.gk = c.gk;
  a.num_pages = c.kv.num_pages;
  a.max_pages = c.kv.max_pages;
  a.T = c.T;
  a.S = c.S;
  a.nq = s.nq;
  a.nkv = s.nkv;
  a.R = c.R;
  a.uniform_n = c.uniform_n;
  a.ks = c.kv.ks;
  a.vs = c.kv.vs;
  a.eps = s.eps;
  a.mag = c.magnitude;
  for (int t = 0; t < c.R / 2; ++t) a.turn[t] = c.turn[t];
  if (c.table.n <= kRotWords) {
    memcpy(a.inl.w, c.table.words, c.table.n * sizeof(int32_t));
  } else {
    a.meta = c.table.dev;
    const hipError_t e = put_words(c.table.words, c.table.n, c.table.dev, st);
    if (e != hipSuccess) return e;
  }
  // A wide call takes up to 1024 units (four per thread, 128 bytes in flight
  // each) of whole rows per block, a narrow one a single unit per thread (rows
  // of 48 heads of 128, narrow and wide: 256 3.7 and 5.0 us, 1000 10.1 both, 2000
  // 17.7 and 16.5).
  const int U = (s.nq + 2 * s.nkv) * (s.hd / 16);
  const bool wide = (long)c.T * U >= 1024L * 512;
  const int per = wide ? 1024 : 256;
  a.rows_per_block = wide ? (per / U < 1 ? 1 : per / U > kMaxRows ? kMaxRows : per / U) : 1;
  const dim3 grid((c.T + a.rows_per_block - 1) / a.rows_per_block, (a.rows_per_block * U + per - 1) / per);
#define EB_ROT(HD_, F8_, QKN_, INTER_)                                                               \
  do {                                                                                               \
    if (wide)                                                                                        \
      hipLaunchKernelGGL((k_rotary_append<HD_, F8_, QKN_, INTER_, 4>), grid, dim3(256), 0, st, a);   \
    else                                                                                             \
      hipLaunchKernelGGL((k_rotary_append<HD_, F8_, QKN_, INTER_, 1>), grid, dim3(256), 0, st, a);   \
    return hipGetLastError();                                                                        \
  } while (0)
#define EB_ROT_I(HD_, F8_, QKN_)              \
  do {                                        \
    if (c.interleaved) EB_ROT(HD_, F8_, QKN_, true); \
    EB_ROT(HD_, F8_, QKN_, false);            \
  } while (0)
#define EB_ROT_N(HD_, F8_)            \
  do {                                \
    if (s.qkn) EB_ROT_I(HD_, F8_, true); \
    EB_ROT_I(HD_, F8_, false);        \
  } while (0)
  if (s.hd == 128) {
    if (c.kv.f8) EB_ROT_N(128, true);
    EB_ROT_N(128, false);
  }
  if (s.hd == 64) {
    if (c.kv.f8) EB_ROT_N(64, true);
    EB_ROT_N(64, false);
  }
#undef EB_ROT_N
#undef EB_ROT_I
#undef EB_ROT
  return hipErrorInvalidValue;
}

}  // namespace eb
