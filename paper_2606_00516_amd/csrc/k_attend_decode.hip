// Decode rows of the modified attention: one new row per request.
//
// A block takes one (request, split of its keys, kv head) and serves the G
// query heads of the kv head, so every cached byte is read once: 4 G hd
// operations for 2 hd elements, far below the matrix cores' rate, bound by
// HBM.  Its four wavefronts stream the split's pages w, w + 4, .. through
// two LDS slots each (direct loads, no registers) with one page in flight
// while another is worked on; at two blocks per CU that is 64 KiB in flight
// per CU (64 rows over 2350 keys on average, 8 kv heads, bf16: 109 us, 5.6 TB/s;
// 13 rows over 69000, 8 bits: 327 us, 5.6 TB/s).  Scores are formed as S^T = K Q^T on 16x16x32 products (16 tokens x
// 16 columns, G of them heads; lane l holds tokens 4 (l / 16) .. + 3 of head
// l % 16), so the cap, the bias and the mask cost 4 values per lane and page
// whatever G is.  O^T += V^T P^T takes V^T by the transposing LDS read; 8-bit
// pages become bf16 on the way and are transposed by a product with a 0/1
// matrix, which is exact.
//
// Splits are joined by k_attend_decode_combine; with weights, the scores are left
// in the workspace (4 G bytes per key beside the 4 hd read: 112 -> 125 us) and
// k_attend_decode_weights turns them into normalised weights once the rows'
// log-sum-exp is known (9 us), instead of reading K a second time.
#include "attend_device.h"

namespace eb {

namespace {

constexpr int kWaves = 4;

struct DecRow {
  int d, seq, row, ctx, first, nkeys;  // first: first key streamed (of a whole page); nkeys = ctx + 1
};
__device__ __forceinline__ DecRow dec_row(const AttendArgs &a, meta_t m, int d) {
  DecRow r;
  // (uniform; said so, so that what follows from them stays in scalar registers)
  r.d = d;
  r.seq = __builtin_amdgcn_readfirstlane(m[DEC_SEQ * a.n + d]);
  r.row = __builtin_amdgcn_readfirstlane(m[DEC_ROW * a.n + d]);
  r.ctx = __builtin_amdgcn_readfirstlane(m[DEC_CTX * a.n + d]);
  r.first = attend_first(r.ctx, a.window);
  r.nkeys = r.ctx + 1;
  return r;
}

// Blocks are dealt round-robin to the 8 XCDs; within a run of 64 blocks, block
// b takes unit 8 (b % 8) + (b % 64) / 8, so that the kv heads of one split,
// whose blocks lie in the same pages, run on one XCD.
__device__ __forceinline__ int xcd_unit(int b, int n) {
  if (b >= (n & ~63)) return b;
  return (b & ~63) + ((b & 7) << 3) + ((b & 63) >> 3);
}

template <int HD, bool F8, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void k_attend_decode(AttendArgs a) {
  using Tr = MdecTraits<HD, F8>;
  constexpr int NKS = HD / 32, NOB = HD / 16, MAXG = 8;
  constexpr int ARRAY = kWaves * Tr::SLOT;
  static_assert(kWaves * MAXG * (HD + 2) * 4 <= 2 * ARRAY, "merge area");
  __shared__ __attribute__((aligned(16))) uint8_t lds[2 * ARRAY];
  extern __shared__ __attribute__((aligned(16))) float stash[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  const int G = a.group;
  const meta_t m = meta_words(a);
  const int unit = xcd_unit(blockIdx.x, gridDim.x);
  const int split = unit / a.nkv, kh = unit - split * a.nkv;
  const DecRow r = dec_row(a, m, last_at_or_below(m + DEC_SPLIT0 * a.n, a.n, split));
  const int sp = __builtin_amdgcn_readfirstlane(split - m[DEC_SPLIT0 * a.n + r.d]);
  const int per = attend_split_keys(r.nkeys - r.first);
  const int k0 = r.first + sp * per, k1 = min(r.nkeys, k0 + per);
  const int nsplit = (r.nkeys - r.first + per - 1) / per;
  const int lo = __builtin_amdgcn_readfirstlane(min(row_first(a, r.row, r.ctx), r.nkeys));
  // (not before the first visible key: pages that the row sees nothing of are not read)
  const int pg0 = max(k0, lo) / kPageSize, pg1 = (k1 + kPageSize - 1) / kPageSize;
  const int32_t *bt = a.kv.bt + (size_t)r.seq * a.kv.max_pages;

  // q of the G heads as the B operand (columns past G zero)
  u32x4_t qb[NKS];
  {
    const int cols = (a.nq + 2 * a.nkv) * HD;
    const bool live = c < G;
    const uint16_t *src = a.qkv + (size_t)r.row * cols + (kh * G + (live ? c : 0)) * HD + g * 8;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {
      const u32x4_t v = ld_u32x4(src + ks * 32);
      qb[ks] = live ? v : u32x4_t{0u, 0u, 0u, 0u};
    }
  }
  // Sel_h[k][c] = 1 where k = c + 16 h: lane (c, g) holds k = 8 g .. 8 g + 7
  u32x4_t sel[2];
  if constexpr (F8) {
    const uint32_t one = (c & 1) ? 0x3F800000u : 0x3F80u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool hit = g == 2 * h + (c >> 3);
#pragma unroll
      for (int e = 0; e < 4; ++e) sel[h][e] = (hit && e == ((c & 7) >> 1)) ? one : 0u;
    }
  }
  float slope = 0.f;
  if constexpr (BIAS) slope = c < G ? a.slopes[kh * G + c] * kLog2e : 0.f;
  const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
  f32x4_t oacc[NOB];
#pragma unroll
  for (int ob = 0; ob < NOB; ++ob) oacc[ob] = zero;
  float mrun = kNoScore, lsum = 0.f;
  f32x4_t s_page = zero;  // the scores of the page worked on last
  uint32_t goff[Tr::NDMA];
#pragma unroll
  for (int i = 0; i < Tr::NDMA; ++i) {
    const int e = i * 1024 + lane * 16;  // byte of the slot block this lane fills
    const int t = e / Tr::ROW, u = (e % Tr::ROW) >> 4;
    goff[i] = (uint32_t)(t * Tr::ROW + ((u ^ mdec_swz<HD, F8>(t)) << 4));
  }
  const int sw = mdec_swz<HD, F8>(c);
  // dims 8 g + 32 ks .. + 7 of token c of a block
  auto dims8 = [&](const uint8_t *blk, int ks) -> u32x4_t {
    const uint8_t *rowp = blk + c * Tr::ROW;
    if constexpr (F8)
      return e4m3x8_to_bf16x8(
          *reinterpret_cast<const u32x2_t *>(rowp + ((((g >> 1) + 2 * ks) ^ sw) << 4) + ((g & 1) << 3)));
    else
      return *reinterpret_cast<const u32x4_t *>(rowp + (((g + 4 * ks) ^ sw) << 4));
  };
  // The transposing read: lane 16 g + 4 e + q points at token 4 g + e, dims
  // 16 ob + 4 q .. + 3, and lane 16 g + i receives dim 16 ob + i of tokens
  // 4 g .. 4 g + 3.
  typedef short v4s_t __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) v4s_t lds_v4s_t;
  const int tt = 4 * g + (c >> 2), tq = c & 3, tsw = mdec_swz<HD, F8>(tt);
  auto vt_read = [&](const uint8_t *blk, int ob) -> u32x2_t {
    const uint8_t *p = blk + tt * Tr::ROW + (((2 * ob + (tq >> 1)) ^ tsw) << 4) + ((tq & 1) << 3);
    return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_t *)p));
  };

  // Online-softmax update with page p in a slot.  The page holds a visible
  // key: it starts below k1 and ends past lo.
  auto update = [&](const uint8_t *slot, int p) {
    const int kp = p * kPageSize;
    f32x4_t sa = zero;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) sa = mfma16x16x32(dims8(slot, ks), qb[ks], sa);
    float s[4];
    if constexpr (CAP) {
      const float big = fmaxf(fmaxf(fabsf(sa[0]), fabsf(sa[1])), fmaxf(fabsf(sa[2]), fabsf(sa[3])));
      if (none(big > a.small_raw)) {
        asm volatile("");  // (a branch: not both forms and a select)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] = small_score(sa[j], a);
      } else {
        asm volatile("");
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] = capped_score(sa[j], a);
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (!CAP) s[j] = sa[j] * a.qscale;
      if constexpr (BIAS) s[j] = fmaf(-slope, (float)(r.ctx - (kp + 4 * g + j)), s[j]);
    }
    const bool edge = kp + kPageSize > k1 || kp < lo;  // uniform
    if (edge) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (kp + 4 * g + j >= k1 || kp + 4 * g + j < lo) s[j] = kNoScore;
    }
    s_page = f32x4_t{s[0], s[1], s[2], s[3]};
    float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
    mx = fmaxf(mx, shfl_xor_f32(mx, 16));
    mx = fmaxf(mx, shfl_xor_f32(mx, 32));
    const float mnew = fmaxf(mrun, mx);
    // (scores of -inf alone, which an infinite key or query can give, keep an offset of 0)
    const float off = mnew == kNoScore ? 0.f : mnew;
    const float alpha = mrun == kNoScore ? 0.f : fast_exp2(mrun - off);
    float pr[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) pr[j] = fast_exp2(s[j] - off);
    lsum = lsum * alpha + ((pr[0] + pr[1]) + (pr[2] + pr[3]));
    mrun = mnew;
    // P^T as the B operand of the 16x16x16 product, rounded to bf16 (half a
    // step, 2^-8 of a probability): it takes bf16 alone, and P in two terms would
    // be two products.  The sum above keeps the fp32 values
    const u32x2_t pt = {pack_bf16x2(pr[0], pr[1]), pack_bf16x2(pr[2], pr[3])};
    u32x2_t keep = {0xFFFFFFFFu, 0xFFFFFFFFu};  // values of masked tokens do not enter (0 x NaN)
    if (edge) {
      const int f = lo - kp - 4 * g;  // tokens below f of this lane's four are masked (those past k1 land as zeros)
      keep[0] = (f <= 0 ? 0xFFFFu : 0u) | (f <= 1 ? 0xFFFF0000u : 0u);
      keep[1] = (f <= 2 ? 0xFFFFu : 0u) | (f <= 3 ? 0xFFFF0000u : 0u);
    }
    if constexpr (F8) {
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) {
        const u32x4_t vv = dims8(slot + Tr::BLK, ks);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const f32x4_t t = mfma16x16x32(vv, sel[h], zero);  // V[4 g + j][32 ks + 16 h + c]
          const u32x2_t av = {bf16_pair_exact(t[0], t[1]) & keep[0], bf16_pair_exact(t[2], t[3]) & keep[1]};
          oacc[2 * ks + h] = mfma16x16x16(av, pt, oacc[2 * ks + h] * alpha);
        }
      }
    } else {
#pragma unroll
      for (int ob = 0; ob < NOB; ++ob) {
        const u32x2_t v = vt_read(slot + Tr::BLK, ob);
        oacc[ob] = mfma16x16x16(u32x2_t{v[0] & keep[0], v[1] & keep[1]}, pt, oacc[ob] * alpha);
      }
    }
  };
  // pages pg0 + wave, + 4, ..; lane l of vbt holds the physical page of page
  // pg0 + l (a split has at most 64)
  const int npg = pg1 - pg0;
  const int vbt = lane < npg ? bt[pg0 + lane] : -1;
  const uint32_t page_bytes = (uint32_t)(a.nkv * Tr::BLK);
  const uint8_t *const kbase = reinterpret_cast<const uint8_t *>(a.kv.k) + (size_t)kh * Tr::BLK;
  const uint8_t *const vbase = reinterpret_cast<const uint8_t *>(a.kv.v) + (size_t)kh * Tr::BLK;
  // (its slot's last reads have been waited for: their products are issued)
  auto dma = [&](uint32_t slot, int i) {
    const int phys = i < npg ? __builtin_amdgcn_readlane(vbt, i) : -1;
    const int bytes = (unsigned)phys < (unsigned)a.kv.num_pages
                          ? min(max(k1 - (pg0 + i) * kPageSize, 0), kPageSize) * Tr::ROW
                          : 0;  // nothing, zeros in LDS
    const uint64_t at = (uint64_t)(uint32_t)phys * page_bytes;
    const u32x4_t rk = range_words<true>(kbase + at, bytes), rv = range_words<true>(vbase + at, bytes);
#pragma unroll
    for (int n = 0; n < Tr::NDMA; ++n) {
      lds_fill16<true>(rk, slot + n * 1024, goff[n]);
      lds_fill16<true>(rv, slot + Tr::BLK + n * 1024, goff[n]);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  const uint8_t *const w0 = lds + 2 * wave * Tr::SLOT, *const w1 = w0 + Tr::SLOT;
  const uint32_t f0 = lds_at(w0), f1 = f0 + Tr::SLOT;
  constexpr int PAGE_LOADS = 2 * Tr::NDMA;
  // The scores of the request: runs of 16, page by page the G heads' (a
  // wavefront stores whole lines).  They wait in LDS for the end of the split:
  // loads and stores count down together in the order they were issued, and
  // waiting for a page's loads behind a store took longer (64 rows over 2350
  // keys, the whole call: 140 us, 138 so; 8 bits 84 and 82; what is left, 11
  // us, is the writing of 19 MB itself).  Where the LDS is short they are stored
  // behind the loads of the next page for their slot, so that the wait for the
  // other slot leaves them (and the store before them) outstanding.
  const bool stores = a.scores && !a.stash;
  float *split_scores = nullptr;
  if (a.scores) {
    const size_t npv = (size_t)((r.nkeys - r.first + kPageSize - 1) / kPageSize);
    split_scores = a.scores + ((size_t)m[DEC_SCORE0 * a.n + r.d] + (size_t)kh * G * npv) * kPageSize +
                   (size_t)(pg0 * kPageSize - r.first) * G;
  }
  auto keep_scores = [&](int p) {
    if (!a.scores || c >= G) return;
    const int to = ((p - pg0) * G + c) * kPageSize + 4 * g;
    if (a.stash)
      *reinterpret_cast<f32x4_t *>(stash + to) = s_page;
    else
      *reinterpret_cast<f32x4_t *>(split_scores + to) = s_page;
  };
  dma(f0, wave);
  dma(f1, wave + kWaves);
  for (int i = wave; i < npg; i += 2 * kWaves) {
    if (stores && i > wave)
      wait_loads<PAGE_LOADS + 2>();  // w0's loads are older than a store, w1's loads and a store
    else
      wait_loads<PAGE_LOADS>();
    update(w0, pg0 + i);
    __builtin_amdgcn_sched_barrier(0);
    dma(f0, i + 2 * kWaves);
    keep_scores(pg0 + i);
    __builtin_amdgcn_sched_barrier(0);
    if (i + kWaves < npg) {
      if (stores && i > wave)
        wait_loads<PAGE_LOADS + 2>();
      else
        wait_loads<PAGE_LOADS>();
      update(w1, pg0 + i + kWaves);
      __builtin_amdgcn_sched_barrier(0);
      dma(f1, i + 3 * kWaves);
      keep_scores(pg0 + i + kWaves);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  wait_loads<0>();
  lsum += shfl_xor_f32(lsum, 16);
  lsum += shfl_xor_f32(lsum, 32);
  // across the waves through LDS, reusing the slots: [wave][h][HD], then [wave][h][2]
  __syncthreads();
  if (a.stash)
    for (int e = 4 * threadIdx.x; e < npg * G * kPageSize; e += 4 * 256)
      *reinterpret_cast<f32x4_t *>(split_scores + e) = *reinterpret_cast<const f32x4_t *>(stash + e);
  float *const mo = reinterpret_cast<float *>(lds) + wave * MAXG * HD;
  float *const ml = reinterpret_cast<float *>(lds) + kWaves * MAXG * HD;
  if (c < G) {
#pragma unroll
    for (int ob = 0; ob < NOB; ++ob) *reinterpret_cast<f32x4_t *>(mo + c * HD + ob * 16 + g * 4) = oacc[ob];
    if (g == 0) {
      ml[(wave * MAXG + c) * 2] = mrun;
      ml[(wave * MAXG + c) * 2 + 1] = lsum;
    }
  }
  __syncthreads();
  const float vscale = F8 ? a.kv.vs : 1.f;
  const bool empty = lo >= r.nkeys;
  for (int e = threadIdx.x; e < G * HD; e += 256) {
    const int h = e / HD, dim = e - h * HD;
    float mx = kNoScore;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) mx = fmaxf(mx, ml[(w * MAXG + h) * 2]);
    float L = 0.f, O = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float mw = ml[(w * MAXG + h) * 2];
      const float f = mw == kNoScore ? 0.f : fast_exp2(mw - mx);
      const float *src = reinterpret_cast<const float *>(lds) + w * MAXG * HD;
      L += f * ml[(w * MAXG + h) * 2 + 1];
      O += f * src[h * HD + dim];
    }
    O *= vscale;
    const int qh = kh * G + h;
    if (nsplit == 1) {
      a.out[((size_t)r.row * a.nq + qh) * HD + dim] = (uint16_t)f32_to_bf16_bits(empty ? 0.f : O / L);
      if (dim == 0 && a.lse) a.lse[(size_t)r.row * a.nq + qh] = empty ? kNoScore : kLn2 * (mx + log2f(L));
    } else {
      const size_t slot = (size_t)split * a.nq + qh;
      a.part_o[slot * HD + dim] = O;
      if (dim == 0) {
        a.part_ml[slot * 2] = mx;
        a.part_ml[slot * 2 + 1] = L;
      }
    }
  }
}

// weights[t] += sum over the G heads of 2^(s - lse): one block per 1024 keys of
// a (request, kv head), four keys per thread.  Reads 4 G bytes per key.
__global__ __launch_bounds__(256) void k_attend_decode_weights(AttendArgs a) {
  const meta_t m = meta_words(a);
  const int unit = blockIdx.x;
  const int blk = unit / a.nkv, kh = unit - blk * a.nkv;
  const DecRow r = dec_row(a, m, last_at_or_below(m + DEC_WBLOCK0 * a.n, a.n, blk));
  const int base = (blk - m[DEC_WBLOCK0 * a.n + r.d]) * kWeightSpan + threadIdx.x * 4;  // from the first key
  if (r.first + base >= r.nkeys) return;
  const int key = r.first + base;
  const int lo = min(row_first(a, r.row, r.ctx), r.nkeys);
  const int page = a.kv.bt[(size_t)r.seq * a.kv.max_pages + key / kPageSize];
  if ((unsigned)page >= (unsigned)a.kv.num_pages) return;
  float *dst = a.weights + ((size_t)page * a.nkv + kh) * kPageSize + key % kPageSize;
  f32x4_t w = *reinterpret_cast<const f32x4_t *>(dst);
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (key + e == r.ctx) w[e] = 0.f;  // the new key's first value
  // (pages before the first visible key hold no scores)
  if (key / kPageSize >= lo / kPageSize && lo < r.nkeys) {
    const size_t npv = (size_t)((r.nkeys - r.first + kPageSize - 1) / kPageSize);
    const float *s = a.scores +
                     ((size_t)m[DEC_SCORE0 * a.n + r.d] + (size_t)a.group * (kh * npv + base / kPageSize)) * kPageSize +
                     base % kPageSize;
    const float *lse = a.lse + (size_t)r.row * a.nq + kh * a.group;
    for (int h = 0; h < a.group; ++h) {
      const f32x4_t v = *reinterpret_cast<const f32x4_t *>(s + h * kPageSize);
      const float z = lse[h] * kLog2e;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (key + e >= lo && key + e < r.nkeys) w[e] += fast_exp2(v[e] - z);
    }
  }
  // slots past the request's last key are not its own to write
  if (key + 3 < r.nkeys) {
    *reinterpret_cast<f32x4_t *>(dst) = w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (key + e < r.nkeys) dst[e] = w[e];
  }
}

// Joins the splits of the decode rows that have several, one wavefront per
// query head.
template <int HD>
__global__ __launch_bounds__(256) void k_attend_decode_combine(AttendArgs a) {
  const meta_t m = meta_words(a);
  const int qh = blockIdx.y * 4 + (threadIdx.x >> 6);
  if (qh >= a.nq) return;
  const DecRow r = dec_row(a, m, blockIdx.x);
  const int per = attend_split_keys(r.nkeys - r.first);
  const int ns = (r.nkeys - r.first + per - 1) / per;
  if (ns < 2) return;
  const bool empty = row_first(a, r.row, r.ctx) >= r.nkeys;
  const size_t base = (size_t)m[DEC_SPLIT0 * a.n + r.d] * a.nq + qh;
  join_splits<HD>(a, base, ns, (size_t)r.row * a.nq + qh, empty, threadIdx.x & 63);
}

}  // namespace

hipError_t launch_attend_decode(const Shape &s, const AttendCall &c, const AttendArgs &a, hipStream_t st) {
  const AttendPlan &p = *c.plan;
  const dim3 grid(p.dec_splits * s.nkv);
#define EB_DEC(HD_, F8_)                                                                                       \
  do {                                                                                                         \
    if (c.softcap > 0.f && c.slopes)                                                                           \
      hipLaunchKernelGGL((k_attend_decode<HD_, F8_, true, true>), grid, dim3(256), a.stash, st, a);            \
    else if (c.softcap > 0.f)                                                                                  \
      hipLaunchKernelGGL((k_attend_decode<HD_, F8_, true, false>), grid, dim3(256), a.stash, st, a);           \
    else if (c.slopes)                                                                                         \
      hipLaunchKernelGGL((k_attend_decode<HD_, F8_, false, true>), grid, dim3(256), a.stash, st, a);           \
    else                                                                                                       \
      hipLaunchKernelGGL((k_attend_decode<HD_, F8_, false, false>), grid, dim3(256), a.stash, st, a);          \
  } while (0)
  if (s.hd == 128) {
    if (a.kv.f8)
      EB_DEC(128, true);
    else
      EB_DEC(128, false);
  } else {
    if (a.kv.f8)
      EB_DEC(64, true);
    else
      EB_DEC(64, false);
  }
#undef EB_DEC
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (p.dec_combine) {
    const dim3 cg(p.n_dec, (s.nq + 3) / 4);
    if (s.hd == 128)
      hipLaunchKernelGGL(k_attend_decode_combine<128>, cg, dim3(256), 0, st, a);
    else
      hipLaunchKernelGGL(k_attend_decode_combine<64>, cg, dim3(256), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (c.weights) {
    hipLaunchKernelGGL(k_attend_decode_weights, dim3(p.dec_wblocks * s.nkv), dim3(256), 0, st, a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace eb
