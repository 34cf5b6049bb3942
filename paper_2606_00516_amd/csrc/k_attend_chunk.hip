// Rows of requests with several new rows (prompt chunks, drafted tokens) in
// the modified attention.
//
// A block takes 128 query rows (128 / G positions of the G heads of one kv
// head) of one request and a range of its keys, in tiles of 64.  Four
// wavefronts hold 32 rows each: S^T = K Q^T and O^T += V^T P^T on 32x32x16
// products, so a row's scores lie in one lane pair, its softmax needs one
// exchange, and P goes from the score registers straight into the second
// product.  Two LDS buffers of a K and a V tile (row-major, swizzled) are
// filled by direct loads, K two tiles and V one tile ahead, so the scores of
// tile t + 1 run on the matrix cores under the exponentials of tile t; 8-bit
// tiles pass through registers to become bf16.  Per tile and wavefront (head
// size 128) 32 products of 32 cycles, 1024 cycles, stand against 32 scores per
// lane: some 45 cycles of vector work each, 1440, where the cap's polynomial
// serves: the vector unit bounds capped attention.  4096 rows over 32768 keys,
// 32 heads: 2.58 to 2.9 ms by the box, 905 to 805 TFLOP/s; the counters put the
// matrix cores at 41 % and the vector unit at 66 %, in part one after the other.
//
// With few rows the keys are split over blocks (the plan's rule) and joined by
// k_attend_chunk_combine.
#include "attend_device.h"

#include <type_traits>

namespace eb {

namespace {

constexpr int kWaves = 4;
// The running maximum moves only when a tile exceeds it by more than this
// (log2 units): probabilities stay below 2^8, exact alike in fp32 and bf16,
// and most tiles skip the rescaling of the outputs.
constexpr float kSlack = 8.0f;

struct PreReq {
  int k, seq, row0, c, n, prefix, nsplit;
};
__device__ __forceinline__ PreReq pre_req(const AttendArgs &a, meta_t m, int k) {
  PreReq r;
  r.k = k;
  // (uniform; said so, so that what follows from them stays in scalar registers)
  r.seq = __builtin_amdgcn_readfirstlane(m[PRE_SEQ * a.n + k]);
  r.row0 = __builtin_amdgcn_readfirstlane(m[PRE_ROW * a.n + k]);
  r.c = __builtin_amdgcn_readfirstlane(m[PRE_CTX * a.n + k]);
  r.n = __builtin_amdgcn_readfirstlane(m[PRE_LEN * a.n + k]);
  r.prefix = __builtin_amdgcn_readfirstlane(m[PRE_PREFIX * a.n + k]);
  r.nsplit = __builtin_amdgcn_readfirstlane(m[PRE_NSPLIT * a.n + k]);
  return r;
}

// How scores are made.  kCapped (a cap, no bias) keeps no running maximum: a
// row's probabilities are 2^(s - offset) with an offset of 0 as long as no
// score of its block's tiles leaves +-kCappedSlack, which the largest of a
// tile's products says (the cap's polynomial asks for it anyway).  Where one
// does, the offset becomes the row's maximum if that is kCappedSlack above it,
// or below -kCappedSlack at the row's first keys: probabilities stay below
// 2^kCappedSlack and a row's largest above 2^-kCappedSlack, whatever the cap.
enum Mode { kPlain = 0, kCapped, kBiased, kCapBiased };

template <int HD, bool F8, int MODE>
__global__ __launch_bounds__(256, 2) void k_attend_chunk(AttendArgs a) {
  constexpr bool CAP = MODE == kCapped || MODE == kCapBiased, BIAS = MODE == kBiased || MODE == kCapBiased;
  constexpr bool FIXED = MODE == kCapped;
  constexpr int KT = kAttendTile;
  constexpr int ROW = HD * 2;        // bytes per key row in LDS
  constexpr int CPR = ROW / 16;      // 16-byte chunks per row
  constexpr int TILE = KT * ROW;     // bytes of the K (and of the V) tile
  constexpr int NKS = HD / 16;       // k-steps of the score product
  constexpr int NOB = HD / 32;       // 32-dim output blocks
  __shared__ __attribute__((aligned(16))) uint8_t lds[4 * TILE];
  __shared__ int red[2], odd[2];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lq = lane & 31, lh = lane >> 5;
  const meta_t m = meta_words(a);
  const int tile_id = blockIdx.x / a.nkv, kh = blockIdx.x - tile_id * a.nkv;
  const PreReq r = pre_req(a, m, last_at_or_below(m + PRE_TILE0 * a.n, a.n, tile_id));
  const int G = a.group, BQ = kAttendRows / G;
  const int nqb = (r.n + BQ - 1) / BQ;
  const int local = __builtin_amdgcn_readfirstlane(tile_id - m[PRE_TILE0 * a.n + r.k]);
  // the last rows, which see the most keys, first
  const int qb = nqb - 1 - local / r.nsplit, sp = local % r.nsplit;
  const int q_lo = qb * BQ, q_hi = min(r.n, q_lo + BQ);
  const int klen = r.c + r.n;
  const int cols = (a.nq + 2 * a.nkv) * HD;

  // this lane's row: 32 rows of a wave are RPH positions of 32 / RPH heads
  const int RPH = min(BQ, 32), HG = G * RPH / 32;
  const int hb = wave % HG, sub = wave / HG;
  const int hrow = hb * (32 / RPH) + lq / RPH;
  const int qrel = q_lo + sub * RPH + lq % RPH;
  const bool qok = qrel < q_hi;
  const int qpos = r.c + qrel;
  u32x4_t qreg[NKS];
  {
    const uint16_t *src = a.qkv + (size_t)(r.row0 + (qok ? qrel : 0)) * cols + (kh * G + hrow) * HD + lh * 8;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {
      const u32x4_t v = ld_u32x4(src + ks * 16);
      qreg[ks] = qok ? v : u32x4_t{0u, 0u, 0u, 0u};
    }
  }
  // keys [rlo, rhi) visible to the row; the block's smallest and largest bounds
  const int rlo = qok ? min(row_first(a, r.row0 + qrel, qpos), klen) : 0;
  const int rhi = qok ? max(qpos + 1, r.prefix) : 0;
  int lo_min = attend_first(r.c + q_lo, a.window), lo_max = a.window > 0 ? max(r.c + q_hi - a.window, 0) : 0;
  if (a.first_key) {
    // every wavefront of a row block sees other positions: through LDS
    int mn = qok ? rlo : 0x7fffffff, mx = qok ? rlo : 0;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
      mn = min(mn, __shfl_xor(mn, o, 64));
      mx = max(mx, __shfl_xor(mx, o, 64));
    }
    if (tid < 2) red[tid] = tid ? 0 : 0x7fffffff;
    __syncthreads();
    if (lane == 0) {
      atomicMin(&red[0], mn);
      atomicMax(&red[1], mx);
    }
    __syncthreads();
    lo_min = __builtin_amdgcn_readfirstlane(red[0]);
    lo_max = __builtin_amdgcn_readfirstlane(red[1]);
  }
  const int hi_min = max(r.c + q_lo + 1, r.prefix), hi_max = max(r.c + q_hi, r.prefix);
  // this split's tiles: an even share of those that the window leaves, cut to
  // those that hold a visible key
  const int all0 = attend_first(r.c + q_lo, a.window) / KT, all1 = (hi_max + KT - 1) / KT;
  const int share = (all1 - all0 + r.nsplit - 1) / r.nsplit;
  const int t0 = max(all0 + sp * share, lo_min / KT), t1 = min(all0 + (sp + 1) * share, all1);

  f32x16_t oacc[NOB];
#pragma unroll
  for (int ob = 0; ob < NOB; ++ob)
#pragma unroll
    for (int i = 0; i < 16; ++i) oacc[ob][i] = 0.f;
  float mrun = FIXED ? 0.f : kNoScore, lrun = 0.f;
  float lbf = 0.f;  // FIXED: the sum of the probabilities as their product takes them
  float slope = 0.f;
  if constexpr (BIAS) slope = a.slopes ? a.slopes[kh * G + hrow] * kLog2e : 0.f;

  const int32_t *bt = a.kv.bt + (size_t)r.seq * a.kv.max_pages;
  const int npages = (klen + kPageSize - 1) / kPageSize;
  constexpr int PPT = KT / kPageSize;
  static_assert(PPT == 4, "tile = 4 pages");
  typedef const __attribute__((address_space(4))) int32_t *bt_ptr_t;
  const bt_ptr_t btc = (bt_ptr_t)bt;
  constexpr int ES = F8 ? 1 : 2;
  constexpr int KPI = 1024 / (HD * ES), NI = KT / (KPI * kWaves);  // keys of one load instruction of a wave; instructions of a tile
  const uint32_t page_bytes = (uint32_t)(a.nkv * kPageSize * HD * ES);
  const size_t head_at = (size_t)kh * (kPageSize * HD * ES);
  const uint8_t *const kbase = reinterpret_cast<const uint8_t *>(a.kv.k) + head_at;
  const uint8_t *const vbase = reinterpret_cast<const uint8_t *>(a.kv.v) + head_at;
  // The page of each of this wave's instructions: its id, then where it starts
  // and how many bytes of it lie below klen (none for an id outside the pool).
  // Loads past the range give zeros, without traffic.  K and V of a tile are
  // found alike, V one tile later: worked out once, for both.
  struct Ids {
    int id[NI];
  };
  struct Ranges {
    uint64_t at[NI];
    int bytes[NI];
  };
  auto page_of = [&](int i) { return (KPI * kWaves * i) / kPageSize + wave * KPI / kPageSize; };
  auto page_ids = [&](int t) {  // pages past the sequence repeat its last id (their ranges are empty)
    Ids v;
#pragma unroll
    for (int i = 0; i < NI; ++i) v.id[i] = btc[min(t * PPT + page_of(i), npages - 1)];
    return v;
  };
  auto ranges = [&](int t, const Ids &v) {
    Ranges g;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int keys = min(max(klen - (t * PPT + page_of(i)) * kPageSize, 0), kPageSize);
      g.bytes[i] =
          __builtin_amdgcn_readfirstlane((unsigned)v.id[i] < (unsigned)a.kv.num_pages ? keys * (HD * ES) : 0);
      g.at[i] = (uint64_t)(uint32_t)v.id[i] * page_bytes;
    }
    return g;
  };
  // --- bf16: load instruction i of wave w fills keys KPI (i 4 + w) .. + KPI - 1
  // of a tile; lane l writes chunk position l % CPR of key .. + l / CPR.
  // K chunk c of key t lies at c ^ (t & 7), V chunk c at c ^ 2 (t & 3).
  uint32_t koff[NI], voff[NI];
  if constexpr (!F8) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int key = KPI * (i * kWaves + wave) + lane / CPR, pos = lane % CPR;
      koff[i] = (uint32_t)((key % kPageSize) * ROW + 16 * (pos ^ (key & 7)));
      voff[i] = (uint32_t)((key % kPageSize) * ROW + 16 * (pos ^ (2 * (key & 3))));
    }
  }
  const uint32_t lds0 = lds_at(lds);
  auto dma = [&](const Ranges &g, int at, bool is_v) {
#pragma unroll
    for (int i = 0; i < NI; ++i)
      lds_fill16(range_words((is_v ? vbase : kbase) + g.at[i], g.bytes[i]),
                 lds0 + at + KPI * (i * kWaves + wave) * ROW, is_v ? voff[i] : koff[i]);
  };
  // --- 8 bits: unit u = tid + 256 i is 16 codes of key u / (HD / 16); they become two chunks
  constexpr int CU = HD / 16;
  u32x4_t kreg[F8 ? NI : 1], vreg[F8 ? NI : 1];
  auto fetch = [&](const Ranges &g, u32x4_t (&reg)[F8 ? NI : 1], bool is_v) {
#pragma unroll
    for (int i = 0; i < (F8 ? NI : 0); ++i)
      reg[i] = buf_ld_u32x4<0>(make_rsrc((is_v ? vbase : kbase) + g.at[i], g.bytes[i]),
                               ((tid + 256 * i) / CU % kPageSize) * HD + (tid % CU) * 16);
  };
  auto land = [&](const u32x4_t (&reg)[F8 ? NI : 1], uint8_t *dst, bool is_v) {
#pragma unroll
    for (int i = 0; i < (F8 ? NI : 0); ++i) {
      const int key = (tid + 256 * i) / CU, ch = 2 * (tid % CU);
      const int x = is_v ? 2 * (key & 3) : key & 7;
      st_u32x4(dst + key * ROW + 16 * (ch ^ x), e4m3x8_to_bf16x8(u32x2_t{reg[i][0], reg[i][1]}));
      st_u32x4(dst + key * ROW + 16 * ((ch + 1) ^ x), e4m3x8_to_bf16x8(u32x2_t{reg[i][2], reg[i][3]}));
    }
  };

  // K operand of the scores: key kb 32 + lq, chunk 2 ks + lh
  int kaddr[4];
#pragma unroll
  for (int k4 = 0; k4 < 4; ++k4) kaddr[k4] = lq * ROW + 16 * ((2 * k4 + lh) ^ (lq & 7));
  // V^T operand, the transposing read: lane 16 g + 4 e + q points at key
  // kb 32 + 16 jj + 8 h + 4 (g / 2) + e, dims ob 32 + 16 (g & 1) + 4 q .. + 3
  const int tg = lane >> 4, te = (lane >> 2) & 3, tq = lane & 3;
  int vaddr[2];
#pragma unroll
  for (int b = 0; b < 2; ++b)
    vaddr[b] = (4 * (tg >> 1) + te) * ROW + 16 * ((4 * b + 2 * (tg & 1) + (tq >> 1)) ^ (2 * te)) + 8 * (tq & 1);
  typedef short v4s_t __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) v4s_t lds_v4s_t;
  auto vt_read = [&](const uint8_t *vt, int ob, int kb, int jj, int h) -> u32x2_t {
    const uint8_t *p = vt + vaddr[ob & 1] + (kb * 32 + 16 * jj + 8 * h) * ROW + 128 * (ob >> 1);
    return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_t *)p));
  };
  // S^T of the K tile at kt: lane value i of block kb at key 32 kb + 8 (i / 4) + 4 lh + i % 4
  auto scores = [&](const uint8_t *kt, f32x16_t (&s)[2]) {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[kb][i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const u32x4_t v = *reinterpret_cast<const u32x4_t *>(kt + kaddr[ks & 3] + 128 * (ks >> 2) + kb * 32 * ROW);
        s[kb] = mfma32x32x16(v, qreg[ks], s[kb]);
      }
  };
  // Values of a tile that some row does not see: a value that is not finite
  // would reach those rows too, as 0 x inf.  Such values are set to zero in
  // LDS, and the rows that do see them take them from the cache one by one.
  // True if any was found; which of the two flags it uses follows the tile.
  auto clean = [&](uint8_t *vt, int which) -> bool {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < TILE / 16 / 256; ++i) {
      u32x4_t *p = reinterpret_cast<u32x4_t *>(vt + (i * 256 + tid) * 16);
      u32x4_t v = *p;
      bool here = false;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool b0 = (v[e] & 0x7F80u) == 0x7F80u, b1 = (v[e] & 0x7F800000u) == 0x7F800000u;
        here |= b0 | b1;
        v[e] &= (b0 ? 0xFFFF0000u : 0xFFFFFFFFu) & (b1 ? 0xFFFFu : 0xFFFFFFFFu);
      }
      if (here) *p = v;
      bad |= here;
    }
    if (bad) odd[which] = 1;
    if (tid == 0) odd[which ^ 1] = 0;  // read last before the barrier that ended the tile before
    __syncthreads();
    return odd[which] != 0;
  };

  if (t0 < t1) {
    if (tid < 2) odd[tid] = 0;
    f32x16_t sc[2];
    // Looks over the products of tile t: whether all are small beside the cap,
    // and whether they move the offset.
    auto look = [&](int t, bool masked) {
      const float big = largest<2>(sc);
      bool small = none(big > (!FIXED ? a.small_raw : mrun < 0.f ? -1.f : a.even_raw));
      if (FIXED && __builtin_expect(!small, 0)) {
        small = none(big > a.small_raw);
        // the row's largest score (the cap keeps their order) over its two lanes, and whether it had a key before
        const int d = t * KT + 4 * lh - rlo;
        const unsigned span = (unsigned)max(rhi - rlo, 0);
        float top = kNoScore;
        if (masked) {
          asm volatile("");
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i)
              top = fmaxf(top, (unsigned)(d + kb * 32 + 8 * (i >> 2) + (i & 3)) < span ? sc[kb][i] : kNoScore);
        } else {
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[kb][i]);
        }
        const auto tw = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        const auto lw = __builtin_amdgcn_permlane32_swap(__float_as_uint(lrun), __float_as_uint(lrun), false, false);
        top = fmaxf(__uint_as_float(tw[0]), __uint_as_float(tw[1]));
        const bool seen = top != kNoScore, first = lw[0] == 0u && lw[1] == 0u;
        top = capped_score(top, a);
        const bool move = seen && (top > mrun + kCappedSlack || (first && top < -kCappedSlack));
        if (!none(move)) {
          const float f = !move ? 1.f : first ? 0.f : fast_exp2(mrun - top);
          lrun *= f;
          lbf *= f;
#pragma unroll
          for (int ob = 0; ob < NOB; ++ob) oacc[ob] = oacc[ob] * f;
          mrun = move ? top : mrun;
        }
      }
      return small;
    };
    const Ids i0 = page_ids(t0), i1 = page_ids(t0 + 1);
    Ids next = page_ids(t0 + 2);
    Ranges vat = ranges(t0 + 1, i1);
    {
      const Ranges g0 = ranges(t0, i0);
      if constexpr (F8) {
        u32x4_t k1[NI];
        fetch(g0, kreg, false);
        fetch(g0, vreg, true);
        fetch(vat, k1, false);
        land(kreg, lds, false);
        land(vreg, lds + TILE, true);
        land(k1, lds + 2 * TILE, false);
      } else {
        dma(g0, 0, false);
        dma(g0, TILE, true);
        if (t0 + 1 < t1) dma(vat, 2 * TILE, false);
      }
    }
    wait_loads<0>();
    __syncthreads();
    scores(lds, sc);
    __syncthreads();  // every wave past the scores of the first tile before K of the third refills its buffer
    auto step = [&](int t, auto lastconst) {
      constexpr bool LAST = decltype(lastconst)::value;
      const int at = ((t - t0) & 1) * (2 * TILE);
      uint8_t *const cur = lds + at, *const nxt = lds + (2 * TILE - at);
      const int k0 = t * KT;
      f32x16_t scn[2];
      // (before the next loads are issued: its barrier would wait for them)
      const bool masked = k0 < lo_max || k0 + KT > hi_min;  // uniform over the block
      const bool odd_values = masked && clean(cur + TILE, t & 1);
      if constexpr (!LAST) {
        // K of tile t and V of tile t - 1 were read before the last barrier
        const Ranges kat = ranges(t + 2, next);
        if constexpr (F8) {
          fetch(kat, kreg, false);
          fetch(vat, vreg, true);
        } else {
          if (t + 2 < t1) dma(kat, at, false);
          dma(vat, 2 * TILE - at + TILE, true);
        }
        vat = kat;
        next = page_ids(t + 3);
      }
      auto hide = [&]() {  // keys outside the row's range
        asm volatile("");  // (a branch, not 32 selects in every tile)
        const int d = k0 + 4 * lh - rlo;
        const unsigned span = (unsigned)max(rhi - rlo, 0);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            sc[kb][i] = (unsigned)(d + kb * 32 + 8 * (i >> 2) + (i & 3)) < span ? sc[kb][i] : kNoScore;
      };
      // plain scores are hidden before the next tile's are formed, so that
      // nothing splits the run of products and exponentials below
      if (MODE == kPlain && masked) hide();
      // Vector work goes before the other wavefront's products, which keep the
      // matrix cores busy from few issued instructions (capped, as above: 2.73
      // ms; without: 2.93).
      __builtin_amdgcn_s_setprio(0);
      if constexpr (!LAST) scores(nxt, scn);
      __builtin_amdgcn_s_setprio(2);
      if constexpr (CAP) {
        if (look(t, masked)) {
          asm volatile("");  // (a branch: not both forms and a select)
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[kb][i] = FIXED ? small_score(sc[kb][i], a, -mrun) : small_score(sc[kb][i], a);
        } else {
          asm volatile("");
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[kb][i] = capped_score(sc[kb][i], a, FIXED ? -mrun : 0.f);
        }
      }
      if constexpr (BIAS) {
        const float d0 = (float)(qpos - k0 - 4 * lh);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float s = CAP ? sc[kb][i] : sc[kb][i] * a.qscale;
            sc[kb][i] = fmaf(-slope, fabsf(d0 - (float)(kb * 32 + 8 * (i >> 2) + (i & 3))), s);
          }
      }
      if (MODE != kPlain && masked) hide();
      constexpr bool RAW = MODE == kPlain;  // scores still to be scaled (qscale > 0 keeps their order)
      float mx = 0.f, alpha = 1.f, neg = 0.f;
      bool bump = false;
      if constexpr (!FIXED) {
        float mraw = kNoScore;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) mraw = fmaxf(mraw, sc[kb][i]);
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mraw), __float_as_uint(mraw), false, false);
        mraw = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
        const float ms = RAW ? mraw * a.qscale : mraw;
        bump = ms > mrun + kSlack;
        mx = bump ? ms : mrun;
        alpha = bump ? fast_exp2(mrun - mx) : 1.0f;
        neg = mx != kNoScore ? -mx : 0.f;
      }
      float l = lrun * alpha;
      uint32_t pk[2][8];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int pr = 0; pr < 8; ++pr) {
          const float s0 = sc[kb][2 * pr], s1 = sc[kb][2 * pr + 1];
          const float p0 = fast_exp2(RAW ? fmaf(s0, a.qscale, neg) : FIXED ? s0 : s0 + neg);
          const float p1 = fast_exp2(RAW ? fmaf(s1, a.qscale, neg) : FIXED ? s1 : s1 + neg);
          // P enters its product rounded to bf16 (half a step, 2^-8 of a
          // probability): the product takes bf16 alone, and P in two terms would
          // be two products.  The sum keeps the fp32 values
          pk[kb][pr] = pack_bf16x2(p0, p1);
          l += p0 + p1;
          // Outputs are divided by the sum of what was multiplied.  Elsewhere a
          // row's largest probability is near 1 of itself (its first maximum
          // is exactly 1); here it is any number, whose rounding would stay in
          // the output: a row that sees one key would miss its value.  (Errors
          // of rows with few keys that count 2.2e-3 -> 1.7e-3, the output's own
          // rounding; costs 3 %, 6 % at head size 64.)
          if constexpr (FIXED) lbf = dot2_bf16(pk[kb][pr], 0x3F803F80u, lbf);
        }
      // (the test on l, true for every finite sum, keeps this branch behind
      // the block above, whose exponentials run under the score products)
      lrun = l;
      if constexpr (!FIXED) {
        const bool rescale = __builtin_amdgcn_ballot_w64(bump && mrun != kNoScore && l >= 0.f) != 0;
        mrun = mx;
        if (__builtin_expect(rescale, 0)) {
#pragma unroll
          for (int ob = 0; ob < NOB; ++ob) oacc[ob] = oacc[ob] * alpha;
        }
      }
      // O^T += V^T P^T: k-step j takes keys 16 (j % 2) + {0..3, 8..11} + 4 lh of key block j / 2
      const uint8_t *const vt = cur + TILE;
      __builtin_amdgcn_s_setprio(0);
#pragma unroll
      for (int ob = 0; ob < NOB; ++ob) {
        f32x16_t acc = oacc[ob];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int kb = j >> 1, jj = j & 1;
          const u32x2_t v0 = vt_read(vt, ob, kb, jj, 0), v1 = vt_read(vt, ob, kb, jj, 1);
          const u32x4_t av = {v0[0], v0[1], v1[0], v1[1]};
          const u32x4_t bv = {pk[kb][4 * jj], pk[kb][4 * jj + 1], pk[kb][4 * jj + 2], pk[kb][4 * jj + 3]};
          acc = mfma32x32x16(av, bv, acc);
        }
        oacc[ob] = acc;
      }
      // The outputs are read by vector instructions next, in the branch below or
      // behind the loop: the wait states that a product's result needs before
      // that are put here, tied to the outputs.  Left to the compiler, a copy
      // of the last outputs at the end of a block followed their product too
      // closely and read old values.
      auto settle = [&]() {
#pragma unroll
        for (int ob = 0; ob < NOB; ++ob) asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 3" : "+v"(oacc[ob]));
      };
      if constexpr (LAST) settle();
      if (__builtin_expect(odd_values, 0)) {
        if constexpr (!LAST) settle();
        // the values that were set to zero, for the rows that see their keys:
        // a sum with one of them is what that value makes of it
        for (int key = max(k0, rlo); key < min(k0 + KT, rhi); ++key) {
          const int phys = bt[key / kPageSize];
          if ((unsigned)phys >= (unsigned)a.kv.num_pages) continue;
          const size_t e0 = ((size_t)phys * a.nkv + kh) * (kPageSize * HD) + (size_t)(key % kPageSize) * HD;
#pragma unroll
          for (int ob = 0; ob < NOB; ++ob)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const size_t e = e0 + ob * 32 + 8 * (i >> 2) + 4 * lh + (i & 3);
              uint32_t w;
              if constexpr (F8)
                w = e4m3x2_to_bf16x2<false>(a.kv.v8()[e]) & 0xFFFFu;
              else
                w = a.kv.v[e];
              if ((w & 0x7F80u) == 0x7F80u) oacc[ob][i] += bf16_lo(w);
            }
        }
      }
      if constexpr (!LAST) {
        if constexpr (F8) {
          land(kreg, cur, false);
          land(vreg, nxt + TILE, true);
        }
        sc[0] = scn[0];
        sc[1] = scn[1];
        wait_loads<0>();
        __syncthreads();
      }
    };
    for (int t = t0; t + 1 < t1; ++t) step(t, std::false_type{});
    step(t1 - 1, std::true_type{});
  }
  float l = lrun;
  l += shfl_xor_f32(l, 32);
  if constexpr (FIXED) lbf += shfl_xor_f32(lbf, 32);
  if (!qok) return;
  const float vscale = F8 ? a.kv.vs : 1.f;
  const int qh = kh * G + hrow;
  if (r.nsplit == 1) {
    const bool empty = rlo >= rhi;
    const float inv = empty ? 0.f : vscale / (FIXED ? lbf : l);
    const size_t at = (size_t)(r.row0 + qrel) * a.nq + qh;
    uint16_t *dst = a.out + at * HD + 4 * lh;
#pragma unroll
    for (int ob = 0; ob < NOB; ++ob)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const u32x2_t w = {pack_bf16x2(oacc[ob][4 * g] * inv, oacc[ob][4 * g + 1] * inv),
                           pack_bf16x2(oacc[ob][4 * g + 2] * inv, oacc[ob][4 * g + 3] * inv)};
        *reinterpret_cast<u32x2_t *>(dst + ob * 32 + 8 * g) = w;
      }
    if (lh == 0 && a.lse) a.lse[at] = empty ? kNoScore : kLn2 * (mrun + log2f(l));
    return;
  }
  const size_t slot = ((size_t)m[PRE_PART0 * a.n + r.k] + (size_t)qrel * r.nsplit + sp) * a.nq + qh;
  float *dst = a.part_o + slot * HD + 4 * lh;
  // (joined with weights of l)
  const float by = FIXED && l > 0.f ? vscale * (l / lbf) : vscale;
#pragma unroll
  for (int ob = 0; ob < NOB; ++ob)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<f32x4_t *>(dst + ob * 32 + 8 * g) =
          f32x4_t{oacc[ob][4 * g] * by, oacc[ob][4 * g + 1] * by, oacc[ob][4 * g + 2] * by, oacc[ob][4 * g + 3] * by};
  if (lh == 0) {
    // (an offset where nothing was seen would count as a maximum where the splits are joined)
    a.part_ml[slot * 2] = FIXED && l == 0.f ? kNoScore : mrun;
    a.part_ml[slot * 2 + 1] = l;
  }
}

// Joins the splits of the rows that have several, one wavefront per query head.
template <int HD>
__global__ __launch_bounds__(256) void k_attend_chunk_combine(AttendArgs a) {
  const meta_t m = meta_words(a);
  // (a request without splits has the first row of the one after it: the last
  // entry at or below a row is that of a request that has splits)
  const PreReq r = pre_req(a, m, last_at_or_below(m + PRE_COMB0 * a.n, a.n, blockIdx.x));
  const int qh = blockIdx.y * 4 + (threadIdx.x >> 6);
  if (qh >= a.nq) return;
  const int j = blockIdx.x - m[PRE_COMB0 * a.n + r.k], p = r.c + j;
  const bool empty = row_first(a, r.row0 + j, p) >= max(p + 1, r.prefix);
  const size_t base = ((size_t)m[PRE_PART0 * a.n + r.k] + (size_t)j * r.nsplit) * a.nq + qh;
  join_splits<HD>(a, base, r.nsplit, (size_t)(r.row0 + j) * a.nq + qh, empty, threadIdx.x & 63);
}

}  // namespace

hipError_t launch_attend_chunk(const Shape &s, const AttendCall &c, const AttendArgs &a, hipStream_t st) {
  const AttendPlan &p = *c.plan;
  const dim3 grid(p.pre_tiles * s.nkv);
  const int mode = c.slopes ? (c.softcap > 0.f ? kCapBiased : kBiased) : c.softcap > 0.f ? kCapped : kPlain;
#define EB_CHUNK_M(HD_, F8_, MODE_)                                                        \
  case MODE_:                                                                              \
    hipLaunchKernelGGL((k_attend_chunk<HD_, F8_, MODE_>), grid, dim3(256), 0, st, a);      \
    break
#define EB_CHUNK(HD_, F8_)             \
  switch (mode) {                      \
    EB_CHUNK_M(HD_, F8_, kPlain);      \
    EB_CHUNK_M(HD_, F8_, kCapped);     \
    EB_CHUNK_M(HD_, F8_, kBiased);     \
    EB_CHUNK_M(HD_, F8_, kCapBiased);  \
  }
  if (s.hd == 128) {
    if (a.kv.f8) {
      EB_CHUNK(128, true)
    } else {
      EB_CHUNK(128, false)
    }
  } else if (a.kv.f8) {
    EB_CHUNK(64, true)
  } else {
    EB_CHUNK(64, false)
  }
#undef EB_CHUNK
#undef EB_CHUNK_M
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (p.pre_comb_rows > 0) {
    const dim3 cg(p.pre_comb_rows, (s.nq + 3) / 4);
    if (s.hd == 128)
      hipLaunchKernelGGL(k_attend_chunk_combine<128>, cg, dim3(256), 0, st, a);
    else
      hipLaunchKernelGGL(k_attend_chunk_combine<64>, cg, dim3(256), 0, st, a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace eb
