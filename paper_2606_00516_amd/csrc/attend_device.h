// What the kernels of the modified attention share: their arguments, the
// score of a key and the rows' visible ranges.
//
//   s = scale q.k;  s = cap tanh(s / cap) with a cap;  s -= slope |p - t| with
//   a distance bias;  key t is visible to the row at position p iff
//   max(first_key, p - window + 1, 0) <= t < max(p + 1, prefix).
// Scores are held in log2 units.
#pragma once
#include <type_traits>

#include "attention_tiles.h"
#include "op_meta.h"
#include "ops.h"

namespace eb {

constexpr float kNoScore = -__builtin_inff();
// Room (log2 units) of a capped chunk row's probabilities above the 1 of an
// ordinary softmax, without an eye on the row's maximum: scores to 22 in size.
// A narrower one costs such rows, not others, 5 % (a look at every tile: 4096
// rows over 32768 keys with scores to 20 in size, 16 units 2.68 ms, 32 units
// 2.55); a wider one takes it from the values, whose sums share fp32's range.
constexpr float kCappedSlack = 32.0f;

struct AttendArgs {
  const uint16_t *qkv;
  uint16_t *out;
  float *lse, *weights, *part_o, *part_ml, *scores, *wparts;
  const int32_t *first_key;
  const float *slopes;
  KV kv;
  int32_t nq, nkv, group, window, n, weight_rows;  // n: requests of the table
  int32_t stash;                                   // bytes of LDS for a decode split's scores; 0: stored as they come
  float qscale;                                    // no cap: to log2 units; cap: 2 log2(e) scale / cap
  float cap2, ratio;                               // cap in log2 units, scale / cap
  // cap tanh(scale raw / cap) log2(e) = raw (tanh_c[0] + tanh_c[1] raw^2 + ..)
  // up to |raw| = small_raw (-1: the coefficients leave fp32)
  float small_raw, tanh_c[5];
  float even_raw;  // up to small_raw, and no score leaves +-kCappedSlack
  const int32_t *meta;
  Words inl;
};
static_assert(sizeof(AttendArgs) < 4096, "kernel arguments");

// tanh(x) = x P(x^2) to |x| = kTanhSmall, of degree 9: minimax of the relative
// error on that range, 1.5e-7 (found by exchange in 64 bits).  Past it 1 - 2 /
// (e^2x + 1), exact at both ends (e^2x = 0 and infinite), whose error is of the
// same size there, but is that of the cap itself and not of a score far below
// it: of caps of hundreds it would leave 1e-4.  Both hold a score to a few fp32
// half steps of its own size.
constexpr float kTanhSmall = 0.65f;
constexpr double kTanhP[5] = {0.999999846, -0.333315002, 0.132978737, -0.0515179164, 0.0146250855};

// One capped score from its raw product, any size of it; add: minus the offset.
EB_DEV float capped_score(float raw, const AttendArgs &a, float add = 0.f) {
  const float x = raw * a.ratio, u = x * x;
  const float p = fmaf(fmaf(fmaf(fmaf((float)kTanhP[4], u, (float)kTanhP[3]), u, (float)kTanhP[2]), u, (float)kTanhP[1]),
                       u, (float)kTanhP[0]);
  const float e = fast_exp2(raw * a.qscale);
  const float large = fmaf(-2.0f * a.cap2, __builtin_amdgcn_rcpf(e + 1.0f), a.cap2 + add);
  return fabsf(x) <= kTanhSmall ? fmaf(a.cap2 * x, p, add) : large;
}

// The largest size of a lane's raw products.  Where all of a wavefront's are
// small (up to small_raw) the polynomial alone serves, the cap and the scale in
// its coefficients: 6 full-rate operations a score and no transcendental,
// against 13 and 2 of a quarter rate.
template <int N>
EB_DEV float largest(const f32x16_t (&s)[N]) {
  float big = 0.f;
#pragma unroll
  for (int b = 0; b < N; ++b)
#pragma unroll
    for (int i = 0; i < 16; i += 2) big = fmaxf(fmaxf(fabsf(s[b][i]), fabsf(s[b][i + 1])), big);
  return big;
}
EB_DEV bool none(bool x) { return __builtin_amdgcn_ballot_w64(x) == 0; }
EB_DEV float small_ratio(float raw, const AttendArgs &a) {
  const float u = raw * raw;
  return fmaf(fmaf(fmaf(fmaf(a.tanh_c[4], u, a.tanh_c[3]), u, a.tanh_c[2]), u, a.tanh_c[1]), u, a.tanh_c[0]);
}
EB_DEV float small_score(float raw, const AttendArgs &a) { return raw * small_ratio(raw, a); }
EB_DEV float small_score(float raw, const AttendArgs &a, float add) { return fmaf(raw, small_ratio(raw, a), add); }

// First key the row at position p may see (the window and its own bound).
EB_DEV int row_first(const AttendArgs &a, int row, int p) {
  int lo = a.window > 0 && p >= a.window ? p - a.window + 1 : 0;
  if (a.first_key) lo = max(lo, a.first_key[row]);
  return lo;
}

// Waits until at most N of the wavefront's vector memory operations are
// outstanding.  The direct loads into LDS are waited for by name: the
// compiler's own count has been seen to leave one out where a loop carries
// them over its back edge.
template <int N>
EB_DEV void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"i"(N) : "memory");
}

// A buffer range (uniform) as the four words of its descriptor.  SAID: says so
// to the compiler, where it does not see it (where it does, the saying cost
// registers: capped chunks 2.99 ms instead of 2.74).
template <bool SAID = false>
EB_DEV u32x4_t range_words(const uint8_t *base, int bytes) {
  const uint64_t b = (uint64_t)base;
  auto u = [](uint32_t v) { return SAID ? (uint32_t)__builtin_amdgcn_readfirstlane((int)v) : v; };
  return u32x4_t{u((uint32_t)b), u((uint32_t)(b >> 32) & 0xFFFFu), u((uint32_t)bytes), 0x00020000u};
}
// One 16-byte-per-lane load from a buffer range (uniform) straight into LDS:
// lane l fills bytes 16 l .. 16 l + 15 from byte address dst (uniform) with the
// bytes at its offset, zeros past the range.  It has no output register, and
// the compiler does not count it: wait_loads before the bytes are read.  (The
// counted form makes the compiler wait for all of them before any read of the
// same array, the loads of later tiles among them.)  It sets m0, which no
// instruction around it keeps a value in.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <bool ONCE = false>
EB_DEV void lds_fill16(u32x4_t range, uint32_t dst, uint32_t off) {
  if constexpr (ONCE)  // data read once
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds"
                 :
                 : "s"(dst), "v"(off), "s"(range)
                 : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :
                 : "s"(dst), "v"(off), "s"(range)
                 : "memory", "m0");
}
#pragma clang diagnostic pop
// Byte address of a __shared__ array for it.
EB_DEV uint32_t lds_at(const void *p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void *)p;
}

constexpr float kLn2 = 0.69314718055994530942f;

// Joins ns partials (entries base, base + nq, ..) into row entry `at` of out
// and lse, by one wavefront: o = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s.
// Lane s % 64 holds partial s's factor, HD / 64 output dims per lane.  Up to 16
// partials' loads are issued together, the first 16 before their factors are
// known, so that few partials take one trip to memory.
template <int HD>
EB_DEV void join_splits(const AttendArgs &a, size_t base, int ns, size_t at, bool empty, int lane) {
  constexpr int DPL = HD / 64, N = 16;
  const size_t stride = (size_t)a.nq;
  const float *po = a.part_o + base * HD + lane * DPL, *pm = a.part_ml + base * 2;
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  float o[N][DPL];
  auto load = [&](int s0) {
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int i = 0; i < DPL; ++i) o[u][i] = po[(size_t)min(s0 + u, ns - 1) * stride * HD + i];
  };
  // maximum and sum of partial s
  auto ml = [&](int s) {
    return s < ns ? *reinterpret_cast<const f32x2_t *>(pm + s * stride * 2) : f32x2_t{kNoScore, 0.f};
  };
  f32x2_t v = ml(lane);
  load(0);
  float mx = v[0];
  for (int s = lane + 64; s < ns; s += 64) mx = fmaxf(mx, ml(s)[0]);
  mx = wave_max(mx);
  float den = 0.f, acc[DPL];
#pragma unroll
  for (int i = 0; i < DPL; ++i) acc[i] = 0.f;
  for (int c = 0; c < ns; c += 64) {
    if (c > 0) v = ml(c + lane);
    const float f = v[0] == kNoScore ? 0.f : fast_exp2(v[0] - mx);
    if (f != 0.f) den += f * v[1];
    for (int j = 0; j < min(64, ns - c); j += N) {
      if (c + j > 0) load(c + j);
#pragma unroll
      for (int u = 0; u < N; ++u) {
        // (past the last split the factor is 0; a split that saw nothing wrote no outputs)
        const float w = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), j + u));
#pragma unroll
        for (int i = 0; i < DPL; ++i) acc[i] = w != 0.f ? fmaf(w, o[u][i], acc[i]) : acc[i];
      }
    }
  }
  den = wave_sum(den);
#pragma unroll
  for (int i = 0; i < DPL; ++i)
    a.out[at * HD + lane * DPL + i] = (uint16_t)f32_to_bf16_bits(empty ? 0.f : acc[i] / den);
  if (lane == 0 && a.lse) a.lse[at] = empty ? kNoScore : kLn2 * (mx + log2f(den));
}

}  // namespace eb
