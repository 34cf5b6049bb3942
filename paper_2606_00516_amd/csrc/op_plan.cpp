#include <hip/hip_runtime.h>

#include "op_plan.h"

#include <algorithm>
#include <cmath>
#include <numeric>

namespace eb {

namespace {
// Splits of the keys of a chunk: enough blocks to fill the chip if this were
// its only request, each long enough that the partials (fp32 rows written and
// read again) and the blocks' starts stay small beside the keys it reads.  Few
// rows: splits of at least 4 tiles suit a request alone, of 12 batches that fill
// the chip (with the join, 32 heads over 8, 4 / 12 tiles: one request of 5 rows
// over 2500 keys 13.9 / 26.1 us, over 4096 16.3 / 26.6; 24 of them over 2000 62 /
// 50, over 4096 112 / 88).  The line at 40 tiles gives short contexts to the one
// and long ones to the other: past it a lone request pays 10 us, below it a full
// batch 20 %.  Many rows: 16 tiles (a chunk of 1000 without context 31 us, 42 with
// splits of 8; 24 and 32 like 16).
int32_t chunk_splits(int32_t rows, int32_t kv_heads, int32_t q_blocks, int32_t tiles) {
  const int32_t items = q_blocks * kv_heads;
  const int32_t least = rows > kAttendRows ? 16 : tiles > 40 ? 12 : 4;  // tiles per split
  return std::max(1, std::min((512 + items - 1) / items, tiles / least));
}

// Parts of the rows in the weights pass of a chunk of `runs` runs of 32 rows,
// where the call has `blocks` blocks of 64 keys of a kv head.  Where these are
// few, enough parts to fill the chip, of four runs a wavefront at least.  Where
// they are many and the runs no more than a block's wavefronts, 0: each
// wavefront takes all of them for 64 keys of its own.  (One prompt of 1009 rows,
// 4 kv heads, 64 blocks: in 8 parts 21 us and 4.5 to join, whole 62; six prompts
// of 1376 blocks: in 2 parts 14 us slower.  Eight requests of 2 or 3 rows over
// 5000 keys, 2560 blocks: keys apart 22.6 us, not 28.3; three of 32 counted rows
// and 480 blocks: 10.8 and 8.0.)
// A row's own results do not depend on its batch; the order of a weight's sum
// may.
int32_t weight_parts(int32_t runs, int64_t blocks) {
  if (runs <= kWeightWaves && blocks >= 1024) return 0;
  return (int32_t)std::max<int64_t>(1, std::min<int64_t>((512 + blocks - 1) / blocks, runs / (4 * kWeightWaves)));
}
}  // namespace

bool plan_attend(const eb_layer_config &cfg, const eb_batch &b, int32_t window, const int32_t *prefix, bool weights,
                 int32_t weight_rows, AttendPlan &p) {
  p = AttendPlan();
  p.T = b.num_tokens;
  const int32_t G = cfg.n_q_heads / cfg.n_kv_heads, nkv = cfg.n_kv_heads, bq = kAttendRows / G;
  std::vector<int32_t> ones, many, row(b.num_seqs + 1, 0);
  for (int i = 0; i < b.num_seqs; ++i) {
    row[i + 1] = row[i] + b.chunk_lens_host[i];
    (b.chunk_lens_host[i] == 1 ? ones : many).push_back(i);
  }
  const auto keys_of = [&](int i) { return b.context_lens_host[i] + b.chunk_lens_host[i]; };
  p.n_dec = (int32_t)ones.size();
  p.dec.assign((size_t)DEC_FIELDS * p.n_dec, 0);
  int64_t runs = 0;
  int32_t part = 0;  // partials of the chunks, behind those of the decode rows
  const auto fits = [&]() {  // (each request adds less than 2^30 to a count: looked at after each, none wraps)
    return std::max({p.dec_splits, p.dec_wblocks, p.pre_tiles, p.pre_wblocks, p.pre_wparts}) <= kMostBlocks / nkv &&
           part <= 0x3FFFFFFF && runs <= 0x7FFFFFFF;
  };
  // the longest splits first: the launch ends on the shortest
  const auto split_of = [&](int i) {
    const int32_t c = b.context_lens_host[i];
    return attend_split_keys(c + 1 - attend_first(c, window));
  };
  std::stable_sort(ones.begin(), ones.end(), [&](int32_t x, int32_t y) { return split_of(x) > split_of(y); });
  for (int32_t d = 0; d < p.n_dec; ++d) {
    const int i = ones[d];
    const int32_t c = b.context_lens_host[i], keys = c + 1 - attend_first(c, window);
    const int32_t per = attend_split_keys(keys), ns = (keys + per - 1) / per;
    int32_t *f = p.dec.data() + d;
    const size_t n = (size_t)p.n_dec;
    f[DEC_SEQ * n] = i;
    f[DEC_ROW * n] = row[i];
    f[DEC_CTX * n] = c;
    f[DEC_SPLIT0 * n] = p.dec_splits;
    f[DEC_WBLOCK0 * n] = p.dec_wblocks;
    f[DEC_SCORE0 * n] = (int32_t)runs;
    p.dec_splits += ns;
    p.dec_most = std::max(p.dec_most, per);
    if (ns > 1) p.dec_combine = true;
    if (weights) {
      p.dec_wblocks += (keys + kWeightSpan - 1) / kWeightSpan;
      runs += (int64_t)((keys + 15) / 16) * cfg.n_q_heads;
    }
    if (!fits()) return false;
  }
  std::stable_sort(many.begin(), many.end(), [&](int32_t x, int32_t y) { return keys_of(x) > keys_of(y); });
  // blocks of so many keys of request i that the rows from j on may see
  const auto key_blocks = [&](int i, int32_t j, int32_t keys) {
    const int32_t c = b.context_lens_host[i];
    return (c + b.chunk_lens_host[i] + keys - 1) / keys - std::min(c, attend_first(c + j, window)) / keys;
  };
  int64_t wblocks = 0;  // (all rows: the workspace's size does not know weight_rows)
  if (weights)
    for (int i : many) wblocks += (int64_t)key_blocks(i, 0, kWeightKeys) * nkv;
  p.n_pre = (int32_t)many.size();
  p.pre.assign((size_t)PRE_FIELDS * p.n_pre, 0);
  part = p.dec_splits;
  for (int32_t k = 0; k < p.n_pre; ++k) {
    const int i = many[k];
    const int32_t c = b.context_lens_host[i], n = b.chunk_lens_host[i], nqb = (n + bq - 1) / bq;
    // the most tiles of any block of rows: the last one's, or with a prefix
    // past it the first one's behind the window
    int32_t tiles = 0;
    for (int32_t q = 0; q < nqb; q = q + 1 < nqb ? nqb - 1 : nqb) {
      const int32_t first = attend_first(c + q * bq, window) / kAttendTile;
      const int32_t end = std::max(c + std::min(n, (q + 1) * bq), prefix ? prefix[i] : 0);
      tiles = std::max(tiles, (end + kAttendTile - 1) / kAttendTile - first);
    }
    const int32_t ns = chunk_splits(n * G, nkv, nqb, tiles);
    const size_t m = (size_t)p.n_pre;
    int32_t *f = p.pre.data() + k;
    f[PRE_SEQ * m] = i;
    f[PRE_ROW * m] = row[i];
    f[PRE_CTX * m] = c;
    f[PRE_LEN * m] = n;
    f[PRE_PREFIX * m] = prefix ? prefix[i] : 0;
    f[PRE_TILE0 * m] = p.pre_tiles;
    f[PRE_NSPLIT * m] = ns;
    f[PRE_PART0 * m] = part;
    f[PRE_COMB0 * m] = p.pre_comb_rows;
    f[PRE_WBLOCK0 * m] = p.pre_wblocks;
    p.pre_tiles += nqb * ns;
    if (ns > 1) {
      part += n * ns;
      p.pre_comb_rows += n;
    }
    if (weights) {
      // every new key gets its first value, every key that a counted row may
      // see gets its share
      const int32_t j0 = weight_rows > 0 ? std::max(0, n - weight_rows) : 0;
      const int32_t parts = weight_parts((n - j0 + 32 / G - 1) / (32 / G), wblocks);
      const int32_t wb = key_blocks(i, j0, parts == 0 ? kWeightKeys * kWeightWaves : kWeightKeys);
      f[PRE_WPARTS * m] = parts;
      f[PRE_WPART0 * m] = p.pre_wparts;
      f[PRE_WJOIN0 * m] = p.pre_wjoins;
      p.pre_wblocks += wb * std::max(1, parts);
      if (parts > 1) {
        p.pre_wparts += wb * parts;
        p.pre_wjoins += wb;
      }
    }
    if (!fits()) return false;
  }
  size_t off = 0;
  const auto take = [&](size_t bytes) {
    const size_t o = off;
    off = (off + bytes + 255) / 256 * 256;
    return o;
  };
  p.o_dec = take(p.dec.size() * 4);
  p.o_pre = take(p.pre.size() * 4);
  p.o_lse = weights ? take((size_t)p.T * cfg.n_q_heads * 4) : 0;
  p.o_part_o = take((size_t)part * cfg.n_q_heads * cfg.head_dim * 4);
  p.o_part_ml = take((size_t)part * cfg.n_q_heads * 8);
  p.o_scores = take((size_t)runs * 64);
  p.o_wparts = take((size_t)p.pre_wparts * nkv * kWeightKeys * 4);
  p.total = off;
  return true;
}

void rotary_frequencies(int R, double theta, double *w) {
  const long double step = std::exp(-2.L / R * std::log((long double)theta));
  long double v = 1.L;
  for (int t = 0; t < R / 2; ++t, v *= step) w[t] = (double)v;
}

bool plan_evict(int32_t n_kv, int32_t S, const int32_t *lens, const int32_t *keep, EvictPlan &p) {
  p = EvictPlan();
  p.S = S;
  p.words.assign((size_t)EV_FIELDS * S, 0);
  int64_t runs = 0;
  for (int i = 0; i < S; ++i) {
    const int32_t c = lens[i], k = std::min(lens[i], keep[i]);
    const size_t n = (size_t)S;
    p.words[EV_LEN * n + i] = c;
    p.words[EV_KEEP * n + i] = keep[i];
    p.words[EV_GROUP0 * n + i] = (int32_t)p.groups;
    p.words[EV_SEG0 * n + i] = (int32_t)p.segments;
    p.words[EV_LIST0 * n + i] = (int32_t)runs;
    p.groups += (k + kEvictGroupKeys - 1) / kEvictGroupKeys;
    p.segments += (c + evict_segment(c) - 1) / evict_segment(c);
    runs += (c + 15) / 16;
    p.max_len = std::max(p.max_len, c);
    p.max_keep = std::max(p.max_keep, k);
    if (std::max(p.groups, p.segments) > kMostBlocks / n_kv || runs > 0x7FFFFFFF) return false;
  }
  size_t off = 0;
  const auto take = [&](size_t bytes) {
    const size_t o = off;
    off = (off + bytes + 255) / 256 * 256;
    return o;
  };
  const size_t heads = (size_t)S * n_kv;
  p.o_words = take(p.words.size() * 4);
  p.o_kept = take(heads * p.max_keep * 4);
  if (p.max_len > kEvictBlock) {
    p.o_hist = take(heads * 2049 * 4);
    p.o_list_v = take((size_t)runs * 16 * n_kv * 4);
    p.o_list_t = take((size_t)runs * 16 * n_kv * 4);
    p.o_seg = take((size_t)p.segments * n_kv * 8);
    p.o_solved = take(heads * 8);
  }
  p.total = off;
  return true;
}

}  // namespace eb
