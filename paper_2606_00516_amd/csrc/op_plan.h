// Host planning of the cache operators: pure C++, no HIP calls.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <vector>

#include "../../include/eb_layer.h"

namespace eb {

constexpr int kAttendTile = 64;    // keys per step of a chunk's rows
constexpr int kAttendRows = 128;   // query rows (positions x heads of the group) per block
constexpr int kWeightKeys = 64;    // keys per wavefront of the weights pass of a chunk
constexpr int kWeightWaves = 4;    // wavefronts of its blocks
constexpr int kWeightSpan = 1024;  // keys per block of the weights pass of a decode row

// Keys per split of a decode row that sees `keys` of them: equal shares, a
// multiple of 64 (a page for each of a block's wavefronts), of at most the
// size below.  They follow from the request alone, so that its result does
// not depend on the batch.  Splits of 128 suit a row alone, larger ones, which
// cost less to start and join, rows in batches.  With the join, 32 heads over 8,
// splits of 128 / 256 / 512: one row over 1500 keys 10.0 / 11.1 / 13.4 us, over
// 2100 10.8 / 11.3 / 12.9, over 4000 11.6 / 11.6 / 13.6, over 16000 28.2 / 19.8 /
// 18.6; 4 rows over 2100 18.6 / 15.4 / 14.3, 64 rows 135 / 106 / 96.  So between
// 2048 and about 8000 keys a lone row pays 2 us for what batches gain.  From 32768
// keys on 1024 (13 rows over 69000: of 512 351 us and 35 to join, of 1024 333
// and 13).
__host__ __device__ inline int32_t attend_split_keys(int32_t keys) {
  const int32_t most = keys <= 512 ? 64 : keys <= 2048 ? 128 : keys <= 32768 ? 512 : 1024;
  const int32_t n = (keys + most - 1) / most;
  return ((keys + n - 1) / n + 63) & ~63;
}
// First key (of a whole page) that the row at position p may see.
__host__ __device__ inline int32_t attend_first(int32_t p, int32_t window) {
  return window > 0 && p >= window ? (p - window + 1) & ~15 : 0;
}

// Tables of one attention call.  Decode part: requests with one new row, the
// longest splits first; chunk part: the others, the most keys first.  Each table is a
// run of arrays (below) of n entries.
struct AttendPlan {
  int32_t T = 0;
  int32_t n_dec = 0, dec_splits = 0, dec_wblocks = 0;
  int32_t dec_most = 0;  // keys of the longest split
  bool dec_combine = false;
  std::vector<int32_t> dec;
  int32_t n_pre = 0, pre_tiles = 0, pre_comb_rows = 0, pre_wblocks = 0, pre_wjoins = 0, pre_wparts = 0;
  std::vector<int32_t> pre;
  // byte offsets in the workspace (256-byte aligned)
  size_t o_dec = 0, o_pre = 0, o_lse = 0, o_part_o = 0, o_part_ml = 0, o_scores = 0, o_wparts = 0, total = 0;
};

// request, row, context, first split, first block of the weights pass, first
// 16-score run
enum DecField { DEC_SEQ = 0, DEC_ROW, DEC_CTX, DEC_SPLIT0, DEC_WBLOCK0, DEC_SCORE0, DEC_FIELDS };
// request, first row, context, rows, prefix, first tile, splits of the keys,
// first partial, first row among those with several splits; of the weights
// pass the first block, the parts of the rows (0: each wavefront has keys of
// its own), and for those with several the first partial and joining block
enum PreField {
  PRE_SEQ = 0, PRE_ROW, PRE_CTX, PRE_LEN, PRE_PREFIX, PRE_TILE0, PRE_NSPLIT, PRE_PART0, PRE_COMB0, PRE_WBLOCK0,
  PRE_WPARTS, PRE_WPART0, PRE_WJOIN0, PRE_FIELDS
};

// window 0: none; prefix: per request, or null.  The batch has passed
// check_batch.  False: more blocks or table entries than a launch holds.
bool plan_attend(const eb_layer_config &cfg, const eb_batch &b, int32_t window, const int32_t *prefix, bool weights,
                 int32_t weight_rows, AttendPlan &p);

// Blocks of a launch: their threads (up to 512 each) are counted in 32 bits.
constexpr int64_t kMostBlocks = 0x7FFFFF;

// w[t] = theta^(-2t/R), t < R / 2: by products of a step in extended precision
// (64 bits: R / 2 <= 64 of them leave 2^-57, far below an fp64 half step of
// 2^-53), rounded once.
void rotary_frequencies(int R, double theta, double *w);

// ---- eviction ----
constexpr int kEvictFew = 512;         // keys of the longest request: one wavefront chooses
constexpr int kEvictBlock = 16384;     // one block chooses; longer: segments
constexpr int kEvictSegment = 4096, kEvictSegments = 512;
constexpr int kEvictGroupKeys = 64;    // kept keys per copy block
// Keys per segment of a request of c keys: at most kEvictSegments of them.
__host__ __device__ inline int32_t evict_segment(int32_t c) {
  const int32_t all = kEvictSegment * kEvictSegments;
  return kEvictSegment * ((c + all - 1) / all > 1 ? (c + all - 1) / all : 1);
}

// length, kept, first copy block, first segment, first 16-key run of the lists
enum EvictField { EV_LEN = 0, EV_KEEP, EV_GROUP0, EV_SEG0, EV_LIST0, EV_FIELDS };
struct EvictPlan {
  int32_t S = 0, max_len = 0, max_keep = 0;
  int64_t groups = 0, segments = 0;
  std::vector<int32_t> words;
  size_t o_words = 0, o_kept = 0, o_hist = 0, o_list_v = 0, o_list_t = 0, o_seg = 0, o_solved = 0, total = 0;
};
// Lengths as given (not negative, at most 2^30).  False: more blocks than a
// launch holds.
bool plan_evict(int32_t n_kv, int32_t S, const int32_t *lens, const int32_t *keep, EvictPlan &p);

}  // namespace eb
