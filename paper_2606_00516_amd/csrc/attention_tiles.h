// Page blocks of the paged cache into LDS, shared by the attention kernels.
#pragma once
#include "device_common.h"
#include "eb_internal.h"

namespace eb {

// Page blocks reach LDS by direct loads (no registers): each 16-byte chunk
// of a block goes to a position swizzled by its token, so that every load
// instruction still covers whole 256-byte token rows of HBM and the MFMA
// operand reads (16 tokens x one chunk per quarter-wave) hit 16 different
// bank groups.  A wavefront owns several page slots (K block then V block) and
// keeps the others in flight while it works on one: four slots in the layer
// step's decode attention, two (on half of the LDS) in the modified one.
template <int HD, bool F8 = false>
struct MdecTraits {
  static constexpr int ES = F8 ? 1 : 2;            // bytes per cached element
  static constexpr int BLK = kPageSize * HD * ES;  // bytes of one (page, kv head) block
  static constexpr int SLOT = 2 * BLK;             // K block, then V block
  static constexpr int NDMA = BLK / 1024;          // 1 KiB load instructions per block
  static constexpr int ROW = HD * ES;              // bytes per token row
  static_assert(NDMA >= 1, "block of at least 1 KiB");
};

// 16-byte chunk position exchange of token row t: rows of 256 bytes (bf16,
// HD 128) take t & 15, 128-byte rows t & 7, 64-byte rows (t >> 1) & 3 ...
template <int HD, bool F8 = false>
EB_DEV int mdec_swz(int t) {
  constexpr int ROW = MdecTraits<HD, F8>::ROW;
  return ROW == 256 ? (t & 15) : ROW == 128 ? ((F8 ? t : (t >> 1)) & 7) : ((t >> 1) & 3);
}

// Upper halves of two fp32 values that hold bf16 numbers exactly, packed.
EB_DEV uint32_t bf16_pair_exact(float lo, float hi) {
  return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}


}  // namespace eb
