// Page blocks of the paged cache into LDS, shared by the attention kernels.
#pragma once
#include "device_common.h"
#include "eb_internal.h"

namespace eb {

// Page blocks reach LDS by direct loads (no registers): each 16-byte chunk
// of a block goes to a position swizzled by its token, so that every load
// instruction still covers whole 256-byte token rows of HBM and the MFMA
// operand reads (16 tokens x one chunk per quarter-wave) hit 16 different
// bank groups.  A wavefront owns four page slots (K block then V block)
// and keeps three pages in flight while it works on the fourth.
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

typedef __attribute__((address_space(3))) void lds_void_t;

// Start the loads of page p (physical page phys, -1 past the end) K and V
// blocks into a slot; slots at or past k1 (and pages past the end or with a
// bad table entry) land as zeros without memory traffic, so cache poison
// never reaches the products.
template <int HD, bool F8>
__device__ __forceinline__ void mdec_dma_page(uint8_t *slot, const uint32_t *goff, const KV kv, int phys, int p,
                                              int k1, int nkv, int kh) {
  using Tr = MdecTraits<HD, F8>;
  const int nvalid = min(max(k1 - p * kPageSize, 0), kPageSize);
  const bool ok = phys >= 0 && phys < kv.num_pages;
  const size_t off = ok ? ((size_t)phys * nkv + kh) * kPageSize * HD : 0;
  // wave-uniform by construction; said so, so the descriptor stays scalar
  const int bytes = __builtin_amdgcn_readfirstlane(ok ? nvalid * Tr::ROW : 0);
  const buf_rsrc_t rk = F8 ? make_rsrc(kv.k8() + off, bytes) : make_rsrc(kv.k + off, bytes);
  const buf_rsrc_t rv = F8 ? make_rsrc(kv.v8() + off, bytes) : make_rsrc(kv.v + off, bytes);
#pragma unroll
  for (int i = 0; i < Tr::NDMA; ++i) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (lds_void_t *)(slot + i * 1024), 16, goff[i], 0, 0, kAuxNT);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (lds_void_t *)(slot + Tr::BLK + i * 1024), 16, goff[i], 0, 0,
                                             kAuxNT);
  }
}

// Upper halves of two fp32 values that hold bf16 numbers exactly, packed.
EB_DEV uint32_t bf16_pair_exact(float lo, float hi) {
  return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}


// One 16-byte-per-lane load from a buffer range straight into LDS: lane l
// fills bytes 16 l .. 16 l + 15 from dst (wave-uniform) with the bytes at its
// offset (zeros past the range).
__device__ __forceinline__ void lds_dma16(buf_rsrc_t r, uint8_t *dst, uint32_t off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void_t *)dst, 16, off, 0, 0, 0);
}

}  // namespace eb
