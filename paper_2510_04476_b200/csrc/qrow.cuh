// A row of the 4-bit cache: its sizes, and how a quantised block of it is stored.
#pragma once
#include "qcache.cuh"
#include "qformat.cuh"

namespace q4 {

template <int DH>
struct Row {                                       // a cache row of one head
  static constexpr int BLK = DH < 128 ? DH : 128;  // channels of a block
  static constexpr int NB = DH / BLK;              // blocks
  static constexpr int NG = BLK / GROUP;           // scale groups of a block
  static constexpr int CODES = DH / 2;             // bytes of codes
  static constexpr int SCALES = DH / GROUP;        // scales
  static constexpr int SW = (SCALES + 1) / 2;      // 32-bit words that hold the scales
};

// What quantise_block gives one of a block's eight lanes, into block `blk` of key (kv = 0) or value (1) row `row`, counted over all
// sequences and heads; with the key's first block, the row's weight (none yet) and position.
template <int DH>
CCA_DEVINL void store_block(const QCache& c, size_t row, int kv, int blk, int lane8, int position,
                            const uint32_t (&code)[(Row<DH>::NG + 1) / 2], const uint32_t (&scale)[(Row<DH>::NG + 1) / 2]) {
  using R = Row<DH>;
  constexpr int NG = R::NG;
  uint8_t* dst = (kv ? c.v_codes : c.k_codes) + row * R::CODES + blk * (R::BLK / 2) + lane8 * 2 * NG;
  bf16* sc = (kv ? c.v_scales : c.k_scales) + row * R::SCALES + blk * NG;
  if constexpr (NG == 4) {
    *reinterpret_cast<uint2*>(dst) = make_uint2(code[0], code[1]);
    if (lane8 == 0) *reinterpret_cast<uint2*>(sc) = make_uint2(scale[0], scale[1]);
  } else if constexpr (NG == 2) {
    *reinterpret_cast<uint32_t*>(dst) = code[0];
    if (lane8 == 0) *reinterpret_cast<uint32_t*>(sc) = scale[0];
  } else {
    *reinterpret_cast<uint16_t*>(dst) = (uint16_t)code[0];
    if (lane8 == 0) *reinterpret_cast<uint16_t*>(sc) = (uint16_t)scale[0];
  }
  if (kv == 0 && blk == 0 && lane8 == 0) {
    if (c.weight) c.weight[row] = 0.f;
    if (c.position) c.position[row] = position;
  }
}

}  // namespace q4
