// How products of block-scaled matrices and gated blocks are cut: tiles, slices of the contraction, workspace.  Host arithmetic.
#pragma once
#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace srq {

constexpr uint32_t FEW_ROWS = 16;  // up to so many rows of X there are no tiles

// A form's stage time is that of all its workgroups at once; half as many, one a CU where two fit, take HALF of it.  Beside the stages a
// launch takes START_US, and slices another launch and their sums to memory and back.  The figures are fitted to 38 launches, among them 1009 x
// 2048 x 5632, 113 and 300 x 11264 x 2048, 4096^3, 500 x 768 x 768 and gated blocks of 20 to 16384 rows, every form with 1 to 22 slices (of those
// within half of the best): what the model takes was within 1 % of the best of them in all but one, 5 % off there and in 24 other launches at most.
struct BlockForm {
  int bm, bn, per_cu;       // tile (gated: bn counts G's and U's columns), workgroups a CU
  float f8_us, exact_us;    // a stage
};
constexpr float START_US = 5.0f, SLICE_BYTES_PER_US = 7.9e6f, HALF = 0.63f;
struct BlockCut {
  int form;
  uint32_t chunk, whole, nsplit, per_split;
  size_t partial_bytes;
  float us;
};

inline BlockCut choose_block_cut(const BlockForm* forms, int nforms, float slices_us, size_t P, size_t columns, size_t R, bool f8) {
  BlockCut best = {};
  best.us = 3e38f;
  const size_t stages = std::max<size_t>(1, (R + 127) / 128);
  for (int f = 0; f < nforms; ++f) {
    const BlockForm& o = forms[f];
    const size_t tiles = ((P + o.bm - 1) / o.bm) * ((columns + o.bn - 1) / o.bn);
    const size_t chunk = (tiles + 7) / 8, slots = 32 * o.per_cu;  // of an XCD
    const size_t whole = chunk / slots * slots, rest = chunk - whole;
    const float stage = f8 ? o.f8_us : o.exact_us;
    for (size_t s = 1; s <= std::min<size_t>(stages, rest ? 32 : 1); ++s) {
      const size_t per = (stages + s - 1) / s;
      if (s > 1 && (stages + per - 1) / per != s) continue;  // no slice without a stage
      const size_t items = rest * s, last = items % slots;
      const float rounds = items / slots + (last == 0 ? 0.0f : 2 * last <= slots && o.per_cu > 1 ? HALF : 1.0f);
      const size_t bytes = s > 1 ? 8 * items * o.bm * o.bn * sizeof(float) : 0;
      const size_t used = s > 1 ? 8 * items * std::min<size_t>(P, o.bm) * o.bn * sizeof(float) : 0;
      const float us = START_US + (chunk / slots * stages + rounds * per) * stage + (s > 1 ? slices_us + 2 * used / SLICE_BYTES_PER_US : 0.0f);
      if (us < best.us) best = {f, (uint32_t)chunk, (uint32_t)(s > 1 ? whole : chunk), (uint32_t)s, (uint32_t)per, bytes, us};
    }
  }
  return best;
}

constexpr BlockForm PRODUCT_FORMS[] = {{256, 256, 1, 1.73f, 2.79f}, {128, 128, 2, 1.12f, 1.61f}, {64, 128, 2, 0.7f, 1.16f}, {64, 64, 2, 0.43f, 0.68f}};
// (the last two have the exact pipeline alone, whatever the flag: nothing of theirs waits for the matrix pipeline, which is busy in 13 % of the cycles)
constexpr BlockForm GATED_FORMS[] = {{256, 256, 1, 1.83f, 3.3f}, {128, 256, 1, 1.24f, 1.9f}, {64, 256, 1, 1.31f, 1.31f}, {32, 256, 1, 1.0f, 1.0f}};
inline BlockCut product_cut(size_t P, size_t Q, size_t R, int f8) { return choose_block_cut(PRODUCT_FORMS, 4, 2.4f, P, Q, R, f8); }
inline BlockCut gated_cut(size_t M, size_t F, size_t K, int f8) { return choose_block_cut(GATED_FORMS, 4, 3.5f, M, 2 * F, K, f8); }

}  // namespace srq
