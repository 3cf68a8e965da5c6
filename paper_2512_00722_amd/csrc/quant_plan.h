// How launches of decode attention over caches in 4 and 8 bits are divided.  Host code
// without anything of the device in it, so that tests can ask for the division that a shape
// gets.
#pragma once

#include <float.h>

#include "internal.h"

namespace spec {

// Sequences whose parts a wavefront can deal out (a lane each).  From the 64th of the
// numbers of chunks, 2.9 times the mean and 63 more, or from 64, parts are at most B and a
// third of all, so that one of them always fits where there are two per sequence.
constexpr int kMostDealt = 64;

// The plan of the least estimated time.  A launch takes the longer of two: the busiest CU's
// share of the bytes (256 of them move 6.9 TB/s; workgroups that read a part of a token's row
// move 7% less per halving, and in 4 bits 45% where it is half a 128-byte line), and its
// wavefronts' chunks one after the other (0.86 us, of two heads 1.5: what a chunk's loads
// take to arrive, fitted with the one that a wavefront loads beyond its last, see quant_unit());
// workgroups beyond those resident cost 2.9 us a round, and parts a second launch and the
// traffic of their results.  Fitted to 4900 launches of 144 shapes (1 to 256 sequences and
// layers of 64 to 131072 tokens, 1 to 16 query heads per KV head, 4 and 8 bits, rows selected or
// not): on average it is 1.6% slower than the best plan, 12% at most.
// Between plans: 32 x 8 x 32768 tokens in 4 bits 1344 us with 8 wavefronts and no parts, 1367
// with 4 and four; 1 x 4096 6.2 and 3.9 to join the parts with 4 wavefronts to a unit in 32
// parts, 7.7 and 2.7 with 8 in 16; 1 x 512 7.6 in one part, 5.4 and 2.6 in four, where
// programs that launch one call after another wait 8.1 and 10.6.
inline QuantPlan make_plan(const QuantDims& d, int k_max, bool ragged) {
  const int heads_groups = d.G / group_heads(d.G);
  const int64_t lb = (int64_t)d.n_layers * d.B, rows = lb * d.H_q;
  const int chunks = (k_max + kDecodeChunk - 1) / kDecodeChunk;
  const int64_t all = lb * d.H_kv * chunks;  // of one head
  QuantPlan best{1, 4, 0, 1, false};
  float least = FLT_MAX;
  int chunks_each = 1;
  for (int nh = 1; nh <= 2; ++nh) {
    if (nh == 2 && (d.bits == 8 || d.H_kv % 2)) continue;
    // half lines pay for themselves only where a chunk or two of loads are all there is
    if (nh == 1 && d.bits == 4 && d.H_kv % 2 == 0 && all > 64 * kCUs) continue;
    const int64_t units = (int64_t)d.H_kv / nh * heads_groups;
    const float chunk_us =
        (float)kCUs * kDecodeChunk * nh * (2 * row_bytes(d.bits) + kScaleBytes) / 6.9e6f;
    const float wait_us = nh == 2 ? 1.5f : 0.86f;
    for (int w = 4; w <= 8; w += 4) {
      // Workgroups of a CU, as the other numbers were fitted with.  Registers and LDS hold as
      // many but for selected rows in 8 bits by 4 wavefronts (194 registers: 2) and, where rows
      // are not selected, one head in 4 bits (126: 4 workgroups of 4 wavefronts, 2 of 8).
      const int resident = w == 8 ? 1 : nh == 2 ? 2 : 3;
      for (int u = 0; 1 << u <= w && units % (1 << u) == 0; ++u) {
        const int64_t one = lb * (units >> u);
        if (one > INT32_MAX / (w * 64)) continue;
        const int waves = w >> u, most = (chunks + waves - 1) / waves;
        float narrow = nh == 1 && d.bits == 4 && d.H_kv > 1 ? 1.45f : 1.f;
        for (int64_t side = (int64_t)nh << u; side < d.H_kv; side *= 2) narrow += 0.07f;
        int last = 0;
        for (int target = 1; target <= 8 * kCUs; target = target == 1 ? 32 : 2 * target) {
          for (int up = 0; up < 2; ++up) {
            const int64_t want = up ? (target + one - 1) / one : target / one;
            const int n = want < 1 ? 1 : want > most ? most : (int)want;
            if (n <= last) continue;
            last = n;
            const int busiest = (int)((one * n + kCUs - 1) / kCUs);
            const int rounds = (busiest + resident - 1) / resident;
            const int own = (chunks + n * waves - 1) / (n * waves);  // of a wavefront
            const float bytes = (float)busiest * own * w * chunk_us * narrow;
            const float wait = (float)rounds * own * wait_us;
            float t = bytes > wait ? bytes + 0.02f * wait : wait + 0.02f * bytes;
            t += 2.9f * (rounds - 1) + (w == 8 ? 0.4f : 0.f) + (nh == 2 ? 0.26f : 0.f);
            if (n > 1) t += 4.7f + 0.71e-6f * 520 * (float)n * rows;
            if (t < least) {
              least = t;
              best = {nh, w, u, n, false};
              chunks_each = own;
            }
          }
        }
      }
    }
  }
  // Whole caches are seldom of one length: two parts per sequence to deal out where they are
  // long (us, in 4 bits of equal and of ragged lengths: 8 layers x 32 of 8192 tokens at most 376
  // and 244, not dealt 364 and 279; 32 x 8 of 32768 1398 and 928, 1389 and 945; in 8 bits 4 x 64
  // of 4096 338 and 230, 350 and 250).
  const bool dealt = d.B > 1 && d.B <= kMostDealt;
  if (ragged && dealt && best.n_split == 1 && chunks_each >= 128) best.n_split = 2;
  best.deal = dealt && best.n_split > 1 && chunks_each >= 8;
  return best;
}
inline int decode_tokens(const QuantDims& d) {
  const int64_t n = (int64_t)d.window + d.n_sink;
  return (int)(n < d.L_cap ? n : d.L_cap);
}

inline QuantPlan plan_of(const QuantDims& d, bool selected) {
  if (selected) return make_plan(d, d.k_max, false);
  return make_plan(d, decode_tokens(d), decode_tokens(d) == d.L_cap);
}

}  // namespace spec
