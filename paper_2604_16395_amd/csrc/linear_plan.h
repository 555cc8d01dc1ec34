// How linear attention cuts a batch into workgroups, from the host lengths: which of its forms (linear_attn.hip) each
// request takes, by an estimate of their times.  Host code; the sizes of the workspace and of the grids follow from it.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "plan_rules.h"
#include "s2l.h"

namespace s2l {

// Requests of at most kLinearShortTokens new tokens are advanced token by token, the others in blocks.  32 heads, token
// by token against in blocks, us: of 5 tokens one request 4.5 against 6.4, 8 requests 10.4 against 11.3, 64 57.5 against
// 73; of 6 5.5 against 6.4, 12.5 against 11.2, 68 against 74; of 8 6.4 against 6.5, 14.7 against 11.3, 81 against 74; of 12
// 8.1 against 6.4, 17.9 against 11.3, 109 against 76.  So the lines cross between 5 and 8, first for a few requests.
constexpr int32_t kLinearShortTokens = 5, kLinearBlockTokens = 32;
struct LinearPlan {          // how the batch is cut, from the host lengths
  int32_t piece_tokens;      // longer requests are cut into pieces of so many tokens (a multiple of a block)
  int32_t unit_tokens;       // the longest piece's
  int32_t pieces;            // of all requests that are not short
  int32_t cut_reqs, ws_states;   // requests of more than one piece; one state before, between and after them
  int32_t short_reqs;
  bool narrow;               // no request is cut, and a workgroup takes half of a head's columns
};

// Estimated time in us of linear attention's blocked form where requests are cut into pieces of
// piece_blocks blocks of 32 tokens.  A workgroup takes the blocks of a (piece, head) one after another, so the longest piece's
// chain is one bound; blocks and states over all CUs are the other, with a part of the longest piece
// where a CU gets more than one.  Cut requests' own states take a launch of the same kind, and the sums between them
// read and write every state once.  Constants: a fit (0.07 rms of the logarithm) to 600 measured layers (51 batches of 1
// to 96 requests of 17 to 32768 tokens, 8 to 64 heads, each in up to 16 piece lengths); single ones make up for one
// another and are no times of parts.
inline double linear_cost(const s2l_batch* b, int32_t hq, int32_t num_cus, int64_t piece_blocks) {
  double units = 0, cut = 0, cut_units = 0, blocks = 0, cut_blocks = 0, states = 0, longest = 0;
  for (int32_t r = 0; r < b->num_reqs; ++r) {
    const int32_t c = b->chunk_lens_host[r];
    if (c <= kLinearShortTokens) continue;
    const int64_t n = ceil_div64(c, kLinearBlockTokens), k = ceil_div64(n, piece_blocks);
    units += (double)k;
    blocks += (double)n;
    longest = std::max(longest, (double)std::min(n, piece_blocks));
    if (k == 1) {
      states += 2;
    } else {
      states += (double)k;
      cut += 1;
      cut_units += (double)k;
      cut_blocks += (double)n;
    }
  }
  const double per_cu = (double)hq / num_cus;   // of units and blocks, each once a head
  // units of equal length come in rounds: a CU takes two of them in less than twice one's time
  const auto rounds = [&](double n, double n_blocks, double one, double two) {
    const double m = std::ceil(n * per_cu - 1e-9), odd = m - 2 * std::floor(m / 2);
    return n_blocks / (n * longest) * (std::floor(m / 2) * two + odd * one);
  };
  const double chain = longest * (1.94 + 0.05 * std::min(1.0, units * per_cu));
  const double uneven = 0.05 * std::min(1.0, std::max(0.0, units * per_cu - 1));
  double t = 6.7 + std::max({chain, (2.16 * blocks + 2.16 * states) * per_cu + uneven * longest * 1.99,
                             rounds(units, blocks, longest * 1.99, 2 * (2.16 * longest + 2.16 * states / units))});
  if (cut_units > 0)
    t += 6.2 + std::max({longest * 0.67, (0.2 * cut_blocks + 2.16 * cut_units) * per_cu,
                         rounds(cut_units, cut_blocks, longest * 0.67, 2 * (0.2 * longest + 2.16))}) +
         8.9 * (cut_units + cut) * per_cu;
  return t;
}

// The same for whole requests with half of a head's columns a workgroup.  A block takes 1.43 us with a CU to itself
// and up to 2.09 us where the others keep two workgroups on every CU; busy CUs take 1.35 us for each and 1.5 us for
// each unit's states, and units of equal length come in rounds, of 1.5 us a block and 2.2 us.
inline double linear_narrow_cost(const s2l_batch* b, int32_t hq, int32_t num_cus) {
  double units = 0, blocks = 0, longest = 0;
  for (int32_t r = 0; r < b->num_reqs; ++r) {
    const int32_t c = b->chunk_lens_host[r];
    if (c <= kLinearShortTokens) continue;
    const double n = (double)ceil_div64(c, kLinearBlockTokens);
    units += 1;
    blocks += n;
    longest = std::max(longest, n);
  }
  const double per_cu = 2.0 * hq / num_cus, rounds = std::ceil(units * per_cu - 1e-9), mean = blocks / units;
  return 5.2 + std::max({longest * (1.43 + 0.33 * std::min(2.0, blocks * per_cu / longest)), (1.35 * blocks + 1.5 * units) * per_cu,
                         rounds * (1.5 * mean * mean / longest + 2.2)});
}

// How linear attention cuts the batch: requests stay whole unless shorter pieces are estimated to be faster, and a
// head of a whole request gets two workgroups where that is estimated to be faster still: its blocks' chain is
// shorter, but a block's K and Q are read twice.  32 heads, one workgroup a head and two: a chunk of 64 tokens
// 10.0 us and 7.9, of 256 22.1 and 17.2; 8 requests of 391 to 1004 tokens 74 and 64, 16 of 512 86 and 97.
// Against the fastest of the measured piece lengths of each of those batches the choice takes 1.01 of the time in the
// geometric mean and 1.08 at most (examples, 32 heads: 2048 tokens whole 131 us, in pieces of 256 46 us; 16 requests
// of 1024 tokens whole 150 to 155 us, in pieces of 512 245).  (Times here are of calls one after another in a graph, over three
// sets of tensors in turn.)
inline LinearPlan linear_plan(const s2l_batch* b, int32_t hq, int32_t num_cus) {
  LinearPlan p = {};
  int64_t longest = 0, total = 0, units = 0;
  for (int32_t r = 0; r < b->num_reqs; ++r) {
    const int32_t c = b->chunk_lens_host[r];
    if (c <= kLinearShortTokens) continue;
    ++units;
    longest = std::max(longest, ceil_div64(c, kLinearBlockTokens));
    total += ceil_div64(c, kLinearBlockTokens);
  }
  int64_t blocks = std::max<int64_t>(longest, 1);
  double best = linear_cost(b, hq, num_cus, blocks);
  // more pieces only add work: of no use where the CUs have enough of it without
  if ((double)total * hq < 2 * (double)longest * num_cus) {
    for (const int64_t n : {2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64}) {
      const int64_t k = ceil_div64(longest, n);
      if (k < 2 && n > 2) break;
      const double cost = linear_cost(b, hq, num_cus, k);
      if (cost < best) best = cost, blocks = k;
    }
  }
  // with more units the CUs are busy either way; the other estimate is some 5 % low for uneven chunks
  if (units > 0 && (double)units * hq <= 16.0 * num_cus && linear_narrow_cost(b, hq, num_cus) < 1.05 * best) {
    p.narrow = true;
    blocks = std::max<int64_t>(longest, 1);
  }
  p.piece_tokens = (int32_t)(blocks * kLinearBlockTokens);
  for (int32_t r = 0; r < b->num_reqs; ++r) {
    const int32_t c = b->chunk_lens_host[r];
    if (c <= kLinearShortTokens) {
      ++p.short_reqs;
      continue;
    }
    const int32_t n = (int32_t)ceil_div64(c, p.piece_tokens);
    p.pieces += n;
    p.unit_tokens = std::max(p.unit_tokens, std::min(c, p.piece_tokens));
    if (n > 1) ++p.cut_reqs, p.ws_states += n + 1;
  }
  return p;
}
inline size_t linear_bytes(const LinearPlan& p, int32_t hq) {
  return (size_t)p.ws_states * hq * kHeadDim * kHeadDim * sizeof(float);
}

}  // namespace s2l
