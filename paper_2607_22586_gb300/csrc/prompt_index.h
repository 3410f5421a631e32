// How attention over whole prompts shares its units out, for the host and the device. A unit is
// (request, KV head, tile of query rows).
#pragma once

#include <stdint.h>

#include <algorithm>

#include "cache_index.h"

namespace mmshift {

constexpr int kPromptRequests = 64;

// Units go to the workers as wholes, longest first: worker i takes the i-th of each round of units,
// in odd rounds from the round's end. No unit is shared then, and there is nothing to merge. Causal:
// requests by falling numbers of tiles, and from segment k's first tile down to segment k + 1's,
// the tiles of the first k + 1 requests. Else: requests by falling length, a segment each.
struct PromptOrder {
  int32_t whole, units, segments;
  int32_t off[kPromptRequests + 1];   // units before a segment
  int32_t req[kPromptRequests];       // its request
  int32_t tiles[kPromptRequests];     // the request's tiles
};

struct PromptUnit {
  int b, h, tile;
};

// The i-th unit.
MMSHIFT_HD PromptUnit prompt_unit(const PromptOrder& O, int n_heads, int causal, int i) {
  const int k = range_of(O.off, O.segments, i), x = i - O.off[k];
  if (!causal) return PromptUnit{O.req[k], x % n_heads, x / n_heads};
  const int per = (k + 1) * n_heads, y = x % per;
  return PromptUnit{O.req[y / n_heads], y % n_heads, O.tiles[k] - 1 - x / per};
}

// Unit of a worker in a round, -1 behind the last.
MMSHIFT_HD int prompt_turn(const PromptOrder& O, int workers, int worker, int round) {
  const int64_t u = (int64_t)round * workers + (round & 1 ? workers - 1 - worker : worker);
  return u < O.units ? (int)u : -1;
}

// Keys of a request's tile of `rows` query rows, r heads a token.
MMSHIFT_HD int prompt_tile_keys(int n, int r, int rows, int causal, int tile) {
  const int64_t last = (int64_t)(tile + 1) * rows - 1, all = (int64_t)n * r - 1;
  return causal ? (int)((last < all ? last : all) / r) + 1 : n;
}

// The order of a batch's units; off: the requests' first tokens, `rows` a tile's.
inline PromptOrder prompt_order(int B, const int32_t* off, int r, int rows, int n_heads, int causal) {
  PromptOrder O = {};
  auto length = [&](int b) { return off[b + 1] - off[b]; };
  for (int b = 0; b < B; ++b)
    if (length(b)) O.req[O.segments++] = b;
  std::stable_sort(O.req, O.req + O.segments, [&](int x, int y) { return length(x) > length(y); });
  for (int k = 0; k < O.segments; ++k) O.tiles[k] = (int32_t)(((int64_t)length(O.req[k]) * r + rows - 1) / rows);
  for (int k = 0; k < O.segments; ++k) {
    const int next = k + 1 < O.segments ? O.tiles[k + 1] : 0;
    O.off[k + 1] = O.off[k] + n_heads * (causal ? (O.tiles[k] - next) * (k + 1) : O.tiles[k]);
  }
  O.units = O.off[O.segments];
  return O;
}

// Whether whole units do: where the workers' costs (sampled, in key tiles of 128; `start` for a
// unit's start and end) differ by less than what sharing units costs, their merge.
inline bool prompt_whole(const PromptOrder& O, const int32_t* off, int r, int rows, int n_heads, int causal, int workers,
                         int start, int merge) {
  // From eight units a worker on always: sharing costs more there than differing workers do but for the
  // extremes. A prompt of 2,500 tokens among 63 of 16, 20 heads, not causal, d = 128: 98 us (101 with shares, though
  // the longest share is 26 % above the mean); 30,000 among them, 32 heads: 9,600 to 9,700 (9,900 to 10,100);
  // but 4,000, 20 heads: 187 (176).
  if (O.units >= 8 * workers) return true;
  constexpr int kSamples = 12;
  int64_t most = 0, sum = 0;
  for (int s = 0; s < kSamples; ++s) {
    const int worker = (int)((int64_t)(workers - 1) * s / (kSamples - 1));
    int64_t cost = 0;
    for (int round = 0; round * workers < O.units; ++round) {
      const int u = prompt_turn(O, workers, worker, round);
      if (u < 0) continue;
      const PromptUnit x = prompt_unit(O, n_heads, causal, u);
      cost += start + (prompt_tile_keys(off[x.b + 1] - off[x.b], r, rows, causal, x.tile) + 127) / 128;
    }
    most = std::max(most, cost);
    sum += cost;
  }
  return most * kSamples <= sum + (int64_t)merge * kSamples;
}

}  // namespace mmshift
