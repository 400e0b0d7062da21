// How the attention of many rows shares its work out (preba_attend_tiles.cu), as arithmetic on sizes alone:
// used on the host and on the device, and plain C++ so that it can be tested without either.
#ifndef PREBA_ATTEND_PLAN_H_
#define PREBA_ATTEND_PLAN_H_

#include <stdint.h>

#if defined(__CUDACC__)
#define PREBA_BOTH __host__ __device__
#else
#define PREBA_BOTH
#endif

namespace preba {
namespace attend {

constexpr uint32_t kTileRows = 128;     // rows of a tile, and keys of a key tile
constexpr uint32_t kMinRun = 2;         // key tiles of a CTA's run in the line, at least
constexpr uint64_t kLineUnits = 1ull << 31;  // a longer line is never formed: its places are 32-bit numbers
constexpr uint32_t kOwnPairs = 480;     // pairs of row tiles that a CTA plans for itself, at most (three for
                                        // each of 160 CTAs; with as many they could be claimed one by one)

// Pairs of row tiles in a step whose requests do not overlap, at most.
PREBA_BOTH inline uint64_t pairs_at_most(uint32_t n, uint32_t tokens, uint32_t group) {
  return tokens / (2 * (kTileRows / group)) + static_cast<uint64_t>(n);
}

struct share_t {
  bool claim;          // pieces are claimed one by one; else they form a line of `units` key tiles
  uint32_t units, per; // of the line, and of a CTA's run of it
};

// total: key tiles of all pairs on one key head, longest: of the longest pair.  Claimed if the longest is
// short beside a CTA's share of the line (prompts, longest a quarter of the share: 324 us; a chunk over a
// long cache, longest 2.3 times the share: 216 us in equal runs, against 1.5 shares and more if each were one
// CTA's), or if there is more work than a line can count: a claim needs no place in it.  In a line of packed states a pair
// counts set-up units beside its tiles, in `total` and not in `longest`: 46 requests of 58 rows over up to 937 states on 12 heads
// of 64 are claimed then and take 49.5 us, with them in both they would form a line and take 55.2; where all states fit one
// tile the two are within 1 us, either way.
PREBA_BOTH inline share_t share_out(uint64_t total, uint32_t heads_kv, uint32_t longest, uint32_t grid) {
  const uint64_t units = total * heads_kv;
  share_t s{3ull * longest * grid <= units || units > kLineUnits, 0, 0};
  if (s.claim) return s;
  s.units = static_cast<uint32_t>(units);
  const uint64_t per = (units + grid - 1) / grid;
  s.per = per > kMinRun ? static_cast<uint32_t>(per) : kMinRun;
  return s;
}

// Whether every CTA plans for itself: few pairs, and a line that it can count whatever the lengths are; set_up: units that a pair
// has in it beside its key tiles.  Without those it is sure that share_out() would form a line too.  With them it might claim
// short pairs instead, and the line is made all the same, because that saves the planning launch: 83 requests of 114 rows over up
// to 66 states on 4 heads of 64 17.4 us, planned and claimed 20.8; 30 of 260 over up to 300 on 8 heads 22.4 and 26.1.
PREBA_BOTH inline bool plans_own(uint64_t pairs, uint32_t heads_kv, uint32_t grid, uint64_t keys_at_most, uint32_t set_up = 0) {
  return pairs < kOwnPairs && pairs * heads_kv < 3ull * grid &&
         pairs * heads_kv * (keys_at_most / kTileRows + 2 + set_up) <= kLineUnits;
}

}  // namespace attend
}  // namespace preba

#endif  // PREBA_ATTEND_PLAN_H_
