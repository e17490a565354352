// How the keys of an attention call are split over the GPU.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace brisk {

constexpr int kCUs = 256;

inline int ceil_div(int64_t a, int64_t b) { return static_cast<int>((a + b - 1) / b); }

// Runs of `keys` keys that `whole` workgroups would cover: the fewest rounds of
// workgroups, each counted as its keys and 512 for its start.  What that constant is
// hardly matters (64 to 1500 plan the timing cases alike): the rule fills a round,
// and weighs neither rows nor the bytes of the partial sums.  (64 caches of up to 2048
// keys, 512 workgroups: whole caches 110 us, runs of 512 keys 119, of 256 147.)
struct Runs { int count, keys; };
constexpr int64_t kMostRuns = 1 << 20;
inline Runs runs_of(int keys, int64_t whole, int step, int slots) {
  Runs best{};
  double least = 1e300;
  for (int s = 1; s <= 64; ++s) {
    const int run = ceil_div(ceil_div(keys, s), step) * step, count = ceil_div(keys, run);
    if (s > 1 && whole * count > kMostRuns) break;  // thousands of rounds: nothing to fill, and a launch has its limit
    const double cost = ((whole * count + slots - 1) / slots) * (run + 512.0);
    if (cost < least) {
      least = cost;
      best = {count, run};
    }
  }
  return best;
}

// Workgroups of a launch, and which one has which row tile of which group (a workgroup without one gets a group past the
// last): tiles of a group follow each other on one XCD (workgroups take turns on the 8 of them), whose cache then has
// its keys; but fewer groups than XCDs spread over all.  (253 blocks of 16 with 16 heads of 64 over one key head, 269 slots of
// prefix and up to 20 own ones in 4 bits: 123 us on one XCD, 58 so.)
__host__ __device__ constexpr int tile_grid(int groups, int tiles) { return (groups < 8 ? groups : (groups + 7) / 8 * 8) * tiles; }
struct GroupTile { int group, tile; };
__host__ __device__ constexpr GroupTile group_tile(int bid, int groups, int tiles) {
  if (groups < 8) return {bid % groups, bid / groups};
  return {bid / 8 / tiles * 8 + bid % 8, bid / 8 % tiles};
}

}  // namespace brisk
