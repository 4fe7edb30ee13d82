// Host check of the blocks that the losses cut a response into: up to the longest response that a call takes they cover each of its slots
// once, and no index on the way leaves an int.
#include <algorithm>
#include <cstdint>
#include <cstdio>
using std::min;
#define LMHEAD_TILE_MAP_HOST 1
#include "../../paper_2603_04411_amd/csrc/tile_map.h"

int main() {
  using namespace lmhead;
  constexpr int k = kLossSlotsPerBlock, most = INT32_MAX;
  long bad = 0, cases = 0;
  for (int T : {1, 2, k - 1, k, k + 1, 3 * k + 5, 1 << 30, most - k, most - k + 1, most - k + 2, most - 1, most}) {
    const int64_t blocks = ((int64_t)T + k - 1) / k;
    if (loss_blocks(T) != blocks) ++bad;
    const int64_t from = blocks > 4 ? blocks - 4 : 0;
    int64_t next = from * k;
    for (int64_t b = from; b < blocks; ++b) {
      ++cases;
      const int t0 = (int)b * k, slots = block_slots(t0, T);
      if (t0 != next || slots < 1 || slots > k) ++bad;
      // a thread's last step over the block, and its last slot
      if ((int64_t)slots - 1 + 256 > most || (int64_t)t0 + slots - 1 > (int64_t)T - 1) ++bad;
      next += slots;
    }
    if (next != T) ++bad;
  }
  std::printf("cases=%ld bad=%ld\n", cases, bad);
  return bad != 0;
}
