// Host check of the overlap test between the tensors of an attention call, byte by byte on small random layouts: what it calls shared is shared, and
// where one of the two is dense it finds all that is.
#include <cstdint>
#include <cstdio>
#include <random>
#include <vector>
#include "../../paper_2603_04411_amd/csrc/attn_regions.h"

using lmhead::Region;

int main() {
  std::mt19937 rng(1);
  auto pick = [&](int lo, int hi) { return (int)(lo + rng() % (unsigned)(hi - lo + 1)); };
  struct Some {
    Region r;
    std::vector<char> bytes;
    bool dense;
  };
  constexpr int kRoom = 6000;
  auto make = [&](Some& s) {
    const int n = pick(1, 3), t = pick(1, 4), h = pick(1, 3), row = pick(1, 6), unit = pick(1, 2), at = pick(1, 400);
    int64_t st[3];
    const int kind = pick(0, 3), gap = pick(0, 1) * pick(0, 9);
    const int order = pick(0, 1);      // heads within slots, or slots within heads
    const int64_t w = (row * 1 + unit - 1) / unit;
    if (kind == 0) {                   // any strides, rows that lie upon each other among them
      for (int64_t& x : st) x = pick(0, 40);
    } else {
      const int64_t inner = w + gap, mid = inner * (order ? t : h) + pick(0, 1) * pick(0, 20);
      st[1] = order ? inner : mid;
      st[2] = order ? mid : inner;
      st[0] = mid * (order ? h : t) + pick(0, 1) * pick(0, 60);
      if (kind == 1) st[pick(0, 2)] = 0;
    }
    attn_layout x{st[0], st[1], st[2]};
    s.r = Region(reinterpret_cast<const void*>((uintptr_t)at), x, n, t, h, row, unit);
    s.bytes.assign(kRoom, 0);
    for (int b = 0; b < n; ++b)
      for (int i = 0; i < t; ++i)
        for (int j = 0; j < h; ++j)
          for (int c = 0; c < row; ++c) {
            const int64_t p = at + (b * st[0] + i * st[1] + j * st[2]) * unit + c;
            if (p < kRoom) s.bytes[p] = 1;
          }
    int64_t last = 0, all = 0;
    for (int p = 0; p < kRoom; ++p)
      if (s.bytes[p]) last = p, ++all;
    s.dense = all == last - at + 1;
    return last + 1 - at == s.r.extent;
  };
  long bad = 0, cases = 0, shared = 0, found = 0;
  for (int x = 0; x < 60000; ++x) {
    Some a, b;
    if (!make(a) || !make(b)) ++bad;
    if (a.r.dense() && !a.dense) ++bad;
    bool truth = false;
    for (int p = 0; p < kRoom && !truth; ++p) truth = a.bytes[p] && b.bytes[p];
    const bool says = lmhead::share(a.r, b.r);
    if (says != lmhead::share(b.r, a.r)) ++bad;
    if (says && !truth) ++bad;
    if (truth && !says && ((a.r.dense() && b.r.nested) || (b.r.dense() && a.r.nested))) ++bad;
    if (lmhead::share(a.r, Region()) || lmhead::share(Region(), b.r)) ++bad;
    ++cases, shared += truth, found += says;
  }
  // strides at their limits do not wrap
  attn_layout far{1ll << 42, 1ll << 42, 1ll << 42};
  if (Region(reinterpret_cast<const void*>(4096), far, 65535, 1 << 30, 1024, 64, 1).extent <= 0) ++bad;
  std::printf("cases=%ld shared=%ld found=%ld bad=%ld\n", cases, shared, found, bad);
  return bad != 0;
}
