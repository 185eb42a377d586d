// Host-side check of pop::meet (csrc/regions.h) against all bytes of both arrays, for random layouts: nested as tensors' are
// (packed halves, gaps, broadcast and single axes, other orders of the axes) and any small strides, negative ones too.
#include <cstdio>
#include <random>
#include <set>
#include "regions.h"

using pop::Region;

static std::set<long long> bytes_of(const Region& r) {
  std::set<long long> all;
  for (int64_t i = 0; i < r.n[0]; ++i)
    for (int64_t j = 0; j < r.n[1]; ++j)
      for (int64_t k = 0; k < r.n[2]; ++k)
        for (int64_t c = 0; c < r.inner; ++c) all.insert((long long)r.at + i * r.stride[0] + j * r.stride[1] + k * r.stride[2] + c);
  return all;
}

int main() {
  int bad = 0, met = 0, near = 0;
  std::mt19937 rng(1);
  const auto in = [&](int lo, int hi) { return (int64_t)(lo + (int)(rng() % (unsigned)(hi - lo + 1))); };
  for (int round = 0; round < 60000; ++round) {
    Region r[2];
    const bool nested = round % 3 != 0, same_strides = round % 2 == 0;
    int64_t n[3], s[3];
    for (int which = 0; which < 2; ++which) {
      const int64_t inner = in(1, 5);
      if (which == 0 || !same_strides) {
        for (int64_t& v : n) v = in(1, 4);
        if (nested) {
          int64_t extent = in(5, 9);
          const int order[3] = {(int)in(0, 2), 0, 0};
          int axes[3] = {order[0], (order[0] + 1) % 3, (order[0] + 2) % 3};
          if (rng() % 2) { const int t = axes[1]; axes[1] = axes[2]; axes[2] = t; }
          for (int k : axes) {
            s[k] = extent + in(0, 3);
            extent = s[k] * n[k];
            if (rng() % 8 == 0) s[k] = 0;
          }
        } else {
          for (int64_t& v : s) v = in(-12, 12);
        }
      }
      r[which] = pop::region(which ? "b" : "a", (const void*)(uintptr_t)(1000 + in(0, nested ? 40 : 25)), inner, 3, n, s, which == 0);
    }
    const std::set<long long> a = bytes_of(r[0]);
    bool want = false;
    for (long long v : bytes_of(r[1])) want = want || a.count(v);
    const bool got = pop::meet(r[0], r[1]);
    met += want;
    near += !want && *a.begin() <= *bytes_of(r[1]).rbegin() && *bytes_of(r[1]).begin() <= *a.rbegin();
    if (got != want && bad++ < 5) std::printf("round %d: %d, want %d\n", round, got, want);
  }
  // halves of wider rows, large: apart; one element further: not
  const int64_t n[3] = {80, 8, 512}, s[3] = {8ll * 512 * 2048, 512 * 2048, 2048};
  const Region x = pop::region("x", (const void*)(1ull << 40), 1024, 3, n, s, false), g = pop::region("g", (const void*)((1ull << 40) + 1024), 1024, 3, n, s, true),
               h = pop::region("h", (const void*)((1ull << 40) + 1022), 1024, 3, n, s, true), far = pop::region("far", (const void*)((1ull << 40) + 79 * 8 * 512 * 2048ll - 1024), 1025, true);
  if (pop::meet(x, g) || !pop::meet(x, h) || !pop::meet(x, far)) { ++bad; std::printf("halves\n"); }
  pop::Regions call;
  const char *one = "", *other = "";
  call.add("x", (const void*)(1ull << 40), 1024, 3, n, s, false, 1);
  call.add("none", nullptr, 1024, true);
  call.add("y", (const void*)(1ull << 40), 1024, 3, n, s, true, 1);
  if (call.clash(one, other)) { ++bad; std::printf("%s %s\n", one, other); }
  call.add("z", (const void*)((1ull << 40) + 1), 8, true, 1);
  if (!call.clash(one, other)) { ++bad; std::printf("z\n"); }
  std::printf("met %d, within each other but apart %d, bad %d\n", met, near, bad);
  return bad != 0 || met < 1000 || near < 1000;
}
