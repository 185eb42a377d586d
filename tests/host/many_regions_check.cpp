// Host-side check of csrc/regions.h: pop::meet for regions of four axes against all bytes of both, and pop::ManyRegions against
// pop::Regions, for random layouts that nest as tensors' do.
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
        for (int64_t l = 0; l < r.n[3]; ++l)
          for (int64_t c = 0; c < r.inner; ++c)
            all.insert((long long)r.at + i * r.stride[0] + j * r.stride[1] + k * r.stride[2] + l * r.stride[3] + c);
  return all;
}

int main() {
  int bad = 0, met = 0, near = 0, clashes = 0;
  std::mt19937 rng(1);
  const auto in = [&](int lo, int hi) { return (int64_t)(lo + (int)(rng() % (unsigned)(hi - lo + 1))); };
  const auto layout = [&](int64_t* n, int64_t* s) {
    int order[4] = {0, 1, 2, 3};
    for (int i = 3; i > 0; --i) std::swap(order[i], order[in(0, i)]);
    int64_t extent = in(4, 9);
    for (int k : order) {
      n[k] = in(1, 3);
      s[k] = extent + in(0, 3);
      extent = s[k] * n[k];
      if (rng() % 8 == 0) s[k] = 0;
    }
  };
  for (int round = 0; round < 30000; ++round) {
    Region r[2];
    int64_t n[4], s[4];
    layout(n, s);
    for (int which = 0; which < 2; ++which) {
      if (which && round % 2) layout(n, s);
      r[which] = pop::region("", (void*)(5000 + in(0, 60)), in(1, 4), 4, n, s, true);
    }
    const std::set<long long> a = bytes_of(r[0]), b = bytes_of(r[1]);
    bool common = false;
    for (long long x : a) common = common || b.count(x);
    met += common;
    near += !common && *a.begin() < *b.rbegin() && *b.begin() < *a.rbegin();
    bad += common != pop::meet(r[0], r[1]);
  }
  for (int round = 0; round < 5000; ++round) {
    pop::Regions few;
    pop::ManyRegions<12> many;
    int64_t n[4], s[4];
    for (int i = 0; i < 10; ++i) {
      layout(n, s);
      const int64_t inner = in(1, 4);
      const void* at = (void*)(5000 + in(0, 6000));
      const bool written = rng() % 2;
      few.add("", at, inner, 4, n, s, written);
      many.add("", at, inner, 4, n, s, written);
    }
    const char *one, *other;
    const bool clash = few.clash(one, other);
    clashes += clash;
    bad += clash != many.clash(one, other);
  }
  std::printf("met %d, near %d, clashes %d, bad %d\n", met, near, clashes, bad);
  return bad != 0 || met < 1000 || near < 1000 || clashes < 500 || clashes > 4500;
}
