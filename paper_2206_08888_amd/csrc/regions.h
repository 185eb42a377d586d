// Whether the arrays of a call share memory (host only): what the checks of op_api.hip ask of outputs and what lies around them.
#pragma once
#include <stdint.h>

namespace pop {

// Up to three axes of n[i] blocks, stride[i] bytes apart, of `inner` adjacent bytes each.
struct Region {
  const char* name;
  uintptr_t at;
  int64_t inner, n[3], stride[3];
  bool written;
  int same;                          // written over an input of the same nonzero `same` where the two coincide: allowed
  __int128 lo, hi;                   // bytes in front of and behind `at`
};

inline Region region(const char* name, const void* at, int64_t inner, bool written, int same = 0) {
  Region r = {name, (uintptr_t)at, inner, {1, 1, 1}, {0, 0, 0}, written, same, 0, inner};
  return r;
}
inline Region region(const char* name, const void* at, int64_t inner, int axes, const int64_t* n, const int64_t* stride, bool written, int same = 0) {
  Region r = region(name, at, inner, written, same);
  for (int i = 0; i < axes; ++i) {
    if (n[i] < 2) continue;          // its stride counts for nothing
    r.n[i] = n[i];
    r.stride[i] = stride[i];
    (stride[i] < 0 ? r.lo : r.hi) += (__int128)stride[i] * (n[i] - 1);
  }
  return r;
}

// Whether two regions have a byte in common.  Arrays that reach into each other may still keep apart (the halves of wider
// rows): then sum_k s_k x_k + r = b.at - a.at is looked for, the difference of an element of a and one of b, with s_k the
// distinct strides, largest first, and x_k, r within their ranges.  Strides of arrays nest, so that two or three values of each
// x_k come into question; if after kMost of them nothing is found, the arrays are taken to be apart.
class Meeting {
 public:
  Meeting(const Region& a, const Region& b) {
    difference_ = (__int128)b.at - (__int128)a.at;
    for (int i = 0; i < 3; ++i) {
      add(a.stride[i], a.n[i] - 1);
      add(-(__int128)b.stride[i], b.n[i] - 1);
    }
    for (int i = 1; i < count_; ++i)
      for (int k = i; k > 0 && term_[k].stride > term_[k - 1].stride; --k) { const Term t = term_[k]; term_[k] = term_[k - 1]; term_[k - 1] = t; }
    lo_[count_] = -((__int128)b.inner - 1);
    hi_[count_] = (__int128)a.inner - 1;
    for (int k = count_ - 1; k >= 0; --k) {
      lo_[k] = lo_[k + 1] + term_[k].stride * term_[k].lo;
      hi_[k] = hi_[k + 1] + term_[k].stride * term_[k].hi;
    }
  }
  bool found() { return find(0, difference_); }

 private:
  struct Term { __int128 stride, lo, hi; };
  static constexpr int kMost = 4096;
  void add(__int128 stride, int64_t most) {
    if (stride == 0 || most == 0) return;
    __int128 lo = 0, hi = most;
    if (stride < 0) { stride = -stride; lo = -hi; hi = 0; }
    int k = 0;
    while (k < count_ && term_[k].stride != stride) ++k;
    if (k == count_) term_[count_++] = {stride, 0, 0};
    term_[k].lo += lo;
    term_[k].hi += hi;
  }
  static __int128 floor_of(__int128 a, __int128 b) { return a >= 0 ? a / b : -((-a + b - 1) / b); }        // b > 0
  bool find(int k, __int128 d) {
    if (d < lo_[k] || d > hi_[k]) return false;
    if (k == count_) return true;
    const Term& t = term_[k];
    __int128 first = -floor_of(hi_[k + 1] - d, t.stride), last = floor_of(d - lo_[k + 1], t.stride);
    if (first < t.lo) first = t.lo;
    if (last > t.hi) last = t.hi;
    for (__int128 x = first; x <= last && looked_ < kMost; ++x) {
      ++looked_;
      if (find(k + 1, d - x * t.stride)) return true;
    }
    return false;
  }
  Term term_[6];
  __int128 lo_[7], hi_[7], difference_;
  int count_ = 0, looked_ = 0;
};

inline bool coincide(const Region& a, const Region& b) {
  bool same = a.at == b.at && a.inner == b.inner;
  for (int i = 0; i < 3; ++i) same = same && a.n[i] == b.n[i] && a.stride[i] == b.stride[i];
  return same;
}
inline bool meet(const Region& a, const Region& b) {
  if ((__int128)a.at + a.hi <= (__int128)b.at + b.lo || (__int128)b.at + b.hi <= (__int128)a.at + a.lo) return false;
  return Meeting(a, b).found();
}

// The arrays of a call; NULL ones and those without a byte are left out.
class Regions {
 public:
  template <typename... A> void add(const char* name, const void* at, int64_t inner, A... rest) {
    if (at && inner > 0) region_[count_++] = region(name, at, inner, rest...);
  }
  // The first two that must not meet and do.
  bool clash(const char*& one, const char*& other) const {
    for (int i = 0; i < count_; ++i)
      for (int k = 0; k < i; ++k) {
        const Region &a = region_[i], &b = region_[k];
        if ((!a.written && !b.written) || !meet(a, b) || (a.same && a.same == b.same && coincide(a, b))) continue;
        one = b.name;
        other = a.name;
        return true;
      }
    return false;
  }

 private:
  Region region_[32];                // three arrays of eight layers, hyperparameters, workspace
  int count_ = 0;
};

}  // namespace pop
