// Which bytes the tensors of a call take, so that a call whose destinations share memory is refused before it races on it.
//
// A tensor is outer_n runs, outer_step bytes apart, of inner_n pieces, inner_step bytes apart, of len bytes each: heads of a
// cache (one piece a run), or heads and rows of bf16 rows in either order.  Layers may lie inside one another's strides ([head]
// [layer][row] or [token][layer][head]), so extents alone do not tell; whether two tensors meet is answered exactly.
// On the host 0.2 us of a call over 32 layers where these lie in one tensor, 1 to 2 where each is allocated by itself.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <memory>
#include <new>

namespace stepkv {

struct Footprint {
  int64_t outer_n, outer_step, inner_n, inner_step, len;
  int64_t run() const { return (inner_n - 1) * inner_step + len; }
  int64_t span() const { return (outer_n - 1) * outer_step + run(); }
  bool folds() const { return (inner_n > 1 && inner_step < len) || (outer_n > 1 && outer_step < run()); }  // meets itself
};

// n1 by n2 pieces of len bytes at strides s1 and s2: the larger stride outside.
inline Footprint make_footprint(int64_t n1, int64_t s1, int64_t n2, int64_t s2, int64_t len) {
  const bool swap = n1 == 1 || (n2 > 1 && s2 > s1);
  return swap ? Footprint{n2, s2, n1, s1, len} : Footprint{n1, s1, n2, s2, len};
}

class Footprints {
 public:
  // n tensors of one footprint; `at` is the caller's and outlives this object.
  void add(const void* const* at, int n, const Footprint& f, bool written) {
    if (at && n > 0 && lists_ < kMaxLists) list_[lists_++] = List{at, n, f, written};
  }

  // Whether a byte of a written tensor is a byte of another tensor too (or of itself twice), or might be.
  bool clash() const {
    for (int i = 0; i < lists_; ++i)
      if (list_[i].written && list_[i].f.folds()) return true;
    return !apart();
  }

 private:
  static constexpr int kMaxLists = 16;
  struct List {
    const void* const* at;
    int n;
    Footprint f;
    bool written;
  };
  List list_[kMaxLists];
  int lists_ = 0;

  static uint64_t addr(const void* p) { return reinterpret_cast<uintptr_t>(p); }
  // a tensor as one number: its address and its list
  static uint64_t at(uint64_t key) { return key / kMaxLists; }
  const List& of(uint64_t key) const { return list_[key % kMaxLists]; }

  // Lists whose tensors lie apart from one another and, all of them, from every list they must not meet are done with.
  // Returns how many tensors the others have.
  int mixed(bool (&done)[kMaxLists]) const {
    uint64_t low[kMaxLists], high[kMaxLists];
    for (int i = 0; i < lists_; ++i) {
      const List& l = list_[i];
      const uint64_t span = (uint64_t)l.f.span();
      uint64_t a = addr(l.at[0]);
      bool up = true, down = true;
      low[i] = high[i] = a;
      for (int j = 1; j < l.n; ++j) {
        const uint64_t b = addr(l.at[j]);
        up &= b >= a + span;
        down &= a >= b + span;
        low[i] = std::min(low[i], b);
        high[i] = std::max(high[i], b);
        a = b;
      }
      high[i] += span;
      done[i] = up || down || !l.written;
    }
    for (int i = 0; i < lists_; ++i)
      for (int j = i + 1; j < lists_; ++j)
        if ((list_[i].written || list_[j].written) && low[i] < high[j] && low[j] < high[i]) done[i] = done[j] = false;
    int n = 0;
    for (int i = 0; i < lists_; ++i) n += done[i] ? 0 : list_[i].n;
    return n;
  }

  bool apart() const {
    bool done[kMaxLists];
    const int n = mixed(done);
    if (n == 0) return true;
    constexpr int kHere = 512;
    uint64_t here[kHere];
    std::unique_ptr<uint64_t[]> heap(n > kHere ? new (std::nothrow) uint64_t[n] : nullptr);
    uint64_t* const p = n > kHere ? heap.get() : here;
    if (!p) return false;
    int k = 0;
    for (int i = 0; i < lists_; ++i)
      for (int j = 0; !done[i] && j < list_[i].n; ++j) p[k++] = addr(list_[i].at[j]) * kMaxLists + i;  // (addresses: 57 bits)
    std::sort(p, p + n);
    // tensors whose extents meet, in groups: apart by how they interleave, else pair by pair
    for (int i0 = 0, i1; i0 < n; i0 = i1) {
      uint64_t end = 0;
      for (i1 = i0; i1 < n && (i1 == i0 || at(p[i1]) < end); ++i1) end = std::max(end, at(p[i1]) + (uint64_t)of(p[i1]).f.span());
      if (i1 - i0 == 1 || interleaved(p + i0, i1 - i0, true) || interleaved(p + i0, i1 - i0, false)) continue;
      for (int i = i0; i < i1; ++i)
        for (int j = i + 1; j < i1; ++j)
          if ((of(p[i]).written || of(p[j]).written) && meet((int64_t)(at(p[j]) - at(p[i])), of(p[i]).f, of(p[j]).f)) return false;
    }
    return true;
  }

  // All of one period (the outer step, or the inner one as well), with their runs (pieces) one after another inside it.
  bool interleaved(const uint64_t* p, int n, bool runs) const {
    const Footprint& f = of(p[0]).f;
    const int64_t period = runs ? f.outer_step : f.inner_step;
    for (int i = 0; i < n; ++i) {
      const Footprint& g = of(p[i]).f;
      if (g.folds() || g.outer_n == 1 || g.outer_step != f.outer_step) return false;
      if (!runs && (g.inner_n == 1 || g.inner_step != f.inner_step || g.outer_step % g.inner_step)) return false;
      const uint64_t end = at(p[i]) + (uint64_t)(runs ? g.run() : g.len);
      if (end > (i + 1 < n ? at(p[i + 1]) : at(p[0]) + (uint64_t)period)) return false;
    }
    return true;
  }

  static int64_t floor_div(int64_t a, int64_t b) { return a / b - (a % b < 0); }

  // Whether pieces at multiples 0, +-1 .. +-(n - 1) of step, of len bytes, meet a piece d bytes from the middle one.
  static bool near_multiple(int64_t d, int64_t n, int64_t step, int64_t len) {
    if (d < 0) d = -d;
    if (n == 1) return d < len;
    const int64_t q = d / step, r = d - q * step;
    return (q < n && r < len) || (q + 1 < n && step - r < len);
  }

  // Whether a tensor of footprint g, d bytes behind one of footprint f, meets it.
  static bool meet(int64_t d, const Footprint& f, const Footprint& g) {
    const bool alike = f.outer_n == g.outer_n && f.inner_n == g.inner_n && f.len == g.len &&
                       (f.outer_n == 1 || f.outer_step == g.outer_step) && (f.inner_n == 1 || f.inner_step == g.inner_step);
    if (alike && !f.folds()) {  // translates: a run of one can only meet the two of the other that lie next to it
      if (f.outer_n == 1) return near_multiple(d, f.inner_n, f.inner_step, f.len);
      const int64_t q = floor_div(d, f.outer_step), r = d - q * f.outer_step;
      return (q < f.outer_n && q > -f.outer_n && near_multiple(r, f.inner_n, f.inner_step, f.len)) ||
             (q + 1 < f.outer_n && q + 1 > -f.outer_n && near_multiple(r - f.outer_step, f.inner_n, f.inner_step, f.len));
    }
    // runs of the one against runs of the other, each run as a whole
    for (int64_t i = 0; i < f.outer_n; ++i) {
      const int64_t e = d - i * f.outer_step;  // j runs: -g.run() < e + j step < f.run()
      if (g.outer_n == 1 || g.outer_step == 0) {
        if (e > -g.run() && e < f.run()) return true;
        continue;
      }
      const int64_t lo = std::max<int64_t>(0, floor_div(-g.run() - e, g.outer_step) + 1);
      const int64_t hi = std::min<int64_t>(g.outer_n - 1, floor_div(f.run() - 1 - e, g.outer_step));
      if (lo <= hi) return true;
    }
    return false;
  }
};

}  // namespace stepkv
