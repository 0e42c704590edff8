// Which bytes the tensors of a call take, so that a call whose destinations share memory is refused before it races on it.
//
// A tensor is outer_n runs, outer_step bytes apart, of inner_n pieces, inner_step bytes apart, of len bytes each: heads of a
// cache (one piece a run), or heads and rows of bf16 rows in either order.  Layers may lie inside one another's strides ([head]
// [layer][row] or [token][layer][head]), so extents alone do not tell; whether two tensors meet is answered exactly.
// The usual case, extents that lie apart, is one walk over the addresses in order: no allocation, 0.1 us for 128 tensors.
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
    return !apart() && !apart_in_detail();
  }

 private:
  static constexpr int kMaxLists = 16;
  struct List {
    const void* const* at;
    int n;
    Footprint f;
    bool written;
  };
  struct Piece {
    uint64_t at;
    const List* of;
    bool operator<(const Piece& o) const { return at < o.at; }
  };
  List list_[kMaxLists];
  int lists_ = 0;

  static uint64_t addr(const void* p) { return reinterpret_cast<uintptr_t>(p); }

  // Every list rises or falls, and in the order of addresses no extent begins inside one it must not meet.
  bool apart() const {
    int next[kMaxLists], step[kMaxLists], left[kMaxLists];
    for (int i = 0; i < lists_; ++i) {
      const List& l = list_[i];
      const bool falls = addr(l.at[l.n - 1]) < addr(l.at[0]);
      step[i] = falls ? -1 : 1;
      next[i] = falls ? l.n - 1 : 0;
      left[i] = l.n;
    }
    uint64_t end = 0, end_written = 0;
    for (;;) {
      int first = -1;
      uint64_t low = UINT64_MAX, second = UINT64_MAX;
      for (int i = 0; i < lists_; ++i) {
        if (!left[i]) continue;
        const uint64_t a = addr(list_[i].at[next[i]]);
        if (first < 0 || a < low) {
          second = low;
          low = a;
          first = i;
        } else {
          second = std::min(second, a);
        }
      }
      if (first < 0) return true;
      const List& l = list_[first];
      const uint64_t span = (uint64_t)l.f.span();
      for (uint64_t a = low; a <= second;) {  // (this list up to the next one's first)
        if (a < (l.written ? end : end_written)) return false;
        end = std::max(end, a + span);
        if (l.written) end_written = std::max(end_written, a + span);
        next[first] += step[first];
        if (--left[first] == 0) break;
        const uint64_t b = addr(l.at[next[first]]);
        if (b < a) return false;  // not in order
        a = b;
      }
    }
  }

  // The same with every tensor looked at: those whose extents meet, in groups, by how they interleave, else pair by pair.
  bool apart_in_detail() const {
    int n = 0;
    for (int i = 0; i < lists_; ++i) n += list_[i].n;
    std::unique_ptr<Piece[]> p(new (std::nothrow) Piece[n]);
    if (!p) return false;
    int k = 0;
    for (int i = 0; i < lists_; ++i)
      for (int j = 0; j < list_[i].n; ++j) p[k++] = Piece{addr(list_[i].at[j]), &list_[i]};
    std::sort(p.get(), p.get() + n);
    for (int i0 = 0, i1; i0 < n; i0 = i1) {
      uint64_t end = 0;
      for (i1 = i0; i1 < n && (i1 == i0 || p[i1].at < end); ++i1)
        end = std::max(end, p[i1].at + (uint64_t)p[i1].of->f.span());
      if (i1 - i0 == 1 || interleaved(&p[i0], i1 - i0, true) || interleaved(&p[i0], i1 - i0, false)) continue;
      for (int i = i0; i < i1; ++i)
        for (int j = i + 1; j < i1; ++j)
          if ((p[i].of->written || p[j].of->written) && meet(p[i], p[j])) return false;
    }
    return true;
  }

  // All of one period (the outer step, or the inner one as well), with their runs (pieces) one after another inside it.
  static bool interleaved(const Piece* p, int n, bool runs) {
    const Footprint& f = p[0].of->f;
    const int64_t period = runs ? f.outer_step : f.inner_step;
    for (int i = 0; i < n; ++i) {
      const Footprint& g = p[i].of->f;
      if (g.folds() || g.outer_n == 1 || g.outer_step != f.outer_step) return false;
      if (!runs && (g.inner_n == 1 || g.inner_step != f.inner_step || g.outer_step % g.inner_step)) return false;
      const uint64_t end = p[i].at + (uint64_t)(runs ? g.run() : g.len);
      if (end > (i + 1 < n ? p[i + 1].at : p[0].at + (uint64_t)period)) return false;
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

  static bool meet(const Piece& a, const Piece& b) {
    const Footprint &f = a.of->f, &g = b.of->f;
    const int64_t d = (int64_t)(b.at - a.at);
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
