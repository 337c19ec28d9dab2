// Whether the pieces of memory that a call reads and writes are apart: host code, for the entry points' checks of arguments.
#pragma once
#include <algorithm>
#include <cstdint>

namespace pbt {

// `count` pieces of `bytes` bytes, `stride` bytes apart (stride >= bytes where there are several); what: whose they are, for the caller's message
struct Region {
  uintptr_t at;
  int64_t bytes, stride, count;
  bool written;
  int what;
};
inline int64_t region_span(const Region& r) { return r.bytes <= 0 || r.count <= 0 ? 0 : (r.count - 1) * r.stride + r.bytes; }

// No byte of `a` is one of `b`.  Exact, but for two of different strides with thousands of pieces each, which are not looked at piece by piece where
// they mix: those count as meeting.
inline bool regions_apart(const Region& a, const Region& b) {
  const int64_t sa = region_span(a), sb = region_span(b);
  if (sa == 0 || sb == 0) return true;
  if (a.at >= b.at + (uintptr_t)sb || b.at >= a.at + (uintptr_t)sa) return true;
  if (a.count > 1 && b.count > 1 && a.stride == b.stride) {   // (the spans meet, so that some piece of one lies between two of the other or on one)
    const int64_t p = a.stride, d = (int64_t)(b.at - a.at), m = ((d % p) + p) % p;
    return m >= a.bytes && p - m >= b.bytes;
  }
  if (a.count > 1 && b.count > 1 && a.count + b.count > 8192) return false;
  // piece by piece, from the first of each that can reach the other
  int64_t i = 0, j = 0;
  if (a.count > 1 && b.at > a.at) i = std::min<int64_t>((int64_t)(b.at - a.at) / a.stride, a.count - 1);
  if (b.count > 1 && a.at > b.at) j = std::min<int64_t>((int64_t)(a.at - b.at) / b.stride, b.count - 1);
  while (i < a.count && j < b.count) {
    const uintptr_t x = a.at + (uintptr_t)(i * a.stride), y = b.at + (uintptr_t)(j * b.stride);
    const uintptr_t xe = x + (uintptr_t)a.bytes, ye = y + (uintptr_t)b.bytes;
    if (x < ye && y < xe) return false;
    if (xe <= ye) ++i;
    else ++j;
  }
  return true;
}

// A place of its own for every region: what is put in order instead of the regions.
struct RegionKey {
  uint64_t at;
  int region;
};
inline void in_order(RegionKey* k, int n) {
  const auto before = [](const RegionKey& a, const RegionKey& b) { return a.at < b.at; };
  if (!std::is_sorted(k, k + n, before)) std::sort(k, k + n, before);
}

// The first pair of regions found that meet, one of them written, to *x and *y; false: there is none.  `key`: room for n.  Regions whose spans
// meet are looked at together: where all are rows of one stride (a flat array's columns) by their places in a row, else pair by pair.
inline bool find_meeting(const Region* r, RegionKey* key, int n, int* x, int* y) {
  for (int k = 0; k < n; ++k) key[k] = RegionKey{r[k].at, k};
  in_order(key, n);
  for (int lo = 0; lo < n;) {
    const Region& first = r[key[lo].region];
    uint64_t end = first.at + (uint64_t)region_span(first);
    int hi = lo + 1;
    bool rows = first.count > 1 && first.stride > 0;
    for (; hi < n && key[hi].at < end; ++hi) {
      const Region& next = r[key[hi].region];
      end = std::max(end, next.at + (uint64_t)region_span(next));
      rows = rows && next.count > 1 && next.stride == first.stride;
    }
    if (hi - lo > 1) {
      bool clear = false;
      if (rows && hi - lo > 8) {
        // places in a row, twice around: what starts before the end of an earlier one meets it (or would, if their spans did: pairs decide then)
        const uint64_t p = (uint64_t)first.stride, base = first.at;
        for (int k = lo; k < hi; ++k) {
          const uint64_t from = key[k].at - base;
          key[k].at = from < p ? from : from % p;
        }
        in_order(key + lo, hi - lo);
        clear = true;
        uint64_t read = 0, wrote = 0;   // ends of what came before
        for (int lap = 0; lap < 2 && clear; ++lap)
          for (int k = lo; k < hi && clear; ++k) {
            const Region& it = r[key[k].region];
            if (region_span(it) == 0) continue;
            const uint64_t at = key[k].at + (lap ? p : 0);
            clear = at >= wrote && (!it.written || at >= read);
            uint64_t& e = it.written ? wrote : read;
            e = std::max(e, at + (uint64_t)it.bytes);
          }
      }
      for (int i = lo; i < hi && !clear; ++i)
        for (int j = i + 1; j < hi; ++j) {
          const Region &a = r[key[i].region], &b = r[key[j].region];
          if ((a.written || b.written) && !regions_apart(a, b)) {
            *x = a.what;
            *y = b.what;
            return true;
          }
        }
    }
    lo = hi;
  }
  return false;
}

// Heads of `width` bytes at at + i row + j head.
struct HeadView { uintptr_t at; int64_t row, head, rows, heads, width; };

// No byte of `a` is one of `b`; false too where strides are too different to tell.
inline bool heads_apart(HeadView a, HeadView b) {
  const auto span = [](const HeadView& v) { return (v.rows - 1) * v.row + (v.heads - 1) * v.head + v.width; };
  if (a.at >= b.at + (uintptr_t)span(b) || b.at >= a.at + (uintptr_t)span(a)) return true;
  if (a.rows == 1 && b.rows == 1) {
    a.row = a.head * a.heads + a.width;
    b.row = b.head * b.heads + b.width;
    a.row = b.row = std::max(a.row, b.row) * 2;
  }
  // the longer of both strides is the same, and what the shorter one spans lies within it: places within one such frame, and in the next one
  const auto frames = [](const HeadView& x, const HeadView& y) {
    if (x.row != y.row || x.row <= 0) return false;
    const Region rx{0, x.width, x.head, x.heads, true, 0};
    if (region_span(rx) > x.row || (y.heads - 1) * y.head + y.width > y.row) return false;
    const int64_t p = x.row, d = (int64_t)(y.at - x.at), m = ((d % p) + p) % p;
    // (addresses within the frame, moved up by one frame so that none is negative)
    const Region x1{(uintptr_t)p, x.width, x.head, x.heads, true, 0};
    const Region y1{(uintptr_t)(p + m), y.width, y.head, y.heads, true, 0}, y0{(uintptr_t)m, y.width, y.head, y.heads, true, 0};
    return regions_apart(x1, y1) && regions_apart(x1, y0);
  };
  if (frames(a, b)) return true;
  // heads outermost
  const auto turned = [](const HeadView& v, int64_t head) { return HeadView{v.at, v.heads > 1 ? v.head : head, v.row, v.heads, v.rows, v.width}; };
  return (a.heads > 1 || b.heads > 1) && frames(turned(a, b.head), turned(b, a.head));
}

}  // namespace pbt
