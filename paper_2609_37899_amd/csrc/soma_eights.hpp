// soma_eights.hpp -- rows of any width in groups of eight elements, i = 8 b .. 8 b + 7 of
// the array as if its rows lay side by side: which of them a row has, what of each is the
// row's own, and which may be read at once.  Arithmetic alone, for kernels and host.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace soma {

// Groups that a row may touch.
constexpr int64_t groups_of(int64_t width) { return width % 8 == 0 ? width / 8 : (width + 14) / 8; }

// Group `index` of a row: its number in the array, the column of its first element (before
// the row's first, if that is negative), and the elements lo to hi - 1 of it that are the
// row's; none if hi <= lo.
struct Eight {
  int64_t block, col;
  int lo, hi;
  constexpr Eight(int64_t row, int64_t width, int64_t index)
      : block((row * width >> 3) + index),
        col(block * 8 - row * width),
        lo(static_cast<int>(col < 0 ? -col : 0)),
        hi(static_cast<int>(width - col < 8 ? width - col : 8)) {}
};

// The same for lane `lane` and its group k, where kLanes lanes share a row of fewer than
// 2^31 elements.  kRagged: the width is no multiple of 8, and groups lie across the rows'
// ends.
template <int kLanes, bool kRagged>
struct Group {
  int64_t block;
  int col, lo, hi;
  constexpr Group(int row, int width, int lane, int k)
      : block((static_cast<int64_t>(row) * width >> 3) + lane + kLanes * k), col(0), lo(0), hi(0) {
    const int64_t c = block * 8 - static_cast<int64_t>(row) * width;
    col = static_cast<int>(c < width ? c : width);
    lo = kRagged && col < 0 ? -col : 0;
    hi = kRagged ? (width - col < 8 ? width - col : 8) : col < width ? 8 : 0;     // <= lo: nothing
  }
};

// Whether groups of eight may be read at once in rows of this stride, from an address that
// is aligned if `aligned`: all of them are then, and those of a row that another follows
// lie inside the array: they reach at most 7 elements past their row's end, and the next
// row's end is `stride` elements behind it.
constexpr bool in_eights(bool aligned, int64_t stride, int64_t width, size_t element) {
  return aligned && stride >= 7 && (stride - width) * static_cast<int64_t>(element) % 16 == 0;
}

// Whether a group is read at once, what is around its row's own elements too; `last`: no
// row follows, so that what lies behind this one's end is not the array's.
constexpr bool reads_whole(bool vec, bool last, int lo, int hi) { return vec && (!last || (lo == 0 && hi == 8)); }

}  // namespace soma
