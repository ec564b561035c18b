// Checks of arguments that the translation units of the C ABI share (not installed).
#pragma once

#include <stdint.h>

#include <algorithm>
#include <utility>

#include "dsp_internal.h"

namespace dsp {
namespace {

inline bool valid_dtype(int dt) { return dt == DSP_F32 || dt == DSP_BF16; }
inline int elem_size(int dt) { return dt == DSP_F32 ? 4 : 2; }
inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }

inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
  return na && nb && pa < pb + nb && pb < pa + na;
}

inline bool mul_ok(int64_t a, int64_t b, int64_t* out) {
  if (a < 0 || b < 0) return false;
  if (a != 0 && b > INT64_MAX / a) return false;
  *out = a * b;
  return true;
}

// Rows of a (B, X, L) grid with element strides st = {b, x, l}, each `width`
// elements wide, do not overlap when, taking the dimensions of extent > 1 by
// increasing stride, every stride is at least the span of the smaller ones.
inline bool rows_disjoint(int64_t B, int64_t X, int64_t L, const int64_t* st, int64_t width) {
  int64_t e[3] = {B, X, L}, s[3] = {st[0], st[1], st[2]};
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (s[j] < s[i]) { std::swap(s[i], s[j]); std::swap(e[i], e[j]); }
  int64_t span = width;
  for (int i = 0; i < 3; ++i) {
    if (e[i] <= 1) continue;
    if (s[i] < span) return false;
    if (!mul_ok(s[i], e[i] - 1, &span) || span > INT64_MAX - width) return false;
    span += width;
  }
  return true;
}

// offsets_ok with room to spare: sums of the terms in bytes stay below 2^63
inline bool spans_ok(int64_t B, int64_t X, int64_t L, const int64_t* st) {
  const int64_t n[3] = {B, X, L};
  for (int i = 0; i < 3; ++i) {
    int64_t t;
    if (st[i] < 0 || !mul_ok(n[i] - 1, st[i], &t) || t > (int64_t(1) << 58)) return false;
  }
  return true;
}

// Two row tensors of (B, X, La) and (B, X, Lb) rows share no element: their spans
// are apart, or they have one layout and lie in different columns of its rows (the shorter
// one's taken on to the longer one's end).
inline bool rows_apart(const void* a, const int64_t* sa, int64_t wa, int64_t La, const void* b, const int64_t* sb, int64_t wb,
                int64_t Lb, int64_t B, int64_t X, int es) {
  auto span = [&](const int64_t* st, int64_t w, int64_t L) {
    return (size_t)((B - 1) * st[0] + (X - 1) * st[1] + (L - 1) * st[2] + w) * es;
  };
  if (!wa || !wb || !La || !Lb || !overlap(a, span(sa, wa, La), b, span(sb, wb, Lb))) return true;
  const int64_t ext[3] = {B, X, std::max(La, Lb)};
  const int64_t st[3] = {sa[0], sa[1], La > 1 ? sa[2] : sb[2]}, other[3] = {sb[0], sb[1], Lb > 1 ? sb[2] : sa[2]};
  int64_t pitch = INT64_MAX;
  for (int i = 0; i < 3; ++i) {
    if (ext[i] <= 1) continue;
    if (st[i] != other[i] || st[i] == 0) return false;
    pitch = st[i] < pitch ? st[i] : pitch;
    for (int j = 0; j < 3; ++j)   // whole pitches: a larger stride starts after the smaller one's rows
      if (j != i && ext[j] > 1 && st[j] >= st[i] && st[j] / st[i] < ext[i]) return false;
  }
  const int64_t off = ((intptr_t)b - (intptr_t)a) / es;
  if (((intptr_t)b - (intptr_t)a) % es) return false;
  return off >= 0 ? off >= wa && off <= pitch - wb : -off >= wb && -off <= pitch - wa;
}
inline bool same_rows(const void* a, const int64_t* sa, const void* b, const int64_t* sb, int64_t B, int64_t X, int64_t L) {
  const int64_t ext[3] = {B, X, L};
  for (int i = 0; i < 3; ++i)
    if (ext[i] > 1 && sa[i] != sb[i]) return false;
  return a == b;
}

// A block of n bytes shares none with the rows of (B, X, L): it is apart from their span or
// lies in one of the gaps between them.  Strides that do not nest leave no gaps to rely on.
inline bool block_apart(const void* block, int64_t n, const void* rows, const int64_t* st, int64_t w, int64_t L, int64_t B,
                 int64_t X, int es) {
  if (n <= 0 || w <= 0 || L <= 0) return true;
  int64_t e[3] = {B, X, L}, s[3] = {st[0], st[1], st[2]}, span = w * es;
  for (int i = 0; i < 3; ++i) {
    for (int j = i + 1; j < 3; ++j)
      if (s[j] > s[i]) { std::swap(s[i], s[j]); std::swap(e[i], e[j]); }
    span += (e[i] - 1) * s[i] * es;
  }
  if (!overlap(block, (size_t)n, rows, (size_t)span)) return true;
  int64_t from = (intptr_t)block - (intptr_t)rows;
  for (int i = 0; i < 3; ++i) {   // from the largest stride down: which of its pieces the block starts in
    if (e[i] <= 1) continue;
    const int64_t step = s[i] * es;
    span -= (e[i] - 1) * step;    // of one piece
    if (from < 0 || step < span) return false;
    const int64_t at = std::min(from / step, e[i] - 1);
    from -= at * step;
    if (at < e[i] - 1 && from + n > step) return false;   // it reaches the next piece
    if (from >= span) return true;
  }
  return false;
}

// What a call reads or writes: rows of the (B, X, L) grid (elements of es bytes), or a block.
struct Mem {
  const void* p;
  const int64_t* st;   // rows: strides; a block: null
  int64_t w, L;        // rows: their width and number; a block: its bytes
};
inline Mem mem_block(const void* p, int64_t bytes) { return {p, nullptr, p ? bytes : 0, 0}; }
inline bool apart(const Mem& a, const Mem& b, int64_t B, int64_t X, int es) {
  if (a.st && b.st) return rows_apart(a.p, a.st, a.w, a.L, b.p, b.st, b.w, b.L, B, X, es);
  if (a.st) return block_apart(b.p, b.w, a.p, a.st, a.w, a.L, B, X, es);
  if (b.st) return block_apart(a.p, a.w, b.p, b.st, b.w, b.L, B, X, es);
  return !overlap(a.p, (size_t)a.w, b.p, (size_t)b.w);
}

}  // namespace
}  // namespace dsp
