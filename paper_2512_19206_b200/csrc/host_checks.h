// Argument checks that the calls of the paged cache and of the partial rotation share (host code).
#pragma once

#include "paged.cuh"

namespace mixkvq {

namespace {

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline bool aligned16(const void* p) { return aligned(p, 16); }

// The memory that a call reads and writes.  Nothing may lie over what it writes.
struct Ranges {
  struct One { uintptr_t lo, hi; bool written; } all[16];
  int n = 0;
  void add(const void* p, size_t bytes, bool written) {
    if (p != nullptr && bytes != 0) all[n++] = {reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes, written};
  }
  void read(const void* p, size_t bytes) { add(p, bytes, false); }
  void write(const void* p, size_t bytes) { add(p, bytes, true); }
  bool clash() const {
    for (int i = 0; i < n; ++i) {
      if (!all[i].written) continue;
      for (int j = 0; j < n; ++j)
        if (i != j && all[i].lo < all[j].hi && all[j].lo < all[i].hi) return true;
    }
    return false;
  }
  // whether anything but the range itself lies over it
  bool touches(const void* p, size_t bytes) const {
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p), hi = lo + bytes;
    for (int i = 0; i < n; ++i)
      if (!(all[i].lo == lo && all[i].hi == hi) && lo < all[i].hi && all[i].lo < hi) return true;
    return false;
  }
};

inline RopeTensor head_major(int H, int n) { return {(long long)H * n * kD, (long long)n * kD, kD}; }

// Whether rows at p with strides t are the head-major rows at `out`: an output over its own input.
inline bool same_rows(const void* p, const RopeTensor& t, const void* out, int B, int H, int n) {
  const RopeTensor w = head_major(H, n);
  return p == out && (B == 1 || t.batch == w.batch) && (H == 1 || t.head == w.head) && (n == 1 || t.token == w.token);
}

// Rows [B, H, n, 128] of 16-bit numbers with strides t (null: none).  in_place: the call writes these very rows.
inline int check_strided(const void* p, const RopeTensor& t, int B, int H, int n, Ranges* r, bool in_place) {
  if (p == nullptr) return MIXKVQ_OK;
  if (!aligned16(p)) return MIXKVQ_E_ALIGNMENT;
  if (t.batch < 0 || t.head < 0 || t.token < 0) return MIXKVQ_E_INVALID_ARG;
  if ((t.batch | t.head | t.token) & 7) return MIXKVQ_E_ALIGNMENT;
  if (!in_place) r->read(p, 2 * ((size_t)(B - 1) * t.batch + (size_t)(H - 1) * t.head + (size_t)(n - 1) * t.token + kD));
  return MIXKVQ_OK;
}

// positions_optional: without them a token turns by its place in its sequence.
inline int check_rotation(const mixkvq_rotation* t, int B, int n, bool positions_optional, RopeTurn* turn, Ranges* r) {
  if (!t || !t->cos_dev || !t->sin_dev || t->n_positions < 1 || (t->interleaved != 0 && t->interleaved != 1) || (!t->positions_dev && !positions_optional))
    return MIXKVQ_E_INVALID_ARG;
  if (t->rotary_dim < 16 || t->rotary_dim > kD || t->rotary_dim % 16) return MIXKVQ_E_UNSUPPORTED;
  if (!aligned16(t->cos_dev) || !aligned16(t->sin_dev) || !aligned(t->positions_dev, 4)) return MIXKVQ_E_ALIGNMENT;
  const size_t table = (size_t)t->n_positions * t->rotary_dim * 2;
  r->read(t->cos_dev, table);
  r->read(t->sin_dev, table);
  r->read(t->positions_dev, (size_t)B * n * 4);
  *turn = RopeTurn{t->cos_dev, t->sin_dev, t->positions_dev, t->n_positions, t->rotary_dim, t->interleaved};
  return MIXKVQ_OK;
}

}  // namespace

}  // namespace mixkvq
