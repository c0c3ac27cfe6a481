// What a rule makes of the attention over a cache of several sequences: which keys a row sees, and what becomes of a score.
// The row of key p sees the first `open` keys of its sequence, and those of [lo, p] with lo = max(first[row], p - window + 1). A
// score s = scale q.k becomes cap tanh(s / cap), less slope |p - key|.
#pragma once
#include "spd_cachefn.h"

namespace spd {
namespace {

// Parts of a rule that a kernel is made for: keys unseen (all rules), capped scores, scores lowered with the distance; caps low
// enough for one offset of the exponents, kFixed. The nearest key that a row sees has a distance of 0 (RowRule), and so the largest of
// its exponents lies in [-top, top]. With top of at most kFixedTop no running maximum is needed: probabilities, 2^-64 to 2^96, have sums
// over 2^20 keys below 2^116, and of keys that the distance lowers below fp32's range none counts beside 2^-64. (Slopes below 0 may raise
// others past top: a piece whose sum reaches kMostSum, behind which its reciprocal is no normal number, is made again by
// plain_query, with its own maximum.) A slope of kSteepest leaves nothing of any key but the nearest, 2^(2 top - 512) of it,
// and so steeper ones are taken as it: in sums of their multiples the nearest key's exponent would be lost.
enum { RULE_KEYS = 1, RULE_CAP = 2, RULE_SLOPES = 4, RULE_FIXED = 8 };
constexpr float kFixed = -16.0f, kFixedTop = 80.0f, kMostSum = 0x1p126f, kSteepest = 512.0f;

// Without a cap the offset starts at the maximum of the first tile, but not below this: a row's nearest key decides, and the offsets that
// keys far from it would set would take the bits of its score. Rows whose sum stays below kLeastSum are computed again (plain_query).
constexpr float kLeastOffset = -64.0f, kLeastSum = 0x1p-60f;

constexpr int kTanhTerms = 7, kNearTerms = 5;  // of fp32 queries; 4 and 3 of bf16 ones

struct RuleArgs {
  float cap;
  int window;
  const float* slopes;
  const int *first, *open;
  // Of products S up to `limit`, top tanh(S / (top to)) = S (c[0] + y (c[1] + ...)), y = S^2, in units of log2 (scaled_polys); up to
  // `near` the fewer of n are enough. limit 0: the exponential formula alone; below 0: neither
  float limit, c[kTanhTerms], near, n[kNearTerms];
};

// Keys below `open` and keys of [lo, lim).
struct Sight {
  int lo, lim, open;
};

// Of a row that stands for key p; before the first key it sees nothing.
__device__ __forceinline__ Sight sight_of(const RuleArgs& R, int row, int p, int open) {
  if (p < 0) return Sight{0, 0, 0};
  int lo = R.first != nullptr ? max(R.first[row], 0) : 0;
  if (R.window > 0) lo = max(lo, p - R.window + 1);
  return Sight{min(lo, p + 1), p + 1, open};
}

__device__ __forceinline__ int open_of(const RuleArgs& R, int i, int len) {
  return R.open != nullptr ? min(max(R.open[i], 0), max(len, 0)) : 0;
}

// What some row of `rows` sees: of [lo, lim), and below open. key(r), open(r): of row row0 + r; `open` where all have one.
template <typename K, typename O>
__device__ __forceinline__ Sight sight_of_rows(const RuleArgs& R, int row0, int rows, K key, O open) {
  Sight h{0x7fffffff, 0, 0};
#pragma unroll 16
  for (int r = 0; r < rows; r++) {
    const Sight s = sight_of(R, row0 + r, key(r), open(r));
    h.open = max(h.open, s.open);
    if (s.lo >= s.lim) continue;
    h.lo = min(h.lo, s.lo);
    h.lim = max(h.lim, s.lim);
  }
  return h;
}
// The same for rows of consecutive keys, the first of which is `key`.
__device__ __forceinline__ Sight sight_of_run(const RuleArgs& R, int row0, int rows, int key, int open) {
  if (R.first != nullptr) {  // four rows a load, all of a tile on the way at once
    Sight h{0x7fffffff, 0, 0};
    auto join = [&](int first, int p) {
      const int lo = max(first, R.window > 0 ? max(p - R.window + 1, 0) : 0);
      const bool any = p >= 0 && lo <= p;
      h.lo = any ? min(h.lo, lo) : h.lo;
      h.lim = any ? p + 1 : h.lim;
    };
    int r = 0;
#pragma unroll 8
    for (; r + 4 <= rows; r += 4) {
      int v[4];
      __builtin_memcpy(v, R.first + row0 + r, sizeof(v));
      for (int i = 0; i < 4; i++) join(v[i], key + r + i);
    }
    for (; r < rows; r++) join(R.first[row0 + r], key + r);
    if (key + rows > 0) h.open = open;
    return h;
  }
  const int from = max(key, 0);  // the first row that sees anything
  if (key + rows <= from) return Sight{0, 0, 0};
  return Sight{R.window > 0 ? max(from - R.window + 1, 0) : 0, key + rows, open};
}

// The keys [a, b) without those that no row sees: keys before `a` or behind `b` are dropped, and a run of them between the open keys
// and the others is a gap. Keys are counted without it: c stands for key c, from gap_at on for key c + gap. gap_at lies whole tiles
// (of `tile` keys) behind the page of a, and gap is whole pages, so that no tile has keys of both sides.
struct Keys {
  int a, b, gap_at, gap;
};
__device__ __forceinline__ Keys keys_of(int a, int b, const Sight& h, int tile) {
  Keys k{a, b, 0x7fffffff, 0};
  const int open = min(b, h.open), lo = max(a, h.lo), lim = min(b, h.lim);
  if (lim <= lo) {
    k.b = max(a, open);
  } else if (open <= a) {
    k.a = lo;
    k.b = lim;
  } else {
    const int start = a & ~(kPage - 1), at = start + (open - start + tile - 1) / tile * tile, to = lo & ~(kPage - 1);
    k.b = max(open, lim);
    if (to > at) {
      k.gap_at = at;
      k.gap = to - at;
      k.b -= k.gap;
    }
  }
  return k;
}

// tanh(x), as spd_ruleattn.hip computes it.
template <int RL>
__device__ float tanh_of(float x);
// 1 / x, within a unit in the last place
template <int RL>
__device__ float reciprocal(float x);

// A row's part of a rule, of one head. In units of log2: a score s becomes top tanh(s to_x) - slope |center - key|. The distance
// is measured from the nearest key that the row sees (its own one, or the last open one): the softmax is the same, and rows that
// see far keys alone keep their scores' bits. RL 0: the keys below lim.
template <int RL>
struct RowRule {
  int lo, lim, open, center;
  float top, to_x, slope;
  __device__ __forceinline__ bool sees(int key) const { return key < open || (key >= lo && key < lim); }
  // some key of [a, b)
  __device__ __forceinline__ bool sees_any(int a, int b) const { return (b > a && a < open) || max(a, lo) < min(b, lim); }
  // to: from s to units of log2; distance: center - key
  __device__ __forceinline__ float shaped(float s, float to, float distance) const {
    float e = s * to;
    if constexpr ((RL & RULE_CAP) != 0) e = top * tanh_of<RL>(e * to_x);
    if constexpr ((RL & RULE_SLOPES) != 0) e = fmaf(-slope, fabsf(distance), e);
    return e;
  }
};
template <>
struct RowRule<0> {
  int lim;
  __device__ __forceinline__ bool sees(int key) const { return key < lim; }
  __device__ __forceinline__ bool sees_any(int a, int) const { return lim > a; }
};

}  // namespace
}  // namespace spd
