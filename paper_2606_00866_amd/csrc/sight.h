// Attention that is told more of its scores and of what a token sees:
//
//   s_ij = scale * q_i . k_j
//   s_ij <- cap * tanh(s_ij / cap)                              (capped)
//   s_ij <- s_ij - slope_h * |i - j|                            (a bias by distance)
//   j is seen by i where  max(first_i, i + 1 - window, 0) <= j < min(end_i, length)
//
// with i, j positions in the program and end_i = i + 1 unless given.  Documents,
// prefixes, spans that see each other and windows are such ranges, so every row's keys
// are an interval: a tile reads the union of its rows' intervals, and only steps that
// some row sees in part are masked.
//
// Items.  As in attend.h, but a tile's keys are those its rows see, so a window over a
// long context gives as many items as the window has work for.  Batches whose sequences
// are one tile each (decode steps) find that from the lengths and ranges themselves: every
// workgroup reads those of all tokens, which are few.  A step of 64 sequences takes 60 us
// with documents and 59 without, of 400 281 and 271, of 400 of four tokens 368 and 297, of
// 1000 921 and 787 (8 key heads of 128, 700 to 1000 keys each).  The others have their tiles
// and items written down by a small kernel first (attend_sight.hip).
//
// tanh.  cap * tanh(x) = cap - 2 cap / (e^2x + 1): an exponential, a reciprocal and three
// more instructions, with an error of 2^-22 of the cap.  For caps up to 64 that is 2^-16
// of a score's unit.  Above, scores below the cap take x P(x^2) instead, P of six terms
// with a relative error of 7e-7 (a minimax fit on [0, 1]), so they keep their relative
// accuracy whatever the cap.  (The polynomial alone, where all of a step's scores are
// small, is no faster: prompts of 20600 tokens 1656 us, 1592 with the other form.)
//
// Reference.  Scores are taken relative to where the maximum was last followed in the
// instruction that finishes them, so neither caps nor biases cost another one for it; a
// row that has seen nothing yet has the reference 0.
#pragma once
#include "attend.h"

namespace mori {

struct SightArgs : AttendArgs {
  float cap, cap_in;   // log2(e) * cap; |scale| / cap.  0: none
  float cap_exp;       // 2 log2(e) * cap_in
  float p[6];          // cap * P's coefficients
  uint32_t exact;      // the cap is above 64
  const float* slopes;
  uint32_t window;     // 0: none
  const int32_t *first, *end;
  // tiles as written down (no array: a sequence is a tile)
  uint32_t tiles;      // bound on their number
  uint32_t align;      // a tile's keys are taken from a multiple of this power of two on
  uint32_t unit_log;
  struct SightTile* tile;  // [tiles]
  uint32_t* list;      // [items] an item's tile; no array: it is the item itself
  uint32_t* split;     // whether any tile has several runs
};
constexpr uint32_t NO_TILE = 0xFFFFFFFFu;

// What a kernel knows of a sight when it is compiled.
constexpr int CAPPED = 1, BIASED = 2, UNKNOWN = 4;
template <int F>
struct Sight : SightArgs {
  static constexpr int FORM = F;
};

// A tile of rows, 48 bytes.
struct SightTile {
  uint32_t lo, hi, from, open;    // keys that its rows see together, and all of them
  uint32_t t0, n, len, tbl;       // of its sequence (Seq)
  uint32_t row0, first, runs;     // its first row, its first item and their number (0: no tile)
  uint32_t run_units;
};

// Keys of token i of a sequence.
__device__ inline Keys token_keys(const SightArgs& a, const Seq& s, uint32_t i) {
  const int32_t pos = s.position(i);
  if (pos < 0) return {0, 0};
  int32_t lo = a.window && (uint32_t)pos >= a.window ? pos + 1 - (int32_t)a.window : 0, hi = pos + 1;
  if (a.first) lo = max(lo, a.first[s.t0 + i]);
  if (a.end) hi = min(a.end[s.t0 + i], (int32_t)s.len);
  if (hi <= lo) return {0, 0};
  return {(uint32_t)lo, (uint32_t)hi};
}
__device__ inline Keys row_keys(const SightArgs& a, const Work& w, uint32_t r) {
  if (r >= w.rows) return {0, 0};
  return token_keys(a, w.s, divide(w.row0 + r, a.by_group));
}

// A sequence as one tile, for the scan over the sequences.  More rows than a tile has
// only where it brings more tokens than it may: padding.
__device__ inline Share share_of(const SightArgs& a, uint32_t b) {
  Share s{0, 1, 0, false};
  Seq q{};
  q.t0 = a.b.seq_off[b];
  const uint32_t end = a.b.seq_off[b + 1];
  q.len = a.b.kv_len[b];
  s.bad = q.t0 > end || end > a.b.T;
  if (s.bad) return s;
  s.n = q.n = end - q.t0;
  if (!q.n) return s;
  s.tiles = 1;
  if (q.n > a.b.max_new) {
    s.tiles = (s.n * a.group + a.tile_rows - 1) / a.tile_rows;
    return s;
  }
  if (q.len > a.b.max_kv) return s;
  uint32_t lo = 0xFFFFFFFFu, hi = 0;
  if (!a.first && !a.end) {  // the first token's and the last one's
    lo = token_keys(a, q, q.len < q.n ? q.n - q.len : 0).lo;
    hi = q.len;
  } else {
    for (uint32_t i = 0; i < q.n; ++i) {
      const Keys k = token_keys(a, q, i);
      if (k.none()) continue;
      lo = min(lo, k.lo);
      hi = max(hi, k.hi);
    }
  }
  if (hi > lo) s.units = (hi - lo + a.unit - 1) >> a.unit_log;
  return s;
}

struct Max {
  __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return max(a, b); }
};
__device__ inline uint32_t wave_max(uint32_t v) { return wave::lane63(wave::incl(v, Max())); }
__device__ inline uint32_t wave_min(uint32_t v) { return ~wave_max(~v); }

// What the rows of some tokens see together, and what all of them see.
struct Union {
  uint32_t lo, hi, from, open;
};
__device__ inline Union union_of(const SightArgs& a, const Seq& s, uint32_t i0, uint32_t i1, uint32_t lane) {
  if (i1 - i0 == 1) {
    const Keys k = token_keys(a, s, i0);
    if (k.none()) return Union{0, 0, 0xFFFFFFFFu, 0};
    return Union{k.lo, k.hi, k.lo, k.hi};
  }
  uint32_t lo = 0xFFFFFFFFu, hi = 0, from = 0, open = 0xFFFFFFFFu;
  for (uint32_t i = i0 + lane; i < i1; i += 64) {
    const Keys k = token_keys(a, s, i);
    if (k.none()) {  // sees nothing: nothing is open to all
      from = 0xFFFFFFFFu;
      open = 0;
      continue;
    }
    lo = min(lo, k.lo);
    hi = max(hi, k.hi);
    from = max(from, k.lo);
    open = min(open, k.hi);
  }
  Union u{wave_min(lo), wave_max(hi), wave_max(from), wave_min(open)};
  if (u.lo >= u.hi) u.lo = u.hi = 0;
  return u;
}

__device__ inline void set_run(const SightArgs& a, Work& w, const Union& u, uint32_t run, uint32_t run_units) {
  const uint32_t start = u.lo & ~(a.align - 1);
  const uint64_t lo = start + (uint64_t)run * run_units * a.unit, hi = lo + (uint64_t)run_units * a.unit;
  w.key0 = same(u.lo);
  w.from = same(u.from);
  w.open = same(u.open);
  w.lo = same((uint32_t)min(lo, (uint64_t)0x7FFFFFFFu));
  w.hi = same((uint32_t)min(hi, (uint64_t)u.hi));
}

// The item of a batch whose sequences are one tile each.
__device__ inline Work work_of(const SightArgs& a, uint32_t block, uint32_t lane) {
  Work w{};
  w.item = divide(block, a.by_kv);
  w.kv = block - w.item * a.kv_heads;
  const uint32_t item = w.item;
  // batches of up to 64: every lane has its sequence's numbers on the way while the item is found
  const bool few = a.b.B <= 64;
  SeqNumbers x{};
  if (few && lane < a.b.B) x = read_sequence(a.b, lane);
  const Item it = find_item(a, lane, [&](uint32_t first, uint32_t n, uint32_t) { return item - first < n; });
  w.some = it.found;
  if (block == 0 && it.bad) report(a.b, MORI_DEV_BAD_TOKENS);
  if (!w.some) return w;
  if (few) {
    const auto of = [&](uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)v, (int)it.b); };
    x = SeqNumbers{of(x.lo), of(x.hi), of(x.len), of(x.p), of(x.first), of(x.last)};
  } else {
    x = read_sequence(a.b, it.b);
    x = SeqNumbers{same(x.lo), same(x.hi), same(x.len), same(x.p), same(x.first), same(x.last)};
  }
  w.s = checked_sequence(a.b, x);
  uint32_t run = w.item - it.first;
  if (w.s.n > a.b.max_new) {
    const uint32_t back = run / it.per_tile, tiles = (w.s.n * a.group + a.tile_rows - 1) / a.tile_rows;
    run -= back * it.per_tile;
    w.row0 = same((tiles - 1 - back) * a.tile_rows);
  }
  w.per_tile = it.per_tile;
  w.rows = min(a.tile_rows, w.s.n * a.group - w.row0);
  Union u{0, 0, 0, 0};
  if (!w.s.error) u = union_of(a, w.s, 0, w.s.n, lane);
  set_run(a, w, u, run, it.run_units);
  return w;
}

// The item of a batch whose tiles are written down.
__device__ inline Work tile_work(const SightArgs& a, uint32_t block) {
  Work w{};
  w.item = divide(block, a.by_kv);
  w.kv = block - w.item * a.kv_heads;
  const uint32_t tile = a.list ? same(a.list[w.item]) : w.item;
  if (tile >= a.tiles) return w;
  const uint4* const at = reinterpret_cast<const uint4*>(a.tile + tile);
  const uint4 x = at[0], y = at[1], z = at[2];
  w.per_tile = same(z.z);
  if (!w.per_tile) return w;
  w.some = true;
  w.s.t0 = same(y.x);
  w.s.n = same(y.y);
  w.s.len = same(y.z);
  w.s.tbl = same(y.w);
  w.s.named = true;
  w.row0 = same(z.x);
  w.rows = min(a.tile_rows, w.s.n * a.group - w.row0);
  set_run(a, w, Union{same(x.x), same(x.y), same(x.z), same(x.w)}, w.item - same(z.y), same(z.w));
  return w;
}

// A tile's keys are what its rows see together, so pages of which none sees a key may lie
// between.  Where reading the run's keys met pages that are not there, those that count: of
// which a row sees a key.  Rare, so no step pays for it.
__device__ inline uint32_t seen_errors(const SightArgs& a, const Work& w, uint32_t lane) {
  const uint32_t lo = max(w.lo, w.key0);
  if (lo >= w.hi) return 0;
  uint32_t err = 0;
  const uint32_t last = divide(w.hi - 1, a.b.by_bt);
  for (uint32_t b0 = divide(lo, a.b.by_bt); b0 <= last; b0 += 64) {
    uint32_t mine = 0;
    if (b0 + lane <= last) checked_page(a.b, a.b.tbl[w.s.tbl + b0 + lane], &mine);
    for (uint64_t bad = __ballot(mine != 0); bad; bad &= bad - 1) {
      const int at = __ffsll((unsigned long long)bad) - 1;
      const uint32_t bit = (uint32_t)__builtin_amdgcn_readlane((int)mine, at);
      if (err & bit) continue;
      const uint32_t k0 = (b0 + at) * a.b.bt, first = max(k0, lo), end = w.hi - k0 < a.b.bt ? w.hi : k0 + a.b.bt;
      bool sees = false;
      for (uint32_t r = lane; r < w.rows; r += 64) {
        const Keys k = row_keys(a, w, r);
        sees |= max(k.lo, first) < min(k.hi, end);
      }
      if (__any(sees)) err |= bit;
    }
  }
  return err;
}

// cap * tanh(scale * s / cap) - ref from a product s, with an error of 2^-22 of the cap
// and with one of 2^-20 of the score.
__device__ inline float capped_any(const SightArgs& a, float s, float ref) {
  const float r = __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(s * a.cap_exp) + 1.f);
  return __builtin_fmaf(-2.f * a.cap, r, a.cap - ref);
}
__device__ inline float capped_exact(const SightArgs& a, float s, float ref) {
  const float x = s * a.cap_in, u = x * x;
  float p = __builtin_fmaf(u, a.p[5], a.p[4]);
#pragma unroll
  for (int k = 3; k >= 0; --k) p = __builtin_fmaf(u, p, a.p[k]);
  return fabsf(x) < 1.f ? __builtin_fmaf(x, p, -ref) : capped_any(a, s, ref);
}

// Scores of one row (or, lane by lane, of several) in the softmax's units and less `ref`,
// from the products of queries and keys; key(i) is what the i-th one's key is ahead of
// `base`, which counts from the row's position.
// On one side of the rows' positions a bias is a straight line, and a constant for each
// key and one for the step take the place of the distance.
template <int FORM, int N, typename K>
__device__ __forceinline__ void shape_scores(const SightArgs& a, float (&y)[N], float ref, float slope, int32_t base,
                                             K key) {
  const bool biased = FORM == UNKNOWN ? a.slopes != nullptr : FORM & BIASED;
  if (FORM == UNKNOWN ? a.cap != 0 : FORM & CAPPED) {
    if (!a.exact) {
#pragma unroll
      for (int i = 0; i < N; ++i) y[i] = capped_any(a, y[i], ref);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) y[i] = capped_exact(a, y[i], ref);
    }
  } else {
    if (FORM == BIASED) {
      const bool behind = __all(base <= -key(N - 1)), ahead = __all(base >= 0);
      if (behind || ahead) {
        const float s = behind ? slope : -slope, b = __builtin_fmaf(s, (float)base, -ref);
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] = __builtin_fmaf(y[i], a.c, __builtin_fmaf(s, (float)key(i), b));
        return;
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = __builtin_fmaf(y[i], a.c, -ref);
  }
  if (biased) {
    const float b = (float)base;
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = __builtin_fmaf(-slope, fabsf(b + (float)key(i)), y[i]);
  }
}
// The reference of a row whose maximum was last followed at `top`.
__device__ inline float ref_of(float top) { return top == NO_TOP ? 0.f : top; }
// log2(e) * slope of a head.
__device__ inline float slope_of(const SightArgs& a, uint32_t h) {
  return a.slopes ? 1.4426950408889634f * a.slopes[h] : 0.f;
}
__device__ inline auto score_of(const SightArgs& a, const Work& w, uint32_t r, uint32_t h) {
  const int32_t pos = w.s.position(divide(w.row0 + r, a.by_group));
  return [&a, slope = slope_of(a, h), pos](float s, uint32_t key) {
    float y = s * a.c;
    if (a.cap != 0) {
      y = a.exact ? capped_exact(a, s, 0.f) : capped_any(a, s, 0.f);
    }
    if (a.slopes) y = __builtin_fmaf(-slope, fabsf((float)((int32_t)key - pos)), y);
    return y;
  };
}

template <typename Args>
struct IsSight {
  static constexpr bool value = false;
  static constexpr int FORM = 0;
};
template <int F>
struct IsSight<Sight<F>> {
  static constexpr bool value = true;
  static constexpr int FORM = F;
};

// The sight in the form that says what it does.
template <typename L>
inline void with_form(const SightArgs& a, L launch) {
  const auto as = [&](auto form) {
    static_cast<SightArgs&>(form) = a;
    launch(form);
  };
  if (a.cap != 0 && a.slopes) as(Sight<CAPPED | BIASED>{});
  else if (a.cap != 0) as(Sight<CAPPED>{});
  else if (a.slopes) as(Sight<BIASED>{});
  else as(Sight<0>{});
}

}  // namespace mori
