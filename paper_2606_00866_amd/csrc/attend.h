// What the attention kernels share: their arguments, the division of a batch into
// work items, and the running softmax's conventions.
//
// Rows.  The query heads that share a key head are stacked: row r of a sequence
// and a key head is token r / group, query head r % group of the group.  So a
// decode step's group fills a matrix tile where single heads would leave it
// empty, and a key is fetched once for all of them.
//
// Items.  A sequence's rows are cut into tiles of a kernel's height; each tile's
// keys into runs of the same whole number c of units, where c follows from the
// batch on the device:
//     c = max(least, ceil(sum over tiles of their units / slots)),
// so that a batch gives about `slots` items however its lengths are spread, and
// at most slots + tiles.  A kernel whose workgroup takes a whole CU runs them in
// rounds of `round` items; there a c is taken that fills one or two rounds.  No
// scheduling pass precedes the kernel: every wavefront finds its item from the
// lengths by a scan over the sequences.
// Tiles of one run write their rows; the others leave partial sums (unnormalised
// rows, their maxima and sums) that a second kernel joins in a fixed order.
//
// Softmax.  Scores are kept in units of log2(e) / scale: weights are
// exp2(score * c - top).  When the running maximum has risen more than RISE over
// where it was last followed, `top` is set LIFT below it, so weights stay at most
// 2^(LIFT + RISE) and most steps leave the accumulators alone.  The weights of the
// sums and of the products are the same numbers but for the rounding of the latter
// to the pool's type, so LIFT takes part in no result; it is there for that rounding.
// The matrix units take 16 bits.  Where they bound a kernel one such number a weight is a
// choice: with a second one for the rest, the tiles' kernel took 571 to 746 us on prompts with
// documents, 180 to 228 on capped chunks, and its error against 64 bits fell from 0.0021 to
// 0.0016, which the rounding of the results makes.  Steps with a sight take pairs.
#pragma once
#include "float16.h"
#include "tokens.h"

namespace mori {

constexpr float NO_TOP = -3.0e38f;  // below any score; finite, so that masked scores (-inf) give weight 0
// bfloat16 has the exponents of 32 bits: any place will do.  float16 has 2^15 down to
// 2^-14 (2^-24 with fewer bits): the maximum is put at 2^12 to 2^15, so that weights
// keep all bits down to 2^-26 of it and vanish below 2^-37 (at 2^0 to 2^8: 2^-14 and
// 2^-25, where 40000 keys 17.5 nats below a first one were lost whole).
template <typename DT>
struct Weight;
template <>
struct Weight<BF16> {
  static constexpr float LIFT = 0.0f, RISE = 8.0f;
};
template <>
struct Weight<F16> {
  static constexpr float LIFT = 12.0f, RISE = 3.0f;
};

struct AttendArgs {
  Batch b;
  Rows q, out;
  uint32_t heads, kv_heads, group;
  FastDiv by_group, by_kv;
  float c;             // |scale| * log2(e) (1 with scale 0)
  uint32_t q_flip;     // XORed into query pairs: the scale's sign
  uint32_t q_keep;     // ANDed into query pairs: 0 with scale 0
  float* lse;
  uint32_t tile_rows;  // rows of a tile
  uint32_t unit;       // keys of a unit
  uint32_t slots, least;
  uint32_t round;      // items that run at a time, where that decides the run length; else 0
  uint32_t splits;     // 0: every tile is one run
  uint32_t items;      // bound on the number of items (grid and workspace)
  float* part;         // [items * kv_heads][tile_rows][value]
  float2* part_ml;     // [items * kv_heads][tile_rows]: top, sum
};

// One sequence as the scan sees it (bounds of its tokens and lengths only).
struct Share {
  uint32_t n, units, tiles;
  bool bad;  // its token range does not fit: it has no rows
};
__device__ inline Share share_of(const AttendArgs& a, uint32_t b) {
  Share s{0, 1, 0, false};
  const uint32_t lo = a.b.seq_off[b], hi = a.b.seq_off[b + 1], len = a.b.kv_len[b];
  s.bad = lo > hi || hi > a.b.T;
  if (s.bad) return s;
  s.n = hi - lo;
  s.tiles = (s.n * a.group + a.tile_rows - 1) / a.tile_rows;
  if (len && len <= a.b.max_kv) s.units = (len + a.unit - 1) / a.unit;
  return s;
}

struct Item {
  uint32_t b;          // sequence
  uint32_t first;      // index of its first item
  uint32_t per_tile;   // runs of each of its tiles
  uint32_t run_units;
  bool found;
  bool bad;            // a sequence of this lane has no usable token range
};

// Among c and the least run lengths (within a sixteenth) whose items fit one round
// and two, the one that takes the least time.  In units: each round its run and an
// item's fixed cost (queries, first keys), about 3, and for every 64 items of split
// tiles one more to write and join 256 KiB of partial sums each.  No choice is below
// c, so the bound on the items stands.  The 3 and the 64 were fitted to the two cases
// measured: 48 sequences of 8600 keys on average, 128 heads, 197-200 us a call, 223
// with c; two chunks of 754 tokens in all at 3550 keys, 32 heads, 296-298, 314 with c.
// Batches of up to 64 sequences, one a lane: more would be summed anew for every length
// tried, which has not been measured.
__device__ inline uint32_t run_of_rounds(const AttendArgs& a, const Share& own, uint64_t total, uint32_t c) {
  const uint32_t tiles = wave::sum(own.tiles);
  const auto items = [&](uint32_t run) { return wave::sum(own.tiles * ((own.units + run - 1) / run)); };
  const auto cost = [&](uint32_t run) {
    const uint32_t n = items(run);
    return (uint64_t)((n + a.round - 1) / a.round) * (run + 3) + (n > tiles ? n / 64 : 0);
  };
  uint32_t best = c;
  uint64_t least = cost(c);
  for (uint32_t fit = a.round; fit <= 2 * a.round; fit += a.round) {
    if (tiles > fit) continue;
    uint32_t run = max(c, (uint32_t)((total + fit - 1) / fit));
    while (items(run) > fit) run += 1 + run / 16;  // ends: `tiles` items are left where run passes the longest
    const uint64_t x = cost(run);
    if (x < least) {
      least = x;
      best = run;
    }
  }
  return best;
}

// The sequence that `want(first item, number of items, b)` picks, the same for
// the whole wavefront (all of whose lanes are active).
template <typename Args, typename F>
__device__ inline Item find_item(const Args& a, uint32_t lane, F want) {
  const uint32_t k = (a.b.B + 63) / 64, b0 = lane * k;
  Share own{0, 1, 0, false};  // the lane's only sequence, for batches of up to 64
  if (b0 < a.b.B) own = share_of(a, b0);
  Item it{};
  it.run_units = 0x7FFFFFFFu;
  if (a.splits) {
    uint64_t total = (uint64_t)own.tiles * own.units;
    for (uint32_t i = 1; i < k && b0 + i < a.b.B; ++i) {
      const Share s = share_of(a, b0 + i);
      total += (uint64_t)s.tiles * s.units;
    }
    total = wave::sum(total);
    it.run_units = (uint32_t)max((uint64_t)a.least, (total + a.slots - 1) / a.slots);
    if (a.round && k == 1) it.run_units = run_of_rounds(a, own, total, it.run_units);
  }
  const auto count = [&](const Share& s) { return s.tiles * ((s.units + it.run_units - 1) / it.run_units); };
  uint32_t mine = count(own);
  for (uint32_t i = 1; i < k && b0 + i < a.b.B; ++i) mine += count(share_of(a, b0 + i));
  uint32_t first = wave::incl_add(mine) - mine;
  uint32_t hit = 0xFFFFFFFFu, hit_first = 0, hit_per = 1;
  Share s = own;
  for (uint32_t i = 0; i < k && b0 + i < a.b.B; ++i) {
    if (i) s = share_of(a, b0 + i);
    const uint32_t n = count(s);
    it.bad |= s.bad;
    if (want(first, n, b0 + i)) {
      hit = b0 + i;
      hit_first = first;
      hit_per = (s.units + it.run_units - 1) / it.run_units;
    }
    first += n;
  }
  const uint64_t who = __ballot(hit != 0xFFFFFFFFu);
  it.found = who != 0;
  if (!it.found) return it;
  const int l = __ffsll((unsigned long long)who) - 1;
  it.b = (uint32_t)__builtin_amdgcn_readlane((int)hit, l);
  it.first = (uint32_t)__builtin_amdgcn_readlane((int)hit_first, l);
  it.per_tile = (uint32_t)__builtin_amdgcn_readlane((int)hit_per, l);
  return it;
}

// One workgroup's work: a run of keys of one tile of rows.
struct Work {
  Seq s;
  uint32_t item, kv;       // index of the item, key head
  uint32_t row0, rows;     // the tile's rows of the sequence: row0 .. row0 + rows - 1
  uint32_t lo, hi;         // keys; lo >= hi: none
  uint32_t open;           // keys below this, and from `from` on, are allowed to every row of the tile
  uint32_t from;
  uint32_t key0;           // no row of the tile may see a key below it
  uint32_t per_tile;
  bool some;
};

// A value that is the same in every lane, in a scalar register.
__device__ inline uint32_t same(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }

__device__ inline Work work_of(const AttendArgs& a, uint32_t block, uint32_t lane) {
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
  const uint32_t tiles = (w.s.n * a.group + a.tile_rows - 1) / a.tile_rows;
  const uint32_t k = w.item - it.first, back = k / it.per_tile, run = k - back * it.per_tile;
  w.per_tile = it.per_tile;
  // the last tile first: with a causal mask it has the most keys
  w.row0 = same((tiles - 1 - back) * a.tile_rows);
  w.rows = min(a.tile_rows, w.s.n * a.group - w.row0);
  // keys of the tile's first and last row: up to and with their own positions
  const int32_t at0 = w.s.position(divide(w.row0, a.by_group)) + 1;
  const int32_t at1 = w.s.position(divide(w.row0 + w.rows - 1, a.by_group)) + 1;
  w.open = same((uint32_t)max(at0, 0));
  const uint64_t lo = (uint64_t)run * it.run_units * a.unit, hi = lo + (uint64_t)it.run_units * a.unit;
  w.lo = same((uint32_t)min(lo, (uint64_t)0x7FFFFFFFu));
  w.hi = same((uint32_t)min(hi, (uint64_t)(uint32_t)max(at1, 0)));
  return w;
}

// Keys a row of the tile may attend to (0 for rows past the tile's).
__device__ inline uint32_t row_limit(const AttendArgs& a, const Work& w, uint32_t r) {
  if (r >= w.rows) return 0;
  return (uint32_t)max(w.s.position(divide(w.row0 + r, a.by_group)) + 1, 0);
}

// Keys that a row may see: lo .. hi - 1, none where that is empty.
struct Keys {
  uint32_t lo, hi;
  __device__ bool none() const { return lo >= hi; }
};
__device__ inline Keys row_keys(const AttendArgs& a, const Work& w, uint32_t r) { return {0, row_limit(a, w, r)}; }

// Where the rows of a tile may see different keys, or none, in this step of n keys.
__device__ inline bool differ(const Work& w, uint32_t k0, uint32_t n) {
  return (k0 + n > w.open && w.open < w.hi) || k0 < w.from;
}
__device__ inline bool differ(const Work& w) { return w.open < w.hi || w.from > w.lo; }

// Token and query head of a row of the tile.
struct RowAt {
  uint32_t t, h;
};
__device__ inline RowAt row_at(const AttendArgs& a, const Work& w, uint32_t r) {
  const uint32_t x = w.row0 + r, i = divide(x, a.by_group);
  return {w.s.t0 + i, w.kv * a.group + (x - i * a.group)};
}

__device__ inline const uint8_t* q_row(const AttendArgs& a, RowAt p) {
  return a.q.data + p.t * a.q.token + p.h * a.q.head;
}

// A query chunk with the scale's sign taken in.
__device__ inline u32x4 q_signed(const AttendArgs& a, u32x4 v) { return (v & a.q_keep) ^ a.q_flip; }

// Row of the pool (page * block_tokens + row in the page) of a key.  The host
// has checked that a plane has fewer than 2^32 rows.
__device__ inline uint32_t pool_row(const Batch& b, uint32_t key, uint32_t entry, uint32_t* err) {
  const uint32_t block = divide(key, b.by_bt);
  return checked_page(b, entry, err) * b.bt + (key - block * b.bt);
}
__device__ inline uint32_t table_entry(const Batch& b, const Seq& s, uint32_t key) {
  return b.tbl[s.tbl + divide(key, b.by_bt)];
}

// Byte offset in a plane of a key's row, all of it in scalar registers; `entry` is its block's.
__device__ inline uint64_t row_bytes_at(const Batch& b, uint32_t key, uint32_t entry, uint32_t* err) {
  const uint32_t block = divide(key, b.by_bt);
  return checked_page(b, entry, err) * b.run + (uint64_t)(key - block * b.bt) * b.row;
}

// Where the logarithm of a row's sum goes; top and sum in the kernels' units.
__device__ inline void store_lse(const AttendArgs& a, RowAt p, float top, float sum, bool none) {
  if (a.lse) a.lse[(uint64_t)p.t * a.heads + p.h] = none ? -INFINITY : (top + __log2f(sum)) * 0.69314718055994531f;
}

// Lanes of the wavefront that hold the same row: l ^ 16, l ^ 32 (and both).
__device__ inline float max_over_32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(bits<uint32_t>(x), bits<uint32_t>(x), false, false);
  return fmaxf(bits<float>(r[0]), bits<float>(r[1]));
}
__device__ inline float max_over_16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(bits<uint32_t>(x), bits<uint32_t>(x), false, false);
  return fmaxf(bits<float>(r[0]), bits<float>(r[1]));
}
__device__ inline float sum_over_32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(bits<uint32_t>(x), bits<uint32_t>(x), false, false);
  return bits<float>(r[0]) + bits<float>(r[1]);
}
__device__ inline float sum_over_16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(bits<uint32_t>(x), bits<uint32_t>(x), false, false);
  return bits<float>(r[0]) + bits<float>(r[1]);
}

// Whether `top` has to follow the step's maximum m, and where to.
template <typename DT>
__device__ inline bool risen(float m, float top) {
  return m > top + (Weight<DT>::LIFT + Weight<DT>::RISE);
}
template <typename DT>
__device__ inline float follow(float m, float top) {
  return fmaxf(top, m - Weight<DT>::LIFT);
}

__device__ inline f32x4 mfma_16x16x32(BF16, u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(bits<BF16::x8>(a), bits<BF16::x8>(b), c, 0, 0, 0);
}
__device__ inline f32x4 mfma_16x16x32(F16, u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(bits<F16::x8>(a), bits<F16::x8>(b), c, 0, 0, 0);
}
typedef float f32x16 __attribute__((ext_vector_type(16)));
__device__ inline f32x16 mfma_32x32x16(BF16, u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(bits<BF16::x8>(a), bits<BF16::x8>(b), c, 0, 0, 0);
}
__device__ inline f32x16 mfma_32x32x16(F16, u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(bits<F16::x8>(a), bits<F16::x8>(b), c, 0, 0, 0);
}

template <typename DT>
__device__ inline uint32_t pair_of(float lo, float hi) {
  typename DT::x2 h;
  h[0] = (typename DT::scalar)lo;
  h[1] = (typename DT::scalar)hi;
  return bits<uint32_t>(h);
}

// 16 B per lane from global memory straight into LDS: lane l's to dst + 16 l (dst
// the same for the wavefront).  Nothing orders a read of dst after it but the
// wait below, and across wavefronts a barrier behind that.
__device__ inline void to_lds(const uint8_t* src, uint8_t* dst) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                   (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
}
// All loads of the wavefront have arrived, those into LDS among them, and no
// read of LDS is still under way.
__device__ inline void wait_loads() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }

// Transposing read: 16 lanes take 4 rows of 16 elements, lane l's address being
// that of elements 4 (l % 4) .. of row (l % 16) / 4; a lane gets one element of each row.
typedef short s16x4 __attribute__((ext_vector_type(4)));
__device__ inline u32x2 read_tr(const uint8_t* p) {
  return bits<u32x2>(__builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p));
}

// N products whose first operand is read from LDS by read(i), AHEAD reads in
// flight.  The order is fixed: left to itself the compiler keeps one operand and
// waits for every read where registers are scarce.
template <int N, int AHEAD, typename R, typename P>
__device__ __forceinline__ void products(R read, P product) {
  u32x4 f[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) f[i] = read(i);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    product(i, f[i % AHEAD]);
    if (i + AHEAD < N) f[i % AHEAD] = read(i + AHEAD);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// The wavefront's index in its workgroup, as the scalar it is.
__device__ inline uint32_t wave_index() { return (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }

// Whether a pair of 16-bit values holds an infinity or a NaN.
__device__ inline bool odd_pair(BF16, uint32_t x) {
  return (x & 0x7F80u) == 0x7F80u || (x & 0x7F800000u) == 0x7F800000u;
}
__device__ inline bool odd_pair(F16, uint32_t x) {
  return (x & 0x7C00u) == 0x7C00u || (x & 0x7C000000u) == 0x7C000000u;
}

// A row's score in the softmax's units from the product of query and key.
__device__ inline auto score_of(const AttendArgs& a, const Work&, uint32_t, uint32_t) {
  return [c = a.c](float s, uint32_t) { return s * c; };
}

// A tile whose rows see different numbers of keys, among them one with an
// infinity or a NaN: in the matrix products it would reach the rows before it
// (weight 0 times NaN).  Such a run of keys is taken again row by row, a wavefront
// a row with plain arithmetic over the keys it may see, and that result counts.
// Nothing of the matrix kernels' state is needed, so this costs them no registers.
template <typename DT, int DK, int DV, typename Args>
__device__ inline void rows_one_by_one(const Args& a, const Work& w, uint32_t first_row, uint32_t row_step,
                                       uint32_t lane) {
  constexpr int W = DV / 64;
  typedef float vec __attribute__((ext_vector_type(W)));  // vectors, not arrays: those would end up in LDS
  typedef float f32x8 __attribute__((ext_vector_type(8)));
  typedef typename DT::scalar scalar;
  const uint64_t v_off = DK == DV ? a.b.plane_bytes : 0;
  uint32_t err = 0;  // reported by the pass before
  for (uint32_t r = first_row; r < w.rows; r += row_step) {
    const RowAt at = row_at(a, w, r);
    const Keys allowed = row_keys(a, w, r);
    const uint32_t lo = max(allowed.lo, w.lo), hi = min(allowed.hi, w.hi);
    const auto shape = score_of(a, w, r, at.h);
    const u32x4* const q = reinterpret_cast<const u32x4*>(q_row(a, at));
    float top = NO_TOP, sum = 0;
    vec o = 0;
    for (uint32_t k0 = lo; k0 < hi; k0 += 64) {
      const uint32_t key = k0 + lane;
      const uint8_t* row = a.b.plane;
      float s = -INFINITY;
      if (key < hi) {
        row += (uint64_t)pool_row(a.b, key, table_entry(a.b, w.s, key), &err) * a.b.row + (uint64_t)w.kv * DK * 2;
        s = 0;
        for (int c = 0; c < DK / 8; ++c) {
          const f32x8 x = __builtin_convertvector(bits<typename DT::x8>(reinterpret_cast<const u32x4*>(row)[c]), f32x8) *
                          __builtin_convertvector(bits<typename DT::x8>(q_signed(a, q[c])), f32x8);
          s += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
        }
        s = shape(s, key);
      }
      float m = s;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
      const float t = fmaxf(top, m), keep = __builtin_amdgcn_exp2f(top - t), f = __builtin_amdgcn_exp2f(s - t);
      top = t;
      sum = sum * keep + f;
      o *= keep;
      const uint64_t v_at = reinterpret_cast<uint64_t>(row) + v_off;
      vec part = 0;
      for (uint32_t j = 0; j < 64 && k0 + j < hi; ++j) {
        const scalar* v = reinterpret_cast<const scalar*>(wave::lane_of(v_at, (int)j));
        const float fj = __shfl(f, (int)j);
#pragma unroll
        for (int i = 0; i < W; ++i) part[i] += fj * (float)v[64 * i + lane];
      }
      o += part;
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
    if (w.per_tile > 1) {
      const uint64_t p = ((uint64_t)w.item * a.kv_heads + w.kv) * a.tile_rows + r;
#pragma unroll
      for (int i = 0; i < W; ++i) a.part[p * DV + 64 * i + lane] = o[i];
      if (lane == 0) a.part_ml[p] = float2{top, sum};
    } else {
      scalar* const out = reinterpret_cast<scalar*>(a.out.data + at.t * a.out.token + at.h * a.out.head);
#pragma unroll
      for (int i = 0; i < W; ++i) out[64 * i + lane] = (scalar)(allowed.none() ? 0.f : o[i] / sum);
      if (lane == 0) store_lse(a, at, top, sum, allowed.none());
    }
  }
}

struct SightArgs;

// Launchers, by kernel.
void launch_attend_step(const AttendArgs& a, bool f16, uint32_t dim, hipStream_t s);
void launch_attend_step(const SightArgs& a, bool f16, uint32_t dim, hipStream_t s);
void launch_attend_tile(const AttendArgs& a, bool f16, uint32_t dim, hipStream_t s);
void launch_attend_tile(const SightArgs& a, bool f16, uint32_t dim, hipStream_t s);
void launch_attend_latent(const AttendArgs& a, bool f16, hipStream_t s);
void launch_attend_join(const AttendArgs& a, bool f16, uint32_t value, hipStream_t s);
void launch_attend_join(const SightArgs& a, bool f16, uint32_t value, hipStream_t s);
void launch_sight_tiles(const SightArgs& a, hipStream_t s);
void launch_sight_join(const SightArgs& a, bool f16, uint32_t dim, hipStream_t s);

}  // namespace mori
