// Attention over a compressed-latent pool: one key row of 576 elements for all
// query heads, whose first 512 elements are the value.
//
// With H heads a key's 1152 bytes take part in 2 * 1088 * H operations, 242 per
// byte at H = 128: bytes bound a few heads, the matrix rate many.  So a key is
// staged in LDS once, as key and value, for as many rows as there are.
//
// Up to 64 rows a wavefront has 16: 128 registers hold their sums (16 x 512), 72
// their queries.  RG of the four wavefronts share their keys and the KG groups take
// different keys, 32 at a time, joined through LDS at the end:
//   RG 1  up to 16 rows, four groups: each wavefront stages and reads its own
//         keys without barriers; four staging areas of 36 KiB, filled while the
//         other wavefronts compute, keep enough loads in flight;
//   RG 2  up to 32 rows, two groups with two areas each: the next keys load behind
//         this step's products;
//   RG 4  up to 64 rows, one group, two workgroups a CU (256 registers a lane, three
//         words of which go to scratch).
// More rows than that have a kernel of their own, below.
//
// 256 sequences of 2.25 M keys in all, 16 heads (2.6 GB): 549 us, 4.7 TB/s of the
// 6.2 that a copy reaches.  Each staged byte is written to LDS once and read there
// nearly twice (as key and as value), beside the products; four areas a CU is what
// LDS holds.
//   scores   S^T = K Q^T, 16x16x32;  values  O^T += V^T P^T, the weights in the
//            order in which they leave the score product (see attend_step.hip).
// A row is 72 chunks of 16 B, permuted within each 8 by a function f of the row:
// rows 2 r and 2 r + 1 lie 128 B apart in the banks, so f takes bits 1..3 of the
// row, reversed: sixteen rows' equal chunks fall on different banks (score reads),
// and so do the 32 B of eight rows (transposing reads of the values).
#include "attend.h"

namespace mori {
namespace {

constexpr uint32_t STEP = 32, ROW = 1152, CH = 72;
constexpr int DK = 576, DV = 512;
constexpr int KS = DK / 32, DB = DV / 16;
constexpr int AHEAD = 5;  // operands read ahead of the products

__device__ inline uint32_t swizzle(uint32_t row) {
  return (row >> 1 & 1) << 2 | (row >> 2 & 1) << 1 | (row >> 3 & 1);
}

// The rows' state of one wavefront.
struct Acc {
  f32x4 o[DB];
  float top, sum;
  bool odd;  // a score was not finite where it could reach rows that must not see it
};

// One step of 32 keys at `at` (LDS): scores, weights, values.  Keys of the step
// from `base` on; a row's keys end at `limit`.
template <typename DT>
__device__ __forceinline__ void take(const AttendArgs& a, const Work& w, const uint8_t* __restrict__ at,
                                     const u32x4 (&q)[KS], Acc& acc, uint32_t base, uint32_t limit, uint32_t lane) {
  const uint32_t n = lane & 15, g = lane >> 4;
  f32x4 s[2] = {f32x4{0, 0, 0, 0}, f32x4{0, 0, 0, 0}};
  const uint32_t kx = swizzle(n);  // the same for key n + 16
  const uint8_t* const ks = at + n * ROW;
  products<2 * KS, AHEAD>(
      [&](int x) {
        const int k = x >> 1;
        return *reinterpret_cast<const u32x4*>(ks + ((((4 * (k & 1) + g) ^ kx) + 8 * (k >> 1)) << 4) + 16 * (x & 1) * ROW);
      },
      [&](int x, u32x4 f) { s[x & 1] = mfma_16x16x32(DT(), f, q[x >> 1], s[x & 1]); });
  if (base + STEP > w.open || base + STEP > w.hi) {
    if (w.open < w.hi) {
      // a key that is not finite shows in the scores of every row
#pragma unroll
      for (int i = 0; i < 8; ++i) acc.odd |= !__builtin_isfinite(s[i / 4][i % 4]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (base + 16 * (i / 4) + 4 * g + i % 4 >= limit) s[i / 4][i % 4] = -INFINITY;
  }
  float m = s[0][0];
#pragma unroll
  for (int i = 1; i < 8; ++i) m = fmaxf(m, s[i / 4][i % 4]);
  m = a.c * max_over_16(max_over_32(m));
  if (__any(risen<DT>(m, acc.top))) {
    const float t = follow<DT>(m, acc.top), keep = __builtin_amdgcn_exp2f(acc.top - t);
    acc.top = t;
    acc.sum *= keep;
#pragma unroll
    for (int d = 0; d < DB; ++d) acc.o[d] *= keep;
  }
  float part = 0;  // of this step: one by one, small weights would be lost in a large sum
  uint32_t p[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float f0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 2][2 * i % 4], a.c, -acc.top));
    const float f1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 2][2 * i % 4 + 1], a.c, -acc.top));
    part += f0 + f1;
    p[i] = pair_of<DT>(f0, f1);
  }
  acc.sum += part;
  // transposing reads: key rows 4 g .. 4 g + 3 of each 16, 16 elements per 16 lanes
  const uint32_t vrow = 4 * g + (lane >> 2 & 3);
  const uint32_t vx = swizzle(vrow), vc = lane >> 1 & 1;
  const uint8_t* const vs = at + vrow * ROW + 8 * (lane & 1);
  const u32x4 pt = {p[0], p[1], p[2], p[3]};
  products<DB, AHEAD>(
      [&](int d) {
        const uint8_t* c = vs + ((((2 * (d & 3) + vc) ^ vx) + 8 * (d >> 2)) << 4);
        const u32x2 lo = read_tr(c), hi = read_tr(c + 16 * ROW);
        return u32x4{lo[0], lo[1], hi[0], hi[1]};
      },
      [&](int d, u32x4 f) { acc.o[d] = mfma_16x16x32(DT(), f, pt, acc.o[d]); });
}

// This group's loads of a step into `to`: whole pool rows, chunks permuted.
// Load i of a thread is chunk (i * RG + rg) * 64 + lane.
template <int RG>
__device__ __forceinline__ void fetch(const AttendArgs& a, uint8_t* __restrict__ to, uint32_t row, uint32_t rg,
                                      uint32_t lane) {
  constexpr uint32_t LOADS = 36 / RG;
  // recomputed at every step: nine places kept over the products cost more registers than there are
  asm volatile("" : "+v"(lane));
  uint32_t place[9];
#pragma unroll
  for (uint32_t i = 0; i < 9; ++i) {
    const uint32_t c = (i * RG + rg) * 64 + lane, r = c / CH, at = c - r * CH;
    place[i] = r << 16 | (at ^ swizzle(r)) * 16;
  }
#pragma unroll
  for (uint32_t i = 0; i < LOADS; ++i) {
    // nine loads of the group cover 8 * RG rows (8 rows on, bit 3 of the row flips the chunk's lowest)
    const uint32_t at = (uint32_t)__shfl((int)row, (int)((place[i % 9] >> 16) + i / 9 * 8 * RG));
    const uint32_t flip = i / 9 * 8 * RG & 8 ? 16 : 0;
    to_lds(a.b.plane + (uint64_t)at * ROW + ((place[i % 9] & 0xFFFFu) ^ flip), to + (i * RG + rg) * 1024);
  }
}

// A group's step: the next keys set out for one area, these taken from the other.
// (The areas' being apart is what lets the reads run beside the loads.)
template <typename DT, int RG>
__device__ __forceinline__ void step(const AttendArgs& a, const Work& w, const uint8_t* __restrict__ now,
                                     uint8_t* __restrict__ then, bool more, uint32_t row, uint32_t rg,
                                     const u32x4 (&q)[KS], Acc& acc, uint32_t base, uint32_t limit, uint32_t lane) {
  if (more) fetch<RG>(a, then, row, rg, lane);
  if (base < w.hi) take<DT>(a, w, now, q, acc, base, limit, lane);
}

template <typename DT, int RG>
__global__ __launch_bounds__(256, RG == 4 ? 2 : 1) void attend_latent_kernel(AttendArgs a) {
  constexpr int NW = 4, KG = NW / RG;
  constexpr uint32_t AREA = STEP * ROW;
  constexpr uint32_t AREAS = RG == 1 ? 1 : 2;  // of each group
  __shared__ __align__(256) uint8_t s_a[AREAS * KG * AREA];
  __shared__ float s_top[KG][RG * 16], s_sum[KG][RG * 16];
  const uint32_t tid = threadIdx.x, lane = tid & 63, wv = wave_index();
  const uint32_t n = lane & 15, g = lane >> 4;
  const uint32_t rg = wv % RG, kg = wv / RG;
  const Work w = work_of(a, blockIdx.x, lane);
  if (!w.some) return;
  uint32_t err = w.s.error;
  const uint32_t last = w.hi - 1;
  const uint32_t r = 16 * rg + n;
  const uint32_t limit = min(row_limit(a, w, r), w.hi);

  u32x4 q[KS];
  {
    const u32x4* src = reinterpret_cast<const u32x4*>(q_row(a, row_at(a, w, min(r, w.rows - 1))) + 16 * g);
#pragma unroll
    for (int k = 0; k < KS; ++k) q[k] = q_signed(a, src[4 * k]);
  }
  Acc acc;
  acc.top = NO_TOP;
  acc.sum = 0;
  acc.odd = false;
#pragma unroll
  for (int d = 0; d < DB; ++d) acc.o[d] = f32x4{0, 0, 0, 0};

  if (w.lo < w.hi) {
    constexpr uint32_t WG_KEYS = STEP * KG;
    const auto key_of = [&](uint32_t base) { return min(base + (lane & (STEP - 1)), last); };
    const auto pool_at = [&](uint32_t base, uint32_t entry) { return pool_row(a.b, key_of(base), entry, &err); };
    uint32_t base = w.lo + kg * STEP;
    uint8_t* const mine = s_a + kg * (AREAS * AREA);
    uint32_t entry = table_entry(a.b, w.s, key_of(base));
    if constexpr (RG == 1) {
      if (base < w.hi) {
        fetch<RG>(a, mine, pool_at(base, entry), rg, lane);
        entry = table_entry(a.b, w.s, key_of(base + WG_KEYS));
        for (;;) {
          wait_loads();
          take<DT>(a, w, mine, q, acc, base, limit, lane);
          base += WG_KEYS;
          if (base >= w.hi) break;
          wait_loads();  // the area has been read
          fetch<RG>(a, mine, pool_at(base, entry), rg, lane);
          entry = table_entry(a.b, w.s, key_of(base + WG_KEYS));
        }
      }
    } else {
      // every group takes the workgroup's number of steps (its keys past the end are masked)
      fetch<RG>(a, mine, pool_at(base, entry), rg, lane);
      entry = table_entry(a.b, w.s, key_of(base + WG_KEYS));
      wait_loads();
      __syncthreads();
      uint32_t now = 0;
      for (uint32_t first = w.lo; first < w.hi; first += WG_KEYS, now ^= AREA) {
        const bool more = first + WG_KEYS < w.hi;
        const uint32_t row = more ? pool_at(base + WG_KEYS, entry) : 0;
        step<DT, RG>(a, w, mine + now, mine + (now ^ AREA), more, row, rg, q, acc, base, limit, lane);
        if (more) entry = table_entry(a.b, w.s, key_of(base + 2 * WG_KEYS));
        base += WG_KEYS;
        wait_loads();
        __syncthreads();
      }
    }
  }
  if (__any(err != 0)) report(a.b, err);
  if (w.open < w.hi && __syncthreads_or(acc.odd)) {
    rows_one_by_one<DT, DK, DV>(a, w, wv, NW, lane);
    return;
  }

  // join the key groups: group 0 takes the others' rows in their order, through LDS
  acc.sum = sum_over_16(sum_over_32(acc.sum));
  if constexpr (KG > 1) {
    if (g == 0) {
      s_top[kg][r] = acc.top;
      s_sum[kg][r] = acc.sum;
    }
    wait_loads();
    __syncthreads();  // also: the staging areas have been read
    float t = NO_TOP;
#pragma unroll
    for (int i = 0; i < KG; ++i) t = fmaxf(t, s_top[i][r]);
    const float keep = __builtin_amdgcn_exp2f(acc.top - t);
    float l = 0;
#pragma unroll
    for (int i = 0; i < KG; ++i) l += s_sum[i][r] * __builtin_amdgcn_exp2f(s_top[i][r] - t);
    acc.top = t;
    acc.sum = l;
    // [kg - 1][rg][d][lane] of four elements: 32 KiB a wavefront
    f32x4* const buf = reinterpret_cast<f32x4*>(s_a) + rg * (DB * 64) + lane;
    constexpr uint32_t GROUP = RG * DB * 64;
    static_assert((KG - 1) * GROUP * 16 <= KG * AREA, "the join fits the staging areas");
#pragma unroll
    for (int d = 0; d < DB; ++d) acc.o[d] *= keep;
    if (kg) {
#pragma unroll
      for (int d = 0; d < DB; ++d) buf[(kg - 1) * GROUP + d * 64] = acc.o[d];
    }
    __syncthreads();
    if (kg) return;
#pragma unroll
    for (int i = 0; i < KG - 1; ++i)
#pragma unroll
      for (int d = 0; d < DB; ++d) acc.o[d] += buf[i * GROUP + d * 64];
  }
  if (r >= w.rows) return;
  if (w.per_tile > 1) {
    const uint64_t at = (uint64_t)w.item * a.tile_rows + r;
#pragma unroll
    for (int d = 0; d < DB; ++d) *reinterpret_cast<f32x4*>(a.part + at * DV + 16 * d + 4 * g) = acc.o[d];
    if (g == 0) a.part_ml[at] = float2{acc.top, acc.sum};
  } else {
    const RowAt at = row_at(a, w, r);
    const bool none = row_limit(a, w, r) == 0;
    const float inv = 1.f / acc.sum;
    uint8_t* out = a.out.data + at.t * a.out.token + at.h * a.out.head;
#pragma unroll
    for (int d = 0; d < DB; ++d) {
      const u32x2 y = {pair_of<DT>(acc.o[d][0] * inv, acc.o[d][1] * inv),
                       pair_of<DT>(acc.o[d][2] * inv, acc.o[d][3] * inv)};
      *reinterpret_cast<u32x2*>(out + 2 * (16 * d + 4 * g)) = none ? u32x2{0, 0} : y;
    }
    if (g == 0) store_lse(a, at, acc.top, acc.sum, none);
  }
}

// ---- up to 128 rows --------------------------------------------------------
// Eight wavefronts of 16 rows would each read every key from LDS: 544 KiB for 32
// keys, and what a wavefront waits for is those reads.  Here two wavefronts share
// 32 rows, so that a read serves two products: of the scores each takes half of the
// elements for all 32 rows (the halves are added through LDS), of the values half
// of the 512.  A wavefront's own 16 rows are its block 0, its partner's block 1; it
// finishes the scores of its own and hands over their weights.
//   scores of half the elements - other block's half to LDS - barrier 1 - earlier loads
//   have arrived, new ones set out - add, weights, to LDS - barrier 2 - values
// Two barriers a step are enough: what is overwritten behind a barrier was last read
// before it (halves before barrier 2, weights and keys before barrier 1 of the next
// step).  Keys are staged in three areas: one is read, one has arrived, one is loaded;
// a step's loads have the whole of the next one to arrive in.
//
// 48 sequences of 0.41 M keys in all, 128 heads (0.49 GB, 0.115 TFLOP): 183 us, 627
// TFLOP/s; two chunks of 754 tokens in all, 32 heads (0.177 TFLOP): 295 us, 599
// TFLOP/s on 189 of 256 CUs.  The matrix units are busy 33% of the first's cycles: the
// products of a step, its weights and its loads follow one another between the
// barriers, and with one workgroup a CU nothing else runs while wavefronts wait there.
// At the same run lengths eight wavefronts that each kept 16 rows to themselves took
// 236 us for the first, this 209.
namespace wide {

constexpr int NW = 8, AREAS = 3, LOADS = 5;
constexpr uint32_t AREA = LOADS * NW * 1024;  // 32 rows and a tail that is loaded but not read
constexpr int KS = DK / 64, DB = DV / 32;  // steps and value blocks of a half

// Barrier for data in LDS that wavefronts wrote themselves.  It does not wait for the
// loads into LDS under way; wait_loads() and the barrier behind it do.
__device__ inline void barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
// Stores to LDS that the compiler does not set behind the loads into LDS under way
// (it orders any store after all of them); barrier() waits for these.
template <typename T>
__device__ inline uint32_t lds_address(T* p) {
  return (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) T*)p);
}
__device__ inline void put(f32x4* p, f32x4 v) {
  asm volatile("ds_write_b128 %0, %1" ::"v"(lds_address(p)), "v"(v) : "memory");
}
__device__ inline void put(u32x4* p, u32x4 v) {
  asm volatile("ds_write_b128 %0, %1" ::"v"(lds_address(p)), "v"(v) : "memory");
}
__device__ inline void put(float* p, float v) {
  asm volatile("ds_write_b32 %0, %1" ::"v"(lds_address(p)), "v"(v) : "memory");
}

// 16-B chunk of a key that lane group g reads for step k of half h: the groups'
// chunks are 128 B apart, so that only the rows decide the banks (but in the last
// step, which takes the row's last 128 B).
__device__ inline uint32_t chunk_of(uint32_t k, uint32_t h, uint32_t g) {
  return k < 8 ? 8 * (4 * (k >> 2) + g) + 4 * h + (k & 3) : 64 + 4 * h + g;
}

// A step's loads (the last four of the 40 bring rows 0 to 3 again).
__device__ __forceinline__ void fetch(const AttendArgs& a, uint8_t* to, uint32_t row, uint32_t wv, uint32_t lane) {
#pragma unroll
  for (uint32_t i = 0; i < LOADS; ++i) {
    const uint32_t c = (i * NW + wv) * 64 + lane, r = c / CH, at = c - r * CH;
    const uint32_t p = (uint32_t)__shfl((int)row, (int)r);
    const uint8_t* const src = a.b.plane + (uint64_t)p * ROW + ((at ^ swizzle(r)) << 4);
    to_lds(src, to + (i * NW + wv) * 1024);
  }
}

struct Shared {
  alignas(16) f32x4 part[NW][2][64];  // scores of the partner's rows over this wavefront's elements
  alignas(16) u32x4 weight[NW][64];
  float keep[NW][16], top[NW][16], sum[NW][16];
};

struct Acc {
  f32x4 o[DB][2];  // this wavefront's elements: its own rows, its partner's
  float top, sum;  // of its own rows
  bool odd;
};

template <typename DT>
__device__ __forceinline__ void step(const AttendArgs& a, const Work& w, const uint8_t* __restrict__ now,
                                     uint8_t* __restrict__ then, Shared& x,
                                     const u32x4 (&q)[KS][2], Acc& acc, uint32_t base, uint32_t limit, uint32_t wv,
                                     uint32_t lane, uint32_t* err) {
  asm volatile("" : "+v"(lane));  // what follows from it is computed at every step: there is no room to keep it
  // the keys after next: their table entry is here when the scores are
  const uint32_t ahead = min(base + 2 * STEP + (lane & (STEP - 1)), w.hi - 1);
  const uint32_t entry = table_entry(a.b, w.s, ahead);
  const uint32_t n = lane & 15, g = lane >> 4, h = wv & 1;
  f32x4 s[2][2];
#pragma unroll
  for (int b = 0; b < 2; ++b) s[b][0] = s[b][1] = f32x4{0, 0, 0, 0};
  const uint32_t kx = swizzle(n);  // the same for key n + 16
  const uint8_t* const ks = now + n * ROW;
  products<2 * KS, 3>(
      [&](int i) {
        return *reinterpret_cast<const u32x4*>(ks + ((chunk_of(i >> 1, h, g) ^ kx) << 4) + 16 * (i & 1) * ROW);
      },
      [&](int i, u32x4 f) {
#pragma unroll
        for (int b = 0; b < 2; ++b) s[b][i & 1] = mfma_16x16x32(DT(), f, q[i >> 1][b], s[b][i & 1]);
      });
  // the compiler sees no store here: the products' delay before their results may be read is kept by hand
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 15\n\ts_nop 3" ::: "memory");
  put(&x.part[wv][0][lane], s[1][0]);
  put(&x.part[wv][1][lane], s[1][1]);
  barrier();  // every wavefront is through with the step before: its area is free
  __builtin_amdgcn_sched_barrier(0);  // the wait for the earlier loads (and the entry) stays behind it
  wait_loads();
  fetch(a, then, pool_row(a.b, ahead, entry, err), wv, lane);
#pragma unroll
  for (int i = 0; i < 2; ++i) s[0][i] += x.part[wv ^ 1][i][lane];
  if (base + STEP > w.open || base + STEP > w.hi) {
    if (w.open < w.hi) {
      // a key that is not finite shows in the scores of every row
#pragma unroll
      for (int i = 0; i < 8; ++i) acc.odd |= !__builtin_isfinite(s[0][i / 4][i % 4]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (base + 16 * (i / 4) + 4 * g + i % 4 >= limit) s[0][i / 4][i % 4] = -INFINITY;
  }
  float m = s[0][0][0];
#pragma unroll
  for (int i = 1; i < 8; ++i) m = fmaxf(m, s[0][i / 4][i % 4]);
  m = a.c * max_over_16(max_over_32(m));
  float keep = 1.f;
  if (__any(risen<DT>(m, acc.top))) {
    const float t = follow<DT>(m, acc.top);
    keep = __builtin_amdgcn_exp2f(acc.top - t);
    acc.top = t;
    acc.sum *= keep;
  }
  float part = 0;  // of this step, as above
  u32x4 p[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float f0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[0][i / 2][2 * i % 4], a.c, -acc.top));
    const float f1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[0][i / 2][2 * i % 4 + 1], a.c, -acc.top));
    part += f0 + f1;
    p[0][i] = pair_of<DT>(f0, f1);
  }
  acc.sum += part;
  put(&x.weight[wv][lane], p[0]);
  put(&x.keep[wv][n], keep);
  barrier();
  p[1] = x.weight[wv ^ 1][lane];
  const float keep1 = x.keep[wv ^ 1][n];
  if (__any(keep != 1.f || keep1 != 1.f)) {
#pragma unroll
    for (int d = 0; d < DB; ++d) {
      acc.o[d][0] *= keep;
      acc.o[d][1] *= keep1;
    }
  }
  // transposing reads: key rows 4 g .. 4 g + 3 of each 16, 16 elements per 16 lanes
  const uint32_t vrow = 4 * g + (lane >> 2 & 3);
  const uint32_t vx = swizzle(vrow), vc = lane >> 1 & 1;
  const uint8_t* const vs = now + vrow * ROW + 8 * (lane & 1) + h * DV;
  products<DB, 4>(
      [&](int d) {
        const uint8_t* c = vs + ((((2 * (d & 3) + vc) ^ vx) + 8 * (d >> 2)) << 4);
        const u32x2 lo = read_tr(c), hi = read_tr(c + 16 * ROW);
        return u32x4{lo[0], lo[1], hi[0], hi[1]};
      },
      [&](int d, u32x4 f) {
#pragma unroll
        for (int b = 0; b < 2; ++b) acc.o[d][b] = mfma_16x16x32(DT(), f, p[b], acc.o[d][b]);
      });
}

template <typename DT>
__global__ __launch_bounds__(64 * NW, 1) void attend_latent_wide_kernel(AttendArgs a) {
  __shared__ __align__(256) uint8_t key[AREAS * AREA];  // apart from the rest: loads into it run beside reads of that
  __shared__ Shared x;
  uint32_t lane = threadIdx.x & 63;
  const uint32_t wv = wave_index();
  uint32_t n = lane & 15, g = lane >> 4;
  const uint32_t h = wv & 1;
  const Work w = work_of(a, blockIdx.x, lane);
  if (!w.some) return;
  uint32_t err = w.s.error;
  const uint32_t last = w.hi - 1;
  const uint32_t limit = min(row_limit(a, w, 16 * wv + n), w.hi);

  const auto key_of = [&](uint32_t base) { return min(base + (lane & (STEP - 1)), last); };
  const auto pool_at = [&](uint32_t base, uint32_t entry) { return pool_row(a.b, key_of(base), entry, &err); };
  if (w.lo < w.hi) {  // the first keys on the way, then the queries
    // (past the end: the last key again)
    fetch(a, key, pool_at(w.lo, table_entry(a.b, w.s, key_of(w.lo))), wv, lane);
    const uint32_t second = min(w.lo + STEP, last);
    fetch(a, key + AREA, pool_at(second, table_entry(a.b, w.s, key_of(second))), wv, lane);
  }
  u32x4 q[KS][2];
  Acc acc;
  acc.odd = false;
  acc.top = NO_TOP;
  acc.sum = 0;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const uint32_t r = 16 * (wv ^ b) + n;
    const u32x4* src = reinterpret_cast<const u32x4*>(q_row(a, row_at(a, w, min(r, w.rows - 1))));
#pragma unroll
    for (int k = 0; k < KS; ++k) q[k][b] = q_signed(a, src[chunk_of(k, h, g)]);
#pragma unroll
    for (int d = 0; d < DB; ++d) acc.o[d][b] = f32x4{0, 0, 0, 0};
  }

  if (w.lo < w.hi) {
    wait_loads();
    barrier();
    uint32_t now = 0, then = 2 * AREA;
    for (uint32_t base = w.lo; base < w.hi; base += STEP) {
      step<DT>(a, w, key + now, key + then, x, q, acc, base, limit, wv, lane, &err);
      now = now == 2 * AREA ? 0 : now + AREA;
      then = then == 2 * AREA ? 0 : then + AREA;
    }
    wait_loads();
  }
  if (__any(err != 0)) report(a.b, err);
  if (w.open < w.hi && __syncthreads_or(acc.odd)) {
    rows_one_by_one<DT, DK, DV>(a, w, wv, NW, lane);
    return;
  }

  // the rows' places are computed again: there was no room to keep them over the steps
  asm volatile("" : "+v"(lane));
  n = lane & 15;
  g = lane >> 4;
  acc.sum = sum_over_16(sum_over_32(acc.sum));
  if (g == 0) {
    x.top[wv][n] = acc.top;
    x.sum[wv][n] = acc.sum;
  }
  __syncthreads();
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const uint32_t r = 16 * (wv ^ b) + n;
    const float top = x.top[wv ^ b][n], sum = x.sum[wv ^ b][n];
    if (r >= w.rows) continue;
    if (w.per_tile > 1) {
      const uint64_t at = (uint64_t)w.item * a.tile_rows + r;
#pragma unroll
      for (int d = 0; d < DB; ++d)
        *reinterpret_cast<f32x4*>(a.part + at * DV + h * (DV / 2) + 16 * d + 4 * g) = acc.o[d][b];
      if (g == 0 && b == 0) a.part_ml[at] = float2{top, sum};
    } else {
      const RowAt at = row_at(a, w, r);
      const bool none = row_limit(a, w, r) == 0;
      const float inv = 1.f / sum;
      uint8_t* out = a.out.data + at.t * a.out.token + at.h * a.out.head + h * DV;
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        const f32x4 y = acc.o[d][b] * inv;
        const u32x2 z = {pair_of<DT>(y[0], y[1]), pair_of<DT>(y[2], y[3])};
        *reinterpret_cast<u32x2*>(out + 2 * (16 * d + 4 * g)) = none ? u32x2{0, 0} : z;
      }
      if (g == 0 && b == 0) store_lse(a, at, top, sum, none);
    }
  }
}

}  // namespace wide

template <typename DT>
void launch(const AttendArgs& a, hipStream_t s) {
  const dim3 grid(a.items);
  switch (a.tile_rows) {
    case 16: hipLaunchKernelGGL((attend_latent_kernel<DT, 1>), grid, dim3(256), 0, s, a); break;
    case 32: hipLaunchKernelGGL((attend_latent_kernel<DT, 2>), grid, dim3(256), 0, s, a); break;
    case 64: hipLaunchKernelGGL((attend_latent_kernel<DT, 4>), grid, dim3(256), 0, s, a); break;
    default: hipLaunchKernelGGL((wide::attend_latent_wide_kernel<DT>), grid, dim3(64 * wide::NW), 0, s, a); break;
  }
}

}  // namespace

void launch_attend_latent(const AttendArgs& a, bool f16, hipStream_t s) {
  if (f16) launch<F16>(a, s);
  else launch<BF16>(a, s);
}

}  // namespace mori
