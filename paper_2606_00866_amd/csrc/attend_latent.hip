// Attention over a compressed-latent pool: one key row of 576 elements for all
// query heads, whose first 512 elements are the value.
//
// With H heads a key's 1152 bytes take part in 2 * 1088 * H operations, 242 per
// byte at H = 128: bytes bound a few heads, the matrix rate many.  So a key is
// staged in LDS once, as key and value, for as many rows as there are.
//
// A wavefront has 16 rows: 128 registers hold their sums (16 x 512), 72 their
// queries.  RG wavefronts share their keys and KG groups take different keys, 32
// (RG 8: 64) at a time, joined through LDS at the end:
//   RG 1  up to 16 rows, four groups: each wavefront stages and reads its own
//         keys without barriers; four staging areas of 36 KiB, filled while the
//         other wavefronts compute, keep enough loads in flight;
//   RG 2  up to 32 rows, two groups with two areas each: the next keys load behind
//         this step's products;
//   RG 4  up to 64 rows, one group, two workgroups a CU;
//   RG 8  up to 128 rows, one group of eight wavefronts.
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
  if (__any(m > acc.top + RISE)) {
    const float t = fmaxf(acc.top, m), keep = __builtin_amdgcn_exp2f(acc.top - t);
    acc.top = t;
    acc.sum *= keep;
#pragma unroll
    for (int d = 0; d < DB; ++d) acc.o[d] *= keep;
  }
  uint32_t p[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float f0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 2][2 * i % 4], a.c, -acc.top));
    const float f1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 2][2 * i % 4 + 1], a.c, -acc.top));
    acc.sum += f0 + f1;
    p[i] = pair_of<DT>(f0, f1);
  }
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

// This group's loads of SUB steps into `to`: whole pool rows, chunks permuted.
// Load i of a thread is chunk (i * RG + rg) * 64 + lane.
template <int RG, int SUB>
__device__ __forceinline__ void fetch(const AttendArgs& a, uint8_t* __restrict__ to, uint32_t row, uint32_t rg,
                                      uint32_t lane) {
  constexpr uint32_t LOADS = 36 * SUB / RG;
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
template <typename DT, int RG, int SUB>
__device__ __forceinline__ void step(const AttendArgs& a, const Work& w, const uint8_t* __restrict__ now,
                                     uint8_t* __restrict__ then, bool more, uint32_t row, uint32_t rg,
                                     const u32x4 (&q)[KS], Acc& acc, uint32_t base, uint32_t limit, uint32_t lane) {
  if (more) fetch<RG, SUB>(a, then, row, rg, lane);
#pragma unroll 1
  for (uint32_t i = 0; i < SUB; ++i)
    if (base + STEP * i < w.hi) take<DT>(a, w, now + i * STEP * ROW, q, acc, base + STEP * i, limit, lane);
}

template <typename DT, int RG>
__global__ __launch_bounds__(RG == 8 ? 512 : 256, RG == 4 ? 2 : 1) void attend_latent_kernel(AttendArgs a) {
  constexpr int NW = RG == 8 ? 8 : 4, KG = NW / RG, SUB = RG == 8 ? 2 : 1;
  constexpr uint32_t KEYS = STEP * SUB;  // a group's keys at a time
  constexpr uint32_t AREA = KEYS * ROW;
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
    constexpr uint32_t WG_KEYS = KEYS * KG;
    const auto key_of = [&](uint32_t base) { return min(base + (lane & (KEYS - 1)), last); };
    const auto pool_at = [&](uint32_t base, uint32_t entry) { return pool_row(a.b, key_of(base), entry, &err); };
    uint32_t base = w.lo + kg * KEYS;
    uint8_t* const mine = s_a + kg * (AREAS * AREA);
    uint32_t entry = table_entry(a.b, w.s, key_of(base));
    if constexpr (RG == 1) {
      if (base < w.hi) {
        fetch<RG, SUB>(a, mine, pool_at(base, entry), rg, lane);
        entry = table_entry(a.b, w.s, key_of(base + WG_KEYS));
        for (;;) {
          wait_loads();
          take<DT>(a, w, mine, q, acc, base, limit, lane);
          base += WG_KEYS;
          if (base >= w.hi) break;
          wait_loads();  // the area has been read
          fetch<RG, SUB>(a, mine, pool_at(base, entry), rg, lane);
          entry = table_entry(a.b, w.s, key_of(base + WG_KEYS));
        }
      }
    } else {
      // every group takes the workgroup's number of steps (its keys past the end are masked)
      fetch<RG, SUB>(a, mine, pool_at(base, entry), rg, lane);
      entry = table_entry(a.b, w.s, key_of(base + WG_KEYS));
      wait_loads();
      __syncthreads();
      uint32_t now = 0;
      for (uint32_t first = w.lo; first < w.hi; first += WG_KEYS, now ^= AREA) {
        const bool more = first + WG_KEYS < w.hi;
        const uint32_t row = more ? pool_at(base + WG_KEYS, entry) : 0;
        step<DT, RG, SUB>(a, w, mine + now, mine + (now ^ AREA), more, row, rg, q, acc, base, limit, lane);
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

template <typename DT>
void launch(const AttendArgs& a, hipStream_t s) {
  const dim3 grid(a.items);
  switch (a.tile_rows) {
    case 16: hipLaunchKernelGGL((attend_latent_kernel<DT, 1>), grid, dim3(256), 0, s, a); break;
    case 32: hipLaunchKernelGGL((attend_latent_kernel<DT, 2>), grid, dim3(256), 0, s, a); break;
    case 64: hipLaunchKernelGGL((attend_latent_kernel<DT, 4>), grid, dim3(256), 0, s, a); break;
    default: hipLaunchKernelGGL((attend_latent_kernel<DT, 8>), grid, dim3(512), 0, s, a); break;
  }
}

}  // namespace

void launch_attend_latent(const AttendArgs& a, bool f16, hipStream_t s) {
  if (f16) launch<F16>(a, s);
  else launch<BF16>(a, s);
}

}  // namespace mori
