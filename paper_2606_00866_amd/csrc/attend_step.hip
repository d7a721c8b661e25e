// Attention of few rows per key head (decode steps, a handful of new tokens):
// up to 16 * NB rows, bound by reading keys and values once.
//
// Nothing is staged in LDS: a wavefront takes 32 keys at a time straight into the
// registers its matrix instructions read.
//   scores   S^T = K Q^T, 16x16x32: a lane holds 16 B of one key row per step, the
//            query rows are the columns, so a row's scores lie in four lanes.
//   values   O^T += V^T P^T.  The weights leave the score product in lanes
//            (row, group g) for keys 4 g .. 4 g + 3 of each 16: taken as the
//            product's k index in that order they need no exchange.  For the
//            values a lane loads 8 keys (those of its group) at the same D / 16
//            elements, whole pool rows per 16 lanes, and transposes the 8 x 8
//            16-bit block with byte permutes.
// The keys' places (page, row) are found one step ahead, keys of the next step
// are loaded behind the scores of this one, values behind the scores' loads, so
// reads are always under way.  Four wavefronts share an item's keys, 32 each in
// turn, and join their sums through LDS at the end.
//
// Why registers: each key and value is read by one wavefront only, so a pass through
// LDS would add writes, reads and barriers and share nothing.
//
// 64 sequences of 1.19 M keys in all (8 key heads of 128, groups of 4; 4.86 GB):
// 892 us, 5.4 TB/s of the 6.2 that a copy reaches, a step's loads ahead in two
// wavefronts a SIMD (200 registers a lane of the 256 they may have at head dimension
// 128; with 17 to 32 rows 292, one wavefront a SIMD).  One sequence of 65502 keys, one key
// head (34 MB): 17 us with the join, 2 TB/s: finding the item, two rounds of dependent
// reads (table, keys) and the second launch.  Eight sequences of 760 keys: 10 us.
//
// With a sight (sight.h) one form serves caps, biases, windows and ranges: it is the bytes
// that bound it.  64 sequences that see 4096 keys each (1.07 GB): 200 us, 5.4 TB/s.  One
// sequence of 65502 keys with a bias: 18.4 us, eight of 760 with a cap 12.2.  So weights are
// pairs of 16-bit numbers there, what is taken and the rest, in two products with the values:
// 2^-16 of a weight (fp16 2^-22) for 2^-8 (2^-11), and an error against 64 bits of 0.0017,
// which the result's own rounding makes, for 0.0021.  That costs 0.3 us of small steps, 0 to 2%
// of larger ones, and up to 6% with 17 to 32 rows (64 sequences of four tokens behind 3000
// keys, 8 heads on one key head: 50.5 to 53.6 us).
#include "sight.h"

namespace mori {
namespace {

constexpr uint32_t NW = 4, STEP = 32;

template <typename DT, int D, int NB, typename Args>
__global__ __launch_bounds__(64 * NW) void attend_step_kernel(Args a) {
  constexpr bool SIGHT = IsSight<Args>::value;
  constexpr int FORM = IsSight<Args>::FORM;
  constexpr int KS = D / 32;       // matrix steps over the head's elements
  constexpr int E = D / 16;        // value elements of a lane: 4 or 8
  constexpr int VW = E / 2;        // their 32-bit words
  __shared__ float s_o[NW][16][D + 4];
  __shared__ float s_top[NW][16 * NB], s_sum[NW][16 * NB];
  const uint32_t tid = threadIdx.x, lane = tid & 63, wv = wave_index();
  const uint32_t n = lane & 15, g = lane >> 4;
  const Work w = work_of(a, blockIdx.x, lane);
  if (!w.some) return;
  uint32_t err = w.s.error;
  const uint32_t last = w.hi - 1;  // used only if lo < hi
  const uint8_t* const kp = a.b.plane + (uint64_t)w.kv * (2 * D) + 16 * g;
  const uint8_t* const vp = a.b.plane + a.b.plane_bytes + (uint64_t)w.kv * (2 * D) + (2 * E) * n;

  u32x4 q[NB][KS];
  uint32_t limit[NB], low[NB];  // a row's keys
  int32_t pos[NB];              // where it stands
  float slope[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const uint32_t r = 16 * nb + n;
    const Keys keys = row_keys(a, w, r);
    limit[nb] = min(keys.hi, w.hi);
    const RowAt at = row_at(a, w, min(r, w.rows - 1));
    const u32x4* src = reinterpret_cast<const u32x4*>(q_row(a, at) + 16 * g);
    if constexpr (SIGHT) {
      low[nb] = keys.lo;
      pos[nb] = w.s.position(at.t - w.s.t0);
      slope[nb] = slope_of(a, at.h);
    }
#pragma unroll
    for (int k = 0; k < KS; ++k) q[nb][k] = q_signed(a, src[4 * k]);
  }
  f32x4 o[NB][E];
  float top[NB], sum[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    top[nb] = NO_TOP;
    sum[nb] = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) o[nb][e] = f32x4{0, 0, 0, 0};
  }

  bool odd = false;  // a value that rows see in part is infinite or NaN
  uint32_t k0 = w.lo + wv * STEP;
  if (k0 < w.hi) {
    u32x4 kr[2][KS];
    uint32_t row, entry;  // this lane's key (lane % 32 of a step): pool row now, table entry of the next step
    const uint32_t kl = lane & 31;
    const auto key_of = [&](uint32_t base) { return min(base + kl, last); };
    const auto load_keys = [&](uint32_t rr) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t at = (uint32_t)__shfl((int)rr, 16 * i + (int)n);
        const u32x4* src = reinterpret_cast<const u32x4*>(kp + (uint64_t)at * a.b.row);
#pragma unroll
        for (int k = 0; k < KS; ++k) kr[i][k] = src[4 * k];
      }
    };
    row = pool_row(a.b, key_of(k0), table_entry(a.b, w.s, key_of(k0)), &err);
    entry = table_entry(a.b, w.s, key_of(min(k0 + NW * STEP, last)));
    load_keys(row);
    for (;;) {
      // values of this step: 8 keys at this lane's elements
      uint32_t vr[8][VW];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t at = (uint32_t)__shfl((int)row, (int)(16 * (j / 4) + 4 * g + j % 4));
        const uint8_t* src = vp + (uint64_t)at * a.b.row;
        if constexpr (VW == 4) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(src);
#pragma unroll
          for (int i = 0; i < 4; ++i) vr[j][i] = x[i];
        } else {
          const u32x2 x = *reinterpret_cast<const u32x2*>(src);
          vr[j][0] = x[0];
          vr[j][1] = x[1];
        }
      }
      f32x4 s[NB][2];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          s[nb][i] = f32x4{0, 0, 0, 0};
#pragma unroll
          for (int k = 0; k < KS; ++k) s[nb][i] = mfma_16x16x32(DT(), kr[i][k], q[nb][k], s[nb][i]);
        }
      const uint32_t next = k0 + NW * STEP;
      const bool more = next < w.hi;
      if (more) {
        row = pool_row(a.b, key_of(next), entry, &err);
        entry = table_entry(a.b, w.s, key_of(min(next + NW * STEP, last)));
        load_keys(row);
      }
      // weights
      const bool mixed = k0 + STEP > w.open || k0 + STEP > w.hi || k0 < w.from;
      uint32_t p[NB][4], rest[NB][4];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        if constexpr (SIGHT) {
          float y[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = s[nb][i / 4][i % 4];
          shape_scores<FORM>(a, y, ref_of(top[nb]), slope[nb], (int32_t)(k0 + 4 * g) - pos[nb], [](int i) { return 16 * (i / 4) + i % 4; });
#pragma unroll
          for (int i = 0; i < 8; ++i) s[nb][i / 4][i % 4] = y[i];
        }
        if (mixed) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t key = k0 + 16 * i + 4 * g + j;
              if (key >= limit[nb] || (SIGHT && key < low[nb])) s[nb][i][j] = -INFINITY;
            }
        }
        float m = s[nb][0][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) m = fmaxf(m, s[nb][i / 4][i % 4]);
        if constexpr (SIGHT) m = max_over_16(max_over_32(m)) + ref_of(top[nb]);
        else m = a.c * max_over_16(max_over_32(m));
        if (__any(risen<DT>(m, top[nb]))) {
          const float t = follow<DT>(m, top[nb]), keep = __builtin_amdgcn_exp2f(top[nb] - t);
          if constexpr (SIGHT) {
            const float further = ref_of(t) - ref_of(top[nb]);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[nb][i / 4][i % 4] -= further;
          }
          top[nb] = t;
          sum[nb] *= keep;
#pragma unroll
          for (int e = 0; e < E; ++e) o[nb][e] *= keep;
        }
        float f[8], part = 0;  // of this step: one by one, small weights would be lost in a large sum
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          f[i] = __builtin_amdgcn_exp2f(SIGHT ? s[nb][i / 4][i % 4]
                                              : __builtin_fmaf(s[nb][i / 4][i % 4], a.c, -top[nb]));
          part += f[i];
        }
        sum[nb] += part;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[nb][i] = pair_of<DT>(f[2 * i], f[2 * i + 1]);
          if constexpr (SIGHT) {
            const typename DT::x2 taken = bits<typename DT::x2>(p[nb][i]);
            rest[nb][i] = pair_of<DT>(f[2 * i] - (float)taken[0], f[2 * i + 1] - (float)taken[1]);
          }
        }
      }
      if (k0 + STEP > w.hi) {
        // behind the end the last key's value is here again: its weight is 0, which an
        // infinity there would turn into NaN
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (k0 + 16 * (j / 4) + 4 * g + j % 4 >= w.hi) {
#pragma unroll
            for (int i = 0; i < VW; ++i) vr[j][i] = 0;
          }
      }
      if (differ(w, k0, STEP)) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int i = 0; i < VW; ++i) odd |= odd_pair(DT(), vr[j][i]);
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        u32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          v[j] = __builtin_amdgcn_perm(vr[2 * j + 1][e / 2], vr[2 * j][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          o[nb][e] = mfma_16x16x32(DT(), v, u32x4{p[nb][0], p[nb][1], p[nb][2], p[nb][3]}, o[nb][e]);
          if constexpr (SIGHT)
            o[nb][e] = mfma_16x16x32(DT(), v, u32x4{rest[nb][0], rest[nb][1], rest[nb][2], rest[nb][3]}, o[nb][e]);
        }
      }
      if (!more) break;
      k0 = next;
    }
  }
  if (__any(err != 0)) {
    if constexpr (SIGHT) err = w.s.error | seen_errors(a, w, lane);
    report(a.b, err);
  }
  bool again = differ(w) && odd;
  if constexpr (SIGHT) {  // an infinite value is NaN next to a rest of 0 or of the other sign
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) again |= o[nb][e][i] != o[nb][e][i];
  }
  if ((SIGHT || differ(w)) && __syncthreads_or(again)) {
    rows_one_by_one<DT, D, D>(a, w, wv, NW, lane);
    return;
  }

  // join the wavefronts, in their order
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    sum[nb] = sum_over_16(sum_over_32(sum[nb]));
    if (g == 0) {
      s_top[wv][16 * nb + n] = top[nb];
      s_sum[wv][16 * nb + n] = sum[nb];
    }
  }
  __syncthreads();
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    float t = NO_TOP;
#pragma unroll
    for (uint32_t i = 0; i < NW; ++i) t = fmaxf(t, s_top[i][16 * nb + n]);
    const float keep = __builtin_amdgcn_exp2f(top[nb] - t);
    if (nb) __syncthreads();  // the rows before have been read
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float* dst = &s_o[wv][n][(4 * g + i) * E];
#pragma unroll
      for (int e = 0; e < E; ++e) dst[e] = o[nb][e][i] * keep;
    }
    __syncthreads();
    const uint32_t rows = w.rows > 16u * nb ? min(16u, w.rows - 16u * nb) : 0u;
    // four elements a thread
    for (uint32_t x = tid; x < rows * (D / 4); x += 64 * NW) {
      const uint32_t r = x / (D / 4), d = 4 * (x % (D / 4)), rr = 16 * nb + r;
      float tt = NO_TOP;
#pragma unroll
      for (uint32_t i = 0; i < NW; ++i) tt = fmaxf(tt, s_top[i][rr]);
      float l = 0;
      f32x4 y{0, 0, 0, 0};
#pragma unroll
      for (uint32_t i = 0; i < NW; ++i) {
        l += s_sum[i][rr] * __builtin_amdgcn_exp2f(s_top[i][rr] - tt);
        y += *reinterpret_cast<const f32x4*>(&s_o[i][r][d]);
      }
      if (w.per_tile > 1) {
        const uint64_t at = ((uint64_t)w.item * a.kv_heads + w.kv) * a.tile_rows + rr;
        *reinterpret_cast<f32x4*>(a.part + at * D + d) = y;
        if (d == 0) a.part_ml[at] = float2{tt, l};
      } else {
        const RowAt at = row_at(a, w, rr);
        const bool none = row_keys(a, w, rr).none();
        const float inv = none ? 0.f : 1.f / l;
        if (none) y = f32x4{0, 0, 0, 0};
        const u32x2 h = {pair_of<DT>(y[0] * inv, y[1] * inv), pair_of<DT>(y[2] * inv, y[3] * inv)};
        *reinterpret_cast<u32x2*>(a.out.data + at.t * a.out.token + at.h * a.out.head + 2 * d) = h;
        if (d == 0) store_lse(a, at, tt, l, none);
      }
    }
  }
}

template <typename DT, int D, typename Args>
void launch(const Args& a, hipStream_t s) {
  const dim3 grid(a.items * a.kv_heads);
  if (a.tile_rows == 16) hipLaunchKernelGGL((attend_step_kernel<DT, D, 1, Args>), grid, dim3(64 * NW), 0, s, a);
  else hipLaunchKernelGGL((attend_step_kernel<DT, D, 2, Args>), grid, dim3(64 * NW), 0, s, a);
}
template <typename Args>
void launch(const Args& a, bool f16, uint32_t dim, hipStream_t s) {
  if (dim == 64) {
    if (f16) launch<F16, 64>(a, s);
    else launch<BF16, 64>(a, s);
  } else {
    if (f16) launch<F16, 128>(a, s);
    else launch<BF16, 128>(a, s);
  }
}

}  // namespace

void launch_attend_step(const AttendArgs& a, bool f16, uint32_t dim, hipStream_t s) { launch(a, f16, dim, s); }
void launch_attend_step(const SightArgs& a, bool f16, uint32_t dim, hipStream_t s) {
  Sight<UNKNOWN> x;  // bound by bytes: one kernel for every form
  static_cast<SightArgs&>(x) = a;
  launch(x, f16, dim, s);
}

}  // namespace mori
