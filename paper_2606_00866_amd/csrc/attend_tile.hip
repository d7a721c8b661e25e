// Attention of many rows per key head (chunks, prompts), bound by the matrix rate.
//
// A workgroup takes NW * 32 * QB rows and walks the keys in steps of 64; keys and
// values of a step are staged in LDS, two steps' worth, so that the next step's
// loads run behind this one's products.
//   scores   S^T = K Q^T, 32x32x16: a wavefront's rows are the columns, so a row's
//            scores lie in two lanes (l, l ^ 32).
//   values   O^T += V^T P^T: the weights leave the score product in lanes (row, h)
//            for keys 4 h .. 4 h + 3 of each 8, which is taken as the product's k
//            order, so they need no exchange; the values come from LDS through
//            transposing reads in that order.
// LDS rows are whole pool rows with their 16-B chunks permuted (the loads go
// straight to LDS, so the permutation is in the address each lane loads from):
// key chunks by the row, so that the lanes of a score read, which want the same
// chunk of consecutive rows, spread over the banks; value chunks by 64 B, so that
// the four rows of a transposing read do.
#include "attend.h"

namespace mori {
namespace {

constexpr uint32_t STEP = 64;
template <typename DT, int D, int NW, int QB>
__global__ __launch_bounds__(64 * NW, QB == 1 && NW == 4 ? 2 : 1) void attend_tile_kernel(AttendArgs a) {
  constexpr uint32_t NT = 64 * NW, ROW = 2 * D, CH = D / 8;  // bytes and chunks of a row
  constexpr uint32_t TILE = STEP * ROW;
  constexpr uint32_t LD = STEP * CH / NT;  // chunks a thread loads of each
  constexpr uint32_t RPL = NT / CH;        // rows of one load of the workgroup
  constexpr int KS = D / 16, DB = D / 32;
  __shared__ __align__(256) uint8_t s_k[2][TILE];
  __shared__ __align__(256) uint8_t s_v[2][TILE];
  const uint32_t tid = threadIdx.x, lane = tid & 63, wv = wave_index();
  const uint32_t n = lane & 31, h = lane >> 5;
  const Work w = work_of(a, blockIdx.x, lane);
  if (!w.some) return;
  uint32_t err = w.s.error;
  const uint32_t last = w.hi - 1;

  // rows: block qb of the wavefront is rows 32 * (wv * QB + qb) + n
  u32x4 q[QB][KS];
  uint32_t limit[QB], wave_hi = 0;
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const uint32_t r = 32 * (wv * QB + qb) + n;
    limit[qb] = min(row_limit(a, w, r), w.hi);
    const u32x4* src = reinterpret_cast<const u32x4*>(q_row(a, row_at(a, w, min(r, w.rows - 1))) + 16 * h);
#pragma unroll
    for (int k = 0; k < KS; ++k) q[qb][k] = q_signed(a, src[2 * k]);
    wave_hi = max(wave_hi, limit[qb]);
  }
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) wave_hi = max(wave_hi, (uint32_t)__shfl_xor((int)wave_hi, d));
  wave_hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)wave_hi);
  f32x16 o[QB][DB];
  float top[QB], sum[QB];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    top[qb] = NO_TOP;
    sum[qb] = 0;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[qb][d][i] = 0;
  }

  bool odd = false;  // a value that rows see in part is infinite or NaN
  if (w.lo < w.hi) {
    // this thread's part of a load: row and permuted chunk
    const uint32_t lr = tid / CH, lc = tid % CH;
    const uint32_t swk = D == 128 ? lr & 15 : (lr >> 1) & 7;
    const uint32_t swv = D == 128 ? (lr & 3) << 2 : ((lr >> 1) & 1) << 2;
    const uint8_t* const kp = a.b.plane + (uint64_t)w.kv * ROW + 16 * (lc ^ swk);
    const uint8_t* const vp = a.b.plane + a.b.plane_bytes + (uint64_t)w.kv * ROW + 16 * (lc ^ swv);
    const auto key_of = [&](uint32_t base, uint32_t i) { return min(base + i * RPL + lr, last); };
    uint32_t entry[LD];
    const auto find = [&](uint32_t base) {
#pragma unroll
      for (uint32_t i = 0; i < LD; ++i) entry[i] = table_entry(a.b, w.s, key_of(base, i));
    };
    const auto fetch = [&](uint32_t base, uint32_t buf) {
#pragma unroll
      for (uint32_t i = 0; i < LD; ++i) {
        const uint64_t at = (uint64_t)pool_row(a.b, key_of(base, i), entry[i], &err) * a.b.row;
        to_lds(kp + at, &s_k[buf][(i * NT + wv * 64) * 16]);
        to_lds(vp + at, &s_v[buf][(i * NT + wv * 64) * 16]);
      }
    };
    // LDS addresses of a lane's reads
    const uint32_t kx = D == 128 ? n & 15 : (n >> 1) & 7;
    const uint32_t vrow = 4 * h + ((lane >> 2) & 3);
    const uint32_t vx = D == 128 ? (vrow & 3) << 2 : ((vrow >> 1) & 1) << 2;
    const uint32_t vc = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), vsub = 8 * (lane & 1);

    find(w.lo);
    fetch(w.lo, 0);
    find(min(w.lo + STEP, last));
    wait_loads();
    __syncthreads();
    uint32_t buf = 0;
    for (uint32_t k0 = w.lo; k0 < w.hi; k0 += STEP, buf ^= 1) {
      if (k0 + STEP < w.hi) {
        fetch(k0 + STEP, buf ^ 1);
        find(min(k0 + 2 * STEP, last));
      }
      const bool mixed = k0 + STEP > w.open || k0 + STEP > w.hi;
      if (k0 + STEP > w.open && w.open < w.hi) {
        for (uint32_t i = 0; i < LD; ++i) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(&s_v[buf][(i * NT + tid) * 16]);
          for (int j = 0; j < 4; ++j) odd |= odd_pair(DT(), x[j]);
        }
      }
      if (k0 < wave_hi) {
        const uint8_t* const ks = s_k[buf] + n * ROW;
        const uint8_t* const vs = s_v[buf] + vrow * ROW + vsub;
        f32x16 s[QB][2];
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[qb][kb][i] = 0;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) {
            const u32x4 kr = *reinterpret_cast<const u32x4*>(ks + kb * 32 * ROW + (((2 * k + h) ^ kx) << 4));
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) s[qb][kb] = mfma_32x32x16(DT(), kr, q[qb][k], s[qb][kb]);
          }
        }
        uint32_t p[QB][16];
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          if (mixed) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
              for (int i = 0; i < 16; ++i)
                if (k0 + 32 * kb + 8 * (i / 4) + 4 * h + i % 4 >= limit[qb]) s[qb][kb][i] = -INFINITY;
          }
          float m = s[qb][0][0];
#pragma unroll
          for (int i = 1; i < 32; ++i) m = fmaxf(m, s[qb][i / 16][i % 16]);
          m = a.c * max_over_32(m);
          if (__any(m > top[qb] + RISE)) {
            const float t = fmaxf(top[qb], m), keep = __builtin_amdgcn_exp2f(top[qb] - t);
            top[qb] = t;
            sum[qb] *= keep;
#pragma unroll
            for (int d = 0; d < DB; ++d) o[qb][d] *= keep;
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float f0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[qb][i / 8][2 * i % 16], a.c, -top[qb]));
            const float f1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[qb][i / 8][2 * i % 16 + 1], a.c, -top[qb]));
            sum[qb] += f0 + f1;
            p[qb][i] = pair_of<DT>(f0, f1);
          }
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
          for (int d = 0; d < DB; ++d) {
            const uint8_t* at = vs + 16 * t * ROW + (((4 * d + vc) ^ vx) << 4);
            const u32x2 lo = read_tr(at), hi = read_tr(at + 8 * ROW);
            const u32x4 v = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
            for (int qb = 0; qb < QB; ++qb)
              o[qb][d] = mfma_32x32x16(DT(), v, u32x4{p[qb][4 * t], p[qb][4 * t + 1], p[qb][4 * t + 2], p[qb][4 * t + 3]},
                                       o[qb][d]);
          }
        }
      }
      wait_loads();
      __syncthreads();
    }
  }
  if (__any(err != 0)) report(a.b, err);
  if (w.open < w.hi && __syncthreads_or(odd)) {
    rows_one_by_one<DT, D, D>(a, w, wv, NW, lane);
    return;
  }

#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const float l = sum_over_32(sum[qb]);
    const uint32_t r = 32 * (wv * QB + qb) + n;
    if (r >= w.rows) continue;
    if (w.per_tile > 1) {
      const uint64_t at = ((uint64_t)w.item * a.kv_heads + w.kv) * a.tile_rows + r;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<f32x4*>(a.part + at * D + 32 * d + 8 * i + 4 * h) =
              f32x4{o[qb][d][4 * i], o[qb][d][4 * i + 1], o[qb][d][4 * i + 2], o[qb][d][4 * i + 3]};
      if (h == 0) a.part_ml[at] = float2{top[qb], l};
    } else {
      const RowAt at = row_at(a, w, r);
      const bool none = row_limit(a, w, r) == 0;
      const float inv = 1.f / l;
      uint8_t* out = a.out.data + at.t * a.out.token + at.h * a.out.head;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const u32x2 y = {pair_of<DT>(o[qb][d][4 * i] * inv, o[qb][d][4 * i + 1] * inv),
                           pair_of<DT>(o[qb][d][4 * i + 2] * inv, o[qb][d][4 * i + 3] * inv)};
          *reinterpret_cast<u32x2*>(out + 2 * (32 * d + 8 * i + 4 * h)) = none ? u32x2{0, 0} : y;
        }
      if (h == 0) store_lse(a, at, top[qb], l, none);
    }
  }
}

template <typename DT, int D>
void launch(const AttendArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((attend_tile_kernel<DT, D, 4, 1>), dim3(a.items * a.kv_heads), dim3(256), 0, s, a);
}

}  // namespace

void launch_attend_tile(const AttendArgs& a, bool f16, uint32_t dim, hipStream_t s) {
  if (dim == 64) {
    if (f16) launch<F16, 64>(a, s);
    else launch<BF16, 64>(a, s);
  } else {
    if (f16) launch<F16, 128>(a, s);
    else launch<BF16, 128>(a, s);
  }
}

}  // namespace mori
