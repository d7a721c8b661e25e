// Attention of many rows per key head (chunks, prompts), bound by the matrix rate.
//
// A workgroup takes 128 rows, 32 a wavefront, and walks the keys in steps of 64; keys and
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
//
// Why 128 rows: two workgroups fit a CU, one's products beside the other's weights.
// (64 rows a wavefront in one workgroup a CU, half the LDS reads, took the same time.)
//
// Three prompts of 19215 tokens in all (32 heads over 8 key heads of 128; 1.05
// TFLOP): 1070 to 1119 us, 937 to 979 TFLOP/s of the 1330 that a large product reaches;
// the matrix units are busy 44 to 49% of the cycles.  A part of it is the clock that the
// chip's power leaves: prompts of 20600 tokens take 1288 us on one card and 1470 on another,
// over a pool and queries of zeros 1064 and 1070; without the weights' arithmetic 1303 and
// 993 on the second.  So what does less work is faster and what only hides latency is not:
// reading operands of the scores six products ahead changed nothing, values four ahead,
// table entries looked up before the weights and not before the wait, and products at a
// higher priority 1% on chunks and 5% on mixed batches.  Chunks of four sequences (0.2
// TFLOP): 281 us, 702 TFLOP/s, with uneven last items and the join; decode steps and chunks
// mixed (32 sequences, 0.51 GB, 0.12 TFLOP): 258 us.
//
// With a sight (sight.h) a workgroup's keys are those its rows see; scores that are
// capped or biased cost what they add to the weights: prompts of 20600 tokens (1.25
// TFLOP) 1303 us with a window past all of them, 1440 with a bias, 1547 with a cap, 1748
// with both.  Prompts with documents take 571 to 636 us by the card, 500 over zeros, 463
// without the weights' arithmetic either; with a prefix and a bias 440 to 508, 401 and 308;
// capped chunks in a window 180 to 205, 165 and 119.
#include "sight.h"

namespace mori {
namespace {

constexpr uint32_t STEP = 64, NW = 4;
constexpr int V_AHEAD = 4;  // values read ahead of their products
// A wavefront's rows and its place in the loads.
template <int D, bool PAGED>
struct Tile {
  static constexpr uint32_t NT = 64 * NW, ROW = 2 * D, CH = D / 8;  // bytes and chunks of a row
  static constexpr uint32_t AREA = STEP * ROW;
  static constexpr uint32_t LD = STEP * CH / NT;  // chunks a thread loads of each
  static constexpr uint32_t RPL = NT / CH;        // rows of one load of the workgroup
  static constexpr uint32_t RPW = 64 / CH;        // and of a wavefront
  static constexpr int KS = D / 16, DB = D / 32;
  static constexpr int BETWEEN = KS / LD;         // steps of the scores from one load to the next

  u32x4 q[KS];
  f32x16 o[DB];
  float top, sum;
  uint32_t limit, wave_hi;  // end of a row's keys, of any row's
  uint32_t low, wave_lo;    // first of them
  int32_t pos;              // where the row stands
  float slope;
  bool odd;                     // a value that rows see in part is infinite or NaN
  uint32_t entry[LD], err;
  // Byte offsets of this thread's chunks from the first row of a load.  They stay
  // where they are: a register that held a load's address counts as busy until the
  // load is done, and these are never anything else.
  uint32_t k_off, v_off;

  __device__ __forceinline__ void place(const AttendArgs& a, uint32_t tid) {
    const uint32_t lr = tid / CH, lc = tid % CH, in_load = PAGED ? lr % RPW * a.b.row : 0;
    k_off = 16 * (lc ^ (D == 128 ? lr & 15 : (lr >> 1) & 7)) + in_load;
    v_off = 16 * (lc ^ (D == 128 ? (lr & 3) << 2 : ((lr >> 1) & 1) << 2)) + in_load;
  }

  // Table entries of the next loads' keys.
  __device__ __forceinline__ void find(const AttendArgs& a, const Work& w, uint32_t base, uint32_t tid) {
#pragma unroll
    for (uint32_t i = 0; i < LD; ++i) entry[i] = table_entry(a.b, w.s, min(base + i * RPL + tid / CH, w.hi - 1));
  }

  // Load i of the keys from `base` on.  A wavefront's rows lie in one page where RPW
  // divides the block (PAGED): their place is a scalar then.  Behind the end a load
  // takes rows that are not the sequence's (drop_tail) or the last group's again.
  __device__ __forceinline__ void fetch(const AttendArgs& a, const Work& w, uint32_t base, uint8_t* __restrict__ to_k,
                                        uint8_t* __restrict__ to_v, uint32_t tid, uint32_t wv, uint32_t i) {
    const uint32_t last = w.hi - 1;
    const uint8_t* const plane = a.b.plane + (uint64_t)w.kv * ROW;
    const uint8_t* at;
    if constexpr (PAGED)
      at = plane + row_bytes_at(a.b, min(base + i * RPL + wv * RPW, last / RPW * RPW), same(entry[i]), &err);
    else
      at = plane + (uint64_t)pool_row(a.b, min(base + i * RPL + tid / CH, last), entry[i], &err) * a.b.row;
    const uint8_t* bt = at + a.b.plane_bytes;
    if constexpr (PAGED) {  // a scalar and a 32-bit offset, not an address per lane
      at = reinterpret_cast<const uint8_t*>(wave::uniform(reinterpret_cast<uint64_t>(at)));
      bt = reinterpret_cast<const uint8_t*>(wave::uniform(reinterpret_cast<uint64_t>(bt)));
    }
    asm("" : "+v"(k_off), "+v"(v_off));  // 32-bit offsets as they are: not widened ahead of the loop
    const uint8_t *const ka = at + k_off, *const va = bt + v_off;
    to_lds(ka, to_k + (i * NT + wv * 64) * 16);
    to_lds(va, to_v + (i * NT + wv * 64) * 16);
  }
};

// The rows behind the end of the last step's values: zeros, so that weights of 0
// meet no infinity or NaN there, be it of a row that is not the sequence's or of the
// last one again.
template <typename T>
__device__ inline void drop_tail(const Work& w, uint8_t* area, uint32_t k0, uint32_t tid) {
  for (uint32_t i = 0; i < T::LD; ++i)
    if (k0 + i * T::RPL + tid / T::CH >= w.hi)
      *reinterpret_cast<u32x4*>(area + (i * T::NT + tid) * 16) = u32x4{0, 0, 0, 0};
  __syncthreads();
}

// The same for keys before the first that a row of the tile sees (a page's rows are
// loaded a few at a time).
template <typename T>
__device__ inline void drop_head(const Work& w, uint8_t* area, uint32_t k0, uint32_t tid) {
  for (uint32_t i = 0; i < T::LD; ++i)
    if (k0 + i * T::RPL + tid / T::CH < w.key0)
      *reinterpret_cast<u32x4*>(area + (i * T::NT + tid) * 16) = u32x4{0, 0, 0, 0};
  __syncthreads();
}

// One step of 64 keys: these taken from the one area, the next ones' loads set out for the other.
template <typename DT, int D, bool PAGED, typename Args>
__device__ __forceinline__ void step(const Args& a, const Work& w, Tile<D, PAGED>& x,
                                     const uint8_t* __restrict__ now_k, const uint8_t* __restrict__ now_v,
                                     uint8_t* __restrict__ then_k, uint8_t* __restrict__ then_v, uint32_t k0,
                                     uint32_t tid, uint32_t wv) {
  typedef Tile<D, PAGED> T;
  constexpr bool SIGHT = IsSight<Args>::value;
  constexpr int FORM = IsSight<Args>::FORM;
  constexpr bool SHAPED = FORM != 0;  // scores are more than products with the scale
  constexpr uint32_t NT = T::NT, ROW = T::ROW, LD = T::LD;
  constexpr int KS = T::KS, DB = T::DB;
  const uint32_t lane = tid & 63, n = lane & 31, h = lane >> 5;
  // LDS addresses of a lane's reads
  const uint32_t kx = D == 128 ? n & 15 : (n >> 1) & 7;
  const uint32_t vrow = 4 * h + ((lane >> 2) & 3);
  const uint32_t vx = D == 128 ? (vrow & 3) << 2 : ((vrow >> 1) & 1) << 2;
  const uint32_t vc = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), vsub = 8 * (lane & 1);
  const uint32_t next = min(k0 + STEP, w.hi - 1);  // behind the last step the last key again, for nothing
  const bool mixed = k0 + STEP > w.open || k0 + STEP > w.hi || k0 < w.from;
  const bool here = k0 < x.wave_hi && (!SIGHT || k0 + STEP > x.wave_lo);
  if (differ(w, k0, STEP)) {
    for (uint32_t i = 0; i < LD; ++i) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(now_v + (i * NT + tid) * 16);
      for (int j = 0; j < 4; ++j) x.odd |= odd_pair(DT(), v[j]);
    }
  }
  if (here) {
    const uint8_t* const ks = now_k + n * ROW;
    const uint8_t* const vs = now_v + vrow * ROW + vsub;
    f32x16 s[2];
#pragma unroll
    for (int i = 0; i < 16; ++i) s[0][i] = s[1][i] = 0;
    __builtin_amdgcn_s_setprio(1);  // the products go first where both wavefronts of a SIMD could
#pragma unroll
    for (int k = 0; k < KS; ++k) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const u32x4 kr = *reinterpret_cast<const u32x4*>(ks + kb * 32 * ROW + (((2 * k + h) ^ kx) << 4));
        s[kb] = mfma_32x32x16(DT(), kr, x.q[k], s[kb]);
      }
      // the next step's loads, a few at a time: issued at once they hold the wavefront up
      if (k % T::BETWEEN == 0) x.fetch(a, w, next, then_k, then_v, tid, wv, k / T::BETWEEN);
    }
    __builtin_amdgcn_s_setprio(0);
    x.find(a, w, k0 + 2 * STEP, tid);  // behind the last use of what was found before, well ahead of the wait
    // the first values on the way behind the weights
    const auto value = [&](int i) {  // of 16 keys, 32 elements
      const uint8_t* at = vs + 16 * (i / DB) * ROW + (((4 * (i % DB) + vc) ^ vx) << 4);
      const u32x2 lo = read_tr(at), hi = read_tr(at + 8 * ROW);
      return u32x4{lo[0], lo[1], hi[0], hi[1]};
    };
    u32x4 v[V_AHEAD];
#pragma unroll
    for (int i = 0; i < V_AHEAD; ++i) v[i] = value(i);
    __builtin_amdgcn_sched_barrier(0);
    uint32_t p[16];
    if constexpr (SHAPED) {
      float y[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) y[i] = s[i / 16][i % 16];
      shape_scores<FORM>(a, y, ref_of(x.top), x.slope, (int32_t)(k0 + 4 * h) - x.pos,
                   [](int i) { return 32 * (i / 16) + 8 * (i % 16 / 4) + i % 4; });
#pragma unroll
      for (int i = 0; i < 32; ++i) s[i / 16][i % 16] = y[i];
    }
    if (mixed) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint32_t key = k0 + 32 * kb + 8 * (i / 4) + 4 * h + i % 4;
          if (SIGHT ? key - x.low >= x.limit - x.low : key >= x.limit) s[kb][i] = -INFINITY;
        }
    }
    float m = s[0][0];
#pragma unroll
    for (int i = 1; i < 32; ++i) m = fmaxf(m, s[i / 16][i % 16]);
    if constexpr (SHAPED) m = max_over_32(m) + ref_of(x.top);
    else m = a.c * max_over_32(m);
    if (__any(risen<DT>(m, x.top))) {
      const float t = follow<DT>(m, x.top), keep = __builtin_amdgcn_exp2f(x.top - t);
      if constexpr (SHAPED) {
        const float further = ref_of(t) - ref_of(x.top);
#pragma unroll
        for (int i = 0; i < 32; ++i) s[i / 16][i % 16] -= further;
      }
      x.top = t;
      x.sum *= keep;
#pragma unroll
      for (int d = 0; d < DB; ++d) x.o[d] *= keep;
    }
    float part = 0;  // of this step: one by one, small weights would be lost in a large sum
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float y0 = s[i / 8][2 * i % 16], y1 = s[i / 8][2 * i % 16 + 1];
      const float f0 = __builtin_amdgcn_exp2f(SHAPED ? y0 : __builtin_fmaf(y0, a.c, -x.top));
      const float f1 = __builtin_amdgcn_exp2f(SHAPED ? y1 : __builtin_fmaf(y1, a.c, -x.top));
      part += f0 + f1;
      p[i] = pair_of<DT>(f0, f1);
    }
    x.sum += part;
    __builtin_amdgcn_s_setprio(1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 4 * DB; ++i) {
      const int t = i / DB, d = i % DB;
      x.o[d] = mfma_32x32x16(DT(), v[i % V_AHEAD], u32x4{p[4 * t], p[4 * t + 1], p[4 * t + 2], p[4 * t + 3]}, x.o[d]);
      if (i + V_AHEAD < 4 * DB) v[i % V_AHEAD] = value(i + V_AHEAD);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
  }
  if (!here) {
#pragma unroll
    for (uint32_t i = 0; i < LD; ++i) x.fetch(a, w, next, then_k, then_v, tid, wv, i);
    x.find(a, w, k0 + 2 * STEP, tid);
  }
}

template <typename DT, int D, bool PAGED, typename Args>
__global__ __launch_bounds__(64 * NW, 2) void attend_tile_kernel(Args a) {
  typedef Tile<D, PAGED> T;
  constexpr bool SIGHT = IsSight<Args>::value;
  constexpr int KS = T::KS, DB = T::DB;
  // Arrays of their own, and the loop written out for both: a read of the one area
  // does not wait for loads into another only where the compiler can tell them apart.
  __shared__ __align__(256) uint8_t s_k0[T::AREA], s_k1[T::AREA];
  __shared__ __align__(256) uint8_t s_v0[T::AREA], s_v1[T::AREA];
  const uint32_t tid = threadIdx.x, lane = tid & 63, wv = wave_index();
  const uint32_t n = lane & 31, h = lane >> 5;
  Work w;
  if constexpr (SIGHT) w = tile_work(a, blockIdx.x);
  else w = work_of(a, blockIdx.x, lane);
  if (!w.some) return;
  T x;
  x.err = w.s.error;
  x.odd = false;
  x.place(a, tid);

  if (w.lo < w.hi) {  // the first keys on the way, then the queries
    x.find(a, w, w.lo, tid);
#pragma unroll
    for (uint32_t i = 0; i < T::LD; ++i) x.fetch(a, w, w.lo, s_k0, s_v0, tid, wv, i);
    x.find(a, w, w.lo + STEP, tid);
  }
  // rows: the wavefront's are 32 * wv + n
  const uint32_t r = 32 * wv + n;
  const Keys keys = row_keys(a, w, r);
  x.limit = min(keys.hi, w.hi);
  const RowAt mine = row_at(a, w, min(r, w.rows - 1));
  const u32x4* src = reinterpret_cast<const u32x4*>(q_row(a, mine) + 16 * h);
  if constexpr (SIGHT) {
    x.low = min(keys.lo, x.limit);
    x.pos = w.s.position(mine.t - w.s.t0);
    x.slope = slope_of(a, mine.h);
    x.wave_lo = wave_min(x.low < x.limit ? x.low : 0xFFFFFFFFu);
  }
#pragma unroll
  for (int k = 0; k < KS; ++k) x.q[k] = q_signed(a, src[2 * k]);
  x.top = NO_TOP;
  x.sum = 0;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) x.o[d][i] = 0;
  x.wave_hi = x.limit;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) x.wave_hi = max(x.wave_hi, (uint32_t)__shfl_xor((int)x.wave_hi, d));
  x.wave_hi = same(x.wave_hi);

  if (w.lo < w.hi) {
    wait_loads();
    __syncthreads();
    const auto turn = [&](uint8_t* now_k, uint8_t* now_v, uint8_t* then_k, uint8_t* then_v, uint32_t k0) {
      if (k0 + STEP > w.hi) drop_tail<T>(w, now_v, k0, tid);
      if (SIGHT && k0 < w.key0) drop_head<T>(w, now_v, k0, tid);
      step<DT>(a, w, x, now_k, now_v, then_k, then_v, k0, tid, wv);
      wait_loads();
      __syncthreads();
    };
    for (uint32_t k0 = w.lo;;) {
      turn(s_k0, s_v0, s_k1, s_v1, k0);
      if ((k0 += STEP) >= w.hi) break;
      turn(s_k1, s_v1, s_k0, s_v0, k0);
      if ((k0 += STEP) >= w.hi) break;
    }
  }
  if (__any(x.err != 0)) {
    if constexpr (SIGHT) x.err = seen_errors(a, w, lane);
    report(a.b, x.err);
  }
  if (differ(w) && __syncthreads_or(x.odd)) {
    rows_one_by_one<DT, D, D>(a, w, wv, NW, lane);
    return;
  }

  const float l = sum_over_32(x.sum);
  if (r >= w.rows) return;
  if (w.per_tile > 1) {
    const uint64_t at = ((uint64_t)w.item * a.kv_heads + w.kv) * a.tile_rows + r;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(a.part + at * D + 32 * d + 8 * i + 4 * h) =
            f32x4{x.o[d][4 * i], x.o[d][4 * i + 1], x.o[d][4 * i + 2], x.o[d][4 * i + 3]};
    if (h == 0) a.part_ml[at] = float2{x.top, l};
  } else {
    const RowAt at = row_at(a, w, r);
    const bool none = row_keys(a, w, r).none();
    const float inv = 1.f / l;
    uint8_t* out = a.out.data + at.t * a.out.token + at.h * a.out.head;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u32x2 y = {pair_of<DT>(x.o[d][4 * i] * inv, x.o[d][4 * i + 1] * inv),
                         pair_of<DT>(x.o[d][4 * i + 2] * inv, x.o[d][4 * i + 3] * inv)};
        *reinterpret_cast<u32x2*>(out + 2 * (32 * d + 8 * i + 4 * h)) = none ? u32x2{0, 0} : y;
      }
    if (h == 0) store_lse(a, at, x.top, l, none);
  }
}

template <typename DT, int D, typename Args>
void launch(const Args& a, hipStream_t s) {
  const dim3 grid(a.items * a.kv_heads), block(64 * NW);
  if (a.b.bt % Tile<D, true>::RPW == 0) hipLaunchKernelGGL((attend_tile_kernel<DT, D, true, Args>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((attend_tile_kernel<DT, D, false, Args>), grid, block, 0, s, a);
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

void launch_attend_tile(const AttendArgs& a, bool f16, uint32_t dim, hipStream_t s) { launch(a, f16, dim, s); }
void launch_attend_tile(const SightArgs& a, bool f16, uint32_t dim, hipStream_t s) {
  with_form(a, [&](const auto& x) { launch(x, f16, dim, s); });
}

}  // namespace mori
