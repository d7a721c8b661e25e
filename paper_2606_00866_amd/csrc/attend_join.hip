// Joins the partial sums of tiles whose keys were split into runs:
//   out = sum_i 2^(top_i - top) part_i / sum_i 2^(top_i - top) sum_i, in run order.
// A token whose tile was one run has nothing to join.  Bound by reading the partial
// sums (2 KiB a row and run where rows are latent): 18 us where 250 items of 128
// latent rows are joined, 30 for 25856 rows of mixed chunks; 5 to 9 us for the rows of
// one to eight sequences, where it is the launch, the search and two dependent reads,
// and 11 us for 24128 latent rows of which none was split (it is launched where tiles
// may be split, which only the device knows).
#include <algorithm>
#include <type_traits>

#include "attend.h"

namespace mori {
namespace {

// WPH wavefronts share a head's runs (8 when there are few rows, so that all runs
// are on the way at once), else a wavefront takes `some` heads of a token.
template <typename DT, int DV, int NW, int WPH>
__global__ __launch_bounds__(64 * NW) void attend_join_kernel(AttendArgs a, uint32_t some) {
  constexpr int W = DV / 64;                // elements of a lane
  typedef float vec __attribute__((ext_vector_type(W)));
  __shared__ float s_y[WPH > 1 ? NW : 1][DV], s_l[NW];
  const uint32_t lane = threadIdx.x & 63, wv = wave_index();
  const uint32_t heads_wg = WPH > 1 ? 1 : NW * some, per_token = (a.heads + heads_wg - 1) / heads_wg;
  const uint32_t t = blockIdx.x / per_token, h0 = (blockIdx.x - t * per_token) * heads_wg + (WPH > 1 ? 0 : wv * some);
  const Item it = find_item(a, lane, [&](uint32_t, uint32_t n, uint32_t b) {
    return n && a.b.seq_off[b] <= t && t < a.b.seq_off[b + 1];
  });
  if (!it.found || it.per_tile < 2) return;
  const uint32_t t0 = same(a.b.seq_off[it.b]), n = same(a.b.seq_off[it.b + 1]) - t0;
  const Seq s = sequence(a.b, it.b);
  const bool none = s.position(t - s.t0) < 0;
  const uint32_t tiles = (n * a.group + a.tile_rows - 1) / a.tile_rows;
  const uint64_t step = (uint64_t)a.kv_heads * a.tile_rows;
  const uint32_t runs = it.per_tile;
  const uint32_t r0 = WPH > 1 ? (uint32_t)((uint64_t)runs * wv / NW) : 0;
  const uint32_t r1 = WPH > 1 ? (uint32_t)((uint64_t)runs * (wv + 1) / NW) : runs;
  for (uint32_t h = h0; h < min(h0 + some, a.heads); ++h) {
    const uint32_t kv = divide(h, a.by_group), x = (t - t0) * a.group + (h - kv * a.group);
    const uint32_t tile = x / a.tile_rows;
    const uint64_t item = it.first + (uint64_t)(tiles - 1 - tile) * it.per_tile;
    if (item + it.per_tile > a.items) continue;  // sequences that overlap: more items than tokens give, which were not run
    const uint64_t at0 = (item * a.kv_heads + kv) * a.tile_rows + (x - tile * a.tile_rows);

    float2 first{NO_TOP, 0};
    if (lane < runs) first = a.part_ml[at0 + lane * step];
    float top = first.x;
    for (uint32_t i = lane + 64; i < runs; i += 64) top = fmaxf(top, a.part_ml[at0 + i * step].x);
    top = max_over_16(max_over_32(top));
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    float l = 0;
    vec y = 0;
    for (uint32_t i0 = r0; i0 < r1; i0 += 64) {
      const uint32_t m = min(64u, r1 - i0);
      float2 ml{NO_TOP, 0};
      if (WPH == 1 && i0 == 0) ml = first;
      else if (lane < m) ml = a.part_ml[at0 + (i0 + lane) * step];
      const float f = ml.x == NO_TOP ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
      l += f * ml.y;
      const uint64_t skip = __ballot(ml.x == NO_TOP);
      const auto add = [&](auto at_once) {  // runs whose rows are on the way at a time
        constexpr uint32_t U = decltype(at_once)::value;
        for (uint32_t i = 0; i < m; i += U) {
          vec v[U];
#pragma unroll
          for (uint32_t u = 0; u < U; ++u)
            v[u] = *reinterpret_cast<const vec*>(a.part + (at0 + (i0 + min(i + u, m - 1)) * step) * DV + W * lane);
#pragma unroll
          for (uint32_t u = 0; u < U; ++u) {
            if (i + u >= m || (skip >> (i + u) & 1)) continue;  // a run without keys
            y += v[u] * bits<float>((uint32_t)__builtin_amdgcn_readlane((int)bits<uint32_t>(f), (int)(i + u)));
          }
        }
      };
      // past the last run it is read again: few runs take the short form
      if (WPH == 1 && m <= 4) add(std::integral_constant<uint32_t, 4>());
      else add(std::integral_constant<uint32_t, (W > 2 ? 8 : 16)>());
    }
    l = sum_over_16(sum_over_32(l));
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) l += __shfl_xor(l, d);
    if constexpr (WPH > 1) {
#pragma unroll
      for (int d = 0; d < W; ++d) s_y[wv][W * lane + d] = y[d];
      if (lane == 0) s_l[wv] = l;
      __syncthreads();
      if (wv) return;
      l = 0;
#pragma unroll
      for (uint32_t i = 0; i < NW; ++i) l += s_l[i];
#pragma unroll
      for (int d = 0; d < W; ++d) {
        y[d] = 0;
#pragma unroll
        for (uint32_t i = 0; i < NW; ++i) y[d] += s_y[i][W * lane + d];
      }
    }
    const float inv = 1.f / l;
    typename DT::scalar* out =
        reinterpret_cast<typename DT::scalar*>(a.out.data + t * a.out.token + h * a.out.head) + W * lane;
#pragma unroll
    for (int d = 0; d < W; ++d) out[d] = (typename DT::scalar)(none ? 0.f : y[d] * inv);
    if (lane == 0) store_lse(a, RowAt{t, h}, top, l, none);
  }
}

template <typename DT, int DV>
void launch(const AttendArgs& a, hipStream_t s) {
  // Few rows: a workgroup each, so that all of their runs are read at once.  Else as many
  // wavefronts as the chip holds: each finds its sequence once for all of its heads
  // (1610 tokens, 32 heads: 302 us for the attention with one head each, 287 so).
  const uint64_t rows = (uint64_t)a.b.T * a.heads;
  if (rows <= 1024) {
    hipLaunchKernelGGL((attend_join_kernel<DT, DV, 8, 8>), dim3((uint32_t)rows), dim3(512), 0, s, a, 1u);
  } else {
    const uint32_t most = (uint32_t)std::min<uint64_t>((rows + 8191) / 8192, (a.heads + 3) / 4);
    const uint32_t per_token = (a.heads + 4 * most - 1) / (4 * most);
    const uint32_t some = (a.heads + 4 * per_token - 1) / (4 * per_token);  // the same for each
    hipLaunchKernelGGL((attend_join_kernel<DT, DV, 4, 1>), dim3(a.b.T * per_token), dim3(256), 0, s, a, some);
  }
}
template <typename DT>
void launch(const AttendArgs& a, uint32_t value, hipStream_t s) {
  if (value == 64) launch<DT, 64>(a, s);
  else if (value == 128) launch<DT, 128>(a, s);
  else launch<DT, 512>(a, s);
}

}  // namespace

void launch_attend_join(const AttendArgs& a, bool f16, uint32_t value, hipStream_t s) {
  if (f16) launch<F16>(a, value, s);
  else launch<BF16>(a, value, s);
}

}  // namespace mori
