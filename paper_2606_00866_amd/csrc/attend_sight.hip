// Writes down the tiles of a batch whose sequences have several, and their items.
//
// Without splits a tile is an item: a wavefront a tile, whose tokens (128 rows at most)
// are two reads a lane; 5 us for 650 tiles.  With splits, or where an order pays, there are
// 2048 tiles at most, and one workgroup more chooses the length of the runs and lists the items.
// Where there are few tiles it does the first part too: it checks the sequences and takes
// the tiles' keys.
//
// Items are listed longest tile first (by eighths of the longest), so the last to start are
// short: documents in 36 sequences 135 us so, 176 in the tiles' order; two prompts of 6000
// with documents 148 and 188, twelve of 900, capped, 94 and 112.
//
// The length of the runs.  An item's time is its steps and a fixed part of about three;
// 512 of them run at a time (two workgroups a CU), 256 of them in two thirds of the time.
// Rounds of the longest are one bound of the whole, all items' steps shared out and a fifth
// of an item, for the last to end, another; the lesser counts, so prompts, whose tiles see
// half of their keys at the mean, are not taken for as many long ones.  Capped, 3000 tokens
// in each of three sequences 302 us by the first bound alone and in the tiles' order; longest
// first 239 so, 240 with half of an item, 311 with three quarters; 50 sequences of 150
// behind 3000 468, 534 and 532; 36 of 650 with documents of 1500 222, 249 and 280; but 8 of
// 500 with these 114, 108 and 111.  Splitting at all costs the join, about two steps, and
// every 88 items one step to write and join 64 KiB of partial sums each (counting split
// tiles' items only splits too much: 282 us, in the tiles' order, where 244 are taken, for the
// first of these).  32 lengths from the shortest allowed to 15 times that are tried, two a
// wavefront, and the one with the least time is taken.  456 workgroups of 65 steps come out
// whole so, 155 us; 235 where 1536 workgroups were aimed at (three rounds and a bit, and
// 31 us of joins).  The kernel takes 5 to 7 us, 9 where it makes the tiles of four
// sequences of 430 tokens too.
#include "sight.h"

namespace mori {
namespace {

// The keys of a tile that starts at row0.
__device__ inline Union tile_union(const SightArgs& a, const Seq& s, uint32_t row0, uint32_t rows, uint32_t lane) {
  if (s.error) return Union{0, 0, 0xFFFFFFFFu, 0};
  return union_of(a, s, divide(row0, a.by_group), divide(row0 + rows - 1, a.by_group) + 1, lane);
}

__device__ inline uint32_t units_of(const SightArgs& a, uint32_t lo, uint32_t hi) {
  const uint32_t n = (hi - (lo & ~(a.align - 1)) + a.unit - 1) >> a.unit_log;
  return n ? n : 1u;  // an empty tile is an item too: its rows are 0
}

__global__ __launch_bounds__(256) void sight_tiles_kernel(SightArgs a) {
  const uint32_t lane = threadIdx.x & 63, tile = blockIdx.x * 4 + wave_index();
  if (tile >= a.tiles) return;
  AttendArgs whole = a;  // a tile is one run here
  whole.splits = 0;
  const Item it = find_item(whole, lane, [&](uint32_t first, uint32_t n, uint32_t) { return tile - first < n; });
  if (tile == 0 && it.bad) report(a.b, MORI_DEV_BAD_TOKENS);  // a lane knows of its own sequences
  uint4* const to = reinterpret_cast<uint4*>(a.tile + tile);
  if (!it.found) {
    if (lane == 0) to[2] = uint4{0, 0, 0, 0};
    return;
  }
  const SeqNumbers x = read_sequence(a.b, it.b);
  const Seq s = checked_sequence(a.b, SeqNumbers{same(x.lo), same(x.hi), same(x.len), same(x.p), same(x.first), same(x.last)});
  const uint32_t tiles = (s.n * a.group + a.tile_rows - 1) / a.tile_rows, back = tile - it.first;
  const uint32_t row0 = (tiles - 1 - back) * a.tile_rows, rows = min(a.tile_rows, s.n * a.group - row0);
  const Union u = tile_union(a, s, row0, rows, lane);
  if (lane) return;
  report(a.b, s.error);
  to[0] = uint4{u.lo, u.hi, u.from, u.open};
  to[1] = uint4{s.t0, s.n, s.len, s.tbl};
  to[2] = uint4{row0, tile, 1, 0x7FFFFFFFu};
}

// Up to so many tiles one workgroup does it all: 27.4 us for four sequences of nine tokens
// with a window and 50.7 for two of 300 so, 28.3 and 52.3 with two kernels.  Above, the tiles
// are taken by a kernel of their own: documents in 36 sequences 197 us so, 246 with one
// workgroup; 3 long and 17 short ones 271 and 305.
constexpr uint32_t FEW = 64;
constexpr uint32_t NT = 1024, WAVES = NT / 64, MOST = 2048, K = MOST / NT, KINDS = 8;

__device__ inline uint32_t scan_before(uint32_t v, uint32_t* s_wave, uint32_t* total) {
  const uint32_t lane = threadIdx.x & 63, wv = threadIdx.x >> 6, in = wave::incl_add(v);
  if (lane == 63) s_wave[wv] = in;
  __syncthreads();
  uint32_t before = in - v, all = 0;
#pragma unroll
  for (uint32_t i = 0; i < WAVES; ++i) {
    const uint32_t x = s_wave[i];
    before += i < wv ? x : 0;
    all += x;
  }
  *total = all;
  __syncthreads();
  return before;
}

__device__ inline uint32_t most_of(uint32_t v, uint32_t* s_wave) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) s_wave[threadIdx.x >> 6] = v;
  __syncthreads();
  uint32_t most = 0;
#pragma unroll
  for (uint32_t i = 0; i < WAVES; ++i) most = max(most, s_wave[i]);
  __syncthreads();
  return most;
}

// The tiles by this workgroup (FEW at most), their units and first rows in LDS; their number.
__device__ inline uint32_t write_tiles(const SightArgs& a, uint32_t* s_units, uint32_t* s_row0, uint32_t* s_wave) {
  __shared__ uint4 s_seq[FEW];  // t0, n, len, tbl
  __shared__ uint32_t s_tile0[FEW];
  const uint32_t tid = threadIdx.x, lane = tid & 63, wv = wave_index();
  // sequences: there are no more of them than tiles may be
  uint32_t have = 0, err = 0;
  if (tid < a.b.B) {
    const Seq q = checked_sequence(a.b, read_sequence(a.b, tid));
    err = q.error;
    s_seq[tid] = uint4{q.t0, q.n, q.len, q.tbl};  // len 0 where something is wrong: padding
    have = (q.n * a.group + a.tile_rows - 1) / a.tile_rows;
  }
  err = wave::all_or(err);
  if (lane == 0) report(a.b, err);
  uint32_t tiles;
  const uint32_t at = scan_before(have, s_wave, &tiles);
  tiles = min(tiles, a.tiles);  // more only where sequences overlap
  if (tid < a.b.B) s_tile0[tid] = at;
  __syncthreads();
  // tiles, a wavefront each
  for (uint32_t tile = wv; tile < tiles; tile += WAVES) {
    uint32_t lo = 0, hi = a.b.B - 1;  // the last sequence whose first tile is not behind this one
    while (lo < hi) {
      const uint32_t mid = (lo + hi + 1) / 2;
      if (same(s_tile0[mid]) <= tile) lo = mid;
      else hi = mid - 1;
    }
    const uint4 q = s_seq[lo];
    Seq s{};
    s.t0 = same(q.x);
    s.n = same(q.y);
    s.len = same(q.z);
    const uint32_t of = (s.n * a.group + a.tile_rows - 1) / a.tile_rows;
    const uint32_t row0 = (of - 1 - (tile - same(s_tile0[lo]))) * a.tile_rows;
    const Union u = tile_union(a, s, row0, min(a.tile_rows, s.n * a.group - row0), lane);
    if (lane == 0) {
      uint4* const to = reinterpret_cast<uint4*>(a.tile + tile);
      to[0] = uint4{u.lo, u.hi, u.from, u.open};
      to[1] = q;
      s_units[tile] = units_of(a, u.lo, u.hi);
      s_row0[tile] = row0;
    }
  }
  return tiles;
}

// READY: the tiles are written down already.
template <bool READY>
__global__ __launch_bounds__(NT) void sight_items_kernel(SightArgs a) {
  __shared__ uint32_t s_units[MOST], s_row0[MOST], s_wave[WAVES], s_run[WAVES];
  __shared__ uint32_t s_kind[KINDS * WAVES];
  __shared__ float s_cost[WAVES];
  const uint32_t tid = threadIdx.x, lane = tid & 63, wv = wave_index();
  uint32_t tiles;
  if constexpr (READY) {
    uint32_t mine = 0;
#pragma unroll
    for (uint32_t k = 0; k < K; ++k) {
      const uint32_t t = K * tid + k;
      if (t >= a.tiles) continue;
      const uint4* const at = reinterpret_cast<const uint4*>(a.tile + t);
      const uint4 x = at[0], z = at[2];
      s_units[t] = z.z ? units_of(a, x.x, x.y) : 0;
      s_row0[t] = z.x;
      mine += z.z;
    }
    scan_before(mine, s_wave, &tiles);
  } else {
    tiles = write_tiles(a, s_units, s_row0, s_wave);
    __syncthreads();
  }
  // the length of the runs
  uint32_t units[K], total;
#pragma unroll
  for (uint32_t k = 0; k < K; ++k) {
    const uint32_t t = K * tid + k;
    units[k] = t < tiles ? s_units[t] : 0;
  }
  scan_before(units[0] + units[1], s_wave, &total);
  const uint32_t least = max(a.least, (total + a.slots - 1) / a.slots);
  const uint32_t longest = most_of(max(units[0], units[1]), s_wave);
  float best = 3.0e38f;
  uint32_t run = a.splits ? least : max(longest, 1u);  // of an empty batch there is none
  for (uint32_t j = 2 * wv; a.splits && j < 2 * wv + 2; ++j) {
    const uint32_t c = (uint32_t)((float)least * __builtin_amdgcn_exp2f(0.125f * (float)j) + 0.999f);
    uint32_t n = 0;
    for (uint32_t t = lane; t < tiles; t += 64) n += (s_units[t] + c - 1) / c;
    n = wave::sum(n);
    const uint32_t groups = n * a.kv_heads, rest = groups % 512, steps = min(c, longest) + 3;
    // by their number, and by their steps and what the last ones take longer
    const float alike = (float)(groups / 512) + (rest == 0 ? 0.f : rest <= 256 ? 0.65f : 1.f);
    const float unlike = fmaxf((float)(total + 3 * n) / (float)steps * (float)a.kv_heads / 512.f + 0.2f, 1.f);
    const float rounds = groups > 512 ? fminf(alike, unlike) : alike;
    const float cost = rounds * (float)steps + (n > tiles ? 2.f + (float)groups / 88.f : 0.f);
    if (cost < best) {
      best = cost;
      run = c;
    }
  }
  if (lane == 0) {
    s_cost[wv] = best;
    s_run[wv] = run;
  }
  __syncthreads();
  best = s_cost[0];
  run = s_run[0];
  for (uint32_t i = 1; i < WAVES; ++i)
    if (s_cost[i] < best) {
      best = s_cost[i];
      run = s_run[i];
    }
  // items, those of longer tiles first: by eighths of the longest, else in order
  uint32_t runs[K], kind[K], at[K]{};
#pragma unroll
  for (uint32_t k = 0; k < K; ++k) {
    runs[k] = (units[k] + run - 1) / run;
    kind[k] = (longest - units[k]) * KINDS / max(longest, 1u);
  }
#pragma unroll
  for (uint32_t c = 0; c < KINDS; ++c) {
    uint32_t mine = 0;
#pragma unroll
    for (uint32_t k = 0; k < K; ++k) mine += kind[k] == c ? runs[k] : 0;
    const uint32_t in = wave::incl_add(mine);
    if (lane == 63) s_kind[c * WAVES + wv] = in;
    uint32_t before = in - mine;
#pragma unroll
    for (uint32_t k = 0; k < K; ++k) {
      if (kind[k] != c) continue;
      at[k] = before;
      before += runs[k];
    }
  }
  __syncthreads();
  static_assert(KINDS * WAVES == 128, "two a lane");
  const uint32_t x = s_kind[2 * lane], y = s_kind[2 * lane + 1], in = wave::incl_add(x + y), items = wave::lane63(in);
#pragma unroll
  for (uint32_t k = 0; k < K; ++k) {
    const uint32_t t = K * tid + k;
    // no runs: of no kind
    at[k] += (uint32_t)__shfl((int)(wv & 1 ? in - y : in - y - x), (int)(min(kind[k], KINDS - 1) * WAVES + wv) / 2);
    if (t < tiles) {
      reinterpret_cast<uint4*>(a.tile + t)[2] = uint4{s_row0[t], at[k], runs[k], run};
      for (uint32_t i = at[k]; i < min(at[k] + runs[k], a.items); ++i) a.list[i] = t;
    } else if (!READY && t < a.tiles) {
      reinterpret_cast<uint4*>(a.tile + t)[2] = uint4{0, 0, 0, 0};
    }
  }
  for (uint32_t i = items + tid; i < a.items; i += NT) a.list[i] = NO_TILE;
  if (tid == 0) *a.split = items > tiles;
}

// Joins the partial sums of the tiles that were split, in run order (as attend_join, but by
// tiles, each of which has runs of its own): a wavefront takes four rows of a tile and a
// key head, whose maxima and sums are on the way together.  Tiles of one run are left at
// once, after one read, and all are where none was split.  Bound by the partial sums' way
// through memory, and by the launch where few are split: 25 us for 3 long and 17 short
// sequences with documents, 55 where each token looked for its sequence and tile first;
// 15 and 30 us for 35000 rows of 64; 3.9 us where none is split.
constexpr uint32_t JOIN_ROWS = 16;  // of a workgroup
template <typename DT, int D>
__global__ __launch_bounds__(256) void sight_join_kernel(SightArgs a) {
  constexpr int W = D / 64, ROWS = JOIN_ROWS / 4;
  typedef float vec __attribute__((ext_vector_type(W)));
  if (!same(*a.split)) return;
  const uint32_t lane = threadIdx.x & 63, wv = wave_index();
  const uint32_t parts = a.tile_rows / JOIN_ROWS, y = blockIdx.x / parts, part = blockIdx.x - y * parts;
  const uint32_t tile = divide(y, a.by_kv);
  Work w{};
  w.kv = y - tile * a.kv_heads;
  const uint4* const at = reinterpret_cast<const uint4*>(a.tile + tile);
  const uint4 q = at[1], z = at[2];
  const uint32_t runs = same(z.z), first = same(z.y);
  if (runs < 2 || (uint64_t)first + runs > a.items) return;  // more items than there is room for: not run
  w.s.t0 = same(q.x);
  w.s.n = same(q.y);
  w.s.len = same(q.z);
  w.row0 = same(z.x);
  w.rows = min(a.tile_rows, w.s.n * a.group - w.row0);
  const uint32_t r0 = part * JOIN_ROWS + wv * ROWS;
  if (r0 >= w.rows) return;
  const uint64_t step = (uint64_t)a.kv_heads * a.tile_rows, at0 = ((uint64_t)first * a.kv_heads + w.kv) * a.tile_rows + r0;
  float2 ml[ROWS];
  Keys keys[ROWS];
#pragma unroll
  for (uint32_t i = 0; i < ROWS; ++i) {
    ml[i] = lane < runs ? a.part_ml[at0 + i + lane * step] : float2{NO_TOP, 0};
    keys[i] = row_keys(a, w, r0 + i);
  }
#pragma unroll
  for (uint32_t i = 0; i < ROWS; ++i) {
    if (r0 + i >= w.rows) break;
    float top = ml[i].x;
    for (uint32_t k = lane + 64; k < runs; k += 64) top = fmaxf(top, a.part_ml[at0 + i + k * step].x);
    top = max_over_16(max_over_32(top));
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    float l = 0;
    vec o = 0;
    for (uint32_t k0 = 0; k0 < runs; k0 += 64) {
      const uint32_t m = min(64u, runs - k0);
      if (k0) ml[i] = lane < m ? a.part_ml[at0 + i + (k0 + lane) * step] : float2{NO_TOP, 0};
      const float f = ml[i].x == NO_TOP ? 0.f : __builtin_amdgcn_exp2f(ml[i].x - top);
      l += f * ml[i].y;
      const uint64_t skip = __ballot(ml[i].x == NO_TOP);
      constexpr uint32_t U = 4;
      for (uint32_t k = 0; k < m; k += U) {
        vec v[U];
#pragma unroll
        for (uint32_t u = 0; u < U; ++u)  // past the last run it is read again
          v[u] = *reinterpret_cast<const vec*>(a.part + (at0 + i + (k0 + min(k + u, m - 1)) * step) * D + W * lane);
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
          if (k + u >= m || (skip >> (k + u) & 1)) continue;  // a run without keys
          o += v[u] * bits<float>((uint32_t)__builtin_amdgcn_readlane((int)bits<uint32_t>(f), (int)(k + u)));
        }
      }
    }
    l = sum_over_16(sum_over_32(l));
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) l += __shfl_xor(l, d);
    const float inv = 1.f / l;
    const RowAt row = row_at(a, w, r0 + i);
    const bool none = keys[i].none();
    typename DT::scalar* const out =
        reinterpret_cast<typename DT::scalar*>(a.out.data + row.t * a.out.token + row.h * a.out.head) + W * lane;
#pragma unroll
    for (int d = 0; d < W; ++d) out[d] = (typename DT::scalar)(none ? 0.f : o[d] * inv);
    if (lane == 0) store_lse(a, row, top, l, none);
  }
}

}  // namespace

void launch_sight_join(const SightArgs& a, bool f16, uint32_t dim, hipStream_t s) {
  const dim3 grid(a.tiles * a.kv_heads * (a.tile_rows / JOIN_ROWS));
  const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a); };
  if (f16) dim == 64 ? launch(sight_join_kernel<F16, 64>) : launch(sight_join_kernel<F16, 128>);
  else dim == 64 ? launch(sight_join_kernel<BF16, 64>) : launch(sight_join_kernel<BF16, 128>);
}

void launch_sight_tiles(const SightArgs& a, hipStream_t s) {
  if (a.list && a.tiles <= FEW) {
    hipLaunchKernelGGL(sight_items_kernel<false>, dim3(1), dim3(NT), 0, s, a);
    return;
  }
  hipLaunchKernelGGL(sight_tiles_kernel, dim3((a.tiles + 3) / 4), dim3(256), 0, s, a);
  if (a.list) hipLaunchKernelGGL(sight_items_kernel<true>, dim3(1), dim3(NT), 0, s, a);
}

}  // namespace mori
