// Writes down the tiles of a batch: which keys each one's rows see together and which all
// of them see.  A wavefront a tile; a tile's tokens (128 rows at most) are two reads a
// lane.  Without splits a tile is an item; with them the attention's wavefronts and the
// join's scan these lines for theirs.
#include "sight.h"

namespace mori {
namespace {

__global__ __launch_bounds__(256) void sight_tiles_kernel(SightArgs a) {
  const uint32_t lane = threadIdx.x & 63, tile = blockIdx.x * 4 + wave_index();
  if (tile >= a.tiles) return;
  AttendArgs whole = a;  // a tile is one run here
  whole.splits = 0;
  const Item it = find_item(whole, lane, [&](uint32_t first, uint32_t n, uint32_t) { return tile - first < n; });
  if (tile == 0 && it.bad && lane == 0) report(a.b, MORI_DEV_BAD_TOKENS);
  if (!it.found) {
    if (lane == 0) a.span[tile] = uint2{1, 0};
    return;
  }
  const SeqNumbers x = read_sequence(a.b, it.b);
  const Seq s = checked_sequence(a.b, SeqNumbers{same(x.lo), same(x.hi), same(x.len), same(x.p), same(x.first), same(x.last)});
  const uint32_t tiles = (s.n * a.group + a.tile_rows - 1) / a.tile_rows, back = tile - it.first;
  const uint32_t row0 = (tiles - 1 - back) * a.tile_rows, rows = min(a.tile_rows, s.n * a.group - row0);
  Union u{0, 0, 0, 0};
  if (!s.error) u = union_of(a, s, divide(row0, a.by_group), divide(row0 + rows - 1, a.by_group) + 1, lane);
  if (lane) return;
  a.span[tile] = uint2{u.lo, u.hi};
  a.tile[tile] = uint4{u.from, u.open, it.b, row0};
  if (back == 0) a.seq_tile[it.b] = it.first;
}

}  // namespace

void launch_sight_tiles(const SightArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(sight_tiles_kernel, dim3((a.tiles + 3) / 4), dim3(256), 0, s, a);
}

}  // namespace mori
