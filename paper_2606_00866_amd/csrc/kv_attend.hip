// Attention of a batch's new tokens over their programs' pages: host side.
//
//   s_j = scale * q . k_j for the program's tokens j up to the row's own position
//   out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m), m at or near the largest s_j
//
// Three kernels by what bounds them (few rows per key head, many, latent rows),
// and one that joins the runs of split contexts; see attend.h for what they share, and
// sight.h for what a call may say of scores and of the keys that a token sees.
#include <algorithm>
#include <cmath>

#include "sight.h"

namespace mori {
namespace {

// How a batch is run.
struct Plan {
  SightArgs a;
  uint32_t dim, value;
  bool f16, step, latent;
  bool listed;  // a sight's items are written down
  uint64_t ml_at, tile_at, list_at, split_at, bytes;  // workspace
};

// Host check of what the call and its workspace size take, and the schedule.
bool plan_of(const mori_pool* pool, uint32_t layer, const mori_tokens* tokens, const mori_attend* at,
             const mori_sight* sight, uint32_t* error, Plan* out) {
  Plan& p = *out;
  SightArgs& a = p.a;
  if (!at || !batch_of(pool, layer, tokens, error, &a.b)) return false;
  if (at->dtype > MORI_DT_BF16 || !at->kv_heads || !at->q_heads || at->q_heads > 1024) return false;
  if (at->q_heads % at->kv_heads || !std::isfinite(at->scale)) return false;
  if ((uint64_t)at->kv_heads * at->head_dim * 2 != pool->row_bytes) return false;
  if (pool->planes == 2) {
    if ((at->head_dim != 64 && at->head_dim != 128) || at->value_dim != at->head_dim) return false;
  } else if (at->kv_heads != 1 || at->head_dim != 576 || at->value_dim != 512) {
    return false;
  }
  if ((uint64_t)a.b.T * at->q_heads >= (1u << 31)) return false;
  if ((uint64_t)pool->num_blocks * pool->block_tokens >= (1ull << 32)) return false;
  p.dim = at->head_dim;
  p.value = at->value_dim;
  p.f16 = at->dtype == MORI_DT_F16;
  a.heads = at->q_heads;
  a.kv_heads = at->kv_heads;
  a.group = at->q_heads / at->kv_heads;
  a.by_group = fast_div(a.group);
  a.by_kv = fast_div(a.kv_heads);
  a.c = at->scale == 0 ? 1.f : std::fabs(at->scale) * 1.4426950408889634f;
  a.q_keep = at->scale == 0 ? 0u : 0xFFFFFFFFu;
  a.q_flip = at->scale < 0 ? 0x80008000u : 0u;
  const uint64_t rows = (uint64_t)a.b.max_new * a.group;
  p.latent = pool->planes == 1;
  p.step = !p.latent && rows <= 32;
  if (p.latent) {
    a.tile_rows = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
    a.unit = 128;
  } else if (p.step) {
    a.tile_rows = rows <= 16 ? 16 : 32;
    a.unit = 128;
  } else {
    a.tile_rows = 128;
    a.unit = 64;
  }
  const uint64_t tiles = (uint64_t)a.b.T * a.group / a.tile_rows + a.b.B;  // no batch has more
  uint64_t most = a.b.max_kv;  // keys of a tile
  bool windowed = false;       // a window bounds them
  if (sight) {
    if (p.latent || !std::isfinite(sight->cap) || sight->cap < 0) return false;
    if ((reinterpret_cast<uintptr_t>(sight->slopes) | reinterpret_cast<uintptr_t>(sight->first) |
         reinterpret_cast<uintptr_t>(sight->end)) & 3u)
      return false;
    if (sight->cap > 0) {
      a.cap = sight->cap * 1.4426950408889634f;
      a.cap_in = at->scale == 0 ? 1.f : std::fabs(at->scale) / sight->cap;
      if (!std::isfinite(a.cap) || !std::isfinite(4.f * a.cap_in) || a.cap == 0) return false;
      a.cap_exp = 2.8853900817779268f * a.cap_in;
      constexpr double P[6] = {0.9999994039535522,    -0.3332904279232025, 0.13281433284282684,
                               -0.051605675369501114, 0.016743116080760956, -0.003067060373723507};
      for (int k = 0; k < 6; ++k) a.p[k] = (float)(P[k] * a.cap);
      a.exact = sight->cap > 64;
    }
    a.slopes = sight->slopes;
    a.window = sight->window;
    a.first = sight->first;
    a.end = sight->end;
    a.unit_log = p.step ? 7 : 6;
    a.align = p.step || a.b.bt % (512 / p.dim) ? 1 : 512 / p.dim;  // rows that a wavefront loads at once from a page
    windowed = a.window && !a.end;
    if (windowed)  // the tokens of a tile and a window before them
      most = std::min<uint64_t>(most, (uint64_t)a.window + std::min(a.b.max_new, (a.tile_rows - 1) / a.group + 2));
    most += a.align;
  }
  // Items that fill the chip a few times over (measured on decode steps, chunks and mixed
  // batches: half of these leave 2-10% to uneven items, twice as many cost that in
  // partial sums and joins); 128 latent rows are 256 KiB of partial sums an item.
  const uint32_t full = p.latent ? (a.tile_rows == 128 ? 512 : 1024) : 1536;
  a.slots = (full + a.kv_heads - 1) / a.kv_heads;
  a.least = p.step ? 2 : 4;
  a.round = p.latent && a.tile_rows == 128 ? 256 : 0;  // one workgroup a CU
  // Nothing is split in short contexts, nor where the tiles alone fill the chip: they would
  // all have room for partial sums and a join behind them.  Measured with 32 query and 8 key
  // heads of 128: 256 programs that decode behind 2000 keys each 365 us, 391 with splits.
  // That holds for lengths alike.  One context far longer than the rest is then one
  // workgroup's a key head: 256 programs behind 500 keys, one of them behind 65536, 866 us
  // against 186; a prompt of 8192 with one such program 2220 against 862.
  a.splits = most > a.least * a.unit && tiles * a.kv_heads < 2048;
  // With a sight, steps of few keys are not split either; where the sequences alone give
  // every CU a workgroup, that holds for more keys.  A workgroup takes 8 us for 1000 keys of
  // two planes of 256 B (a CU reads no faster), the second launch 5 us.  Whole and split, key
  // heads of 128, 8 of them: one sequence of 500 keys 10.8 and 14.3 us, of 1000 15.1 and
  // 14.6, of 2000 23.7 and 14.7; 8 sequences of about 500 (up to 1100) 17.4 and 14.3; 32 of
  // about 500 21.7 and 32.1, of 1000 39.1 and 45.2, of 2000 (up to 5000) 82.0 and 74.6; 64 of
  // 500 31.2 and 37.9, of 1000 (up to 3000) 67.3 and 60.1.
  if (sight && p.step && most <= (tiles * a.kv_heads < 256 ? 768 : 2048)) a.splits = 0;
  // Nor are tiles of few keys: the choice of the runs and the join take 7 to 9 us.  Tiles of
  // 128 rows, 128 wide, whole and split: 20 workgroups of 500 keys 24.8 and 27.5 us, of 1000
  // 35.6 and 30.5; 64 of 700 29.4 and 32.6, of 1000 36.3 and 35.4; 30 sequences behind 500 keys
  // (up to 1100) 56.1 and 64.1, but 8 of these 48.3 and 41.0; 16 with a window of 2400 and
  // documents 78.1 and 63.2.
  // A window makes tiles alike, so more of them stay whole.  128 wide, and 64 wide in brackets:
  // 160 workgroups of 1100 keys 37 and 43 us (27 and 33), of 2000 55 and 51 (40 and 41); 272 of
  // 2500 69 and 75 (51 and 57), of 5000 119 and 116 (89 and 82).  From 400 on the chip, 512 at
  // a time, is about full: of 5000 keys 472 173 and 182 (112 and 120), 656 257 and 265 (136 and
  // 144), 1136 437 and 447 (248 and 257); of 6000 416, capped, 245 and 237 (200 and 185), 824 358
  // and 348; of 12000 552 620 and 540 (322 and 320), 1136 947 and 868 (513 and 499).
  if (sight && !p.step) {
    const uint64_t groups = tiles * a.kv_heads;
    const bool alike = windowed && !a.first;
    uint64_t whole = groups < 256 ? 768 : 1280;
    if (alike && groups >= 128) whole = groups < 256 ? 1024 : groups < 400 ? 2560 : 5120;
    if (most <= whole) a.splits = 0;
  }
  // runs have `least` units or more, so short contexts give fewer items than slots
  const uint64_t runs = tiles * ((most + a.unit - 1) / a.unit) / a.least;
  const uint64_t items = tiles + (a.splits ? std::min<uint64_t>(a.slots, runs + 1) : 0);
  const uint64_t threads = p.latent && a.tile_rows == 128 ? 512 : 256;  // of a workgroup
  if (items * a.kv_heads * threads >= (1ull << 32)) return false;  // a launch has fewer
  a.items = (uint32_t)items;
  const uint64_t n = a.splits ? items * a.kv_heads * a.tile_rows : 0;
  p.ml_at = n * p.value * sizeof(float);
  p.bytes = p.ml_at + n * sizeof(float2);
  if (sight && !p.step) {
    p.tile_at = (p.bytes + 15) / 16 * 16;
    p.list_at = p.tile_at + tiles * sizeof(SightTile);
    // Items run longest first.  That pays for tiles which are not split, too, where these fill
    // the chip many times and do not come in such an order by themselves, as those of few
    // sequences do: one prompt of 8200 with documents of 1500 378 us so, 388 else, and 687 and
    // 681 without documents; 64 sequences of 300 behind 2000 789 and 812.
    const bool room = a.splits || (tiles * a.kv_heads >= 2048 && tiles <= 2048);  // whatever the sight
    p.listed = a.splits || (room && (a.first || (!windowed && a.b.B >= 16)));
    p.split_at = p.list_at + (room ? items * sizeof(uint32_t) : 0);
    p.bytes = p.split_at + (room ? sizeof(uint32_t) : 0);
    a.tiles = (uint32_t)tiles;
  }
  return true;
}

int workspace_of(const mori_pool* pool, const mori_tokens* tokens, const mori_attend* attend, const mori_sight* sight,
                 uint64_t* bytes) {
  Plan p{};
  if (!bytes || !plan_of(pool, 0, tokens, attend, sight, nullptr, &p)) return MORI_EINVAL;
  *bytes = p.bytes;
  return MORI_OK;
}

int attend_of(const mori_pool* pool, uint32_t layer, const mori_tokens* tokens, const mori_attend* attend,
              const mori_sight* sight, void* workspace, uint64_t workspace_bytes, uint32_t* error, void* stream) {
  Plan p{};
  if (!plan_of(pool, layer, tokens, attend, sight, error, &p)) return MORI_EINVAL;
  SightArgs& a = p.a;
  if (a.b.T == 0) return MORI_OK;
  if (!rows_valid(attend->q) || !rows_valid(attend->out)) return MORI_EINVAL;
  if (p.bytes && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < p.bytes))
    return MORI_EINVAL;
  a.q = rows_of(attend->q);
  a.out = rows_of(attend->out);
  a.lse = attend->lse;
  uint8_t* const ws = static_cast<uint8_t*>(workspace);
  a.part = static_cast<float*>(workspace);
  a.part_ml = reinterpret_cast<float2*>(ws + p.ml_at);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const auto run = [&](const auto& args) {
    if (p.step) launch_attend_step(args, p.f16, p.dim, s);
    else launch_attend_tile(args, p.f16, p.dim, s);
    if (a.splits) launch_attend_join(args, p.f16, p.value, s);
  };
  if (sight && !p.step) {
    a.tile = reinterpret_cast<SightTile*>(ws + p.tile_at);
    if (p.listed) {
      a.list = reinterpret_cast<uint32_t*>(ws + p.list_at);
      a.split = reinterpret_cast<uint32_t*>(ws + p.split_at);
    }
    launch_sight_tiles(a, s);
    launch_attend_tile(a, p.f16, p.dim, s);
    if (a.splits) launch_sight_join(a, p.f16, p.dim, s);
  } else if (sight) {
    run(a);
  } else if (p.latent) {
    launch_attend_latent(a, p.f16, s);
    if (a.splits) launch_attend_join(static_cast<const AttendArgs&>(a), p.f16, p.value, s);
  } else {
    run(static_cast<const AttendArgs&>(a));
  }
  if (hipGetLastError() != hipSuccess) return MORI_EHIP;
  return MORI_OK;
}

}  // namespace
}  // namespace mori

extern "C" int mori_kv_attend_workspace(const mori_pool* pool, const mori_tokens* tokens, const mori_attend* attend,
                                        uint64_t* bytes) {
  return mori::workspace_of(pool, tokens, attend, nullptr, bytes);
}

extern "C" int mori_kv_attend(const mori_pool* pool, uint32_t layer, const mori_tokens* tokens,
                              const mori_attend* attend, void* workspace, uint64_t workspace_bytes, uint32_t* error,
                              void* stream) {
  return mori::attend_of(pool, layer, tokens, attend, nullptr, workspace, workspace_bytes, error, stream);
}

extern "C" int mori_kv_attend_sight_workspace(const mori_pool* pool, const mori_tokens* tokens,
                                              const mori_attend* attend, const mori_sight* sight, uint64_t* bytes) {
  if (!sight) return MORI_EINVAL;
  return mori::workspace_of(pool, tokens, attend, sight, bytes);
}

extern "C" int mori_kv_attend_sight(const mori_pool* pool, uint32_t layer, const mori_tokens* tokens,
                                    const mori_attend* attend, const mori_sight* sight, void* workspace,
                                    uint64_t workspace_bytes, uint32_t* error, void* stream) {
  if (!sight) return MORI_EINVAL;
  return mori::attend_of(pool, layer, tokens, attend, sight, workspace, workspace_bytes, error, stream);
}
