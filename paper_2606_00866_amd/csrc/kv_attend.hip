// Attention of a batch's new tokens over their programs' pages: host side.
//
//   s_j = scale * q . k_j for the program's tokens j up to the row's own position
//   out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m), m at or near the largest s_j
//
// Three kernels by what bounds them (few rows per key head, many, latent rows),
// and one that joins the runs of split contexts; see attend.h for what they share.
#include <algorithm>
#include <cmath>

#include "attend.h"

namespace mori {
namespace {

// How a batch is run.
struct Plan {
  AttendArgs a;
  uint32_t dim, value;
  bool f16, step, latent;
  uint64_t ml_at, bytes;  // workspace
};

// Host check of what the call and its workspace size take, and the schedule.
bool plan_of(const mori_pool* pool, uint32_t layer, const mori_tokens* tokens, const mori_attend* at, uint32_t* error,
             Plan* out) {
  Plan& p = *out;
  AttendArgs& a = p.a;
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
  a.splits = a.b.max_kv > a.least * a.unit && tiles * a.kv_heads < 2048;
  // runs have `least` units or more, so short contexts give fewer items than slots
  const uint64_t runs = tiles * (((uint64_t)a.b.max_kv + a.unit - 1) / a.unit) / a.least;
  const uint64_t items = tiles + (a.splits ? std::min<uint64_t>(a.slots, runs + 1) : 0);
  const uint64_t threads = p.latent && a.tile_rows == 128 ? 512 : 256;  // of a workgroup
  if (items * a.kv_heads * threads >= (1ull << 32)) return false;  // a launch has fewer
  a.items = (uint32_t)items;
  const uint64_t n = a.splits ? items * a.kv_heads * a.tile_rows : 0;
  p.ml_at = n * p.value * sizeof(float);
  p.bytes = p.ml_at + n * sizeof(float2);
  return true;
}

}  // namespace
}  // namespace mori

extern "C" int mori_kv_attend_workspace(const mori_pool* pool, const mori_tokens* tokens, const mori_attend* attend,
                                        uint64_t* bytes) {
  using namespace mori;
  Plan p{};
  if (!bytes || !plan_of(pool, 0, tokens, attend, nullptr, &p)) return MORI_EINVAL;
  *bytes = p.bytes;
  return MORI_OK;
}

extern "C" int mori_kv_attend(const mori_pool* pool, uint32_t layer, const mori_tokens* tokens,
                              const mori_attend* attend, void* workspace, uint64_t workspace_bytes, uint32_t* error,
                              void* stream) {
  using namespace mori;
  Plan p{};
  if (!plan_of(pool, layer, tokens, attend, error, &p)) return MORI_EINVAL;
  AttendArgs& a = p.a;
  if (a.b.T == 0) return MORI_OK;
  if (!rows_valid(attend->q) || !rows_valid(attend->out)) return MORI_EINVAL;
  if (p.bytes && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < p.bytes))
    return MORI_EINVAL;
  a.q = rows_of(attend->q);
  a.out = rows_of(attend->out);
  a.lse = attend->lse;
  a.part = static_cast<float*>(workspace);
  a.part_ml = reinterpret_cast<float2*>(static_cast<uint8_t*>(workspace) + p.ml_at);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (p.step) launch_attend_step(a, p.f16, p.dim, s);
  else if (p.latent) launch_attend_latent(a, p.f16, s);
  else launch_attend_tile(a, p.f16, p.dim, s);
  if (a.splits) launch_attend_join(a, p.f16, p.value, s);
  if (hipGetLastError() != hipSuccess) return MORI_EHIP;
  return MORI_OK;
}
