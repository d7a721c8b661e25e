// Attention of a batch's new tokens over their programs' pages.
//
//   s_j = scale * q . k_j for the program's tokens j up to the row's own position
//   out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m), m the largest s_j so far
//
// One wavefront per (token, query head): 64 keys at a time, a key per lane for
// the scores, the value's elements over the lanes for the sum.
#include <cmath>

#include "attend.h"

namespace mori {
namespace {

constexpr uint32_t NT = 256;

template <typename DT, int DK, int DV>
__global__ __launch_bounds__(NT) void attend_rows_kernel(AttendArgs a, float scale, uint64_t v_off) {
  __shared__ float s_q[NT / 64][DK];
  const uint32_t lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const uint64_t row = (uint64_t)blockIdx.x * (NT / 64) + wv;
  const uint32_t t = (uint32_t)(row / a.heads), h = (uint32_t)(row - (uint64_t)t * a.heads);
  if (t >= a.b.T) return;
  uint32_t b = 0;
  while (b + 1 < a.b.B && a.b.seq_off[b + 1] <= t) ++b;
  const Seq sq = sequence(a.b, b);
  uint32_t err = sq.error;
  if (!sq.named || t < sq.t0 || t - sq.t0 >= sq.n) {
    if (lane == 0) report(a.b, err);
    return;
  }
  const int32_t pos = sq.error ? -1 : sq.position(t - sq.t0);
  const typename DT::scalar* q = reinterpret_cast<const typename DT::scalar*>(a.q.data + t * a.q.token + h * a.q.head);
  for (int d = lane; d < DK; d += 64) s_q[wv][d] = (float)q[d] * scale;
  float o[DV / 64] = {}, m = -INFINITY, l = 0;
  for (int32_t k0 = 0; k0 <= pos; k0 += 64) {
    const int32_t key = k0 + (int32_t)lane;
    float s = -INFINITY;
    const uint8_t* at = a.b.plane;
    if (key <= pos) {
      const uint32_t block = divide((uint32_t)key, a.b.by_bt);
      const uint32_t page = checked_page(a.b, a.b.tbl[sq.tbl + block], &err);
      at += page * a.b.run + (uint64_t)((uint32_t)key - block * a.b.bt) * a.b.row + (uint64_t)(h / a.group) * DK * 2;
      s = 0;
      for (int c = 0; c < DK / 8; ++c) {
        float f[8];
        widen<DT>(reinterpret_cast<const u32x4*>(at)[c], f);
        for (int i = 0; i < 8; ++i) s += f[i] * s_q[wv][8 * c + i];
      }
    }
    float top = s;
    for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float m2 = fmaxf(m, top), keep = expf(m - m2), p = expf(s - m2);
    float sum = p;
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
    l = l * keep + sum;
    m = m2;
    for (int i = 0; i < DV / 64; ++i) o[i] *= keep;
    const uint64_t v_at = (uint64_t)at + v_off;
    for (int j = 0; j < 64 && k0 + j <= pos; ++j) {
      const typename DT::scalar* v = reinterpret_cast<const typename DT::scalar*>(wave::lane_of(v_at, j));
      const float pj = __shfl(p, j);
      for (int i = 0; i < DV / 64; ++i) o[i] += pj * (float)v[64 * i + lane];
    }
  }
  typename DT::scalar* out = reinterpret_cast<typename DT::scalar*>(a.out.data + t * a.out.token + h * a.out.head);
  const float inv = pos < 0 ? 0.f : 1.f / l;
  for (int i = 0; i < DV / 64; ++i) out[64 * i + lane] = (typename DT::scalar)(o[i] * inv);
  if (a.lse && lane == 0) a.lse[(uint64_t)t * a.heads + h] = pos < 0 ? -INFINITY : m + logf(l);
  report(a.b, err);
}

// How a batch is run.
struct Plan {
  AttendArgs a;
  uint32_t dim, value, blocks;
  float scale;
  bool f16, step, tile;
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
  p.scale = at->scale;
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
  p.step = pool->planes == 2 && rows <= 32;
  p.tile = pool->planes == 2 && !p.step;
  p.blocks = rows <= 16 ? 1 : 2;
  a.tile_rows = p.step ? 16 * p.blocks : 128;
  a.unit = p.step ? 128 : 64;
  const uint64_t tiles = (uint64_t)a.b.T * a.group / a.tile_rows + a.b.B;  // no batch has more
  a.slots = ((p.step ? 1536 : 1024) + a.kv_heads - 1) / a.kv_heads;
  a.least = (p.step ? 2 : 4);
  a.splits = a.b.max_kv > a.least * a.unit && (p.step || tiles * a.kv_heads < 2048);
  const uint64_t items = tiles + (a.splits ? a.slots : 0);
  if (items * a.kv_heads >= (1ull << 31)) return false;
  a.items = (uint32_t)items;
  const uint64_t n = (p.step || p.tile) && a.splits ? items * a.kv_heads * a.tile_rows : 0;
  p.ml_at = n * p.value * sizeof(float);
  p.bytes = p.ml_at + n * sizeof(float2);
  return true;
}

template <typename DT>
void launch(const Plan& p, hipStream_t s) {
  const AttendArgs& a = p.a;
  const uint64_t v_off = p.value == p.dim ? a.b.plane_bytes : 0;
  const dim3 grid((uint32_t)(((uint64_t)a.b.T * a.heads + NT / 64 - 1) / (NT / 64)));
  if (p.dim == 64) hipLaunchKernelGGL((attend_rows_kernel<DT, 64, 64>), grid, dim3(NT), 0, s, a, p.scale, v_off);
  else if (p.dim == 128) hipLaunchKernelGGL((attend_rows_kernel<DT, 128, 128>), grid, dim3(NT), 0, s, a, p.scale, v_off);
  else hipLaunchKernelGGL((attend_rows_kernel<DT, 576, 512>), grid, dim3(NT), 0, s, a, p.scale, v_off);
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
  if (p.step) {
    launch_attend_step(a, p.f16, p.dim, p.blocks, s);
    if (a.splits) launch_attend_join(a, p.f16, p.value, s);
  } else if (p.tile) {
    launch_attend_tile(a, p.f16, p.dim, s);
    if (a.splits) launch_attend_join(a, p.f16, p.value, s);
  } else if (p.f16) {
    launch<F16>(p, s);
  } else {
    launch<BF16>(p, s);
  }
  if (hipGetLastError() != hipSuccess) return MORI_EHIP;
  return MORI_OK;
}
