// New tokens' keys and values into the paged pool, the position rotation
// applied on the way, and the same rotation of their queries.
//
// The rotation of a pair by position p: (a, b) -> (a c - b s, b c + a s) with
// c, s from the table row of p, in 32 bits, rounded once to the pool's type.
//
// The work is cut into units of 32 bytes of one head of one token: two 16-B
// chunks half a region apart, which hold whole pairs in both rotation styles
// (and are two coalesced runs for values, latents and unrotated elements). A
// workgroup takes 256 consecutive units, so it covers a few tokens; it issues its
// loads, then its wavefronts find the tokens' places (sequence, position, page)
// while those are in flight, then it rotates and stores.
//
// Bound by bytes: prompt chunks of five programs (16587 tokens, 32 query and 8 key
// heads of 128; 416 MB) take 77 us, 5.4 TB/s; a decode step of eight agents (4 key
// heads of 64) 3.7 us, where the launch and two dependent reads are the time.
#include "float16.h"
#include "tokens.h"

namespace mori {
namespace {

constexpr uint32_t NT = 256;

struct AppendArgs {
  Batch b;
  Rows k, v, q, q_out;
  uint32_t rope_len, rot, pairs;  // pairs: MORI_ROPE_PAIRS
  uint32_t hd, kv_heads, latent;
  const float* rope;
  uint32_t units;                 // of one token
  uint32_t q_units, k_units;      // units of all queries, of all keys (latent: of the latent part)
  FastDiv by_units, by_q, by_k;   // by units of a token, of a query head, of a key head
  uint32_t uq, uk;                // units of one query head, of one key (and value) head
};

struct Place {
  uint64_t slot;   // byte offset of the token's row in a plane
  uint32_t pos;
  uint32_t state;  // LEFT_ALONE, PADDING, ROTATED (queries only) or STORED
};
constexpr uint32_t LEFT_ALONE = 0, PADDING = 1, ROTATED = 2, STORED = 3;

// Sequence of token t by a search of a whole wavefront: 64 (then up to 64 more)
// offsets at once, the number of them that are not past t.
__device__ inline uint32_t find_sequence(const Batch& b, uint32_t t, uint32_t lane) {
  const uint32_t stride = (b.B + 63) / 64;
  uint32_t first = 0;
  if (stride > 1) {
    const uint32_t i = min((lane + 1) * stride, b.B);
    first = (uint32_t)__popcll(__ballot(b.seq_off[i] <= t && i < b.B)) * stride;
  }
  const uint32_t j = first + lane + 1;
  const bool in = lane < stride && j < b.B;
  return min(first + (uint32_t)__popcll(__ballot(stride > 1 ? in && b.seq_off[in ? j : 0] <= t
                                                             : j < b.B && b.seq_off[min(j, b.B)] <= t)),
             b.B - 1);
}

__device__ inline Place place_of(const AppendArgs& a, uint32_t t, uint32_t lane, uint32_t* err) {
  Place p{};
  const uint32_t b = find_sequence(a.b, t, lane);
  const Seq s = sequence(a.b, b);
  *err |= s.error;
  if (!s.named || t < s.t0 || t - s.t0 >= s.n) return p;
  const int32_t pos = s.position(t - s.t0);
  p.state = PADDING;
  if (s.error || pos < 0) return p;
  if (a.rot && (uint32_t)pos >= a.rope_len) {
    *err |= MORI_DEV_BAD_TOKENS;
    return p;
  }
  p.pos = (uint32_t)pos;
  const uint32_t block = divide(p.pos, a.b.by_bt);
  uint32_t bad = 0;
  const uint32_t page = checked_page(a.b, a.b.tbl[s.tbl + block], &bad);
  *err |= bad;
  p.slot = page * a.b.run + (uint64_t)(p.pos - block * a.b.bt) * a.b.row;
  p.state = bad ? ROTATED : STORED;
  return p;
}

// Where a unit reads and writes.
struct Unit {
  const uint8_t* src;
  uint8_t* dst;     // of a query; of a key or value, the row's start is added later
  uint32_t at;      // byte offset of its first chunk in the head
  uint32_t gap;     // bytes to its second chunk
  uint32_t pair;    // first chunk's index among the rotated ones
  bool query, turn;
};

__device__ inline Unit unit_of(const AppendArgs& a, uint32_t t, uint32_t u) {
  Unit x;
  uint32_t n, r, c, head;  // the head's elements, how many of them turn, the unit in it
  if (u < a.q_units) {
    head = divide(u, a.by_q);
    c = u - head * a.uq;
    n = a.latent ? a.rot : a.hd;
    r = a.rot;
    x.query = true;
    x.src = a.q.data + t * a.q.token + head * a.q.head;
    x.dst = a.q_out.data + t * a.q_out.token + head * a.q_out.head;
  } else {
    x.query = false;
    u -= a.q_units;
    const bool first = u < a.k_units;
    if (!first) u -= a.k_units;
    const Rows& in = first ? a.k : a.v;
    if (a.latent) {
      head = 0;
      c = u;
      n = first ? a.hd - a.rot : a.rot;
      r = first ? 0 : a.rot;
      x.dst = a.b.plane + (first ? 0 : 2 * (a.hd - a.rot));
    } else {
      head = divide(u, a.by_k);
      c = u - head * a.uk;
      n = a.hd;
      r = first ? a.rot : 0;
      x.dst = a.b.plane + (first ? 0 : a.b.plane_bytes) + 2 * head * a.hd;
    }
    x.src = in.data + t * in.token + head * in.head;
  }
  x.turn = c < r / 16;
  x.pair = c;
  if (x.turn) {
    x.at = 16 * c;
    x.gap = r;  // r / 16 chunks of 16 B
  } else {
    c -= r / 16;
    x.at = 2 * r + 16 * c;
    x.gap = n - r;
  }
  return x;
}

template <typename DT>
__device__ inline void rotate(const AppendArgs& a, const Unit& x, uint32_t pos, u32x4& lo, u32x4& hi) {
  const float* row = a.rope + (uint64_t)pos * a.rot;
  const uint32_t half = a.rot / 2;
  float p[8], q[8];
  widen<DT>(lo, p);
  widen<DT>(hi, q);
  if (!a.pairs) {  // element 8 pair + i of the first half with the same of the second
    const f32x4* cs = reinterpret_cast<const f32x4*>(row + 8 * x.pair);
    const f32x4* sn = reinterpret_cast<const f32x4*>(row + half + 8 * x.pair);
    const f32x4 c0 = cs[0], c1 = cs[1], s0 = sn[0], s1 = sn[1];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float c = i < 4 ? c0[i & 3] : c1[i & 3], s = i < 4 ? s0[i & 3] : s1[i & 3];
      const float f = p[i], g = q[i];
      p[i] = f * c - g * s;
      q[i] = g * c + f * s;
    }
  } else {  // neighbours within each chunk
    const uint32_t i0 = 4 * x.pair, i1 = i0 + a.rot / 4;
    const f32x4 c0 = *reinterpret_cast<const f32x4*>(row + i0), s0 = *reinterpret_cast<const f32x4*>(row + half + i0);
    const f32x4 c1 = *reinterpret_cast<const f32x4*>(row + i1), s1 = *reinterpret_cast<const f32x4*>(row + half + i1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float f = p[2 * i], g = p[2 * i + 1];
      p[2 * i] = f * c0[i] - g * s0[i];
      p[2 * i + 1] = g * c0[i] + f * s0[i];
      f = q[2 * i], g = q[2 * i + 1];
      q[2 * i] = f * c1[i] - g * s1[i];
      q[2 * i + 1] = g * c1[i] + f * s1[i];
    }
  }
  lo = narrow<DT>(p);
  hi = narrow<DT>(q);
}

template <typename DT>
__global__ __launch_bounds__(NT) void append_kernel(AppendArgs a) {
  __shared__ Place s_place[NT / 2 + 2];  // a token has two units at least
  const uint32_t tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const uint64_t u_first = (uint64_t)blockIdx.x * NT;
  const uint32_t t_first = (uint32_t)(u_first / a.units);
  const uint32_t u_in = (uint32_t)(u_first - (uint64_t)t_first * a.units);
  const uint32_t t_last = min(t_first + divide(u_in + NT - 1, a.by_units), a.b.T - 1);
  const uint32_t u = u_in + tid, tl = divide(u, a.by_units);
  // past the batch: loads the last token's, stores nothing
  const Unit x = unit_of(a, min(t_first + tl, t_last), u - tl * a.units);
  u32x4 lo = *reinterpret_cast<const u32x4*>(x.src + x.at);
  u32x4 hi = *reinterpret_cast<const u32x4*>(x.src + x.at + x.gap);
  uint32_t err = 0;
  for (uint32_t i = wv; i <= t_last - t_first; i += NT / 64) {
    const Place p = place_of(a, t_first + i, lane, &err);
    if (lane == 0) s_place[i] = p;
  }
  if (lane == 0) report(a.b, err);
  __syncthreads();
  if (t_first + tl > t_last) return;
  const Place p = s_place[tl];
  if (p.state == LEFT_ALONE || (!x.query && p.state != STORED)) return;
  if (p.state == PADDING) lo = hi = u32x4{0, 0, 0, 0};
  else if (x.turn) rotate<DT>(a, x, p.pos, lo, hi);
  uint8_t* dst = x.dst + (x.query ? 0 : p.slot) + x.at;
  *reinterpret_cast<u32x4*>(dst) = lo;
  *reinterpret_cast<u32x4*>(dst + x.gap) = hi;
}

template <typename DT>
void launch(const AppendArgs& a, hipStream_t s) {
  const uint64_t total = (uint64_t)a.b.T * a.units;
  hipLaunchKernelGGL(append_kernel<DT>, dim3((uint32_t)((total + NT - 1) / NT)), dim3(NT), 0, s, a);
}

}  // namespace
}  // namespace mori

extern "C" int mori_kv_append(const mori_pool* pool, uint32_t layer, const mori_tokens* tokens, const mori_append* ap,
                              uint32_t* error, void* stream) {
  using namespace mori;
  AppendArgs a{};
  if (!ap || !batch_of(pool, layer, tokens, error, &a.b)) return MORI_EINVAL;
  if (ap->dtype > MORI_DT_BF16 || ap->rope_style > MORI_ROPE_PAIRS) return MORI_EINVAL;
  a.latent = pool->planes == 1;
  a.hd = ap->head_dim;
  a.kv_heads = ap->kv_heads;
  a.rot = ap->rot_dim;
  if (!a.hd || a.hd > 4096 || (a.hd & 15u) || (a.rot & 15u) || a.rot > a.hd || !a.kv_heads) return MORI_EINVAL;
  if ((uint64_t)a.kv_heads * a.hd * 2 != pool->row_bytes) return MORI_EINVAL;
  if (a.latent && (a.kv_heads != 1 || a.rot < 16 || a.rot > a.hd - 16)) return MORI_EINVAL;
  if (a.rot && (!ap->rope || (reinterpret_cast<uintptr_t>(ap->rope) & 15u) || !ap->rope_len)) return MORI_EINVAL;
  if (a.b.T == 0) return MORI_OK;
  if (!rows_valid(ap->k) || !rows_valid(ap->v)) return MORI_EINVAL;
  const bool with_q = ap->q.data != nullptr;
  if (with_q && (!rows_valid(ap->q) || !rows_valid(ap->q_out) || !ap->q_heads || ap->q_heads > 1024)) return MORI_EINVAL;
  a.k = rows_of(ap->k);
  a.v = rows_of(ap->v);
  if (with_q) a.q = rows_of(ap->q), a.q_out = rows_of(ap->q_out);
  a.rope = ap->rope;
  a.rope_len = ap->rope_len;
  a.pairs = ap->rope_style == MORI_ROPE_PAIRS;
  a.uq = (a.latent ? a.rot : a.hd) / 16;
  a.uk = a.hd / 16;
  a.q_units = with_q ? ap->q_heads * a.uq : 0;
  a.k_units = a.latent ? (a.hd - a.rot) / 16 : a.kv_heads * a.uk;
  a.units = a.q_units + (a.latent ? a.uk : 2 * a.k_units);
  a.by_units = fast_div(a.units);
  a.by_q = fast_div(a.uq);
  a.by_k = fast_div(a.uk);
  if ((uint64_t)a.b.T * a.units > (1ull << 32) - NT) return MORI_EINVAL;  // a launch has fewer threads than 2^32
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (ap->dtype == MORI_DT_F16) launch<F16>(a, s);
  else launch<BF16>(a, s);
  if (hipGetLastError() != hipSuccess) return MORI_EHIP;
  return MORI_OK;
}
