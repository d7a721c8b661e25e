// Block tables of programs that take new tokens, and what a batch of those tokens
// needs, from the numbers of tokens alone.
//
//   more_b  = max(0, ceil((held_p + n_b) / block_tokens) - blocks_p)     p = program_b
//   off'    = exclusive scan over p of blocks_p + more_p
//   tbl'    = each program's entries, then the pages it takes: the lowest free ids, in
//             batch order, a sequence's blocks in their order
//   seq_off = exclusive scan over b of n_b,  kv_len_b = held'_p = held_p + n_b
//   slot_t  = page of t's block * block_tokens + its row,  position_t = held_p + i
//
// One or two launches, bound by their latency and dependent reads: a byte of the free map
// per page, an entry of the tables in and out, 12 bytes a token.  A step of 8 programs (a
// pool of 401 pages) takes 6.1 us, of 400 of 1024 (309 450 pages) 11.2, of 3000 of 4096
// 16.6; chunks of 24 of 64 programs (72 620 tokens, about 4540 of 87 830 pages) 9.
//   grow_small   everything, in one workgroup, for small pools and batches
//   grow_count   one workgroup checks and scans the sequences and programs; the others
//                count free pages, 512 at a time, and, where the tables grow in place,
//                copy the old entries aside
//   grow_assign  workgroups take a tile each (pages to table entries and to the slots of
//                the tokens in new blocks), or old entries (to where they lie now), or
//                tokens in old blocks, or programs.  Every workgroup sums the tile counts
//                for itself, so all of them know whether there are pages enough: nothing
//                is changed unless everything is.
#include <algorithm>

#include "tokens.h"

namespace mori {
namespace {

constexpr uint32_t NT = 256;
// Pages of a count: the smallest tile.  A tile's workgroup also writes the slots of all
// tokens in its pages: with 4096 pages a tile chunks of 72 620 tokens took 28 us there,
// with 512 5.5.
constexpr uint32_t COUNTED = 512;
constexpr uint32_t ENTRIES = 1024;  // table entries of a workgroup
constexpr uint32_t MOST = MORI_MAX_PROGRAMS;

struct Head {
  uint32_t error;     // MORI_DEV_* bits: nothing grows
  uint32_t more;      // pages taken
  uint32_t tokens;    // of the batch
  uint32_t entries;   // of the old tables
  uint32_t sound;     // the old offsets can be used as indexes
};

struct GrowArgs {
  uint32_t B, T, max_new, max_kv, P, tbl_len, bt, num_blocks, counts, ntiles, tile;
  FastDiv by_bt;
  const uint32_t *new_tokens, *program;
  const uint8_t* tier;
  const uint32_t *tbl_off, *tbl, *held;
  const uint8_t* free_map;
  uint32_t *tbl_off_to, *tbl_to, *held_to;
  uint8_t* free_to;
  uint32_t *seq_off, *kv_len;
  int64_t* slots;
  int32_t* positions;
  uint32_t* error;
  uint32_t in_place, copies;  // the tables'; workgroups that copy them aside
  // workspace
  Head* head;
  uint32_t *tile_cnt, *old_off, *new_off, *held_new, *tok, *ahead, *len, *prog;
  uint32_t* aside;
};

// Bytes that are not 0, a bit for each.
__device__ inline uint32_t set_bytes(uint32_t w) {
  return (((w & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | w) & 0x80808080u;
}

// N pages of the free map from `page` on (N = 2 or 16, a multiple of it), 4 a word; those
// past the pool are not free.
template <int N>
struct Pages {
  static constexpr int W = N < 4 ? 1 : N / 4;
  uint32_t w[W];
  __device__ __forceinline__ void load(const uint8_t* map, uint32_t num_blocks, uint64_t page) {
    if (page + N <= num_blocks) {
      if constexpr (N == 2) {
        w[0] = *reinterpret_cast<const uint16_t*>(map + page);
      } else {
        const uint4 x = *reinterpret_cast<const uint4*>(map + page);
        w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
      }
      return;
    }
    uint8_t x[N];  // all reads at once, of the last page where there is none
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = map[page + i < num_blocks ? page + i : num_blocks - 1u];
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) w[i / 4] |= page + i < num_blocks ? (uint32_t)x[i] << (8 * (i % 4)) : 0u;
  }
  __device__ __forceinline__ void store(uint8_t* map, uint32_t num_blocks, uint64_t page) const {
    if (page + N <= num_blocks) {
      if constexpr (N == 2) *reinterpret_cast<uint16_t*>(map + page) = (uint16_t)w[0];
      else *reinterpret_cast<uint4*>(map + page) = uint4{w[0], w[1], w[2], w[3]};
      return;
    }
#pragma unroll
    for (int i = 0; i < W; ++i) {
#pragma unroll 1
      for (int j = 0; j < 4 && 4 * i + j < N; ++j)
        if (page + 4 * i + j < num_blocks) map[page + 4 * i + j] = (uint8_t)(w[i] >> (8 * j));
    }
  }
  // Takes free pages out, the first one as the r-th, while r is below `end`: to(r, its index here).
  template <typename F>
  __device__ __forceinline__ void take(uint32_t r, uint32_t end, F to) {
#pragma unroll
    for (int i = 0; i < W; ++i) {
      for (uint32_t bits = set_bytes(w[i]); bits && r < end; bits &= bits - 1, ++r) {
        const uint32_t j = (uint32_t)__builtin_ctz(bits) / 8;
        to(r, 4 * i + j);
        w[i] &= ~(0xFFu << (8 * j));
      }
    }
  }
  __device__ __forceinline__ uint32_t count() const {
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) n += __popc(set_bytes(w[i]));
    return n;
  }
};

// Exclusive scans over i = k W + thread of values v[k], after the wavefronts' sums of every
// k have met in LDS: `part` has K * WAVES of them, in that order.
template <int K, int WAVES>
__device__ inline void scan_parts(const uint32_t* part, const uint32_t (&incl)[K], const uint32_t (&v)[K], uint32_t lane,
                                  uint32_t wv, uint32_t (&before)[K], uint32_t* total) {
  static_assert(K * WAVES <= 64, "a wavefront scans them");
  const uint32_t x = lane < K * WAVES ? part[lane] : 0, in = wave::incl_add(x);
#pragma unroll
  for (int k = 0; k < K; ++k) before[k] = (uint32_t)__shfl((int)(in - x), (int)(k * WAVES + wv)) + incl[k] - v[k];
  *total = wave::lane63(in);
}

// The batch and the programs: checks, scans, and what grow_assign reads of them.  One
// workgroup of W threads, thread t with the programs and sequences t, W + t, ...: every read
// of global memory is under way before the first barrier, the rest is in LDS and three
// barriers long.  Totals are of 64 bits, so none wraps unseen; where something does not
// fit, what is written here is not used.
template <int W, int K>
__device__ void scan_batch(const GrowArgs& a) {
  constexpr uint32_t WAVES = W / 64, NONE = 0xFFFFFFFFu, CLAIMED = 0xFFFFFFFEu;
  __shared__ uint32_t s_more[W * K], s_len[W * K], s_held[W * K], s_blocks[W * K];  // by program
  __shared__ uint8_t s_tier[W * K];
  __shared__ uint64_t s_total[WAVES][3];
  __shared__ uint32_t s_part[3][K * WAVES];
  __shared__ uint32_t s_error[WAVES], s_bad[WAVES];
  const uint32_t tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  uint32_t lo[K], blocks[K], held[K], n[K], prog[K], bad = 0, err = 0;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const uint32_t p = k * W + tid;
    prog[k] = p < a.B ? a.program ? a.program[p] : p : NONE;
    n[k] = p < a.B ? a.new_tokens[p] : 0;
    lo[k] = blocks[k] = held[k] = 0;
    s_more[p] = NONE;
    if (p < a.P) {
      lo[k] = a.tbl_off[p];
      const uint32_t hi = a.tbl_off[p + 1];
      held[k] = a.held[p];
      s_tier[p] = a.tier ? a.tier[p] : (uint8_t)MORI_TIER_GPU;
      bad |= lo[k] > hi || hi > a.tbl_len || (p == 0 && lo[k]);
      blocks[k] = hi - lo[k];
      s_held[p] = held[k];
      s_blocks[p] = blocks[k];
    }
  }
  bad = __ballot(bad) != 0;
  if (lane == 0) s_bad[wv] = bad;
  __syncthreads();
  uint32_t more[K], len[K], n_in[K], m_in[K];
  uint64_t n_sum = 0, m_sum = 0;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const uint32_t p = prog[k], x = n[k];
    more[k] = len[k] = n[k] = 0;
    if (k * W + tid < a.B) {
      if (p >= a.P || atomicCAS(&s_more[p], NONE, CLAIMED) != NONE) {  // no program, or one that is here already
        err |= MORI_DEV_BAD_TOKENS;
      } else {
        const uint32_t h = s_held[p], have = s_blocks[p];
        if (s_tier[p] != MORI_TIER_GPU) err |= MORI_DEV_NOT_RESIDENT;
        if (x > a.max_new || (uint64_t)h + x > a.max_kv || h > (uint64_t)have * a.bt) {
          err |= MORI_DEV_BAD_TOKENS;
        } else {
          n[k] = x;
          len[k] = h + x;  // with the rounding below 2^31
          const uint32_t need = divide(len[k] + a.bt - 1, a.by_bt);
          more[k] = need > have ? need - have : 0;
          s_more[p] = more[k];
          s_len[p] = len[k];
        }
      }
    }
    n_in[k] = wave::incl_add(n[k]);
    m_in[k] = wave::incl_add(more[k]);
    if (lane == 63) {
      s_part[0][k * WAVES + wv] = n_in[k];
      s_part[1][k * WAVES + wv] = m_in[k];
    }
    n_sum += n[k];
    m_sum += more[k];
  }
  n_sum = wave::sum(n_sum);
  m_sum = wave::sum(m_sum);
  err = wave::all_or(err);
  if (lane == 0) {
    s_total[wv][0] = n_sum;
    s_total[wv][1] = m_sum;
    s_error[wv] = err;
  }
  __syncthreads();
  uint64_t e_sum = 0;
  uint32_t grown[K], e_in[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const uint32_t p = k * W + tid;
    grown[k] = 0;
    if (p < a.P) {
      const uint32_t x = s_more[p];
      const bool takes = x < CLAIMED;
      grown[k] = blocks[k] + (takes ? x : 0);
      a.held_new[p] = takes ? s_len[p] : held[k];
    }
    e_in[k] = wave::incl_add(grown[k]);
    if (lane == 63) s_part[2][k * WAVES + wv] = e_in[k];
    e_sum += grown[k];
  }
  e_sum = wave::sum(e_sum);
  if (lane == 0) s_total[wv][2] = e_sum;
  __syncthreads();
  uint32_t tok[K], ahead[K], off[K], t_all, m_all, e_all;
  scan_parts<K, WAVES>(s_part[0], n_in, n, lane, wv, tok, &t_all);
  scan_parts<K, WAVES>(s_part[1], m_in, more, lane, wv, ahead, &m_all);
  scan_parts<K, WAVES>(s_part[2], e_in, grown, lane, wv, off, &e_all);
  uint64_t sums[3];  // in full
#pragma unroll
  for (int j = 0; j < 3; ++j) sums[j] = wave::sum(lane < WAVES ? s_total[lane][j] : (uint64_t)0);
  err = wave::all_or(lane < WAVES ? s_error[lane] : 0u);
  bad = wave::all_or(lane < WAVES ? s_bad[lane] : 0u);
  if (sums[0] > a.T) err |= MORI_DEV_BAD_TOKENS;
  if (bad) err |= MORI_DEV_BAD_TBL_OFF;
  else if (sums[1] > a.num_blocks || sums[2] > a.tbl_len) err |= MORI_DEV_NOSPC;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const uint32_t i = k * W + tid;
    if (i < a.B) {
      a.tok[i] = tok[k];
      a.ahead[i] = ahead[k];
      a.len[i] = len[k];
      a.prog[i] = prog[k];
    }
    if (i < a.P) {
      a.new_off[i] = off[k];
      a.old_off[i] = lo[k];
      if (i == a.P - 1) {
        a.new_off[a.P] = e_all;
        a.old_off[a.P] = lo[k] + blocks[k];
        *a.head = Head{err, m_all, t_all, bad ? 0 : lo[k] + blocks[k], !bad};
        a.tok[a.B] = t_all;
        a.ahead[a.B] = m_all;
        if (err && a.error) atomicOr(a.error, err);
      }
    }
  }
}

template <int W, int K>
__global__ __launch_bounds__(W) void grow_count_kernel(GrowArgs a) {
  if (blockIdx.x == 0) {
    scan_batch<W, K>(a);
    return;
  }
  const uint32_t tid = threadIdx.x, i = blockIdx.x - 1;
  if (i < a.copies) {
    const uint32_t n = min(a.tbl_off[a.P], a.tbl_len);
    const uint64_t e0 = (uint64_t)i * ENTRIES + tid;
#pragma unroll
    for (uint32_t k = 0; k < ENTRIES / W; ++k)
      if (e0 + k * W < n) a.aside[e0 + k * W] = a.tbl[e0 + k * W];
    return;
  }
  // a wavefront takes 1024 pages: two small tiles or a quarter of a large one
  const uint64_t page = ((uint64_t)(i - a.copies) * W + tid) * 16;
  Pages<16> x;
  x.load(a.free_map, a.num_blocks, page);
  const uint32_t in = wave::incl_add(x.count());
  const uint64_t at = page / 1024;
  if ((tid & 31) == 31) {
    const uint32_t half = tid & 32 ? in - (uint32_t)__builtin_amdgcn_readlane((int)in, 31) : in;
    const uint64_t c = 2 * at + (tid & 32 ? 1 : 0);
    if (c < a.counts) a.tile_cnt[c] = half;
  }
}

// The last of x[0..n-1] (ascending, x[0] <= v) that is not above v: 64 of them at a time.
// The same v for the whole wavefront.
__device__ inline uint32_t wave_last_not_above(const uint32_t* x, uint32_t n, uint32_t v, uint32_t lane) {
  uint32_t at = 0, step = (n + 63) / 64;
  for (;;) {
    const uint32_t i = at + lane * step;
    const uint64_t in = __ballot(i < n && x[min(i, n - 1)] <= v);
    at += (63 - __clzll((long long)in)) * step;
    if (step == 1) return at;
    step = (step + 63) / 64;
  }
}
// The same by a thread between two indexes.  X: a pointer, or an array in LDS, which stays
// one to the compiler so.
template <typename X>
__device__ __forceinline__ uint32_t last_not_above(const X& x, uint32_t lo, uint32_t hi, uint32_t v) {
  while (lo < hi) {
    const uint32_t mid = (lo + hi + 1) / 2;
    if (x[mid] <= v) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// A tile's pages, N a thread: to the programs that take them, and out of the free map.
template <int N>
__device__ void assign_tile(const GrowArgs& a, const Head& h, bool ok, uint32_t tile, uint32_t base) {
  constexpr uint32_t TILE = N * NT;
  struct Taken {
    uint32_t page, pos, rows;  // position of its first token, tokens in it
    uint32_t t;                // index of its first token in the batch
  };
  __shared__ Taken s_taken[TILE];
  __shared__ uint32_t s_ahead[MOST], s_wave[NT / 64];
  const uint32_t tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const uint64_t page0 = (uint64_t)tile * TILE + (uint64_t)N * tid;
  const uint32_t more = ok ? h.more : 0;
  const bool some = base < more;  // pages from here on are taken
  if (!some && a.free_to == a.free_map) return;
  Pages<N> x;
  x.load(a.free_map, a.num_blocks, page0);
  if (some) {
    for (uint32_t b = tid; b < a.B; b += NT) s_ahead[b] = a.ahead[b];
    const uint32_t mine = x.count(), in = wave::incl_add(mine);
    if (lane == 63) s_wave[wv] = in;
    __syncthreads();
    uint32_t r = in - mine, count = 0;  // index among the tile's free pages
#pragma unroll
    for (uint32_t i = 0; i < NT / 64; ++i) {
      if (i < wv) r += s_wave[i];
      count += s_wave[i];
    }
    count = min(count, more - base);
    x.take(r, count, [&](uint32_t at, uint32_t i) { s_taken[at].page = (uint32_t)page0 + i; });
    __syncthreads();
    for (uint32_t i = tid; i < count; i += NT) {
      // sequences that take none share their number with the next: the last of them takes it
      const uint32_t b = last_not_above(s_ahead, 0, a.B - 1, base + i), p = a.prog[b];
      const uint32_t block = a.old_off[p + 1] - a.old_off[p] + (base + i - s_ahead[b]);
      const uint32_t pos = block * a.bt, len = a.len[b];  // the block holds a token: pos < len
      a.tbl_to[a.new_off[p] + block] = s_taken[i].page;
      s_taken[i].pos = pos;
      s_taken[i].rows = min(a.bt, len - pos);
      s_taken[i].t = a.tok[b + 1] - (len - pos);
    }
    __syncthreads();
    if (a.slots || a.positions) {  // every token of a new block is new
      for (uint32_t y = tid; y < count * a.bt; y += NT) {  // below 2^30
        const uint32_t i = divide(y, a.by_bt), row = y - i * a.bt;
        const Taken k = s_taken[i];
        if (row >= k.rows) continue;
        if (a.slots) a.slots[k.t + row] = (int64_t)((uint64_t)k.page * a.bt + row);
        if (a.positions) a.positions[k.t + row] = (int32_t)(k.pos + row);
      }
    }
  }
  x.store(a.free_to, a.num_blocks, page0);
}

// Old entries to where they lie now.
__device__ void move_entries(const GrowArgs& a, const Head& h, bool ok, uint32_t first) {
  const uint32_t tid = threadIdx.x, lane = tid & 63;
  if (first >= h.entries || (a.in_place && !(ok && h.more))) return;  // in place nothing moves
  const uint32_t* const from = a.in_place ? a.aside : a.tbl;
  const uint32_t last = min(first + ENTRIES, h.entries) - 1;
  const uint32_t p0 = wave_last_not_above(a.old_off, a.P, first, lane), p1 = wave_last_not_above(a.old_off, a.P, last, lane);
  uint32_t page[ENTRIES / NT];
#pragma unroll
  for (uint32_t k = 0; k < ENTRIES / NT; ++k) page[k] = from[min(first + k * NT + tid, last)];
#pragma unroll
  for (uint32_t k = 0; k < ENTRIES / NT; ++k) {
    const uint32_t e = first + k * NT + tid;
    if (e > last) continue;
    const uint32_t p = last_not_above(a.old_off, p0, p1, e);
    a.tbl_to[ok ? a.new_off[p] + (e - a.old_off[p]) : e] = page[k];
  }
}

// Slots and positions of the tokens in blocks that were there.
__device__ void place_tokens(const GrowArgs& a, const Head& h, bool ok, uint32_t t0, uint32_t* err) {
  const uint32_t t = t0 + threadIdx.x, lane = threadIdx.x & 63;
  uint32_t b0 = 0, b1 = 0;
  if (ok && t0 < h.tokens) {
    b0 = wave_last_not_above(a.tok, a.B, t0, lane);
    b1 = wave_last_not_above(a.tok, a.B, min(t0 + NT, h.tokens) - 1, lane);
  }
  if (t >= a.T) return;
  int64_t slot = -1;
  int32_t at = -1;
  if (ok && t < h.tokens) {
    const uint32_t b = last_not_above(a.tok, b0, b1, t), p = a.prog[b];
    const uint32_t pos = a.len[b] - (a.tok[b + 1] - t), block = divide(pos, a.by_bt);
    const uint32_t first = a.old_off[p];
    if (block >= a.old_off[p + 1] - first) return;  // in a new block
    const uint32_t page = (a.in_place ? a.aside : a.tbl)[first + block];
    at = (int32_t)pos;
    if (page < a.num_blocks) slot = (int64_t)((uint64_t)page * a.bt + (pos - block * a.bt));
    else *err |= page == MORI_NO_PAGE ? MORI_DEV_NOT_RESIDENT : MORI_DEV_PAGE_RANGE;
  }
  if (a.slots) a.slots[t] = slot;
  if (a.positions) a.positions[t] = at;
}

// What the batch and the programs are afterwards, by thread x of all.
__device__ inline void store_batch(const GrowArgs& a, const Head& h, bool ok, uint32_t x) {
  if (x == 0 && !h.error && !ok && a.error) atomicOr(a.error, MORI_DEV_NOSPC);
  if (x <= a.B) a.seq_off[x] = ok ? a.tok[x] : 0;
  if (x < a.B) a.kv_len[x] = ok ? a.len[x] : 0;
  if (x < a.P && (ok || a.held_to != a.held)) a.held_to[x] = ok ? a.held_new[x] : a.held[x];
  if (x <= a.P && h.sound) a.tbl_off_to[x] = ok ? a.new_off[x] : a.old_off[x];
}

template <int N>
__global__ __launch_bounds__(NT) void grow_assign_kernel(GrowArgs a, uint32_t movers, uint32_t placers) {
  __shared__ uint32_t s_before[NT / 64], s_total[NT / 64];
  const uint32_t tid = threadIdx.x, lane = tid & 63;
  uint32_t i = blockIdx.x;
  const Head h = *a.head;
  // free pages in the tiles before this one and in all; neither is needed where nothing is taken
  uint32_t before = 0, total = 0;
  if (h.more) {
    const uint64_t mine = (uint64_t)i * (a.tile / COUNTED);
    for (uint32_t k = tid; k < a.counts; k += NT) {
      const uint32_t n = a.tile_cnt[k];
      total += n;
      if (k < mine) before += n;
    }
    before = wave::sum(before);
    total = wave::sum(total);
    if (lane == 0) {
      s_before[tid >> 6] = before;
      s_total[tid >> 6] = total;
    }
    __syncthreads();
    before = s_before[0] + s_before[1] + s_before[2] + s_before[3];
    total = s_total[0] + s_total[1] + s_total[2] + s_total[3];
  }
  const bool ok = !h.error && total >= h.more;
  if (i < a.ntiles) {
    assign_tile<N>(a, h, ok, i, before);
    return;
  }
  i -= a.ntiles;
  if (i < movers) {
    move_entries(a, h, ok, i * ENTRIES);
    return;
  }
  i -= movers;
  if (i < placers) {
    uint32_t err = 0;
    place_tokens(a, h, ok, i * NT, &err);
    err = wave::all_or(err);
    if (lane == 0 && err && a.error) atomicOr(a.error, err);
    return;
  }
  store_batch(a, h, ok, (i - placers) * NT + tid);
}

// All of it in one workgroup, where a pool and a batch are small (16 pages, 8 entries, 4
// tokens and a program a thread at most): one launch, no workspace.  What the scan finds
// and the grown table lie in LDS, and tokens find their pages there whether their blocks
// are new or old.  Everything is read before the first barrier, so in place is as good.
// A pool of 401 pages and 377 entries, 8 programs that take a token each: 6.1 us a call (64
// threads; 6.5 with 256), 8.7 with the two launches, which in a graph take 5.6.
template <int W>
__global__ __launch_bounds__(W) void grow_small_kernel(GrowArgs a) {
  constexpr uint32_t E = 8;
  __shared__ uint32_t s_wave[W / 64], s_tbl[E * W], s_page[E * W];
  __shared__ uint32_t s_old_off[W + 1], s_new_off[W + 1], s_held[W], s_tok[W + 1], s_ahead[W + 1], s_len[W], s_prog[W];
  __shared__ Head s_head;
  const uint32_t tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  Pages<16> x;
  const uint64_t page0 = 16ull * tid;
  x.load(a.free_map, a.num_blocks, page0);
  uint32_t entry[E];  // neighbours
#pragma unroll
  for (uint32_t k = 0; k < E; ++k) entry[k] = E * tid + k < a.tbl_len ? a.tbl[E * tid + k] : 0;
  a.head = &s_head;
  a.old_off = s_old_off;
  a.new_off = s_new_off;
  a.held_new = s_held;
  a.tok = s_tok;
  a.ahead = s_ahead;
  a.len = s_len;
  a.prog = s_prog;
  scan_batch<W, 1>(a);
  const uint32_t mine = x.count(), in = wave::incl_add(mine);
  if (lane == 63) s_wave[wv] = in;
  __syncthreads();
  uint32_t r = in - mine, total = 0;  // index among the free pages
#pragma unroll 4
  for (uint32_t i = 0; i < W / 64; ++i) {
    if (i < wv) r += s_wave[i];
    total += s_wave[i];
  }
  const Head h = s_head;
  const bool ok = !h.error && total >= h.more;
  const uint32_t more = ok ? h.more : 0;
  if (E * tid < h.entries) {
    uint32_t p = 0, end = 0xFFFFFFFFu, up = 0;  // how far an entry moves: it stays where nothing is taken
    if (more) {
      p = last_not_above(s_old_off, 0, a.P - 1, E * tid);
      end = s_old_off[p + 1];
      up = s_new_off[p] - s_old_off[p];
    }
#pragma unroll
    for (uint32_t k = 0; k < E; ++k) {
      const uint32_t e = E * tid + k;
      if (e >= h.entries) break;
      while (e >= end) {
        ++p;
        end = s_old_off[p + 1];
        up = s_new_off[p] - s_old_off[p];
      }
      s_tbl[e + up] = entry[k];  // below tbl_len
    }
  }
  const bool taken = r < more && mine;
  x.take(r, more, [&](uint32_t at, uint32_t i) { s_page[at] = (uint32_t)page0 + i; });  // no more than entries
  if (more) {
    __syncthreads();
    for (uint32_t i = tid; i < more; i += W) {
      const uint32_t b = last_not_above(s_ahead, 0, a.B - 1, i), p = s_prog[b];
      s_tbl[s_new_off[p] + (s_old_off[p + 1] - s_old_off[p]) + (i - s_ahead[b])] = s_page[i];
    }
  }
  __syncthreads();
  // every store from here on: a barrier behind one would wait for it
  if (more || !a.in_place) {
    for (uint32_t e = tid; e < h.entries + more; e += W) a.tbl_to[e] = s_tbl[e];
  }
  if (taken || a.free_to != a.free_map) x.store(a.free_to, a.num_blocks, page0);
  store_batch(a, h, ok, tid);
  if (tid == 0) store_batch(a, h, ok, W);  // one more of each offset than programs and sequences
  if (!a.slots && !a.positions) return;
  uint32_t err = 0;
  for (uint32_t t = tid; t < a.T; t += W) {
    int64_t slot = -1;
    int32_t at = -1;
    if (ok && t < h.tokens) {
      const uint32_t b = last_not_above(s_tok, 0, a.B - 1, t), p = s_prog[b];
      const uint32_t pos = s_len[b] - (s_tok[b + 1] - t), block = divide(pos, a.by_bt);
      const uint32_t page = s_tbl[s_new_off[p] + block];
      at = (int32_t)pos;
      if (page < a.num_blocks) slot = (int64_t)((uint64_t)page * a.bt + (pos - block * a.bt));
      else err |= page == MORI_NO_PAGE ? MORI_DEV_NOT_RESIDENT : MORI_DEV_PAGE_RANGE;
    }
    if (a.slots) a.slots[t] = slot;
    if (a.positions) a.positions[t] = at;
  }
  if (err && a.error) atomicOr(a.error, err);
}

struct Layout {
  uint64_t tile_cnt, old_off, new_off, held_new, tok, ahead, len, prog, aside, bytes;
};
Layout layout_of(const GrowArgs& a) {
  Layout l{};
  uint64_t at = 64;  // the head
  const auto take = [&](uint64_t n) {
    const uint64_t here = at;
    at += (4 * n + 63) / 64 * 64;
    return here;
  };
  l.tile_cnt = take(a.counts);
  l.old_off = take(a.P + 1);
  l.new_off = take(a.P + 1);
  l.held_new = take(a.P);
  l.tok = take(a.B + 1);
  l.ahead = take(a.B + 1);
  l.len = take(a.B);
  l.prog = take(a.B);
  l.aside = take(a.in_place ? a.tbl_len : 0);
  l.bytes = at;
  return l;
}

bool args_of(const mori_pool* pool, const mori_growth* g, GrowArgs* out) {
  GrowArgs& a = *out;
  if (!pool || !g || !pool->block_tokens || !pool->num_blocks || pool->num_blocks == MORI_NO_PAGE) return false;
  if (pool->block_tokens > (1u << 18)) return false;
  if (!g->num_seqs || g->num_seqs > MORI_MAX_PROGRAMS || !g->num_programs || g->num_programs > MORI_MAX_PROGRAMS) return false;
  if (!g->max_kv || (uint64_t)g->max_kv + pool->block_tokens >= (1u << 31) || g->num_tokens >= (1u << 31)) return false;
  if (!g->new_tokens || !g->tbl_off || !g->tbl || !g->held || !g->free_map) return false;
  if (!g->tbl_off_to || !g->tbl_to || !g->held_to || !g->free_to || !g->seq_off || !g->kv_len || !g->tbl_len) return false;
  if ((reinterpret_cast<uintptr_t>(g->free_map) | reinterpret_cast<uintptr_t>(g->free_to)) & 15u) return false;
  a.B = g->num_seqs;
  a.T = g->num_tokens;
  a.max_new = g->max_new;
  a.max_kv = g->max_kv;
  a.P = g->num_programs;
  a.tbl_len = g->tbl_len;
  a.bt = pool->block_tokens;
  a.num_blocks = pool->num_blocks;
  a.counts = (uint32_t)(((uint64_t)a.num_blocks + COUNTED - 1) / COUNTED);
  a.tile = a.counts <= 1024 ? 512 : 4096;
  a.ntiles = (uint32_t)(((uint64_t)a.num_blocks + a.tile - 1) / a.tile);
  a.by_bt = fast_div(a.bt);
  a.new_tokens = g->new_tokens;
  a.program = g->program;
  a.tier = g->tier;
  a.tbl_off = g->tbl_off;
  a.tbl = g->tbl;
  a.held = g->held;
  a.free_map = g->free_map;
  a.tbl_off_to = g->tbl_off_to;
  a.tbl_to = g->tbl_to;
  a.held_to = g->held_to;
  a.free_to = g->free_to;
  a.seq_off = g->seq_off;
  a.kv_len = g->kv_len;
  a.slots = g->slots;
  a.positions = g->positions;
  a.in_place = g->tbl_to == g->tbl;
  a.copies = a.in_place ? (uint32_t)(((uint64_t)a.tbl_len + ENTRIES - 1) / ENTRIES) : 0;
  return true;
}

}  // namespace
}  // namespace mori

extern "C" int mori_tables_grow_workspace(const mori_pool* pool, const mori_growth* growth, uint64_t* bytes) {
  using namespace mori;
  GrowArgs a{};
  if (!bytes || !args_of(pool, growth, &a)) return MORI_EINVAL;
  *bytes = layout_of(a).bytes;
  return MORI_OK;
}

extern "C" int mori_tables_grow(const mori_pool* pool, const mori_growth* growth, void* workspace,
                                uint64_t workspace_bytes, uint32_t* error, void* stream) {
  using namespace mori;
  GrowArgs a{};
  if (!args_of(pool, growth, &a)) return MORI_EINVAL;
  const Layout l = layout_of(a);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < l.bytes) return MORI_EINVAL;
  uint8_t* const w = static_cast<uint8_t*>(workspace);
  const auto at = [&](uint64_t x) { return reinterpret_cast<uint32_t*>(w + x); };
  a.head = reinterpret_cast<Head*>(w);
  a.tile_cnt = at(l.tile_cnt);
  a.old_off = at(l.old_off);
  a.new_off = at(l.new_off);
  a.held_new = at(l.held_new);
  a.tok = at(l.tok);
  a.ahead = at(l.ahead);
  a.len = at(l.len);
  a.prog = at(l.prog);
  a.aside = at(l.aside);
  a.error = error;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const uint32_t most = std::max(a.P, a.B);
  const auto fits = [&](uint32_t w) {
    return most <= w && a.num_blocks <= 16 * w && a.tbl_len <= 8 * w && a.T <= 4 * w;
  };
  if (fits(1024)) {
    if (fits(64)) hipLaunchKernelGGL(grow_small_kernel<64>, dim3(1), dim3(64), 0, s, a);
    else if (fits(256)) hipLaunchKernelGGL(grow_small_kernel<256>, dim3(1), dim3(256), 0, s, a);
    else hipLaunchKernelGGL(grow_small_kernel<1024>, dim3(1), dim3(1024), 0, s, a);
    return hipGetLastError() == hipSuccess ? MORI_OK : MORI_EHIP;
  }
  const auto count = [&](auto kernel, uint32_t threads) {
    const uint64_t pages = 16ull * threads;
    hipLaunchKernelGGL(kernel, dim3(1 + a.copies + (uint32_t)((a.num_blocks + pages - 1) / pages)), dim3(threads), 0, s, a);
  };
  if (most <= 64) count(grow_count_kernel<64, 1>, 64);
  else if (most <= 256) count(grow_count_kernel<256, 1>, 256);
  else if (most <= 1024) count(grow_count_kernel<1024, 1>, 1024);
  else count(grow_count_kernel<1024, 4>, 1024);
  const uint32_t movers = (uint32_t)(((uint64_t)a.tbl_len + ENTRIES - 1) / ENTRIES);
  const uint32_t placers = a.slots || a.positions ? (a.T + NT - 1) / NT : 0;
  const dim3 grid(a.ntiles + movers + placers + (most + NT) / NT);
  if (a.tile == 512) hipLaunchKernelGGL(grow_assign_kernel<2>, grid, dim3(NT), 0, s, a, movers, placers);
  else hipLaunchKernelGGL(grow_assign_kernel<16>, grid, dim3(NT), 0, s, a, movers, placers);
  if (hipGetLastError() != hipSuccess) return MORI_EHIP;
  return MORI_OK;
}
