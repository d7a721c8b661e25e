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
// Two launches, bound by their latency and dependent reads: a byte of the free map per
// page, an entry of the tables in and out, 12 bytes a token.
//   grow_count   one workgroup checks and scans the sequences and programs; the others
//                count free pages by tiles of 4096 and, where the tables grow in place,
//                copy the old entries aside
//   grow_assign  workgroups take a tile each (pages to table entries and to the slots of
//                the tokens in new blocks), or old entries (to where they lie now), or
//                tokens in old blocks, or programs.  Every workgroup sums the tile counts
//                for itself, so all of them know whether there are pages enough: nothing
//                is changed unless everything is.
#include "tokens.h"

namespace mori {
namespace {

constexpr uint32_t TILE = 4096;    // pages of a workgroup of grow_assign, 16 a thread
constexpr uint32_t COUNT_NT = 1024, NT = 256;
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
  uint32_t B, T, max_new, max_kv, P, tbl_len, bt, num_blocks, ntiles;
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

// Sums of every thread's value before it (by thread) and of all; a workgroup of up to
// 16 wavefronts, all of it here.
struct Scan {
  uint32_t before, total;
};
__device__ inline Scan scan_of(uint32_t v, uint32_t* s_wave, uint32_t waves) {
  const uint32_t lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const uint32_t in = wave::incl_add(v);
  if (lane == 63) s_wave[wv] = in;
  __syncthreads();
  Scan s{in - v, 0};
  for (uint32_t i = 0; i < waves; ++i) {
    const uint32_t x = s_wave[i];
    if (i < wv) s.before += x;
    s.total += x;
  }
  __syncthreads();
  return s;
}

// Bytes that are not 0.
__device__ inline uint32_t set_bytes(uint32_t w) {
  return (((w & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | w) & 0x80808080u;
}

// 16 pages of the free map from `page` on; those past the pool are not free.
__device__ inline uint4 free_pages(const GrowArgs& a, uint32_t page) {
  if ((uint64_t)page + 16 <= a.num_blocks) return *reinterpret_cast<const uint4*>(a.free_map + page);
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (uint32_t i = 0; i < 16; ++i)
    if ((uint64_t)page + i < a.num_blocks) w[i / 4] |= (uint32_t)a.free_map[page + i] << (8 * (i % 4));
  return uint4{w[0], w[1], w[2], w[3]};
}
__device__ inline uint32_t count_set(uint4 w) {
  return __popc(set_bytes(w.x)) + __popc(set_bytes(w.y)) + __popc(set_bytes(w.z)) + __popc(set_bytes(w.w));
}

// The batch and the programs: checks, scans, and what grow_assign reads of them.
__device__ void scan_batch(const GrowArgs& a) {
  constexpr uint32_t K = MOST / COUNT_NT;
  __shared__ uint32_t s_more[MOST], s_len[MOST];  // by program; NONE: no sequence of the batch
  __shared__ uint32_t s_wave[COUNT_NT / 64], s_error;
  constexpr uint32_t NONE = 0xFFFFFFFFu, CLAIMED = 0xFFFFFFFEu;
  const uint32_t tid = threadIdx.x;
  uint32_t err = 0, bad_off = 0;
  if (tid == 0) s_error = 0;
  for (uint32_t p = tid; p < a.P; p += COUNT_NT) s_more[p] = NONE;
  // neighbouring programs and sequences a thread
  uint32_t lo[K], hi[K], n[K], prog[K], more[K], len[K];
#pragma unroll
  for (uint32_t k = 0; k < K; ++k) {
    const uint32_t p = K * tid + k;
    lo[k] = hi[k] = 0;
    if (p < a.P) {
      lo[k] = a.tbl_off[p];
      hi[k] = a.tbl_off[p + 1];
      bad_off |= lo[k] > hi[k] || hi[k] > a.tbl_len || (p == 0 && lo[k]);
    }
  }
  __syncthreads();
  const bool sound = !__syncthreads_or(bad_off);
  if (!sound) err |= MORI_DEV_BAD_TBL_OFF;
#pragma unroll
  for (uint32_t k = 0; k < K; ++k) {
    const uint32_t b = K * tid + k;
    n[k] = more[k] = len[k] = 0;
    prog[k] = NONE;
    if (b >= a.B) continue;
    const uint32_t p = a.program ? a.program[b] : b, x = a.new_tokens[b];
    if (p >= a.P || atomicCAS(&s_more[p], NONE, CLAIMED) != NONE) {  // no program, or one that is here already
      err |= MORI_DEV_BAD_TOKENS;
      continue;
    }
    prog[k] = p;
    const uint32_t h = a.held[p], blocks = sound ? a.tbl_off[p + 1] - a.tbl_off[p] : 0;
    if (a.tier && a.tier[p] != MORI_TIER_GPU) err |= MORI_DEV_NOT_RESIDENT;
    if (x > a.max_new || (uint64_t)h + x > a.max_kv || h > (uint64_t)blocks * a.bt) {
      err |= MORI_DEV_BAD_TOKENS;
      continue;
    }
    n[k] = x;
    len[k] = h + x;  // below 2^31
    const uint32_t need = divide(len[k] + a.bt - 1, a.by_bt);
    more[k] = need > blocks ? need - blocks : 0;
  }
  __syncthreads();
#pragma unroll
  for (uint32_t k = 0; k < K; ++k)
    if (prog[k] != NONE) {
      s_more[prog[k]] = more[k];
      s_len[prog[k]] = len[k];
    }
  // sums in 64 bits first, so that none wraps unseen
  uint64_t n_sum = 0, m_sum = 0, e_sum = 0;
#pragma unroll
  for (uint32_t k = 0; k < K; ++k) {
    n_sum += n[k];
    m_sum += more[k];
  }
  __shared__ uint64_t s_n, s_m, s_e;
  if (tid == 0) s_n = s_m = s_e = 0;
  __syncthreads();
#pragma unroll
  for (uint32_t k = 0; k < K; ++k) {
    const uint32_t p = K * tid + k;
    if (p < a.P) {
      const uint32_t m = s_more[p];
      hi[k] -= lo[k];  // blocks from here on
      e_sum += (uint64_t)(sound ? hi[k] : 0) + (m < CLAIMED ? m : 0);
    }
  }
  n_sum = wave::sum(n_sum);
  m_sum = wave::sum(m_sum);
  e_sum = wave::sum(e_sum);
  if ((tid & 63) == 0) {
    atomicAdd(reinterpret_cast<unsigned long long*>(&s_n), n_sum);
    atomicAdd(reinterpret_cast<unsigned long long*>(&s_m), m_sum);
    atomicAdd(reinterpret_cast<unsigned long long*>(&s_e), e_sum);
  }
  __syncthreads();
  if (s_n > a.T) err |= MORI_DEV_BAD_TOKENS;
  if (s_m > a.num_blocks || s_e > a.tbl_len) err |= MORI_DEV_NOSPC;
  if (err) atomicOr(&s_error, err);
  __syncthreads();
  const uint32_t error = s_error;
  if (error) {  // nothing grows
#pragma unroll
    for (uint32_t k = 0; k < K; ++k) n[k] = more[k] = len[k] = 0;
  }
  uint32_t v = 0, w = 0;
#pragma unroll
  for (uint32_t k = 0; k < K; ++k) {
    v += n[k];
    w += more[k];
  }
  const Scan t = scan_of(v, s_wave, COUNT_NT / 64), m = scan_of(w, s_wave, COUNT_NT / 64);
  v = t.before;
  w = m.before;
#pragma unroll
  for (uint32_t k = 0; k < K; ++k) {
    const uint32_t b = K * tid + k;
    if (b < a.B) {
      a.tok[b] = v;
      a.ahead[b] = w;
      a.len[b] = len[k];
      a.prog[b] = prog[k];
    }
    v += n[k];
    w += more[k];
  }
  uint32_t e = 0;
#pragma unroll
  for (uint32_t k = 0; k < K; ++k) {
    const uint32_t p = K * tid + k;
    more[k] = 0;
    if (p < a.P && sound) {
      const uint32_t x = s_more[p];
      more[k] = hi[k] + (x < CLAIMED && !error ? x : 0);
    }
    e += more[k];
  }
  const Scan all = scan_of(e, s_wave, COUNT_NT / 64);
  e = all.before;
#pragma unroll
  for (uint32_t k = 0; k < K; ++k) {
    const uint32_t p = K * tid + k;
    if (p < a.P) {
      a.new_off[p] = e;
      a.old_off[p] = lo[k];
      a.held_new[p] = s_more[p] < CLAIMED && !error ? s_len[p] : a.held[p];
    }
    e += more[k];
    if (p == a.P - 1) {
      a.new_off[a.P] = e;
      a.old_off[a.P] = lo[k] + hi[k];
      *a.head = Head{error, m.total, t.total, sound ? lo[k] + hi[k] : 0, sound};
    }
  }
  if (tid == 0) {
    a.tok[a.B] = t.total;
    a.ahead[a.B] = m.total;
    if (error && a.error) atomicOr(a.error, error);
  }
}

__global__ __launch_bounds__(COUNT_NT) void grow_count_kernel(GrowArgs a) {
  if (blockIdx.x == 0) {
    scan_batch(a);
    return;
  }
  const uint32_t tid = threadIdx.x, i = blockIdx.x - 1;
  if (i < a.copies) {
    const uint32_t n = min(a.tbl_off[a.P], a.tbl_len);
    const uint64_t e0 = (uint64_t)i * (4 * COUNT_NT) + tid;
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k)
      if (e0 + k * COUNT_NT < n) a.aside[e0 + k * COUNT_NT] = a.tbl[e0 + k * COUNT_NT];
    return;
  }
  // four tiles, four wavefronts each
  __shared__ uint32_t s_count[COUNT_NT / 64];
  const uint32_t tile0 = (i - a.copies) * (COUNT_NT / NT);
  const uint64_t page = (uint64_t)tile0 * TILE + 16ull * tid;
  const uint32_t n = page < a.num_blocks ? count_set(free_pages(a, (uint32_t)page)) : 0;
  const uint32_t sum = wave::sum(n);
  if ((tid & 63) == 0) s_count[tid >> 6] = sum;
  __syncthreads();
  if (tid < COUNT_NT / NT && tile0 + tid < a.ntiles)
    a.tile_cnt[tile0 + tid] = s_count[4 * tid] + s_count[4 * tid + 1] + s_count[4 * tid + 2] + s_count[4 * tid + 3];
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
// The same by a thread between two indexes.
__device__ inline uint32_t last_not_above(const uint32_t* x, uint32_t lo, uint32_t hi, uint32_t v) {
  while (lo < hi) {
    const uint32_t mid = (lo + hi + 1) / 2;
    if (x[mid] <= v) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// A tile's pages: to the programs that take them, and out of the free map.
__device__ void assign_tile(const GrowArgs& a, const Head& h, bool ok, uint32_t tile, uint32_t base) {
  __shared__ uint32_t s_page[TILE], s_seq[TILE], s_ahead[MOST + 1], s_wave[NT / 64];
  const uint32_t tid = threadIdx.x;
  const uint64_t page0 = (uint64_t)tile * TILE + 16ull * tid;
  uint4 w{0, 0, 0, 0};
  if (page0 < a.num_blocks) w = free_pages(a, (uint32_t)page0);
  const uint32_t mine = count_set(w), more = ok ? h.more : 0;
  const bool some = base < more;  // of this tile's pages some are taken
  if (some) {
    for (uint32_t b = tid; b <= a.B; b += NT) s_ahead[b] = a.ahead[b];
    const Scan s = scan_of(mine, s_wave, NT / 64);
    uint32_t r = base + s.before;
    uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (uint32_t i = 0; i < 16; ++i) {
      const uint32_t bit = 0xFFu << (8 * (i % 4));
      if (v[i / 4] & bit) {
        if (r < more) {
          s_page[r - base] = (uint32_t)page0 + i;
          v[i / 4] &= ~bit;
        }
        ++r;
      }
    }
    w = uint4{v[0], v[1], v[2], v[3]};
    __syncthreads();
    const uint32_t count = min(more - base, s.total);
    for (uint32_t i = tid; i < count; i += NT) {
      // sequences that take none share their number with the next: the last of them takes it
      const uint32_t b = last_not_above(s_ahead, 0, a.B - 1, base + i), p = a.prog[b];
      s_seq[i] = b;
      const uint32_t block = a.old_off[p + 1] - a.old_off[p] + (base + i - s_ahead[b]);
      a.tbl_to[a.new_off[p] + block] = s_page[i];
    }
    __syncthreads();
    if (a.slots || a.positions) {  // every token of a new block is new
      for (uint32_t x = tid; x < count * a.bt; x += NT) {  // below 2^30
        const uint32_t i = divide(x, a.by_bt), row = x - i * a.bt, b = s_seq[i], p = a.prog[b];
        const uint32_t block = a.old_off[p + 1] - a.old_off[p] + (base + i - s_ahead[b]);
        const uint64_t pos = (uint64_t)block * a.bt + row;
        const uint32_t len = a.len[b], held = len - (a.tok[b + 1] - a.tok[b]);
        if (pos >= len) continue;
        const uint32_t t = a.tok[b] + ((uint32_t)pos - held);
        if (a.slots) a.slots[t] = (int64_t)((uint64_t)s_page[i] * a.bt + row);
        if (a.positions) a.positions[t] = (int32_t)pos;
      }
    }
  }
  if (page0 < a.num_blocks && (some || a.free_to != a.free_map)) {
    if (page0 + 16 <= a.num_blocks) {
      *reinterpret_cast<uint4*>(a.free_to + page0) = w;
    } else {
      const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (uint32_t i = 0; i < 16; ++i)
        if (page0 + i < a.num_blocks) a.free_to[page0 + i] = (uint8_t)(v[i / 4] >> (8 * (i % 4)));
    }
  }
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

__global__ __launch_bounds__(NT) void grow_assign_kernel(GrowArgs a, uint32_t movers, uint32_t placers) {
  __shared__ uint32_t s_before[NT / 64], s_total[NT / 64];
  const uint32_t tid = threadIdx.x, lane = tid & 63;
  uint32_t i = blockIdx.x;
  const Head h = *a.head;
  // free pages in the tiles before this one and in all; neither is needed where nothing is taken
  uint32_t before = 0, total = 0;
  if (h.more) {
    for (uint32_t k = tid; k < a.ntiles; k += NT) {
      const uint32_t n = a.tile_cnt[k];
      total += n;
      if (k < i) before += n;
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
    assign_tile(a, h, ok, i, before);
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
  i -= placers;
  if (i == 0 && tid == 0 && !h.error && !ok && a.error) atomicOr(a.error, MORI_DEV_NOSPC);
  const uint32_t x = i * NT + tid;
  if (x <= a.B) a.seq_off[x] = ok ? a.tok[x] : 0;
  if (x < a.B) a.kv_len[x] = ok ? a.len[x] : 0;
  if (x < a.P && (ok || a.held_to != a.held)) a.held_to[x] = ok ? a.held_new[x] : a.held[x];
  if (x <= a.P && h.sound) a.tbl_off_to[x] = ok ? a.new_off[x] : a.old_off[x];
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
  l.tile_cnt = take(a.ntiles);
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
  a.ntiles = (uint32_t)(((uint64_t)a.num_blocks + TILE - 1) / TILE);
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
  a.copies = a.in_place ? (uint32_t)(((uint64_t)a.tbl_len + 4 * COUNT_NT - 1) / (4 * COUNT_NT)) : 0;
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
  const uint32_t counters = (a.ntiles + COUNT_NT / NT - 1) / (COUNT_NT / NT);
  hipLaunchKernelGGL(grow_count_kernel, dim3(1 + a.copies + counters), dim3(COUNT_NT), 0, s, a);
  const uint32_t movers = (uint32_t)(((uint64_t)a.tbl_len + ENTRIES - 1) / ENTRIES);
  const uint32_t placers = a.slots || a.positions ? (a.T + NT - 1) / NT : 0;
  const uint32_t rest = (max(a.P, a.B) + NT) / NT;
  hipLaunchKernelGGL(grow_assign_kernel, dim3(a.ntiles + movers + placers + rest), dim3(NT), 0, s, a, movers, placers);
  if (hipGetLastError() != hipSuccess) return MORI_EHIP;
  return MORI_OK;
}
