// The tokens of a batch on the device: which sequence a token belongs to, where
// it stands in its program, and which pool page holds a position.  Shared by the
// append and the attention kernels.
//
// Every index that comes from device memory is checked before it is used: a
// sequence whose numbers do not fit becomes padding, a page id outside the pool
// is never turned into an address.
#pragma once
#include "mori_internal.h"
#include "wave.h"

namespace mori {

// Division of n < 2^31 by a d that stays the same: (2 n * m) >> (32 + l) with
// l = ceil(log2 d), m = ceil(2^(31 + l) / d) < 2^32, which is exact for such n.
struct FastDiv {
  uint32_t m, l;
};
inline FastDiv fast_div(uint32_t d) {
  uint32_t l = 0;
  while ((1ull << l) < d) ++l;
  return {(uint32_t)(((1ull << (31 + l)) + d - 1) / d), l};
}
__device__ inline uint32_t divide(uint32_t n, FastDiv d) { return __umulhi(n << 1, d.m) >> d.l; }

// The batch and the pool's layer as the kernels take them.
struct Batch {
  uint32_t B, T, max_new, max_kv;
  const uint32_t* seq_off;
  const uint32_t* kv_len;
  const uint32_t* program;
  uint32_t P, tbl_len;
  const uint32_t* tbl_off;
  const uint32_t* tbl;
  uint32_t bt, num_blocks;
  FastDiv by_bt;
  uint64_t run;          // bytes of one page in one plane
  uint32_t row;          // bytes of one token in one plane
  uint8_t* plane;        // the layer's first plane
  uint64_t plane_bytes;  // from one plane to the next
  uint32_t* error;
};

// Host check of what both calls take; fills the kernel's form.
inline bool batch_of(const mori_pool* pool, uint32_t layer, const mori_tokens* t, uint32_t* error, Batch* out) {
  if (!pool || !t || !pool_valid(*pool) || layer >= pool->layers) return false;
  if (pool->planes != 1 && pool->planes != 2) return false;
  if (!t->num_seqs || t->num_seqs > MORI_MAX_PROGRAMS || !t->seq_off || !t->kv_len || !t->tbl_off) return false;
  if (!t->num_programs || !t->max_kv || t->max_kv >= (1u << 31) || t->num_tokens >= (1u << 31)) return false;
  if (t->tbl_len && !t->tbl) return false;
  Batch& b = *out;
  b.B = t->num_seqs;
  b.T = t->num_tokens;
  b.max_new = t->max_new;
  b.max_kv = t->max_kv;
  b.seq_off = t->seq_off;
  b.kv_len = t->kv_len;
  b.program = t->program;
  b.P = t->num_programs;
  b.tbl_len = t->tbl_len;
  b.tbl_off = t->tbl_off;
  b.tbl = t->tbl;
  b.bt = pool->block_tokens;
  b.num_blocks = pool->num_blocks;
  b.by_bt = fast_div(b.bt);
  b.row = pool->row_bytes;
  b.run = (uint64_t)b.bt * b.row;
  b.plane_bytes = b.run * b.num_blocks;
  b.plane = static_cast<uint8_t*>(pool->base) + (uint64_t)layer * pool->planes * b.plane_bytes;
  b.error = error;
  return true;
}

// A [tokens][heads][elements] array of 16-bit floats: 16-B chunks stay aligned.
inline bool rows_valid(const mori_rows& r) {
  return r.data && !(reinterpret_cast<uintptr_t>(r.data) & 15u) && !(r.token_stride & 7u) && !(r.head_stride & 7u);
}

struct Rows {
  uint8_t* data;
  uint64_t token, head;  // strides in bytes
};
inline Rows rows_of(const mori_rows& r) {
  return {static_cast<uint8_t*>(r.data), 2 * r.token_stride, 2 * r.head_stride};
}

// One sequence of the batch.
struct Seq {
  uint32_t t0, n;     // its tokens
  uint32_t len;       // the program's tokens with them
  uint32_t tbl;       // its first entry in the table
  uint32_t error;     // MORI_DEV_* bits; padding then (len 0)
  bool named;         // its token range is in bounds
  __device__ int32_t position(uint32_t i) const { return (int32_t)(len + i) - (int32_t)n; }
};

// What the batch and the tables say of a sequence.
struct SeqNumbers {
  uint32_t lo, hi, len, p, first, last;
};
__device__ inline SeqNumbers read_sequence(const Batch& a, uint32_t b) {
  SeqNumbers x{a.seq_off[b], a.seq_off[b + 1], a.kv_len[b], a.program ? a.program[b] : b, 1, 0};
  if (x.p < a.P) {
    x.first = a.tbl_off[x.p];
    x.last = a.tbl_off[x.p + 1];
  }
  return x;
}

// A sequence, checked.  Every bound that later indexing relies on holds
// afterwards: t0 + n <= T, and len <= blocks * bt with tbl + blocks <= tbl_len.
__device__ inline Seq checked_sequence(const Batch& a, const SeqNumbers& x) {
  Seq s{};
  if (x.lo > x.hi || x.hi > a.T) {
    s.error = MORI_DEV_BAD_TOKENS;
    return s;
  }
  s.named = true;
  s.t0 = x.lo;
  s.n = x.hi - x.lo;
  if (s.n > a.max_new || x.len > a.max_kv || x.p >= a.P || x.first > x.last || x.last > a.tbl_len ||
      (uint64_t)(x.last - x.first) * a.bt < x.len) {
    s.error = MORI_DEV_BAD_TOKENS;
    return s;
  }
  s.tbl = x.first;
  s.len = x.len;
  return s;
}
__device__ inline Seq sequence(const Batch& a, uint32_t b) { return checked_sequence(a, read_sequence(a, b)); }

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

// The page of a block as the table has it: its id, or 0 and the error bit.
__device__ inline uint32_t checked_page(const Batch& a, uint32_t id, uint32_t* err) {
  if (id < a.num_blocks) return id;
  *err |= id == MORI_NO_PAGE ? MORI_DEV_NOT_RESIDENT : MORI_DEV_PAGE_RANGE;
  return 0;
}

__device__ inline void report(const Batch& a, uint32_t err) {
  if (err && a.error) atomicOr(a.error, err);
}

}  // namespace mori
