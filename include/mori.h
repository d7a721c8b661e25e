/*
 * mori.h -- C ABI of libmori: the MI355X (gfx950) hot path of MORI's
 * idleness-ranked KV-cache placement (arXiv 2606.00866, "Idleness is
 * Relative: Exploiting Tool-Call Idle Windows for Offloading in Agentic
 * Systems with MORI").
 *
 * One rebalance of the three-tier placement of Sec. 4.1 (GPU HBM, CPU DRAM,
 * Waiting), as three calls:
 *
 *   mori_rank_partition  Eq. 1 idleness of every program (Sec. 4.2), the
 *                        relative ranking (Sec. 1, Sec. 4.3), the
 *                        capacity-matched GPU and CPU boundaries (Sec. 4.1
 *                        per-tier capacity, Sec. 7.2 fill from the busiest
 *                        end), the sticky diff (Sec. 4.3: only programs that
 *                        cross the boundary move), page allocation and the
 *                        block-table rewrite.
 *   mori_kv_swap_out     gathers the demoted programs' scattered KV pages into
 *                        one contiguous buffer per program (GPU -> CPU).
 *   mori_kv_swap_in      scatters the promoted programs' bytes into the pages
 *                        allocated for them (CPU -> GPU, Sec. 4.1: a CPU-tier
 *                        program resumes over PCIe).
 *
 * Beside them the calls of a model's step: mori_tables_grow gives programs that
 * take new tokens the pages they need, and in every layer mori_kv_append writes
 * the tokens' keys and values and mori_kv_attend reads them (mori_kv_append_axes and
 * mori_kv_attend_sight: with positions of several axes, and with more to say of
 * scores and of what a token sees).
 *
 * Conventions
 *   - Every call returns an int: MORI_OK (0) or a negative MORI_E* code.
 *     Nothing throws across the ABI.  Errors found on the host are reported
 *     before anything is enqueued and leave all caller memory untouched.
 *   - Device-side validation (program data, pool consistency, host
 *     addresses) sets bits of a device error word (MORI_DEV_*).  A plan that
 *     fails validation modifies no caller memory; its error is returned by
 *     mori_plan_wait and mori_query.
 *   - Streams are hipStream_t values passed as void*; NULL is the default
 *     stream.  The library never synchronises the device.  It blocks the host
 *     in mori_plan_wait, in copy-engine swaps (which need the plan), in
 *     mori_query(MORI_Q_DEVICE_ERROR), mori_profile_read, mori_register and
 *     mori_destroy; a kernel-mode swap waits until the previous one of its
 *     direction has read its address table.
 *   - Threads: a context is driven by one host thread at a time (its calls
 *     are not synchronised against each other); distinct contexts share no
 *     state, and mori_evict_order, mori_replica_admit, mori_tables_grow and
 *     the calls on tokens keep none.
 *   - Ownership: the caller owns the pool, the program arrays, the host
 *     buffers and the streams.  The context owns its device scratch, a small
 *     pinned mirror of the plan and, for copy-engine swaps, device staging
 *     buffers, all allocated in mori_create and freed in mori_destroy.
 *
 * Layouts
 *   pool   [layers * planes][num_blocks][block_tokens][row_bytes] bytes in
 *          HBM.  A "run" is one (plane, page): block_tokens * row_bytes
 *          contiguous bytes.  A page of a program spans every plane.
 *   host   one contiguous buffer per CPU-resident program p:
 *          [layers * planes][nblk_p][block_tokens][row_bytes], so each
 *          program's runs of one plane are adjacent.
 *   nblk_p = tbl_off[p+1] - tbl_off[p] whole blocks; a program is never split
 *          across tiers (Sec. 1: a program sits in exactly one tier at a time).
 */
#ifndef MORI_H
#define MORI_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- return codes ---------------------------------------------------- */
#define MORI_OK 0
#define MORI_EINVAL (-1)  /* bad argument: null/misaligned pointer, size, flag or mode */
#define MORI_ENOSPC (-2)  /* capacity: too many programs, staging too small, registry full */
#define MORI_ESTATE (-3)  /* call out of order (swap without a plan, swap twice, ...) */
#define MORI_EHIP (-4)    /* a HIP runtime call failed; mori_query(MORI_Q_LAST_HIP_ERROR) */
#define MORI_EDEVICE (-5) /* device-side validation failed; see the MORI_DEV_* bits */

/* ---- device error word bits ------------------------------------------- */
#define MORI_DEV_BAD_WINDOW 0x001u    /* window value negative, NaN or inf, or a total overflowed */
#define MORI_DEV_BAD_IDLENESS 0x002u  /* given idleness outside [0, 1] */
#define MORI_DEV_BAD_TIER 0x004u      /* tier value > 2 */
#define MORI_DEV_BAD_TBL_OFF 0x008u   /* tbl_off not starting at 0, decreasing, or past tbl_len */
#define MORI_DEV_PAGE_RANGE 0x010u    /* a GPU program's page id >= num_blocks */
#define MORI_DEV_PAGE_DUP 0x020u      /* a page owned twice, or owned and marked free */
#define MORI_DEV_PAGE_LEAK 0x040u     /* a page neither free nor owned */
#define MORI_DEV_NONRES_PAGE 0x080u   /* a CPU/Waiting program's table holds a page */
#define MORI_DEV_NOSPC 0x100u         /* not enough pages (plans: unreachable for a consistent pool) or table entries */
#define MORI_DEV_HOST_ADDR 0x200u     /* swap address not 16-B aligned or outside registered memory */
#define MORI_DEV_BAD_BLOCK 0x400u     /* eviction order: type label > 2 or last access >= 2^62 */
#define MORI_DEV_BAD_STATUS 0x800u    /* incremental policy: status value > 2 */
#define MORI_DEV_STALL 0x1000u        /* reserved (no kernel waits for another workgroup) */
#define MORI_DEV_BAD_TOKENS 0x2000u   /* tokens: offsets, a length or a program out of their bounds */
#define MORI_DEV_NOT_RESIDENT 0x4000u /* tokens: a block they need has no page (MORI_NO_PAGE) */
/* classes: program data = 0x00F and 0x800, pool state = 0x0F0, capacity = 0x100, swap = 0x200,
   blocks = 0x400, tokens = 0x6000 (and PAGE_RANGE) */

/* ---- tiers, table sentinel, flags, copy modes -------------------------- */
#define MORI_TIER_GPU 0u
#define MORI_TIER_CPU 1u
#define MORI_TIER_WAIT 2u
#define MORI_TIER_SSD 3u /* only with MORI_F_SSD_TIER (Sec. 7.1: storage below the CPU tier) */
#define MORI_NO_PAGE 0xFFFFFFFFu

#define MORI_F_STATUS_KEY 1u     /* Acting programs (status 1) rank after all Reasoning ones */
#define MORI_F_SKIP_FIT 2u       /* greedy fit in rank order instead of a strict prefix */
#define MORI_F_IDLENESS_GIVEN 4u /* use programs.idleness instead of windows */
#define MORI_F_INCREMENTAL 8u    /* incremental sticky policy of Sec. 4.3.1 instead of the boundary */
#define MORI_F_SSD_TIER 16u      /* a third boundary in the ranking: the SSD tier (Sec. 7.1) */

/* program status (Sec. 4.1), read with MORI_F_STATUS_KEY or MORI_F_INCREMENTAL */
#define MORI_ST_REASONING 0u /* running inference or waiting for it */
#define MORI_ST_ACTING 1u    /* inside a tool call */
#define MORI_ST_NEW 2u       /* newly arrived, waiting for its first inference (Reasoning elsewhere) */

#define MORI_COPY_AUTO 0u   /* copy engines (chosen by measurement on MI355X) */
#define MORI_COPY_KERNEL 1u /* kernels load/store host-mapped memory directly; no host sync */
#define MORI_COPY_CE 2u     /* kernel gather/scatter through device staging + SDMA copies */

/* transition categories (mori_plan.category) */
#define MORI_CAT_KEPT 0u
#define MORI_CAT_OUT 1u       /* GPU -> CPU or SSD: bytes gathered to the host */
#define MORI_CAT_IN 2u        /* CPU or SSD -> GPU: bytes scattered into new pages */
#define MORI_CAT_DROP_GPU 3u  /* GPU -> Waiting: pages released, KV discarded */
#define MORI_CAT_DROP_CPU 4u  /* CPU -> Waiting */
#define MORI_CAT_ADMIT_GPU 5u /* Waiting -> GPU: pages reserved, no copy */
#define MORI_CAT_ADMIT_CPU 6u /* Waiting -> CPU: no copy */
#define MORI_CAT_CPU_SSD 7u   /* CPU -> SSD: the caller writes the host buffer to storage */
#define MORI_CAT_SSD_CPU 8u   /* SSD -> CPU: the caller reads it back into a host buffer */
#define MORI_CAT_DROP_SSD 9u  /* SSD -> Waiting */
#define MORI_CAT_ADMIT_SSD 10u /* Waiting -> SSD: no copy */

#define MORI_MAX_PROGRAMS 4096u
#define MORI_MAX_WINDOW 64u
#define MORI_MAX_RANGES 64u

typedef struct mori_ctx mori_ctx;

/* The paged KV pool in HBM (PagedAttention-style blocks, Sec. 2.1). */
typedef struct {
  uint32_t layers;       /* >= 1 */
  uint32_t planes;       /* >= 1: 2 for K and V, 1 for a compressed latent */
  uint32_t block_tokens; /* >= 1 tokens per block */
  uint32_t row_bytes;    /* bytes per token per (layer, plane); multiple of 16 */
  uint32_t num_blocks;   /* pages in the pool, < 2^32 - 1 */
  void* base;            /* device pointer, 256-B aligned, layout in the header comment */
} mori_pool;

/* Per-program state (Sec. 4.1: status, context size and recent durations). */
typedef struct {
  uint32_t num_programs;   /* P <= max_programs of the context */
  uint32_t window_k;       /* cycles per idleness window, 1..MORI_MAX_WINDOW (the paper uses 5) */
  const float* window;     /* device [P][window_k][2]: (reasoning s, acting s), oldest cycle
                              first; the newest acting entry is the ongoing call's elapsed time */
  const float* idleness;   /* device [P]; read only with MORI_F_IDLENESS_GIVEN */
  const uint8_t* status;   /* device [P] MORI_ST_*; read only with MORI_F_STATUS_KEY (where only
                              MORI_ST_ACTING counts) or MORI_F_INCREMENTAL */
  const uint32_t* tbl_off; /* device [P+1] CSR offsets into tbl; nblk_p = tbl_off[p+1]-tbl_off[p] */
  uint32_t tbl_len;        /* entries allocated in tbl (>= tbl_off[P]) */
  uint32_t* tbl;           /* device [tbl_len], in/out: page id of each logical block of a
                              GPU-resident program, MORI_NO_PAGE for every other program */
  uint8_t* tier;           /* device [P], in/out: current tier -> new tier */
  uint8_t* free_map;       /* device [num_blocks], in/out: 1 = page free */
} mori_programs;

/* Per-tier capacity (Sec. 4.1: neither tier may exceed its memory). */
typedef struct {
  uint64_t gpu_bytes; /* <= num_blocks * block bytes */
  uint64_t cpu_bytes;
  uint32_t flags;     /* MORI_F_* */
  uint64_t ssd_bytes; /* read only with MORI_F_SSD_TIER */
} mori_budget;

/* The plan of the last mori_rank_partition, as mirrored on the host.  The
 * array pointers refer to context-owned pinned memory, valid until the next
 * mori_rank_partition or mori_destroy. */
typedef struct {
  uint32_t num_programs, m_gpu, m_cpu;
  uint32_t n_out, n_in, n_drop_gpu, n_drop_cpu, n_admit_gpu, n_admit_cpu;
  uint32_t device_error; /* MORI_DEV_* bits; 0 when the plan is valid */
  uint32_t m_ssd;        /* programs on the SSD tier (0 without MORI_F_SSD_TIER) */
  uint64_t pages_out, pages_in, pages_admit;
  uint64_t pages_free_before, pages_released, pages_recycled, pages_free_after;
  uint64_t bytes_out, bytes_in, gpu_bytes_after, cpu_bytes_after, ssd_bytes_after;
  uint64_t pages_dropped; /* released pages of idle programs dropped to Waiting (nothing uses them) */
  const uint32_t* order;        /* [P] program ids, busiest first (incremental: see below) */
  const uint64_t* prefix;       /* [P] inclusive KV-byte prefix in rank order */
  const uint8_t* tier_old;      /* [P] */
  const uint8_t* tier_new;      /* [P] */
  const uint8_t* category;      /* [P] MORI_CAT_* */
  const uint32_t* out_programs; /* [n_out] in rank order */
  const uint32_t* in_programs;  /* [n_in] in rank order */
} mori_plan;

/* ---- context ----------------------------------------------------------- */

/* Creates a context for one pool on the current HIP device.  max_programs <=
 * MORI_MAX_PROGRAMS bounds P of every later call.  staging_bytes is the
 * device staging of copy-engine swaps per direction (0: 512 MiB), used as two
 * halves of whole runs (it must hold at least two runs); copy-engine swaps
 * move the bytes in chunks of one half.  flags:
 *   MORI_CREATE_COPY_STREAMS  the context owns one copy stream per direction,
 *     so the copy engines drain one staging half while the gather/scatter
 *     kernel works on the other.  HIP maps a process's streams onto
 *     GPU_MAX_HW_QUEUES hardware queues (4 by default, read when HIP starts)
 *     and streams beyond that share queues, where one stream's waits block
 *     the other's work and the two swap directions serialise; set the flag
 *     only when the process has at least 8 queues (the two swap streams, the
 *     two copy streams).  Without it the copies run on the caller's stream,
 *     in order with the kernels.
 * The two streams given to the swaps should be distinct and created early
 * (streams beyond the queue count share queues).  *out is set on success.
 * EINVAL: null pool/out, unknown flags, bad geometry or alignment; EHIP:
 * allocation. */
#define MORI_CREATE_COPY_STREAMS 1u
int mori_create(const mori_pool* pool, uint32_t max_programs, uint64_t staging_bytes, uint32_t flags,
                mori_ctx** out);

/* Waits for the context's outstanding work and frees it.  NULL is a no-op. */
int mori_destroy(mori_ctx* ctx);

/* Registers a range that swap buffers may live in: pinned host memory from
 * hipHostMalloc / mori_host_alloc (used through its device mapping), or
 * device memory (then swaps are device-to-device gathers and scatters).  The
 * swap kernels touch no address outside registered ranges.  EINVAL: null,
 * zero size, or memory HIP does not know; ENOSPC: MORI_MAX_RANGES reached. */
int mori_register(mori_ctx* ctx, void* ptr, uint64_t bytes);

/* Pinned, device-mapped host memory for the CPU tier (hipHostMalloc with the
 * mapped and portable flags), and its release. */
int mori_host_alloc(uint64_t bytes, void** out);
int mori_host_free(void* ptr);

/* ---- the hot path ------------------------------------------------------ */

/* Computes the new placement and rewrites tbl, tier and free_map in stream
 * order.  Waits (on the stream) for the previous plan's swaps.  The plan is
 * stored into the context's pinned host mirror by the kernels; read it with
 * mori_plan_wait.
 *
 * Pages for programs entering the GPU are handed out in this order: pages
 * free before the step; then pages of programs dropped to Waiting that
 * nothing uses any more; then, together, pages of swapped-out programs (free
 * once the swap-out has read them) and pages of programs dropped while they
 * may still be running an inference step (free once that step has ended);
 * each group in ascending page id.  A dropped program counts as running when
 * the plan reads statuses (MORI_F_STATUS_KEY or MORI_F_INCREMENTAL) and its
 * status is not MORI_ST_ACTING (Sec. 4.3.1 demotes a Reasoning victim lazily:
 * its current step is not interrupted); without statuses the caller vouches
 * that dropped programs are idle.  The caller orders such a program's current
 * step before mori_kv_swap_out on the swap-out stream.  Programs promoted
 * from a lower tier take the pages first, then programs admitted from
 * Waiting, each group in rank order, blocks in logical order.  A slot at or
 * past pages_free_before + pages_dropped is on a page still in use: the
 * swap-in waits for the swap-out stream before writing it, and the caller
 * (MORI_Q_OUT_EVENT) before prefilling it.
 *
 * Default policy (Sec. 4.3, Sec. 7.2): rank all programs by idleness (Eq. 1),
 * busiest first, and fill the GPU tier, then the CPU tier, from the busiest
 * end; a program moves only when it crosses a boundary.
 *
 * MORI_F_INCREMENTAL (Sec. 4.3.1; status required): tiers change only to
 * repair a capacity violation or to fill free GPU room.  (1) While the CPU
 * tier exceeds its budget, its programs go to Waiting in demotion order
 * (Acting before Reasoning, highest idleness first, ties highest id first).
 * (2) While the GPU tier exceeds its budget, the next program in demotion
 * order leaves it, to the CPU tier if it fits in the CPU room left, else to
 * Waiting; a Reasoning victim is demoted lazily: the caller lets its current
 * inference step finish (orders it before the swap-out on the swap-out
 * stream), and its pages are handed out only after that (see above).
 * (3) The GPU room left is filled from, in order: CPU programs waiting for
 * inference, returning Waiting programs waiting for inference, new arrivals
 * smallest context first; lowest idleness first within a level, ties lowest
 * id.  Programs moved by (1)-(2) and Acting programs are no candidates; the
 * walk stops at the first candidate that does not fit (MORI_F_SKIP_FIT:
 * skips it).  Waiting programs are never placed on the CPU tier.  plan.order
 * then lists programs by old tier -- GPU, CPU, then Waiting as returning,
 * new (by context size), Acting -- each group by (Reasoning before Acting,
 * idleness, id) or, for new arrivals, (context size, idleness, id); m_gpu and
 * m_cpu count the programs on each tier afterwards.  A new arrival must have
 * fewer than 2^31 blocks (MORI_DEV_BAD_TBL_OFF otherwise).
 *
 * MORI_F_SSD_TIER (Sec. 7.1, boundary policy only): tier 3 is valid and the
 * ranking gets a third run -- after the CPU tier's, the longest run within
 * ssd_bytes goes to the SSD tier (skip-fit: the first of GPU, CPU, SSD with
 * room).  An SSD program owns no page; its KV is the caller's, in storage.
 * A program leaving the GPU for the SSD tier is swapped out like one going to
 * the CPU tier (into a host buffer the caller then writes to storage), and one
 * coming back is swapped in from a host buffer the caller has filled; page
 * slots go to every swapped-in program (from CPU or SSD) in rank order.
 *
 * A new plan supersedes the last one.  It waits (on the stream) for the last
 * plan's swaps that were enqueued; swaps that were not are abandoned, and the
 * tables, tiers and free map stand as that plan wrote them -- programs it sent
 * off the GPU then have no copy of their KV (placement-only use).
 *
 * EINVAL: null pointers (status with MORI_F_STATUS_KEY or MORI_F_INCREMENTAL),
 * window_k out of range, unknown flags, MORI_F_SSD_TIER with
 * MORI_F_INCREMENTAL, gpu_bytes > num_blocks * block bytes.  ENOSPC: P above
 * the context's max_programs.  Both are raised before anything is enqueued. */
int mori_rank_partition(mori_ctx* ctx, const mori_programs* programs, const mori_budget* budget,
                        void* stream);

/* Blocks the host until the last plan is on the host and fills *out.
 * Returns MORI_EDEVICE (with out->device_error set) if the plan was rejected
 * on the device, ESTATE if there is no plan. */
int mori_plan_wait(mori_ctx* ctx, mori_plan* out);

/* Swap-out of the last plan: for every program p with category OUT, copies
 * each run (plane q, logical block i) from its old page to
 * host_dst[p] + (q * nblk_p + i) * run_bytes.  host_dst is a host array of P
 * addresses (read during the call; entries of other programs are ignored),
 * each 16-B aligned inside a registered range with room for nblk_p * block
 * bytes.  Pages released by these programs may be reused only after this
 * swap completes.  ESTATE: no plan, or swap-out already enqueued for it. */
int mori_kv_swap_out(mori_ctx* ctx, const uint64_t* host_dst, uint32_t mode, void* stream);

/* Swap-in of the last plan: for every program p with category IN, copies
 * host_src[p] + (q * nblk_p + i) * run_bytes into its newly allocated page of
 * block i, plane q.  Waits (on the stream) for the plan and, before writing a
 * page that is still in use (the swap-out of the same plan reads it, or a
 * dropped program's step ordered before that swap-out uses it), for that
 * swap-out (pages free before the step and pages of idle dropped programs
 * need no wait).  The host buffers may be reused after it completes.  ESTATE: no plan, swap-in already
 * enqueued, or swap-out of the plan not yet enqueued. */
int mori_kv_swap_in(mori_ctx* ctx, const uint64_t* host_src, uint32_t mode, void* stream);

/* ---- introspection ----------------------------------------------------- */
#define MORI_Q_LAST_HIP_ERROR 1 /* last hipError_t seen by the context */
#define MORI_Q_DEVICE_ERROR 2   /* device error word of the last plan and swaps (waits for them) */
#define MORI_Q_LAST_MODE 3      /* copy mode actually used by the last swap */
#define MORI_Q_PLAN_EVENT 4     /* hipEvent_t recorded when the plan is complete */
#define MORI_Q_OUT_EVENT 5      /* hipEvent_t recorded when the last swap-out is complete */
#define MORI_Q_IN_EVENT 6       /* hipEvent_t recorded when the last swap-in is complete */
int mori_query(mori_ctx* ctx, int what, uint64_t* value);

/* Static description of a return code. */
const char* mori_strerror(int code);

/* ---- typed eviction order (Sec. 4.3.2) -------------------------------------- */
/* The engine-side companion of the placement: every KV block carries the type
 * label of its program -- busy (GPU queue), idle (CPU queue), inactive
 * (Waiting) -- and its last access time.  A tier evicts by type first, in
 * tier-reversed order (GPU: inactive, idle, busy; CPU: inactive, busy, idle),
 * least recently used first within a type, so each tier keeps the programs
 * the placement assigned to it.  Equal type and time: lowest block id first. */
#define MORI_TYPE_BUSY 0u
#define MORI_TYPE_IDLE 1u
#define MORI_TYPE_INACTIVE 2u

typedef struct {
  uint32_t num_blocks;          /* N */
  const uint8_t* type;          /* device [N] MORI_TYPE_* */
  const uint64_t* last_access;  /* device [N] access times, larger = more recent, < 2^62 */
  const uint32_t* size;         /* device [N] block sizes in units of unit_bytes, or NULL: one unit each */
  uint64_t unit_bytes;
} mori_blocks;

/* Bytes of device workspace mori_evict_order needs for num_blocks blocks
 * (about 33 bytes per block, plus 1 MiB). */
int mori_evict_workspace(uint32_t num_blocks, uint64_t* bytes);

/* Eviction order of one tier (MORI_TIER_GPU or MORI_TIER_CPU), enqueued on
 * `stream`: order[j] (device [N]) = block evicted j-th; prefix[j] (device [N],
 * may be NULL) = bytes freed by the first j+1 evictions; result (device [2]) =
 * {fewest evictions that free at least need_bytes (N if all of them free
 * less, 0 when need_bytes is 0), MORI_DEV_* error bits}.  The time depends
 * little on how types and times lie over the block ids; only times made to miss
 * the blocks the call samples make it long (2^20 blocks: up to 9 ms).
 * workspace: device memory of at least mori_evict_workspace bytes, 256-B
 * aligned, owned by the caller and used only while the call's work runs.
 * Nothing is allocated.
 * EINVAL: null pointers, misaligned or short workspace, bad tier. */
int mori_evict_order(const mori_blocks* blocks, uint32_t tier, uint64_t need_bytes, void* workspace,
                     uint64_t workspace_bytes, uint32_t* order, uint64_t* prefix, uint32_t* result,
                     void* stream);

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, serving loops that forbid allocation): mori_evict_order with the
 * workspace in a device array the library holds on each GPU for the life of
 * the process, instead of a caller buffer.  Same result for the same input;
 * at most MORI_EVICT_NOALLOC_MAX_BLOCKS blocks (ENOSPC above; the array is
 * about 6.1 MiB per GPU).  Nothing is allocated: the array's device address
 * is looked up on the first call on each GPU (call it once before a capture
 * starts), and each call enqueues kernels only, which clear what must start
 * at zero.  Every call on one GPU uses the same array: calls whose work
 * overlaps on one GPU (other streams, other host threads) race and give
 * wrong results, so the caller serialises them, e.g. on one stream.
 * EINVAL: null pointers, bad tier; EHIP: the address lookup failed. */
#define MORI_EVICT_NOALLOC_MAX_BLOCKS 524288u /* 2^19 */
int mori_evict_order_noalloc(const mori_blocks* blocks, uint32_t tier, uint64_t need_bytes, uint32_t* order,
                             uint64_t* prefix, uint32_t* result, void* stream);

/* ---- tokens: writing and reading the pool's pages for a model ------------ */
/* The calls a model makes in every layer, on the pages of the GPU-resident
 * programs: mori_kv_append writes new tokens' keys and values into the pool,
 * mori_kv_attend lets their queries attend to everything the program holds.
 * Both read the same block tables that mori_rank_partition rewrites, in stream
 * order; neither needs a context, allocates or waits.
 *
 * A pool row (row_bytes, one token in one plane) is
 *   planes 2   plane 0: keys [kv_heads][head_dim], plane 1: values, the same
 *   planes 1   a compressed latent [head_dim] shared by all query heads: the
 *              latent part, which is key and value, then the rotated key part
 * of 16-bit floats.  Layer l has planes l * planes ... l * planes + planes - 1.
 * Token j of a program is row j % block_tokens of its block j / block_tokens. */
#define MORI_DT_F16 0u
#define MORI_DT_BF16 1u

/* A batch: new tokens of some programs, packed one program after the other.
 * Sequence b is tokens seq_off[b] .. seq_off[b+1]-1 of the batch, the last
 * n_b of the kv_len[b] tokens that its program holds after the append; token i
 * of them is at position kv_len[b] - n_b + i of the program.  A token whose
 * position is negative is padding (kv_len[b] < n_b): nothing is stored for it
 * and it attends to nothing.  num_tokens, max_new and max_kv are bounds that
 * the host vouches for (they size the launch): tokens before seq_off[0] or
 * past seq_off[num_seqs] are left alone.  A program appears once in a batch.
 * On the device: n_b above max_new, kv_len above max_kv or above the program's
 * blocks, a program id out of range: MORI_DEV_BAD_TOKENS, and the sequence counts
 * as all padding; offsets that decrease or pass num_tokens: the same bit, and
 * that sequence's tokens are left alone.
 * A block without a page: MORI_DEV_NOT_RESIDENT; a page id past the pool:
 * MORI_DEV_PAGE_RANGE; such a token is not stored, and what attends to it is
 * unspecified.  No call touches memory outside the pool and the arrays given. */
typedef struct {
  uint32_t num_seqs;        /* B, 1..MORI_MAX_PROGRAMS */
  uint32_t num_tokens;      /* T, rows of the token arrays */
  uint32_t max_new;         /* no n_b is larger; 1 for a decode step */
  uint32_t max_kv;          /* no kv_len is larger; < 2^31 */
  const uint32_t* seq_off;  /* device [B+1] */
  const uint32_t* kv_len;   /* device [B] */
  const uint32_t* program;  /* device [B], or NULL: sequence b is program b */
  uint32_t num_programs;    /* P */
  uint32_t tbl_len;         /* entries allocated in tbl */
  const uint32_t* tbl_off;  /* device [P+1], as in mori_programs */
  const uint32_t* tbl;      /* device [tbl_len] */
} mori_tokens;

/* Programs that take new tokens: their tables grow by pages of the free map, and
 * what the batch's calls need is made in the same go, all of it on the device.
 * Sequence b is new_tokens[b] new tokens of its program, behind the held[p] that it
 * holds.  Its program gets the pages that are missing for them: the lowest free ids,
 * in batch order, a sequence's blocks in their order.  Tables stay contiguous:
 * entries behind a program's move up.  tbl_len bounds the grown tables; entries past
 * them are left alone.  No page is ever given back (a plan does that).
 *
 * What was before (tbl_off, tbl, free_map, held) is read, what is after goes to
 * tbl_off_to, tbl_to, free_to and held_to: each the array itself (then a captured
 * graph of steps replays with programs that grow) or one that overlaps no other.
 * seq_off, kv_len, program and the grown tables are a mori_tokens' arrays.
 * slots[t] = page * block_tokens + row of token t, positions[t] its position; -1 for
 * places of the arrays past the batch's tokens.
 *
 * All or nothing: where something does not fit, the arrays after are those before,
 * the batch is empty (offsets and lengths 0, slots and positions -1) and error gets
 *   MORI_DEV_BAD_TOKENS    a program out of range or twice in the batch, held past the
 *                          program's blocks, new_tokens above max_new, a length above
 *                          max_kv, more than num_tokens tokens in all
 *   MORI_DEV_NOT_RESIDENT  a program whose tier is not MORI_TIER_GPU
 *   MORI_DEV_NOSPC         too few free pages or table entries
 *   MORI_DEV_BAD_TBL_OFF   offsets that do not start at 0, decrease or pass tbl_len;
 *                          tables and offsets after are then not written
 * An old block of a new token without a page (or with one past the pool) gives slot -1
 * and MORI_DEV_NOT_RESIDENT (MORI_DEV_PAGE_RANGE); the rest stands.
 *
 * A plan's swap-out may still be reading pages that the plan has marked free: grow once
 * it is enqueued, ordered behind MORI_Q_OUT_EVENT.  Swaps move what the plan placed, so a
 * program that is on its way in may grow. */
typedef struct {
  uint32_t num_seqs;          /* B, 1..MORI_MAX_PROGRAMS */
  uint32_t num_tokens;        /* T, places of slots and positions */
  uint32_t max_new, max_kv;   /* as in mori_tokens */
  const uint32_t* new_tokens; /* device [B] */
  const uint32_t* program;    /* device [B], or NULL: sequence b is program b */
  uint32_t num_programs;      /* P, 1..MORI_MAX_PROGRAMS */
  uint32_t tbl_len;           /* entries allocated in tbl and in tbl_to */
  const uint8_t* tier;        /* device [P], or NULL: every program is on the GPU */
  const uint32_t* tbl_off;    /* device [P+1] */
  const uint32_t* tbl;        /* device [tbl_len] */
  const uint8_t* free_map;    /* device [num_blocks], 16-B aligned: 0 = in use */
  const uint32_t* held;       /* device [P] tokens that each program holds */
  uint32_t* tbl_off_to;
  uint32_t* tbl_to;
  uint8_t* free_to;
  uint32_t* held_to;
  uint32_t* seq_off;          /* device [B+1] */
  uint32_t* kv_len;           /* device [B] */
  int64_t* slots;             /* device [T], or NULL */
  int32_t* positions;         /* device [T], or NULL */
} mori_growth;

/* Device workspace mori_tables_grow needs (more where tbl_to is tbl). */
int mori_tables_grow_workspace(const mori_pool* pool, const mori_growth* growth, uint64_t* bytes);

/* Enqueues the above; of the pool block_tokens (at most 2^18) and num_blocks are read.
 * workspace: 256-B aligned device memory of at least mori_tables_grow_workspace bytes, used only
 * while the call's work runs; its contents before do not matter.  *error (device, may
 * be NULL) collects MORI_DEV_* bits by OR; the caller clears it.  EINVAL: null pointers,
 * alignment, counts out of range, a short workspace. */
int mori_tables_grow(const mori_pool* pool, const mori_growth* growth, void* workspace, uint64_t workspace_bytes,
                     uint32_t* error, void* stream);

/* A [tokens][heads][elements] array of 16-bit floats on the device: element e
 * of head h of token t is at data + 2 * (t * token_stride + h * head_stride + e).
 * data is 16-B aligned and both strides are multiples of 8 elements. */
typedef struct {
  void* data;
  uint64_t token_stride, head_stride; /* in elements */
} mori_rows;

#define MORI_ROPE_HALF 0u  /* element i turns with i + rot_dim / 2 */
#define MORI_ROPE_PAIRS 1u /* element 2i turns with 2i + 1 */

/* What mori_kv_append stores.  The rotation by position p of the pair i:
 * (a, b) -> (a c - b s, b c + a s) with c = rope[p][i], s = rope[p][rot_dim/2 + i],
 * computed in 32 bits and rounded once.
 *   planes 2   k and v [T][kv_heads][head_dim]; the first rot_dim elements of
 *              every key head are rotated, the rest and the values are copied.
 *   planes 1   k [T][1][head_dim - rot_dim], the latent part, copied; v
 *              [T][1][rot_dim], the key part, rotated and stored behind it.
 *   q          optional (NULL data): the tokens' queries, [T][q_heads][head_dim]
 *              with planes 2, rotated like the keys; [T][q_heads][rot_dim] with
 *              planes 1, rotated whole.  Written to q_out (which may be q
 *              itself, with its strides); padding tokens get zeros. */
typedef struct {
  uint32_t dtype;      /* MORI_DT_* */
  uint32_t kv_heads;   /* 1 with planes 1 */
  uint32_t head_dim;   /* multiple of 16, <= 4096; kv_heads * head_dim * 2 == row_bytes */
  uint32_t q_heads;    /* <= 1024; read only with q */
  uint32_t rot_dim;    /* multiple of 16, <= head_dim (planes 1: 16..head_dim-16); 0: no rotation */
  uint32_t rope_style; /* MORI_ROPE_* */
  uint32_t rope_len;   /* positions in rope; a token past them: MORI_DEV_BAD_TOKENS, not stored */
  const float* rope;   /* device [rope_len][rot_dim], 16-B aligned: cosines, then sines */
  mori_rows k, v, q, q_out;
} mori_append;

/* Writes the batch's keys and values of one layer into the pool.  *error
 * (device, may be NULL) collects MORI_DEV_* bits by OR; the caller clears it.
 * EINVAL: null pointers, alignment, sizes that do not fit each other, 2^36
 * elements or more in a batch (queries, keys and values; a launch's threads). */
int mori_kv_append(const mori_pool* pool, uint32_t layer, const mori_tokens* tokens, const mori_append* append,
                   uint32_t* error, void* stream);

/* Positions with several axes (time, height and width of a patch in an image or a
 * video): the pair i of token t turns by rope[at[a][t]][i] with a the axis of i, in place
 * of the token's position in its program, which still says where it is stored.
 *   MORI_AXES_BLOCKS  the first sections[0] pairs have axis 0, the next sections[1]
 *                     axis 1 and so on
 *   MORI_AXES_TURNS   pair i has axis i % num_axes, if i / num_axes < sections of it,
 *                     else axis 0, whose section is the rest
 * A column of the table has its own frequency, so axes whose frequencies start anew are
 * a table made that way.  A position below 0 or past rope_len: MORI_DEV_BAD_TOKENS, the
 * token is not stored and its query is 0; padding's positions do not matter. */
#define MORI_MAX_AXES 4u
#define MORI_AXES_BLOCKS 0u
#define MORI_AXES_TURNS 1u
typedef struct {
  uint32_t num_axes;                /* 1..MORI_MAX_AXES */
  uint32_t order;                   /* MORI_AXES_* */
  uint32_t sections[MORI_MAX_AXES]; /* pairs of each axis: rot_dim / 2 together */
  const int32_t* at;                /* device [num_axes][axis_stride], a token an entry */
  uint64_t axis_stride;             /* >= num_tokens, where there is more than one axis */
} mori_axes;

/* mori_kv_append with such positions.  EINVAL: as there, no axes, sections that do not
 * give every axis its pairs, rot_dim 0. */
int mori_kv_append_axes(const mori_pool* pool, uint32_t layer, const mori_tokens* tokens, const mori_append* append,
                        const mori_axes* axes, uint32_t* error, void* stream);

/* What attends: out[t][h] = sum over the program's tokens j up to and with t's
 * own position of softmax_j(scale * q[t][h] . key_j) value_j, with head h
 * reading key head h / (q_heads / kv_heads); an empty sum is 0.
 *   planes 2   head_dim 64 or 128, value_dim the same
 *   planes 1   head_dim 576, value_dim 512 (the row's first 512 elements)
 * Scores, maxima, sums and outputs are kept in 32 bits; the weights are rounded
 * to dtype for the matrix product with the values.  fp16 weights keep all their
 * bits down to 2^-26 of the largest and are 0 below 2^-37 (bf16: where 32 bits end);
 * an infinite value under a weight that is 0 so gives NaN. */
typedef struct {
  uint32_t dtype;     /* MORI_DT_* */
  uint32_t q_heads;   /* multiple of kv_heads, <= 1024 */
  uint32_t kv_heads;  /* kv_heads * head_dim * 2 == row_bytes */
  uint32_t head_dim, value_dim;
  float scale;        /* finite */
  mori_rows q;        /* [T][q_heads][head_dim] */
  mori_rows out;      /* [T][q_heads][value_dim]; overlaps no input */
  float* lse;         /* device [T][q_heads] or NULL: log of the sum of exp(scores), -inf for an empty sum */
} mori_attend;

/* Device workspace mori_kv_attend needs for this batch (0: none; it grows with
 * num_tokens, num_seqs and the heads, and is bounded by max_new and max_kv). */
int mori_kv_attend_workspace(const mori_pool* pool, const mori_tokens* tokens, const mori_attend* attend,
                             uint64_t* bytes);

/* Attention of the batch's tokens in one layer, as above.  workspace: 256-B
 * aligned device memory of at least mori_kv_attend_workspace bytes, used only
 * while the call's work runs; its contents before do not matter.  The result is
 * the same for every call with the same arguments, bit for bit.  error as in
 * mori_kv_append.  EINVAL: null pointers, alignment, sizes or head dimensions
 * other than the above, a short workspace, a batch of more tokens than a launch has
 * threads for (num_tokens * q_heads below 2^27 always fits). */
int mori_kv_attend(const mori_pool* pool, uint32_t layer, const mori_tokens* tokens, const mori_attend* attend,
                   void* workspace, uint64_t workspace_bytes, uint32_t* error, void* stream);

/* What a call may say of scores and of what a token sees, K/V pools only:
 *   s = scale * q . key_j
 *   cap > 0:  s = cap * tanh(s / cap)
 *   slopes:   s = s - slopes[h] * |i - j|, i and j positions in the program
 * and token i of the program sees key j where
 *   max(first[t], i + 1 - window, 0) <= j < min(end[t], the program's length)
 * with end[t] = i + 1 unless it is given, so one may also see what is behind it.  Ranges
 * make documents that do not see each other (first: where a token's document starts),
 * prefixes that all of it see (end: the larger of the prefix's and the token's own) and
 * the like.  A token that sees nothing gets 0, lse -inf.  Pages of which no token of the
 * sequence sees a key need not be there. */
typedef struct {
  float cap;            /* 0: none; finite, not negative */
  uint32_t window;      /* positions up to and with the token's own; 0: all */
  const float* slopes;  /* device [q_heads] or NULL */
  const int32_t* first; /* device [T] or NULL */
  const int32_t* end;   /* device [T] or NULL */
} mori_sight;

/* mori_kv_attend and its workspace with that; EINVAL as there, and for a cap or
 * alignment that does not fit, no sight, or a latent pool.  A workspace for a sight
 * without a window serves all others of the batch. */
int mori_kv_attend_sight_workspace(const mori_pool* pool, const mori_tokens* tokens, const mori_attend* attend,
                                   const mori_sight* sight, uint64_t* bytes);
int mori_kv_attend_sight(const mori_pool* pool, uint32_t layer, const mori_tokens* tokens, const mori_attend* attend,
                         const mori_sight* sight, void* workspace, uint64_t workspace_bytes, uint32_t* error,
                         void* stream);

/* ---- kernel timing ------------------------------------------------------ */
/* With profiling on, every gather/scatter kernel launch of the swaps is
 * bracketed by timing events recorded on the stream it is launched on (up to
 * 4096 launches per direction between reads).  mori_profile_read waits for
 * those events and returns, for direction 0 (swap-out) or 1 (swap-in), the
 * number of launches, the payload bytes they moved and their summed duration
 * in milliseconds, then clears the record.  EINVAL: null pointers or a bad
 * direction; ENOSPC (from a swap) is never raised: launches beyond the record
 * capacity are simply not timed. */
int mori_profile(mori_ctx* ctx, int enable);
int mori_profile_read(mori_ctx* ctx, int direction, uint64_t* launches, uint64_t* payload_bytes,
                      double* kernel_ms);

/* ---- multi-replica admission (host) ----------------------------------- */
#define MORI_MAX_REPLICAS 1024u
#define MORI_ADMIT_BEST_FIT 1u /* least room that holds the program, instead of the most */

/* Admission of the Waiting queue that all replicas share (Sec. 4.1: a GPU and
 * a CPU queue per replica, one global Waiting queue; Sec. 4.3.1: Waiting
 * promotions are bin-packed across replicas in decreasing size onto the
 * replica with the most available capacity, while CPU-tier programs keep their
 * replica -- each replica's own mori_rank_partition promotes those).  Host
 * memory only; no GPU work.
 *   bytes[P], idleness[P], status[P]: the Waiting programs' KV bytes, Eq. 1
 *     idleness in [0, 1] and MORI_ST_* status.  Candidates are the Reasoning
 *     (returning) programs, then the new arrivals; Acting programs stay.
 *     Within a level: larger KV first, then lower idleness, then lower index.
 *   room[R]: free GPU bytes of each replica after its own plan.
 *   flags: 0 or MORI_ADMIT_BEST_FIT.
 *   replica[P] (out): the replica each program goes to, -1 if it stays
 *     waiting (it fits no replica when its turn comes; later ones are tried).
 *   room_after[R] (out; may be room itself): room less what was admitted.
 * Ties between replicas go to the lower index.  Each replica then admits its
 * programs as Waiting->GPU in its next plan (prefill rebuilds their KV).
 * EINVAL: num_replicas 0 or above MORI_MAX_REPLICAS, null arrays, unknown
 * flags, a status above 2 or idleness outside [0, 1]. */
int mori_replica_admit(uint32_t num_programs, const uint64_t* bytes, const float* idleness, const uint8_t* status,
                       uint32_t num_replicas, const uint64_t* room, uint32_t flags, int32_t* replica,
                       uint64_t* room_after);

#ifdef __cplusplus
}
#endif
#endif /* MORI_H */
