"""Cases of the operators around a step whose tokens the device counts: tables that
grow, positions with several axes, attention that does not see everything.

  grow    TokenGrowth: the block tables of programs that take new tokens grow by
          pages of the free map; the batch's offsets, lengths, slots and positions
          are made in the same call
  append  kv_append with positions of several axes (time, height, width) in place
          of the one that a token has in its program
  attend  kv_attend with capped scores, a bias by distance, a window, and ranges of
          keys that each token may see (documents, prefixes)

A case names a batch: ``seqs`` programs with about ``new`` new tokens each behind
about ``ctx`` cached ones (0: whole prompts), and ``decode`` further programs with
one new token.  Token counts, contexts and what tokens may see follow from the case
alone; values, page order and the programs' order follow from the seed.  ``own``
chooses between the plain form (elementary torch operations) and the framework's
calls.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

THETA = 500000.0
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
GPU, CPU = 0, 1  # tiers


def _grow(programs, seqs, new, ctx, block=16, room=64, name=None):
    """``seqs`` of ``programs`` programs take tokens; ``room``: the token arrays'
    length is a multiple of it (the bucket of a captured step)."""
    c = {"kind": "grow", "programs": programs, "seqs": seqs, "new": new, "ctx": ctx, "block": block, "room": room}
    return {"name": name, **c} if name else c


def _append(dtype, seqs, new, ctx, q_heads, kv_heads, dim, sections, order="blocks", style="half", block=16,
            name=None):
    """``sections``: pairs of each axis, as text; twice their sum is what is rotated."""
    c = {"kind": "append", "dtype": dtype, "seqs": seqs, "new": new, "ctx": ctx, "q_heads": q_heads,
         "kv_heads": kv_heads, "dim": dim, "sections": sections, "order": order, "style": style, "block": block,
         "decode": 0}
    return {"name": name, **c} if name else c


def _attend(dtype, seqs, new, ctx, q_heads, kv_heads, dim, block=16, decode=0, cap=0.0, bias=False, window=0,
            docs=0, prefix=0.0, name=None):
    """``docs``: mean length of the documents a program's tokens are cut into (0: one);
    ``prefix``: the share of the new tokens that all of them see."""
    c = {"kind": "attend", "dtype": dtype, "seqs": seqs, "new": new, "ctx": ctx, "q_heads": q_heads,
         "kv_heads": kv_heads, "dim": dim, "block": block, "decode": decode, "cap": cap, "bias": bias,
         "window": window, "docs": docs, "prefix": prefix}
    return {"name": name, **c} if name else c


def listed():
    return [
        # the tiny workload's eight agents take a token each: launch latency
        _grow(8, 8, 1, 700, room=8, name="grow_step_tiny"),
        # a decode step of the churn workload's programs, those that are resident and running
        _grow(1024, 400, 1, 4096, name="grow_step_churn"),
        # chunks and prompts of some of the Llama-3-8B workload's programs
        _grow(64, 24, 4096, 16384, name="grow_chunks_8b"),
        # the tiny workload's decode step, three axes: launch latency
        _append("fp16", 8, 1, 700, 8, 4, 64, "8,12,12", name="append_axes_step_tiny"),
        # agents that look at screenshots: image patches in prompt chunks of five programs
        _append("bf16", 5, 4096, 6000, 32, 8, 128, "16,24,24", name="append_axes_chunk_8b"),
        # the same with axes that take turns, on one rank at tensor parallelism 4, a few frames each
        _append("bf16", 16, 600, 2000, 16, 2, 128, "24,20,20", "turns", name="append_turns_chunk_tp4"),
        # the tiny workload's decode step with capped scores
        _attend("fp16", 8, 1, 700, 8, 4, 64, cap=50.0, name="step_capped_tiny"),
        # decode step of the Llama-3-8B workload's programs in a layer that sees the last 4096 tokens
        _attend("bf16", 64, 1, 16384, 32, 8, 128, window=4096, name="step_window_8b"),
        # one agent with a long context on one rank at tensor parallelism 8, distances in place of rotations
        _attend("bf16", 1, 1, 65501, 8, 1, 128, bias=True, name="step_bias_long_tp8"),
        # resumed agents send a tool's output, capped scores in a layer with a window
        _attend("bf16", 4, 512, 12000, 32, 8, 128, cap=50.0, window=4096, name="chunk_capped_window_8b"),
        # prompts packed out of documents that do not see each other
        _attend("bf16", 3, 8192, 0, 32, 8, 128, docs=1500, name="prompt_documents_8b"),
        # prompts whose first half is seen by all of their tokens, with a bias by distance
        _attend("bf16", 4, 4096, 0, 32, 8, 128, bias=True, prefix=0.5, name="prompt_prefix_bias_8b"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(8, 4, 64), (12, 4, 64), (16, 16, 64), (32, 8, 128), (64, 8, 128), (32, 4, 128), (16, 2, 128), (8, 1, 128),
         (10, 2, 128), (16, 16, 128)]
SECTIONS = {64: [("8,12,12", "blocks"), ("12,10,10", "turns"), ("16,16", "blocks"), ("16,16", "turns"), ("8,8", "blocks")],
            128: [("16,24,24", "blocks"), ("24,20,20", "turns"), ("32,32", "blocks"), ("16,16,16,16", "blocks"),
                  ("16,16,16,16", "turns"), ("64", "blocks"), ("8,12,12", "blocks")]}


def draw(rng):
    while True:
        kind = rng.choice(["grow"] * 2 + ["append"] * 2 + ["attend"] * 5)
        if kind == "grow":
            programs = _log_int(rng, 1, 4096)
            seqs = min(programs, _log_int(rng, 1, 4096))
            new = 1 if rng.random() < 0.4 else _log_int(rng, 2, 8192)
            case = _grow(programs, seqs, new, _log_int(rng, 16, 32768), rng.choice([16, 16, 32, 64]),
                         rng.choice([1, 8, 64, 256]))
            if programs * case["ctx"] > 1 << 23 or seqs * new > 1 << 17:
                continue
            return case
        q, kv, dim = rng.choice(HEADS)
        dtype, block = rng.choice(["bf16", "bf16", "fp16"]), rng.choice([16, 16, 32, 64])
        if kind == "append":
            sections, order = rng.choice(SECTIONS[dim])
            case = _append(dtype, _log_int(rng, 1, 64), _log_int(rng, 1, 4096), _log_int(rng, 16, 8192), q, kv, dim,
                           sections, order, rng.choice(["half", "pairs"]), block)
        else:
            shape = rng.choice(["step", "step", "few", "chunk", "prompt"])
            new = {"step": 1, "few": rng.randint(2, 16)}.get(shape) or _log_int(rng, 17, 8192)
            ctx = 0 if shape == "prompt" else _log_int(rng, 64, 65536)
            sight = rng.choice(["window", "window", "docs", "prefix", "none"])
            case = _attend(dtype, _log_int(rng, 1, 64), new, ctx, q, kv, dim, block,
                           rng.choice([0, 0, _log_int(rng, 1, 64)]) if new > 1 else 0,
                           rng.choice([0.0, 0.0, 20.0, 50.0]), rng.random() < 0.35,
                           _log_int(rng, 16, 16384) if sight == "window" else 0,
                           _log_int(rng, 16, 8192) if sight == "docs" else 0,
                           rng.choice([0.1, 0.35, 1.0]) if sight == "prefix" else 0.0)
            if not (case["cap"] or case["bias"] or case["window"] or case["docs"] or case["prefix"]):
                continue
        n, length = _lengths(case)
        w = work(case)
        pool = int(length.sum()) * _row(case) * 2
        pairs = sum(int(a) * int(b) for a, b in zip(n, length)) * case["q_heads"]  # scores that the plain form makes
        if w["flops"] > 4e11 or w["bytes"] > 2e9 or pool > (4e8 if kind == "append" else 4e9) or \
                (kind == "attend" and pairs > 6e9):
            continue
        return case


# --------------------------------------------------------------------------
# shapes
# --------------------------------------------------------------------------
def _rng_of(case, *more):
    return np.random.default_rng([case[k] for k in ("seqs", "new", "ctx", "block")] + list(more))


def _lengths(case):
    """New tokens of each program and its length in the pool with them."""
    rng = _rng_of(case, case["q_heads"], case["decode"])
    seqs, extra = case["seqs"], case["decode"]
    n = np.full(seqs, case["new"], np.int64)
    if case["new"] > 1:
        n = np.maximum(1, (case["new"] * np.exp(-0.7 * rng.random(seqs))).astype(np.int64))
        n[0] = case["new"]
    n = np.concatenate([n, np.ones(extra, np.int64)])
    base = case["ctx"] or (case["new"] if extra else 0)
    cached = np.full(n.size, base, np.int64)
    if n.size > 1:
        cached = np.clip(base * np.exp(0.5 * rng.standard_normal(n.size)), base // 4, 4 * base).astype(np.int64)
    if not case["ctx"]:
        cached[:seqs] = 0
    return n, cached + n


def _sight(case):
    """Keys that each token sees: from the first of these numbers up to the second (not
    with it); the window is not in them."""
    n, length = _lengths(case)
    rng = _rng_of(case, case["docs"])
    first, end = [], []
    for a, L in zip(n.tolist(), length.tolist()):
        pos = np.arange(L - a, L)
        lo, hi = np.zeros(a, np.int64), pos + 1
        if case["docs"]:
            cuts = np.cumsum(np.maximum(1, rng.exponential(case["docs"], 2 + 4 * L // case["docs"]).astype(np.int64)))
            starts = np.concatenate([[0], cuts])
            lo = starts[np.searchsorted(starts, pos, side="right") - 1]
        if case["prefix"]:
            hi = np.maximum(hi, L - a + int(case["prefix"] * a))
        first.append(lo)
        end.append(hi)
    return np.concatenate(first), np.concatenate(end)


def _seen(case):
    """The same with the window."""
    n, length = _lengths(case)
    lo, hi = _sight(case)
    if case["window"]:
        pos = np.concatenate([np.arange(L - a, L) for a, L in zip(n.tolist(), length.tolist())])
        lo = np.maximum(lo, pos + 1 - case["window"])
    return lo, np.maximum(lo, hi)


def _row(case):
    return 2 * case["kv_heads"] * case["dim"]


def _sections(case):
    return [int(x) for x in case["sections"].split(",")]


def _growth(case):
    """Tokens that every program holds, its blocks, which take new ones and how many."""
    rng = _rng_of(case, case["programs"])
    P, B, bt = case["programs"], case["seqs"], case["block"]
    ctx = case["ctx"]
    held = np.clip(ctx * np.exp(0.5 * rng.standard_normal(P)), 1, 4 * ctx).astype(np.int64)
    blocks = np.maximum(1, -(-held // bt))
    n = np.full(B, case["new"], np.int64)
    if case["new"] > 1:
        n = np.maximum(1, (case["new"] * np.exp(-0.7 * rng.random(B))).astype(np.int64))
    return held, blocks, n


def _rooms(case):
    """Places of the token arrays, of the table and of the pool."""
    held, blocks, n = _growth(case)
    entries = int(blocks.sum()) + int((n // case["block"] + 1).sum())
    return -(-int(n.sum()) // case["room"]) * case["room"], entries, entries + entries // 16 + 1


def work(case):
    if case["kind"] == "grow":
        held, blocks, n = _growth(case)
        P, B = case["programs"], case["seqs"]
        T, entries, pages = _rooms(case)
        grown = int(blocks.sum()) + int((n // case["block"]).sum())
        # tables, offsets, lengths and the free map in and out, programs and counts in; offsets, lengths,
        # slots and positions of the batch out
        return {"bytes": 4 * (int(blocks.sum()) + grown) + 17 * P + 2 * pages + 8 * B + 8 * B + 12 * T, "flops": 0}
    n, length = _lengths(case)
    T, q, kv, dim = int(n.sum()), case["q_heads"], case["kv_heads"], case["dim"]
    if case["kind"] == "append":
        axes, rot = len(_sections(case)), 2 * sum(_sections(case))
        return {"bytes": 2 * 2 * T * dim * (q + 2 * kv) + 4 * T * (rot + axes), "flops": 3 * T * (q + kv) * rot}
    lo, hi = _seen(case)
    off = np.concatenate([[0], np.cumsum(n)])
    read = sum(int(hi[a:b].max() - lo[a:b].min()) for a, b in zip(off[:-1].tolist(), off[1:].tolist()))
    given = 4 * T * (bool(case["docs"]) + bool(case["prefix"]))
    return {"bytes": read * 2 * _row(case) + 2 * T * q * 2 * dim + given, "flops": 4 * dim * q * int((hi - lo).sum())}


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
class Geometry:
    """Of the pool: one layer of a model's."""

    def __init__(self, block_tokens, row_bytes, num_blocks):
        self.layers, self.planes = 1, 2
        self.block_tokens, self.row_bytes, self.num_blocks = block_tokens, row_bytes, num_blocks


class State:
    pass


def _normal(gen, shape, dtype, scale=1.0):
    x = torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=gen)
    return x if scale == 1.0 else x.mul_(scale)


def _pages(rng, count):
    """Page ids of a used pool: chunks of mean 4 consecutive pages, shuffled."""
    cuts = np.cumsum(rng.geometric(0.25, size=count))
    cuts = np.concatenate([[0], cuts[cuts < count], [count]])
    order = rng.permutation(cuts.size - 1)
    return np.concatenate([np.arange(cuts[i], cuts[i + 1]) for i in order]).astype(np.int32)


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _axis_positions(rng, n, length, axes):
    """Positions of every axis: text, where they are alike, and grids of image patches
    (frames, rows, columns), after which text goes on behind the largest."""
    out = []
    for a, L in zip(n.tolist(), length.tolist()):
        at, base, parts = 0, L - a, []
        while at < a:
            text = int(rng.integers(1, 64))
            parts.append(np.repeat(base + np.arange(text)[None], axes, 0))
            base, at = base + text, at + text
            t, h, w = int(rng.integers(1, 4)), int(rng.integers(4, 24)), int(rng.integers(4, 24))
            grid = np.stack([x.ravel() for x in np.meshgrid(np.arange(t), np.arange(h), np.arange(w), indexing="ij")])
            parts.append(base + grid[[min(i, 2) for i in range(axes)]])
            base, at = base + max(t, h, w), at + grid.shape[1]
        out.append(np.concatenate(parts, 1)[:, :a])
    return np.concatenate(out, 1).astype(np.int32)


def prepare(case, seed):
    st = State()
    st.case = case
    rng = np.random.default_rng([seed, 0x6B77])
    if case["kind"] == "grow":
        _prepare_grow(st, rng)
        return st
    st.n, st.length = _lengths(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype, B, T = DTYPES[case["dtype"]], st.n.size, int(st.n.sum())
    q, kv, dim, bt = case["q_heads"], case["kv_heads"], case["dim"], case["block"]
    # tables: programs in another order than the batch, some blocks to grow into, free pages between
    blocks = -(-st.length // bt) + np.arange(B) % 3
    st.prog = rng.permutation(B).astype(np.int32)
    per_program = np.empty(B, np.int64)
    per_program[st.prog] = blocks
    st.tbl_off = np.concatenate([[0], np.cumsum(per_program)]).astype(np.int32)
    total = int(blocks.sum())
    st.pages = _pages(rng, total + total // 16 + 1)[:total]
    nb = total + total // 16 + 1
    st.geom = Geometry(bt, _row(case), nb)
    st.pool = _normal(gen, (2, nb, bt, kv, dim), dtype)
    st.seq_off = np.concatenate([[0], np.cumsum(st.n)]).astype(np.int32)
    st.d_tbl, st.d_tbl_off, st.d_prog = _dev(st.pages), _dev(st.tbl_off), _dev(st.prog)
    st.d_seq_off, st.d_length = _dev(st.seq_off), _dev(st.length.astype(np.int32))
    if case["kind"] == "append":
        rot, axes = 2 * sum(_sections(case)), len(_sections(case))
        st.at = _axis_positions(rng, st.n, st.length, axes)
        st.d_at = _dev(st.at)
        angle = torch.arange(int(st.at.max()) + 1, dtype=torch.float64)[:, None] * \
            THETA ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
        st.rope = torch.cat([angle.cos(), angle.sin()], 1).float().cuda()
        # the fused projection's output: queries, keys, values side by side
        x = _normal(gen, (T, q + 2 * kv, dim), dtype)
        st.q, st.k, st.v = x[:, :q], x[:, q:q + kv], x[:, q + kv:]
        st.q_out = torch.empty(T, q, dim, dtype=dtype, device="cuda")
    else:
        # scores that reach into the cap, or ordinary ones
        st.q = _normal(gen, (T, q, dim), dtype, 8.0 if case["cap"] else 2.5)
        st.out = torch.empty(T, q, dim, dtype=dtype, device="cuda")
        st.scale = dim ** -0.5
        lo, hi = _sight(case)
        st.first = _dev(lo.astype(np.int32)) if case["docs"] else None
        st.end = _dev(hi.astype(np.int32)) if case["prefix"] else None
        st.slopes = _dev(np.exp2(-8.0 * np.arange(1, q + 1) / q).astype(np.float32)) if case["bias"] else None
        st.lo, st.hi = _seen(case)
    if own:
        _plan(st)
    return st


def _prepare_grow(st, rng):
    """A pool in use: programs on the GPU, a few on the CPU tier (their tables hold no
    pages), the rest of the pages free; the batch takes some of those on the GPU."""
    case = st.case
    P, B, bt = case["programs"], case["seqs"], case["block"]
    held, blocks, n = _growth(case)
    runs = np.sort(rng.permutation(P)[:B])  # the same number of programs take tokens, others each time
    held, blocks = held.copy(), blocks.copy()
    order = rng.permutation(P)
    held, blocks = held[order], blocks[order]
    tier = np.where(rng.random(P) < 0.8, GPU, CPU).astype(np.uint8)
    tier[runs] = GPU
    prog = rng.permutation(runs).astype(np.int32)
    total, here = int(blocks.sum()), int(blocks[tier == GPU].sum())
    st.T, entries, pages = _rooms(case)
    ids = _pages(rng, pages)
    tbl = np.full(entries, -1, np.int32)
    tbl[:total][np.repeat(tier, blocks) == GPU] = ids[:here]
    free = np.zeros(pages, np.uint8)
    free[ids[here:]] = 1
    st.geom = Geometry(bt, 256, pages)
    st.host = dict(tbl_off=np.concatenate([[0], np.cumsum(blocks)]).astype(np.int32), tbl=tbl, free=free,
                   held=held.astype(np.int32), tier=tier, prog=prog, new=n.astype(np.int32))
    for name, a in st.host.items():
        setattr(st, name, _dev(a))
    st.max_new, st.max_kv = int(n.max()), int((held[prog] + n).max())
    st.o_off, st.o_tbl = torch.empty_like(st.tbl_off), torch.full_like(st.tbl, -1)
    st.o_free, st.o_held = torch.empty_like(st.free), torch.empty_like(st.held)
    if own:
        from paper_2606_00866_amd import attention as A

        st.growth = A.TokenGrowth(st.geom, st.tbl_off, st.tbl, st.free, st.held, st.new, st.prog, tier=st.tier,
                                  num_tokens=st.T, max_new=st.max_new, max_kv=st.max_kv,
                                  into=(st.o_off, st.o_tbl, st.o_free, st.o_held))


def _plan(st):
    from paper_2606_00866_amd import attention as A

    st.batch = A.TokenBatch(st.geom, st.d_tbl_off, st.d_tbl, st.d_seq_off, st.d_length, program=st.d_prog,
                            num_tokens=int(st.n.sum()), max_new=int(st.n.max()), max_kv=int(st.length.max()))
    if st.case["kind"] == "attend":
        st.workspace = A.kv_attend_workspace(st.geom, st.batch, st.q, sight=True)


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------
def run(state):
    st, case = state, state.case
    if not own:
        return {"grow": _plain_grow, "append": _plain_append, "attend": _plain_attend}[case["kind"]](st)
    from paper_2606_00866_amd import attention as A

    if case["kind"] == "grow":
        b = st.growth.run()
        return {"tbl_off": st.o_off, "tbl": st.o_tbl, "free": st.o_free, "held": st.o_held, "seq_off": b.seq_off,
                "kv_len": b.kv_len, "slots": st.growth.slots, "positions": st.growth.positions}
    if case["kind"] == "append":
        A.kv_append(st.pool, st.geom, 0, st.batch, st.k, st.v, q=st.q, q_out=st.q_out, rope=st.rope,
                    style=case["style"], positions=st.d_at, sections=_sections(case), order=case["order"])
        return {"pool": st.pool, "q": st.q_out}
    A.kv_attend(st.pool, st.geom, 0, st.batch, st.q, scale=st.scale, out=st.out, workspace=st.workspace,
                cap=case["cap"] or None, slopes=st.slopes, window=case["window"] or None, first=st.first, end=st.end)
    return st.out


def _plain_grow(st):
    bt, P, B, T = st.case["block"], st.held.numel(), st.new.numel(), st.T
    prog, n = st.prog.long(), st.new.long()
    blocks = (st.tbl_off[1:] - st.tbl_off[:-1]).long()
    after = st.held.long()
    kv_len = after[prog] + n
    after[prog] = kv_len
    more = ((kv_len + bt - 1) // bt - blocks[prog]).clamp_min(0)  # pages of each sequence
    ahead = torch.cumsum(more, 0) - more
    grown = blocks.clone()
    grown[prog] = blocks[prog] + more
    zero = torch.zeros(1, dtype=torch.long, device="cuda")
    off = torch.cat([zero, torch.cumsum(grown, 0)])
    # the r-th free page, lowest ids first
    free = st.free.long()
    rank = torch.cumsum(free, 0) - 1
    N = free.numel()
    of_rank = torch.zeros(N + 1, dtype=torch.long, device="cuda")
    of_rank[torch.where(free > 0, rank, N)] = torch.arange(N, device="cuda")
    taken = (free > 0) & (rank < more.sum())
    ahead_of = torch.zeros(P, dtype=torch.long, device="cuda")
    ahead_of[prog] = ahead
    # table entries: what was there, then the pages taken
    e = torch.arange(st.tbl.numel(), device="cuda")
    p = torch.searchsorted(off[1:], e, right=True).clamp_max(P - 1)
    j = e - off[p]
    old = st.tbl[(st.tbl_off[p] + torch.minimum(j, blocks[p] - 1)).long().clamp(0, st.tbl.numel() - 1)].long()
    page = torch.where(j < blocks[p], old, of_rank[(ahead_of[p] + j - blocks[p]).clamp(0, N)])
    st.o_tbl.copy_(torch.where(e < off[P], page, st.o_tbl.long()))
    st.o_off.copy_(off)
    st.o_free.copy_((free > 0) & ~taken)
    st.o_held.copy_(after)
    seq_off = torch.cat([zero, torch.cumsum(n, 0)])
    t = torch.arange(T, device="cuda")
    b = torch.searchsorted(seq_off[1:], t, right=True).clamp_max(B - 1)
    pos = kv_len[b] - n[b] + t - seq_off[b]
    there = t < seq_off[B]
    at = off[prog[b]] + pos // bt
    slot = st.o_tbl[torch.where(there, at, 0)].long() * bt + pos % bt
    return {"tbl_off": st.o_off, "tbl": st.o_tbl, "free": st.o_free, "held": st.o_held, "seq_off": seq_off.int(),
            "kv_len": kv_len.int(), "slots": torch.where(there, slot, -1), "positions": torch.where(there, pos, -1).int()}


def _slots(st):
    """Page and row of every new token."""
    bt = st.case["block"]
    n = st.d_seq_off[1:] - st.d_seq_off[:-1]
    T = int(st.n.sum())
    seq = torch.repeat_interleave(torch.arange(st.n.size, device="cuda"), n.long(), output_size=T)
    pos = (st.d_length - n)[seq] + torch.arange(T, device="cuda") - st.d_seq_off[seq]
    page = st.d_tbl[(st.d_tbl_off[st.d_prog.long()][seq] + pos // bt).long()]
    return page.long(), (pos % bt).long()


def _axis_of(case):
    """The axis of every pair: one section after the other, or in turns until an axis has
    its pairs, where the first one takes the rest."""
    s = _sections(case)
    if case["order"] == "blocks":
        return [a for a, m in enumerate(s) for _ in range(m)]
    return [i % len(s) if i // len(s) < s[i % len(s)] else 0 for i in range(sum(s))]


def _rotate(x, cos, sin, style):
    """x [T][H][D] in 32 bits, the first elements turned by cos, sin [T][pairs]."""
    m = cos.shape[1]
    c, s = cos[:, None], sin[:, None]
    if style == "half":
        a, b = x[..., :m], x[..., m:2 * m]
        return torch.cat([a * c - b * s, b * c + a * s, x[..., 2 * m:]], -1)
    a, b = x[..., 0:2 * m:2], x[..., 1:2 * m:2]
    return torch.cat([torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2), x[..., 2 * m:]], -1)


def _plain_append(st):
    page, row = _slots(st)
    axis = torch.tensor(_axis_of(st.case), device="cuda")
    pair = torch.arange(axis.numel(), device="cuda")
    at = st.d_at.long()[axis].t()  # [T][pairs]
    cos, sin = st.rope[at, pair], st.rope[at, pair + axis.numel()]
    st.q_out.copy_(_rotate(st.q.float(), cos, sin, st.case["style"]))
    st.pool[0, page, row] = _rotate(st.k.float(), cos, sin, st.case["style"]).to(st.k.dtype)
    st.pool[1, page, row] = st.v
    return {"pool": st.pool, "q": st.q_out}


def _plain_attend(st):
    case = st.case
    H, kv, bt = case["q_heads"], case["kv_heads"], case["block"]
    G = H // kv
    for b in range(st.n.size):
        n, L, p = int(st.n[b]), int(st.length[b]), int(st.prog[b])
        t0, off = int(st.seq_off[b]), int(st.tbl_off[p])
        start, stop = int(st.lo[t0:t0 + n].min()), int(st.hi[t0:t0 + n].max())  # what the sequence's tokens see
        count = stop - start
        pages = st.d_tbl[off + start // bt:off + -(-stop // bt)].long()
        skip = start - start // bt * bt
        rows = [st.pool[i, pages].flatten(0, 1)[skip:skip + count].float().transpose(0, 1) for i in range(2)]
        keys, values = rows[0].transpose(1, 2).contiguous(), rows[1].contiguous()  # [kv][dim][keys], [kv][keys][dim]
        at = torch.arange(start, stop, device="cuda")
        pos = torch.arange(L - n, L, device="cuda")
        low = torch.zeros_like(pos) if st.first is None else st.first[t0:t0 + n]
        if case["window"]:
            low = torch.maximum(low, pos + 1 - case["window"])
        high = pos + 1 if st.end is None else st.end[t0:t0 + n]
        step = max(1, (1 << 28) // (H * count))
        for i in range(0, n, step):
            m = min(step, n - i)
            q = st.q[t0 + i:t0 + i + m].float().unflatten(1, (kv, G)).transpose(0, 1).flatten(1, 2)  # [kv][m * G][dim]
            s = torch.bmm(q.contiguous(), keys).mul_(st.scale)
            if case["cap"]:
                s = s.div_(case["cap"]).tanh_().mul_(case["cap"])
            s = s.unflatten(1, (m, G))  # [kv][m][G][keys]
            if case["bias"]:
                far = (pos[i:i + m, None] - at[None, :]).abs().float()
                s -= st.slopes.view(kv, 1, G, 1) * far[None, :, None, :]
            hidden = (at[None, :] < low[i:i + m, None]) | (at[None, :] >= high[i:i + m, None])
            s = s.masked_fill_(hidden[None, :, None, :], -math.inf).flatten(1, 2)
            s.sub_(s.amax(-1, keepdim=True).clamp_min(-1e30)).exp_()
            total = s.sum(-1, keepdim=True)
            o = torch.bmm(s, values) / torch.where(total > 0, total, 1)
            st.out[t0 + i:t0 + i + m] = o.unflatten(1, (m, G)).transpose(0, 1).flatten(1, 2).to(st.out.dtype)
        del keys, values, rows
    return st.out


# --------------------------------------------------------------------------
# the definition, in whole numbers and in 64 bits
# --------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    return {"grow": _exact_grow, "append": _exact_append, "attend": _exact_attend}[case["kind"]](st)


def _exact_grow(st):
    """Program by program, on the host."""
    h, bt = st.host, st.case["block"]
    off = h["tbl_off"].astype(np.int64)
    tables = [h["tbl"][off[p]:off[p + 1]].tolist() for p in range(off.size - 1)]
    held, free = h["held"].astype(np.int64), h["free"].copy()
    pages = iter(np.flatnonzero(free).tolist())
    slots, positions, kv_len = np.full(st.T, -1, np.int64), np.full(st.T, -1, np.int64), []
    t = 0
    for p, n in zip(h["prog"].tolist(), h["new"].tolist()):
        while len(tables[p]) * bt < held[p] + n:
            tables[p].append(next(pages))
            free[tables[p][-1]] = 0
        pos = np.arange(held[p], held[p] + n)
        slots[t:t + n] = np.array(tables[p], np.int64)[pos // bt] * bt + pos % bt
        positions[t:t + n] = pos
        t += n
        held[p] += n
        kv_len.append(int(held[p]))
    tbl = np.full(h["tbl"].size, -1, np.int64)
    flat = [x for table in tables for x in table]
    tbl[:len(flat)] = flat
    return {"tbl_off": np.concatenate([[0], np.cumsum([len(x) for x in tables])]), "tbl": tbl, "free": free,
            "held": held, "seq_off": np.concatenate([[0], np.cumsum(h["new"], dtype=np.int64)]),
            "kv_len": np.array(kv_len), "slots": slots, "positions": positions}


def _exact_append(st):
    """Token by token of the batch's numbering, the rotation as a product of complex numbers."""
    case = st.case
    T, bt, s = int(st.n.sum()), case["block"], _sections(case)
    m = sum(s)
    seq = np.repeat(np.arange(st.n.size), st.n)
    pos = st.length[seq] - st.n[seq] + np.arange(T) - st.seq_off[seq]
    at = _dev(st.pages[st.tbl_off[st.prog[seq]] + pos // bt].astype(np.int64))
    row = _dev(pos % bt)
    turn = torch.empty(T, m, dtype=torch.complex128, device="cuda")
    start = np.concatenate([[0], np.cumsum(s)])
    for i in range(m):
        if case["order"] == "blocks":
            axis = int(np.searchsorted(start, i, side="right")) - 1
        else:
            turns, axis = divmod(i, len(s))
            axis = axis if turns < s[axis] else 0
        z = st.rope[_dev(st.at[axis].astype(np.int64))].double()
        turn[:, i] = torch.complex(z[:, i], z[:, m + i])
    turn = turn[:, None]

    def rotated(x):
        x, rest = x[..., :2 * m].double(), x[..., 2 * m:].double()
        if case["style"] == "half":
            z = torch.complex(x[..., :m].contiguous(), x[..., m:].contiguous()) * turn
            return torch.cat([z.real, z.imag, rest], -1)
        z = torch.view_as_complex(x.contiguous().unflatten(-1, (m, 2))) * turn
        return torch.cat([torch.view_as_real(z).flatten(-2), rest], -1)

    pool = st.pool.double()
    pool[0, at, row] = rotated(st.k)
    pool[1, at, row] = st.v.double()
    return {"pool": pool, "q": rotated(st.q)}


def _exact_attend(st):
    """Head by head: the logarithm of each row's sum, then the weighted values."""
    case = st.case
    H, G = case["q_heads"], case["q_heads"] // case["kv_heads"]
    if sum(int(a) * int(b) for a, b in zip(st.n, st.length)) * H * case["dim"] * 4 > 4e12:
        return None
    out = torch.empty(st.out.shape, dtype=torch.float64, device="cuda")
    low, high = _dev(st.lo), _dev(st.hi)
    for b in range(st.n.size):
        n, L, p = int(st.n[b]), int(st.length[b]), int(st.prog[b])
        t0 = int(st.seq_off[b])
        j = np.arange(int(st.lo[t0:t0 + n].min()), int(st.hi[t0:t0 + n].max()))
        page = _dev(st.pages[st.tbl_off[p] + j // case["block"]].astype(np.int64))
        row = _dev(j % case["block"])
        at = _dev(j)
        shared = range(0, H, G) if n * G <= 4096 else range(H)  # heads of a group together, or one by one
        for h in shared:
            g = G if len(shared) < H else 1
            k, v = (st.pool[i, page, row, h // G].double() for i in range(2))
            part = max(1, (1 << 27) // (g * j.size))
            for i in range(0, n, part):
                m = min(part, n - i)
                t = slice(t0 + i, t0 + i + m)
                s = (st.q[t, h:h + g].double().flatten(0, 1) @ k.t() * st.scale).unflatten(0, (m, g))
                if case["cap"]:
                    s = case["cap"] * torch.tanh(s / case["cap"])
                if case["bias"]:
                    pos = torch.arange(L - n + i, L - n + i + m, device="cuda").double()
                    s = s - st.slopes[h:h + g].double()[None, :, None] * (pos[:, None, None] - at).abs()
                seen = (at >= low[t, None]) & (at < high[t, None])
                s = torch.where(seen[:, None], s, -math.inf)
                lse = torch.logsumexp(s, -1, keepdim=True)
                w = torch.where(torch.isfinite(lse), torch.exp(s - lse.nan_to_num(neginf=0.0)), 0)
                out[t, h:h + g] = (w.flatten(0, 1) @ v).unflatten(0, (m, g))
    return out
