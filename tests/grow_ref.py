"""Plain definition of tables that grow (numpy, program by program), and instances for
its tests: used pools with programs on and off the GPU."""
from __future__ import annotations

from dataclasses import dataclass, field

import numpy as np

NONE = -1


@dataclass
class Geom:
    block_tokens: int
    num_blocks: int
    layers: int = 1
    planes: int = 2
    row_bytes: int = 256


@dataclass
class State:
    geom: Geom
    tbl_off: np.ndarray
    tbl: np.ndarray       # with room behind the last entry
    free: np.ndarray
    held: np.ndarray
    tier: np.ndarray
    prog: np.ndarray
    new: np.ndarray
    T: int
    extra: dict = field(default_factory=dict)

    @property
    def max_new(self):
        return max(1, int(self.new.max(initial=1)))

    @property
    def max_kv(self):
        return int((self.held[self.prog] + self.new).max(initial=1))


def instance(seed, programs, seqs, new, *, bt=16, held=60, spare_blocks=2, spare_pages=40, room=7, off_gpu=0.2, pad=5,
             free_first=False):
    """`new`: a number, or (lo, hi).  A program holds up to `held` tokens in as many blocks
    as they need and up to `spare_blocks` more."""
    rng = np.random.default_rng(seed)
    h = rng.integers(0, held + 1, programs)
    blocks = -(-h // bt) + rng.integers(0, spare_blocks + 1, programs)
    tier = (rng.random(programs) < off_gpu).astype(np.uint8)
    prog = rng.permutation(programs)[:seqs]
    tier[prog] = 0
    n = np.full(seqs, new) if np.isscalar(new) else rng.integers(new[0], new[1] + 1, seqs)
    off = np.concatenate([[0], np.cumsum(blocks)])
    grown = int(np.maximum(0, -(-(h[prog] + n) // bt) - blocks[prog]).sum())
    here = np.repeat(tier, blocks) == 0
    pages = int(here.sum()) + grown + spare_pages
    ids = np.arange(pages) if free_first else rng.permutation(pages)
    if free_first:
        ids = ids[::-1]
    tbl = np.full(int(off[-1]) + grown + room, NONE, np.int64)
    tbl[:off[-1]][here] = ids[:int(here.sum())]
    free = np.zeros(pages, np.uint8)
    free[ids[int(here.sum()):]] = 1
    return State(Geom(bt, pages), off, tbl, free, h, tier, prog, n, int(n.sum()) + pad, {"grown": grown})


def grow(s):
    """What the arrays are afterwards; None where there are too few pages or entries."""
    bt = s.geom.block_tokens
    tables = [s.tbl[s.tbl_off[p]:s.tbl_off[p + 1]].tolist() for p in range(s.held.size)]
    free, held = s.free.copy(), s.held.copy()
    slots, positions, kv_len, t = np.full(s.T, -1, np.int64), np.full(s.T, -1, np.int64), [], 0
    pages = np.flatnonzero(free).tolist()[::-1]
    for p, n in zip(s.prog.tolist(), s.new.tolist()):
        while len(tables[p]) * bt < held[p] + n:
            if not pages:
                return None
            free[pages[-1]] = 0
            tables[p].append(pages.pop())
        for pos in range(held[p], held[p] + n):
            slots[t], positions[t] = tables[p][pos // bt] * bt + pos % bt, pos
            t += 1
        held[p] += n
        kv_len.append(held[p])
    flat = [x for table in tables for x in table]
    if len(flat) > s.tbl.size:
        return None
    tbl = s.tbl.copy()
    tbl[:len(flat)] = flat
    return dict(tbl_off=np.concatenate([[0], np.cumsum([len(x) for x in tables])]), tbl=tbl, free=free, held=held,
                seq_off=np.concatenate([[0], np.cumsum(s.new)]), kv_len=np.array(kv_len), slots=slots,
                positions=positions)


def refused(s):
    """What a call that does not fit leaves."""
    B = s.prog.size
    return dict(tbl_off=s.tbl_off, tbl=s.tbl, free=s.free, held=s.held, seq_off=np.zeros(B + 1, int),
                kv_len=np.zeros(B, int), slots=np.full(s.T, -1), positions=np.full(s.T, -1))
