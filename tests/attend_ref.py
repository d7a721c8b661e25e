"""Plain 64-bit definitions of the token operators (numpy, one token at a time),
and instances for their tests: pools whose free pages, unused rows and other
layers hold NaN, so that anything read from them shows."""
from __future__ import annotations

from dataclasses import dataclass

import numpy as np
import torch

NONE = 0xFFFFFFFF
# half a unit in the last place, relative: 11 and 8 significant bits
ROUND = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -126}  # below the smallest normal number: absolute


@dataclass
class Geom:
    layers: int
    planes: int
    block_tokens: int
    row_bytes: int
    num_blocks: int


@dataclass
class Inst:
    geom: Geom
    dtype: torch.dtype
    kv: int
    dim: int
    n: np.ndarray         # new tokens per sequence
    length: np.ndarray    # tokens held with them
    prog: np.ndarray
    tbl_off: np.ndarray   # int64
    tbl: np.ndarray       # int64 page ids
    seq_off: np.ndarray
    pool: torch.Tensor    # [layers][planes][blocks][bt][kv][dim], host
    layer: int

    def slot(self, b, pos):
        e = self.tbl_off[self.prog[b]] + pos // self.geom.block_tokens
        return int(self.tbl[e]), int(pos % self.geom.block_tokens)

    def rows(self, plane, b, count):
        """float64 [count][kv][dim]: the first tokens of sequence b's program in one plane."""
        j = np.arange(count)
        pages = self.tbl[self.tbl_off[self.prog[b]] + j // self.geom.block_tokens]
        return self.pool[self.layer, plane, torch.from_numpy(pages), torch.from_numpy(j % self.geom.block_tokens)].double().numpy()


def instance(seed, n, length, *, kv, dim, dtype=torch.bfloat16, bt=16, planes=2, layers=2, layer=1, spare=1, extra=3,
             value_scale=1.0):
    """Sequences of n[b] new tokens, length[b] held, in programs of a shuffled
    order, each with `spare` more blocks than it needs."""
    rng = np.random.default_rng(seed)
    n, length = np.asarray(n, np.int64), np.asarray(length, np.int64)
    B = n.size
    prog = rng.permutation(B).astype(np.int64)
    blocks = np.zeros(B, np.int64)
    blocks[prog] = -(-length // bt) + spare
    tbl_off = np.concatenate([[0], np.cumsum(blocks)])
    nb = int(tbl_off[-1]) + extra
    tbl = rng.permutation(nb)[:int(tbl_off[-1])].astype(np.int64)
    pool = torch.full((layers, planes, nb, bt, kv, dim), float("nan"), dtype=dtype)
    inst = Inst(Geom(layers, planes, bt, kv * dim * 2, nb), dtype, kv, dim, n, length, prog, tbl_off, tbl,
                np.concatenate([[0], np.cumsum(n)]), pool, layer)
    for b in range(B):
        for q in range(planes):
            j = np.arange(int(length[b]))
            pages = tbl[tbl_off[prog[b]] + j // bt]
            x = rng.standard_normal((j.size, kv, dim)) * (value_scale if q else 1.0)
            pool[layer, q, torch.from_numpy(pages), torch.from_numpy(j % bt)] = torch.from_numpy(x).to(dtype)
    return inst


def dev32(a):
    return torch.from_numpy(np.ascontiguousarray(a).astype(np.uint32).view(np.int32).copy()).cuda()


def batch(inst, max_new=None, max_kv=None, tokens=None):
    from paper_2606_00866_amd import attention as A
    return A.TokenBatch(inst.geom, dev32(inst.tbl_off), dev32(inst.tbl), dev32(inst.seq_off), dev32(inst.length),
                        dev32(inst.prog), num_tokens=int(inst.n.sum()) if tokens is None else tokens,
                        max_new=int(inst.n.max(initial=0)) if max_new is None else max_new,
                        max_kv=max(1, int(inst.length.max(initial=1))) if max_kv is None else max_kv)


def attend(inst, q, scale, value_dim):
    """out, lse and the weighted mean of |v| (what the bound is made of), the
    largest score's error bound and the largest |v|: float64."""
    T, H = q.shape[:2]
    G = H // inst.kv
    q = q.double().numpy()
    out, lse = np.zeros((T, H, value_dim)), np.full((T, H), -np.inf)
    mean, delta, count = np.zeros((T, H, value_dim)), np.zeros((T, H, 1)), np.zeros((T, H, 1))
    top = np.zeros((T, H, 1))
    for b in range(inst.n.size):
        n, L = int(inst.n[b]), int(inst.length[b])
        k = inst.rows(0, b, L)
        v = k[..., :value_dim] if inst.geom.planes == 1 else inst.rows(1, b, L)
        for i in range(n):
            t, m = int(inst.seq_off[b]) + i, L - n + i + 1
            if m <= 0:
                continue
            for h in range(H):
                kk, vv = k[:m, h // G], v[:m, h // G]
                s = kk @ q[t, h] * scale
                top_s = s.max()
                w = np.exp(s - top_s)
                lse[t, h] = top_s + np.log(w.sum())
                w /= w.sum()
                out[t, h] = w @ vv
                mean[t, h] = w @ np.abs(vv)
                # products of 16-bit floats are exact in 32 bits; their sum of dim terms is off by at most
                # dim ulps of the sum of magnitudes, the scaling by another three
                delta[t, h] = (q.shape[2] + 3) * 2.0 ** -23 * (np.abs(kk) @ np.abs(q[t, h])).max() * abs(scale)
                count[t, h], top[t, h] = m, np.abs(vv).max()
    return out, lse, mean, delta, count, top


def attend_bound(dtype, out, mean, delta, count, top):
    """What the formula's evaluation may be off by: every weight by its rounding to
    dtype and by the error of its score (in the weight and in the sum), the 32-bit
    sums by 2^-16, weights below dtype's normal numbers by its smallest step, the
    result by its rounding."""
    weights = ROUND[dtype] * 1.01 + 2 * np.expm1(2 * delta) + 2.0 ** -16
    return weights * mean + ROUND[dtype] * (np.abs(out) + weights * mean) + (TINY[dtype] * count) * top + TINY[dtype]


def rotated(x, table, style):
    """x float64 [..., D], table float64 [r]: cosines, then sines."""
    r = table.size
    y = x.copy()
    c, s = table[:r // 2], table[r // 2:]
    for i in range(r // 2):
        a, b = (i, i + r // 2) if style == "half" else (2 * i, 2 * i + 1)
        y[..., a] = x[..., a] * c[i] - x[..., b] * s[i]
        y[..., b] = x[..., b] * c[i] + x[..., a] * s[i]
    return y
