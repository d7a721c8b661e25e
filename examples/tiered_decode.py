"""A model's side of the tiering: agents whose KV cache moves between HBM and host
memory keep decoding as if it had not.

Eight programs of the tiny workload run a toy decoder (random projections, two
layers) on a pool that holds only some of them.  Every rebalance is one
``TierPool.step``: programs that enter the GPU for the first time are prefilled,
those that come back go on where they were.  The same tokens also run on a second
pool in which every program is always resident; since nothing else differs, all
outputs have to be equal, bit for bit.

    python examples/tiered_decode.py
"""
from __future__ import annotations

import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np
import torch

from paper_2606_00866_amd import mori as M
from paper_2606_00866_amd.attention import TokenBatch, kv_append, kv_attend, rope_table
from paper_2606_00866_amd.tiering import TierPool
from workload import TINY, Geometry, budget_bytes, make_instance

HEADS, KV, DIM = 8, 4, 64
GROWTH = 12  # tokens a program decodes at most


class Decoder:
    """x -> x + attention(x) W_o, layer by layer, over one pool."""

    def __init__(self, tier_pool, layers, positions, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: (torch.randn(*s, device="cuda", generator=g) * s[0] ** -0.5).half()
        self.tp = tier_pool
        self.qkv = [rnd(HEADS * DIM, (HEADS + 2 * KV) * DIM) for _ in range(layers)]
        self.o = [rnd(HEADS * DIM, HEADS * DIM) for _ in range(layers)]
        self.rope = rope_table(positions, DIM)

    def __call__(self, x, batch):
        """x [T][HEADS * DIM] of the batch's tokens."""
        tp = self.tp
        for layer, (w, o) in enumerate(zip(self.qkv, self.o)):
            y = (x @ w).view(len(x), HEADS + 2 * KV, DIM)
            q, k, v = y[:, :HEADS], y[:, HEADS:HEADS + KV], y[:, HEADS + KV:]
            kv_append(tp.pool, tp.geom, layer, batch, k, v, q=q, q_out=q, rope=self.rope)
            x = x + kv_attend(tp.pool, tp.geom, layer, batch, q).flatten(1) @ o
        return torch.nn.functional.layer_norm(x.float(), x.shape[1:]).half()


def empty_pool(geom, nblk, num_blocks, resident):
    """A TierPool without content: every program on the GPU, or every one waiting."""
    off = np.concatenate([[0], np.cumsum(nblk)]).astype(np.uint32)
    total = int(off[-1])
    tbl = np.arange(total, dtype=np.uint32) if resident else np.full(total, M.MORI_NO_PAGE, np.uint32)
    free = np.ones(num_blocks, np.uint8)
    if resident:
        free[:total] = 0
    tier = np.full(len(nblk), M.MORI_TIER_GPU if resident else M.MORI_TIER_WAIT, np.uint8)
    block = geom.layers * geom.planes * geom.block_tokens * geom.row_bytes
    return TierPool(Geometry(geom.layers, geom.planes, geom.block_tokens, geom.row_bytes, num_blocks), off, tbl, tier,
                    free, arena_bytes=2 * total * block + (1 << 20))


def main(rounds=4, steps=3):
    inst = make_instance(TINY)
    g, nblk = inst.geom, np.asarray(inst.nblk, np.int64)
    prompt = np.maximum(1, nblk * g.block_tokens - GROWTH)
    budget = budget_bytes(inst.total_bytes, TINY.gpu_pct)
    moving = empty_pool(g, nblk, -(-budget // g.block_bytes), resident=False)
    still = empty_pool(g, nblk, int(nblk.sum()), resident=True)
    models = [Decoder(tp, g.layers, int(prompt.max()) + GROWTH) for tp in (moving, still)]
    gen = torch.Generator(device="cuda").manual_seed(1)
    held = np.zeros(inst.P, np.int64)  # tokens of a program in its cache
    last = torch.zeros(inst.P, HEADS * DIM, dtype=torch.half, device="cuda")
    moved = {"in": 0, "out": 0, "tokens": 0}
    try:
        for r in range(rounds):
            window = inst.window if r % 2 == 0 else inst.window[:, :, ::-1].copy()
            plan = moving.step(gpu_bytes=budget, cpu_bytes=inst.total_bytes if r else 0,
                               window=torch.from_numpy(window).cuda())
            moved["in"] += plan.n_in
            moved["out"] += plan.n_out
            resident = np.flatnonzero(moving.state()[1] == M.MORI_TIER_GPU)
            for step in range(steps):
                # programs new to the GPU bring their prompt, the others one token: one mixed batch
                new = np.where(held[resident] == 0, prompt[resident], 1)
                here = resident[held[resident] + new <= nblk[resident] * g.block_tokens]
                new = np.where(held[here] == 0, prompt[here], 1)
                x = torch.randn(int(new.sum()), HEADS * DIM, device="cuda", generator=gen).half()
                ends = np.cumsum(new) - 1
                for i, p in enumerate(here):
                    if held[p]:
                        x[ends[i]] = last[p]
                batches = [TokenBatch.of(tp, here, new, held[here] + new) for tp in (moving, still)]
                a, b = (m(x, t) for m, t in zip(models, batches))
                for t in batches:
                    t.check()
                if not torch.equal(a, b):
                    raise AssertionError(f"round {r}, step {step}: outputs differ by {(a - b).abs().max().item()}")
                held[here] += new
                last[torch.from_numpy(here).cuda()] = a[torch.from_numpy(ends).cuda()]
                moved["tokens"] += int(new.sum())
    finally:
        moving.close()
        still.close()
    print(f"{moved['tokens']} tokens over {rounds} rebalances ({moved['out']} programs out, {moved['in']} back in): "
          "outputs equal those of a pool that never moves")
    return moved


if __name__ == "__main__":
    main()
