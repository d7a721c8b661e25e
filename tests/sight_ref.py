"""Plain 64-bit definition of attention with caps, biases by distance, windows and
ranges (numpy, one token at a time), and what its evaluation may be off by."""
from __future__ import annotations

import numpy as np

import attend_ref as R


def attend(inst, q, scale, cap=None, slopes=None, window=None, first=None, end=None):
    """out, lse (float64) and the bound of out's error."""
    T, H = q.shape[:2]
    D, G, dtype = q.shape[2], q.shape[1] // inst.kv, inst.dtype
    q = q.double().numpy()
    out, lse = np.zeros((T, H, D)), np.full((T, H), -np.inf)
    mean, delta, count, top = np.zeros((T, H, D)), np.zeros((T, H, 1)), np.zeros((T, H, 1)), np.zeros((T, H, 1))
    for b in range(inst.n.size):
        n, L = int(inst.n[b]), int(inst.length[b])
        k, v = inst.rows(0, b, L), inst.rows(1, b, L)
        for i in range(n):
            t, pos = int(inst.seq_off[b]) + i, L - n + i
            if pos < 0:
                continue
            lo, hi = 0, pos + 1
            if window is not None:
                lo = max(lo, pos + 1 - window)
            if first is not None:
                lo = max(lo, int(first[t]))
            if end is not None:
                hi = min(L, int(end[t]))
            if lo >= hi:
                continue
            for h in range(H):
                kk, vv = k[lo:hi, h // G], v[lo:hi, h // G]
                s = kk @ q[t, h] * scale
                # as in attend_ref; a cap does not stretch differences.  Its tanh as 1 - 2 r, r = 1 / (e + 1): r is
                # off by the exponential's and the reciprocal's 2^-23, the argument's rounding (2x 2^-24 of e) and
                # the sum's, together below 2 r (1 - r) (2^-23 + x 2^-23) + 2 r 2^-23 + 2^-24 < 2^-22 of the cap;
                # above a cap of 64 by 2^-20 of the score (a polynomial's 7e-7 and roundings, or the above next to
                # a tanh of 0.76 at least).  A bias adds two roundings of itself and one of the sum
                d = (D + 3) * 2.0 ** -23 * (np.abs(kk) @ np.abs(q[t, h])).max() * abs(scale)
                if cap is not None:
                    s = cap * np.tanh(s / cap)
                    d += 2.0 ** -20 * np.abs(s).max() + (cap * 2.0 ** -22 if cap <= 64 else 0)
                if slopes is not None:
                    far = float(slopes[h]) * np.abs(pos - np.arange(lo, hi))
                    s = s - far
                    # keys far below the largest score weigh nothing whatever their score's error is
                    near = s >= s.max() - 40
                    d += 2.0 ** -22 * (np.abs(far[near]).max() + np.abs(s[near]).max())
                top_s = s.max()
                w = np.exp(s - top_s)
                lse[t, h] = top_s + np.log(w.sum())
                w /= w.sum()
                out[t, h] = w @ vv
                mean[t, h] = w @ np.abs(vv)
                delta[t, h], count[t, h], top[t, h] = d, hi - lo, np.abs(vv).max()
    return out, lse, R.attend_bound(dtype, out, mean, delta, count, top), delta[..., 0]
