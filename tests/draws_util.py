"""Draws of dsbd_sample_rows against the definition in 64 bits, and the exact size of a prefix."""
import numpy as np
import torch

import paper_2409_16560_b200 as dsbd
import rows_util as ru

F32, I32 = torch.float32, torch.int32


def f32(x):
    return float(torch.tensor(x, dtype=F32))


def check(z, u, T=1.0, k=0, p=1.0, m=0.0):
    """Every draw of every row: equal tokens; logp is fp32 of a sum in 64 bits, half a step."""
    token, logp, status = dsbd.sample_rows(z, u.cuda(), temperature=T, top_k=k, top_p=p, min_p=m)
    assert int(status) == 0
    x, uu, got, got_p = z.double().cpu(), u.double().cpu(), token.cpu(), logp.double().cpu()
    for r in range(z.shape[0]):
        for j in range(u.shape[1]):
            t, lp = ru.draw(x[r], float(uu[r, j]), f32(T), k, f32(p), f32(m))
            assert int(got[r, j]) == t, (r, j, int(got[r, j]), t)
            assert abs(float(got_p[r, j]) - lp) <= 2.0 ** -24 * abs(lp) + 1e-12, (r, j)


def prefix(x, T, p, k=0):
    """Of a row x that falls from token to token: how many tokens the shortest prefix of p of the (first k tokens') mass has, the logarithm of its mass relative to the
    largest token's, and how far, in parts of the whole, the goal is from either end of the prefix's last token; in 80 bits."""
    x = np.asarray(x, dtype=np.longdouble)
    assert bool((np.diff(x) <= 0).all())
    w = np.exp((x - x[0]) / np.longdouble(f32(T)))
    s = np.cumsum(w[:k or None])
    goal = np.longdouble(f32(p)) * s[-1]
    n = int((s < goal).sum()) + 1
    below = s[n - 2] if n > 1 else np.longdouble(0)
    return n, float(np.log(s[n - 1])), float(min(goal - below, s[n - 1] - goal) / s[-1])
