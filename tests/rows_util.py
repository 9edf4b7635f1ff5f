"""Rows of logits for the tests of the draws, the largest logits and the distillation, and the same from the definitions in 64 bits."""
import math

import torch

LN2 = math.log(2.0)


def rows_of(R, V, dtype, seed, pad=0, start=0, spread=3.0, zipf=True, device="cuda"):
    """[R, V] view of a buffer whose rows lie V + pad apart, its first row `start` elements behind a 16-byte boundary; NaN around the rows."""
    g = torch.Generator().manual_seed(seed)
    x = spread * torch.randn(R, V, generator=g)
    if zipf:
        x -= torch.log1p(torch.randperm(V, generator=g).float())
    buf = torch.full((start + R * (V + pad) + 16,), math.nan, dtype=dtype, device=device)
    z = buf[start:start + R * (V + pad)].view(R, V + pad)[:, :V]
    z.copy_(x)
    return z


def order_of(x):
    """Tokens by falling logit, of equal ones the lower token first."""
    return torch.sort(x, descending=True, stable=True).indices


def draw(x, u, T, k=0, p=1.0, m=0.0):
    """The token and log-probability that a uniform number u draws from one row x (all doubles)."""
    V = len(x)
    order = order_of(x)
    if T == 0:
        return int(order[0]), 0.0
    w = torch.exp((x - x.max()) / T)
    if 0 < k < V:
        order = order[:k]
    if p < 1:
        s = w[order].cumsum(0)
        order = order[:int((s < p * s[-1]).sum()) + 1]
    order = order[w[order] >= m]
    kept = order[w[order] > 0].sort().values
    s = w[kept].cumsum(0)
    i = min(int((s <= u * s[-1]).sum()), len(kept) - 1)
    return int(kept[i]), float((x[kept[i]] - x.max()) / T - s[-1].log())


def top(x, K, T):
    order = order_of(x)
    at, left = order[:K], order[K:]
    rest = torch.logsumexp(x[left] / T, 0) if len(left) else torch.tensor(-math.inf, dtype=torch.float64)
    return x[at], at, rest


def distill(x, value, index, rest, T):
    """Loss (differentiable by x) of one row x against entries (value, index; index -1 is none) and `rest` (None: without)."""
    there = index >= 0
    at, teacher = index[there].long(), value[there] / T
    log_q = torch.log_softmax(x / T, 0)
    told = log_q[at]
    if rest is not None:
        others = torch.ones(len(x), dtype=torch.bool, device=x.device)
        others[at] = False
        told = torch.cat([told, torch.logsumexp(log_q[others], 0)[None] if others.any() else told.new_full((1,), -math.inf)])
        teacher = torch.cat([teacher, rest[None]])
    log_p = torch.log_softmax(teacher, 0)
    some = log_p > -math.inf
    p = log_p.exp()
    return T * T * (p[some] * (log_p[some] - told[some])).sum()
