"""Plain 64-bit forms of the operators between a model's projections and the decode step, for the tests."""
import numpy as np
import torch

PAGE = 64


def turned(x, w, rows, layout, eps):
    """Rows x [T, H, d] normed (w [d] or None) and rotated by the table rows [T, 2, rot / 2] (None: not rotated)."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
    if rows is None:
        return x
    rows = rows.double()
    half = rows.shape[2]
    y = x.clone()
    for i in range(half):
        a, b = (i, i + half) if layout == "half" else (2 * i, 2 * i + 1)
        c, s = rows[:, 0, i, None], rows[:, 1, i, None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def turned_bar(x, w, rows, layout, eps, bf16):
    """Largest error that fp32 arithmetic and the output's rounding allow: each term of a pair and the norm's factor carry a
    few roundings of 2^-24 (16 are allowed: mean, rsqrt, products, sum), the output one of 2^-8 in bf16 (8 significant bits)."""
    pairs = turned(x.abs(), w.abs() if w is not None else None, rows.abs() if rows is not None else None, layout, eps)
    y = turned(x, w, rows, layout, eps)
    if rows is not None:                   # |a c| + |b s| of the first of a pair: its difference became a sum
        half = rows.shape[2]
        z = turned(x.abs(), w.abs() if w is not None else None, None, layout, eps)
        for i in range(half):
            a, b = (i, i + half) if layout == "half" else (2 * i, 2 * i + 1)
            c, s = rows.double().abs()[:, 0, i, None], rows.double().abs()[:, 1, i, None]
            pairs[..., a] = z[..., a] * c + z[..., b] * s
    return y, 16 * 2.0 ** -24 * pairs + (2.0 ** -8 * 1.01 * y.abs() if bf16 else 2.0 ** -24 * y.abs()) + 1e-37


def paged_problem(new, old, Hkv, d, dtype, seed, extra_pages=3, device="cuda"):
    """Pools, tables and offsets of sequences with old[b] cached tokens that get new[b] more."""
    new, old = np.asarray(new, np.int64), np.asarray(old, np.int64)
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    need = -(-(new + old) // PAGE)
    page_off = np.concatenate([[0], np.cumsum(need)]).astype(np.int64)
    n_pages = int(page_off[-1]) + extra_pages
    perm = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed))
    randn = lambda *s: torch.randn(*s, generator=gen, device=device).to(dtype)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device)
    new_off = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    prefix_off = np.concatenate([[0], np.cumsum(old)]).astype(np.int64)
    table = perm[:int(page_off[-1])].to(torch.int32)
    return dict(new=new, old=old, new_off_host=new_off, prefix_off_host=prefix_off, page_off_host=page_off, table_host=table.numpy(),
                new_off=dev(new_off), prefix_off=dev(prefix_off), page_off=dev(page_off),
                page_table=table.to(device) if len(table) else torch.zeros(1, dtype=torch.int32, device=device),
                k_pool=randn(n_pages, Hkv, PAGE, d), v_pool=randn(n_pages, Hkv, PAGE, d), randn=randn, T=int(new.sum()))


def chunk_of(p):
    import paper_2409_16560_b200 as dsbd
    return dsbd.Chunk(p["new_off"], p["new_off_host"], p["prefix_off"], p["prefix_off_host"], p["page_table"], p["page_off"])


def cache_of(pool, p, b, tokens):
    """The first `tokens` rows of sequence b, [tokens, Hkv, d]."""
    pages = torch.as_tensor(p["table_host"][p["page_off_host"][b]:p["page_off_host"][b + 1]]).long().to(pool.device)
    return pool[pages].permute(0, 2, 1, 3).flatten(0, 1)[:tokens]


def attention_reference(q, p, scale, rows_at_once=512):
    """out, and sum_j w_j |v_j| (what the error bar is made of), in 64 bits."""
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    mass = torch.zeros_like(out)
    group = q.shape[1] // p["k_pool"].shape[1]
    for b in range(len(p["new"])):
        n, L = int(p["new"][b]), int(p["old"][b])
        if n == 0:
            continue
        k, v = (cache_of(x, p, b, L + n).double() for x in (p["k_pool"], p["v_pool"]))
        first = int(p["new_off_host"][b])
        for i0 in range(0, n, rows_at_once):
            i1 = min(n, i0 + rows_at_once)
            for g in range(k.shape[1]):
                z = torch.einsum("nhd,td->nht", q[first + i0:first + i1, g * group:(g + 1) * group].double(), k[:, g]) * scale
                hidden = torch.arange(L + n, device=q.device)[None, :] > L + torch.arange(i0, i1, device=q.device)[:, None]
                w = torch.softmax(z.masked_fill(hidden[:, None, :], float("-inf")), -1)
                out[first + i0:first + i1, g * group:(g + 1) * group] = torch.einsum("nht,td->nhd", w, v[:, g])
                mass[first + i0:first + i1, g * group:(g + 1) * group] = torch.einsum("nht,td->nhd", w, v[:, g].abs())
    return out, mass


def attention_bar(mass):
    """Weights are rounded to bf16 (2^-8: 8 significant bits) in the sum over the values and in the row sum, the result once
    more; fp32 sums of d products move a logit by less than 1e-4 at the tests' sizes, which moves a weight by as much."""
    return (2.0 ** -7 + 2.0 ** -8 + 2e-4) * mass + 1e-30
