"""The operators between a model's QKV projection and the decode step, with the sizes they come in.

Rotation of queries and keys by position (with the per-head norms), the append of a chunk's keys and
values to the paged cache, the attention of the chunk over that cache, and the positions of a forest's
nodes.  A case is one pass through one of them; buffers, workspaces and launch facts are made in
`prepare`, as a serving program makes them once per step or per model.

`run` has two forms: the library's calls (`own`), and the same formulas in elementary torch operations,
in 32 bits and rounded once at the end.
"""
import math

import numpy as np
import torch

own = False
DEVICE = "cuda"
PAGE = 64


# ------------------------------------------------------------------------------------ cases
def listed():
    gqa = dict(Hq=32, Hkv=8, d=128, dtype="bf16")
    mha = dict(Hq=32, Hkv=32, d=128, dtype="bf16")
    small = dict(Hq=32, Hkv=8, d=64, dtype="bf16")
    full = dict(rot=128, layout="half", norm=True)
    return [
        # one request of a 7B-shaped model: four chains of five nodes before the forest attention; latency
        dict(name="rotate-one-request", op="rotate", T=20, **mha, rot=128, layout="half", norm=False, max_position=600),
        # a toy model in fp32 with interleaved pairs over half of each head (unit tests, debugging a port)
        dict(name="rotate-toy-f32", op="rotate", T=301, Hq=4, Hkv=4, d=64, dtype="f32", rot=32, layout="interleaved",
             norm=True, max_position=700),
        # the forest of the large serving step: 64 requests x 8 beams x 9 nodes, normed heads
        dict(name="rotate-forest-large", op="rotate", T=4608, **gqa, **full, max_position=4200),
        # the same forest's positions, and those of one request
        dict(name="positions-one-request", op="positions", B=4, tree="chain", depth=4, L_lo=200, L_hi=512),
        dict(name="positions-forest-large", op="positions", B=512, tree="wide", depth=6, L_lo=1024, L_hi=4096),
        # one new token of each of 64 sequences (the small model between two draws)
        dict(name="append-one-token-each", op="append", B=64, n_lo=1, n_hi=1, L_lo=100, L_hi=1000, **small,
             rot=64, layout="half", norm=False, with_q=True),
        # a batch of ragged prompts, nothing cached yet
        dict(name="append-prompts", op="append", B=16, n_lo=70, n_hi=1500, L_lo=0, L_hi=0, **gqa, **full, with_q=True),
        # one long prompt
        dict(name="append-long-prompt", op="append", B=1, n_lo=16384, n_hi=16384, L_lo=0, L_hi=0, **gqa, **full,
             with_q=True),
        # the smallest attention: the small model's four beams of one request, a token each, heads of 64
        dict(name="attend-one-request-d64", op="attend", B=4, n_lo=1, n_hi=1, L_lo=512, L_hi=516, **small),
        # a batch that decodes plainly, one token a sequence, ragged caches
        dict(name="attend-one-token-each", op="attend", B=64, n_lo=1, n_hi=1, L_lo=1024, L_hi=4096, **gqa),
        # a serving step that mixes pieces of prompts behind caches of any length
        dict(name="attend-mixed", op="attend", B=12, n_lo=1, n_hi=777, L_lo=0, L_hi=6000, **gqa),
        # one long prompt at once
        dict(name="attend-long-prompt", op="attend", B=1, n_lo=16384, n_hi=16384, L_lo=0, L_hi=0, **gqa),
    ]


# a drawn case stays below the largest listed one of its operator
MAX_ROTATE_BYTES = 0.34e9
MAX_APPEND_BYTES = 0.41e9
MAX_ATTEND_FLOPS = 2.1e12
MAX_ATTEND_BYTES = 0.7e9
MAX_ATTEND_PAD = 2.2e9           # entries of the padded score matrix of one KV head's queries, over the sequences


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng, dtype):
    if dtype == "f32":
        Hq, Hkv = rng.choice([(4, 4), (8, 2), (12, 12)])
    else:
        Hq, Hkv = rng.choice([(32, 8), (32, 8), (32, 32), (40, 40), (16, 4), (28, 4), (12, 12)])
    return dict(Hq=Hq, Hkv=Hkv, d=rng.choice([64, 128, 128]), dtype=dtype)


def _rope(rng, d):
    return dict(rot=rng.choice([d, d, d // 2, d // 4]), layout=rng.choice(["half", "half", "interleaved"]),
                norm=rng.random() < 0.5)


def draw(rng):
    op = rng.choice(["rotate", "append", "attend", "attend", "positions"])
    if op == "positions":
        c = dict(op=op, B=_log_int(rng, 1, 512), tree=rng.choice(["chain", "wide"]), depth=rng.randint(1, 8),
                 L_lo=rng.randint(0, 1024), L_hi=rng.randint(1024, 8192))
        c["depth"] = 6 if c["tree"] == "wide" else c["depth"]
        return c
    heads = _heads(rng, "f32" if op != "attend" and rng.random() < 0.2 else "bf16")
    if op == "rotate":
        c = dict(op=op, T=_log_int(rng, 1, 16384), **heads, **_rope(rng, heads["d"]),
                 max_position=_log_int(rng, 64, 32768))
        while work(c)["bytes"] > MAX_ROTATE_BYTES:
            c["T"] = c["T"] * 3 // 4
        return c
    B = _log_int(rng, 1, 64)
    n_lo = rng.choice([1, _log_int(rng, 1, 1024)])
    n_hi = rng.choice([n_lo, _log_int(rng, n_lo, 16384 if B == 1 else 2048)])
    L_lo = rng.choice([0, _log_int(rng, 1, 8192)])
    L_hi = rng.choice([L_lo, _log_int(rng, max(L_lo, 1), 16384)])
    c = dict(op=op, B=B, n_lo=n_lo, n_hi=n_hi, L_lo=L_lo, L_hi=L_hi, **heads)
    if op == "append":
        c.update(_rope(rng, heads["d"]))
        c.update(with_q=rng.random() < 0.7, L_lo=min(L_lo, 1024), L_hi=min(L_hi, 1024))
    while _too_large(c):
        if c["B"] > 1:
            c["B"] = max(1, c["B"] * 3 // 4)
        elif c["n_hi"] > 256:
            c["n_hi"] = c["n_hi"] * 3 // 4
            c["n_lo"] = min(c["n_lo"], c["n_hi"])
        else:
            c["L_hi"] = c["L_hi"] * 3 // 4
            c["L_lo"] = min(c["L_lo"], c["L_hi"])
    return c


def _too_large(c):
    w = work(c)
    if c["op"] == "append":
        return w["bytes"] > MAX_APPEND_BYTES
    new, old = _lengths(c)
    pad = c["B"] * (c["Hq"] // c["Hkv"]) * int(new.max()) * int((new + old).max())
    return w["flops"] > MAX_ATTEND_FLOPS or w["bytes"] > MAX_ATTEND_BYTES or pad > MAX_ATTEND_PAD


# ------------------------------------------------------------------------------------ sizes
def _lengths(c):
    """New tokens and cached tokens of every sequence: spread evenly over the logarithm, in a fixed mixed order."""
    def spread(lo, hi, mult):
        i = (np.arange(c["B"]) * mult + 3) % c["B"]
        x = i / max(c["B"] - 1, 1)
        return np.round(np.exp(np.log(lo + 1) + x * (np.log(hi + 1) - np.log(lo + 1))) - 1).astype(np.int64)
    coprime = [m for m in (7, 11, 13) if c["B"] % m] or [1]
    return np.maximum(spread(c["n_lo"], c["n_hi"], coprime[0]), 1), spread(c["L_lo"], c["L_hi"], coprime[-1])


def _tree(c):
    if c["tree"] == "chain":
        return [-1] + list(range(c["depth"]))
    return [-1, 0, 0, 1, 1, 2, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15]


def _elem(c):
    return 2 if c["dtype"] == "bf16" else 4


def work(c):
    if c["op"] == "positions":
        N = c["B"] * len(_tree(c))
        return dict(bytes=8 * N + 4 * (c["B"] + 1) + 8 * (c["B"] + 1), flops=2 * N)
    if c["op"] == "rotate":
        el = c["T"] * (c["Hq"] + c["Hkv"]) * c["d"]
        table = min(c["T"], c["max_position"]) * c["rot"] * 4
        return dict(bytes=2 * el * _elem(c) + table + 4 * c["T"], flops=el * (7 if c["norm"] else 3))
    new, old = _lengths(c)
    T = int(new.sum())
    if c["op"] == "append":
        q = c["Hq"] if c["with_q"] else 0
        table = int((new + old).max() - old.min()) * c["rot"] * 4
        return dict(bytes=2 * T * (q + 2 * c["Hkv"]) * c["d"] * _elem(c) + table,
                    flops=T * (q + c["Hkv"]) * c["d"] * (7 if c["norm"] else 3))
    seen = int((new * old + new * (new + 1) // 2).sum())
    return dict(bytes=int((new + old).sum()) * c["Hkv"] * c["d"] * 2 * _elem(c) + 2 * T * c["Hq"] * c["d"] * _elem(c),
                flops=4 * c["Hq"] * c["d"] * seen)


# ------------------------------------------------------------------------------------ inputs
def _table(n, rot, base=500000.0):
    """Rows (cos, sin) of the angles position * base^(-2 i / rot)."""
    inv = base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEVICE) / rot)
    ang = torch.arange(n, dtype=torch.float64, device=DEVICE)[:, None] * inv[None, :]
    return torch.stack([ang.cos(), ang.sin()], dim=1).float().contiguous()


def _inputs(c, seed):
    """Tensors and host facts, the same for every form of the operator."""
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    s = dict(case=c)
    if c["op"] == "positions":
        tree = np.asarray(_tree(c))
        B, n = c["B"], len(tree)
        off = np.arange(B + 1, dtype=np.int32) * n
        s["parent_host"] = np.where(tree[None, :] >= 0, tree[None, :] + off[:-1, None], -1).reshape(-1).astype(np.int32)
        s["node_off_host"] = off
        L = torch.randint(c["L_lo"], c["L_hi"] + 1, (B,), generator=gen, device=DEVICE)
        s["prefix_off"] = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEVICE), L.cumsum(0)])
        s["parent"] = torch.from_numpy(s["parent_host"]).to(DEVICE)
        s["node_off"] = torch.from_numpy(off).to(DEVICE)
        return s
    Hq, Hkv, d = c["Hq"], c["Hkv"], c["d"]
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    randn = lambda *shape: torch.randn(*shape, generator=gen, device=DEVICE).to(dt)
    if c["op"] == "rotate":
        T, new, old = c["T"], None, None
        # beams of nearby lengths, a few nodes each
        s["position"] = torch.randint(0, c["max_position"], (T,), generator=gen, device=DEVICE, dtype=torch.int32)
    else:
        new, old = _lengths(c)
        T = int(new.sum())
        s["new_off_host"] = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        s["prefix_off_host"] = np.concatenate([[0], np.cumsum(old)]).astype(np.int64)
        need = -(-(new + old) // PAGE)
        page_off = np.concatenate([[0], np.cumsum(need)]).astype(np.int64)
        s["n_pages"] = int(page_off[-1]) + 3
        perm = torch.randperm(s["n_pages"], generator=torch.Generator().manual_seed(seed))
        s["page_table"] = perm[:int(page_off[-1])].to(torch.int32).to(DEVICE)
        s["page_off"] = torch.from_numpy(page_off).to(DEVICE)
        s["new_off"] = torch.from_numpy(s["new_off_host"]).to(DEVICE)
        s["prefix_off"] = torch.from_numpy(s["prefix_off_host"]).to(DEVICE)
        s["k_pool"] = randn(s["n_pages"], Hkv, PAGE, d)
        s["v_pool"] = randn(s["n_pages"], Hkv, PAGE, d)
    if c["op"] == "attend":
        s["q"] = randn(T, Hq, d)
        return s
    # the output of a fused projection, and the views of it that a model takes
    qkv = randn(T, (Hq + 2 * Hkv) * d)
    s["q"] = qkv[:, :Hq * d].unflatten(1, (Hq, d))
    s["k"] = qkv[:, Hq * d:(Hq + Hkv) * d].unflatten(1, (Hkv, d))
    s["v"] = qkv[:, (Hq + Hkv) * d:].unflatten(1, (Hkv, d))
    positions = c["max_position"] if c["op"] == "rotate" else int((new + old).max())
    s["table"] = _table(positions, c["rot"])
    for name in ("q_norm", "k_norm"):
        s[name] = 1 + 0.2 * torch.randn(d, generator=gen, device=DEVICE) if c["norm"] else None
    return s


def prepare(case, seed):
    c = dict(case)
    s = _inputs(c, seed)
    if not own:
        if c["op"] == "attend":
            s["plan"] = _padded_plan(s["new_off_host"], s["prefix_off_host"])
        if c["op"] == "append":
            s["plan"] = _slots(s)
        if c["op"] == "positions":
            s["tree_of"] = torch.from_numpy(np.repeat(np.arange(c["B"]), len(_tree(c)))).to(DEVICE)
        return s
    import paper_2409_16560_b200 as dsbd
    s["status"] = torch.zeros(1, dtype=torch.int32, device=DEVICE)
    if c["op"] == "positions":
        B = c["B"]
        s["forest"] = dsbd.Forest(dict(R=B, B=B, N=len(s["parent_host"]), max_depth=8, req_beam_off=np.arange(B + 1),
                                       beam_node_off=s["node_off_host"], parent=s["parent_host"],
                                       token=np.zeros(len(s["parent_host"]))), DEVICE)
        s["out"] = torch.empty(len(s["parent_host"]), dtype=torch.int32, device=DEVICE)
        return s
    if c["op"] != "attend":
        s["rope"] = dsbd.Rope(s["table"], layout=c["layout"], q_norm=s["q_norm"], k_norm=s["k_norm"], eps=1e-6)
        s["q_out"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device=DEVICE)
        s["k_out"] = torch.empty(s["k"].shape, dtype=s["k"].dtype, device=DEVICE)
    if c["op"] != "rotate":
        s["chunk"] = dsbd.Chunk(s["new_off"], s["new_off_host"], s["prefix_off"], s["prefix_off_host"],
                                s["page_table"], s["page_off"])
    if c["op"] == "attend":
        s["out"] = torch.empty_like(s["q"])
        need = dsbd.chunk_attention_workspace(s["chunk"], c["Hq"], c["Hkv"], c["d"], s["q"].dtype, c["d"] ** -0.5)
        s["workspace"] = torch.empty(max(need, 256), dtype=torch.uint8, device=DEVICE)
    return s


def run(s):
    if own:
        return _run_own(s)
    return dict(rotate=_plain_rotate, append=_plain_append, attend=_plain_attend, positions=_plain_positions)[s["case"]["op"]](s)


def _run_own(s):
    import paper_2409_16560_b200 as dsbd
    c = s["case"]
    if c["op"] == "positions":
        dsbd.forest_positions(s["forest"], s["prefix_off"], position=s["out"], status=s["status"])
        return s["out"]
    if c["op"] == "rotate":
        dsbd.rotate_qk(s["q"], s["k"], s["position"], s["rope"], q_out=s["q_out"], k_out=s["k_out"], status=s["status"])
        return s["q_out"], s["k_out"]
    if c["op"] == "append":
        dsbd.kv_append_paged(s["chunk"], s["k"], s["v"], s["k_pool"], s["v_pool"], rope=s["rope"],
                             q=s["q"] if c["with_q"] else None, q_out=s["q_out"] if c["with_q"] else None,
                             status=s["status"])
        return (s["k_pool"], s["v_pool"]) + ((s["q_out"],) if c["with_q"] else ())
    dsbd.chunk_attention_paged(s["chunk"], c["Hq"], c["Hkv"], c["d"], c["d"] ** -0.5, s["q"], s["k_pool"], s["v_pool"],
                               out=s["out"], workspace=s["workspace"], status=s["status"])
    return s["out"]


# ------------------------------------------------------------------------------------ the plain forms
def _normed(x, w):
    x = x.float()
    return x if w is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w


def _rotated(x, w, rows, c):
    """x [T, H, d] normed and rotated by the table rows [T, 2, rot / 2], in the type of x."""
    y, rot = _normed(x, w), c["rot"]
    cos, sin = rows[:, None, 0], rows[:, None, 1]
    a, b = (y[..., :rot // 2], y[..., rot // 2:rot]) if c["layout"] == "half" else (y[..., 0:rot:2], y[..., 1:rot:2])
    u, v = a * cos - b * sin, b * cos + a * sin
    head = torch.cat([u, v], -1) if c["layout"] == "half" else torch.stack([u, v], -1).flatten(-2)
    return torch.cat([head, y[..., rot:]], -1).to(x.dtype)


def _plain_rotate(s):
    c, rows = s["case"], s["table"][s["position"].long()]
    return _rotated(s["q"], s["q_norm"], rows, c), _rotated(s["k"], s["k_norm"], rows, c)


def _slots(s):
    """Where a chunk's rows go: positions and rows of the pools, and the rows that become zeros."""
    new, old = np.diff(s["new_off_host"]), np.diff(s["prefix_off_host"])
    seq = np.repeat(np.arange(len(new)), new)
    pos = old[seq] + np.arange(len(seq)) - s["new_off_host"][seq]
    # behind the last token of a page that the chunk opened
    end = old + new
    fill = np.where((end % PAGE != 0) & (end // PAGE * PAGE >= old), PAGE - end % PAGE, 0)
    zseq = np.repeat(np.arange(len(new)), fill)
    zpos = end[zseq] + np.arange(len(zseq)) - np.repeat(np.cumsum(fill) - fill, fill)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEVICE)
    return dict(seq=dev(seq), pos=dev(pos), zseq=dev(zseq), zpos=dev(zpos))


def _plain_append(s):
    c, p = s["case"], s["plan"]
    rows = s["table"][p["pos"]]
    page = s["page_table"][s["page_off"][p["seq"]] + p["pos"] // PAGE].long()
    zpage = s["page_table"][s["page_off"][p["zseq"]] + p["zpos"] // PAGE].long()
    s["k_pool"][page, :, p["pos"] % PAGE] = _rotated(s["k"], s["k_norm"], rows, c)
    s["v_pool"][page, :, p["pos"] % PAGE] = s["v"]
    s["k_pool"][zpage, :, p["zpos"] % PAGE] = 0
    s["v_pool"][zpage, :, p["zpos"] % PAGE] = 0
    return (s["k_pool"], s["v_pool"]) + ((_rotated(s["q"], s["q_norm"], rows, c),) if c["with_q"] else ())


def _padded_plan(new_off, prefix_off):
    """Indices that lay ragged sequences out as one padded batch."""
    new, old = np.diff(new_off), np.diff(prefix_off)
    rows, pages = int(new.max()), int((-(-(new + old) // PAGE)).max())
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEVICE)
    i = np.arange(rows)[None, :]
    return dict(rows=rows, pages=pages, row=dev(np.minimum(new_off[:-1, None] + i, new_off[-1] - 1)),
                last=dev(old[:, None] + i), valid=dev(i < new[:, None]), end=dev(new + old))


def _plain_attend(s):
    """Padded batch, a block of KV heads at a time."""
    c, p = s["case"], s["plan"]
    Hq, Hkv, d, B = c["Hq"], c["Hkv"], c["d"], c["B"]
    n, L = p["rows"], p["pages"] * PAGE
    at = s["page_off"][:-1, None] + torch.arange(p["pages"], device=DEVICE)
    page = s["page_table"][at.clamp(max=len(s["page_table"]) - 1)].long()
    token = torch.arange(L, device=DEVICE)
    hidden = token[None, None, :] > torch.minimum(p["last"], p["end"][:, None] - 1)[:, :, None]        # [B, n, L]
    beyond = (token[None, :] >= p["end"][:, None])[:, None, :, None]
    out = torch.empty_like(s["q"])
    per_head = B * (Hq // Hkv) * n * L
    step = max(1, min(Hkv, (1 << 30) // per_head))
    for g in range(0, Hkv, step):
        h = min(step, Hkv - g)
        q = s["q"][:, g * (Hq // Hkv):(g + h) * (Hq // Hkv)][p["row"]].float()                        # [B, n, h group, d]
        q = q.unflatten(2, (h, Hq // Hkv)).permute(0, 2, 3, 1, 4).flatten(2, 3)                       # [B, h, group n, d]
        k = s["k_pool"][page, g:g + h].float().permute(0, 2, 1, 3, 4).flatten(2, 3)                   # [B, h, L, d]
        v = s["v_pool"][page, g:g + h].float().permute(0, 2, 1, 3, 4).flatten(2, 3)
        v = v.masked_fill(beyond, 0.0)
        z = (q * d ** -0.5) @ k.transpose(-1, -2)                                                     # [B, h, group n, L]
        z.unflatten(2, (Hq // Hkv, n)).masked_fill_(hidden[:, None, None], -math.inf)
        z -= z.amax(-1, keepdim=True)
        z.exp_()
        o = (z @ v) / z.sum(-1, keepdim=True)
        o = o.unflatten(2, (Hq // Hkv, n)).permute(0, 3, 1, 2, 4).flatten(2, 3)                       # [B, n, h group, d]
        out[:, g * (Hq // Hkv):(g + h) * (Hq // Hkv)] = o[p["valid"]].to(out.dtype)
    return out


def _plain_positions(s):
    """Depths by pointer doubling (trees of up to 64 levels)."""
    up, depth = s["parent"].long(), (s["parent"] >= 0).int()
    L = (s["prefix_off"][1:] - s["prefix_off"][:-1]).int()
    for _ in range(6):
        j = up.clamp(min=0)
        live = up >= 0
        depth = depth + torch.where(live, depth[j], 0)
        up = torch.where(live, up[j], up)
    return L[s["tree_of"]] + depth


# ------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """The operators from their definitions, in 64 bits: rotations as complex products, attention sequence by
    sequence, positions by walking up the trees."""
    c = dict(case)
    s = _inputs(c, seed)
    if c["op"] == "positions":
        depth = np.zeros(len(s["parent_host"]), np.int64)
        for i, p in enumerate(s["parent_host"]):
            depth[i] = depth[p] + 1 if p >= 0 else 0
        L = np.diff(s["prefix_off"].cpu().numpy())
        return torch.from_numpy((np.repeat(L, len(_tree(c))) + depth).astype(np.int32))
    if c["op"] == "rotate":
        rows = s["table"][s["position"].long()].double()
        return _turn(s["q"], s["q_norm"], rows, c), _turn(s["k"], s["k_norm"], rows, c)
    new, old = np.diff(s["new_off_host"]), np.diff(s["prefix_off_host"])
    first = s["page_off"].cpu().numpy()
    if c["op"] == "append":
        at = torch.from_numpy(np.concatenate([np.arange(l, l + n) for l, n in zip(old, new)])).to(DEVICE)
        rows = s["table"][at].double()
        k, v = _turn(s["k"], s["k_norm"], rows, c), s["v"].double()
        k_pool, v_pool = s["k_pool"].double(), s["v_pool"].double()
        for b in range(c["B"]):
            pages = s["page_table"][first[b]:first[b + 1]].long()
            for pool, x in ((k_pool, k), (v_pool, v)):
                cache = pool[pages].permute(0, 2, 1, 3).flatten(0, 1).clone()                          # [tokens, Hkv, d]
                lo, hi = int(old[b]), int(old[b] + new[b])
                cache[lo:hi] = x[s["new_off_host"][b]:s["new_off_host"][b + 1]]
                if hi // PAGE * PAGE >= lo:
                    cache[hi:] = 0
                pool[pages] = cache.unflatten(0, (len(pages), PAGE)).permute(0, 2, 1, 3)
        return (k_pool, v_pool) + ((_turn(s["q"], s["q_norm"], rows, c),) if c["with_q"] else ())
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEVICE)
    group = c["Hq"] // c["Hkv"]
    for b in range(c["B"]):
        pages = s["page_table"][first[b]:first[b + 1]].long()
        for lo in range(0, int(new[b]), 1024):
            hi = min(lo + 1024, int(new[b]))
            end = int(old[b]) + hi
            for g in range(c["Hkv"]):
                k = s["k_pool"][pages[:-(-end // PAGE)], g].double().flatten(0, 1)[:end]
                v = s["v_pool"][pages[:-(-end // PAGE)], g].double().flatten(0, 1)[:end]
                r = slice(int(s["new_off_host"][b]) + lo, int(s["new_off_host"][b]) + hi)
                q = s["q"][r, g * group:(g + 1) * group].double()
                z = torch.einsum("nhd,td->nht", q, k) * c["d"] ** -0.5
                seen = torch.arange(end, device=DEVICE)[None, :] <= (int(old[b]) + torch.arange(lo, hi, device=DEVICE))[:, None]
                w = torch.softmax(z.masked_fill(~seen[:, None, :], -math.inf), -1)
                out[r, g * group:(g + 1) * group] = torch.einsum("nht,td->nhd", w, v)
    return out


def _turn(x, w, rows, c):
    x = x.double()
    if w is not None:
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + 1e-6) * w.double()
    rot = c["rot"]
    y = x.clone()
    even, odd = (slice(0, rot // 2), slice(rot // 2, rot)) if c["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    z = torch.complex(x[..., even], x[..., odd]) * torch.complex(rows[:, 0], rows[:, 1])[:, None]
    y[..., even], y[..., odd] = z.real, z.imag
    return y
