"""The operators on rows of next-token logits beside the decode step, with the sizes they come in.

Drawing tokens with each row's own settings (temperature, top-k, top-p, min-p) from given uniforms, the largest logits
of each row with what the rest amounts to, and the loss that pulls a small model's rows to such a teacher, with its
gradient.  A case is one pass through one of them; logits, settings and output buffers are made in `prepare`.

`run` has two forms: the library's calls (`own`), and the same formulas in elementary torch operations.  The plain form
of the draw is in 64 bits, because a token changes when a sum moves across it; the others are in 32 bits and rounded
once at the end, but for the loss's short sums over the teacher's entries, whose terms cancel.
"""
import math

import torch

own = False
DEVICE = "cuda"


# ------------------------------------------------------------------------------------ cases
def listed():
    return [
        # the first beams of one request, drawn behind its prompt with the paper's settings; latency
        dict(name="sample-one-request", op="sample", rows=1, V=32000, pad=0, dtype="f32", draws=4, settings="paper", masked=0.0),
        # a serving step that decodes plainly: each request with settings of its own, some of them constrained to a few tokens
        dict(name="sample-requests", op="sample", rows=64, V=128256, pad=0, dtype="f32", draws=1, settings="rows", masked=0.2),
        # the same with the nucleus alone, rows of an odd vocabulary in a padded buffer
        dict(name="sample-nucleus-odd", op="sample", rows=96, V=50257, pad=47, dtype="bf16", draws=1, settings="nucleus", masked=0.0),
        # a large batch at plain temperature: several samples of each prompt
        dict(name="sample-large", op="sample", rows=512, V=128256, pad=0, dtype="f32", draws=8, settings="plain", masked=0.0),
        # the forest of one request: what the large model said at its nodes
        dict(name="top-one-tree", op="top", rows=20, V=50257, pad=0, dtype="f32", K=16, temperature=1.0),
        # a batch of training rows, many entries of each
        dict(name="top-many-entries", op="top", rows=2048, V=32000, pad=0, dtype="bf16", K=256, temperature=2.0),
        # every node of the large serving step
        dict(name="top-forest-large", op="top", rows=4608, V=128256, pad=0, dtype="f32", K=64, temperature=1.0),
        # an evaluation: losses without gradients, rows of an odd vocabulary
        dict(name="distill-evaluate-odd", op="distill", rows=517, V=50257, pad=0, dtype="bf16", K=16, temperature=1.0, rest=False,
             grad=False),
        # the nodes of one request's forest
        dict(name="distill-one-tree", op="distill", rows=20, V=32000, pad=0, dtype="f32", K=16, temperature=1.0, rest=True, grad=True),
        # a training batch in bf16
        dict(name="distill-batch", op="distill", rows=2048, V=128256, pad=0, dtype="bf16", K=128, temperature=2.0, rest=True, grad=True),
        # every node of the large serving step, from the logits that the verification reads
        dict(name="distill-forest-large", op="distill", rows=4608, V=128256, pad=0, dtype="f32", K=64, temperature=1.0, rest=True,
             grad=True),
    ]


MAX_SAMPLE = 512 * 128256
MAX_ROWS = 4608 * 128256


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["sample", "sample", "top", "distill", "distill"])
    V = rng.choice([32000, 50257, 128256, 151936, 262144, _log_int(rng, 16, 262144), _log_int(rng, 16, 262144)])
    c = dict(op=op, rows=_log_int(rng, 1, 512 if op == "sample" else 4608), V=V, pad=rng.choice([0, 0, 1, 8, 47]),
             dtype=rng.choice(["f32", "bf16"]))
    if op == "sample":
        c.update(draws=rng.choice([1, 1, 4, 8, 16]), settings=rng.choice(["paper", "rows", "rows", "nucleus", "plain"]),
                 masked=rng.choice([0.0, 0.0, 0.3, 1.0]))
    else:
        c.update(K=min(V, _log_int(rng, 1, 512)), temperature=rng.choice([1.0, 1.0, 0.7, 2.0, 4.0]))
    if op == "distill":
        c.update(rest=rng.random() < 0.6, grad=rng.random() < 0.8)
    while c["rows"] * V > (MAX_SAMPLE if op == "sample" else MAX_ROWS):
        c["rows"] = c["rows"] * 3 // 4
    return c


def _size(c):
    return 2 if c["dtype"] == "bf16" else 4


def work(c):
    R, V, el = c["rows"], c["V"], c["rows"] * c["V"]
    if c["op"] == "sample":
        settings = 16 * R if c["settings"] == "rows" else 0
        return dict(bytes=el * _size(c) + 12 * R * c["draws"] + settings, flops=4 * el)
    if c["op"] == "top":
        return dict(bytes=el * _size(c) + R * (8 * c["K"] + 4), flops=4 * el)
    passes = 2 if c["grad"] else 1
    return dict(bytes=passes * el * _size(c) + R * (8 * c["K"] + 4 + (4 if c["rest"] else 0) + (4 if c["grad"] else 0)),
                flops=(7 if c["grad"] else 4) * el)


# ------------------------------------------------------------------------------------ inputs
def _logits(c, gen, base=None):
    """Rows as a model gives them: a long-tailed vocabulary and a spread of each row's own, or another model's rows with noise."""
    R, V, dt = c["rows"], c["V"], torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    z = torch.empty(R, V + c["pad"], dtype=dt, device=DEVICE)
    x = torch.randn(R, V, generator=gen, device=DEVICE)
    if base is None:
        rank = torch.randperm(V, generator=gen, device=DEVICE)
        x = x.mul_(3.0).sub_(torch.log1p(rank.float()))
    else:
        x = x.add_(base)
    z[:, V:] = 1e4                                     # what stands behind a row's vocabulary is not read
    z[:, :V] = x
    return z[:, :V], x


def _inputs(c, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    R, V, s = c["rows"], c["V"], dict(case=c)
    uniform = lambda *shape: torch.rand(*shape, generator=gen, device=DEVICE)
    if c["op"] != "distill":
        s["z"], _ = _logits(c, gen)
    if c["op"] == "sample":
        # a constrained request may use about two hundred tokens
        held = uniform(R, 1) < c["masked"]
        s["z"].masked_fill_(held & (uniform(R, V) > 200.0 / V) & (torch.arange(V, device=DEVICE) != V // 2), -math.inf)
        s["u"] = uniform(R, c["draws"])
        if c["settings"] == "rows":
            pick = lambda values, dtype: torch.tensor(values, dtype=dtype, device=DEVICE)[torch.randint(
                0, len(values), (R,), generator=gen, device=DEVICE)]
            s["how"] = dict(temperature=pick([0.0, 0.6, 0.8, 1.0, 1.3], torch.float32), top_k=pick([0, 0, 20, 50, 1000], torch.int32),
                            top_p=pick([1.0, 0.8, 0.9, 0.95], torch.float32), min_p=pick([0.0, 0.0, 0.02, 0.1], torch.float32))
        else:
            s["how"] = dict(paper=dict(temperature=1.0, top_k=10, top_p=0.8, min_p=0.0),
                            nucleus=dict(temperature=0.9, top_k=0, top_p=0.95, min_p=0.0),
                            plain=dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0))[c["settings"]]
        s["token"] = torch.empty(R, c["draws"], dtype=torch.int32, device=DEVICE)
        s["logp"] = torch.empty(R, c["draws"], device=DEVICE)
        return s
    f32 = lambda *shape: torch.empty(*shape, device=DEVICE)
    if c["op"] == "top":
        s["value"], s["rest"] = f32(R, c["K"]), f32(R)
        s["index"] = torch.empty(R, c["K"], dtype=torch.int32, device=DEVICE)
        return s
    # the teacher's entries, stored when it ran, and the student's rows near them
    T = c["temperature"]
    _, teacher = _logits(dict(c, dtype="f32", pad=0), gen)
    value, index = torch.topk(teacher, c["K"], dim=1)
    s["value"], s["index"], s["rest"] = value.contiguous(), index.int(), None
    if c["rest"]:
        s["rest"] = torch.logsumexp(teacher.scatter(1, index, -math.inf).div_(T), 1)
    s["z"], _ = _logits(c, gen, teacher)
    s["loss"], s["weight"], s["grad"] = f32(R), None, None
    if c["grad"]:
        s["weight"] = (uniform(R) > 0.05).float() / R          # padding rows count for nothing
        s["grad"] = torch.empty(R, V, dtype=s["z"].dtype, device=DEVICE)
    return s


def prepare(case, seed):
    s = _inputs(dict(case), seed)
    s["status"] = torch.zeros(1, dtype=torch.int32, device=DEVICE)
    return s


def run(s):
    if own:
        return _run_own(s)
    return dict(sample=_plain_sample, top=_plain_top, distill=_plain_distill)[s["case"]["op"]](s)


def _run_own(s):
    import paper_2409_16560_b200 as dsbd
    c = s["case"]
    if c["op"] == "sample":
        dsbd.sample_rows(s["z"], s["u"], token=s["token"], logp=s["logp"], status=s["status"], **s["how"])
        return s["token"], s["logp"]
    if c["op"] == "top":
        dsbd.top_logits(s["z"], c["K"], temperature=c["temperature"], value=s["value"], index=s["index"], rest=s["rest"],
                        status=s["status"])
        return s["value"], s["index"], s["rest"]
    dsbd.distill(s["z"], s["value"], s["index"], rest=s["rest"], weight=s["weight"], temperature=c["temperature"], loss=s["loss"],
                 grad=s["grad"], status=s["status"])
    return (s["loss"], s["grad"]) if c["grad"] else s["loss"]


# ------------------------------------------------------------------------------------ the plain forms
def _column(x, like):
    """A setting as a column in 64 bits; a number is the 32-bit number that a call gets."""
    x = x if torch.is_tensor(x) else torch.tensor(float(x), dtype=torch.float32, device=DEVICE).expand(like.shape[0])
    return x.double()[:, None]


def _plain_sample(s):
    """Masses in descending order (ties: lower token first) for the cuts, in the order of the tokens for the draw."""
    z, V = s["z"].float(), s["case"]["V"]
    T, k, p, m = (_column(s["how"][name], z) for name in ("temperature", "top_k", "top_p", "min_p"))
    down, order = torch.sort(z, dim=1, descending=True, stable=True)
    mass = ((down.double() - down[:, :1].double()) / T.clamp(min=1e-30)).exp()
    rank = torch.arange(V, device=DEVICE)[None, :]
    mass = mass * (rank < torch.where(k > 0, k, V))
    before = mass.cumsum(1)
    total = before[:, -1:]
    before = torch.cat([torch.zeros_like(total), before[:, :-1]], 1)
    mass = mass * ((before < p * total) | (p >= 1)) * (mass >= m)
    mass = torch.where(T == 0, (rank == 0).double(), mass)
    mass = torch.zeros_like(mass).scatter_(1, order, mass)
    upto = mass.cumsum(1)
    total = upto[:, -1:]
    # the first token whose cumulative mass exceeds u times the whole (u just below 1 may round up to the whole)
    last = V - 1 - (mass > 0).flip(1).int().argmax(1, keepdim=True)
    token = torch.searchsorted(upto, s["u"].double() * total, right=True).minimum(last)
    return token.int(), (mass.gather(1, token) / total).log().float()


def _plain_top(s):
    c, z = s["case"], s["z"].float()
    down, order = torch.sort(z, dim=1, descending=True, stable=True)
    below = down[:, c["K"]:] / c["temperature"]
    if c["K"] == c["V"]:
        return down, order.int(), torch.full((c["rows"],), -math.inf, device=DEVICE)
    top = below[:, :1].contiguous()
    return down[:, :c["K"]].contiguous(), order[:, :c["K"]].int(), top[:, 0] + below.sub_(top).exp_().sum(1).log()


def _plain_distill(s):
    """The student's softmax in 32 bits; the teacher's entries, K a row, in 64, where their terms cancel."""
    c, T, at = s["case"], s["case"]["temperature"], s["index"].long()
    z = s["z"].float() / T
    top = z.amax(1, keepdim=True)
    e = (z - top).exp()
    whole = e.sum(1, keepdim=True, dtype=torch.float64)
    t = s["value"].double() / T
    logq = z.gather(1, at).double() - top.double() - whole.log()
    if c["rest"]:
        others = e.scatter(1, at, 0.0).sum(1, keepdim=True, dtype=torch.float64)
        t = torch.cat([t, s["rest"][:, None].double()], 1)
        logq = torch.cat([logq, others.log() - whole.log()], 1)
    t = t - t.amax(1, keepdim=True)
    logp = t - t.exp().sum(1, keepdim=True).log()
    p = logp.exp()
    # an entry without mass adds nothing, whatever the student gives it
    loss = (T * T * torch.where(p > 0, p * (logp - logq), 0.0).sum(1)).float()
    if not c["grad"]:
        return loss
    loss = torch.where(s["weight"] == 0, 0.0, loss)
    q = e / whole.float()
    g = q * (1 - p[:, -1:] / logq[:, -1:].exp()).float() if c["rest"] and c["K"] < c["V"] else q
    K = c["K"]
    g = g.scatter(1, at, (logq[:, :K].exp() - p[:, :K]).float())
    return loss, (s["weight"][:, None] * T * g).to(s["z"].dtype)


# ------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """The operators from their definitions, row by row, in 64 bits."""
    c = dict(case)
    s = _inputs(c, seed)
    z, V = s["z"], c["V"]
    if c["op"] == "sample":
        rows = [_exact_row(z[r].double(), s["u"][r].double(), {k: float(v[r] if torch.is_tensor(v) else torch.tensor(v, dtype=torch.float32))
                                                              for k, v in s["how"].items()}) for r in range(c["rows"])]
        return torch.stack([t for t, _ in rows]).int(), torch.stack([p for _, p in rows])
    out = []
    for r in range(c["rows"]):
        x = z[r].double()
        if c["op"] == "top":
            # larger values first, and of equal ones the lower index
            kth = torch.topk(x, c["K"]).values[-1]
            sure, tied = torch.nonzero(x > kth)[:, 0], torch.nonzero(x == kth)[:, 0]
            at = torch.cat([sure[torch.sort(-x[sure], stable=True).indices], tied[:c["K"] - len(sure)]])
            left = torch.ones(V, dtype=torch.bool, device=DEVICE)
            left[at] = False
            out.append((x[at], at.int(), torch.logsumexp(x[left] / c["temperature"], 0)))
            continue
        T, at = c["temperature"], s["index"][r].long()
        teacher = s["value"][r].double() / T
        logq = torch.log_softmax(x / T, 0)
        inside = torch.zeros(V, dtype=torch.bool, device=DEVICE)
        inside[at] = True
        told = logq[at]
        if c["rest"]:
            teacher = torch.cat([teacher, s["rest"][r:r + 1].double()])
            told = torch.cat([told, torch.logsumexp(logq[~inside], 0)[None]])
        logp = torch.log_softmax(teacher, 0)
        p = logp.exp()
        some = p > 0
        loss = T * T * (p[some] * (logp[some] - told[some])).sum()
        if not c["grad"]:
            out.append((loss,))
            continue
        w = s["weight"][r].double()
        g = logq.exp()
        if c["rest"]:
            g[~inside] -= p[-1] * torch.softmax(logq[~inside], 0)
        g[at] -= p[:c["K"]]
        out.append((loss * (w != 0), w * T * g))
    cols = [torch.stack(col) for col in zip(*out)]
    return cols[0] if len(cols) == 1 else tuple(cols)


def _exact_row(x, u, how):
    n = len(x)
    T, k, p, m = how["temperature"], int(how["top_k"]), how["top_p"], how["min_p"]
    if T == 0:
        best = torch.nonzero(x == x.max())[0, 0]
        return best.repeat(len(u)), torch.zeros(len(u), dtype=torch.float64, device=DEVICE)
    w = torch.exp((x - x.max()) / T)
    # tokens by falling logit, of equal ones the lower token first
    order = torch.sort(-x, stable=True).indices
    if 0 < k < n:
        order = order[:k]
    if p < 1:
        upto = torch.cumsum(w[order], 0)
        order = order[:int((upto < p * upto[-1]).sum()) + 1]
    order = order[w[order] >= m]
    kept = torch.sort(order[w[order] > 0]).values
    upto = torch.cumsum(w[kept], 0)
    i = (upto[None, :] <= u[:, None] * upto[-1]).sum(1).clamp(max=len(kept) - 1)
    return kept[i], torch.log(w[kept[i]] / upto[-1])
