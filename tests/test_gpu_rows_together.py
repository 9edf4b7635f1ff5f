"""Draws, largest logits and distillation as they are used together: behind a verified step, on streams side by side, captured as one
graph, and along a small model's training."""
import math
import os
import sys

import pytest
import torch

import paper_2409_16560_b200 as dsbd
import rows_util as ru

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu
F32, I32 = torch.float32, torch.int32


def test_the_example_s_plain_draws_and_what_the_small_model_learns():
    """Tokens by the definition; the loss and its gradient by the small model's rows by the formula in 64 bits.  The bars are those of
    test_gpu_distill with a thousand logits within 30 octaves: sums and terms off by less than 2e-5."""
    import prompt_to_step as ex
    r = ex.run()
    assert r["status"] == 0
    zp, zq, fit = r["zp"].double().cpu(), r["zq"].double().cpu(), r["fit"]
    roots = r["roots"].cpu()
    for i, root in enumerate(roots.tolist()):
        how = {k: float(v[i]) for k, v in r["settings"].items()}
        for j in range(r["uniform"].shape[1]):
            t, lp = ru.draw(zp[root], float(r["uniform"][i, j]), how["temperature"], int(how["top_k"]), how["top_p"])
            assert int(r["plain"][i, j]) == t and abs(float(r["plain_logp"][i, j]) - lp) <= 2.0 ** -24 * abs(lp) + 1e-12
    for n in range(len(zp)):
        v, at, left = ru.top(zp[n], 16, 2.0)
        assert torch.equal(fit["index"][n].long().cpu(), at) and torch.equal(fit["value"][n].double().cpu(), v)
        assert abs(float(fit["rest"][n]) - float(left)) <= 2e-5 + 2.0 ** -24 * abs(float(left))
        x = zq[n].clone().requires_grad_()
        loss = ru.distill(x, fit["value"][n].double().cpu(), fit["index"][n].cpu(), fit["rest"][n].double().cpu(), 2.0)
        g, = torch.autograd.grad(loss, x)
        assert abs(float(fit["loss"][n]) - float(loss.detach())) <= 4 * 2e-5
        w = float(fit["weight"][n])
        assert float((fit["slope"][n].double().cpu() - w * g).abs().max()) <= w * 2 * 2e-5 * 2


def problem(seed, R=24, V=30011):
    z = ru.rows_of(R, V, F32, seed=seed).contiguous()
    student = (z + torch.randn(R, V, device="cuda", generator=torch.Generator("cuda").manual_seed(seed))).bfloat16()
    u = torch.rand(R, 5, device="cuda", generator=torch.Generator("cuda").manual_seed(seed + 1))
    T = torch.tensor([0.0, 0.7, 1.0, 1.4] * (R // 4), device="cuda")
    k = torch.tensor([0, 0, 30, 700, 5, 2000] * (R // 6), dtype=I32, device="cuda")
    p = torch.tensor([1.0, 0.9, 0.95] * (R // 3), device="cuda")
    return dict(z=z, student=student, u=u, how=dict(temperature=T, top_k=k, top_p=p))


def outputs(q):
    R, V = q["z"].shape
    e = lambda *s, dtype=F32: torch.zeros(*s, dtype=dtype, device="cuda")
    return dict(token=e(R, 5, dtype=I32), logp=e(R, 5), value=e(R, 40), index=e(R, 40, dtype=I32), rest=e(R), loss=e(R),
                grad=e(R, V, dtype=torch.bfloat16), status=e(1, dtype=I32))


def chain(q, o, stream=None):
    dsbd.sample_rows(q["z"], q["u"], token=o["token"], logp=o["logp"], status=o["status"], stream=stream, **q["how"])
    dsbd.top_logits(q["z"], 40, temperature=1.5, value=o["value"], index=o["index"], rest=o["rest"], status=o["status"], stream=stream)
    dsbd.distill(q["student"], o["value"], o["index"], rest=o["rest"], temperature=1.5, loss=o["loss"], grad=o["grad"], status=o["status"],
                 stream=stream)


def same(a, b):
    return all(torch.equal(a[n], b[n]) for n in a)


def test_two_streams_at_once():
    q = [problem(s) for s in (1, 2)]
    want = [outputs(x) for x in q]
    for x, o in zip(q, want):
        chain(x, o)
    torch.cuda.synchronize()
    assert int(want[0]["status"]) == 0
    streams = [torch.cuda.Stream() for _ in q]
    got = [outputs(x) for x in q]
    torch.cuda.synchronize()
    for _ in range(20):
        for x, o, s in zip(q, got, streams):
            chain(x, o, s)
    torch.cuda.synchronize()
    assert same(got[0], want[0]) and same(got[1], want[1])


def test_one_graph_of_the_chain_replayed_on_new_logits():
    q = problem(3)
    o = outputs(q)
    chain(q, o)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain(q, o)
    for seed in (4, 5):
        new = problem(seed)
        for name in ("z", "student", "u"):
            q[name].copy_(new[name])
        graph.replay()
        torch.cuda.synchronize()
        want = outputs(new)
        chain(new, want)
        torch.cuda.synchronize()
        assert same(o, want)


def test_a_call_behind_another_of_the_same_stream_sees_what_that_wrote():
    """Launches overlap at their ends: a chain of calls, each on the outputs of the one before, many times over."""
    q = problem(6)
    want = outputs(q)
    chain(q, want)
    torch.cuda.synchronize()
    for _ in range(50):
        o = outputs(q)
        z = q["z"] + 0.0                                       # written by a kernel just before
        for _ in range(3):
            chain(dict(q, z=z), o)
        torch.cuda.synchronize()
        assert same(o, want)


def test_a_step_of_training_through_the_loss():
    """Hidden states times an unembedding: the gradient by the weights against differences of the summed loss in 64 bits along a random
    direction; the calls' own losses move the same way."""
    g = torch.Generator("cuda").manual_seed(5)
    h = torch.randn(48, 64, device="cuda", generator=g)
    W = (0.3 * torch.randn(64, 5003, device="cuda", generator=g)).requires_grad_()
    teacher = (h @ (0.3 * torch.randn(64, 5003, device="cuda", generator=g)))
    value, index, rest, _ = dsbd.top_logits(teacher, 32)
    weight = torch.rand(48, device="cuda", generator=g) / 48
    logits = h @ W
    loss, slope, status = dsbd.distill(logits, value, index, rest=rest, weight=weight)
    logits.backward(slope)
    assert int(status) == 0
    d = torch.randn(64, 5003, device="cuda", generator=g)
    d /= d.norm()

    def total(eps):
        x = (h.double() @ (W.detach().double() + eps * d.double())).cpu()
        return sum(float(weight[r]) * float(ru.distill(x[r], value[r].double().cpu(), index[r].cpu(), rest[r].double().cpu(), 1.0))
                   for r in range(48))
    step = 1e-3
    slope64 = (total(step) - total(-step)) / (2 * step)
    along = float((W.grad.double() * d.double()).sum())
    # fp32 products of 64 and 48 terms and the gradient's 2e-5 of each share; the differences' third derivative times step^2
    assert abs(along - slope64) <= 1e-4 * float(W.grad.norm()) + 1e-5 and math.isfinite(along)
