"""Distillation of rows from a teacher's entries: losses and gradients against the formula in 64 bits (its gradient by autograd) and against
differences of losses."""
import itertools
import math

import pytest
import torch

import paper_2409_16560_b200 as dsbd
import rows_util as ru

pytestmark = pytest.mark.gpu
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def problem(R, V, K, dtype, seed, rest=True, weight=True, pad=0, start=0, noise=1.0):
    """A student's rows near a teacher's, the teacher's entries and what is left of it (at temperature 1), weights of which one is 0."""
    teacher = ru.rows_of(R, V, F32, seed).double().cpu()
    g = torch.Generator().manual_seed(seed + 1)
    z = ru.rows_of(R, V, dtype, seed, pad=pad, start=start)
    z.copy_((teacher + noise * torch.randn(R, V, generator=g)).float())
    value, index, left = zip(*[ru.top(teacher[r], K, 1.0) for r in range(R)])
    w = torch.rand(R, generator=g) + 0.1
    w[R // 2] = 0.0 if R > 1 else w[0]
    return dict(z=z, value=torch.stack(value).float().cuda(), index=torch.stack(index).int().cuda(),
                rest=torch.stack(left).float().cuda() if rest else None, weight=w.cuda() if weight else None)


def check(q, T=1.0, expect=0, grad=True):
    """The bar.  A term of the student's sums: 2^-22 by the exponential, three roundings of its argument (a octaves below the reference:
    a ln 2 * 3 * 2^-24), a thread's up to 256 terms added in 32 bits: `part`, of every q.  Loss: T^2 sum p |d log q| <= T^2 part, and half
    a step.  Gradient: part of w T q (and once more for its own term; of w T p for the others, which p_rest is shared out to), the factor's
    rounding and the product's, and half a step of its type."""
    z = q["z"]
    loss, g, status = dsbd.distill(z, q["value"], q["index"], rest=q["rest"], weight=q["weight"], temperature=T, grad=grad or None)
    assert int(status) == expect
    T = float(torch.tensor(T, dtype=F32))
    x = z.double().cpu()
    value, index = q["value"].double().cpu(), q["index"].cpu()
    half = torch.finfo(z.dtype).eps / 2
    for r in range(z.shape[0]):
        w = 1.0 if q["weight"] is None else float(q["weight"][r])
        if w == 0:
            assert float(loss[r]) == 0 and (g is None or bool((g[r] == 0).all()))
            continue
        xr = x[r].clone().requires_grad_()
        want = ru.distill(xr, value[r], index[r], None if q["rest"] is None else q["rest"][r].double().cpu(), T)
        a = ((xr.max() - xr) / (T * ru.LN2)).detach().clamp(max=150.0)
        prob = torch.softmax(xr.detach() / T, 0)
        part = 2.0 ** -22 + 3 * 2.0 ** -24 * ru.LN2 * float((prob * a).sum()) + 256 * 2.0 ** -24
        want_loss = float(want.detach())
        if math.isinf(want_loss):
            assert float(loss[r]) == want_loss
        else:
            assert abs(float(loss[r]) - want_loss) <= T * T * part + 2.0 ** -24 * abs(want_loss), (r, float(loss[r]), want_loss)
        if g is None:
            continue
        ref, = torch.autograd.grad(want, xr)
        named = torch.zeros(len(xr), dtype=torch.bool)
        named[index[r][index[r] >= 0].long()] = True
        share = prob.clone()
        if q["rest"] is not None and bool((~named).any()):
            # what p_rest gives to a token that is not named
            share[~named] += (T * prob[~named] - ref[~named]).abs() / T
        own = part + 2.0 ** -22 + 3 * 2.0 ** -24 * (1 + ru.LN2 * a)
        bar = w * T * own * share + half * w * ref.abs() + 1e-37
        err = (g[r].double().cpu() - w * ref).abs()
        assert bool((err <= bar).all()), (r, float((err / bar).max()))
    return loss, g


CASES = [(1, 1), (2, 1), (2, 2), (7, 3), (16, 16), (100, 16), (1000, 200), (4099, 1024), (32000, 64), (50257, 16), (128256, 128)]


@pytest.mark.parametrize("size,dtype,rest", list(itertools.product(CASES, [F32, BF], [True, False])))
def test_every_size(size, dtype, rest):
    V, K = size
    check(problem(4, V, K, dtype, seed=V, rest=rest, pad=V % 3, start=V % 5))


@pytest.mark.parametrize("T", [0.5, 2.0, 10.0])
@pytest.mark.parametrize("rest", [True, False])
def test_temperatures(T, rest):
    q = problem(3, 9000, 50, F32, seed=3, rest=rest)
    if rest:
        teacher = ru.rows_of(3, 9000, F32, 3).double().cpu()
        q["rest"] = torch.stack([ru.top(teacher[r], 50, T)[2] for r in range(3)]).float().cuda()
    check(q, T)
    check(q, T, grad=False)


@pytest.mark.parametrize("T", [2.0 ** -40, 2.0 ** 40])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_logits_of_the_temperature_s_size(T, dtype):
    """Powers of two scale everything but the rest: p and q are those of a temperature of 1, the loss T^2 and the gradient T times theirs."""
    q = problem(3, 9000, 50, dtype, seed=6)
    loss, g = check(q)
    scaled = dsbd.distill(q["z"] * T, q["value"] * T, q["index"], rest=q["rest"], weight=q["weight"], temperature=T)
    assert torch.equal(scaled[0], loss * T * T) and torch.equal(scaled[1], g * T)


@pytest.mark.parametrize("V,dtype", [(262144, F32), (393216, F32), (786432, BF)])
def test_long_rows(V, dtype):
    check(problem(2, V, 100, dtype, seed=V, start=1))


def test_the_gradient_is_the_losses_difference():
    """Central differences of the kernel's own losses: off by the losses' rounding over the step and by its square times a third
    derivative, at most T^2 / T^3 * 1 here."""
    for rest in (True, False):
        q = problem(1, 40, 6, F32, seed=9, rest=rest, weight=False)
        for T in (1.0, 2.0):
            loss, g, _ = dsbd.distill(q["z"], q["value"], q["index"], rest=q["rest"], temperature=T)
            h = 2.0 ** -5
            z = q["z"].repeat(80, 1)
            z[torch.arange(40), torch.arange(40)] += h
            z[torch.arange(40, 80), torch.arange(40)] -= h
            up = lambda t: None if t is None else t.repeat_interleave(80, 0)
            l = dsbd.distill(z, up(q["value"]), up(q["index"]), rest=up(q["rest"]), temperature=T, grad=None)[0].double()
            step = (z[:40].diagonal().double() - z[40:].diagonal().double())
            d = (l[:40] - l[40:]) / step
            bar = 2 * (2.0 ** -20 * T * T + 2.0 ** -24 * float(l.max())) / (2 * h) + h * h / T
            assert float((d - g[0].double()).abs().max()) <= bar


def test_a_student_far_from_its_teacher():
    """One token with all of the student's mass, named or not: the others' share is e^-200, and the loss and the gradient see it."""
    for named in (True, False):
        q = problem(2, 6000, 20, F32, seed=5, weight=False)
        for r in range(2):
            inside = set(q["index"][r].tolist())
            t = int(q["index"][r, 3]) if named else next(t for t in range(6000) if t not in inside)
            q["z"][r, t] = 200.0
        loss, _ = check(q)
        assert bool((loss > 50).all())


def test_masked_students():
    """-inf logits: no gradient there; where the teacher has mass there, an infinite loss; named by an entry without mass, nothing."""
    q = problem(3, 5000, 30, F32, seed=6, weight=False)
    outside = torch.ones(5000, dtype=torch.bool)
    outside[q["index"].long().cpu().flatten()] = False
    q["z"][:, outside.nonzero()[::2, 0].cuda()] = -math.inf
    check(q)
    q["z"][1, int(q["index"][1, 0])] = -math.inf
    loss, g, _ = dsbd.distill(q["z"], q["value"], q["index"], rest=q["rest"])
    assert float(loss[1]) == math.inf and bool(g.isfinite().all())
    q["value"][1, 0] = -math.inf
    loss, g, status = dsbd.distill(q["z"], q["value"], q["index"], rest=q["rest"])
    assert bool(loss.isfinite().all()) and float(g[1, int(q["index"][1, 0])]) == 0 and int(status) == 0


def test_entries_that_are_not_there():
    """Rows of fewer entries than K: index -1 with any value."""
    q = problem(4, 3000, 20, F32, seed=7)
    q["index"][0, 5:] = -1
    q["value"][0, 5:] = math.nan
    q["index"][1, ::2] = -1
    q["value"][3, 7] = -math.inf
    check(q)
    q["rest"] = None
    check(q)


def test_the_same_token_twice():
    """Outcomes that share a token: the gradient has both."""
    for rest in (True, False):
        q = problem(3, 2000, 700, F32, seed=8, rest=rest, weight=False)
        q["index"][0, 9] = q["index"][0, 2]
        q["index"][1, [3, 100, 650]] = int(q["index"][1, 600])
        q["index"][2] = q["index"][2, 0].clone()
        first = check(q)
        again = dsbd.distill(q["z"], q["value"], q["index"], rest=q["rest"])
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_indices_out_of_range_are_left_out():
    q = problem(3, 3000, 20, F32, seed=7, weight=False)
    q["index"][1, 4], q["index"][2, 0] = 3000, -2
    got = dsbd.distill(q["z"], q["value"], q["index"], rest=q["rest"])
    assert int(got[2]) == 1
    q["index"][1, 4], q["index"][2, 0] = -1, -1
    want = check(q)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_rows_without_anything():
    """Nothing but -inf in a student's row, in a teacher's, no entries: no loss, no gradient, and a report."""
    for rest in (True, False):
        for what in ("student", "teacher", "entries"):
            q = problem(4, 2500, 9, F32, seed=2, rest=rest, weight=False)
            want = dsbd.distill(q["z"], q["value"], q["index"], rest=q["rest"])
            if what == "student":
                q["z"][2] = -math.inf
            else:
                if what == "teacher":
                    q["value"][2] = -math.inf
                else:
                    q["index"][2] = -1
                if rest:
                    q["rest"][2] = -math.inf
            loss, g, status = dsbd.distill(q["z"], q["value"], q["index"], rest=q["rest"])
            assert int(status) == 2 and float(loss[2]) == 0 and bool((g[2] == 0).all())
            rows = [0, 1, 3]
            assert torch.equal(loss[rows], want[0][rows]) and torch.equal(g[rows], want[1][rows])


def test_rest_alone_and_all_tokens_named():
    q = problem(2, 600, 4, F32, seed=2, weight=False)
    q["index"][0] = -1
    check(q)
    q = problem(3, 50, 50, F32, seed=2, weight=False)          # no other tokens: rest is -inf
    assert bool((q["rest"] == -math.inf).all())
    check(q)
    q["rest"][1] = 0.0                                         # a teacher with mass where the student can have none
    loss, g, status = dsbd.distill(q["z"], q["value"], q["index"], rest=q["rest"])
    assert float(loss[1]) == math.inf and bool(g.isfinite().all()) and int(status) == 0


def test_nan_goes_through_and_rows_of_weight_zero_are_not_read():
    q = problem(4, 3001, 12, F32, seed=4)
    q["weight"][:] = torch.tensor([1.0, 0.0, 1.0, 1.0])
    q["z"][1], q["value"][1], q["index"][1], q["rest"][1] = math.nan, math.nan, -7, math.nan
    loss, g, status = dsbd.distill(q["z"], q["value"], q["index"], rest=q["rest"], weight=q["weight"])
    assert int(status) == 0 and float(loss[1]) == 0 and bool((g[1] == 0).all())
    q["z"][2, 100] = math.nan
    q["value"][3, 2] = math.nan
    loss, g, status = dsbd.distill(q["z"], q["value"], q["index"], rest=q["rest"], weight=q["weight"])
    assert bool(loss[2:].isnan().all()) and bool(loss[:2].isfinite().all())
    assert bool(g[2].isnan().all()) and bool(g[:2].isfinite().all()) and bool(g[3].isnan().any())
    q["z"][2] = math.nan
    assert bool(dsbd.distill(q["z"], q["value"], q["index"], rest=q["rest"])[0][2].isnan())


@pytest.mark.parametrize("dtype", [F32, BF])
def test_in_place_and_into_rows_of_another_alignment(dtype):
    q = problem(5, 50257, 16, dtype, seed=5, pad=2, start=1)
    loss, g, _ = dsbd.distill(q["z"], q["value"], q["index"], rest=q["rest"], weight=q["weight"])
    for pad, start in [(0, 0), (1, 0), (5, 3), (2, 1)]:
        to = ru.rows_of(5, 50257, dtype, 1, pad=pad, start=start)
        around = to._base
        to.fill_(1.0)
        whole = around.isnan()
        got = dsbd.distill(q["z"], q["value"], q["index"], rest=q["rest"], weight=q["weight"], grad=to)
        assert got[1] is to and torch.equal(to, g) and torch.equal(got[0], loss)
        assert torch.equal(around.isnan(), whole)              # nothing between the rows is written
    around, whole = q["z"]._base, q["z"]._base.isnan()
    got = dsbd.distill(q["z"], q["value"], q["index"], rest=q["rest"], weight=q["weight"], grad=q["z"])
    assert torch.equal(q["z"], g) and torch.equal(got[0], loss) and torch.equal(around.isnan(), whole)


def test_the_gradient_goes_on_to_what_made_the_logits():
    """loss, grad = distill(logits); logits.backward(grad): against the formula through autograd, for a small projection in 64 bits."""
    g = torch.Generator().manual_seed(1)
    h, W = torch.randn(6, 32, generator=g), torch.randn(32, 500, generator=g) * 0.2
    q = problem(6, 500, 10, F32, seed=3)
    Wd = W.cuda().requires_grad_()
    logits = h.cuda() @ Wd
    loss, grad, _ = dsbd.distill(logits, q["value"], q["index"], rest=q["rest"], weight=q["weight"])
    logits.backward(grad)
    W64 = W.double().requires_grad_()
    rows = h.double() @ W64
    sum(float(q["weight"][r]) * ru.distill(rows[r], q["value"][r].double().cpu(), q["index"][r].cpu(), q["rest"][r].double().cpu(), 1.0)
        for r in range(6)).backward()
    # products in 32 bits of 32 and 6 terms, and what the logits' rounding moves
    assert float((Wd.grad.double().cpu() - W64.grad).abs().max()) <= 1e-5 * float(W64.grad.abs().max()) * 6


def test_the_same_call_gives_the_same_bits_and_a_graph_s_replay_new_ones():
    q = problem(64, 32000, 64, BF, seed=3)
    call = lambda **kw: dsbd.distill(q["z"], q["value"], q["index"], rest=q["rest"], weight=q["weight"], **kw)
    first = call()
    for _ in range(5):
        again = call()
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    out = dict(loss=torch.zeros(64, device="cuda"), grad=torch.zeros(64, 32000, dtype=BF, device="cuda"),
               status=torch.zeros(1, dtype=I32, device="cuda"))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call(**out)
    q["z"].copy_(ru.rows_of(64, 32000, BF, seed=9))
    graph.replay()
    torch.cuda.synchronize()
    want = call(stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    assert torch.equal(out["loss"], want[0]) and torch.equal(out["grad"], want[1]) and not torch.equal(want[0], first[0])


def test_what_is_refused():
    q = problem(3, 50, 5, F32, seed=1)
    base = dict(logits=q["z"], value=q["value"], index=q["index"], rest=q["rest"], weight=q["weight"])
    for bad in (dict(temperature=0.0), dict(temperature=math.nan), dict(temperature=math.inf)):
        with pytest.raises(dsbd.DsbdError, match="invalid argument"):
            dsbd.distill(**dict(base, **bad))
    with pytest.raises(dsbd.DsbdError, match="invalid argument"):
        dsbd.distill(**dict(base, value=torch.zeros(3, 51, device="cuda"), index=torch.zeros(3, 51, dtype=I32, device="cuda")))
    with pytest.raises(dsbd.DsbdError, match="unsupported"):
        z = torch.zeros(1, 5000, device="cuda")
        dsbd.distill(z, torch.zeros(1, 1025, device="cuda"), torch.zeros(1, 1025, dtype=I32, device="cuda"))
    cuda = lambda *s, **kw: torch.zeros(*s, device="cuda", **kw)
    for bad in (dict(logits=q["z"].half()), dict(logits=q["z"].cpu()), dict(value=q["value"].double()), dict(value=q["value"][:2]),
                dict(index=q["index"].long()), dict(index=q["index"][:, :4]), dict(rest=cuda(2)), dict(rest=cuda(3, 1)), dict(weight=cuda(3, dtype=BF)),
                dict(weight=q["weight"].cpu()), dict(loss=cuda(4)), dict(grad=cuda(3, 49)), dict(grad=cuda(3, 50, dtype=BF)),
                dict(grad=cuda(50, 3).t()), dict(status=cuda(1)), dict(value=q["value"].t().contiguous().t())):
        with pytest.raises((AssertionError, RuntimeError)):
            dsbd.distill(**dict(base, **bad))
    assert dsbd.distill(q["z"][:0], q["value"][:0], q["index"][:0])[0].shape == (0,)
