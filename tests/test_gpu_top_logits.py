"""The largest logits of rows and what the rest amounts to, against the definition in 64 bits."""
import itertools
import math

import pytest
import torch

import paper_2409_16560_b200 as dsbd
import rows_util as ru

pytestmark = pytest.mark.gpu
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def rest_bar(x, K, T, rest):
    """Half a step of the result, and of the sum: each term 2^-22 by the exponential and three roundings of its argument (a octaves below the
    smallest kept logit: a ln 2 * 3 * 2^-24, over the terms on average), a thread's up to 256 terms added in 32 bits."""
    down = x.sort(descending=True).values
    a = (down[K - 1] - down[K:]) / (T * ru.LN2)
    w = torch.exp2(-a)
    mean = float((w * a.clamp(max=1e4)).sum() / w.sum()) if float(w.sum()) else 0.0
    return 2.0 ** -24 * abs(rest) + 2.0 ** -22 + 3 * 2.0 ** -24 * ru.LN2 * mean + 256 * 2.0 ** -24


def check(z, K, T=1.0, expect=0):
    value, index, rest, status = dsbd.top_logits(z, K, temperature=T)
    assert int(status) == expect
    assert value.dtype == F32 and index.dtype == I32 and value.shape == index.shape == (z.shape[0], K) and rest.shape == (z.shape[0],)
    T = float(torch.tensor(T, dtype=F32))
    x = z.double().cpu()
    for r in range(z.shape[0]):
        v, at, left = ru.top(x[r], K, T)
        assert torch.equal(index[r].long().cpu(), at), r
        assert torch.equal(value[r].double().cpu(), v), r
        got, left = float(rest[r]), float(left)
        if math.isinf(left):
            assert got == left
        else:
            assert abs(got - left) <= rest_bar(x[r], K, T, left), r


SIZES = [1, 2, 5, 16, 33, 1000, 4099, 32000, 50257, 128256]


@pytest.mark.parametrize("V,dtype", list(itertools.product(SIZES, [F32, BF])))
def test_every_size(V, dtype):
    z = ru.rows_of(4, V, dtype, seed=V, pad=V % 7, start=V % 5)
    for K in sorted({1, 2, 16, 100, 511, 1024, V - 1, V}):
        if 1 <= K <= min(V, 1024):
            check(z, K, 0.9)


@pytest.mark.parametrize("T", [0.01, 0.5, 1.0, 4.0, 1e3])
def test_temperatures(T):
    check(ru.rows_of(3, 20000, F32, seed=2), 64, T)


@pytest.mark.parametrize("T", [2.0 ** -126, 1e-30, 1e20, 2.0 ** 100])
def test_temperatures_of_every_size(T):
    """Ordinary logits where T is large, with a mask of the type's lowest value, and logits of T's size."""
    z = ru.rows_of(4, 5000, F32, seed=4)
    z[2:] = (z[2:].double() * T).float()
    z[1, ::2] = torch.finfo(F32).min
    check(z if T > 1 else z[2:], 20, T)


@pytest.mark.parametrize("V,dtype", [(262144, F32), (393216, F32), (786432, BF)])
def test_long_rows(V, dtype):
    check(ru.rows_of(2, V, dtype, seed=V, start=3), 200)


@pytest.mark.parametrize("levels", [1, 2, 40])
@pytest.mark.parametrize("V", [9, 3000, 60000])
def test_equal_logits_go_by_token(V, levels):
    """More equal logits than the list holds, at either side of the cut."""
    z = torch.randint(0, levels, (3, V), generator=torch.Generator().manual_seed(V)).float().cuda()
    for K in (1, 5, 700, 1024):
        if K <= V:
            check(z, K)
            check(z.to(BF), K)


@pytest.mark.parametrize("left", [1, 3, 200, 2000])
def test_masked_rows(left):
    """Where the mask leaves fewer than K tokens, the first masked ones follow and nothing is left over."""
    V = 20000
    z = ru.rows_of(3, V, F32, seed=left)
    for r in range(3):
        keep = torch.randperm(V, generator=torch.Generator().manual_seed(r))[:left].cuda()
        x = z[r, keep].clone()
        z[r] = -math.inf
        z[r, keep] = x
    for K in (1, 2, 64, 300, 1000):
        check(z, K)


def test_extreme_logits():
    """Ranges over the whole of fp32, the type's lowest value, denormals and zeros of both signs; a rest 200 below the kept logits."""
    g = torch.Generator().manual_seed(1)
    x = torch.randn(6, 7000, generator=g)
    x[0] *= 1e38
    x[1] *= 1e-42
    x[2, 10:] = torch.finfo(F32).min
    x[3, ::2], x[3, 1::2] = 0.0, -0.0
    x[4, :30] += 200
    x[5] *= 1e5
    assert bool((x[0] == math.inf).any())                      # 3.4 standard deviations are beyond fp32: such a row has no result
    assert int(dsbd.top_logits(x[:1].cuda(), 5)[3]) == 8
    x[0].clamp_(-torch.finfo(F32).max, torch.finfo(F32).max)
    for K in (1, 12, 30, 600):
        check(x.cuda(), K)


def test_rows_without_a_result():
    for bad, code in [(math.nan, 8), (math.inf, 8), (-math.inf, 2)]:
        z = ru.rows_of(4, 5000, F32, seed=1)
        want = dsbd.top_logits(z, 20)
        z[1] = bad if bad == -math.inf else z[1]
        z[1, 33] = bad
        value, index, rest, status = dsbd.top_logits(z, 20)
        assert int(status) == code and bool(value[1].isnan().all()) and bool((index[1] == -1).all()) and math.isnan(float(rest[1]))
        rows = [0, 2, 3]
        assert all(torch.equal(a[rows], b[rows]) for a, b in zip((value, index, rest), want))


def test_outputs_of_the_caller_a_graph_and_another_stream():
    z = ru.rows_of(8, 32000, BF, seed=1).contiguous()
    out = dict(value=torch.zeros(8, 50, device="cuda"), index=torch.zeros(8, 50, dtype=I32, device="cuda"), rest=torch.zeros(8, device="cuda"),
               status=torch.zeros(1, dtype=I32, device="cuda"))
    dsbd.top_logits(z, 50, **out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dsbd.top_logits(z, 50, **out)
    z.copy_(ru.rows_of(8, 32000, BF, seed=2))
    graph.replay()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    torch.cuda._sleep(50_000_000)
    want = dsbd.top_logits(z, 50, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(out[n], w) for n, w in zip(("value", "index", "rest"), want))


def test_the_same_call_gives_the_same_bits():
    z = ru.rows_of(100, 50257, BF, seed=3)
    first = dsbd.top_logits(z, 128)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first[:3], dsbd.top_logits(z, 128)))


def test_what_is_refused():
    z = torch.zeros(3, 50, device="cuda")
    for bad in (dict(K=0), dict(K=51), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=math.inf), dict(temperature=math.nan)):
        with pytest.raises(dsbd.DsbdError, match="invalid argument"):
            dsbd.top_logits(**dict(dict(logits=z, K=5), **bad))
    with pytest.raises(dsbd.DsbdError, match="unsupported"):
        dsbd.top_logits(torch.zeros(1, 5000, device="cuda"), 1025)
    for bad in (dict(logits=z.half()), dict(logits=z.cpu()), dict(logits=z.t()), dict(value=torch.zeros(3, 4, device="cuda")),
                dict(index=torch.zeros(3, 5, dtype=torch.int64, device="cuda")), dict(rest=torch.zeros(3, 1, device="cuda")),
                dict(status=torch.zeros(1, device="cuda"))):
        with pytest.raises((AssertionError, RuntimeError)):
            dsbd.top_logits(**dict(dict(logits=z, K=5), **bad))
    assert dsbd.top_logits(z[:0], 5)[0].shape == (0, 5)
