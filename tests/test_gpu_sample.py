"""Draws from rows with each row's own settings, against the definition in 64 bits.  Tokens are equal: both sides' sums are in 64 bits, so a
uniform number would have to lie within 1e-13 of a cell's edge."""
import itertools
import math

import pytest
import torch

import paper_2409_16560_b200 as dsbd
import rows_util as ru

pytestmark = pytest.mark.gpu
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def check(z, u, T=1.0, k=0, p=1.0, m=0.0, expect=0):
    """Every draw of every row; settings are numbers or lists of the rows' own.  logp is fp32 of a sum in 64 bits: half a step."""
    R = z.shape[0]
    own = lambda x, dtype: torch.tensor(x, dtype=dtype, device="cuda") if isinstance(x, list) else x
    u = u.cuda()
    token, logp, status = dsbd.sample_rows(z, u, temperature=own(T, F32), top_k=own(k, I32), top_p=own(p, F32), min_p=own(m, F32))
    assert int(status) == expect
    f32 = lambda x, r: float(torch.tensor(x[r] if isinstance(x, list) else x, dtype=F32))
    x, uu = z.double().cpu(), u.double().cpu()
    got, got_p = token.cpu(), logp.double().cpu()
    for r in range(R):
        for j in range(u.shape[1]):
            t, lp = ru.draw(x[r], float(uu[r, j]), f32(T, r), int(f32(k, r)), f32(p, r), f32(m, r))
            assert int(got[r, j]) == t, (r, j)
            assert abs(float(got_p[r, j]) - lp) <= 2.0 ** -24 * abs(lp) + 1e-12, (r, j)
    return token, logp


def uniform(R, n, seed):
    u = torch.rand(R, n, generator=torch.Generator().manual_seed(seed))
    u[0, 0] = 0.0
    u[-1, -1] = 1.0
    return u


SIZES = [1, 2, 3, 7, 16, 31, 100, 1000, 4099, 8192, 32000, 50257, 128256]


@pytest.mark.parametrize("V,dtype", list(itertools.product(SIZES, [F32, BF])))
def test_settings_at_every_size(V, dtype):
    z = ru.rows_of(6, V, dtype, seed=V, pad=V % 5, start=V % 3)
    u = uniform(6, 3, V + 1)
    for T, k, p, m in [(1.0, 0, 1.0, 0.0), (0.7, 0, 0.9, 0.0), (1.3, 10, 0.8, 0.0), (1.0, 50, 1.0, 0.05), (0.8, 0, 1.0, 0.02),
                       (0.0, 5, 0.5, 0.0), (2.0, V, 0.3, 0.0), (1.0, 1, 1.0, 0.0)]:
        check(z, u, T, k, p, m)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_rows_settings_of_their_own(dtype):
    z = ru.rows_of(40, 20011, dtype, seed=1, pad=3)
    g = torch.Generator().manual_seed(2)
    pick = lambda xs: [xs[i] for i in torch.randint(0, len(xs), (40,), generator=g).tolist()]
    check(z, uniform(40, 4, 3), pick([0.0, 0.5, 0.9, 1.0, 1.7, 30.0]), pick([-1, 0, 1, 3, 40, 900, 1024, 1025, 5000, 30000]),
          pick([1.0, 2.0, 0.9, 0.5, 0.05]), pick([0.0, 0.0, 0.01, 0.3, 1.0]))


@pytest.mark.parametrize("k", [1, 2, 31, 32, 33, 511, 512, 513, 1023, 1024, 1025, 2047, 5000, 50000])
@pytest.mark.parametrize("V,dtype", [(50257, F32), (50257, BF), (128256, F32)])
def test_top_k_of_any_size(V, dtype, k):
    z = ru.rows_of(2, V, dtype, seed=k)
    check(z, uniform(2, 5, k), 1.5, k, 1.0)
    check(z, uniform(2, 5, k), 3.0, k, 0.93)


@pytest.mark.parametrize("p", [1e-30, 1e-6, 0.1, 0.5, 0.95, 0.999, 0.999999, 1 - 2.0 ** -24])
@pytest.mark.parametrize("dtype,T", [(F32, 1.0), (BF, 1.0), (F32, 8.0), (F32, 0.05)])
def test_top_p_of_any_size(dtype, T, p):
    z = ru.rows_of(3, 30011, dtype, seed=7)
    check(z, uniform(3, 8, 8), T, 0, p)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("V", [20000, 50257, 151936])
@pytest.mark.parametrize("spread", [0.05, 0.5, 3.0])
def test_prefixes_longer_than_a_list(V, dtype, spread):
    """Flat rows, whose top-p and min-p keep thousands of tokens, among ties (bf16) and without (fp32)."""
    z = ru.rows_of(3, V, dtype, seed=V + 1, pad=5, start=3, spread=spread, zipf=False)
    u = uniform(3, 6, V)
    for T, p, m in [(1.0, 0.5, 0.0), (1.0, 0.9, 0.0), (2.5, 0.97, 0.0), (8.0, 0.3, 0.0), (1.0, 0.9, 0.2), (3.0, 0.999, 0.7), (0.5, 0.8, 1e-3)]:
        check(z, u, T, 0, p, m)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("k,p,m", [(600, 1.0, 0.0), (1000, 0.9, 0.0), (1500, 0.95, 0.0), (2500, 1.0, 0.01), (0, 0.9, 0.0), (0, 0.99, 0.3), (0, 1.0, 0.05)])
def test_many_short_rows(dtype, k, p, m):
    """Rows of one CTA each, with fewer threads than a top-k has tokens, some of them masked to less than that."""
    z = ru.rows_of(160, 9001, dtype, seed=k + 3, pad=2, zipf=False)
    z[::7, 300:] = -math.inf
    z[1::7, 1::2] = -math.inf
    check(z, uniform(160, 2, 4), 1.2, k, p, m)


@pytest.mark.parametrize("T", [1e36, 3e37, 1e38])
def test_temperatures_of_the_largest_logits_size(T):
    z = ru.rows_of(4, 9000, F32, seed=8, spread=1.0)
    z[1] *= 1e37
    z[2] = z[2] * 1e37 - 3e38
    z[3, ::3] = torch.finfo(F32).min
    z = z.clamp(torch.finfo(F32).min)
    for k, p, m in [(0, 1.0, 0.0), (20, 0.9, 0.0), (0, 0.9, 0.0), (0, 0.3, 0.9), (2000, 0.9, 0.1)]:
        check(z, uniform(4, 5, 6), T, k, p, m)


@pytest.mark.parametrize("T", [1e-30, 1e-36, 1e-38, 1e-40])
def test_temperatures_that_leave_no_scale(T):
    """Differences of the logits over the temperature: beyond fp32, or of ordinary size where the logits are as small."""
    z = ru.rows_of(4, 9000, F32, seed=5)
    z[2:] = (z[2:].double() * T).float()
    for k, p, m in [(0, 1.0, 0.0), (20, 0.9, 0.0), (0, 0.9, 0.0), (2000, 0.9, 0.1)]:
        check(z, uniform(4, 5, 6), T, k, p, m)


@pytest.mark.parametrize("V", [5, 700, 3000, 40000, 128256])
@pytest.mark.parametrize("levels", [1, 2, 3])
def test_equal_logits_go_by_token(V, levels):
    """Rows of one, two and three different logits: cuts lie inside long ties, and a top-p of 0.5 of equal masses exactly between two."""
    g = torch.Generator().manual_seed(V)
    z = (torch.randint(0, levels, (4, V), generator=g).float() - 1.0).cuda()
    u = uniform(4, 4, V)
    for k, p in [(0, 0.5), (0, 0.25), (0, 0.7), (3, 1.0), (V // 2, 1.0), (V - 1, 0.5), (2000, 0.5), (0, 1.0), (0, 1e-5)]:
        check(z, u, 1.0, k, p)


def test_zeros_of_both_signs_are_equal():
    z = torch.zeros(1, 4000)
    z[0, ::2] = -0.0
    for k, p in [(3, 1.0), (0, 0.25), (0, 1.0), (1500, 1.0)]:
        check(z.cuda(), uniform(1, 6, 5), 1.0, k, p)
    assert int(dsbd.sample_rows(z.cuda(), torch.zeros(1, 1, device="cuda"), temperature=0.0)[0]) == 0


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("left", [1, 2, 30, 700, 3000])
def test_masked_rows(dtype, left):
    """Rows of which a mask leaves a few tokens: settings that would keep more keep these."""
    V = 33000
    z = ru.rows_of(3, V, dtype, seed=left)
    for r in range(3):
        keep = torch.randperm(V, generator=torch.Generator().manual_seed(r))[:left].cuda()
        x = z[r, keep].clone()
        z[r] = -math.inf
        z[r, keep] = x
    for T, k, p, m in [(1.0, 0, 1.0, 0.0), (1.0, 10, 1.0, 0.0), (1.0, 1024, 0.9, 0.0), (1.0, 5000, 1.0, 0.0), (1.0, 5000, 0.8, 0.0),
                       (2.0, 0, 0.99, 0.1), (0.0, 0, 1.0, 0.0)]:
        check(z, uniform(3, 4, left), T, k, p, m)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_masks_of_the_type_s_lowest_value(dtype):
    """A mask of finite numbers is a logit like others: without mass beside one of 0, all of the mass where there is nothing else."""
    low = torch.finfo(dtype).min
    z = torch.full((3, 9000), low, dtype=dtype)
    z[0, 77] = 0.0
    z[1, [5, 8000]] = torch.tensor([1.0, 2.0], dtype=dtype)
    for k, p in [(0, 1.0), (0, 0.9), (4, 1.0), (2000, 0.9)]:
        check(z.cuda(), uniform(3, 5, 1), 1.0, k, p)


def test_wide_and_narrow_ranges_of_logits():
    V = 12000
    g = torch.Generator().manual_seed(3)
    x = torch.randn(5, V, generator=g)
    z = torch.stack([x[0] * 1e38 * 2, x[1] * 1e-38, x[2] * 1e-44, x[3] * 1e5, 1e6 + x[4]]).clamp(-3.4e38, 3.4e38).cuda()
    for T, k, p in [(1.0, 0, 1.0), (1.0, 20, 0.9), (1.0, 0, 0.9), (1.0, 3000, 1.0), (1e38, 0, 0.8), (1e-3, 0, 0.99), (1e4, 700, 0.5)]:
        check(z, uniform(5, 4, 9), T, k, p)


@pytest.mark.parametrize("V,dtype", [(151936, F32), (151936, BF), (262144, F32), (393216, F32), (786432, BF)])
def test_long_rows(V, dtype):
    z = ru.rows_of(2, V, dtype, seed=V, start=1)
    for T, k, p in [(1.0, 0, 1.0), (1.0, 0, 0.9), (1.0, 40, 0.9), (1.0, 20000, 1.0)]:
        check(z, uniform(2, 3, 4), T, k, p)


def test_many_draws_and_one():
    z = ru.rows_of(2, 5000, F32, seed=5)
    for k in (0, 100):
        check(z, uniform(2, 700, 6), 1.0, k, 0.9)
    u = torch.rand(2, device="cuda")
    token, logp, _ = dsbd.sample_rows(z, u)
    again = dsbd.sample_rows(z, u[:, None])
    assert token.shape == logp.shape == (2,) and torch.equal(token[:, None], again[0]) and torch.equal(logp[:, None], again[1])


def test_the_share_of_draws_is_the_probability():
    """A row's draws at the centres of 4096 equal strips: each token's count is within one of 4096 times its probability."""
    z = ru.rows_of(1, 300, F32, seed=8)
    u = ((torch.arange(4096) + 0.5) / 4096)[None].cuda()
    token, _, _ = dsbd.sample_rows(z, u, temperature=0.9)
    n = torch.bincount(token[0].long(), minlength=300).double().cpu()
    want = torch.softmax(z[0].double().cpu() / float(torch.tensor(0.9)), 0) * 4096
    assert float((n - want).abs().max()) < 1.0 + 1e-6


@pytest.mark.parametrize("dtype", [F32, BF])
def test_rows_without_a_result(dtype):
    """NaN, +inf, nothing but -inf: token -1, logp NaN and a report; the rows beside them are as ever."""
    for bad, code in [("nan", 8), ("inf", 8), ("empty", 2)]:
        for k, p in [(0, 1.0), (7, 0.9), (0, 0.9)]:
            z = ru.rows_of(5, 9001, dtype, seed=4)
            u = uniform(5, 2, 4).cuda()
            want, want_p, _ = dsbd.sample_rows(z, u, top_k=k, top_p=p)
            z[2] = -math.inf if bad == "empty" else z[2]
            z[2, 4500] = {"nan": math.nan, "inf": math.inf, "empty": -math.inf}[bad]
            for T in (1.0, 0.0):
                token, logp, status = dsbd.sample_rows(z, u, temperature=T, top_k=k, top_p=p)
                assert int(status) == code
                assert token[2].tolist() == [-1, -1] and bool(logp[2].isnan().all())
                if T:
                    rows = [0, 1, 3, 4]
                    assert torch.equal(token[rows], want[rows]) and torch.equal(logp[rows], want_p[rows])


def test_settings_and_uniforms_out_of_range():
    z = ru.rows_of(6, 3000, F32, seed=4)
    u = uniform(6, 3, 4).cuda()
    want, want_p, _ = dsbd.sample_rows(z, u)
    t = lambda *x: torch.tensor(x, dtype=F32, device="cuda")
    for how in (dict(temperature=t(1, 1, -1, 1, math.nan, math.inf)), dict(top_p=t(1, 1, 0, 1, -0.5, math.nan)),
                dict(min_p=t(0, 0, -0.1, 0, 1.1, math.nan))):
        token, logp, status = dsbd.sample_rows(z, u, **how)
        assert int(status) == 6
        assert bool((token[[2, 4, 5]] == -1).all()) and bool(logp[[2, 4, 5]].isnan().all())
        assert torch.equal(token[[0, 1, 3]], want[[0, 1, 3]]) and torch.equal(logp[[0, 1, 3]], want_p[[0, 1, 3]])
    for k in (0, 20):
        want, want_p, _ = dsbd.sample_rows(z, u, top_k=k)
        for T in (1.0, 0.0):
            bad = u.clone()
            bad[1, 1], bad[2, 0], bad[3, 2] = -1e-6, 1.0 + 2.0 ** -23, math.nan
            token, logp, status = dsbd.sample_rows(z, bad, temperature=T, top_k=k)
            out = torch.zeros(6, 3, dtype=torch.bool, device="cuda")
            out[1, 1] = out[2, 0] = out[3, 2] = True
            assert int(status) == 6 and bool((token[out] == -1).all()) and bool(logp[out].isnan().all())
            if T:
                assert torch.equal(token[~out], want[~out]) and torch.equal(logp[~out], want_p[~out])


def test_no_rows_no_draws():
    z = torch.zeros(0, 100, device="cuda")
    token, logp, status = dsbd.sample_rows(z, torch.zeros(0, 3, device="cuda"))
    assert token.shape == (0, 3) and int(status) == 0
    token, logp, status = dsbd.sample_rows(torch.zeros(2, 100, device="cuda"), torch.zeros(2, 0, device="cuda"))
    assert token.shape == (2, 0) and int(status) == 0


@pytest.mark.parametrize("how", [dict(), dict(top_k=30, top_p=0.9), dict(top_p=0.9), dict(top_k=3000, top_p=0.95)])
def test_the_same_call_gives_the_same_bits(how):
    z = ru.rows_of(64, 50257, BF, seed=11)
    u = uniform(64, 2, 1).cuda()
    first = dsbd.sample_rows(z, u, **how)
    for _ in range(5):
        again = dsbd.sample_rows(z, u, **how)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_a_captured_call_draws_from_new_logits():
    z = ru.rows_of(5, 20000, F32, seed=1).contiguous()
    u = uniform(5, 2, 2).cuda()
    token, logp, status = (torch.zeros(5, 2, dtype=I32, device="cuda"), torch.zeros(5, 2, device="cuda"),
                           torch.zeros(1, dtype=I32, device="cuda"))
    call = lambda: dsbd.sample_rows(z, u, top_p=0.9, token=token, logp=logp, status=status)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in (3, 4):
        z.copy_(ru.rows_of(5, 20000, F32, seed=seed))
        u.copy_(uniform(5, 2, seed))
        graph.replay()
        torch.cuda.synchronize()
        want = dsbd.sample_rows(z, u, top_p=0.9)
        assert torch.equal(token, want[0]) and torch.equal(logp, want[1])


def test_a_call_on_another_stream_makes_what_it_needs_there():
    z = ru.rows_of(3, 4000, F32, seed=1)
    z[1] = math.nan
    u = uniform(3, 1, 2).cuda()
    side = torch.cuda.Stream()
    dsbd.sample_rows(z, u)
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)
    token, _, status = dsbd.sample_rows(z, u, stream=side)
    torch.cuda.synchronize()
    assert int(status) == 8 and token[:, 0].tolist()[1] == -1


def test_what_the_binding_refuses():
    z, u = torch.zeros(3, 50, device="cuda"), torch.zeros(3, 2, device="cuda")
    f = torch.ones(3, device="cuda")
    for bad in (dict(logits=z.half()), dict(logits=z.cpu()), dict(logits=z.t()), dict(logits=z[0]), dict(uniform=u[:2]), dict(uniform=u.double()),
                dict(uniform=u.cpu()), dict(uniform=torch.zeros(2, 3, device="cuda").t()), dict(token=torch.zeros(3, 2, device="cuda")),
                dict(token=torch.zeros(3, 1, dtype=I32, device="cuda")), dict(logp=torch.zeros(3, 2, dtype=BF, device="cuda")),
                dict(temperature=f.double()), dict(temperature=f[:2]), dict(top_k=f), dict(top_p=f.cpu()), dict(min_p=f[:, None]),
                dict(status=torch.zeros(1, device="cuda")), dict(status=torch.zeros(1, dtype=I32))):
        with pytest.raises((AssertionError, RuntimeError)):
            dsbd.sample_rows(**dict(dict(logits=z, uniform=u), **bad))
    for bad in (dict(temperature=-1.0), dict(temperature=math.nan), dict(temperature=math.inf), dict(top_p=0.0), dict(top_p=-1.0),
                dict(top_p=math.nan), dict(min_p=-0.1), dict(min_p=1.5), dict(min_p=math.nan)):
        with pytest.raises(dsbd.DsbdError, match="invalid argument"):
            dsbd.sample_rows(z, u, **bad)
    with pytest.raises(dsbd.DsbdError, match="unsupported"):
        dsbd.sample_rows(torch.empty(1, 393217, device="cuda"), u[:1])
