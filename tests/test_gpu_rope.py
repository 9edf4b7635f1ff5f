"""Rotation with the heads' norms, append to the paged cache, positions of a forest's nodes, on the GPU against plain 64-bit
forms."""
import numpy as np
import pytest
import torch

import paper_2409_16560_b200 as dsbd
from chunk_util import PAGE, cache_of, chunk_of, paged_problem, turned, turned_bar

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _close(got, x, w, rows, layout, eps):
    ref, bar = turned_bar(x, w, rows, layout, eps, got.dtype == BF)
    err = (got.double() - ref).abs()
    assert torch.all(err <= bar), float((err - bar).max())


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("dtype,d,rot", [(BF, 128, 128), (BF, 128, 32), (BF, 128, 96), (BF, 64, 64), (BF, 64, 16),
                                         (F32, 128, 128), (F32, 128, 48), (F32, 64, 64), (F32, 64, 16)])
def test_rotation_against_64_bits(dtype, d, rot, norm, layout):
    g = _gen(rot + d)
    table = dsbd.rope_table(4096, rot, base=10000.0)
    for T, Hq, Hkv in [(1, 4, 4), (3, 32, 8), (65, 28, 4), (130, 1, 1), (7, 40, 40)]:
        # views of a fused projection's output whose rows are a little longer than the heads
        qkv = torch.randn(T, (Hq + 2 * Hkv) * d + 16, generator=g, device="cuda").to(dtype)
        q = qkv[:, :Hq * d].unflatten(1, (Hq, d))
        k = qkv[:, Hq * d:(Hq + Hkv) * d].unflatten(1, (Hkv, d))
        wq, wk = (torch.randn(d, generator=g, device="cuda") if norm else None for _ in range(2))
        position = torch.randint(0, 4096, (T,), generator=g, device="cuda", dtype=torch.int32)
        rope = dsbd.Rope(table, layout=layout, q_norm=wq, k_norm=wk, eps=1e-5)
        before = qkv.clone()
        qo, ko, st = dsbd.rotate_qk(q, k, position, rope)
        assert int(st.item()) == 0 and torch.equal(qkv, before)
        rows = table[position.long()]
        _close(qo, q, wq, rows, layout, 1e-5)
        _close(ko, k, wk, rows, layout, 1e-5)
        # in place gives the same bits, and touches nothing else of the rows
        dsbd.rotate_qk(q, k, position, rope, q_out=q, k_out=k)
        assert torch.equal(q, qo) and torch.equal(k, ko)
        assert torch.equal(qkv[:, (Hq + Hkv) * d:], before[:, (Hq + Hkv) * d:])


def test_norms_without_rotation_and_one_tensor_alone():
    g = _gen(3)
    q = torch.randn(9, 6, 128, generator=g, device="cuda").to(BF)
    w = torch.rand(128, generator=g, device="cuda") + 0.5
    qo, none, st = dsbd.rotate_qk(q, None, None, dsbd.Rope(None, q_norm=w))
    assert none is None and int(st.item()) == 0
    _close(qo, q, w, None, "half", 1e-6)
    table = dsbd.rope_table(64, 64)
    position = torch.arange(9, dtype=torch.int32, device="cuda")
    none, ko, st = dsbd.rotate_qk(None, q, position, dsbd.Rope(table))
    assert none is None and int(st.item()) == 0
    _close(ko, q, None, table[position.long()], "half", 1e-6)


def test_position_zero_and_the_part_behind_the_rotation_keep_their_bits():
    """cos 0 = 1, sin 0 = 0: the row comes back; infinities and NaN outside the rotated part stay where they are."""
    table = dsbd.rope_table(100, 32)
    x = torch.randn(2, 3, 128, generator=_gen(4), device="cuda").to(BF)
    x[..., 40], x[..., 41], x[..., 127] = float("inf"), float("nan"), float("-inf")
    for layout in ("half", "interleaved"):
        y, _, st = dsbd.rotate_qk(x, None, torch.tensor([0, 99], dtype=torch.int32, device="cuda"), dsbd.Rope(table, layout=layout))
        assert int(st.item()) == 0
        assert torch.equal(y[0].view(torch.int16), x[0].view(torch.int16))
        assert torch.equal(y[1, :, 32:].view(torch.int16), x[1, :, 32:].view(torch.int16))
        assert torch.isfinite(y[1, :, :32]).all()


def test_positions_out_of_the_table_are_left_out_and_reported():
    table = dsbd.rope_table(50, 128)
    x = torch.randn(4, 2, 128, generator=_gen(5), device="cuda")
    out = torch.full_like(x, 7.0)
    position = torch.tensor([0, 50, -1, 49], dtype=torch.int32, device="cuda")
    _, _, st = dsbd.rotate_qk(x, None, position, dsbd.Rope(table), q_out=out)
    assert int(st.item()) == 7
    assert (out[1:3] == 7.0).all() and torch.equal(out[0], x[0]) and not (out[3] == 7.0).any()


def test_rotations_keep_inner_products_by_distance():
    """What the rotation is for: (rotated q at m) . (rotated k at n) depends on m - n alone."""
    g = _gen(6)
    table = dsbd.rope_table(5000, 128)
    q = torch.randn(1, 1, 128, generator=g, device="cuda").expand(3, 1, 128).contiguous()
    k = torch.randn(1, 1, 128, generator=g, device="cuda").expand(3, 1, 128).contiguous()
    m = torch.tensor([10, 1010, 4010], dtype=torch.int32, device="cuda")
    qo, _, _ = dsbd.rotate_qk(q, None, m, dsbd.Rope(table))
    ko, _, _ = dsbd.rotate_qk(k, None, m - 7, dsbd.Rope(table))
    dots = (qo.double() * ko.double()).sum(-1).flatten()
    # angles carry 2^-24 each: 128 terms of size about 1
    assert (dots - dots[0]).abs().max() < 128 * 4 * 2.0 ** -24 * float((q.abs() * k.abs()).sum())


@pytest.mark.parametrize("scaling", [None, dict(kind="linear", factor=4.0), dict(kind="base", factor=8.0),
                                     dict(kind="wavelength", factor=8.0, original=8192, low=1.0, high=4.0),
                                     dict(kind="ramp", factor=16.0, original=4096, low=1.0, high=32.0)])
def test_table_against_64_bits(scaling):
    n, rot = 40000, 96
    table = dsbd.rope_table(n, rot, base=500000.0, scaling=scaling)
    f, att = dsbd.rope_frequencies(rot, base=500000.0, scaling=scaling)
    ang = np.arange(n)[:, None] * f[None, :]
    t = table.cpu().numpy()
    # one rounding of the result; the library's and numpy's sine in double differ in the last place
    assert np.abs(t[:, 0] - np.cos(ang) * att).max() <= 2.0 ** -24 * att * 1.001
    assert np.abs(t[:, 1] - np.sin(ang) * att).max() <= 2.0 ** -24 * att * 1.001


def _append(p, k, v, rope, q=None):
    qo, st = dsbd.kv_append_paged(chunk_of(p), k, v, p["k_pool"], p["v_pool"], rope=rope, q=q)
    torch.cuda.synchronize()
    return qo, int(st.item())


LENGTHS = [([1], [0]), ([1, 1, 1, 1], [0, 63, 64, 130]), ([64, 0, 65, 1], [0, 5, 1, 127]), ([200, 3, 0, 0, 61], [30, 0, 0, 64, 3]),
           ([1] * 70, list(range(70)))]


@pytest.mark.parametrize("new,old", LENGTHS)
@pytest.mark.parametrize("dtype,d,Hq,Hkv,rot,layout,norm", [(BF, 128, 32, 8, 128, "half", True), (BF, 64, 4, 4, 32, "interleaved", False),
                                                            (F32, 128, 6, 2, 64, "half", False), (F32, 64, 5, 5, 64, "interleaved", True)])
def test_append_against_64_bits(new, old, dtype, d, Hq, Hkv, rot, layout, norm):
    p = paged_problem(new, old, Hkv, d, dtype, seed=sum(new) + d)
    table = dsbd.rope_table(512, rot)
    wq, wk = (1 + p["randn"](d).float() * 0.3 if norm else None for _ in range(2))
    qkv = p["randn"](p["T"], (Hq + 2 * Hkv) * d)
    q, k, v = (x.unflatten(1, (-1, d)) for x in qkv.split([Hq * d, Hkv * d, Hkv * d], 1))
    k0, v0 = p["k_pool"].clone(), p["v_pool"].clone()
    qo, st = _append(p, k, v, dsbd.Rope(table, layout=layout, q_norm=wq, k_norm=wk), q=q)
    assert st == 0
    k1, v1 = k0.clone(), v0.clone()                    # what the pools have to be, rows of k by their bar
    for b, (n, L) in enumerate(zip(new, old)):
        r = slice(int(p["new_off_host"][b]), int(p["new_off_host"][b]) + n)
        rows = table[L:L + n]
        _close(qo[r], q[r], wq, rows, layout, 1e-6)
        got_k, got_v = cache_of(p["k_pool"], p, b, L + n)[L:], cache_of(p["v_pool"], p, b, L + n)[L:]
        _close(got_k, k[r], wk, rows, layout, 1e-6)
        assert torch.equal(got_v, v[r])
        pages = p["table_host"][p["page_off_host"][b]:p["page_off_host"][b + 1]]
        for i in range(n):
            k1[pages[(L + i) // PAGE], :, (L + i) % PAGE] = got_k[i]
            v1[pages[(L + i) // PAGE], :, (L + i) % PAGE] = v[r][i]
        end = L + n
        if n and end % PAGE and end // PAGE * PAGE >= L:     # a page that the call opened is written whole
            k1[pages[end // PAGE], :, end % PAGE:] = 0
            v1[pages[end // PAGE], :, end % PAGE:] = 0
    assert torch.equal(p["k_pool"], k1) and torch.equal(p["v_pool"], v1)


def test_append_without_rotation_copies_bits():
    p = paged_problem([70, 2], [10, 0], 3, 128, BF, seed=1)
    k, v = p["randn"](72, 3, 128), p["randn"](72, 3, 128)
    k[0, 0, 0], v[71, 2, 127] = float("nan"), float("inf")
    none, st = _append(p, k, v, None)
    assert none is None and st == 0
    for b, r in ((0, slice(0, 70)), (1, slice(70, 72))):
        L, n = int(p["old"][b]), int(p["new"][b])
        for pool, x in ((p["k_pool"], k), (p["v_pool"], v)):
            assert torch.equal(cache_of(pool, p, b, L + n)[L:].contiguous().view(torch.int16), x[r].contiguous().view(torch.int16))


def test_append_leaves_out_what_contradicts_the_call():
    # a table that is too short, and a page id outside the pool: those rows alone are left out
    for what in ("short", "page"):
        p = paged_problem([70, 5], [0, 60], 2, 64, F32, seed=2)
        k, v = p["randn"](75, 2, 64), p["randn"](75, 2, 64)
        k0 = p["k_pool"].clone()
        if what == "short":                            # the second sequence loses its second page (from token 64 on)
            p["page_off"][-1] -= 1
        else:
            p["page_table"][int(p["page_off_host"][1]) + 1] = p["k_pool"].shape[0]
        _, st = _append(p, k, v, None)
        assert st == (3 if what == "short" else 7)
        assert torch.equal(cache_of(p["k_pool"], p, 0, 70), k[:70])
        pages = p["table_host"][int(p["page_off_host"][1]):]
        assert torch.equal(p["k_pool"][pages[0], :, 60:64].transpose(0, 1), k[70:74])
        assert torch.equal(p["k_pool"][pages[1]], k0[pages[1]])


def test_appends_and_rotations_on_another_stream():
    p = paged_problem([33, 1], [0, 7], 2, 128, BF, seed=3)
    table = dsbd.rope_table(64, 128)
    k, v, q = p["randn"](34, 2, 128), p["randn"](34, 2, 128), p["randn"](34, 4, 128)
    want_q, st = dsbd.kv_append_paged(chunk_of(p), k, v, p["k_pool"], p["v_pool"], rope=dsbd.Rope(table), q=q)
    want = p["k_pool"].clone()
    p["k_pool"].zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got_q, st = dsbd.kv_append_paged(chunk_of(p), k, v, p["k_pool"], p["v_pool"], rope=dsbd.Rope(table), q=q,
                                     q_out=torch.empty_like(q), status=torch.zeros(1, dtype=torch.int32, device="cuda"), stream=side)
    side.synchronize()
    assert torch.equal(got_q, want_q) and torch.equal(cache_of(p["k_pool"], p, 0, 33), cache_of(want, p, 0, 33))


def test_refusals_of_rotation_and_append():
    table = dsbd.rope_table(16, 64)
    position = torch.zeros(2, dtype=torch.int32, device="cuda")

    def code(call):
        with pytest.raises(dsbd.DsbdError) as e:
            call()
        return e.value.code

    x = torch.zeros(2, 2, 96, device="cuda")
    assert code(lambda: dsbd.rotate_qk(x, None, position, dsbd.Rope(table))) == -2                       # d = 96
    x = torch.zeros(2, 2, 64, device="cuda")
    assert code(lambda: dsbd.rotate_qk(x, None, position, dsbd.Rope(torch.zeros(4, 2, 64, device="cuda")))) == -1      # rot > d
    assert code(lambda: dsbd.rotate_qk(x, None, position, dsbd.Rope(torch.zeros(4, 2, 4, device="cuda")))) == -1       # rot = 8
    assert code(lambda: dsbd.rotate_qk(x, None, None, dsbd.Rope(table))) == -1                           # no positions
    odd = torch.zeros(2 * 2 * 64 + 1, device="cuda")[1:].view(2, 2, 64)
    assert code(lambda: dsbd.rotate_qk(odd, None, position, dsbd.Rope(table))) == -2                     # alignment
    q, k = torch.zeros(2, 3, 64, device="cuda"), torch.zeros(2, 2, 64, device="cuda")
    assert code(lambda: dsbd.rotate_qk(q, k, position, dsbd.Rope(table))) == -1                          # 3 heads over 2
    with pytest.raises(AssertionError):
        dsbd.rotate_qk(x, None, position, dsbd.Rope(table, q_norm=torch.ones(128, device="cuda")))
    with pytest.raises(AssertionError):
        dsbd.rotate_qk(x.transpose(0, 1), None, position, dsbd.Rope(table))
    with pytest.raises(ValueError):
        dsbd.rope_table(16, 64, scaling=dict(kind="nothing"))
    p = paged_problem([2], [0], 2, 64, F32, seed=0)
    with pytest.raises(AssertionError):                                                                  # pools of another type
        dsbd.kv_append_paged(chunk_of(p), x.to(BF), x.to(BF), p["k_pool"], p["v_pool"])
    odd = torch.zeros(2 * 2 * 64 + 1, device="cuda")[1:].view(2, 2, 64)
    assert code(lambda: dsbd.kv_append_paged(chunk_of(p), odd, x, p["k_pool"], p["v_pool"])) == -2


def test_nothing_to_append():
    p = paged_problem([0, 0], [5, 64], 2, 64, F32, seed=0)
    k0 = p["k_pool"].clone()
    e = torch.zeros(0, 2, 64, device="cuda")
    _, st = _append(p, e, e, None)
    assert st == 0 and torch.equal(k0, p["k_pool"])
    qo, ko, st = dsbd.rotate_qk(e, e, torch.zeros(0, dtype=torch.int32, device="cuda"), dsbd.Rope(dsbd.rope_table(4, 64)))
    assert qo.shape == (0, 2, 64) and int(st.item()) == 0


# ------------------------------------------------------------------------------------ positions
def _forest(sizes, rng, chain=False):
    off = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    parent = np.concatenate([[-1] + [o + (i - 1 if chain else int(rng.integers(0, i))) for i in range(1, n)] for o, n in zip(off, sizes)])
    return dict(R=1, B=len(sizes), N=int(off[-1]), max_depth=max(sizes), req_beam_off=[0, len(sizes)], beam_node_off=off,
                parent=parent.astype(np.int32), token=np.zeros(int(off[-1])))


@pytest.mark.parametrize("sizes,chain", [([1], False), ([9] * 8, True), ([1, 20, 64, 3, 128, 33], False), ([1025, 2], False),
                                         ([3000, 1, 40], False), ([1056, 1057], True)])
def test_positions_of_a_forest(sizes, chain):
    rng = np.random.default_rng(len(sizes))
    arrays = _forest(sizes, rng, chain)
    depth = np.zeros(arrays["N"], np.int64)
    for i, p in enumerate(arrays["parent"]):
        depth[i] = depth[p] + 1 if p >= 0 else 0
    L = rng.integers(0, 5000, size=len(sizes))
    prefix_off = torch.as_tensor(np.concatenate([[0], np.cumsum(L)]).astype(np.int64)).cuda()
    f = dsbd.Forest(arrays, "cuda")
    pos, st = dsbd.forest_positions(f, prefix_off)
    assert int(st.item()) == 0
    assert np.array_equal(pos.cpu().numpy(), np.repeat(L, sizes) + depth)


def test_positions_report_a_parent_outside_its_tree():
    arrays = _forest([4, 4], np.random.default_rng(0), chain=True)
    for node, bad in ((5, 3), (6, 6), (2, 7), (1, -1)):
        a = dict(arrays, parent=arrays["parent"].copy())
        a["parent"][node] = bad
        prefix_off = torch.tensor([0, 10, 30], device="cuda")
        f = dsbd.Forest.from_device(1, 2, 8, 4, {k: torch.as_tensor(np.asarray(a[k], dtype=np.int32)).cuda() for k in
                                                 ("req_beam_off", "beam_node_off", "parent", "token")}, 4, 2, 2)
        pos, st = dsbd.forest_positions(f, prefix_off)
        assert int(st.item()) == 4, (node, bad)
        other = slice(0, 4) if node >= 4 else slice(4, 8)
        assert pos[other].tolist() == ([10, 11, 12, 13] if node >= 4 else [20, 21, 22, 23])
