"""Rotation and append of so many tokens that a warp takes several groups of a token's heads, one after the other: from the queries over
the keys to the values, whole tokens, and last warps that get fewer groups than the others."""
import numpy as np
import pytest
import torch

import paper_2409_16560_b200 as dsbd
from chunk_util import PAGE, cache_of, chunk_of, paged_problem, turned_bar

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _close(got, x, w, rows, layout, eps=1e-6):
    for i in range(0, x.shape[0], 1024):                     # (64-bit copies of a piece at a time)
        r = slice(i, i + 1024)
        ref, bar = turned_bar(x[r], w, rows[r], layout, eps, got.dtype == BF)
        err = (got[r].double() - ref).abs()
        assert torch.all(err <= bar), (i, float((err - bar).max()))


def _problem(T, Hq, Hkv, d, rot, dtype, norm, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    qkv = torch.randn(T, (Hq + 2 * Hkv) * d, generator=g, device="cuda").to(dtype)
    q, k, v = (x.unflatten(1, (-1, d)) for x in qkv.split([Hq * d, Hkv * d, Hkv * d], 1))
    wq, wk = (1 + 0.3 * torch.randn(d, generator=g, device="cuda") if norm else None for _ in range(2))
    return g, qkv, q, k, v, wq, wk, dsbd.rope_table(6000, rot)


# A group is 8 heads of 128 or 16 of 64 in bf16, half as many in fp32; 3552 warps or more share a call.  900, 1900 and 4000 tokens:
# up to 4 warps, 2 warps and 1 warp a token.  (Hq, Hkv): 6 groups (2 2 2, 3 3, 6), 5 with an uneven last warp (2 2 1, 3 2), 7 (2 2 2 1, 4 3).
SHAPES = [(BF, 128, 40, 8, 128, "half", True), (BF, 128, 28, 4, 64, "interleaved", False), (BF, 64, 64, 16, 64, "half", True),
          (BF, 64, 96, 12, 32, "interleaved", True), (F32, 128, 16, 4, 128, "interleaved", True), (F32, 64, 24, 8, 48, "half", False)]


@pytest.mark.parametrize("T", [900, 1900, 4000])
@pytest.mark.parametrize("dtype,d,Hq,Hkv,rot,layout,norm", SHAPES)
def test_rotation(T, dtype, d, Hq, Hkv, rot, layout, norm):
    g, qkv, q, k, v, wq, wk, table = _problem(T, Hq, Hkv, d, rot, dtype, norm, T + d)
    position = torch.randint(0, 6000, (T,), generator=g, device="cuda", dtype=torch.int32)
    rope = dsbd.Rope(table, layout=layout, q_norm=wq, k_norm=wk)
    before = qkv.clone()
    qo, ko, st = dsbd.rotate_qk(q, k, position, rope)
    assert int(st.item()) == 0 and torch.equal(qkv, before)
    rows = table[position.long()]
    _close(qo, q, wq, rows, layout)
    _close(ko, k, wk, rows, layout)
    dsbd.rotate_qk(q, k, position, rope, q_out=q, k_out=k)    # in place
    assert torch.equal(q, qo) and torch.equal(k, ko)
    assert torch.equal(qkv[:, (Hq + Hkv) * d:], before[:, (Hq + Hkv) * d:])
    # either alone gives the same
    none, k1, _ = dsbd.rotate_qk(None, before[:, Hq * d:(Hq + Hkv) * d].unflatten(1, (Hkv, d)), position, rope)
    q1, none, _ = dsbd.rotate_qk(before[:, :Hq * d].unflatten(1, (Hq, d)), None, position, rope)
    assert torch.equal(k1, ko) and torch.equal(q1, qo)


@pytest.mark.parametrize("T", [900, 1900, 4000])
@pytest.mark.parametrize("dtype,d,Hq,Hkv,rot,layout,norm", SHAPES)
def test_append(T, dtype, d, Hq, Hkv, rot, layout, norm):
    new = [T // 3, 0, 1, T - T // 3 - 1 - T // 5, T // 5]
    old = [70, 5, 127, 0, 1]
    for with_q in (True, False):
        p = paged_problem(new, old, Hkv, d, dtype, seed=T + d)
        _, _, q, k, v, wq, wk, table = _problem(T, Hq, Hkv, d, rot, dtype, norm, T + d)
        k0, v0 = p["k_pool"].clone(), p["v_pool"].clone()
        qo, st = dsbd.kv_append_paged(chunk_of(p), k, v, p["k_pool"], p["v_pool"],
                                      rope=dsbd.Rope(table, layout=layout, q_norm=wq, k_norm=wk), q=q if with_q else None)
        assert int(st.item()) == 0 and (qo is None) == (not with_q)
        position = torch.as_tensor(np.concatenate([np.arange(L, L + n) for n, L in zip(new, old)])).cuda()
        rows = table[position]
        if with_q:
            _close(qo, q, wq, rows, layout)
        got_k = torch.cat([cache_of(p["k_pool"], p, b, old[b] + new[b])[old[b]:] for b in range(len(new))])
        got_v = torch.cat([cache_of(p["v_pool"], p, b, old[b] + new[b])[old[b]:] for b in range(len(new))])
        _close(got_k, k, wk, rows, layout)
        assert torch.equal(got_v, v)
        # all else: zeros behind the last token of a page that the call opened, untouched rows elsewhere
        for pool, before in ((p["k_pool"], k0), (p["v_pool"], v0)):
            left = torch.ones(pool.shape[0], PAGE, dtype=torch.bool, device="cuda")
            for b in range(len(new)):
                pages = p["table_host"][p["page_off_host"][b]:p["page_off_host"][b + 1]]
                end = old[b] + new[b]
                for t in range(old[b], end):
                    left[pages[t // PAGE], t % PAGE] = False
                if new[b] and end % PAGE and end // PAGE * PAGE >= old[b]:
                    left[pages[end // PAGE], end % PAGE:] = False
                    assert not pool[pages[end // PAGE], :, end % PAGE:].any()
            rest = left[:, None, :, None].expand(pool.shape)
            assert torch.equal(pool[rest], before[rest])
