"""Attention of a chunk of new tokens over the paged cache, on the GPU against a plain 64-bit form."""
import numpy as np
import pytest
import torch

import paper_2409_16560_b200 as dsbd
from chunk_util import PAGE, attention_bar, attention_reference, chunk_of, paged_problem

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _attend(p, q, Hkv, scale, **kw):
    out, st = dsbd.chunk_attention_paged(chunk_of(p), q.shape[1], Hkv, q.shape[2], scale, q, p["k_pool"], p["v_pool"], **kw)
    torch.cuda.synchronize()
    return out, int(st.item())


def _check(p, q, Hkv, scale):
    out, st = _attend(p, q, Hkv, scale)
    assert st == 0
    ref, mass = attention_reference(q, p, scale)
    err = (out.double() - ref).abs()
    assert torch.all(err <= attention_bar(mass)), (float(err.max()), [int(i) for i in torch.nonzero(err > attention_bar(mass))[0]])
    return out


# tokens per sequence (new, cached): one token, ends of pages and tiles, row tiles that are just full or one over,
# nothing cached, nothing new, long caches that are cut between CTAs
LENGTHS = {
    "one": ([1], [0]),
    "ones": ([1] * 9, [0, 1, 62, 63, 64, 126, 127, 128, 300]),
    "ends": ([64, 65, 63, 2], [0, 63, 1, 126]),
    "tiles": ([31, 32, 33, 64, 65], [97, 96, 95, 64, 63]),
    "mixed": ([1, 0, 200, 1, 17, 0, 300], [1000, 500, 0, 40, 2111, 0, 77]),
    "long": ([1, 5], [9000, 20000]),
    "prompt": ([1500], [0]),
    "whole": ([0, 1, 0, 70, 3], [5, 0, 9, 100, 64]),
    "blocks": ([0, 129, 65, 300], [64, 0, 700, 5]),
    "many": ([1, 2, 3] * 130, [17 * (i % 23) for i in range(390)]),
}


@pytest.mark.parametrize("lengths", list(LENGTHS))
@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 128), (2, 2, 128), (8, 2, 64), (3, 3, 64)])
def test_attention_against_64_bits(lengths, Hq, Hkv, d):
    new, old = LENGTHS[lengths]
    p = paged_problem(new, old, Hkv, d, BF, seed=len(new) + d)
    _check(p, p["randn"](p["T"], Hq, d), Hkv, d ** -0.5)


@pytest.mark.parametrize("Hq,Hkv", [(5, 1), (14, 2), (40, 8), (33, 1), (64, 1), (128, 1), (100, 1), (12, 12), (32, 32)])
def test_head_layouts(Hq, Hkv):
    """Groups that fill the 128 rows of a tile and ones that do not, up to one token a tile."""
    for d in (64, 128):
        p = paged_problem([3, 130, 1, 70], [5, 0, 700, 60], Hkv, d, BF, seed=Hq)
        _check(p, p["randn"](p["T"], Hq, d), Hkv, d ** -0.5)


def test_peaked_and_shifted_logits():
    """Logits far apart, maxima that keep growing along the cache, and a common offset of all of a row's logits: references
    move, and rows of heavy weights have the rounding of their weights cancelled."""
    Hq, Hkv, d = 8, 2, 128
    for what in ("peaked", "growing", "falling", "offset"):
        p = paged_problem([70, 1], [900, 1500], Hkv, d, BF, seed=5)
        q = p["randn"](p["T"], Hq, d)
        if what == "peaked":
            q = q * 8
        elif what == "offset":
            p["k_pool"] += 3
            q = q + 2
        else:
            for b in range(2):
                pages = torch.as_tensor(p["table_host"][p["page_off_host"][b]:p["page_off_host"][b + 1]]).long().cuda()
                ramp = torch.linspace(0, 4, len(pages), device="cuda") if what == "growing" else torch.linspace(4, 0, len(pages), device="cuda")
                p["k_pool"][pages] = (p["k_pool"][pages].float() * 0.2 + ramp[:, None, None, None] * torch.sign(p["k_pool"][pages[0], 0, 0]).float()).to(BF)
            q = torch.sign(p["k_pool"][int(p["table_host"][0]), 0, 0].float()).to(BF).expand(q.shape).contiguous()
        out, st = _attend(p, q, Hkv, d ** -0.5)
        ref, mass = attention_reference(q, p, d ** -0.5)
        # larger logits: an fp32 sum of 128 products of size s carries up to 128 * 2^-24 * s on the logit
        size = float((q.float().abs().amax() * p["k_pool"].float().abs().amax()) * 128 * d ** -0.5)
        bar = attention_bar(mass) + 128 * 2.0 ** -24 * size * mass
        assert st == 0 and torch.all((out.double() - ref).abs() <= bar), what


def test_an_output_at_16_bytes():
    """32-byte stores are for outputs that allow them."""
    for new, old in (([40, 1], [10, 300]), ([200], [3000])):
        p = paged_problem(new, old, 2, 128, BF, seed=20)
        q = p["randn"](p["T"], 8, 128)
        want, _ = _attend(p, q, 2, 128 ** -0.5)
        out = torch.empty(q.numel() + 8, dtype=BF, device="cuda")[8:].view(q.shape)
        assert out.data_ptr() % 32 == 16
        got, st = _attend(p, q, 2, 128 ** -0.5, out=out)
        assert st == 0 and torch.equal(got, want)


def test_scales():
    p = paged_problem([40, 2], [100, 300], 1, 64, BF, seed=8)
    q = p["randn"](42, 4, 64)
    for scale in (1e-3, 0.5, 1.0):
        _check(p, q, 1, scale)


def test_what_lies_behind_the_last_token_does_not_count():
    """NaN and infinities behind a sequence's end, in its last page, in pages that are not its own and in whole pages of the
    table that it does not reach."""
    Hq, Hkv, d = 4, 2, 128
    for new, old in (([1, 1, 30], [5, 70, 100]), ([100, 3], [90, 0]), ([300], [0]), ([1], [63])):
        p = paged_problem(new, old, Hkv, d, BF, seed=9, extra_pages=5)
        q = p["randn"](p["T"], Hq, d)
        want = _check(p, q, Hkv, d ** -0.5)
        used = torch.zeros(p["k_pool"].shape[0], PAGE, dtype=torch.bool, device="cuda")
        for b in range(len(new)):
            for t in range(new[b] + old[b]):
                used[p["table_host"][p["page_off_host"][b] + t // PAGE], t % PAGE] = True
        for fill in (float("nan"), float("inf"), float("-inf")):
            for pool in (p["k_pool"], p["v_pool"]):
                pool.copy_(torch.where(used[:, None, :, None], pool, torch.full_like(pool, fill)))
            got, st = _attend(p, q, Hkv, d ** -0.5)
            assert st == 0 and torch.equal(got, want)


@pytest.mark.parametrize("Hq,Hkv,d", [(62, 2, 128), (8, 2, 128), (8, 8, 64)])
def test_what_lies_behind_many_wide_blocks_does_not_count(Hq, Hkv, d):
    """Either row tile of a wide block may be the first to come to the block's last tile."""
    new, old = [122, 5, 300, 71, 1, 257, 130] * 6, [3, 475, 0, 65, 65, 30, 700] * 6
    p = paged_problem(new, old, Hkv, d, BF, seed=19)
    used = torch.zeros(p["k_pool"].shape[0], PAGE, dtype=torch.bool, device="cuda")
    for b in range(len(new)):
        pages = torch.as_tensor(p["table_host"][p["page_off_host"][b]:p["page_off_host"][b + 1]]).long().cuda()
        used[pages] = (torch.arange(len(pages) * PAGE, device="cuda") < new[b] + old[b]).view(-1, PAGE)
    for pool in (p["k_pool"], p["v_pool"]):
        pool[~used[:, None].expand(-1, Hkv, -1)] = float("nan")
    q = p["randn"](p["T"], Hq, d)
    first = _check(p, q, Hkv, d ** -0.5)
    for _ in range(20):
        out, st = _attend(p, q, Hkv, d ** -0.5)
        assert st == 0 and torch.equal(out, first)


def test_rows_of_bad_numbers_stay_their_own():
    """A query row of NaN or infinities gives NaN and leaves its neighbours alone."""
    p = paged_problem([60, 1], [200, 40], 2, 128, BF, seed=10)
    q = p["randn"](61, 8, 128)
    want, _ = _attend(p, q, 2, 128 ** -0.5)
    bad = q.clone()
    bad[7, 3], bad[50, 0, 5], bad[60, 7, 0] = float("nan"), float("inf"), float("nan")
    got, st = _attend(p, bad, 2, 128 ** -0.5)
    hit = torch.zeros(61, 8, dtype=torch.bool, device="cuda")
    hit[7, 3] = hit[50, 0] = hit[60, 7] = True
    assert st == 0 and torch.isnan(got[hit]).all() and torch.equal(got[~hit], want[~hit])


def test_results_do_not_depend_on_the_rest_of_the_batch_beyond_rounding():
    """A sequence alone and the same in a batch: other cuts between CTAs, the same numbers up to the bar."""
    p = paged_problem([40, 1, 200], [3000, 77, 10], 2, 128, BF, seed=11)
    q = p["randn"](p["T"], 8, 128)
    out, _ = _attend(p, q, 2, 128 ** -0.5)
    ref, mass = attention_reference(q, p, 128 ** -0.5)
    for b in range(3):
        lo, hi = int(p["new_off_host"][b]), int(p["new_off_host"][b + 1])
        dev = lambda a, t: torch.as_tensor(np.asarray(a, dtype=t)).cuda()
        no, po = [0, hi - lo], [0, int(p["old"][b])]
        pages = p["table_host"][p["page_off_host"][b]:p["page_off_host"][b + 1]]
        c = dsbd.Chunk(dev(no, np.int32), no, dev(po, np.int64), po, dev(pages, np.int32), dev([0, len(pages)], np.int64))
        one, st = dsbd.chunk_attention_paged(c, 8, 2, 128, 128 ** -0.5, q[lo:hi].contiguous(), p["k_pool"], p["v_pool"])
        assert int(st.item()) == 0
        assert torch.all((one.double() - ref[lo:hi]).abs() <= attention_bar(mass[lo:hi]))
    again, _ = _attend(p, q, 2, 128 ** -0.5)
    assert torch.equal(out, again)                            # the same call gives the same bits


def test_shared_pages_and_a_pool_beyond_32_bits():
    """Sequences that share their prefix pages, and pages at the end of pools of more than 2^32 bytes."""
    Hq, Hkv, d = 8, 8, 128
    n_pages = 34000                                           # 64 KB a page and head group: 4.4 GB a pool
    assert n_pages * Hkv * PAGE * d * 2 > 2 ** 32
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    k_pool = torch.zeros(n_pages, Hkv, PAGE, d, dtype=BF, device="cuda")
    v_pool = torch.zeros_like(k_pool)
    ids = [n_pages - 1, 0, n_pages - 2, n_pages - 7, 3, n_pages - 3]
    for i in ids:
        k_pool[i] = torch.randn(Hkv, PAGE, d, generator=g, device="cuda").to(BF)
        v_pool[i] = torch.randn(Hkv, PAGE, d, generator=g, device="cuda").to(BF)
    table = np.array(ids[:3] + ids[3:4] + ids[:3] + ids[4:], np.int32)          # both start with the same three pages
    p = dict(new=np.array([10, 64]), old=np.array([210, 250]), new_off_host=np.array([0, 10, 74], np.int32),
             prefix_off_host=np.array([0, 210, 460]), page_off_host=np.array([0, 4, 9]), table_host=table, k_pool=k_pool, v_pool=v_pool, T=74)
    dev = lambda a, t: torch.as_tensor(np.asarray(a, dtype=t)).cuda()
    p.update(new_off=dev(p["new_off_host"], np.int32), prefix_off=dev(p["prefix_off_host"], np.int64),
             page_off=dev(p["page_off_host"], np.int64), page_table=dev(table, np.int32))
    _check(p, torch.randn(74, Hq, d, generator=g, device="cuda").to(BF), Hkv, d ** -0.5)


def test_reports():
    base = paged_problem([5, 40, 1], [100, 20, 300], 2, 128, BF, seed=12)
    q = base["randn"](46, 4, 128)
    want, _ = _attend(base, q, 2, 128 ** -0.5)
    # a sequence whose table is too short: its missing pages read as zeros, the others are as before
    p = dict(base, page_off=base["page_off"].clone())
    p["page_off"][3] -= 1
    got, st = _attend(p, q, 2, 128 ** -0.5)
    assert st == 3 and torch.equal(got[:45], want[:45]) and torch.isfinite(got).all()
    # a page id outside the pool
    for bad in (base["k_pool"].shape[0], -1, 2 ** 31 - 1):
        p = dict(base, page_table=base["page_table"].clone())
        p["page_table"][0] = bad
        got, st = _attend(p, q, 2, 128 ** -0.5)
        assert st == 7 and torch.equal(got[5:], want[5:]) and torch.isfinite(got).all()
    # offsets that contradict the call: that sequence's rows are not written
    for field, at, to in (("new_off", 2, 47), ("new_off", 2, 3), ("prefix_off", 2, 90), ("prefix_off", 2, 10 ** 12)):
        p = {**base, field: base[field].clone()}
        p[field][at] = to
        out = torch.full_like(q, 9.0)
        got, st = _attend(p, q, 2, 128 ** -0.5, out=out)
        assert st == 7 and torch.isfinite(got).all()
        assert torch.equal(got[:5], want[:5])


def test_refusals():
    p = paged_problem([2, 3], [10, 0], 2, 128, BF, seed=13)
    c = chunk_of(p)
    q = p["randn"](5, 4, 128)

    def code(**kw):
        a = dict(Hq=4, Hkv=2, d=128, scale=0.1, q=q, k_pool=p["k_pool"], v_pool=p["v_pool"])
        a.update(kw)
        with pytest.raises(dsbd.DsbdError) as e:
            dsbd.chunk_attention_paged(c, a["Hq"], a["Hkv"], a["d"], a["scale"], a["q"], a["k_pool"], a["v_pool"], **{k: v for k, v in kw.items() if k in ("out", "workspace")})
        return e.value.code

    assert code(scale=0.0) == -1 and code(scale=-1.0) == -1 and code(scale=float("inf")) == -1 and code(scale=float("nan")) == -1
    assert code(q=q.float(), k_pool=p["k_pool"].float(), v_pool=p["v_pool"].float()) == -2
    f = paged_problem([2, 3], [10, 0], 2, 96, BF, seed=13)
    assert code(d=96, q=f["randn"](5, 4, 96), k_pool=f["k_pool"], v_pool=f["v_pool"]) == -2
    assert code(Hq=3, q=p["randn"](5, 3, 128)) == -1
    assert code(out=q) == -1
    odd = torch.zeros(5 * 4 * 128 + 1, dtype=BF, device="cuda")[1:].view(5, 4, 128)
    assert code(q=odd) == -2
    big = paged_problem([1], [5000], 2, 128, BF, seed=1)
    cb = chunk_of(big)
    need = dsbd.chunk_attention_workspace(cb, 4, 2, 128, BF, 0.1)
    with pytest.raises(dsbd.DsbdError) as e:
        dsbd.chunk_attention_paged(cb, 4, 2, 128, 0.1, big["randn"](1, 4, 128), big["k_pool"], big["v_pool"],
                                   workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    assert e.value.code == -3
    assert dsbd.chunk_attention_workspace(cb, 3, 2, 128, BF, 0.1) == 0
    assert dsbd.chunk_attention_launches(cb, 4, 2, 128, BF, 0.1) == 2 and dsbd.chunk_attention_launches(c, 4, 2, 128, BF, 0.1) == 1


def test_nothing_new():
    p = paged_problem([0, 0], [10, 100], 2, 128, BF, seed=14)
    out, st = _attend(p, torch.zeros(0, 4, 128, dtype=BF, device="cuda"), 2, 0.1)
    assert out.shape == (0, 4, 128) and st == 0


def test_another_stream_and_a_graph():
    p = paged_problem([30, 1, 1], [500, 2000, 4], 2, 128, BF, seed=15)
    q = p["randn"](32, 8, 128)
    want, _ = _attend(p, q, 2, 128 ** -0.5)
    c = chunk_of(p)
    out, status = torch.empty_like(q), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(dsbd.chunk_attention_workspace(c, 8, 2, 128, BF, 128 ** -0.5), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    dsbd.chunk_attention_paged(c, 8, 2, 128, 128 ** -0.5, q, p["k_pool"], p["v_pool"], out=out, workspace=ws, status=status, stream=side)
    side.synchronize()
    assert torch.equal(out, want) and int(status.item()) == 0
    # a graph of append and attention reads the offsets and tables that are there at its replay
    k, v = p["randn"](32, 2, 128), p["randn"](32, 2, 128)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dsbd.kv_append_paged(c, k, v, p["k_pool"], p["v_pool"], status=status)
        dsbd.chunk_attention_paged(c, 8, 2, 128, 128 ** -0.5, q, p["k_pool"], p["v_pool"], out=out, workspace=ws, status=status)
    for old in ([500, 2000, 4], [499, 1700, 0]):
        p["prefix_off"].copy_(torch.tensor([0] + list(np.cumsum(old))))
        graph.replay()
        torch.cuda.synchronize()
        p["old"] = np.array(old)
        ref, mass = attention_reference(q, p, 128 ** -0.5)
        assert int(status.item()) == 0 and torch.all((out.double() - ref).abs() <= attention_bar(mass))


def test_a_wait_that_runs_out_sets_the_status_and_leaves_the_context_usable():
    """In a second library, built with short waits, CTA 0's second stage never comes: the call returns with the status set, the rows of
    the other CTAs are right, and the product library's next launch is.  (Whole units, then units that are cut.)"""
    import ctypes as C
    from paper_2409_16560_b200 import build
    lib = C.CDLL(build.build_wait_test())
    lib.dsbd_chunk_attention_paged.argtypes = [C.c_void_p] * 8 + [C.c_size_t, C.c_void_p, C.c_void_p]
    from paper_2409_16560_b200 import binding as bd
    for new, old in (([5, 70, 2], [600, 300, 500]), ([40, 300, 7], [9000, 700, 6000])):
        p = paged_problem(new, old, 2, 128, BF, seed=16)
        q = p["randn"](p["T"], 8, 128)
        want, st = _attend(p, q, 2, 128 ** -0.5)
        assert st == 0
        c = chunk_of(p)
        desc = bd._desc(8, 2, 128, BF, 128 ** -0.5)
        ws = torch.empty(dsbd.chunk_attention_workspace(c, 8, 2, 128, BF, 128 ** -0.5), dtype=torch.uint8, device="cuda")
        for _ in range(2):                                    # (the first launch loads the kernel)
            out, status = torch.zeros_like(q), torch.zeros(1, dtype=torch.int32, device="cuda")
            begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            begin.record()
            rc = lib.dsbd_chunk_attention_paged(c.address, C.addressof(desc), q.data_ptr(), p["k_pool"].data_ptr(), p["v_pool"].data_ptr(),
                                                c.pages(p["k_pool"].shape[0]), out.data_ptr(), ws.data_ptr(), ws.numel(),
                                                status.data_ptr(), torch.cuda.current_stream().cuda_stream)
            end.record()
            assert rc == 0
            torch.cuda.synchronize()
            assert int(status.item()) == 5
        assert begin.elapsed_time(end) < 20.0                 # a millisecond a wait that runs out, and a few of them
        assert torch.equal(out[-new[-1]:], want[-new[-1]:])   # the last sequence is other CTAs'
        again, st = _attend(p, q, 2, 128 ** -0.5)
        assert st == 0 and torch.equal(again, want)
