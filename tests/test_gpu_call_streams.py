"""Calls that are given a stream other than the current one make what they need (status word, workspace, outputs) on that stream:
its filling comes before the call's kernels, and its memory does not go to work of the current stream while they run."""
import pytest
import torch

import paper_2409_16560_b200 as dsbd
from chunk_util import attention_bar, attention_reference, chunk_of, paged_problem

pytestmark = pytest.mark.gpu
BF, I32 = torch.bfloat16, torch.int32
BUSY = 100_000_000                                            # cycles: 50 ms and more


def _calls():
    """Name -> (call on a stream that returns its status word, the code that it has to report)."""
    p = paged_problem([2, 3], [10, 0], 2, 128, BF, seed=3)
    q, k, v = p["randn"](5, 4, 128), p["randn"](5, 2, 128), p["randn"](5, 2, 128)
    table = dsbd.rope_table(8, 128)
    position = torch.full((5,), 8, dtype=I32, device="cuda")             # none of the table's
    bad = dict(p, page_table=torch.full_like(p["page_table"], -1))
    c = chunk_of(bad)
    f = dsbd.Forest.from_device(1, 1, 2, 1, dict(req_beam_off=torch.tensor([0, 1], dtype=I32, device="cuda"),
                                                beam_node_off=torch.tensor([0, 2], dtype=I32, device="cuda"),
                                                parent=torch.tensor([-1, -1], dtype=I32, device="cuda"),
                                                token=torch.zeros(2, dtype=I32, device="cuda")), 2, 1, 1)
    prefix = torch.tensor([0, 10], device="cuda")
    return {"rotate": (lambda s: dsbd.rotate_qk(q, k, position, dsbd.Rope(table), stream=s)[2], 7),
            "positions": (lambda s: dsbd.forest_positions(f, prefix, stream=s)[1], 4),
            "append": (lambda s: dsbd.kv_append_paged(c, k, v, p["k_pool"], p["v_pool"], stream=s)[1], 7),
            "attend": (lambda s: dsbd.chunk_attention_paged(c, 4, 2, 128, 0.1, q, p["k_pool"], p["v_pool"], stream=s)[1], 7)}


@pytest.mark.parametrize("name", ["rotate", "positions", "append", "attend"])
def test_what_a_call_reports_is_not_cleared_behind_it(name):
    """The current stream is busy: a status word that it is to clear is cleared when the call has long reported."""
    call, code = _calls()[name]
    side = torch.cuda.Stream()
    assert int(call(None).item()) == code                    # (the kernels are loaded)
    torch.cuda.synchronize()
    torch.cuda._sleep(BUSY)
    status = call(side)
    torch.cuda.synchronize()
    assert int(status.item()) == code


def test_a_workspace_is_not_given_to_the_current_stream_while_the_call_waits():
    """The side stream is busy when the call is made, so its kernels run later; what the current stream allocates and fills meanwhile
    stays as it is, and so does the result."""
    p = paged_problem([40, 300, 7], [9000, 700, 6000], 2, 128, BF, seed=16)
    q = p["randn"](p["T"], 8, 128)
    c = chunk_of(p)
    need = dsbd.chunk_attention_workspace(c, 8, 2, 128, BF, 128 ** -0.5)
    out = torch.empty_like(q)
    status = torch.zeros(1, dtype=I32, device="cuda")
    dsbd.chunk_attention_paged(c, 8, 2, 128, 128 ** -0.5, q, p["k_pool"], p["v_pool"], out=out, status=status)
    torch.cuda.synchronize()
    want = out.clone()
    out.zero_()
    torch.full((16,), 77, dtype=torch.uint8, device="cuda")              # (a kernel's first use waits for the device)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
    dsbd.chunk_attention_paged(c, 8, 2, 128, 128 ** -0.5, q, p["k_pool"], p["v_pool"], out=out, status=status, stream=side)
    mine = [torch.full((need,), 77, dtype=torch.uint8, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert all(bool((m == 77).all()) for m in mine)
    assert int(status.item()) == 0 and torch.equal(out, want)
    ref, mass = attention_reference(q, p, 128 ** -0.5)
    assert torch.all((out.double() - ref).abs() <= attention_bar(mass))


def test_outputs_on_another_stream():
    p = paged_problem([33, 1], [0, 7], 2, 128, BF, seed=3)
    rope = dsbd.Rope(dsbd.rope_table(64, 128))
    k, v, q = p["randn"](34, 2, 128), p["randn"](34, 2, 128), p["randn"](34, 4, 128)
    c = chunk_of(p)

    def chain(stream):
        qo, _ = dsbd.kv_append_paged(c, k, v, p["k_pool"], p["v_pool"], rope=rope, q=q, stream=stream)
        out, st = dsbd.chunk_attention_paged(c, 4, 2, 128, 0.1, qo, p["k_pool"], p["v_pool"], stream=stream)
        return out, st

    want, _ = chain(None)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda._sleep(BUSY)
    for _ in range(3):
        got, st = chain(side)
        side.synchronize()
        assert int(st.item()) == 0 and torch.equal(got, want)
