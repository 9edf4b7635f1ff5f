"""The calls of a decode step, given a stream other than the current one, make everything that they make on that stream (the library is
replaced by one that launches nothing)."""
import pytest
import torch

import paper_2409_16560_b200 as dsbd
from paper_2409_16560_b200 import binding

pytestmark = pytest.mark.gpu
I32, I64, F32 = torch.int32, torch.int64, torch.float32


class _Library:
    def __getattr__(self, name):
        return lambda *args: 256 if name.endswith("_workspace") else 0


@pytest.fixture
def made(monkeypatch):
    """The current streams at every allocation that the binding makes."""
    streams = []
    monkeypatch.setattr(binding, "load", lambda: _Library())
    for name in ("empty", "zeros", "full", "empty_like", "zeros_like", "full_like"):
        real = getattr(torch, name)
        monkeypatch.setattr(torch, name, lambda *a, _real=real, **kw: (streams.append(torch.cuda.current_stream()), _real(*a, **kw))[1])
    return streams


def _t(*values, dtype=I32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _calls():
    f = dsbd.Forest(dict(R=1, B=1, N=2, max_depth=1, req_beam_off=[0, 1], beam_node_off=[0, 2], parent=[-1, 0], token=[0, 1]), "cuda")
    prm = dict(V=8)
    z = torch.randn(2, 8, device="cuda")
    node = torch.randn(2, 4, 64, device="cuda")
    prefix, prefix_dev = [0, 3], _t(0, 3, dtype=I64)
    pool, pages, page_off = torch.randn(2, 4, 64, 64, device="cuda"), _t(0), _t(0, 1, dtype=I64)
    outs = (_t(0, 1), _t(1), _t(0), _t(0), torch.zeros(1, device="cuda"))
    out = dsbd.alloc_verify_out(f, [0, 2], "cuda")
    one = torch.zeros(1, device="cuda")
    return {
        "forest_attention": lambda s: dsbd.forest_attention(f, 4, 4, 64, 0.1, node, node, node, pool, pool, prefix_dev, prefix, stream=s),
        "forest_attention_paged": lambda s: dsbd.forest_attention_paged(f, 4, 4, 64, 0.1, node, node, node, pool, pool, pages, page_off,
                                                                        prefix_dev, prefix, stream=s),
        "forest_build": lambda s: dsbd.forest_build(_t(0, 1), [0, 1], 1, 1, _t(0).view(1, 1), _t(1).view(1, 1), stream=s, exact=True),
        "draft_layer": lambda s: dsbd.draft_layer(_t(0, 1), [0, 1], prm, 1, 1, z[:1], one, _t(0, 1), 1, stream=s),
        "kv_commit": lambda s: dsbd.kv_commit(f, 4, 64, *outs, node, node, pool, pool, prefix_dev, prefix, 1, 8, stream=s),
        "kv_commit_paged": lambda s: dsbd.kv_commit_paged(f, 4, 64, *outs, node, node, pool, pool, pages, page_off, prefix_dev, prefix,
                                                          _t(1), _t(1), 1, 4, stream=s),
        "verify_step": lambda s: dsbd.verify_step(f, prm, z, z, one, one, out, stream=s),
        "node_stats": lambda s: dsbd.node_stats(f, prm, z, z, stream=s),
        "select_width": lambda s: dsbd.select_width(f, prm, z, z, one, one, _t(0, 1), _t(0), _t(1), 4, stream=s),
    }


@pytest.mark.parametrize("name", ["forest_attention", "forest_attention_paged", "forest_build", "draft_layer", "kv_commit", "kv_commit_paged",
                                  "verify_step", "node_stats", "select_width"])
def test_everything_is_made_on_the_stream_of_the_call(made, name):
    call = _calls()[name]
    side = torch.cuda.Stream()
    made.clear()
    call(side)
    assert made and all(s == side for s in made)
    made.clear()
    call(None)
    assert made and all(s == torch.cuda.current_stream() for s in made)


def test_the_largest_tree_is_read_behind_the_build(monkeypatch):
    """exact=True reads the size of the largest tree back: of the call's own stream, which may be busy."""
    rbo, parent, token = _t(0, 1), _t(0, 0, 1, 1).view(2, 2), _t(1, 2, 3, 4).view(2, 2)
    want, _, _ = dsbd.forest_build(rbo, [0, 1], 2, 2, parent, token, exact=True)
    assert want.max_tree_nodes == 5
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
    got, _, status = dsbd.forest_build(rbo, [0, 1], 2, 2, parent, token, exact=True, stream=side)
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and got.max_tree_nodes == 5
