"""What the binding of the rotation, the positions, the append and the chunk attention refuses before anything reaches the library (which
is replaced here by one that only tells that it was called)."""
import numpy as np
import pytest
import torch

import paper_2409_16560_b200 as dsbd
from chunk_util import chunk_of, paged_problem
from paper_2409_16560_b200 import binding

pytestmark = pytest.mark.gpu
BF, I32, I64 = torch.bfloat16, torch.int32, torch.int64


class Reached(Exception):
    pass


class _Library:
    def __getattr__(self, name):
        def call(*args):
            raise Reached(name)
        return call


@pytest.fixture
def no_library(monkeypatch):
    monkeypatch.setattr(binding, "load", lambda: _Library())


def _chain(device="cuda"):
    return dsbd.Forest(dict(R=1, B=2, N=5, max_depth=2, req_beam_off=[0, 2], beam_node_off=[0, 3, 5], parent=[-1, 0, 1, -1, 3],
                            token=np.zeros(5)), device)


PREFIX = [0, 10, 30]


def test_positions_want_offsets_and_outputs_of_their_types_on_the_device(no_library):
    prefix = torch.tensor(PREFIX, device="cuda")
    with pytest.raises(Reached):
        dsbd.forest_positions(_chain(), prefix)
    for bad in (prefix.to(I32), prefix[:2], torch.cat([prefix, prefix]), prefix.cpu(), prefix.double()):
        with pytest.raises((AssertionError, RuntimeError)):
            dsbd.forest_positions(_chain(), bad)
    position = torch.zeros(5, dtype=I32, device="cuda")
    with pytest.raises(Reached):
        dsbd.forest_positions(_chain(), prefix, position=position)
    for bad in (position.cpu(), position.to(I64), position[:4]):
        with pytest.raises((AssertionError, RuntimeError)):
            dsbd.forest_positions(_chain(), prefix, position=bad)
    with pytest.raises((AssertionError, RuntimeError)):
        dsbd.forest_positions(_chain("cpu"), prefix)


def _calls():
    """The four device operators, as functions of the status tensor."""
    p = paged_problem([2, 3], [10, 0], 2, 128, BF, seed=3)
    q, k, v = p["randn"](5, 4, 128), p["randn"](5, 2, 128), p["randn"](5, 2, 128)
    c, position, prefix = chunk_of(p), torch.zeros(5, dtype=I32, device="cuda"), torch.tensor(PREFIX, device="cuda")
    rope = dsbd.Rope(torch.zeros(8, 2, 64, device="cuda"))
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    return {"rotate": lambda s: dsbd.rotate_qk(q, k, position, rope, status=s),
            "positions": lambda s: dsbd.forest_positions(_chain(), prefix, status=s),
            "append": lambda s: dsbd.kv_append_paged(c, k, v, p["k_pool"], p["v_pool"], status=s),
            "attend": lambda s: dsbd.chunk_attention_paged(c, 4, 2, 128, 0.1, q, p["k_pool"], p["v_pool"], workspace=ws, status=s)}


@pytest.mark.parametrize("name", ["rotate", "positions", "append", "attend"])
def test_a_status_word_is_an_int32_on_the_device(no_library, name):
    call = _calls()[name]
    status = torch.zeros(1, dtype=I32, device="cuda")
    with pytest.raises(Reached):
        call(status)
    for bad in (status.cpu(), status.to(I64), status.to(torch.uint8), status[:0]):
        with pytest.raises((AssertionError, RuntimeError)):
            call(bad)


def test_the_attention_wants_its_workspace_on_the_device_and_in_one_piece(no_library):
    p = paged_problem([2, 3], [10, 0], 2, 128, BF, seed=3)
    q, c = p["randn"](5, 4, 128), chunk_of(p)
    call = lambda w: dsbd.chunk_attention_paged(c, 4, 2, 128, 0.1, q, p["k_pool"], p["v_pool"], workspace=w)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    with pytest.raises(Reached):
        call(ws)
    for bad in (ws.cpu(), ws.view(1024, 1024)[:, ::2], ws.expand(2, -1)):
        with pytest.raises((AssertionError, RuntimeError)):
            call(bad)
