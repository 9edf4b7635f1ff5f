"""Calls from two host threads at once, whose rows want different shared memory of the same kernels."""
import ctypes as C
import threading

import pytest
import torch

import paper_2409_16560_b200 as dsbd
import rows_util as ru
from paper_2409_16560_b200.binding import DTYPE_F32, DistillParamsT, RowsT, SampleParamsT

pytestmark = pytest.mark.gpu
F32, I32 = torch.float32, torch.int32


class Calls:
    """A top-p draw and a loss with its gradient of one row of V logits on a stream of their own, through the C ABI with arguments made once, so that the
    threads spend their time in the library."""

    def __init__(self, V, seed):
        z = ru.rows_of(1, V, F32, seed=seed).contiguous()
        value, index, rest, _ = dsbd.top_logits(ru.rows_of(1, V, F32, seed=seed + 1), 8)
        e = lambda *s, dtype=F32: torch.zeros(*s, dtype=dtype, device="cuda")
        self.out = dict(token=e(1, 3, dtype=I32), logp=e(1, 3), loss=e(1), grad=e(1, V), status=e(1, dtype=I32))
        o = {n: t.data_ptr() for n, t in self.out.items()}
        u = torch.rand(1, 3, device="cuda", generator=torch.Generator("cuda").manual_seed(seed))
        self.stream = torch.cuda.Stream()
        rows = RowsT(z.data_ptr(), V, 1, V, DTYPE_F32)
        draw = SampleParamsT(1.0, 0.9, 0.0, 0, None, None, None, None, 3)
        fit = DistillParamsT(8, 1.0, value.data_ptr(), index.data_ptr(), rest.data_ptr(), None)
        self.kept = (z, u, value, index, rest, rows, draw, fit)
        at, s = C.addressof, self.stream.cuda_stream
        self.sample = (at(rows), at(draw), u.data_ptr(), o["token"], o["logp"], o["status"], s)
        self.distill = (at(rows), at(fit), o["loss"], o["grad"], V, o["status"], s)

    def run(self, times):
        lib = dsbd.load()
        for i in range(times):
            for rc in (lib.dsbd_sample_rows(*self.sample), lib.dsbd_distill(*self.distill)):
                if rc:
                    raise dsbd.DsbdError("call %d" % i, rc)
            if i % 100 == 99:
                self.stream.synchronize()


@pytest.mark.parametrize("lengths", [(2000, 393216), (128256, 393216), (20000, 128256)])
def test_two_threads_with_rows_of_different_length(lengths):
    both = [Calls(V, seed) for seed, V in enumerate(lengths)]
    torch.cuda.synchronize()
    for c in both:
        c.run(1)
    torch.cuda.synchronize()
    want = [{n: t.clone() for n, t in c.out.items()} for c in both]
    torch.cuda.synchronize()
    raised, start = [], threading.Barrier(2)

    def work(c):
        try:
            start.wait(10)
            c.run(3000)
        except Exception as e:                                 # (the main thread reports it)
            raised.append(e)
    threads = [threading.Thread(target=work, args=(c,)) for c in both]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not raised, raised
    for c, w in zip(both, want):
        assert all(torch.equal(c.out[n], w[n]) for n in w)
