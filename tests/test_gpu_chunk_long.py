"""Attention of a chunk behind long caches, on values with which every page counts: page i of a sequence holds ones in column
i mod d and zeros elsewhere, so a column of the result is the weight of a few pages.  With values of random signs the result of a long
cache is small beside the bar, and a page or a run of pages less would go unnoticed; here the test shows that it would not."""
import pytest
import torch

import paper_2409_16560_b200 as dsbd
from chunk_util import PAGE, attention_bar, attention_reference, cache_of, chunk_of, paged_problem

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _one_hot_pages(p, d):
    p["v_pool"].zero_()
    for b in range(len(p["new"])):
        pages = torch.as_tensor(p["table_host"][p["page_off_host"][b]:p["page_off_host"][b + 1]]).long().cuda()
        p["v_pool"][pages, :, :, torch.arange(len(pages), device="cuda") % d] = 1.0


def _page_weights(p, q, b, row, head, group, scale):
    """Weights of the pages that a row sees, in 64 bits."""
    n = int(p["old"][b]) + row + 1
    k = cache_of(p["k_pool"], p, b, n)[:, head // group].double()
    w = torch.softmax(k @ q[int(p["new_off_host"][b]) + row, head].double() * scale, 0)
    return torch.nn.functional.pad(w, (0, -n % PAGE)).view(-1, PAGE).sum(1)


# (new, old, Hkv): units of hundreds of pages, cut into dozens of parts (the 70000 tokens into all the runs of a call, so that the
# join takes several rounds of 32), wide blocks behind more pages than a warp holds ids of, and short units among them
CASES = {"tokens": ([1, 5], [9000, 20000], 2), "one": ([3], [70000], 1), "wide": ([300, 1], [9000, 40], 2),
         "blocks": ([700], [2500], 4), "among": ([1, 2, 130, 1], [30000, 64, 4000, 130], 2)}


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", list(CASES))
@pytest.mark.parametrize("even", [True, False])
def test_every_page_counts(case, even, d):
    new, old, Hkv = CASES[case]
    Hq = 4 * Hkv
    p = paged_problem(new, old, Hkv, d, BF, seed=41)
    _one_hot_pages(p, d)
    q = p["randn"](p["T"], Hq, d)
    if even:
        q.zero_()
    out, st = dsbd.chunk_attention_paged(chunk_of(p), Hq, Hkv, d, d ** -0.5, q, p["k_pool"], p["v_pool"])
    assert int(st.item()) == 0
    ref, mass = attention_reference(q, p, d ** -0.5)
    # even: all weights are 1 and every sum is a whole number below 2^24, so there are a reciprocal, a product and the output's rounding
    bar = (2.0 ** -8 + 2.0 ** -21) * ref if even else attention_bar(mass)
    err = (out.double() - ref).abs()
    assert torch.all(err <= bar), float((err - bar).max())
    # a page that is left out puts its column over the bar, by more than the rounding of that result could take back
    for b in range(len(new)):
        for row, head in ((new[b] - 1, 0), (0, Hq - 1)):
            w = _page_weights(p, q, b, row, head, Hq // Hkv, d ** -0.5)
            column = torch.arange(len(w), device="cuda") % d
            whole = torch.zeros(d, dtype=torch.float64, device="cuda").index_add_(0, column, w)[column]
            if len(w) == 1:
                continue
            without = (whole - w) / (1 - w)
            at = bar[int(p["new_off_host"][b]) + row, head][column]
            seen = w > 1e-2 / len(w)                          # (the last page may hold a token or two)
            assert torch.all(((whole - without).abs() > at + 2.0 ** -7 * without)[seen]) and seen.sum() >= len(w) - 1
