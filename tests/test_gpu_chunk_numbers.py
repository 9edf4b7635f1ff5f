"""What numbers in the cache do to the attention of a chunk: keys that are not finite at positions that a row sees."""
import pytest
import torch

import paper_2409_16560_b200 as dsbd
from chunk_util import PAGE, attention_bar, attention_reference, chunk_of, paged_problem

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _attend(p, q, Hkv, scale):
    out, st = dsbd.chunk_attention_paged(chunk_of(p), q.shape[1], Hkv, q.shape[2], scale, q, p["k_pool"], p["v_pool"])
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    return out


def _place(p, b, position):
    """Page and row of a position of sequence b."""
    return int(p["table_host"][p["page_off_host"][b] + position // PAGE]), position % PAGE


# (new, old): whole units, single tokens and chunks; units that are cut between CTAs, the same
SHAPES = {"whole": ([1, 70, 3], [130, 64, 65]), "cut": ([1, 300, 2], [5000, 3000, 9000])}


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_a_key_that_is_no_number_reaches_every_row_that_sees_it(shape, d):
    """One key with a NaN, at each of the 64 slots of a page in turn: NaN for the query heads of its KV head and the tokens that
    see it, the bits of before for all others."""
    Hq, Hkv = 8, 2
    new, old = SHAPES[shape]
    p = paged_problem(new, old, Hkv, d, BF, seed=d)
    q = p["randn"](p["T"], Hq, d)
    want = _attend(p, q, Hkv, d ** -0.5)
    for slot in range(PAGE):
        b = slot % 3
        position = (old[b] // PAGE - (slot // 3) % 2) * PAGE + slot          # the last page that was cached, or the one before
        position = min(max(position, 0), old[b] + new[b] - 1) // PAGE * PAGE + slot
        if position >= old[b] + new[b]:
            position -= PAGE
        page, row = _place(p, b, position)
        g = slot % Hkv
        keep = p["k_pool"][page, g, row].clone()
        p["k_pool"][page, g, row, (7 * slot) % d] = float("nan")
        got = _attend(p, q, Hkv, d ** -0.5)
        p["k_pool"][page, g, row] = keep
        hit = torch.zeros(p["T"], Hq, dtype=torch.bool, device="cuda")
        first = int(p["new_off_host"][b])
        sees = max(position - old[b], 0)                                     # the first token of the chunk that sees it
        hit[first + sees:first + new[b], g * (Hq // Hkv):(g + 1) * (Hq // Hkv)] = True
        assert hit.any()
        assert torch.isnan(got[hit]).all(), (slot, position)
        assert torch.equal(got[~hit], want[~hit]), (slot, position)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_infinite_keys(shape, d):
    """Keys with infinities give logits of +inf (NaN out), -inf (weight 0) or inf - inf (NaN), as in 64 bits."""
    Hq, Hkv = 8, 2
    new, old = SHAPES[shape]
    p = paged_problem(new, old, Hkv, d, BF, seed=d + 1)
    q = p["randn"](p["T"], Hq, d)
    kinds = set()
    for i in range(16):
        b = i % 3
        position = (old[b] // PAGE - 1) * PAGE + 4 * (i // 2) + i // 4       # (at most 34: over two sixteens of slots and more)
        page, row = _place(p, b, position)
        keep = p["k_pool"][page, :, row].clone()
        p["k_pool"][page, :, row, 3] = float("inf")
        if i % 2:
            p["k_pool"][page, :, row, 9] = float("-inf")
        got = _attend(p, q, Hkv, d ** -0.5)
        ref, mass = attention_reference(q, p, d ** -0.5)
        p["k_pool"][page, :, row] = keep
        bad = torch.isnan(ref)
        assert torch.equal(torch.isnan(got), bad), (i, position)
        assert torch.all(((got.double() - ref).abs() <= attention_bar(mass))[~bad]), (i, position)
        r = slice(int(p["new_off_host"][b]), int(p["new_off_host"][b + 1]))
        kinds |= {bool(x) for x in bad[r].flatten()[:: max(bad[r].numel() // 4096, 1)]}
    assert kinds == {True, False}


def _constant_values(p, q, Hkv, scale, c):
    p["v_pool"].fill_(c)
    return _attend(p, q, Hkv, scale)


# Just below 2 and 1: the neighbour above 255/128 is 2, half a step of 2^-8 = 1.96e-3 away; the one below 1 is 2^-9 away.
CONSTANTS = (255 / 128, 1.0, -1.0, -255 / 128)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lengths", [([300], [0]), ([1, 40, 2], [3000, 700, 20000]), ([1] * 20, [40 + 50 * i for i in range(20)])])
def test_values_that_are_all_alike_come_back(lengths, d):
    """Weights that sum to one give back a value that all positions share.  The weights are rounded to bf16 for the product; when the
    row sum adds those same rounded weights the rounding cancels, and what is left are fp32 sums of up to 20002 terms of one
    sign, errors of a random walk: sqrt(20002) 2^-24 < 1e-5, far below the half step of 1.95e-3 to a neighbouring bf16, so
    the result is exact.  A sum of the weights before their rounding is off by up to 3.9e-3 where a row's weights round alike."""
    new, old = lengths
    p = paged_problem(new, old, 2, d, BF, seed=31)
    for peak in (1.0, 6.0):                                   # broad rows, and rows of one or two heavy weights
        q = (p["randn"](p["T"], 8, d).float() * peak).to(BF)
        for c in CONSTANTS:
            out = _constant_values(p, q, 2, d ** -0.5, c)
            assert torch.all(out == c), (peak, c, float((out.float() - c).abs().max()))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("weight", [0.50205, 0.50185, 0.2511, 0.2508, 0.7285])
def test_equal_weights_beside_a_heavier_one(weight, d):
    """The first key of a sequence is the maximum, all others have the same weight just off the middle between two bf16 values (at
    0.50205 it rounds up by 3.7e-3 of itself, at 0.50185 down by as much)."""
    import math
    for new, old in (([70], [300]), ([1, 1], [2000, 6000])):
        p = paged_problem(new, old, 1, d, BF, seed=1)
        q = torch.zeros(p["T"], 4, d, dtype=BF, device="cuda")
        q[..., 0] = 1.0
        p["k_pool"].zero_()
        p["k_pool"][..., 0] = -1.0
        for b in range(len(new)):
            page, row = _place(p, b, 0)
            p["k_pool"][page, :, row, 0] = 0.0
        for c in CONSTANTS:
            out = _constant_values(p, q, 1, -math.log(weight), c)
            assert torch.all(out == c), (c, float((out.float() - c).abs().max()))
