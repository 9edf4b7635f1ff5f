"""The example's chain from prompts to a verified step: the logits that the large model gives a forest's nodes (prompt in two chunks,
rotated nodes, forest attention) have to be those of the same tokens read as one prompt (appended, chunk attention), and
the caches that the step leaves those of reading the output beams."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def _path(parent, n):
    p = [n]
    while parent[p[-1]] >= 0:
        p.append(parent[p[-1]])
    return p[::-1]


def test_forest_logits_are_those_of_the_same_tokens_as_a_prompt():
    import prompt_to_step as ex
    r = ex.run()
    assert r["status"] == 0
    large, f = r["large"], r["forest"]
    parent, tokens, bno = (x.cpu().numpy() for x in (f.dev["parent"], r["tokens"], f.dev["beam_node_off"]))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def read_alone(text):
        """Logits behind the text's last token, read from an empty cache at once; keys of all layers."""
        need = r["need"](len(text))
        m = object.__new__(type(large))
        m.__dict__.update(large.__dict__, k_pool=torch.zeros_like(large.k_pool), v_pool=torch.zeros_like(large.v_pool))
        z = m.read(torch.as_tensor(np.asarray(text)).cuda(), ex.chunk([len(text)], [0], [list(range(need))]), status)
        cache = lambda pool: pool[:, :need].permute(0, 1, 3, 2, 4).flatten(1, 2)[:, :len(text)].float()
        return z[-1], cache(m.k_pool), cache(m.v_pool)

    # Two bf16 models that differ in the rounding of two layers' activations (2^-8 each) and of the attention's weights: logits of standard
    # deviation 3 that are sums of 256 products agree to a few hundredths; a wrong position, mask or page moves them by ones.
    for b in range(len(bno) - 1):
        for n in (int(bno[b]), int(bno[b + 1]) - 1, (int(bno[b]) + int(bno[b + 1])) // 2):
            text = np.concatenate([r["prompts"][b][:-1], tokens[_path(parent, n)]])
            z, _, _ = read_alone(text)
            err = (z - r["zp"][n]).abs()
            assert float(err.mean()) < 0.06 and float(err.max()) < 0.5, (b, n, float(err.mean()), float(err.max()))
    # the kept beams' caches
    c, out = r["commit"], {k: v.cpu().numpy() for k, v in r["out"].items()}
    poff, pgoff, table = (c[k].cpu().numpy() for k in ("new_prefix_off", "new_page_off", "new_page_table"))
    slots = c["new_beam_slot"].cpu().numpy()
    kept = [int(s) for s in slots if s >= 0]
    assert kept
    for j, s in enumerate(kept):
        text = np.concatenate([r["prompts"][out["out_root_beam"][s]][:-1], tokens[_path(parent, out["out_parent"][s])]])
        assert poff[j + 1] - poff[j] == len(text)
        _, k, v = read_alone(text)
        pages = table[pgoff[j]:pgoff[j + 1]]
        for pool, want in ((large.k_pool, k), (large.v_pool, v)):
            got = pool[:, torch.as_tensor(pages).long().cuda()].permute(0, 1, 3, 2, 4).flatten(1, 2)[:, :len(text)].float()
            assert float((got - want).abs().mean()) < 0.02 and float((got - want).abs().max()) < 0.5
    assert int(status.item()) == 0
