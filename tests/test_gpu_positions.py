"""Positions of a forest's nodes: behind the kernel that builds the forest, and of large trees."""
import numpy as np
import pytest
import torch

import paper_2409_16560_b200 as dsbd

pytestmark = pytest.mark.gpu


def test_positions_right_behind_the_build():
    """Nothing waits between the build and the positions, and the arrays are the same memory again and again, with other trees."""
    R, gamma, W_S = 32, 6, 12
    rng = np.random.default_rng(0)
    rbo = torch.arange(R + 1, dtype=torch.int32, device="cuda")
    L = rng.integers(0, 5000, R)
    prefix_off = torch.as_tensor(np.concatenate([[0], np.cumsum(L)])).cuda()
    token = torch.zeros(gamma, R * W_S, dtype=torch.int32, device="cuda")
    draws, results = [], []
    for _ in range(20):
        parent = np.empty((gamma, R * W_S), np.int32)
        parent[0] = np.repeat(np.arange(R), W_S)
        for l in range(1, gamma):
            parent[l] = np.repeat(np.arange(R), W_S) * W_S + rng.integers(0, W_S, R * W_S)
        draws.append(torch.as_tensor(parent).cuda())
    torch.cuda.synchronize()
    for d in draws:
        f, node_of_draw, status = dsbd.forest_build(rbo, np.arange(R + 1), gamma, W_S, d, token)
        position, status = dsbd.forest_positions(f, prefix_off, status=status)
        results.append((position[node_of_draw.long().flatten()].view(gamma, -1), status))
    want = np.repeat(L, W_S)[None, :] + np.arange(1, gamma + 1)[:, None]
    for got, status in results:
        assert int(status.item()) == 0 and np.array_equal(got.cpu().numpy(), want)
