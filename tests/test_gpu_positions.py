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


def _forest(parents):
    """A forest of one request from each tree's parents (local numbers, -1 for the root)."""
    off = np.concatenate([[0], np.cumsum([len(p) for p in parents])]).astype(np.int32)
    parent = np.concatenate([np.where(np.asarray(p) >= 0, np.asarray(p) + o, -1) for p, o in zip(parents, off)]).astype(np.int32)
    dev = lambda a: torch.as_tensor(np.asarray(a, np.int32)).cuda()
    f = dsbd.Forest.from_device(1, len(parents), int(off[-1]), 1, dict(req_beam_off=dev([0, len(parents)]), beam_node_off=dev(off),
                                                                      parent=dev(parent), token=dev(np.zeros(off[-1]))), 1, 1, 1)
    return f, off, parent


def _depths(parent):
    depth = np.zeros(len(parent), np.int64)
    for i, p in enumerate(parent):
        depth[i] = depth[p] + 1 if p >= 0 else 0
    return depth


def test_large_trees():
    """Trees beyond those that fit in shared memory: chains of any length (a walk up from every node would take the square of it),
    bushes, and steps that jump over a few nodes, over 31, 32 and 33."""
    rng = np.random.default_rng(1)
    for trees in ([list(range(-1, 50000 - 1))], [list(range(-1, 1057 - 1)), [-1], list(range(-1, 4096 - 1))],
                  [[-1] + [int(rng.integers(0, i)) for i in range(1, 20000)], [-1, 0, 0]],
                  [[-1] + [max(i - s, 0) for i in range(1, 3000)] for s in (2, 7, 31, 32, 33, 64)],
                  [[-1] + [max(i - int(rng.integers(1, 40)), 0) for i in range(1, n)] for n in (1058, 2000, 5001)]):
        f, off, parent = _forest(trees)
        L = rng.integers(0, 5000, len(trees))
        prefix_off = torch.as_tensor(np.concatenate([[0], np.cumsum(L)])).cuda()
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        position, status = dsbd.forest_positions(f, prefix_off)
        end.record()
        assert int(status.item()) == 0
        assert np.array_equal(position.cpu().numpy(), np.repeat(L, np.diff(off)) + _depths(parent))
        assert begin.elapsed_time(end) < 50.0                 # 50000 nodes: 1563 steps of a microsecond or two


def test_large_trees_report_a_parent_outside():
    for node, bad in ((1, 1), (40, 40), (40, 1999), (40, 2500), (1999, -1), (0, 5), (64, -7), (100, 2 ** 31 - 1), (100, -2 ** 31)):
        f, off, parent = _forest([list(range(-1, 1999)), list(range(-1, 1999))])
        f.dev["parent"][node] = bad
        position, status = dsbd.forest_positions(f, torch.tensor([0, 10, 30]).cuda())
        assert int(status.item()) == 4, (node, bad)
        want = np.arange(2000)
        want[node:] -= node if node else 0                    # what hangs below the node counts from it
        assert position[:2000].tolist() == (10 + want).tolist(), (node, bad)
        assert position[2000:].tolist() == list(range(20, 2020))
