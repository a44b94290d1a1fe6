"""Tree attention over long sequences as the planner cuts them by itself: eight blocks of a cluster, pieces through the
workspace, and items of dozens of tiles in blocks that take over work, so that rings and buffers go round many times."""
import numpy as np
import pytest
import torch

from tests.test_gpu_tree import Setup, dsa  # noqa: F401  (dsa: the module's fixture)

pytestmark = pytest.mark.gpu


def _workspace(dsa, s):  # noqa: F811
    return dsa.dsa_tree_workspace_size(s.problem, s.diag, s.tree)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window", [0, 700])
@pytest.mark.parametrize("page", [0, 16, 48])
@pytest.mark.parametrize("lens,hkv", [((1100,), 1), ((4000,), 2), ((2049, 1), 2)])
def test_clusters(dsa, d, window, page, lens, hkv):  # noqa: F811
    s = Setup(dsa, d=d, hq=4 * hkv, hkv=hkv, n=7, lens=lens, window=window, sinks=4, page=page)
    assert _workspace(dsa, s) == 0                                 # (merged on chip)
    s.check(*s.run())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window", [0, 8300])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("length,hkv", [(8300, 2), (9001, 1), (12345, 1)])
def test_pieces_through_the_workspace(dsa, d, window, page, length, hkv):  # noqa: F811
    s = Setup(dsa, d=d, hq=2 * hkv, hkv=hkv, n=5, lens=(length,), window=window, sinks=3, page=page)
    assert _workspace(dsa, s) > 0                                  # (eight blocks would be too few)
    s.check(*s.run())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,page", [(0, 16), (0, 0), (1500, 16)])
def test_long_items_in_blocks_that_take_over(dsa, d, window, page):  # noqa: F811
    """More items than places, most of them short: a block's few long ones run through its rings again and again."""
    rng = np.random.default_rng(d)
    lens = [int(x) for x in rng.integers(0, 150, size=40)]
    for r, length in ((0, 2111), (7, 3000), (22, 2500), (39, 2048)):
        lens[r] = length
    counts = [int(x) for x in rng.integers(0, 5, size=40)]
    counts[0] = counts[7] = counts[22] = counts[39] = 4
    s = Setup(dsa, d=d, hq=8, hkv=8, n=4, lens=lens, counts=counts, window=window, sinks=3, page=page)
    assert _workspace(dsa, s) == 0
    s.check(*s.run())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("batch,hkv,length", [(1, 2, 3000), (1, 1, 9000), (20, 16, 2200)])
@pytest.mark.parametrize("rising", [True, False])
def test_logits_that_keep_growing(dsa, d, batch, hkv, length, rising):  # noqa: F811
    """Keys that grow along the sequence: the maximum moves, and O is rescaled, in late tiles and in every piece (or, turned
    round, in the first ones only)."""
    lens = [length if r in (0, batch - 1) else 40 + r for r in range(batch)]
    s = Setup(dsa, d=d, hq=hkv, hkv=hkv, n=3, lens=lens, page=16, seed=2)
    for r in (0, batch - 1):
        pos = torch.arange(length)
        size = 0.05 + 4.0 * (pos if rising else length - 1 - pos) / length
        for i in range(length):
            o, t = s.place(r, i)
            s.full[0][o, t] *= size[i]
    s.dev_full[0].copy_(s.full[0])
    s.check(*s.run())
