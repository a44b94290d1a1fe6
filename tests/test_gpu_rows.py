"""Token maps and row copies (dsa_map_tokens, dsa_store_rows, dsa_gather_rows) against plain Python, byte by byte."""
import random

import pytest
import torch

from tests import latent_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dsa():
    from paper_2609_19702_b200 import binding
    return binding


def run_map(dsa, count, base, table, page, blocks, room, n, outputs=3):
    dev = lambda x, t=torch.int32: None if x is None else torch.tensor(x, dtype=t).cuda()  # noqa: E731
    start = torch.full((len(count) + 1,), 7, dtype=torch.int32).cuda()
    slot = torch.full((n,), 7, dtype=torch.int64).cuda()
    position, request = torch.full((n,), 7, dtype=torch.int32).cuda(), torch.full((n,), 7, dtype=torch.int32).cuda()
    dsa.dsa_map_tokens(dev(count).view(-1), start, slot, position if outputs > 1 else None, request if outputs > 2 else None,
                       base=dev(base), block_table=dev(table), block_size=page, num_blocks=blocks, max_seq_len=room)
    want = latent_ref.map_expected(count, base, table, page, blocks, room, n)
    assert start.tolist() == want[0]
    assert slot.tolist() == want[1]
    if outputs > 1:
        assert position.tolist() == want[2]
    if outputs > 2:
        assert request.tolist() == want[3]


def test_map_small(dsa):
    run_map(dsa, [1], [5], [[2, 0]], 4, 3, 8, 1)
    run_map(dsa, [0, 3, -2, 0, 2], [9, 2, 0, 1, 6], [[0, 1, 2], [3, 4, 5], [6, 7, 8], [0, 0, 0], [9, 9, 10]], 3, 11, 9, 12)
    run_map(dsa, [2, 2], [0, 1], None, 0, 0, 10, 4, outputs=1)
    run_map(dsa, [4, 4], None, None, 0, 0, 3, 8, outputs=2)                          # the last ones have no room
    run_map(dsa, [3], [-2], [[0]], 2, 1, 2, 3)                                       # positions below 0
    run_map(dsa, [4], [0], [[0, -1]], 2, 1, 4, 4)                                    # a page that is missing
    run_map(dsa, [4], [0], [[5, 1]], 2, 2, 4, 4)                                     # and one outside the pool
    run_map(dsa, [5, 5], [0, 0], [[0, 1], [2, 3]], 4, 4, 8, 7)                       # more tokens than entries
    run_map(dsa, [5, 5], [0, 0], [[0, 1], [2, 3]], 4, 4, 8, 0)
    run_map(dsa, [], None, None, 0, 0, 8, 5)                                         # no requests
    run_map(dsa, [0, 0], [1, 1], [[0], [1]], 4, 2, 4, 3)


@pytest.mark.parametrize("batch,page,most", [(1, 16, 5000), (300, 16, 40), (1000, 5, 7), (8192, 1, 2), (17, 64, 700)])
def test_map_ragged(dsa, batch, page, most):
    rng = random.Random(batch)
    count = [rng.choice([0, 1, rng.randrange(0, most + 1)]) for _ in range(batch)]
    base = [rng.randrange(0, 100) for _ in range(batch)]
    room = most + 90
    per = -(-room // page)
    blocks = batch * per
    ids = list(range(blocks))
    rng.shuffle(ids)
    table = [ids[b * per:(b + 1) * per] for b in range(batch)]
    run_map(dsa, count, base, table, page, blocks, room, sum(count) + 3)


def test_slots_beyond_32_bits(dsa):
    """Pages whose slots pass 2^31: the numbers only, no such cache."""
    run_map(dsa, [3], [70], [[0, 2 ** 30]], 64, 2 ** 30 + 1, 128, 4)


def _latent(dsa, dtype, blocks, page, width, paged, latent, pad=0):
    cache = torch.randn((blocks, page, width + pad), dtype=torch.float32).to(dtype).cuda()
    seq = torch.zeros((blocks,), dtype=torch.int32).cuda()
    return cache, dsa.Latent(cache, strides=(cache.stride(0), cache.stride(1)), seq_len=seq, latent_dim=latent, rope_dim=width - latent,
                             max_seq_len=page, sm_scale=1.0, block_table=torch.zeros((blocks, 1), dtype=torch.int32).cuda() if paged else None,
                             block_size=page if paged else 0, num_blocks=blocks if paged else 0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("paged", [True, False])
@pytest.mark.parametrize("count,latent,rope,pad,ld", [(1, 512, 64, 0, 0), (0, 512, 64, 0, 0), (15, 256, 32, 0, 0), (17, 256, 8, 16, 0), (700, 512, 24, 8, 40)])
def test_store_and_gather(dsa, dtype, paged, count, latent, rope, pad, ld):
    torch.manual_seed(count)
    blocks, page, width = 67, 12, latent + rope
    cache, lat = _latent(dsa, dtype, blocks, page, width, paged, latent, pad)
    slot = torch.randperm(blocks * page)[:count]
    slot[::5] = torch.tensor([-1, -2 ** 40, blocks * page, 2 ** 40])[torch.arange(len(slot[::5])) % 4]
    rows = torch.randn((count, width + ld)).to(dtype).cuda()[:, :width]
    want = cache.clone()
    for t, s in enumerate(slot.tolist()):
        if 0 <= s < blocks * page:
            want[s // page, s % page, :width] = rows[t]
    dsa.dsa_store_rows(lat, slot.cuda(), rows)
    assert torch.equal(cache, want)
    back = torch.randn((count, width + ld)).to(dtype).cuda()[:, :width]
    want = back.clone()
    for t, s in enumerate(slot.tolist()):
        if 0 <= s < blocks * page:
            want[t] = cache[s // page, s % page, :width]
    dsa.dsa_gather_rows(lat, slot.cuda(), back)
    assert torch.equal(back, want)


def test_rows_beyond_32_bits(dsa):
    """A cache of more than 2^32 bytes, its last slots among those used."""
    blocks, page, width = 70000, 64, 512 + 64
    cache = torch.zeros((blocks, page, width), dtype=torch.bfloat16, device="cuda")
    lat = dsa.Latent(cache, strides=(cache.stride(0), cache.stride(1)), seq_len=torch.zeros((1,), dtype=torch.int32).cuda(), latent_dim=512,
                     rope_dim=64, max_seq_len=page, sm_scale=1.0, block_table=torch.zeros((1, 1), dtype=torch.int32).cuda(), block_size=page,
                     num_blocks=blocks)
    slot = torch.tensor([blocks * page - 1, 0, 2 ** 22 + 5], dtype=torch.int64).cuda()
    rows = torch.randn((3, width), device="cuda").bfloat16()
    dsa.dsa_store_rows(lat, slot, rows)
    assert torch.equal(cache[-1, -1], rows[0]) and torch.equal(cache[0, 0], rows[1])
    assert torch.equal(cache[(2 ** 22 + 5) // page, (2 ** 22 + 5) % page], rows[2])
    back = torch.zeros_like(rows)
    dsa.dsa_gather_rows(lat, slot, back)
    assert torch.equal(back, rows)
