"""Attention of new tokens over a latent cache (dsa_latent_step) against a float64 reference, and every byte of the cache."""
import math

import pytest
import torch

from tests import latent_ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def dsa():
    from paper_2609_19702_b200 import binding
    return binding


class Case:
    """A batch on the host in its own type, and the same on the device: cache rows that no token may see are NaN."""

    def __init__(self, dtype, heads, new, lens, page, latent=512, rope=64, counts=None, seed=0, room=None, pad=0, spare=1):
        g = torch.Generator().manual_seed(seed)
        dt = DT[dtype]
        rand = lambda *s: torch.randn(s, generator=g).to(dt)  # noqa: E731
        self.dtype, self.heads, self.new, self.lens, self.page, self.latent, self.rope = dtype, heads, new, lens, page, latent, rope
        self.w, b = latent + rope, len(lens)
        self.room = room if room is not None else max(max(lens), 0) + new
        self.scale = 1.0 / math.sqrt(128 + rope)
        self.counts = counts
        self.q, self.c_new = rand(b, new, heads, self.w), rand(b, new, self.w)
        ld = self.w + pad
        if page:
            per = max(1, -(-self.room // page))
            self.blocks = b * per + spare
            self.table = torch.randperm(self.blocks, generator=g)[:b * per].view(b, per).to(torch.int32)
            self.cache = torch.full((self.blocks, page, ld), math.nan, dtype=dt)
        else:
            self.blocks, self.table = 0, None
            self.cache = torch.full((b, max(self.room, 1), ld), math.nan, dtype=dt)
        self.rows = []
        for r, s in enumerate(lens):
            s = max(0, min(s, self.room))
            rows = rand(s, self.w)
            self.rows.append(rows)
            for i in range(s):
                self.place(r, i)[:] = rows[i]
        self.n = []
        for r, s in enumerate(lens):
            n = new if counts is None else max(0, min(counts[r], new))
            self.n.append(0 if s < 0 else max(0, min(n, self.room - min(s, self.room))))

    def place(self, r, i, cache=None):
        cache = self.cache if cache is None else cache
        if self.table is None:
            return cache[r, i, :self.w]
        return cache[int(self.table[r, i // self.page]), i % self.page, :self.w]

    def device(self, dsa):
        self.d_cache = self.cache.cuda()
        self.d_seq = torch.tensor(self.lens, dtype=torch.int32).cuda()
        self.d_table = None if self.table is None else self.table.cuda()
        lat = dsa.Latent(self.d_cache, strides=(self.d_cache.stride(0), self.d_cache.stride(1)), seq_len=self.d_seq, latent_dim=self.latent,
                         rope_dim=self.rope, max_seq_len=self.room, sm_scale=self.scale, block_table=self.d_table, block_size=self.page,
                         num_blocks=self.blocks)
        self.d_q, self.d_new = self.q.cuda(), self.c_new.cuda()
        self.d_count = None if self.counts is None else torch.tensor(self.counts, dtype=torch.int32).cuda()
        return lat

    def expected(self, r):
        return latent_ref.step_expected(self.q[r].double(), self.rows[r].double(), self.c_new[r].double(), self.n[r], self.latent,
                                        self.scale, self.dtype == "bf16")

    def check(self, out, lse, cache=None, stored=None):
        want = self.cache.clone()
        for r, n in enumerate(self.n):
            o, l, tol, ltol = self.expected(r)
            latent_ref.assert_near(out[r], o, tol, "out of request %d" % r)
            latent_ref.assert_near(lse[r], l, ltol, "lse of request %d" % r)
            for i in range(n):
                if stored is None or stored(r, self.lens[r] + i):
                    self.place(r, self.lens[r] + i, want)[:] = self.c_new[r, i]
        got = (self.d_cache if cache is None else cache).cpu()
        as_bits = torch.int16 if self.dtype == "bf16" else torch.int32
        assert torch.equal(got.view(as_bits), want.view(as_bits)), "cache"


def run(dsa, c, lat=None):
    lat = c.device(dsa) if lat is None else lat
    out, lse = dsa.alloc_latent_outputs(lat, c.d_q)
    out.fill_(math.nan), lse.fill_(math.nan)
    ws = dsa.alloc_latent_workspace(lat, c.d_q)
    if ws is not None:
        ws.fill_(0xff)
    dsa.dsa_latent_step(lat, c.d_q, c.d_new, out, lse, ws, new_count=c.d_count)
    torch.cuda.synchronize()
    assert dsa.dsa_wait_timeouts() == 0
    return out, lse


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,new,lens,page,kw", [
    (1, 1, [0, 1, 63, 64, 65, 200], 16, {}),
    (16, 1, [600, 17, 0, 129], 16, {}),
    (16, 1, [0], 64, {}),
    (128, 1, [300, 70], 64, {}),
    (20, 3, [0, 1, 144, 511], 0, dict(latent=256, rope=32)),
    (3, 7, [5, 130, 64, 17], 5, dict(counts=[0, 7, 3, 5])),
    (8, 64, [100, 3], 24, {}),
    (96, 2, [150, 33, 1], 1, dict(rope=16)),
    (64, 1, [256, 255, 257], 128, dict(rope=8, latent=256)),
    (5, 33, [95, 64], 48, dict(counts=[33, 32], pad=24)),
    (64, 3, [77, 191], 0, dict(pad=8)),
    (130, 2, [129], 16, {}),
])
def test_step(dsa, dtype, heads, new, lens, page, kw):
    c = Case(dtype, heads, new, lens, page, **kw)
    c.check(*run(dsa, c))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [0, 16])
def test_lengths_at_their_limits(dsa, dtype, page):
    """Requests that are full, nearly full, over-long, negative, or without new tokens; counts outside [0, N]."""
    lens, counts = [40, 38, 37, 60, -3, 20, 20, 0], [4, 4, 4, 4, 4, -2, 99, 4]
    c = Case(dtype, 16, 4, lens, page, counts=counts, room=40)
    c.lens = [min(x, 40) for x in lens]
    c.d_lens = None
    lat = c.device(dsa)
    c.d_seq.copy_(torch.tensor(lens, dtype=torch.int32))
    assert c.n == [0, 2, 3, 0, 0, 0, 4, 4]
    # what a token that does not exist would have brought may be anything
    for r, n in enumerate(c.n):
        c.d_q[r, n:] = math.nan
        c.d_new[r, n:] = math.nan
    c.check(*run(dsa, c, lat))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_missing_pages_store_nothing(dsa, dtype):
    c = Case(dtype, 16, 3, [31, 16, 47], 16, room=64)
    lat = c.device(dsa)
    c.d_table[0, 2:] = -1                                    # position 32 and 33 have no page
    c.d_table[1, 1] = c.blocks + 5                           # 16 .. 18 neither
    c.check(*run(dsa, c, lat), stored=lambda r, at: not (r == 0 and at >= 32) and r != 1)


@pytest.mark.parametrize("dtype,lens,heads,new", [("bf16", [12345, 1, 4000, 640], 16, 1), ("bf16", [5000, 9], 128, 2),
                                                  ("f32", [3000, 100], 8, 1), ("bf16", [700] * 150 + [1, 0, 64], 8, 1),
                                                  ("bf16", [64 * 37], 64, 5)])
def test_long_and_many(dsa, dtype, lens, heads, new):
    """Pieces of one sequence on many blocks, and blocks with pieces of many sequences."""
    c = Case(dtype, heads, new, lens, 64 if len(lens) < 10 else 16)
    c.check(*run(dsa, c))


def test_large_scores(dsa):
    """Maxima that keep growing along the sequence, and scores far below zero."""
    for sign in (1.0, -1.0):
        c = Case("bf16", 16, 2, [400, 130], 16, seed=5)
        ramp = torch.linspace(0, 6, 400)
        for r in range(2):
            for i in range(c.lens[r]):
                c.rows[r][i] = (c.rows[r][i].float() + sign * ramp[i] * c.q[r, 0, 0].float() / 4).bfloat16()
                c.place(r, i)[:] = c.rows[r][i]
        c.check(*run(dsa, c))


def test_same_inputs_same_bits(dsa):
    c = Case("bf16", 32, 1, [3000, 777, 64, 2], 16)
    first = run(dsa, c)
    for _ in range(3):
        again = run(dsa, c)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
