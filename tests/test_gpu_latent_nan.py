"""Rows without a number inside live requests of dsa_latent_step, under every plan: what sees them has no number either, whichever blocks
merge it, and nobody else notices."""
import math

import pytest
import torch

from tests import latent_ref
from tests.test_gpu_latent import Case, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dsa():
    from paper_2609_19702_b200 import binding
    return binding


def _lens(batch, top):
    return [top if b % 5 == 0 else 1 + (b * 37) % top for b in range(batch)]


# (type, requests, heads, new tokens, longest, page, whether parts are joined through the workspace)
PLANS = [("bf16", 4, 16, 1, 300, 16, False),                 # clusters
         ("bf16", 64, 16, 1, 1500, 16, True),                # shares of single blocks
         ("bf16", 64, 16, 2, 900, 64, True),
         ("bf16", 20, 128, 1, 1500, 64, True),               # shares of pairs
         ("bf16", 20, 100, 2, 1200, 16, True),
         ("bf16", 24, 128, 1, 700, 8, True),                 # single blocks, two row tiles a request
         ("f32", 6, 8, 1, 900, 16, True)]


@pytest.mark.parametrize("dtype,batch,heads,new,top,page,joined", PLANS)
def test_rows_without_a_number(dsa, dtype, batch, heads, new, top, page, joined):
    c = Case(dtype, heads, new, _lens(batch, top), page)
    lat = c.device(dsa)
    assert (dsa.dsa_latent_workspace_size(lat, heads, new) > 0) == joined
    good = [x.clone() for x in run(dsa, c, lat)]

    def alone(r, first=0):
        """What tokens `first`.. of request r are has no number; all others have the bits that they had."""
        out, lse = run(dsa, c, lat)
        for x, y in ((out, good[0]), (lse, good[1])):
            assert x[r, first:].isnan().all()
            for b in range(batch):
                if b != r:
                    assert torch.equal(x[b], y[b]), "request %d" % b

    for r in (0, 1, batch - 1):                              # long, short, last
        keep = c.d_new[r].clone()
        c.d_new[r] = math.nan                                # a new token's row, which every token of one behind it sees
        alone(r)
        c.d_new[r] = keep
        for at in sorted({0, 1, 63, 64, 127, 128, c.lens[r] // 2, c.lens[r] - 1}):
            if at < c.lens[r]:                               # one cached row, in the first, in a middle, in the last tile
                row = c.place(r, at, c.d_cache)
                keep = row.clone()
                row.fill_(math.nan)
                alone(r)
                row.copy_(keep)
    keep = c.d_cache.clone()                                 # and all of them
    for at in range(c.lens[0]):
        c.place(0, at, c.d_cache).fill_(math.nan)
    c.d_new[0] = math.nan
    alone(0)
    c.d_cache.copy_(keep)
    c.d_new.copy_(c.c_new)
    for x, y in zip(run(dsa, c, lat), good):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype,batch,heads,new,top,page,joined", PLANS)
def test_queries_without_a_number(dsa, dtype, batch, heads, new, top, page, joined):
    """One head's query of one token: that head's result alone."""
    c = Case(dtype, heads, new, _lens(batch, top), page)
    lat = c.device(dsa)
    for r, h in ((0, 0), (0, heads - 1), (batch // 2, heads // 2)):
        c.d_q.copy_(c.q)
        c.d_q[r, new - 1, h] = math.nan
        out, lse = run(dsa, c, lat)
        assert out[r, new - 1, h].isnan().all() and lse[r, new - 1, h].isnan()
        want, l, tol, ltol = c.expected(r)
        got, got_l = out[r].cpu(), lse[r].cpu()
        got[new - 1, h], got_l[new - 1, h] = want[new - 1, h].to(got.dtype), l[new - 1, h].to(got_l.dtype)
        latent_ref.assert_near(got, want, tol, "the other heads")
        latent_ref.assert_near(got_l, l, ltol, "the other heads, lse")
        for b in (1, batch - 1):
            want, l, tol, ltol = c.expected(b)
            latent_ref.assert_near(out[b], want, tol, "request %d" % b)
            latent_ref.assert_near(lse[b], l, ltol, "lse of request %d" % b)
