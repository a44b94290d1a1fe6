"""How the blocks of a prompt call (dsa_latent_prompt) find their work: long runs of requests without a token, very many requests,
bounds of the queries far above what the requests have."""
import json
import math

import pytest
import torch

from tests import latent_ref
from tests.test_gpu_prompt import DT, run_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dsa():
    from paper_2609_19702_b200 import binding
    return binding


def test_runs_of_requests_without_a_token(dsa):
    """A running block passes over hundreds of blocks without a query between one item and the next, each time the same."""
    lens = [0] * 3000
    for b, n in ((0, 3), (700, 260), (701, 1), (1999, 40), (2999, 129)):
        lens[b] = n
    first = run_case(dsa, "bf16", 8, 64, 8, lens)
    for _ in range(10):
        again = run_case(dsa, "bf16", 8, 64, 8, lens)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_a_run_longer_than_a_wait_may_take(dsa):
    """A million requests of 1024 heads, hardly any with a token: what a block finds behind seconds of nothing is computed too."""
    lens = [0] * 2 ** 20
    for b, n in ((0, 1), (2 ** 19 + 3, 2), (2 ** 20 - 1, 3)):
        lens[b] = n
    run_case(dsa, "bf16", 1024, 64, 8, lens)


def blocks_of(call, tmp_path):
    """Thread blocks that the prompt kernel of this call is launched with."""
    from torch.profiler import ProfilerActivity, profile
    call()
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as p:
        call()
        torch.cuda.synchronize()
    p.export_chrome_trace(str(tmp_path / "trace.json"))
    events = json.load(open(tmp_path / "trace.json"))["traceEvents"]
    grids = [e["args"]["grid"] for e in events if "dsa_prompt" in e.get("name", "") and "grid" in e.get("args", {})]
    if not any("grid" in e.get("args", {}) for e in events):
        pytest.skip("no launch is shown by the profiler here")
    assert len(grids) == 1
    return grids[0][0]


class Shared:
    """A batch whose heads are all the same (strides of 0), so that it stays small; `front` rows in front belong to nobody."""

    def __init__(self, dsa, dtype, heads, lens, d=64, rope=8, front=0, seed=0):
        g = torch.Generator().manual_seed(seed)
        n, dt = sum(lens), DT[dtype]
        self.dsa, self.dtype, self.heads, self.lens, self.d, self.front = dsa, dtype, heads, lens, d, front
        self.q, self.kv, self.kr = (torch.randn(s, generator=g).to(dt) for s in ((front + n, d + rope), (front + n, 2 * d), (front + n, rope)))
        self.start = torch.tensor([0] + lens).cumsum(0).int() + front
        dq, dkv = self.q.cuda()[:, None].expand(-1, heads, -1), self.kv.cuda()[:, None].expand(-1, heads, -1)
        self.prompt = dsa.Prompt(dq, dkv[..., :d], self.kr.cuda(), dkv[..., d:], self.start.cuda())
        self.out, self.lse = dsa.alloc_prompt_outputs(self.prompt)

    def call(self, bound=0):                                 # (0: all tokens, as the call has it by itself)
        self.prompt.max_q_len = bound
        self.dsa.dsa_latent_prompt(self.prompt, self.out, self.lse)

    def run(self, bound=0):
        self.out.fill_(7.0), self.lse.fill_(7.0)
        self.call(bound)
        assert self.dsa.dsa_wait_timeouts() == 0
        return self.out.clone(), self.lse.clone()

    def check(self, out, lse, requests, bound=0):
        assert torch.equal(out, out[:, :1].expand_as(out)) and torch.equal(lse, lse[:, :1].expand_as(lse))
        assert bool((out[:self.front] == 7.0).all()) and bool((lse[:self.front] == 7.0).all())
        out, lse, d = out[:, :1].cpu(), lse[:, :1].cpu(), self.d
        for r in requests:
            a, b = int(self.start[r]), int(self.start[r + 1])
            if a == b:
                continue
            kv = self.kv[a:b, None].double()
            o, l, tol, ltol = latent_ref.prompt_expected(self.q[a:b, None].double(), kv[..., :d], self.kr[a:b].double(), kv[..., d:], True,
                                                         1 / math.sqrt(self.q.shape[1]), self.dtype == "bf16")
            top = min(b - a, bound or b - a)
            latent_ref.assert_near(out[a:a + top], o[:top], tol[:top], "out of request %d" % r)
            latent_ref.assert_near(lse[a:a + top], l[:top], ltol[:top], "lse of request %d" % r)
            assert bool((out[a + top:b] == 7.0).all()) and bool((lse[a + top:b] == 7.0).all())


def ragged(batch, most, seed, zeros=0.3):
    g = torch.Generator().manual_seed(seed)
    return torch.where(torch.rand((batch,), generator=g) < zeros, 0, torch.randint(0, most + 1, (batch,), generator=g)).tolist()


@pytest.mark.parametrize("dtype,rows", [("bf16", 256), ("f32", 32)])
@pytest.mark.parametrize("batch,most,zeros,front", [(257, 70, 0.3, 0), (600, 100, 0.3, 1000), (4096, 9, 0.5, 0), (40, 1500, 0.1, 300), (200, 20, 0.3, 0),
                                                    (1025, 33, 0.9, 5), (256, 600, 0.0, 0), (3, 700, 0.0, 4000)])
def test_a_loose_bound_changes_nothing(dsa, tmp_path, dtype, rows, batch, most, zeros, front):
    """All tokens as the bound of a request's queries: the same bits as with the longest request, and no more blocks than the
    tokens fill and one a request."""
    lens = ragged(batch, most, batch, zeros)
    lens[batch // 2] = most
    c = Shared(dsa, dtype, 3, lens, front=front)
    loose = c.run()
    c.check(*loose, requests=range(0, batch, max(1, batch // 60)))
    c.check(*loose, requests=[0, batch // 2, batch - 1])
    tight = c.run(most)
    assert torch.equal(loose[0], tight[0]) and torch.equal(loose[1], tight[1])
    assert blocks_of(lambda: c.call(), tmp_path) <= 3 * 2 * (len(c.q) // rows + batch)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_bound_below_some_of_many_requests(dsa, dtype):
    """Queries beyond the bound are left out; the blocks that they would have had do nothing."""
    lens = ragged(2000, 5, 3)
    lens[0], lens[777], lens[1999] = 900, 1500, 601
    c = Shared(dsa, dtype, 2, lens)
    c.check(*c.run(600), requests=[0, 776, 777, 778, 1998, 1999], bound=600)


@pytest.mark.parametrize("dtype,batch,tokens,heads", [("f32", 4096, 32, 128), ("bf16", 65536, 2, 128)])
def test_batches_that_a_loose_bound_made_too_large(dsa, dtype, batch, tokens, heads):
    """A grid of every request's share of all tokens would have more than 2^31 blocks."""
    lens = ragged(batch, 2 * tokens, batch, 0.0)
    lens[batch // 3] += 300
    c = Shared(dsa, dtype, heads, lens)
    c.check(*c.run(), requests=list(range(0, batch, batch // 50)) + [batch // 3, batch - 1])
