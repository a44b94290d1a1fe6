"""The latent-cache calls as a server uses them, one behind the other: pages reserved, the tokens of a ragged batch mapped, their
rows stored, the rows behind them gathered and expanded, prompt attention, then steps of one or several tokens, pages given
back.  The host keeps every request's rows; what each call gives is compared with float64 over those."""
import math
import os
import subprocess
import sys

import pytest
import torch

from tests import draft_ref, latent_ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
H, D, R, P = 4, 64, 256, 32
W = R + P


@pytest.fixture(scope="module")
def dsa():
    from paper_2609_19702_b200 import binding
    return binding


class Server:
    """Static buffers, so that a pass can be captured: a prompt pass and a step pass over them."""

    def __init__(self, dsa, dtype, batch, page, cap, most, new):
        g = torch.Generator().manual_seed(batch * 100 + page)
        self.dsa, self.b, self.page, self.cap, self.most, self.new, self.bf16 = dsa, batch, page, cap, most, new, dtype == "bf16"
        self.room = min(cap // 2 - 3 * new, most // batch)   # of a request, in each of two prompts
        dt = DT[dtype]
        self.rand = lambda *s: torch.randn(s, generator=g).to(dt)  # noqa: E731
        self.g = g
        per = -(-cap // page)
        blocks = batch * per
        self.cache = torch.full((blocks, page, W), math.nan, dtype=dt, device="cuda")
        self.table = torch.full((batch, per), -1, dtype=torch.int32, device="cuda")
        self.pool = dsa.PagePool(torch.zeros((blocks,), dtype=torch.int32, device="cuda"), page)
        self.seq, self.count, self.status = (torch.zeros((batch,), dtype=torch.int32, device="cuda") for _ in range(3))
        self.lat = dsa.Latent(self.cache, strides=(page * W, W), seq_len=self.seq, latent_dim=R, rope_dim=P, max_seq_len=cap, sm_scale=1 / math.sqrt(D + P),
                              block_table=self.table, block_size=page, num_blocks=blocks)
        self.up = (torch.randn((R, H * 2 * D), generator=g) / 16).to(dt).cuda()          # keys and values of all heads
        full = batch * cap
        z = lambda *s, t=dt: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
        self.q, self.c = z(most, H, D + P), z(most, W)
        self.q_start, self.kv_start = z(batch + 1, t=torch.int32), z(batch + 1, t=torch.int32)
        self.slot, self.position, self.request = z(most, t=torch.int64), z(most, t=torch.int32), z(most, t=torch.int32)
        self.kv_slot, self.kv_rows, self.kv = z(full, t=torch.int64), z(full, W), z(full, H, 2 * D)
        self.out, self.lse = z(most, H, D), z(most, H, t=torch.float32)
        self.prompt = dsa.Prompt(self.q, self.kv[..., :D], self.kv_rows[:, R:], self.kv[..., D:], self.q_start, self.kv_start, max_q_len=most)
        self.sq, self.sc = z(batch, new, H, W), z(batch, new, W)
        self.s_out, self.s_lse = dsa.alloc_latent_outputs(self.lat, self.sq)
        self.ws = dsa.alloc_latent_workspace(self.lat, self.sq)
        self.rows = [torch.zeros((0, W), dtype=dt) for _ in range(batch)]

    def prompt_pass(self):
        """The tokens of self.c and self.q, self.count[b] of request b, behind what is cached."""
        d, lat = self.dsa, self.lat
        d.dsa_reserve_pages(self.pool, self.table, self.seq, self.room, self.status)
        args = dict(block_table=self.table, block_size=self.page, num_blocks=lat.num_blocks, max_seq_len=self.cap)
        d.dsa_map_tokens(self.count, self.q_start, self.slot, self.position, self.request, base=self.seq, **args)
        d.dsa_store_rows(lat, self.slot, self.c)
        self.seq += self.count
        d.dsa_map_tokens(self.seq, self.kv_start, self.kv_slot, **args)
        d.dsa_gather_rows(lat, self.kv_slot, self.kv_rows)
        torch.mm(self.kv_rows[:, :R], self.up, out=self.kv.view(-1, H * 2 * D))
        d.dsa_latent_prompt(self.prompt, self.out, self.lse)
        d.dsa_release_pages(self.pool, self.table, self.seq)

    def step_pass(self):
        d = self.dsa
        d.dsa_reserve_pages(self.pool, self.table, self.seq, self.new, self.status)
        d.dsa_latent_step(self.lat, self.sq, self.sc, self.s_out, self.s_lse, self.ws, new_count=self.count)
        self.seq += self.count
        d.dsa_release_pages(self.pool, self.table, self.seq)

    def check_cache(self):
        lens = [len(r) for r in self.rows]
        assert self.seq.tolist() == lens and self.status.tolist() == [0] * self.b
        held = [-(-n // self.page) for n in lens]
        assert (self.table >= 0).sum(1).tolist() == held and int(self.pool.ref_count.sum()) == sum(held)
        for r, n in enumerate(lens):
            at = torch.arange(n, device="cuda")
            assert torch.equal(self.cache[self.table[r].long()[at // self.page], at % self.page].cpu(), self.rows[r])

    def run_prompt(self, counts, launch):
        c, q, total = self.rand(self.most, W), self.rand(self.most, H, D + P), sum(counts)
        self.c.copy_(c), self.q.copy_(q), self.count.copy_(torch.tensor(counts, dtype=torch.int32))
        self.out.fill_(7.0), self.lse.fill_(7.0), self.kv_rows.fill_(math.nan)
        launch()
        torch.cuda.synchronize()
        at, bt = 0, 0
        kv = self.kv.cpu()
        for r, n in enumerate(counts):
            base = len(self.rows[r])
            self.rows[r] = torch.cat([self.rows[r], c[at:at + n]])
            assert self.position[at:at + n].tolist() == list(range(base, base + n)) and self.request[at:at + n].tolist() == [r] * n
            end = bt + len(self.rows[r])
            assert torch.equal(self.kv_rows[bt:end].cpu(), self.rows[r])
            if n:
                k = kv[bt:end].double()
                o, l, tol, ltol = latent_ref.prompt_expected(q[at:at + n].double(), k[..., :D], self.rows[r][:, R:].double(), k[..., D:], True,
                                                             1 / math.sqrt(D + P), self.bf16)
                latent_ref.assert_near(self.out[at:at + n], o, tol, "prompt of request %d" % r)
                latent_ref.assert_near(self.lse[at:at + n], l, ltol, "prompt lse of request %d" % r)
            at, bt = at + n, end
        assert self.q_start.tolist()[-1] == total and (self.out[total:] == 7.0).all() and (self.lse[total:] == 7.0).all()
        self.check_cache()

    def run_step(self, counts, launch):
        c, q = self.rand(self.b, self.new, W), self.rand(self.b, self.new, H, W)
        self.sc.copy_(c), self.sq.copy_(q), self.count.copy_(torch.tensor(counts, dtype=torch.int32))
        self.s_out.fill_(math.nan), self.s_lse.fill_(math.nan)
        launch()
        torch.cuda.synchronize()
        for r, n in enumerate(counts):
            o, l, tol, ltol = latent_ref.step_expected(q[r].double(), self.rows[r].double(), c[r].double(), n, R, 1 / math.sqrt(D + P), self.bf16)
            latent_ref.assert_near(self.s_out[r], o, tol, "step of request %d" % r)
            latent_ref.assert_near(self.s_lse[r], l, ltol, "step lse of request %d" % r)
            self.rows[r] = torch.cat([self.rows[r], c[r, :n]])
        self.check_cache()


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("dtype,batch,page,cap,most,new", [("f32", 3, 4, 120, 70, 3), ("bf16", 3, 16, 400, 250, 1), ("bf16", 5, 24, 300, 200, 4),
                                                          ("bf16", 70, 8, 150, 1500, 2)])
def test_prompts_and_steps(dsa, dtype, batch, page, cap, most, new, captured):
    s = Server(dsa, dtype, batch, page, cap, most, new)
    launch = [s.prompt_pass, s.step_pass]
    if captured:
        dsa.dsa_prepare()
        launch, graphs = [], []
        state = [t.clone() for t in (s.cache, s.table, s.pool.ref_count, s.seq)]
        side = torch.cuda.Stream()
        for one in (s.prompt_pass, s.step_pass):
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):                    # (the library product wants a first run outside a capture)
                one()
            torch.cuda.current_stream().wait_stream(side)
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1]):
                one()
            launch.append(graphs[-1].replay)
        for t, was in zip((s.cache, s.table, s.pool.ref_count, s.seq), state):
            t.copy_(was)
    rng = torch.Generator().manual_seed(batch)
    draw = lambda top: torch.randint(0, top + 1, (batch,), generator=rng).tolist()  # noqa: E731
    s.run_prompt(draw(s.room), launch[0])                      # no cached rows yet
    for _ in range(2):
        s.run_step(draw(new), launch[1])
    s.run_prompt(draw(s.room), launch[0])                      # behind a cached prefix, some without a new token
    for _ in range(3):
        s.run_step(draw(new), launch[1])
    assert dsa.dsa_wait_timeouts() == 0


@pytest.mark.parametrize("n,cached", [(40, 0), (7, 90), (64, 300)])
def test_both_forms_agree(dsa, n, cached):
    """float32: the same tokens by expanded keys and values, and by queries with the keys' map absorbed, both against one float64
    attention.  What the maps' own rounding to float32 adds: one more half step for every element of keys and queries, one
    for every value."""
    g = torch.Generator().manual_seed(n)
    rand = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    rows, q, up_k, up_v = rand(cached + n, W), rand(n, H, D + P), rand(H, R, D) / 16, rand(H, R, D) / 16
    k64, v64 = torch.einsum("lr,hrd->lhd", rows[:, :R].double(), up_k.double()), torch.einsum("lr,hrd->lhd", rows[:, :R].double(), up_v.double())
    scale = 1 / math.sqrt(D + P)
    key = torch.cat([k64, rows[:, None, R:].double().expand(-1, H, -1)], -1)
    limit = [cached + i + 1 for i in range(n)]
    o, l, weight, size, count = latent_ref.attend(q.double(), key, v64, limit, scale)

    tol, ltol = draft_ref.tree_tolerances(o, l, weight, size, count, D + P + 1, False)
    starts = [torch.tensor([0, x], dtype=torch.int32).cuda() for x in (n, cached + n)]
    p = dsa.Prompt(q.cuda(), k64.float().cuda(), rows[:, R:].cuda(), v64.float().cuda(), starts[0], starts[1], max_q_len=n)
    out, lse = dsa.alloc_prompt_outputs(p)
    dsa.dsa_latent_prompt(p, out, lse)
    latent_ref.assert_near(out, o, tol + draft_ref.F32_HALF_STEP * weight, "expanded")
    latent_ref.assert_near(lse, l, ltol, "expanded lse")

    # the absorbed form's scores are sums of R + P products, and its result is mapped behind the call (in 64 bits)
    absorbed = torch.cat([torch.einsum("nhd,hrd->nhr", q[..., :D].double(), up_k.double()), q[..., D:].double()], -1)
    lo, ll, lweight, lsize, lcount = latent_ref.attend(absorbed, rows[:, None].double(), rows[:, None, :R].double(), limit, scale)
    ltol_, lltol = draft_ref.tree_tolerances(lo, ll, lweight, lsize, lcount, W + 1, False)
    assert torch.allclose(ll, l, atol=1e-9) and torch.allclose(torch.einsum("nhr,hrd->nhd", lo, up_v.double()), o, atol=1e-9)
    cache = torch.full((1, cached + n, W), math.nan)
    cache[0, :cached] = rows[:cached]
    lat = dsa.Latent(cache.cuda(), strides=((cached + n) * W, W), seq_len=torch.tensor([cached], dtype=torch.int32).cuda(), latent_dim=R, rope_dim=P,
                     max_seq_len=cached + n, sm_scale=scale)
    dq, dc = absorbed.float()[None].cuda(), rows[None, cached:].contiguous().cuda()
    s_out, s_lse = dsa.alloc_latent_outputs(lat, dq)
    dsa.dsa_latent_step(lat, dq, dc, s_out, s_lse, dsa.alloc_latent_workspace(lat, dq))
    up = up_v.double()
    latent_ref.assert_near(torch.einsum("nhr,hrd->nhd", s_out[0].cpu().double(), up), o, torch.einsum("nhr,hrd->nhd", ltol_, up.abs()) + 1e-9, "absorbed")
    latent_ref.assert_near(s_lse[0], l, lltol, "absorbed lse")
    assert torch.equal(lat.cache[0].cpu(), rows)


CHILD = r"""
import torch
from paper_2609_19702_b200 import binding as dsa

def latent(dt, batch, heads, new, room):
    cache = torch.randn((batch, room, 576), device="cuda").to(dt)
    seq = torch.arange(batch, device="cuda", dtype=torch.int32) * 31 % (room - new)
    lat = dsa.Latent(cache, strides=(room * 576, 576), seq_len=seq, latent_dim=512, rope_dim=64, max_seq_len=room, sm_scale=0.07)
    q, c = torch.randn((batch, new, heads, 576), device="cuda").to(dt), torch.randn((batch, new, 576), device="cuda").to(dt)
    return lat, q, c, dsa.alloc_latent_outputs(lat, q), dsa.alloc_latent_workspace(lat, q)

steps = [latent(torch.bfloat16, 2, 16, 1, 200), latent(torch.bfloat16, 200, 16, 2, 300), latent(torch.bfloat16, 60, 128, 1, 900),
         latent(torch.float32, 3, 8, 2, 200), latent(torch.bfloat16, 10, 16, 1, 1000)]
prompts = []
for dt, d in ((torch.bfloat16, 128), (torch.float32, 64), (torch.bfloat16, 64)):
    q, kv, kr = (torch.randn(s, device="cuda").to(dt) for s in ((300, 2, d + 64), (300, 2, 2 * d), (300, 64)))
    p = dsa.Prompt(q, kv[..., :d], kr, kv[..., d:], torch.tensor([0, 7, 300], dtype=torch.int32, device="cuda"), max_q_len=293)
    prompts.append((p, dsa.alloc_prompt_outputs(p)))
count = torch.tensor([3, 4], dtype=torch.int32, device="cuda")
start, slot = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(9, dtype=torch.int64, device="cuda")
rows, back = torch.randn((9, 576), device="cuda").bfloat16(), torch.zeros((9, 576), device="cuda").bfloat16()

def calls():
    for lat, q, c, (out, lse), ws in steps:
        dsa.dsa_latent_step(lat, q, c, out, lse, ws)
    for p, (out, lse) in prompts:
        dsa.dsa_latent_prompt(p, out, lse)
    dsa.dsa_map_tokens(count, start, slot, max_seq_len=200)
    dsa.dsa_store_rows(steps[0][0], slot, rows)
    dsa.dsa_gather_rows(steps[0][0], slot, back)

state = [t for s in steps for t in (s[0].cache, *s[3])] + [t for p in prompts for t in p[1]] + [start, slot, back]
was = [t.clone() for t in state]
torch.cuda.synchronize()
dsa.dsa_prepare()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):          # the very first calls of this process
    calls()
graph.replay()
torch.cuda.synchronize()
got = [t.clone() for t in state]
for t, w in zip(state, was):
    t.copy_(w)
calls()
torch.cuda.synchronize()
bits = lambda t: t.contiguous().view(torch.uint8)
for i, (a, b) in enumerate(zip(got, state)):
    assert torch.equal(bits(a), bits(b)), i
assert slot.tolist() == [0, 1, 2, 200, 201, 202, 203, -1, -1] and torch.equal(back[:7], rows[:7]) and dsa.dsa_wait_timeouts() == 0
print("CAPTURED-FIRST-CALLS-OK")
"""


def test_first_calls_of_a_process_can_be_captured_after_prepare():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    env = dict(os.environ, PYTHONPATH=root + os.pathsep + os.environ.get("PYTHONPATH", ""))
    res = subprocess.run([sys.executable, "-c", CHILD], cwd=root, env=env, capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stdout[-2000:] + res.stderr[-4000:]
    assert "CAPTURED-FIRST-CALLS-OK" in res.stdout
