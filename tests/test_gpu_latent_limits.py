"""Latent-cache calls where sizes, layouts, streams and graphs could go wrong: every plan of the step, pages of all sizes, shared
pages, offsets beyond 32 bits, infinities, heads that share keys, two calls at once, graphs over one workspace."""
import math

import pytest
import torch

from tests import latent_ref
from tests.test_gpu_latent import DT, Case, run
from tests.test_gpu_prompt import run_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dsa():
    from paper_2609_19702_b200 import binding
    return binding


def _lens(batch, top, seed):
    g = torch.Generator().manual_seed(seed)
    lens = torch.randint(0, top + 1, (batch,), generator=g).tolist()
    lens[0] = top
    return lens


@pytest.mark.parametrize("latent", [512, 256])
@pytest.mark.parametrize("batch,heads,new,top", [
    (1, 16, 1, 3000), (5, 16, 1, 700), (20, 16, 1, 600), (40, 8, 2, 300), (148, 16, 1, 70), (149, 16, 1, 130), (75, 64, 1, 900),
    (1, 128, 1, 2000), (3, 128, 2, 500), (8, 96, 1, 700), (33, 128, 1, 260), (16, 100, 3, 350), (90, 65, 1, 200), (2, 1024, 1, 300),
])
def test_every_plan(dsa, latent, batch, heads, new, top):
    """Clusters of one to eight blocks, shares of single blocks and of pairs."""
    c = Case("bf16", heads, new, _lens(batch, top, batch + heads), 64 if batch % 2 else 16, latent=latent, rope=64 if heads > 16 else 24, seed=batch)
    c.check(*run(dsa, c))


@pytest.mark.parametrize("page", [1, 2, 3, 4, 6, 8, 12, 24, 32, 40, 100, 256])
@pytest.mark.parametrize("batch,heads,top", [(2, 16, 500), (100, 16, 150), (30, 128, 300)])
def test_pages(dsa, page, batch, heads, top):
    c = Case("bf16", heads, 2, _lens(batch, top, page), page, seed=page, pad=8 * (page % 3))
    c.check(*run(dsa, c))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page,extra", [(1, 8), (2, 72), (16, 8), (64, 584 + 8)])
def test_page_stride_of_its_own(dsa, dtype, page, extra):
    """Pages that do not lie a whole number of tokens apart."""
    c = Case(dtype, 16, 3, [130, 0, 77, 400], page, pad=8)
    lat = c.device(dsa)
    step = page * lat.strides[1] + extra
    flat = torch.full((c.blocks * step,), math.nan, dtype=DT[dtype], device="cuda")
    view = flat.as_strided(c.d_cache.shape, (step, lat.strides[1], 1))
    view.copy_(c.d_cache)
    lat.cache, lat.strides = flat, (step, lat.strides[1])
    out, lse = run(dsa, c, lat)
    c.check(out, lse, cache=view)
    gaps = flat.view(c.blocks, step)[:, page * lat.strides[1]:]
    assert gaps.isnan().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [16, 128])
def test_pages_of_a_common_prefix(dsa, dtype, heads):
    """Ten requests whose first pages are the same ones."""
    page, common = 16, 5
    lens = [common * page + 13 * r for r in range(10)]
    c = Case(dtype, heads, 1, lens, page)
    for r in range(1, 10):
        c.table[r, :common] = c.table[0, :common]
        for i in range(common * page):
            c.rows[r][i] = c.rows[0][i]
    c.check(*run(dsa, c))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("heads", [16, 96])
def test_cache_offsets_beyond_32_bits(dsa, dtype, paged, heads):
    """Requests or pages more than 2^31 elements apart, and pages whose numbers times their size pass 2^32 bytes."""
    room, w = 400, 576
    lens = [333, 0, 399]
    c = Case(dtype, heads, 1, lens, 0, room=room)
    step = 2 ** 30 + 2 ** 29 + 64 * 9                        # elements: the third one lies beyond 2^31
    flat = torch.empty((2 * step + 512 * w,), dtype=DT[dtype], device="cuda")
    where = flat.as_strided((3, room, w), (step, w, 1))
    where.copy_(c.cache)
    seq = torch.tensor(lens, dtype=torch.int32).cuda()
    c.d_q, c.d_new, c.d_count = c.q.cuda(), c.c_new.cuda(), None
    kw = dict(seq_len=seq, latent_dim=512, rope_dim=64, max_seq_len=room, sm_scale=c.scale)
    if paged:                                                # one page a request, whose numbers go the other way
        order = torch.tensor([[2], [0], [1]], dtype=torch.int32)
        for r in range(3):
            where[int(order[r, 0])].copy_(c.cache[r])
        lat = dsa.Latent(flat, strides=(step, w), block_table=order.cuda(), block_size=room, num_blocks=3, **kw)
    else:
        lat = dsa.Latent(flat, strides=(step, w), **kw)
    out, lse = run(dsa, c, lat)
    got = where if not paged else torch.stack([where[int(order[r, 0])] for r in range(3)])
    c.check(out, lse, cache=got)


def test_many_pages_beyond_32_bits(dsa):
    """The last pages of a pool of 5 GB, in bf16 with a page's tokens as they come and gathered one by one."""
    for page in (64, 1):
        w = 576
        blocks = 2 ** 32 // (w * page) + 700
        c = Case("bf16", 16, 1, [300, 64], page, spare=0)
        cache = torch.empty((blocks, page, w), dtype=torch.bfloat16, device="cuda")
        far = blocks - 1 - torch.arange(c.blocks)
        cache[far.cuda()] = c.cache.cuda()
        c.d_seq = torch.tensor(c.lens, dtype=torch.int32).cuda()
        c.d_q, c.d_new, c.d_count = c.q.cuda(), c.c_new.cuda(), None
        lat = dsa.Latent(cache, strides=(page * w, w), seq_len=c.d_seq, latent_dim=512, rope_dim=64, max_seq_len=c.room, sm_scale=c.scale,
                         block_table=far[c.table.long()].int().cuda(), block_size=page, num_blocks=blocks)
        out, lse = run(dsa, c, lat)
        c.check(out, lse, cache=cache[far.cuda()])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_offsets_beyond_32_bits(dsa, dtype):
    """The last tokens of batches of more than 2^31 elements; the first tokens belong to nobody."""
    heads, d, rope, tokens = 64, 128, 64, 2 ** 31 // (64 * 128) + 1000
    g = torch.Generator().manual_seed(3)
    dt = DT[dtype]
    lens = [150, 0, 70]
    n = sum(lens)
    q, kv, kr = (torch.randn(s, generator=g).to(dt) for s in ((n, heads, d + rope), (n, heads, 2 * d), (n, rope)))
    bq, bk, br = (torch.empty((tokens, *x.shape[1:]), dtype=dt, device="cuda") for x in (q, kv, kr))
    for big, x in ((bq, q), (bk, kv), (br, kr)):
        big[-n:] = x.cuda()
    start = torch.tensor([tokens - n, tokens - n + 150, tokens - n + 150, tokens], dtype=torch.int32).cuda()
    p = dsa.Prompt(bq, bk[..., :d], br, bk[..., d:], start, max_q_len=150)
    out, lse = dsa.alloc_prompt_outputs(p)
    out.fill_(7.0), lse.fill_(7.0)
    dsa.dsa_latent_prompt(p, out, lse)
    at = 0
    for length in lens:
        if length:
            k = kv[at:at + length].double()
            o, l, tol, ltol = latent_ref.prompt_expected(q[at:at + length].double(), k[..., :d], kr[at:at + length].double(), k[..., d:], True,
                                                         1 / math.sqrt(d + rope), dtype == "bf16")
            latent_ref.assert_near(out[tokens - n + at:tokens - n + at + length], o, tol, "out")
            latent_ref.assert_near(lse[tokens - n + at:tokens - n + at + length], l, ltol, "lse")
        at += length
    assert bool((out[:tokens - n] == 7.0).all()) and bool((lse[:tokens - n] == 7.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [128, 64])
def test_prompt_heads_that_share_keys(dsa, dtype, d):
    """Keys and values with a head stride of 0, and queries whose tokens lie further apart than their heads fill."""
    g = torch.Generator().manual_seed(d)
    dt = DT[dtype]
    q = torch.randn((333, 5 * (d + 64) + 40), generator=g).to(dt).cuda()[:, :5 * (d + 64)].view(333, 5, d + 64)
    k, r, v = (torch.randn((333, w + 8), generator=g).to(dt).cuda()[:, :w] for w in (d, 64, d))
    start = torch.tensor([0, 200, 333], dtype=torch.int32).cuda()
    p = dsa.Prompt(q, k[:, None].expand(-1, 5, -1), r, v[:, None].expand(-1, 5, -1), start, max_q_len=200)
    out, lse = dsa.alloc_prompt_outputs(p)
    dsa.dsa_latent_prompt(p, out, lse)
    for a, b in ((0, 200), (200, 333)):
        h = [x[a:b].cpu().double() for x in (q, k, r, v)]
        o, l, tol, ltol = latent_ref.prompt_expected(h[0], h[1][:, None].expand(-1, 5, -1), h[2], h[3][:, None].expand(-1, 5, -1), True,
                                                     1 / math.sqrt(d + 64), dtype == "bf16")
        latent_ref.assert_near(out[a:b], o, tol, "out")
        latent_ref.assert_near(lse[a:b], l, ltol, "lse")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_lens,kv_lens", [([1], None), ([1], [1]), ([1], [700]), ([1, 1], [81, 80]), ([0, 0, 1], None), ([79, 81, 160, 161], None),
                                            ([255, 1, 512], [256, 300, 513]), ([40, 600], [0, 3])])
def test_prompt_sizes(dsa, dtype, q_lens, kv_lens):
    for heads, d in ((1, 128), (2, 64)):
        run_case(dsa, dtype, heads, d, 64, q_lens, kv_lens, behind=0 if len(q_lens) == 1 else 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_many_requests(dsa, dtype):
    """More row blocks than places on the device, most of them without a token."""
    g = torch.Generator().manual_seed(8)
    lens = torch.where(torch.rand((700,), generator=g) < 0.5, 0, torch.randint(0, 9, (700,), generator=g)).tolist()
    lens[350] = 520
    run_case(dsa, dtype, 1, 64, 32, lens)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinities_and_nan_that_nobody_sees(dsa, dtype):
    """Cached rows behind the length, rows of tokens that do not exist and their queries: anything may stand there."""
    for bad in (math.inf, -math.inf, math.nan, torch.finfo(DT[dtype]).max):
        c = Case(dtype, 16, 4, [70, 64, 0, 1], 16, counts=[1, 4, 2, 0])
        c.cache[c.cache.isnan()] = bad
        c.device(dsa)
        lat = c.device(dsa)
        for r, n in enumerate(c.n):
            c.d_q[r, n:] = bad
            c.d_new[r, n:] = bad
        c.check(*run(dsa, c, lat))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_request_without_a_number_leaves_the_others_alone(dsa, dtype):
    for heads, lens in ((16, [300, 200, 64, 5]), (128, [300, 200, 64, 5])):
        c = Case(dtype, heads, 1, lens, 16)
        good = run(dsa, c)
        good = [x.clone() for x in good]
        lat = c.device(dsa)
        c.d_new[1] = math.nan
        out, lse = run(dsa, c, lat)
        assert out[1].isnan().all() and lse[1].isnan().all()
        for r in (0, 2, 3):
            assert torch.equal(out[r], good[0][r]) and torch.equal(lse[r], good[1][r])


def test_two_calls_at_once(dsa):
    """Steps and prompts on streams of their own, a workspace for each step."""
    cases = [Case("bf16", 16, 1, _lens(64, 900, 1), 16), Case("bf16", 128, 1, _lens(20, 700, 2), 64), Case("f32", 8, 2, _lens(5, 300, 3), 16)]
    lats = [c.device(dsa) for c in cases]
    outs = [dsa.alloc_latent_outputs(l, c.d_q) for l, c in zip(lats, cases)]
    works = [dsa.alloc_latent_workspace(l, c.d_q) for l, c in zip(lats, cases)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, l, (o, s), w, st in zip(cases, lats, outs, works, streams):
            dsa.dsa_latent_step(l, c.d_q, c.d_new, o, s, w, stream=st)
    torch.cuda.synchronize()
    for c, (o, s) in zip(cases, outs):
        c.check(o, s)
    assert dsa.dsa_wait_timeouts() == 0


def test_graphs_over_one_workspace(dsa):
    """Two captured steps of different sizes that share a workspace, replayed in turns with new lengths."""
    a, b = Case("bf16", 16, 1, _lens(64, 800, 5), 16), Case("bf16", 128, 1, _lens(24, 600, 6), 16)
    lats = [c.device(dsa) for c in (a, b)]
    size = max(dsa.dsa_latent_workspace_size(l, c.heads, 1) for l, c in zip(lats, (a, b)))
    ws = torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")
    outs = [dsa.alloc_latent_outputs(l, c.d_q) for l, c in zip(lats, (a, b))]
    dsa.dsa_prepare()
    graphs = []
    for c, l, (o, s) in zip((a, b), lats, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            dsa.dsa_latent_step(l, c.d_q, c.d_new, o, s, ws)
    for _ in range(3):
        for g in graphs:
            g.replay()
    for c, (o, s) in zip((a, b), outs):
        torch.cuda.synchronize()
        c.check(o, s)
    # shorter sequences than at the capture: the lengths are read on the device
    for c, (o, s), g in zip((a, b), outs, graphs):
        short = [x // 3 for x in c.lens]
        c.d_seq.copy_(torch.tensor(short, dtype=torch.int32))
        o.fill_(math.nan), s.fill_(math.nan)
        g.replay()
        torch.cuda.synchronize()
        for r, n in enumerate(short):
            want, l, tol, ltol = latent_ref.step_expected(c.q[r].double(), c.rows[r][:n].double(), c.c_new[r].double(), 1, c.latent, c.scale, True)
            latent_ref.assert_near(o[r], want, tol, "out of request %d" % r)
            latent_ref.assert_near(s[r], l, ltol, "lse of request %d" % r)
    assert dsa.dsa_wait_timeouts() == 0


def test_steps_one_behind_the_other(dsa):
    """Calls in one stream without a gap, the next one's cache the last one's, as the layers of a model and its tokens follow."""
    c = Case("bf16", 16, 1, [100, 0, 37], 16, room=130)
    lat = c.device(dsa)
    g = torch.Generator().manual_seed(4)
    qs, news = torch.randn((25, 3, 1, 16, 576), generator=g).bfloat16(), torch.randn((25, 3, 1, 576), generator=g).bfloat16()
    dq, dn = qs.cuda(), news.cuda()
    outs = [dsa.alloc_latent_outputs(lat, dq[0]) for _ in range(25)]
    ws = dsa.alloc_latent_workspace(lat, dq[0])
    torch.cuda.synchronize()
    for i in range(25):
        dsa.dsa_latent_step(lat, dq[i], dn[i], outs[i][0], outs[i][1], ws)
        dsa.dsa_advance_seq_len(lat.seq_len, 130)
    torch.cuda.synchronize()
    for i in range(25):
        for r in range(3):
            rows = torch.cat([c.rows[r]] + [news[j, r] for j in range(i)])
            o, l, tol, ltol = latent_ref.step_expected(qs[i, r].double(), rows.double(), news[i, r].double(), 1, 512, c.scale, True)
            latent_ref.assert_near(outs[i][0][r], o, tol, "step %d of request %d" % (i, r))
            latent_ref.assert_near(outs[i][1][r], l, ltol, "lse of step %d of request %d" % (i, r))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,bound", [([3] * 200, 600), ([0, 700, 0, 1, 257, 256, 0], 1214), ([5] * 256, 1280), ([5] * 257, 1285), ([0] * 40, 1),
                                        ([0] * 255 + [300], 300), ([90, 400] * 10, 250), ([1], 1), ([1, 1], 2), ([2000, 10, 3, 900], 2913)])
def test_prompt_bounds_that_are_loose(dsa, dtype, lens, bound):
    """Upper bounds of the queries far above what most requests have (all tokens, say), and below what some have."""
    run_case(dsa, dtype, 2, 64, 32, lens, max_q=bound, seed=len(lens))
    if sum(lens) < 1500:
        run_case(dsa, dtype, 1, 128, 64, lens, [2 * n + 1 for n in lens], max_q=bound, seed=len(lens), causal=len(lens) % 2 == 0)
