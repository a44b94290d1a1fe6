"""Attention of drafted trees against the 64-bit reference (draft_ref): types, head layouts, lengths from nothing to
several splits, odd pages and strides, masks, requests without nodes or room, and rows that nobody sees holding NaN."""
import math

import numpy as np
import pytest
import torch

from tests import draft_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dsa():
    from paper_2609_19702_b200 import binding
    return binding


class Setup:
    """One batch: host copies in float64, device tensors, the cache's rows addressed by [page or request, token]."""

    def __init__(self, dsa, *, dtype=torch.bfloat16, d=128, hq=8, hkv=2, n=8, page=16, lens=(100, 37), prompt=20, branch=2,
                 counts=None, window=0, sinks=0, split=0, scale=0.0, cap=None, layout="token", shared=False, seed=0, poison=True,
                 chain=False):
        g = torch.Generator().manual_seed(seed * 1000 + d + hq + n + page + sum(lens))
        rng = np.random.default_rng(seed + n + len(lens))
        b = len(lens)
        self.dsa, self.b, self.n, self.d, self.hq, self.hkv, self.dtype = dsa, b, n, d, hq, hkv, dtype
        self.lens, self.prompt, self.window, self.sinks = list(lens), prompt, window, sinks
        self.cap = cap if cap is not None else max(list(lens) + [0]) + n
        rand = lambda *s: torch.randn(s, generator=g).to(dtype)  # noqa: E731
        blocks = -(-max(self.cap, 1) // page) if page else 0
        if page:
            self.table = torch.from_numpy(rng.permutation(b * blocks + 3)[:b * blocks].reshape(b, blocks).astype(np.int32))
            outer, inner = b * blocks + 3, page
        else:
            self.table, outer, inner = None, (1 if shared else b), max(self.cap, 1)
        # "token": [outer, token, head, D]; "head": [outer, head, token, D]; "wide": padded tokens and pages
        shape = {"token": (outer, inner, hkv, d), "head": (outer, hkv, inner, d), "wide": (outer, inner + 1, hkv + 1, d + 16)}[layout]
        full_k, full_v = rand(*shape), rand(*shape)
        view = {"token": lambda t: t, "head": lambda t: t.transpose(1, 2),
                "wide": lambda t: t[:, :inner, :hkv, :d]}[layout]
        self.shared, self.page = shared, page
        self.full = [full_k, full_v]
        self.view = view
        if poison:                                           # nothing but the cached rows is a number
            keep_k, keep_v = full_k.clone(), full_v.clone()
            full_k.fill_(math.nan)
            full_v.fill_(math.nan)
            for r in range(b):
                for s in range(max(0, min(self.lens[r], self.cap))):
                    if not self._seen_by_some(r, s):
                        continue
                    o, i = self.place(r, s)
                    view(full_k)[o, i] = view(keep_k)[o, i]
                    view(full_v)[o, i] = view(keep_v)[o, i]
        self.q, self.k_new, self.v_new = rand(b, n, hq, d), rand(b, n, hkv, d), rand(b, n, hkv, d)
        parent = np.full((b, n), -1, np.int32)
        for r in range(b):
            for i in range(1, n):
                parent[r, i] = i - 1 if chain else max(-1, i - 1 - int(rng.integers(0, 2 * branch + 1)))
        self.parent = parent
        counts = [n] * b if counts is None else list(counts)
        self.live = [0 if self.lens[r] < 0 else max(0, min(counts[r], n, self.cap - min(self.lens[r], self.cap))) for r in range(b)]
        if poison:
            for r in range(b):
                for t in (self.q, self.k_new, self.v_new):
                    t[r, self.live[r]:] = math.nan
        self.scale = scale or 1 / math.sqrt(d)
        dev = lambda t: t.cuda()  # noqa: E731
        self.dev_full = [dev(t) for t in self.full]
        kc, vc = (view(t) for t in self.dev_full)
        self.kc, self.vc = kc, vc
        self.problem = dsa.Problem(
            q=dev(self.q), k_cache=kc, v_cache=vc, strides=(0 if shared else kc.stride(0), kc.stride(1), kc.stride(2)),
            seq_len=torch.tensor(self.lens, dtype=torch.int32).cuda(), prompt_len=torch.full((b,), prompt, dtype=torch.int32).cuda(),
            num_kv_heads=hkv, max_seq_len=self.cap, max_prompt_len=prompt, block_table=None if self.table is None else dev(self.table),
            block_size=page, num_blocks=outer if page else 0, split_tokens=split, sm_scale=scale)
        self.diag = dsa.Diag(dsa.DSA_MASK_WINDOW, window, n_sink=sinks) if window else None
        self.tree = dsa.Tree(n, parent=None if chain else torch.from_numpy(parent).cuda(),
                             node_count=torch.tensor(counts, dtype=torch.int32).cuda())
        self.dk, self.dv = dev(self.k_new), dev(self.v_new)

    def _seen_by_some(self, r, s):
        p0 = min(self.prompt, self.lens[r]) + self.sinks
        return not self.window or s < p0 or self.lens[r] - s < self.window

    def place(self, r, s):
        if self.page:
            return int(self.table[r, s // self.page]), s % self.page
        return (0 if self.shared else r), s

    def run(self, out=None, lse=None, ws="new", stream=None):
        if out is None:
            out, lse = self.dsa.alloc_tree_outputs(self.problem)
            out.fill_(7.0)
            lse.fill_(7.0)
        if isinstance(ws, str):
            ws = self.dsa.alloc_tree_workspace(self.problem, self.diag, self.tree)
            if ws is not None:
                ws.fill_(255)                                # (NaN for whoever reads what nobody wrote)
        self.dsa.dsa_tree_step(self.problem, self.diag, self.tree, self.dk, self.dv, out, lse, ws, stream)
        return out, lse

    def reference(self, r):
        s = max(0, min(self.lens[r], self.cap))
        rows = [torch.stack([self.view(f)[self.place(r, i)] for i in range(s)]) if s else torch.zeros((0, self.hkv, self.d))
                for f in self.full]
        m = self.live[r]
        clean = lambda t: torch.cat([t[r, :m], torch.zeros_like(t[r, m:])]).double()  # noqa: E731
        return draft_ref.tree_reference(clean(self.q), rows[0].double(), rows[1].double(), clean(self.k_new), clean(self.v_new),
                                        self.parent[r], s, self.prompt, m, self.scale, self.window, self.sinks)

    def check(self, out, lse):
        torch.cuda.synchronize()
        assert self.dsa.dsa_wait_timeouts() == 0
        for r in range(self.b):
            ro, rl, weight, size, count = self.reference(r)
            tol, ltol = draft_ref.tree_tolerances(ro, rl, weight, size, count, self.d, self.dtype == torch.bfloat16)
            o, s = out[r].cpu().double(), lse[r].cpu().double()
            m = self.live[r]
            assert torch.equal(o[m:], torch.zeros_like(o[m:])) and torch.isneginf(s[m:]).all(), "request %d: nodes that are not there" % r
            assert torch.isfinite(o).all(), "request %d: a row that nobody sees came through" % r
            if m:
                assert ((o[:m] - ro[:m]).abs() <= tol[:m]).all(), "request %d: out off by %.3g of its bound" % (
                    r, ((o[:m] - ro[:m]).abs() / tol[:m]).max())
                assert ((s[:m] - rl[:m]).abs() <= ltol[:m]).all(), "request %d: lse off by %.3g of its bound" % (
                    r, ((s[:m] - rl[:m]).abs() / ltol[:m]).max())
        self.check_cache()

    def check_cache(self):
        """The new rows at their places, every other byte as it was."""
        for f, dev, new in zip(self.full, self.dev_full, (self.k_new, self.v_new)):
            want = f.clone()
            for r in range(self.b):
                for i in range(self.live[r]):
                    self.view(want)[self.place(r, self.lens[r] + i)] = new[r, i]
            bits = torch.int16 if self.dtype == torch.bfloat16 else torch.int32
            assert torch.equal(dev.cpu().view(bits), want.view(bits))


BOTH = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (4, 2), (8, 2), (16, 2)])
def test_head_layouts(dsa, dtype, d, hq, hkv):
    s = Setup(dsa, dtype=dtype, d=d, hq=hq, hkv=hkv, n=11, lens=(70, 3, 129), counts=(11, 4, 9))
    s.check(*s.run())


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 33, 63, 64])
def test_node_counts(dsa, dtype, n):
    s = Setup(dsa, dtype=dtype, n=n, hq=8, hkv=2, lens=(65, 40, 12), counts=(n, max(n - 1, 0), 1))
    s.check(*s.run())


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("hq,n", [(8, 64), (8, 17), (4, 64), (2, 64)])
def test_several_row_tiles(dsa, dtype, hq, n):
    s = Setup(dsa, dtype=dtype, hq=hq, hkv=1, n=n, lens=(130, 64), counts=(n, 16), window=50, sinks=2)
    s.check(*s.run())


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("lens", [(0,), (1,), (63, 64, 65), (127, 128, 129), (0, 500, 1)])
@pytest.mark.parametrize("page", [0, 16])
def test_lengths(dsa, dtype, lens, page):
    s = Setup(dsa, dtype=dtype, lens=lens, page=page, prompt=7)
    s.check(*s.run())


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("page", [1, 5, 7, 8, 24, 64, 100, 128, 192])
def test_pages(dsa, dtype, page):
    s = Setup(dsa, dtype=dtype, lens=(150, 33), page=page, counts=(8, 5))
    s.check(*s.run())


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("layout", ["token", "head", "wide"])
@pytest.mark.parametrize("page", [0, 16])
def test_strides(dsa, dtype, layout, page):
    s = Setup(dsa, dtype=dtype, lens=(90, 41), page=page, layout=layout)
    s.check(*s.run())


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("window,sinks,prompt", [(1, 0, 0), (1, 4, 0), (3, 0, 20), (16, 4, 20), (64, 1, 64), (65, 0, 1),
                                                 (1000, 4, 20), (2 ** 31 - 1, 2 ** 31 - 1, 20), (30, 4, 500)])
@pytest.mark.parametrize("page", [0, 5, 16])
def test_windows(dsa, dtype, window, sinks, prompt, page):
    s = Setup(dsa, dtype=dtype, lens=(200, 22, 0), window=window, sinks=sinks, prompt=prompt, page=page, n=9, branch=1)
    s.check(*s.run())


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("window", [0, 100])
@pytest.mark.parametrize("split", [64, 100, 256])
def test_splits(dsa, dtype, window, split):
    s = Setup(dsa, dtype=dtype, lens=(700, 1, 64, 310), split=split, window=window, sinks=4, counts=(8, 0, 8, 3))
    if not window or split < 256:                                 # (a window of 100 is seen in at most four tiles)
        assert dsa.alloc_tree_workspace(s.problem, s.diag, s.tree) is not None
    s.check(*s.run())


@pytest.mark.parametrize("dtype", BOTH)
def test_requests_without_nodes_or_room(dsa, dtype):
    # negative length; no node; a count beyond N; room for three nodes only; no room at all; a length beyond the cap
    s = Setup(dsa, dtype=dtype, lens=(-1, 30, 20, 57, 60, 75), counts=(8, 0, 99, 8, 8, 8), cap=60, prompt=5)
    assert s.live == [0, 0, 8, 3, 0, 0]
    s.check(*s.run())


@pytest.mark.parametrize("dtype", BOTH)
def test_chain_and_empty_parents(dsa, dtype):
    s = Setup(dsa, dtype=dtype, n=13, chain=True, lens=(40,))
    s.check(*s.run())
    s = Setup(dsa, dtype=dtype, n=13, lens=(40,))
    s.parent[:] = np.array([5, -7, 2, 99, 4, 4, 6, 5, 13, 8, 9, -1, 11], np.int32)      # roots wherever it is not in [0, i)
    s.tree.parent.copy_(torch.from_numpy(s.parent))
    s.check(*s.run())


@pytest.mark.parametrize("dtype", BOTH)
def test_scale_and_large_logits(dsa, dtype):
    s = Setup(dsa, dtype=dtype, lens=(300,), scale=1.5, n=5)          # softmax of a few weights, many rescalings
    s.check(*s.run())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,page", [(0, 16), (40, 16), (0, 0)])
def test_more_blocks_than_places(dsa, d, window, page):
    """Blocks that take over others' work: several hundred (request, kv head) pairs of very different lengths, among them
    requests without nodes, without cached tokens and without either."""
    rng = np.random.default_rng(d + window + page)
    lens = [int(x) for x in rng.integers(0, 200, size=130)]
    counts = [int(x) for x in rng.integers(0, 6, size=130)]
    lens[3] = lens[7] = counts[7] = 0
    s = Setup(dsa, d=d, hq=8, hkv=8, n=5, lens=lens, counts=counts, window=window, sinks=3, page=page, prompt=9)
    s.check(*s.run())


@pytest.mark.parametrize("b", [2, 100, 128, 129, 200, 256, 257])
def test_requests_of_unequal_length_and_number(dsa, b):
    """More blocks than places, so that requests are taken in the order of their tiles (up to 256 of them)."""
    rng = np.random.default_rng(b)
    hkv = max(2, -(-320 // b))
    lens = [int(x) for x in rng.choice([0, 1, 5, 64, 65, 130, 300, 301, -1], size=b)]
    s = Setup(dsa, d=64, hq=hkv, hkv=hkv, n=3, page=16, lens=lens, counts=[int(x) for x in rng.integers(0, 5, size=b)])
    s.check(*s.run())


def test_requests_share_a_cache(dsa):
    # a batch stride of 0: every request reads the same rows; nodes without room append nothing
    s = Setup(dsa, lens=(48, 48, 48), page=0, shared=True, cap=48, counts=(8, 8, 8))
    assert s.live == [0, 0, 0]
    s.check(*s.run())
    s = Setup(dsa, lens=(48, 20, 48), page=0, shared=True, cap=49, counts=(1, 0, 0))
    s.check(*s.run())


@pytest.mark.parametrize("dtype", BOTH)
def test_one_node_is_a_decode_step(dsa, dtype):
    s = Setup(dsa, dtype=dtype, n=1, lens=(130, 0, 77), window=64, sinks=4, chain=True, poison=False)
    out, lse = s.run()
    torch.cuda.synchronize()
    p = dsa.Problem(**{**s.problem.__dict__, "q": s.problem.q[:, 0].contiguous()})
    o1, l1 = dsa.alloc_outputs(p)
    dsa.dsa_decode_step(p, s.diag, s.dk[:, 0].contiguous(), s.dv[:, 0].contiguous(), o1, l1, dsa.alloc_workspace(p, s.diag))
    torch.cuda.synchronize()
    for r in range(3):
        _, rl, weight, size, count = s.reference(r)
        ro = s.reference(r)[0]
        tol, ltol = draft_ref.tree_tolerances(ro, rl, weight, size, count, s.d, dtype == torch.bfloat16)
        assert ((out[r].cpu().double() - o1[r].cpu().double()).abs() <= 2 * tol).all()
        assert ((lse[r].cpu().double() - l1[r].cpu().double()).abs() <= 2 * ltol).all()


@pytest.mark.parametrize("dtype", BOTH)
def test_same_bits_again_on_another_stream_and_replayed(dsa, dtype):
    s = Setup(dsa, dtype=dtype, lens=(700, 90, 300), split=128, n=20)
    out, lse = s.run()
    s.check(out, lse)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o2, l2 = dsa.alloc_tree_outputs(s.problem)
    w2 = dsa.alloc_tree_workspace(s.problem, s.diag, s.tree)
    s.run(o2, l2, w2, stream=side)
    side.synchronize()
    assert torch.equal(out, o2) and torch.equal(lse, l2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run(o2, l2, w2)
    for _ in range(3):
        o2.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, o2) and torch.equal(lse, l2)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("hq,n", [(2, 6), (8, 20)])
def test_nodes_without_a_page_are_stored_nowhere(dsa, dtype, hq, n):
    s = Setup(dsa, dtype=dtype, hq=hq, hkv=2, n=n, lens=(32, 40, 7), page=8, chain=True)
    table = s.problem.block_table
    spare = [x for x in range(s.problem.num_blocks) if x not in set(table.flatten().tolist())]
    table[0, 4:], table[1, 6:] = -1, s.problem.num_blocks                # the pages behind the cached tokens (and, of one, some new ones)
    s.table[0, 4:], s.table[1, 6:] = spare[0], spare[1]
    rows = [n, n, n]
    s.run()
    out, lse = s.run()
    # what the kernel may have written: rows 0 lacks all its pages, row 1 those from token 48 on
    live = s.live
    s.live = [0, min(n, 8), n]
    s.check_cache()
    s.live, s.check_cache = live, lambda: None
    assert live == rows
    s.check(out, lse)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("layout", ["pages", "requests", "tokens"])
def test_offsets_beyond_32_bits(dsa, dtype, layout):
    """Rows more than 2^31 elements behind the start of the cache: pages, a request's start, or a request's own tokens."""
    b, n, hq, hkv, d, length = 2, 6, 4, 2, 128, 40
    blocks = 2 ** 31 // (16 * hkv * d) + 1000
    size, strides = {"pages": (blocks * 16 * hkv * d, (16 * hkv * d, hkv * d, d)),
                     "requests": (2 ** 31 + 64 * hkv * d, (2 ** 31, hkv * d, d)),
                     "tokens": (2 ** 26 * 46, (hkv * d, 2 ** 26, d))}[layout]
    g = torch.Generator().manual_seed(3)
    rand = lambda *s: torch.randn(s, generator=g).to(dtype)  # noqa: E731
    flat = [torch.empty(size, dtype=dtype, device="cuda") for _ in range(2)]
    pages = [[blocks - 1, 2, blocks - 700], [0, blocks - 3, 1]]
    at = lambda r, s: (pages[r][s // 16] * strides[0] + s % 16 * strides[1] if layout == "pages" else  # noqa: E731
                       r * strides[0] + s * strides[1])
    rows = [rand(b, length, hkv, d) for _ in range(2)]
    for f, x in zip(flat, rows):
        for r in range(b):
            for s in range(length):
                f[at(r, s):at(r, s) + hkv * d] = x[r, s].reshape(-1).cuda()
    q, kn, vn = rand(b, n, hq, d), rand(b, n, hkv, d), rand(b, n, hkv, d)
    problem = dsa.Problem(q=q.cuda(), k_cache=flat[0], v_cache=flat[1], strides=strides, seq_len=torch.tensor([length] * b, dtype=torch.int32).cuda(),
                          prompt_len=torch.zeros((b,), dtype=torch.int32).cuda(), num_kv_heads=hkv, max_seq_len=length + n,
                          block_table=torch.tensor(pages, dtype=torch.int32).cuda() if layout == "pages" else None, block_size=16,
                          num_blocks=blocks)
    tree = dsa.Tree(n)
    out, lse = dsa.alloc_tree_outputs(problem)
    dsa.dsa_tree_step(problem, None, tree, kn.cuda(), vn.cuda(), out, lse, dsa.alloc_tree_workspace(problem, None, tree))
    torch.cuda.synchronize()
    assert dsa.dsa_wait_timeouts() == 0
    for r in range(b):
        ro, rl, weight, big, count = draft_ref.tree_reference(q[r].double(), rows[0][r].double(), rows[1][r].double(), kn[r].double(),
                                                              vn[r].double(), list(range(-1, n - 1)), length, 0, n, 1 / math.sqrt(d))
        tol, ltol = draft_ref.tree_tolerances(ro, rl, weight, big, count, d, dtype == torch.bfloat16)
        assert ((out[r].cpu().double() - ro).abs() <= tol).all() and ((lse[r].cpu().double() - rl).abs() <= ltol).all()
        for f, new in zip(flat, (kn, vn)):
            for i in range(n):
                assert torch.equal(f[at(r, length + i):at(r, length + i) + hkv * d].cpu(), new[r, i].reshape(-1))


def test_no_requests(dsa):
    q = torch.zeros((0, 4, 4, 64), device="cuda")
    none = torch.zeros((0,), dtype=torch.int32, device="cuda")
    cache = torch.zeros((4, 16, 2, 64), device="cuda")
    problem = dsa.Problem(q=q, k_cache=cache, v_cache=cache, strides=(2048, 128, 64), seq_len=none, prompt_len=none, num_kv_heads=2,
                          max_seq_len=64, block_table=none.view(0, 4), block_size=16, num_blocks=4)
    tree = dsa.Tree(4, parent=none.view(0, 4))
    out, lse = dsa.alloc_tree_outputs(problem)
    dsa.dsa_tree_step(problem, None, tree, q[:, :, :2].contiguous(), q[:, :, :2].contiguous(), out, lse)
    ver = dsa.Verify(none.view(0, 4), torch.zeros((0, 4, 100), device="cuda"))
    dsa.dsa_verify_tree(ver, tree, *dsa.alloc_verify_outputs(ver))
    problem.q = q[:, 0].contiguous()
    dsa.dsa_compact_kv(problem, none.view(0, 4), none, base=none, len_out=none)
    pool = dsa.PagePool(torch.zeros((4,), dtype=torch.int32, device="cuda"), 16)
    dsa.dsa_reserve_pages(pool, none.view(0, 4), none, 3, none)
    dsa.dsa_release_pages(pool, none.view(0, 4), none)
    dsa.dsa_fork_pages(pool, problem, none, none, none, dsa.alloc_fork_workspace(none))
    dsa.dsa_copy_pages(problem, none, none)
    torch.cuda.synchronize()


def test_two_calls_at_once(dsa):
    a = Setup(dsa, lens=(2000, 900, 1500, 60), split=256, n=30, poison=False)
    b = Setup(dsa, lens=(1700, 1900), split=192, n=64, hq=16, poison=False, seed=3)
    streams = [torch.cuda.Stream() for _ in range(2)]
    want = [x.run() for x in (a, b)]
    torch.cuda.synchronize()
    outs = [(*dsa.alloc_tree_outputs(x.problem), dsa.alloc_tree_workspace(x.problem, x.diag, x.tree)) for x in (a, b)]
    for _ in range(10):
        for x, o, st in zip((a, b), outs, streams):
            x.run(*o, stream=st)
    torch.cuda.synchronize()
    for (o, l), got in zip(want, outs):
        assert torch.equal(o, got[0]) and torch.equal(l, got[1])


def test_binding_refuses(dsa):
    s = Setup(dsa, lens=(20,))
    out, lse = dsa.alloc_tree_outputs(s.problem)
    with pytest.raises(ValueError):
        dsa.dsa_tree_step(s.problem, None, dsa.Tree(9), s.dk, s.dv, out, lse)
    with pytest.raises(ValueError):
        dsa.dsa_tree_step(s.problem, None, s.tree, s.dk[:, :, :1], s.dv, out, lse)
    with pytest.raises(ValueError):
        dsa.dsa_tree_step(s.problem, None, s.tree, s.dk.float(), s.dv, out, lse)
    with pytest.raises(ValueError):
        dsa.dsa_tree_step(s.problem, None, s.tree, s.dk, s.dv, out.float(), lse)
    with pytest.raises(ValueError):
        dsa.dsa_tree_step(s.problem, None, s.tree, s.dk, s.dv, out, lse[:, :, :1])
    with pytest.raises(ValueError):
        dsa.dsa_tree_step(s.problem, None, s.tree, s.dk, s.dv, out.cpu(), lse)
    grid = dsa.Diag(dsa.DSA_MASK_GRID, 16, 8, 4)
    with pytest.raises(dsa.DsaError):
        dsa.dsa_tree_step(s.problem, grid, s.tree, s.dk, s.dv, out, lse)
