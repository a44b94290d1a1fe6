"""Verification of drafted tokens against the 64-bit walk of draft_ref: whole numbers, equal ones."""
import numpy as np
import pytest
import torch

from tests import draft_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dsa():
    from paper_2609_19702_b200 import binding
    return binding


def _draw(rng, b, n, v, branch, mode, dtype, sharp=1.0, counts=None, pad=0, chain=False):
    """Inputs as in use: the children of a node drawn from the draft's row there."""
    logits = rng.normal(size=(b, n, v)) * 2 * sharp
    soft = lambda x: np.exp(x - x.max(-1, keepdims=True)) / np.exp(x - x.max(-1, keepdims=True)).sum(-1, keepdims=True)  # noqa: E731
    rounded = lambda x: torch.from_numpy(x).to(dtype)  # noqa: E731
    p, q = rounded(soft(logits)), rounded(soft(logits + 0.4 * rng.normal(size=logits.shape)))
    parent = np.full((b, n), -1, np.int32)
    tokens = rng.integers(0, v, size=(b, n)).astype(np.int32)
    for r in range(b):
        for i in range(1, n):
            parent[r, i] = i - 1 if chain else max(0, i - 1 - int(rng.integers(0, 2 * branch + 1)))
            row = q[r, parent[r, i]].double().numpy()
            if mode == "greedy":
                row = p[r, parent[r, i]].double().numpy()
                tokens[r, i] = np.argsort(-row, kind="stable")[int(rng.integers(0, min(v, 3)))]
            else:
                tokens[r, i] = rng.choice(v, p=row / row.sum())
    u = rng.random((b, n), dtype=np.float32)
    padded = lambda t: torch.cat([t, torch.full((b, n, pad), 9.0, dtype=dtype)], -1)  # noqa: E731
    return dict(p=p, q=q, dp=padded(p).cuda()[..., :v], dq=padded(q).cuda()[..., :v], parent=parent, tokens=tokens, u=u,
                counts=[n] * b if counts is None else counts, mode=mode, chain=chain)


def _run(dsa, c, stream=None, outs=None):
    mode = c["mode"]
    b, n = c["tokens"].shape
    tree = dsa.Tree(n, parent=None if c["chain"] else torch.from_numpy(c["parent"]).cuda(),
                    node_count=torch.tensor(c["counts"], dtype=torch.int32).cuda())
    ver = dsa.Verify(torch.from_numpy(c["tokens"]).cuda(), c["dp"], c["dq"] if mode == "sample" else None,
                     None if mode == "greedy" else torch.from_numpy(c["u"]).cuda())
    outs = outs or dsa.alloc_verify_outputs(ver)
    for t in outs:
        t.fill_(77)
    dsa.dsa_verify_tree(ver, tree, *outs, stream)
    torch.cuda.synchronize()
    return outs


def _check(dsa, c):
    path, accepted, word = (t.cpu().numpy() for t in _run(dsa, c))
    b, n = c["tokens"].shape
    lengths = []
    for r in range(b):
        m = max(0, min(c["counts"][r], n))
        want, w = draft_ref.verify_reference(c["tokens"][r], c["p"][r].double().numpy(), c["q"][r].double().numpy(), c["u"][r],
                                             c["parent"][r], m, c["mode"])
        assert accepted[r] == len(want) and list(path[r]) == want + [-1] * (n - len(want)) and word[r] == w, (
            r, list(path[r]), want, word[r], w)
        lengths.append(len(want))
    return lengths


MODES = ["sample", "point", "greedy"]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("v", [1, 2, 127, 128, 129, 1000, 8193, 20000])
def test_vocabularies(dsa, dtype, mode, v):
    rng = np.random.default_rng(v)
    _check(dsa, _draw(rng, 5, 9, v, 2, mode, dtype, counts=[9, 0, 1, 5, 20]))


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("v", [2049, 65537, 100003, 131072, 150001, 230003])
def test_large_vocabularies(dsa, mode, v):
    rng = np.random.default_rng(v)
    _check(dsa, _draw(rng, 3, 5, v, 1, mode, torch.bfloat16, sharp=0.2))
    _check(dsa, _draw(rng, 2, 6, v, 0, mode, torch.float32, pad=1))


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("n,branch,chain", [(1, 1, False), (2, 1, False), (33, 1, False), (64, 4, False), (64, 0, False), (17, 0, True)])
def test_trees(dsa, mode, n, branch, chain):
    rng = np.random.default_rng(n + branch)
    lengths = []
    for dtype in (torch.float32, torch.bfloat16):
        lengths += _check(dsa, _draw(rng, 12, n, 300, branch, mode, dtype, chain=chain))
    if n >= 17 and mode != "point":                               # (a drawn token seldom stands as a chosen one)
        assert max(lengths) > 2                                   # (walks of some length were walked)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("b", [1, 2, 40, 160, 400])
def test_batches(dsa, mode, b):
    rng = np.random.default_rng(b)
    _check(dsa, _draw(rng, b, 6, 9000 if b <= 40 else 500, 1, mode, torch.float32))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("pad", [1, 3, 8])
def test_padded_rows(dsa, dtype, mode, pad):
    rng = np.random.default_rng(pad)
    _check(dsa, _draw(rng, 4, 8, 1001, 1, mode, dtype, pad=pad))


@pytest.mark.parametrize("mode", ["sample", "point"])
def test_many_rejections(dsa, mode):
    """One node with all others as its children, numbers near 1: turned down one after the other."""
    rng = np.random.default_rng(4)
    c = _draw(rng, 6, 20, 50, 1, mode, torch.float32, sharp=0.3)
    c["parent"][:, 1:] = 0
    c["u"][:, 1:] = np.nextafter(np.float32(1), np.float32(0))
    c["tokens"][2, 1:] = c["tokens"][2, 1]                         # the same token again and again
    _check(dsa, c)
    c["u"][:, :] = 0.0
    _check(dsa, c)
    c["u"][:, 0] = np.nextafter(np.float32(1), np.float32(0))
    _check(dsa, c)


def test_tokens_outside_the_vocabulary_change_nothing(dsa):
    rng = np.random.default_rng(5)
    for mode in MODES:
        c = _draw(rng, 4, 8, 100, 2, mode, torch.float32)
        c["tokens"][:, 2], c["tokens"][:, 5] = -1, 100
        c["tokens"][3] = 2 ** 31 - 1
        assert _check(dsa, c)[3] == 1


def test_draft_equal_to_target_always_stands(dsa):
    rng = np.random.default_rng(6)
    c = _draw(rng, 8, 10, 3000, 0, "sample", torch.float32, chain=True)
    c["q"], c["dq"] = c["p"], c["dp"]
    for r in range(8):
        for i in range(1, 10):
            row = c["p"][r, i - 1].double().numpy()
            c["tokens"][r, i] = rng.choice(3000, p=row / row.sum())
    assert _check(dsa, c) == [10] * 8


def test_nothing_left_and_nothing_there(dsa):
    """The draft covers the target everywhere: the residual is empty, the token comes from the target's row itself;
    a row without a positive entry gives -1."""
    p = torch.zeros((2, 2, 256))
    p[0, :, 10], p[0, :, 200] = 0.25, 0.25
    q = torch.full((2, 2, 256), 0.5)
    c = dict(p=p, q=q, dp=p.cuda(), dq=q.cuda(), parent=np.array([[-1, 0]] * 2, np.int32), tokens=np.array([[0, 10]] * 2, np.int32),
             u=np.array([[0.6, 0.9]] * 2, np.float32), counts=[2, 2], mode="sample", chain=False)
    path, accepted, word = _run(dsa, c)
    assert path.tolist() == [[0, -1]] * 2 and accepted.tolist() == [1, 1] and word.tolist() == [200, -1]


def test_greedy_ties_and_equal_scores(dsa):
    for v in (7, 300, 20000):
        p = torch.zeros((3, 2, v))
        p[1, :, v // 2:], p[2] = 1.0, -float("inf")
        c = dict(p=p, q=p, dp=p.cuda(), dq=p.cuda(), parent=np.array([[-1, 0]] * 3, np.int32),
                 tokens=np.array([[0, 0], [0, v // 2], [0, 0]], np.int32), u=np.zeros((3, 2), np.float32), counts=[2] * 3,
                 mode="greedy", chain=True)
        path, accepted, word = _run(dsa, c)
        assert word.tolist() == [0, v // 2, 0] and accepted.tolist() == [2, 2, 2]


def test_rows_beyond_32_bits(dsa):
    b, n, v = 520, 64, 65536
    p = torch.empty((b, n, v), dtype=torch.bfloat16, device="cuda")
    last = torch.zeros((2, n, v), dtype=torch.bfloat16)
    word = np.random.default_rng(0).integers(0, v, size=(2, n))
    for r in range(2):
        last[r, np.arange(n), word[r]] = 1.0
    p[-2:] = last.cuda()
    tokens = np.zeros((b, n), np.int32)
    tokens[-2:, 1:] = word[:, :-1]
    tokens[-1, 40] = (word[1, 39] + 1) % v
    ver = dsa.Verify(torch.from_numpy(tokens).cuda(), p)
    path, accepted, nxt = dsa.alloc_verify_outputs(ver)
    dsa.dsa_verify_tree(ver, dsa.Tree(n), path, accepted, nxt)
    assert accepted[-2:].tolist() == [64, 40] and nxt[-2:].tolist() == [int(word[0, 63]), int(word[1, 39])]
    ver = dsa.Verify(ver.tokens, p, None, torch.zeros((b, n), device="cuda"))
    dsa.dsa_verify_tree(ver, dsa.Tree(n), path, accepted, nxt)
    assert accepted[-2:].tolist() == [64, 40] and nxt[-2:].tolist() == [int(word[0, 63]), int(word[1, 39])]


def test_greedy_counts_a_nan_as_the_lowest(dsa):
    for v in (7, 300, 20000):
        p = torch.full((3, 2, v), float("nan"))
        p[0, :, v // 2], p[1, :, v - 1] = -3.0, -float("inf")
        c = dict(p=p, q=p, dp=p.cuda(), dq=p.cuda(), parent=np.array([[-1, 0]] * 3, np.int32),
                 tokens=np.array([[0, v // 2], [0, 0], [0, 0]], np.int32), u=np.zeros((3, 2), np.float32), counts=[2] * 3,
                 mode="greedy", chain=True)
        path, accepted, word = _run(dsa, c)
        assert word.tolist() == [v // 2, 0, 0] and accepted.tolist() == [2, 2, 2]


@pytest.mark.parametrize("mode", ["sample", "point"])
def test_probabilities_that_are_none(dsa, mode):
    """NaN, infinite or negative entries, and numbers of 1 or NaN: a token or -1, and the other requests' tokens as they are."""
    rng = np.random.default_rng(3)
    c = _draw(rng, 6, 9, 5000, 2, mode, torch.float32)
    want = [t.clone() for t in _run(dsa, c)]
    for r, x in enumerate((float("nan"), float("inf"), -1.0)):
        c["dp"][r, :, ::7] = x
        c["dq"][r, :, ::5] = x
    c["u"][3] = 1.0
    c["u"][4] = float("nan")
    path, accepted, word = _run(dsa, c)
    assert torch.equal(path[5], want[0][5]) and accepted[5] == want[1][5] and word[5] == want[2][5]
    assert ((word >= -1) & (word < 5000)).all() and ((accepted >= 1) & (accepted <= 9)).all()


def test_accepted_tokens_follow_the_target(dsa):
    """One drafted token and the last one: over many numbers the first of the two that stands is distributed as p says,
    whatever q is.  64 cells of 200000 draws: every cell within five standard deviations, for fixed numbers."""
    rng = np.random.default_rng(7)
    b, v = 200000, 64
    row = lambda: np.exp(rng.normal(size=v))  # noqa: E731
    p, q = row(), row()
    p, q = p / p.sum(), q / q.sum()
    dp = torch.from_numpy(np.stack([p, np.full(v, 1 / v)])).float().cuda().expand(b, 2, v).contiguous()
    dq = torch.from_numpy(np.stack([q, q])).float().cuda().expand(b, 2, v).contiguous()
    tokens = np.zeros((b, 2), np.int32)
    tokens[:, 1] = rng.choice(v, size=b, p=q)
    c = dict(dp=dp, dq=dq, parent=np.array([[-1, 0]] * b, np.int32), tokens=tokens, u=rng.random((b, 2), dtype=np.float32),
             counts=[2] * b, mode="sample", chain=True)
    _, accepted, word = (t.cpu().numpy() for t in _run(dsa, c))
    got = np.bincount(np.where(accepted == 2, tokens[:, 1], word), minlength=v)
    sd = np.sqrt(b * p * (1 - p))
    assert (np.abs(got - b * p) <= 5 * sd).all()


def test_streams_and_graphs(dsa):
    rng = np.random.default_rng(8)
    c = _draw(rng, 9, 16, 30000, 2, "sample", torch.float32)
    want = [t.clone() for t in _run(dsa, c)]
    tree = dsa.Tree(16, parent=torch.from_numpy(c["parent"]).cuda())
    ver = dsa.Verify(torch.from_numpy(c["tokens"]).cuda(), c["dp"], c["dq"], torch.from_numpy(c["u"]).cuda())
    outs = dsa.alloc_verify_outputs(ver)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    dsa.dsa_verify_tree(ver, tree, *outs, side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dsa.dsa_verify_tree(ver, tree, *outs)
    for t in outs:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))
