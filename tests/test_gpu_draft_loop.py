"""The drafted-token calls as a decode loop uses them, one behind the other: pages reserved, every layer's tree
attention, verification, accepted rows moved up in all layers, pages given back.  A small model whose greedy tokens the
loop has to reproduce whatever the drafts are, in fp32 so that both ways of computing agree far better than two logits
lie apart."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

V, E, LAYERS, HQ, HKV, D, PAGE, CAP = 61, 96, 3, 4, 2, 64, 4, 64


@pytest.fixture(scope="module")
def dsa():
    from paper_2609_19702_b200 import binding
    return binding


class Model:
    """Layers of attention over a paged cache; the token's logical position is added to its embedding."""

    def __init__(self, dsa, batch, nodes):
        g = torch.Generator().manual_seed(11)
        r = lambda *s, scale=1.0: (torch.randn(s, generator=g) * scale).cuda()  # noqa: E731
        self.dsa, self.b, self.n = dsa, batch, nodes
        self.emb, self.pos, self.out = r(V, E), r(CAP + 16, E), r(E, V)              # (the same whatever `nodes` is)
        self.w = [{"q": r(E, HQ * D, scale=E ** -0.5), "k": r(E, HKV * D, scale=E ** -0.5), "v": r(E, HKV * D, scale=E ** -0.5),
                   "o": r(HQ * D, E, scale=(HQ * D) ** -0.5 * 3)} for _ in range(LAYERS)]
        blocks = batch * (CAP // PAGE) + 3
        self.k = torch.full((LAYERS, blocks, PAGE, HKV, D), float("nan"), device="cuda")
        self.v = torch.full_like(self.k, float("nan"))
        self.table = torch.full((batch, CAP // PAGE), -1, dtype=torch.int32, device="cuda")
        self.refs = torch.zeros((blocks,), dtype=torch.int32, device="cuda")
        self.refs[torch.tensor([0, 5, 6])] = 1                                   # pages that somebody else holds
        self.pool = dsa.PagePool(self.refs, PAGE)
        self.seq = torch.zeros((batch,), dtype=torch.int32, device="cuda")
        self.prompt = torch.zeros((batch,), dtype=torch.int32, device="cuda")
        self.status = torch.zeros((batch,), dtype=torch.int32, device="cuda")

    def problem(self, q, layer):
        return self.dsa.Problem(q=q, k_cache=self.k[layer], v_cache=self.v[layer], strides=(PAGE * HKV * D, HKV * D, D),
                                seq_len=self.seq, prompt_len=self.prompt, num_kv_heads=HKV, max_seq_len=CAP, block_table=self.table,
                                block_size=PAGE, num_blocks=self.refs.numel())

    def reserve(self, extra):
        self.dsa.dsa_reserve_pages(self.pool, self.table, self.seq, extra, self.status)

    def step(self, tokens):
        """One token per request, by dsa_decode_step; logits [B, V]."""
        x = self.emb[tokens] + self.pos[self.seq.long()]
        for layer, w in enumerate(self.w):
            q, k, v = ((x @ w[c]).view(self.b, -1, D).contiguous() for c in "qkv")
            p = self.problem(q, layer)
            out, lse = self.dsa.alloc_outputs(p)
            self.dsa.dsa_decode_step(p, None, k, v, out, lse, self.dsa.alloc_workspace(p))
            x = x + out.view(self.b, -1) @ w["o"]
        self.dsa.dsa_advance_seq_len(self.seq, CAP)
        return x @ self.out

    def tree_logits(self, tokens, depth, tree):
        """Logits [B, N, V] of a tree of drafted tokens."""
        x = self.emb[tokens] + self.pos[self.seq.long()[:, None] + depth]
        for layer, w in enumerate(self.w):
            q, k, v = ((x @ w[c]).view(self.b, self.n, -1, D).contiguous() for c in "qkv")
            p = self.problem(q, layer)
            out, lse = self.dsa.alloc_tree_outputs(p)
            self.dsa.dsa_tree_step(p, None, tree, k, v, out, lse, self.dsa.alloc_tree_workspace(p, None, tree))
            x = x + out.view(self.b, self.n, -1) @ w["o"]
        return x @ self.out

    def settle(self, path, accepted):
        """The accepted rows of all layers move up, and the pages behind them go back to the pool."""
        self.dsa.dsa_compact_kv(self.problem(torch.zeros((self.b, HQ, D), device="cuda"), 0), path, accepted, base=self.seq,
                                len_out=self.seq, num_layers=LAYERS, stride_layer=self.k.stride(0))
        self.dsa.dsa_release_pages(self.pool, self.table, self.seq)


def _drafts(rng, last, truth, at, n):
    """A tree of n nodes behind the settled token `last` of every request: parents, tokens, depths.  Its tokens are the
    true continuation's with probability 3/4."""
    b = len(last)
    parent, tokens, depth = (np.full((b, n), x, np.int32) for x in (-1, 0, 0))
    for r in range(b):
        tokens[r, 0] = last[r]
        for i in range(1, n):
            p = max(0, i - 1 - int(rng.integers(0, 3)))
            parent[r, i], depth[r, i] = p, depth[r, p] + 1
            # the truth behind this node, if the whole line so far is true
            line, j = [], i
            while j > 0:
                line.append(j)
                j = parent[r, j]
            true = all(tokens[r, x] == truth[r][at[r] + depth[r, x] - 1] for x in line[1:])
            tokens[r, i] = truth[r][at[r] + depth[r, i] - 1] if true and rng.random() < 0.75 else int(rng.integers(0, V))
    return parent, tokens, depth


def _sequential(dsa, first, steps):
    m = Model(dsa, len(first), 1)
    tokens, out = torch.tensor(first).cuda(), []
    for _ in range(steps):
        m.reserve(1)
        logits = m.step(tokens)
        top = logits.topk(2, -1).values
        assert (top[:, 0] - top[:, 1]).min() > 1e-3                              # no near ties in this model
        tokens = logits.argmax(-1)
        out.append(tokens.cpu().numpy())
    return np.stack(out, 1), m


def _rows(m, request, length):
    pages = m.table[request].long()
    pos = torch.arange(length, device="cuda")
    return m.k[:, pages[pos // PAGE], pos % PAGE], m.v[:, pages[pos // PAGE], pos % PAGE]


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("nodes", [1, 6, 11])
def test_greedy_loop_reproduces_the_models_tokens(dsa, nodes, captured):
    first, steps = [3, 17, 42], 40
    truth, ref = _sequential(dsa, first, steps + nodes + 1)
    rng = np.random.default_rng(nodes)
    m = Model(dsa, 3, nodes)
    tokens = torch.zeros((3, nodes), dtype=torch.int32, device="cuda")
    parent, depth = torch.zeros_like(tokens), torch.zeros_like(tokens)
    tree = dsa.Tree(nodes, parent=parent)
    logits = torch.zeros((3, nodes, V), device="cuda")
    ver = dsa.Verify(tokens, logits)
    path, accepted, word = dsa.alloc_verify_outputs(ver)

    def one_pass():
        m.reserve(nodes)
        logits.copy_(m.tree_logits(tokens.long(), depth.long(), tree))
        dsa.dsa_verify_tree(ver, tree, path, accepted, word)
        m.settle(path, accepted)

    graph = None
    if captured:
        dsa.dsa_prepare()
        state = [t.clone() for t in (m.seq, m.table, m.refs)]
        one_pass()                                                               # (the matrix products' own set-up)
        torch.cuda.synchronize()
        for t, s in zip((m.seq, m.table, m.refs), state):
            t.copy_(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            one_pass()
    out, last, passes = [[] for _ in first], list(first), 0
    while min(len(o) for o in out) < steps - nodes:
        p, t, d = _drafts(rng, last, truth, [len(o) for o in out], nodes)
        parent.copy_(torch.from_numpy(p))
        tokens.copy_(torch.from_numpy(t))
        depth.copy_(torch.from_numpy(d))
        if graph is not None:
            graph.replay()
        else:
            one_pass()
        assert m.status.tolist() == [0, 0, 0]
        for r in range(3):
            k = int(accepted[r])
            out[r] += [int(t[r, i]) for i in path[r, 1:k].tolist()] + [int(word[r])]
            last[r] = out[r][-1]
        passes += 1
        # a request that is far ahead has run out of room in this little cache: nothing is left to compare then
        if max(len(o) for o in out) > steps:
            break
    assert dsa.dsa_wait_timeouts() == 0
    for r in range(3):
        assert out[r] == truth[r][:len(out[r])].tolist()
    if nodes > 1:
        assert sum(len(o) for o in out) > 3 * passes                             # (drafts were accepted)
    # the rows in the cache are those of the tokens one by one, and the pool holds exactly the tables' pages
    for r in range(3):
        length = int(m.seq[r])
        assert length == len(out[r])
        for a, b in zip(_rows(m, r, length), _rows(ref, r, length)):
            assert torch.allclose(a, b, rtol=1e-4, atol=1e-4)
    held = torch.bincount(m.table[m.table >= 0].long(), minlength=m.refs.numel())
    held[torch.tensor([0, 5, 6])] += 1
    assert torch.equal(held.int(), m.refs)


def test_forked_requests_go_their_own_ways(dsa):
    """A request is branched in two; both continue with different tokens, and each has the rows that it would have alone."""
    n = 5
    m = Model(dsa, 2, n)
    alone = [Model(dsa, 2, n) for _ in range(2)]
    rng = np.random.default_rng(1)
    start = rng.integers(0, V, size=9)
    tree = dsa.Tree(n)

    def run(model, row, tokens, keep):
        """A chain of n tokens for one row (the other has no nodes), `keep` of which stand."""
        counts = torch.tensor([n if r == row else 0 for r in range(2)], dtype=torch.int32).cuda()
        tr = dsa.Tree(n, node_count=counts)
        need = torch.where(counts > 0, model.seq, -1)
        dsa.dsa_reserve_pages(model.pool, model.table, need.int(), n, model.status)
        tok = torch.from_numpy(np.tile(tokens, (2, 1))).long().cuda()
        out = model.tree_logits(tok, torch.arange(n).cuda()[None].expand(2, -1), tr)
        path = torch.arange(n, dtype=torch.int32).cuda()[None].expand(2, -1).contiguous()
        model.settle(path, torch.where(counts > 0, keep, 0).int())
        return out[row, :keep]

    for model in [m] + alone:
        for s in range(0, 9, 3):
            run(model, 0, np.concatenate([start[s:s + 3], [0, 0]]), 3)
    assert m.seq.tolist() == [9, 0]
    status, src, dst = (torch.tensor([x], dtype=torch.int32).cuda() for x in (9, 0, 1))
    dsa.dsa_fork_pages(m.pool, m.problem(torch.zeros((2, HQ, D), device="cuda"), 0), src, dst, status, dsa.alloc_fork_workspace(src),
                       num_layers=LAYERS, stride_layer=m.k.stride(0))
    assert status.tolist() == [0] and m.seq.tolist() == [9, 9]
    assert m.table[0, :2].tolist() == m.table[1, :2].tolist() and int(m.table[0, 2]) != int(m.table[1, 2])
    more = [rng.integers(0, V, size=(3, n)) for _ in range(2)]
    for i in range(3):
        for row in range(2):
            got = run(m, row, more[row][i], 4)
            want = run(alone[row], 0, more[row][i], 4)
            assert torch.allclose(got, want, rtol=1e-4, atol=1e-4)
    for row in range(2):
        for a, b in zip(_rows(m, row, 21), _rows(alone[row], 0, 21)):
            assert torch.allclose(a, b, rtol=1e-4, atol=1e-4)
    dsa.dsa_release_pages(m.pool, m.table)
    assert int(m.refs.sum()) == 3


def test_sampled_loop(dsa):
    """The same loop with probabilities and numbers: its tokens are those of the walk on the same probabilities."""
    from tests import draft_ref
    n, b = 7, 2
    m = Model(dsa, b, n)
    rng = np.random.default_rng(5)
    last = [4, 8]
    for _ in range(5):
        parent = np.array([[-1] + [max(0, i - 1 - int(rng.integers(0, 3))) for i in range(1, n)] for _ in range(b)], np.int32)
        depth = np.zeros((b, n), np.int64)
        tokens = rng.integers(0, V, size=(b, n)).astype(np.int32)
        tokens[:, 0] = last
        for r in range(b):
            for i in range(1, n):
                depth[r, i] = depth[r, parent[r, i]] + 1
        u = rng.random((b, n), dtype=np.float32)
        tree = dsa.Tree(n, parent=torch.from_numpy(parent).cuda())
        m.reserve(n)
        target = torch.softmax(m.tree_logits(torch.from_numpy(tokens).long().cuda(), torch.from_numpy(depth).cuda(), tree) * 0.2, -1)
        draft = torch.softmax(torch.randn((b, n, V), generator=torch.Generator().manual_seed(3)).cuda(), -1)
        ver = dsa.Verify(torch.from_numpy(tokens).cuda(), target, draft, torch.from_numpy(u).cuda())
        path, accepted, word = dsa.alloc_verify_outputs(ver)
        dsa.dsa_verify_tree(ver, tree, path, accepted, word)
        before = m.seq.tolist()
        m.settle(path, accepted)
        for r in range(b):
            want, w = draft_ref.verify_reference(tokens[r], target[r].cpu().double().numpy(), draft[r].cpu().double().numpy(), u[r],
                                                 parent[r], n, "sample")
            assert path[r, :len(want)].tolist() == want and int(word[r]) == w
            assert int(m.seq[r]) == before[r] + len(want)
        last = word.tolist()


CHILD = r"""
import torch
from paper_2609_19702_b200 import binding as dsa

torch.manual_seed(0)
i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
refs, table, seq, prompt = i32([1, 1, 1, 1] + [0] * 12), i32([[0, 1, -1, -1], [2, 3, -1, -1], [-1] * 4]), i32([30, 20, 0]), i32([4, 4, 0])
pool, status = dsa.PagePool(refs, 16), i32([9, 9, 9])
calls, state = [], [refs, table, seq, prompt, status]
for dtype, d, hq, n, split in ((torch.bfloat16, 128, 8, 6, 0), (torch.bfloat16, 64, 2, 6, 64), (torch.float32, 64, 2, 4, 0),
                               (torch.float32, 128, 8, 12, 0), (torch.float32, 128, 8, 4, 64)):
    k, v = torch.randn((2, 16, 16, 2, d), device="cuda").to(dtype), torch.randn((2, 16, 16, 2, d), device="cuda").to(dtype)
    prob = dsa.Problem(q=torch.randn((3, n, hq, d), device="cuda").to(dtype), k_cache=k, v_cache=v, strides=(32 * d, 2 * d, d), seq_len=seq,
                       prompt_len=prompt, num_kv_heads=2, max_seq_len=64, block_table=table, block_size=16, num_blocks=16,
                       split_tokens=split and 16)
    tree = dsa.Tree(n)
    out, lse = dsa.alloc_tree_outputs(prob)
    args = (prob, None, tree, torch.randn((3, n, 2, d), device="cuda").to(dtype), torch.randn((3, n, 2, d), device="cuda").to(dtype), out, lse,
            dsa.alloc_tree_workspace(prob, None, tree))
    calls.append(lambda a=args: dsa.dsa_tree_step(*a))
    state += [k, v, out, lse]
flat = dsa.Problem(q=torch.zeros((3, 2, d), dtype=dtype, device="cuda"), k_cache=k, v_cache=v, strides=prob.strides, seq_len=seq, prompt_len=prompt,
                   num_kv_heads=2, max_seq_len=64, block_table=table, block_size=16, num_blocks=16)
for dtype in (torch.float32, torch.bfloat16):
    for vocab in (1000, 30000, 230000):
        for u in (None, torch.rand((3, 3)).cuda()):
            probs = torch.softmax(torch.randn((3, 3, vocab), device="cuda") * 3, -1).to(dtype)
            ver = dsa.Verify(probs.argmax(-1).roll(1, 1).int(), probs, None if u is None else probs.roll(1, 0), u)
            outs = dsa.alloc_verify_outputs(ver)
            calls.append(lambda a=(ver, dsa.Tree(3), *outs): dsa.dsa_verify_tree(*a))
            state += list(outs)
ws, one, two = dsa.alloc_fork_workspace(i32([0])), i32([0]), i32([2])
keep, count, pages = i32([[0, 2, 3]] * 3), i32([3, 2, 0]), [i32([0]), i32([15])]
calls = [lambda: dsa.dsa_reserve_pages(pool, table, seq, 16, status)] + calls + [
    lambda: dsa.dsa_compact_kv(flat, keep, count, base=seq, len_out=seq, num_layers=2, stride_layer=k.stride(0)),
    lambda: dsa.dsa_release_pages(pool, table, seq),
    lambda: dsa.dsa_fork_pages(pool, flat, one, two, status[:1], ws, 2, k.stride(0)),
    lambda: dsa.dsa_copy_pages(flat, *pages, 2, k.stride(0))]
start = [t.clone() for t in state]
torch.cuda.synchronize()

dsa.dsa_prepare()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):          # the very first of these calls in this process
    for call in calls:
        call()
graph.replay()
torch.cuda.synchronize()
got = [t.clone() for t in state]
for t, s in zip(state, start):
    t.copy_(s)
for call in calls:
    call()
torch.cuda.synchronize()
bits = lambda t: t.contiguous().view(torch.uint8)
for i, (a, b) in enumerate(zip(got, state)):
    assert torch.equal(bits(a), bits(b)), i
assert seq.tolist() == [33, 22, 33] and status[0] == 0 and dsa.dsa_wait_timeouts() == 0
print("CAPTURED-FIRST-CALLS-OK")
"""


def test_first_calls_of_a_process_can_be_captured_after_prepare():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    env = dict(os.environ, PYTHONPATH=root + os.pathsep + os.environ.get("PYTHONPATH", ""))
    res = subprocess.run([sys.executable, "-c", CHILD], cwd=root, env=env, capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stdout[-2000:] + res.stderr[-4000:]
    assert "CAPTURED-FIRST-CALLS-OK" in res.stdout
