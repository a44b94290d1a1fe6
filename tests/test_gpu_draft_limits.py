"""Decoding with drafted tokens where pages or room run out: lengths count nothing that was stored nowhere, and a loop that
leaves nodes without room out of node_count gives the model's tokens all the same."""
import os
import re

import numpy as np
import pytest
import torch

from tests import draft_ref
from tests.test_gpu_draft_loop import CAP, LAYERS, PAGE, V, Model, _drafts, _rows, _sequential
from tests.test_gpu_pages import Cache, _int

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dsa():
    from paper_2609_19702_b200 import binding
    return binding


@pytest.mark.parametrize("where", ["apart", "base", "counts"])
def test_lengths_stop_at_rows_that_are_nowhere(dsa, where):
    """Rows whose own place or the one they go to lies outside the cache or has no page end the kept ones."""
    page, m = 8, 12
    c = Cache(dsa, 9, m, page)
    for r, e in ((1, 4), (2, 2), (3, 0), (5, 11), (8, 3)):
        c.table[r, e] = -1
    c.table[4, 5] = 10 ** 6
    lists = [list(range(0, 80, 2)) for _ in range(9)]
    lists[6] = list(range(40))                                     # nothing moves
    lists[7] = list(range(10)) + list(range(60, 90))
    lists[8] = list(range(40))                                     # nothing moves, but a page is missing
    base = [3, 0, 6, 0, 1, 7, 50, 12, 5]
    counts = [40, 40, 40, 40, 40, 40, 40, 99, 30]
    want = []
    for r in range(9):
        kept = min(counts[r], 40)
        gone = [i for i in range(kept) for at in (base[r] + lists[r][i], base[r] + i)
                if not (at < m * page and 0 <= int(c.table[r, at // page]) < c.problem.num_blocks)]
        want.append(base[r] + min(gone + [kept]))
    assert want == [43, 16, 11, 0, 21, 47, 90, 46, 24]
    first, keep, n = _int(base), _int(lists), _int(counts)
    out = {"apart": _int([0] * 9), "base": first, "counts": n}[where]
    dsa.dsa_compact_kv(c.problem, keep, n, base=first, len_out=out)
    assert out.tolist() == want


def test_lengths_of_long_lists(dsa):
    # the missing page lies behind several stretches of the list; and positions outside the cache
    c = Cache(dsa, 4, 200, 4)
    c.table[0, 160] = c.table[1, 199] = c.table[2, 0] = -1
    keep = [list(range(100, 700)), list(range(200, 800)), list(range(600)), list(range(201, 801))]
    out = _int([7] * 4)
    dsa.dsa_compact_kv(c.problem, _int(keep), _int([600] * 4), len_out=out)
    assert out.tolist() == [540, 596, 0, 599]
    dsa.dsa_compact_kv(c.problem, _int([[0, 1]] * 4), _int([2] * 4), base=_int([798, 799, -1, 2 ** 31 - 1]), len_out=out)
    assert out.tolist() == [800, 799, -1, 2 ** 31 - 1]


@pytest.mark.parametrize("rows,m", [(6, 6), (1300, 70)])
def test_a_source_without_its_pages_is_not_branched(dsa, rows, m):
    """A page that is missing within the source's length (the part-filled last one, or one in front of it): the branch is
    refused and nothing changes; what is missing behind the length matters to nobody."""
    page, hkv = 4, 1
    held = min(m, 6)                                               # pages that a source has
    lens = [held * page - 2] * rows + [0] * rows
    table = np.full((2 * rows, m), -1, np.int32)
    table[:rows, :held] = np.arange(rows * held).reshape(rows, held)
    blocks = rows * held + rows
    c = Cache(dsa, 2 * rows, m, page, blocks=blocks, hkv=hkv, table=table, lens=lens)
    was = np.array(table)
    for r, (e, x) in {0: (held - 1, -1), 1: (0, -1), 2: (2, blocks), 3: (1, 10 ** 9), rows - 1: (held - 2, -5)}.items():
        was[r, e] = x
    c.table.copy_(torch.from_numpy(was))
    refs = np.zeros(blocks, np.int32)
    refs[:rows * held] = 1
    pool, status = dsa.PagePool(torch.from_numpy(refs).cuda(), page), _int([9] * rows)
    src, dst = list(range(rows)), list(range(2 * rows - 1, rows - 1, -1))
    dsa.dsa_fork_pages(pool, c.problem, _int(src), _int(dst), status, dsa.alloc_fork_workspace(status))
    bad = {0, 1, 2, 3, rows - 1}
    assert status.tolist() == [2 if r in bad else 0 for r in src]
    want, fresh = np.array(was), rows * held
    for r in src:
        if r in bad:
            continue
        want[dst[r], :held] = was[r, :held]
        want[dst[r], held - 1] = fresh
        refs[was[r, :held - 1]] += 1
        refs[fresh] = 1
        lens[dst[r]] = lens[r]
        for t in c.host:
            t[:, fresh, :page - 2] = t[:, was[r, held - 1], :page - 2]
        fresh += 1
    assert np.array_equal(c.table.cpu().numpy(), want) and pool.ref_count.tolist() == refs.tolist()
    assert c.seq.tolist() == lens and c.same()


@pytest.mark.parametrize("blocks", [40, 20000])
def test_reserve_passes_over_negative_counts(dsa, blocks):
    """A count below 0 (a caller's own mark, say) is no free page, stays as it is and shifts nobody's pages."""
    rng = np.random.default_rng(blocks)
    rows, m, page = 12, 5, 4
    refs = np.where(rng.random(blocks) < 0.4, -rng.integers(1, 9, size=blocks), 0).astype(np.int32)
    refs[0], refs[1], refs[-1] = -1, -(2 ** 31) + m, -3
    table = np.full((rows, m), -1, np.int32)
    table[3, 1] = 2                                                # (a row with a hole)
    refs[2] = 1
    lens = rng.integers(0, 2 * page, size=rows).tolist()
    lens[3] = 3 * page
    pool, dt, status = dsa.PagePool(torch.from_numpy(refs).cuda(), page), torch.from_numpy(table).cuda(), _int([9] * rows)
    dsa.dsa_reserve_pages(pool, dt, _int(lens), 0, status)
    model = draft_ref.Pool(refs, table, page)
    assert status.tolist() == model.reserve(lens, 0)               # (the small pool runs out)
    assert dt.tolist() == model.table and pool.ref_count.tolist() == model.refs
    assert (refs < 0).sum() == sum(x < 0 for x in model.refs)


def _loop(dsa, m, rng, last, out, truth, gate, passes, between=None):
    """Passes of the loop; `gate`: nodes without room or pages are left out of node_count."""
    b, n = m.b, m.n
    parent, tokens, depth = (torch.zeros((b, n), dtype=torch.int32, device="cuda") for _ in range(3))
    count = torch.full((b,), n, dtype=torch.int32, device="cuda")
    tree = dsa.Tree(n, parent=parent, node_count=count)
    logits = torch.zeros((b, n, V), device="cuda")
    ver = dsa.Verify(tokens, logits)
    path, accepted, word = dsa.alloc_verify_outputs(ver)
    for step in range(passes):
        p, t, d = _drafts(rng, last, truth, [len(o) for o in out], n)
        for x, y in zip((parent, tokens, depth), (p, t, d)):
            x.copy_(torch.from_numpy(y))
        m.reserve(n)
        if gate:
            count.copy_(torch.where((m.status == 0) & (m.seq >= 0), (CAP - m.seq).clamp(0, n), 0))
        logits.copy_(m.tree_logits(tokens.long(), depth.long().clamp(max=15), tree))
        dsa.dsa_verify_tree(ver, tree, path, accepted, word)
        m.settle(path, accepted)
        for r in range(b):
            k = int(accepted[r])
            if k:
                out[r] += [int(t[r, i]) for i in path[r, 1:k].tolist()] + [int(word[r])]
                last[r] = out[r][-1]
        if between is not None:
            between(step)


@pytest.mark.parametrize("nodes", [3, 7])
def test_a_pool_that_runs_out(dsa, nodes):
    """Two requests share too few pages.  The one that gets none waits with no nodes, and goes on when the other's are given
    back; what it says in the end is what it says alone."""
    first, steps = [3, 17], 45
    truth, ref = _sequential(dsa, first, steps + nodes + 1)
    m = Model(dsa, 2, nodes)
    free = (m.refs == 0).nonzero()[:, 0]
    m.refs[free[9:]] = 1                                           # nine pages are left: not enough for both
    rng, out, last = np.random.default_rng(nodes), [[], []], list(first)
    lengths, waited = [], []

    def between(step):
        lengths.append(m.seq.tolist())
        waited.append(m.status.tolist())

    _loop(dsa, m, rng, last, out, truth, True, 12, between)
    assert any(s != [0, 0] for s in waited)
    for r in range(2):
        assert out[r] == truth[r][:len(out[r])].tolist() and int(m.seq[r]) == len(out[r])
    far = max(range(2), key=lambda r: len(out[r]))                 # the request that is further gives all of its pages back
    other = 1 - far
    keep = torch.full((2,), -1, dtype=torch.int32, device="cuda")
    keep[far] = 0
    dsa.dsa_release_pages(m.pool, m.table, keep)
    m.seq[far] = -1                                                # (and is no longer served)
    had = len(out[other])
    _loop(dsa, m, rng, last, out, truth, True, 4)
    assert len(out[other]) > had and int(m.seq[far]) == -1
    assert out[other] == truth[other][:len(out[other])].tolist()
    for a, b in zip(_rows(m, other, int(m.seq[other])), _rows(ref, other, int(m.seq[other]))):
        assert torch.allclose(a, b, rtol=1e-4, atol=1e-4)
    assert dsa.dsa_wait_timeouts() == 0


@pytest.mark.parametrize("nodes", [2, 7])
def test_lengths_without_the_gate(dsa, nodes):
    """A caller who does not gate: some tokens of the answer are lost to it, but no length counts a row without a page or
    beyond the cache, so that later passes read nothing that is another request's."""
    first = [3, 17, 42]
    truth, _ = _sequential(dsa, first, 50)
    m = Model(dsa, 3, nodes)
    free = (m.refs == 0).nonzero()[:, 0]
    m.refs[free[20:]] = 1
    rng, out, last = np.random.default_rng(nodes), [[], [], []], list(first)
    before, seen = [[0, 0, 0]], []

    def between(step):
        now = m.seq.tolist()
        seen.append(m.status.tolist())
        for r in range(3):
            assert before[0][r] <= now[r] <= CAP
            pages = m.table[r, :-(-now[r] // PAGE)]
            assert ((pages >= 0) & (pages < m.refs.numel())).all()
            for rows in _rows(m, r, now[r]):                       # every row that is counted was stored (the cache began as NaN)
                assert torch.isfinite(rows).all()
        before[0] = now
        for o in out:
            del o[40:]                                             # (drafts are taken from a table of 50 tokens)

    _loop(dsa, m, rng, last, out, truth, False, 40, between)
    assert any(s != [0, 0, 0] for s in seen)
    assert dsa.dsa_wait_timeouts() == 0


def test_a_request_that_reaches_the_end_of_the_cache(dsa):
    nodes, first = 5, [3, 17]
    truth, _ = _sequential(dsa, first, CAP)
    m = Model(dsa, 2, nodes)
    rng, out, last = np.random.default_rng(2), [[], []], list(first)

    def between(step):
        assert max(m.seq.tolist()) <= CAP
        for r in range(2):                                         # (drafts beyond the model's tokens are not looked up)
            assert len(out[r]) <= len(truth[r])

    _loop(dsa, m, rng, last, out, np.concatenate([truth, np.zeros((2, nodes), truth.dtype)], 1), True, 60, between)
    for r in range(2):
        assert int(m.seq[r]) == len(out[r]) > CAP - nodes
        assert out[r] == truth[r][:len(out[r])].tolist()
    assert m.status.tolist() != [0, 0] and LAYERS > 1


def test_the_documented_loop_runs(dsa):
    """README's pass with drafted tokens, as it stands there, twice: the second one behind the lengths of the first."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "README.md")).read()
    code = next(x for x in re.findall(r"```python\n(.*?)```", text, flags=re.S) if "dsa_tree_step" in x)
    b, n, hq, hkv, d, layers, vocab, s_max = 3, 5, 4, 2, 128, 2, 50, 96
    blocks = 20
    g = torch.Generator().manual_seed(0)
    rand = lambda *s: torch.randn(s, generator=g).bfloat16().cuda()  # noqa: E731
    k, v = rand(layers, blocks, 16, hkv, d), rand(layers, blocks, 16, hkv, d)
    seq = _int([30, 16, -1])                                       # (row 2 is free for a branch)
    table = torch.full((b, s_max // 16), -1, dtype=torch.int32, device="cuda")
    table[0, :2], table[1, 0] = _int([4, 7]), 2
    refs = _int([0] * blocks)
    refs[_int([2, 4, 7]).long()] = 1
    probs = torch.softmax(torch.randn((b, n, vocab), generator=g) * 3, -1).cuda()
    names = dict(dsa=dsa, torch=torch, N=n, S_max=s_max, L=layers, layer_stride=k.stride(0), diag=None, block_table=table, seq_len=seq,
                 ref_count=refs, parent=_int([[-1, 0, 0, 1, 2]] * b), count=_int([0] * b), status=_int([9] * b), k_new=rand(b, n, hkv, d),
                 v_new=rand(b, n, hkv, d), tokens=_int([[0, 1, 2, 3, 4]] * b), target_probs=probs, draft_probs=probs.roll(1, 0),
                 uniforms=torch.rand((b, n), generator=g).cuda(), path=_int([[9] * n] * b), accepted=_int([9] * b), next_token=_int([9] * b),
                 src=_int([0]), dst=_int([2]), forked=_int([9]))
    names["layers"] = [dsa.Problem(q=rand(b, n, hq, d), k_cache=k[i], v_cache=v[i], strides=k[i].stride()[:3], seq_len=seq,
                                   prompt_len=_int([0] * b), num_kv_heads=hkv, max_seq_len=s_max, block_table=table, block_size=16,
                                   num_blocks=blocks) for i in range(layers)]
    names["out"], names["lse"] = dsa.alloc_tree_outputs(names["layers"][0])
    names["ws"] = dsa.alloc_tree_workspace(names["layers"][0], None, dsa.Tree(n))
    for _ in range(2):
        before = seq.tolist()
        exec(code, names)
        torch.cuda.synchronize()
        stands = names["accepted"].tolist()
        assert names["status"].tolist() == [0] * b and names["forked"].tolist() == [0] and min(stands[:2]) >= 1 and stands[2] == 0
        assert seq.tolist() == [before[0] + stands[0], before[1] + stands[1], before[0] + stands[0]]     # (a branch of row 0)
        assert torch.isfinite(names["out"]).all() and names["next_token"].tolist()[2] == -1 and int(names["next_token"][:2].min()) >= 0
        dsa.dsa_release_pages(names["pool"], table, torch.where(torch.arange(b).cuda() == 2, 0, -1).int())
        seq[2] = -1
    assert dsa.dsa_wait_timeouts() == 0


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("last", ["compact", "release", "reserve", "fork"])
def test_promise_behind_calls_that_write_lengths_and_tables(dsa, last, captured):
    """Layers of decode steps behind each of the calls that write lengths or block tables: the first without
    DSA_PLAN_METADATA_STABLE, the others with it.  What comes out is what comes out without it."""
    b, h, d, page, m, layers, steps = 8, 8, 64, 16, 12, 3, 25
    rng = np.random.default_rng(3)
    g = torch.Generator().manual_seed(5)
    lens = rng.integers(10, (m - 1) * page, size=(steps, b))
    counts = [_int((x + (x % page == 0)).tolist()) for x in lens]  # (part-filled last pages: the step's token has a place in them)
    table0 = torch.from_numpy(rng.permutation(3 * b * m)[:b * m].reshape(b, m).astype(np.int32)).cuda()
    caches = torch.randn((2, layers, 3 * b * m, page, h, d), generator=g).bfloat16()
    q, kn, vn = (torch.randn((steps, layers, b, h, d), generator=g).bfloat16().cuda() for _ in range(3))
    diag = dsa.Diag(dsa.DSA_MASK_GRID, 24, 10, 6, 1)
    keep = torch.arange(m * page, dtype=torch.int32, device="cuda").expand(b, -1).contiguous()
    whole = _int([(m - 1) * page] * b)

    def run(flag):
        k, v = (caches[i].cuda() for i in range(2))
        table, seq, prompt, status = table0.clone(), whole.clone(), _int([9] * b), _int([0] * b)
        refs = torch.zeros((3 * b * m,), dtype=torch.int32, device="cuda")
        refs[table.long().flatten()] = 1
        pool, count = dsa.PagePool(refs, page), counts[0].clone()
        src, dst = _int([0, 1]), _int([b - 1, b - 2])
        ws, forked = dsa.alloc_fork_workspace(src), _int([9, 9])
        give_up = _int([-1] * (b - 2) + [0, 0])
        qs, ks, vs = (torch.empty_like(t[0]) for t in (q, kn, vn))
        probs = [dsa.Problem(q=qs[i], k_cache=k[i], v_cache=v[i], strides=k[i].stride()[:3], seq_len=seq, prompt_len=prompt, num_kv_heads=h,
                             max_seq_len=m * page, max_prompt_len=9, block_table=table, block_size=page, num_blocks=3 * b * m,
                             plan_flags=dsa.plan_group(4, 1) | (flag if i else 0)) for i in range(layers)]
        assert dsa.dsa_query_plan(probs[1], diag).block_warps == 4
        outs = [dsa.alloc_outputs(p) for p in probs]
        spaces = [dsa.alloc_workspace(p, diag) for p in probs]

        def one_pass():
            # every call writes what the layers read, `last` right in front of them
            dsa.dsa_compact_kv(probs[0], keep, whole if last == "reserve" else count, len_out=seq, num_layers=layers, stride_layer=k.stride(0))
            if last in ("release", "reserve"):
                dsa.dsa_release_pages(pool, table, count)
            if last == "reserve":
                dsa.dsa_compact_kv(probs[0], keep, count, len_out=seq, num_layers=layers, stride_layer=k.stride(0))
                dsa.dsa_reserve_pages(pool, table, seq, page, status)
            if last == "fork":
                dsa.dsa_release_pages(pool, table, give_up)
                dsa.dsa_fork_pages(pool, probs[0], src, dst, forked, ws, layers, k.stride(0))
            for p, (out, lse), space, i in zip(probs, outs, spaces, range(layers)):
                dsa.dsa_decode_step(p, diag, ks[i], vs[i], out, lse, space)

        got, graph = [], None
        for t in range(steps):
            for x, y in ((qs, q), (ks, kn), (vs, vn)):
                x.copy_(y[t])
            count.copy_(counts[t])
            if last == "release":                                  # (the pages that a pass gives back are taken again outside it)
                dsa.dsa_reserve_pages(pool, table, whole, 0, status)
            if captured and t == 1:
                dsa.dsa_prepare()
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    one_pass()
            if graph is not None:
                graph.replay()
            else:
                one_pass()
            got.append([(out.clone(), lse.clone()) for out, lse in outs] + [seq.clone(), table.clone()])
        torch.cuda.synchronize()
        return got

    for a, e in zip(run(dsa.DSA_PLAN_METADATA_STABLE), run(0)):
        for (o1, l1), (o2, l2) in zip(a[:layers], e[:layers]):
            assert torch.equal(o1, o2) and torch.equal(l1, l2)
        assert torch.equal(a[layers], e[layers]) and torch.equal(a[layers + 1], e[layers + 1])
        assert all(torch.isfinite(o).all() for o, _ in a[:layers])
    assert dsa.dsa_wait_timeouts() == 0


@pytest.mark.parametrize("spare", [2000, 700])
def test_fork_of_many_entry_by_entry(dsa, spare):
    """More branches than the planning block has threads: every table entry, count, length and byte of the cache; with too
    few pages the branches that get none change nothing, and those that need none are made all the same."""
    n, page, m = 1500, 4, 3
    rng = np.random.default_rng(spare)
    lens = [(i * 7) % 12 for i in range(n)] + [0] * n
    prompts = [min(x, 5) for x in lens]
    table = np.full((2 * n, m), -1, np.int32)
    ids, used = rng.permutation(n * m + spare), 0
    for i in range(n):
        need = -(-lens[i] // page)
        table[i, :need] = ids[used:used + need]
        used += need
    refs = np.ones(n * m + spare, np.int32)
    free = np.sort(rng.choice(ids[used:], size=spare, replace=False))
    refs[free] = 0
    c = Cache(dsa, 2 * n, m, page, blocks=n * m + spare, hkv=1, layers=2, table=table, lens=lens)
    c.prompt.copy_(_int(prompts))
    pool, status = dsa.PagePool(torch.from_numpy(refs).cuda(), page), _int([9] * n)
    src, dst = rng.integers(0, n, size=n).tolist(), (n + rng.permutation(n)).tolist()
    dsa.dsa_fork_pages(pool, c.problem, _int(src), _int(dst), status, dsa.alloc_fork_workspace(status), num_layers=2,
                       stride_layer=c.dev[0].stride(0))
    left, want = free.tolist(), []
    for s, d in zip(src, dst):
        full, part = divmod(lens[s], page)
        if part and not left:
            want.append(1)
            continue
        want.append(0)
        refs[table[s, :full]] += 1
        table[d, :full] = table[s, :full]
        if part:
            fresh = left.pop(0)
            table[d, full], refs[fresh] = fresh, 1
            for t in c.host:
                t[:, fresh, :part] = t[:, int(table[s, full]), :part]
        lens[d], prompts[d] = lens[s], prompts[s]
    assert want.count(1) == 0 if spare >= n else 0 < want.count(1) < n
    assert status.tolist() == want and np.array_equal(c.table.cpu().numpy(), table)
    assert pool.ref_count.tolist() == refs.tolist() and c.seq.tolist() == lens and c.prompt.tolist() == prompts and c.same()
