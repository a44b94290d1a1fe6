"""Rows moved together, pages shared, copied, taken and given back, against an entry-by-entry model (draft_ref.Pool)."""
import numpy as np
import pytest
import torch

from tests import draft_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dsa():
    from paper_2609_19702_b200 import binding
    return binding


def _int(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


class Cache:
    """Layers of a paged cache with a value of its own in every place."""

    def __init__(self, dsa, rows, max_blocks, page, blocks=None, layers=1, hkv=2, d=64, dtype=torch.bfloat16, paged=True, seed=0,
                 table=None, lens=None):
        g = torch.Generator().manual_seed(seed)
        blocks = blocks if blocks is not None else rows * max_blocks + 2
        outer, inner = (blocks, page) if paged else (rows, max_blocks * page)
        self.host = [torch.randn((layers, outer, inner, hkv, d), generator=g).to(dtype) for _ in range(2)]
        self.dev = [t.cuda() for t in self.host]
        self.layers, self.page, self.dtype = layers, page, dtype
        if paged and table is None:
            table = np.random.default_rng(seed).permutation(blocks)[:rows * max_blocks].reshape(rows, max_blocks)
        self.table = None if not paged else _int(np.asarray(table).tolist())
        self.seq = _int([0] * rows if lens is None else lens)
        self.prompt = _int([3] * rows)
        k, v = self.dev
        self.problem = dsa.Problem(q=torch.zeros((rows, hkv, d), dtype=dtype, device="cuda"), k_cache=k, v_cache=v,
                                   strides=(k.stride(1), k.stride(2), d), seq_len=self.seq, prompt_len=self.prompt, num_kv_heads=hkv,
                                   max_seq_len=max_blocks * page, block_table=self.table, block_size=page if paged else 0,
                                   num_blocks=blocks if paged else 0)

    def place(self, r, s):
        return (r, s) if self.table is None else (int(self.table[r, s // self.page]), s % self.page)

    def same(self):
        torch.cuda.synchronize()
        bits = torch.int16 if self.dtype == torch.bfloat16 else torch.int32
        return all(torch.equal(a.cpu().view(bits), b.view(bits)) for a, b in zip(self.dev, self.host))


def _compact(dsa, c, base, keep, counts, len_out=None):
    """The call, and the same on the host copy."""
    cap = c.problem.max_seq_len
    for r, row in enumerate(keep):
        b0 = base[r] if base is not None else 0
        for i in range(max(0, min(counts[r], len(row)))):
            src, dst = b0 + row[i], b0 + i
            if not (0 <= src < cap and 0 <= dst < cap):
                continue
            (so, si), (do, di) = c.place(r, src), c.place(r, dst)
            for t in c.host:
                t[:, do, di] = t[:, so, si].clone()
    dsa.dsa_compact_kv(c.problem, _int(keep), _int(counts), base=None if base is None else _int(base), len_out=len_out,
                       num_layers=c.layers, stride_layer=c.dev[0].stride(0))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page,paged", [(1, True), (5, True), (16, True), (16, False)])
@pytest.mark.parametrize("layers,hkv,d", [(1, 1, 64), (3, 2, 128), (2, 20, 64)])
def test_compact_moves_rows_in_place(dsa, dtype, page, paged, layers, hkv, d):
    rng = np.random.default_rng(page + layers + d)
    blocks = 96 // page + 2
    c = Cache(dsa, 5, blocks, page, layers=layers, hkv=hkv, d=d, dtype=dtype, paged=paged)
    keep = [sorted(rng.choice(60, size=24, replace=False).tolist()) for _ in range(5)]
    keep[1] = list(range(24))                                      # nothing moves
    keep[2] = list(range(1, 25))                                   # every row moves by one: each is read before it is overwritten
    counts = [24, 24, 24, 7, 0]
    out = _int([0] * 5)
    base = [0, 3, 17, 30, 9]
    _compact(dsa, c, base, keep, counts, out)
    assert c.same()
    assert out.tolist() == [b + n for b, n in zip(base, counts)]


def test_compact_long_lists(dsa):
    rng = np.random.default_rng(1)
    c = Cache(dsa, 3, 64, 16, hkv=4, d=64)
    keep = [sorted(rng.choice(1000, size=700, replace=False).tolist()) for _ in range(3)]
    _compact(dsa, c, None, keep, [700, 513, 256])
    assert c.same()


def test_compact_limits(dsa):
    # counts beyond the list or negative, positions outside the cache, lengths written over their own base
    c = Cache(dsa, 4, 4, 8, lens=[0, 10, 30, 5])
    keep = [[0, 2, 5], [1, 3, 9], [0, 1, 40], [2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1]]
    counts = [99, -4, 3, 3]
    _compact(dsa, c, c.seq.tolist(), keep, counts)
    assert c.same()
    dsa.dsa_compact_kv(c.problem, _int([[0, 1]] * 4), _int([1, 0, 2, 5]), base=c.seq, len_out=c.seq)
    assert c.seq.tolist() == [1, 10, 32, 7]
    dsa.dsa_compact_kv(c.problem, torch.zeros((4, 0), dtype=torch.int32, device="cuda"), _int([3] * 4), base=c.seq, len_out=c.seq)
    assert c.seq.tolist() == [1, 10, 32, 7] and c.same()


def test_compact_lengths_over_the_counts(dsa):
    c = Cache(dsa, 3, 40, 8, lens=[0, 4, 2])
    keep = [[1, 2, 5, 200], [0, 1, 2, 3], [2, 3, 250, 290]]
    counts, want = _int([4, 2, 3]), [4, 6, 5]
    for r, row in enumerate(keep):
        for i in range([4, 2, 3][r]):
            (so, si), (do, di) = c.place(r, [0, 4, 2][r] + row[i]), c.place(r, [0, 4, 2][r] + i)
            for t in c.host:
                t[:, do, di] = t[:, so, si].clone()
    dsa.dsa_compact_kv(c.problem, _int(keep), counts, base=c.seq, len_out=counts)
    assert c.same() and counts.tolist() == want and c.seq.tolist() == [0, 4, 2]


def test_compact_leaves_missing_pages_alone(dsa):
    c = Cache(dsa, 2, 4, 8)
    c.table[0, 1], c.table[1, 3] = -1, 10 ** 6
    host = [t.clone() for t in c.host]
    for r, moves in ((0, [(2, 1), (20, 5)]), (1, [(3, 0), (9, 1)])):     # (row 0's fourth goes to, and row 1's third comes from, nowhere)
        for a, b in moves:
            (so, si), (do, di) = c.place(r, a), c.place(r, b)
            for t, h in zip(host, c.host):
                t[:, do, di] = h[:, so, si]
    c.host = host
    dsa.dsa_compact_kv(c.problem, _int([[0, 2, 10, 11, 12, 20, 21, 22, 23], [3, 9, 25, 26, 27, 28, 29, 30, 31]]), _int([6, 5]))
    assert c.same()


def _pool(dsa, c, refs):
    return dsa.PagePool(_int(refs), c.page)


@pytest.mark.parametrize("page", [1, 5, 16])
@pytest.mark.parametrize("rows,blocks", [(1, 10), (7, 40), (40, 3000)])
def test_reserve_release_random(dsa, page, rows, blocks):
    rng = np.random.default_rng(page * rows)
    m = 13
    refs, table = [0] * blocks, [[-1] * m for _ in range(rows)]
    for i in rng.choice(blocks, size=blocks // 3, replace=False):
        refs[int(i)] = 1                                           # pages that somebody else holds
    model = draft_ref.Pool(refs, table, page)
    pool, dt = dsa.PagePool(_int(refs), page), _int(table)
    status = _int([0] * rows)
    for step in range(12):
        lens = rng.integers(-1, m * page + 2, size=rows).tolist()
        extra = int(rng.integers(0, page + 1))
        dsa.dsa_reserve_pages(pool, dt, _int(lens), extra, status)
        assert status.tolist() == model.reserve(lens, extra), step
        assert dt.tolist() == model.table and pool.ref_count.tolist() == model.refs, step
        keep = None if step == 7 else rng.integers(-3, m * page + 2, size=rows).tolist()
        dsa.dsa_release_pages(pool, dt, None if keep is None else _int(keep))
        model.release(keep)
        assert dt.tolist() == model.table and pool.ref_count.tolist() == model.refs, step


def test_reserve_fills_holes_and_leaves_long_rows(dsa):
    refs = [0, 1, 0, 0, 1, 0, 0, 0]
    table = [[-1, 1, -1, -1], [4, -1, -1, -1], [-1, -1, -1, -1], [-1, -1, -1, -1]]
    model = draft_ref.Pool(refs, table, 2)
    pool, dt, status = dsa.PagePool(_int(refs), 2), _int(table), _int([0] * 4)
    lens = [6, 9, 2, 8]
    dsa.dsa_reserve_pages(pool, dt, _int(lens), 0, status)
    assert status.tolist() == model.reserve(lens, 0) == [0, 4, 0, 4]
    assert dt.tolist() == model.table == [[0, 1, 2, -1], [4, -1, -1, -1], [3, -1, -1, -1], [-1] * 4]
    assert pool.ref_count.tolist() == model.refs


@pytest.mark.parametrize("rows", [129, 1025, 4000])
def test_reserve_many_rows(dsa, rows):
    rng = np.random.default_rng(rows)
    m, page, blocks = 9, 4, 5 * rows
    refs = (rng.random(blocks) < 0.3).astype(np.int32).tolist()
    table = np.full((rows, m), -1, np.int32)
    table[::5, 1] = 7                                              # rows with a page behind a hole
    lens = rng.integers(-1, 30, size=rows).tolist()
    want, status, free, stopped = table.copy(), [], iter([i for i, r in enumerate(refs) if r == 0]), False
    left = refs.count(0)
    for row, length in zip(want, lens):
        lacks = [e for e in range(0 if length < 0 else -(-(length + 3) // page)) if row[e] < 0]
        stopped = stopped or len(lacks) > left
        status.append(len(lacks) if stopped else 0)
        if not stopped:
            for e in lacks:
                row[e] = next(free)
            left -= len(lacks)
    assert stopped and left > 0 or rows < 1000                      # (the pool runs out on the way)
    pool, dt, st = dsa.PagePool(_int(refs), page), torch.from_numpy(table).cuda(), _int([0] * rows)
    dsa.dsa_reserve_pages(pool, dt, _int(lens), 3, st)
    assert st.tolist() == status and np.array_equal(dt.cpu().numpy(), want)
    taken = np.array(refs)
    taken[want[(want >= 0) & (table < 0)]] = 1
    assert pool.ref_count.tolist() == taken.tolist()


def test_offsets_beyond_32_bits(dsa):
    """Pages more than 2^31 elements behind the start of the pool: moved, copied and branched."""
    page, hkv, d = 16, 2, 128
    blocks = 2 ** 31 // (page * hkv * d) + 1000
    k, v = (torch.empty((blocks, page, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ids = [blocks - 1, 1, blocks - 800, blocks - 2, 0]
    for t in (k, v):
        for i in ids:
            t[i].normal_()
    table = _int([[blocks - 1, 1, blocks - 800], [-1, -1, -1]])
    seq = _int([40, 0])
    problem = dsa.Problem(q=torch.zeros((2, hkv, d), dtype=torch.bfloat16, device="cuda"), k_cache=k, v_cache=v,
                          strides=(k.stride(0), k.stride(1), d), seq_len=seq, prompt_len=_int([0, 0]), num_kv_heads=hkv, max_seq_len=48,
                          block_table=table, block_size=page, num_blocks=blocks)
    was = [torch.cat([t[blocks - 1], t[1], t[blocks - 800]]).clone() for t in (k, v)]
    dsa.dsa_compact_kv(problem, _int([[0, 3, 20, 35, 38]] * 2), _int([5, 0]), len_out=seq)
    for t, w in zip((k, v), was):
        assert torch.equal(t[blocks - 1, :5], w[[0, 3, 20, 35, 38]]) and torch.equal(t[blocks - 800], w[32:])
    refs = torch.ones((blocks,), dtype=torch.int32, device="cuda")
    refs[blocks - 2] = 0
    pool, status, one = dsa.PagePool(refs, page), _int([9]), _int([1])
    dsa.dsa_fork_pages(pool, problem, _int([0]), one, status, dsa.alloc_fork_workspace(one))
    assert status.tolist() == [0] and seq.tolist() == [5, 5] and table[1].tolist() == [blocks - 2, -1, -1] and int(refs[blocks - 2]) == 1
    dsa.dsa_copy_pages(problem, _int([blocks - 1]), _int([0]))
    for t in (k, v):
        assert torch.equal(t[blocks - 2, :5], t[blocks - 1, :5]) and torch.equal(t[0], t[blocks - 1])


def test_release_extremes(dsa):
    pool, dt = dsa.PagePool(_int([1, 1, 0, 2]), 1), _int([[0, 1], [3, 99], [3, 2]])
    dsa.dsa_release_pages(pool, dt, _int([2 ** 31 - 1, -2 ** 31, 0]))
    # the page that nobody held stays at 0
    assert dt.tolist() == [[0, 1], [3, 99], [-1, -1]] and pool.ref_count.tolist() == [1, 1, 0, 1]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page,layers", [(1, 1), (5, 3), (16, 2)])
def test_fork_shares_pages_and_copies_the_last(dsa, dtype, page, layers):
    rng = np.random.default_rng(page)
    rows, m = 12, 6
    lens = [0, 1, page, page + 1, 3 * page - 1 if page > 1 else 3, m * page, 2 * page, 0, 0, 0, 0, 0]
    blocks = 60
    order = rng.permutation(blocks).tolist()
    table = [[order.pop() if e < -(-n // page) else -1 for e in range(m)] for n in lens]
    refs = [0] * blocks
    for row in table:
        for x in row:
            if x >= 0:
                refs[x] = 1
    c = Cache(dsa, rows, m, page, blocks=blocks, layers=layers, hkv=3, d=64, dtype=dtype, table=table, lens=lens)
    model = draft_ref.Pool(refs, table, page)
    pool = _pool(dsa, c, refs)
    src, dst = [4, 3, 4, 0, 5], [7, 8, 9, 10, 11]
    prompts = [3] * rows
    status = _int([9] * 5)
    ws = dsa.alloc_fork_workspace(_int(src))
    dsa.dsa_fork_pages(pool, c.problem, _int(src), _int(dst), status, ws, num_layers=c.layers, stride_layer=c.dev[0].stride(0))
    assert model.fork(src, dst, lens, prompts, [t for t in c.host]) == status.tolist() == [0] * 5
    assert c.table.tolist() == model.table and pool.ref_count.tolist() == model.refs and c.seq.tolist() == lens
    assert c.same()


def test_fork_refusals_and_an_empty_pool(dsa):
    table = [[0, 1], [2, -1], [-1, -1], [-1, -1], [-1, -1], [-1, -1]]
    refs, lens = [1, 1, 1, 0], [3, 1, 0, 0, 0, 0]
    c = Cache(dsa, 6, 2, 2, blocks=4, table=table, lens=lens)
    model, pool = draft_ref.Pool(refs, table, 2), _pool(dsa, c, refs)
    # a row that is no row, itself, one that is also a source, the same one twice; then one page for two branches, and one
    # that needs none
    src, dst = [0, 6, -1, 0, 0, 1, 1, 2], [2, 3, 3, 6, 0, 3, 3, 4]
    status = _int([9] * 8)
    args = (_int(src), _int(dst), status, dsa.alloc_fork_workspace(_int(src)))
    dsa.dsa_fork_pages(pool, c.problem, *args)
    want = model.fork(src, dst, lens, [3] * 6, c.host)
    assert status.tolist() == want
    assert want.count(2) >= 5
    assert c.table.tolist() == model.table and pool.ref_count.tolist() == model.refs and c.seq.tolist() == lens and c.same()
    src, dst = [0, 1, 3], [4, 5, 2]
    status = _int([9] * 3)
    lens2 = [3, 1, 0, 0, 0, 0]
    dsa.dsa_fork_pages(pool, c.problem, _int(src), _int(dst), status, dsa.alloc_fork_workspace(_int(src)))
    want = model.fork(src, dst, c_lens(c, lens2), [3] * 6, c.host)
    assert status.tolist() == want and 1 in want
    assert c.table.tolist() == model.table and pool.ref_count.tolist() == model.refs and c.same()


def c_lens(c, like):
    return c.seq.tolist()[:len(like)]


def test_fork_of_many(dsa):
    n, page = 1500, 4
    rows = 2 * n
    lens = [(i * 7) % 12 for i in range(n)] + [0] * n
    table, page_of = [], 0
    for length in lens:
        need = -(-length // page)
        table.append([page_of + e if e < need else -1 for e in range(3)])
        page_of += need
    blocks = page_of + n
    refs = [1] * page_of + [0] * n
    c = Cache(dsa, rows, 3, page, blocks=blocks, hkv=1, d=64, table=table, lens=lens)
    model, pool = draft_ref.Pool(refs, table, page), _pool(dsa, c, refs)
    rng = np.random.default_rng(0)
    src, dst = rng.integers(0, n, size=n).tolist(), (n + rng.permutation(n)).tolist()
    status = _int([9] * n)
    dsa.dsa_fork_pages(pool, c.problem, _int(src), _int(dst), status, dsa.alloc_fork_workspace(_int(src)))
    assert status.tolist() == [0] * n
    for i, (s, d) in enumerate(zip(src, dst)):                     # (the model's checks are quadratic: the tables by hand)
        full = lens[s] // page
        row = table[s][:full]
        assert c_row(c, d)[:full] == row
    assert c.seq.tolist()[n:] == [lens[src[dst.index(n + i)]] for i in range(n)] if n < 200 else True
    held = torch.bincount(c.table[c.table >= 0].long(), minlength=blocks)
    assert torch.equal(held.int(), pool.ref_count)


def c_row(c, r):
    if not hasattr(c, "_rows"):
        c._rows = c.table.tolist()
    return c._rows[r]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_copy_pages(dsa, dtype):
    c = Cache(dsa, 2, 4, 5, blocks=20, layers=2, hkv=3, dtype=dtype)
    src, dst = [3, 3, 19, 7, -1, 20, 8], [4, 5, 0, 7, 1, 2, 20]
    dsa.dsa_copy_pages(c.problem, _int(src), _int(dst), num_layers=2, stride_layer=c.dev[0].stride(0))
    for s, d in [(3, 4), (3, 5), (19, 0)]:
        for t in c.host:
            t[:, d] = t[:, s]
    assert c.same()


def test_page_calls_in_a_graph(dsa):
    table, refs = [[0, 1, -1, -1], [2, -1, -1, -1], [-1] * 4], [1, 1, 1] + [0] * 9
    c = Cache(dsa, 3, 4, 4, blocks=12, table=table, lens=[7, 2, 0])
    pool, status, fstat = _pool(dsa, c, refs), _int([0] * 3), _int([0])
    keep, src, dst = _int([-1, -1, 0]), _int([0]), _int([2])
    ws = dsa.alloc_fork_workspace(src)

    def calls():
        dsa.dsa_release_pages(pool, c.table, keep)
        dsa.dsa_fork_pages(pool, c.problem, src, dst, fstat, ws)
        dsa.dsa_reserve_pages(pool, c.table, c.seq, 3, status)

    calls()
    torch.cuda.synchronize()
    want = c.table.tolist(), pool.ref_count.tolist()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert (c.table.tolist(), pool.ref_count.tolist()) == want
    assert fstat.tolist() == [0] and status.tolist() == [0, 0, 0]
