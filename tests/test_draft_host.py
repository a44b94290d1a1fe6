"""Host-only checks of the drafted-token calls: bad arguments are refused before a device is touched, and the
plain references of the GPU tests agree with hand-made values.  No compute call is made here."""
import ctypes
import math

import numpy as np
import pytest
import torch

from tests import draft_ref
from tests.test_abi_host import _diag, _problem

FAKE = 0x50000
INVALID, UNSUPPORTED, SMALL = -1, -2, -3


@pytest.fixture(scope="module")
def dsa():
    from paper_2609_19702_b200 import build
    build.build()
    from paper_2609_19702_b200 import binding
    return binding


def _tree(dsa, n=16, parent=FAKE, count=None):
    return dsa.dsa_tree(n, parent, count)


def _window(dsa, **kw):
    return _diag(dsa, mode=dsa.DSA_MASK_WINDOW, window=512, n_att=0, grid_w=0, **kw)


def _size(dsa, p, d, t):
    n = ctypes.c_size_t(0)
    rc = dsa._lib.dsa_tree_workspace_size(ctypes.addressof(p), ctypes.addressof(d) if d is not None else None,
                                          ctypes.addressof(t) if t is not None else None, ctypes.byref(n))
    return rc, n.value


def _step(dsa, p, d, t, k=FAKE, v=FAKE, out=FAKE, lse=FAKE, ws=None, n=0):
    return dsa._lib.dsa_tree_step(ctypes.addressof(p), ctypes.addressof(d) if d is not None else None,
                                  ctypes.addressof(t) if t is not None else None, k, v, out, lse, ws, n, None)


def test_tree_refusals(dsa):
    p, t = _problem(dsa), _tree(dsa)
    assert _size(dsa, p, None, t)[0] == 0
    assert _size(dsa, p, _window(dsa, n_sink=4), t)[0] == 0
    assert _size(dsa, p, None, None)[0] == INVALID
    assert _size(dsa, p, None, _tree(dsa, n=0))[0] == INVALID
    assert _size(dsa, p, None, _tree(dsa, n=65))[0] == UNSUPPORTED
    assert _size(dsa, p, None, _tree(dsa, n=64))[0] == 0
    assert _size(dsa, p, _diag(dsa), t)[0] == UNSUPPORTED                           # grid mask
    assert _size(dsa, p, _window(dsa, n_sink=-1), t)[0] == INVALID
    ring = _problem(dsa, ring_size=2048, ring_sinks=4)
    assert _size(dsa, ring, _window(dsa), t)[0] == UNSUPPORTED
    assert _size(dsa, _problem(dsa, head_dim=96), None, t)[0] == UNSUPPORTED
    assert _size(dsa, _problem(dsa, max_seq_len=2 ** 31 - 1), None, t)[0] == UNSUPPORTED
    assert _size(dsa, _problem(dsa, stride_token=100), None, t)[0] == INVALID
    for bad in (dict(k=None), dict(v=None), dict(out=None), dict(lse=None), dict(k=FAKE + 4), dict(v=FAKE + 8), dict(out=FAKE + 2)):
        assert _step(dsa, p, None, t, **bad) == INVALID
    assert _size(dsa, p, None, t)[1] == 0                                          # pieces of a request merge on chip
    p = _problem(dsa, split_tokens=256)
    rc, need = _size(dsa, p, None, t)
    assert need > 0
    assert _step(dsa, p, None, t) == INVALID                                       # no workspace
    assert _step(dsa, p, None, t, ws=FAKE + 16, n=need) == INVALID                 # misaligned
    assert _step(dsa, p, None, t, ws=0x60000, n=need - 1) == SMALL
    assert _step(dsa, _problem(dsa, batch=0), None, t) == 0


def test_tree_workspace_follows_split_tokens(dsa):
    t = _tree(dsa)
    sizes = [_size(dsa, _problem(dsa, split_tokens=s), None, t)[1] for s in (64, 100, 128, 8254)]
    assert sizes[0] > sizes[1] == sizes[2] > sizes[3] == 0
    parts = math.ceil(8254 / 64)
    assert sizes[0] >= 4 * 16 * 32 * parts * (128 + 1) * 4


def test_verify_refusals(dsa):
    def call(tree=True, **kw):
        v = dsa.dsa_verify(4, 1000, dsa.DSA_F32, FAKE, FAKE, 1000, FAKE, 1000, FAKE)
        outs = [kw.pop(k, FAKE) for k in ("path", "accepted", "next_token")]
        n = kw.pop("nodes", 8)
        for k, x in kw.items():
            setattr(v, k, x)
        t = dsa.dsa_tree(n, None, None)
        return dsa._lib.dsa_verify_tree(ctypes.addressof(v), ctypes.addressof(t) if tree else None, *outs, None)
    assert call(tree=False) == INVALID
    assert call(nodes=0) == INVALID and call(nodes=65) == UNSUPPORTED
    assert call(vocab=0) == INVALID and call(vocab=1001) == INVALID
    assert call(draft_stride=999) == INVALID and call(target_stride=999) == INVALID
    assert call(dtype=7) == UNSUPPORTED and call(batch=-1) == INVALID
    assert call(tokens=None) == INVALID and call(target_probs=None) == INVALID and call(target_probs=FAKE + 2) == INVALID
    assert call(uniforms=None) == INVALID                                          # draft probabilities without numbers
    for k in ("path", "accepted", "next_token"):
        assert call(**{k: None}) == INVALID
    assert call(batch=0) == 0


def test_page_refusals(dsa):
    L = dsa._lib
    pool = lambda **kw: dsa.dsa_page_pool(kw.get("num_blocks", 64), kw.get("block_size", 16), kw.get("ref_count", FAKE))  # noqa: E731
    a = ctypes.addressof
    paged = dict(block_table=FAKE, block_size=16, num_blocks=64, max_blocks=600)
    p = _problem(dsa, **paged)
    ok = pool()
    # compact
    assert L.dsa_compact_kv(a(p), 0, 0, None, FAKE, FAKE, 4, None, None) == INVALID        # no layer
    assert L.dsa_compact_kv(a(p), 2, 0, None, FAKE, FAKE, 4, None, None) == INVALID        # layers on top of each other
    assert L.dsa_compact_kv(a(p), 2, 1001, None, FAKE, FAKE, 4, None, None) == INVALID     # not a multiple of 16 bytes
    assert L.dsa_compact_kv(a(p), 1, 0, None, None, FAKE, 4, None, None) == INVALID
    assert L.dsa_compact_kv(a(p), 1, 0, None, FAKE, None, 4, None, None) == INVALID
    assert L.dsa_compact_kv(a(p), 1, 0, None, FAKE, FAKE, -1, None, None) == INVALID
    assert L.dsa_compact_kv(a(p), 1 << 17, 4096, None, FAKE, FAKE, 4, None, None) == UNSUPPORTED
    assert L.dsa_compact_kv(a(_problem(dsa, batch=64)), 1, 0, None, FAKE, FAKE, 2 ** 31 - 1, None, None) == UNSUPPORTED
    ring = _problem(dsa, ring_size=2048, **paged)
    assert L.dsa_compact_kv(a(ring), 1, 0, None, FAKE, FAKE, 4, None, None) == UNSUPPORTED
    # reserve, release
    assert L.dsa_reserve_pages(a(pool(num_blocks=0)), FAKE, 4, 8, FAKE, 1, FAKE, None) == INVALID
    assert L.dsa_reserve_pages(a(pool(ref_count=None)), FAKE, 4, 8, FAKE, 1, FAKE, None) == INVALID
    for args in ((None, 4, 8, FAKE, 1, FAKE), (FAKE, -1, 8, FAKE, 1, FAKE), (FAKE, 4, 0, FAKE, 1, FAKE), (FAKE, 4, 8, None, 1, FAKE),
                 (FAKE, 4, 8, FAKE, -1, FAKE), (FAKE, 4, 8, FAKE, 1, None)):
        assert L.dsa_reserve_pages(a(ok), *args, None) == INVALID
    assert L.dsa_reserve_pages(a(ok), FAKE, 5000, 8, FAKE, 1, FAKE, None) == UNSUPPORTED
    assert L.dsa_reserve_pages(a(ok), FAKE, 0, 8, FAKE, 1, FAKE, None) == 0
    assert L.dsa_release_pages(a(ok), None, 4, 8, None, None) == INVALID
    assert L.dsa_release_pages(a(pool(block_size=0)), FAKE, 4, 8, None, None) == INVALID
    # fork, copy
    def fork(prob=p, pl=ok, src=FAKE, dst=FAKE, n=4, st=FAKE, ws=0x60000, size=64):
        return L.dsa_fork_pages(a(pl), a(prob), 1, 0, src, dst, n, st, ws, size, None)
    assert fork(prob=_problem(dsa)) == INVALID                                     # not paged
    assert fork(pl=pool(num_blocks=63)) == INVALID and fork(pl=pool(block_size=8)) == INVALID
    assert fork(src=None) == INVALID and fork(dst=None) == INVALID and fork(st=None) == INVALID and fork(n=-1) == INVALID
    assert fork(ws=None) == INVALID and fork(ws=0x60010) == INVALID and fork(size=63) == SMALL
    assert fork(n=0) == 0
    assert L.dsa_copy_pages(a(_problem(dsa)), 1, 0, FAKE, FAKE, 4, None) == INVALID
    assert L.dsa_copy_pages(a(p), 1, 0, None, FAKE, 4, None) == INVALID
    assert L.dsa_copy_pages(a(p), 1, 0, FAKE, FAKE, 0, None) == 0


def test_binding_refuses_shapes(dsa):
    tok = torch.zeros((3, 5), dtype=torch.int32)
    probs = torch.zeros((3, 5, 16))
    assert dsa.Verify(tok, probs[..., :10], probs[..., 1:11], torch.zeros(3, 5)).c_struct().target_stride == 16
    with pytest.raises(ValueError):
        dsa.Verify(tok, probs[:, ::2]).c_struct()
    with pytest.raises(ValueError):
        dsa.Verify(tok, probs.transpose(1, 2)).c_struct()
    with pytest.raises(ValueError):
        dsa.Verify(tok, probs, probs.bfloat16(), torch.zeros(3, 5)).c_struct()
    with pytest.raises(ValueError):
        dsa.Verify(tok, probs, None, torch.zeros(3, 5, dtype=torch.float64)).c_struct()
    with pytest.raises(TypeError):
        dsa.Verify(tok, probs.double()).c_struct()
    with pytest.raises(ValueError):
        dsa.Tree(5, parent=torch.zeros((3, 4), dtype=torch.int32)).c_struct(3)
    with pytest.raises(ValueError):
        dsa.Tree(5, node_count=torch.zeros(3)).c_struct(3)
    with pytest.raises(ValueError):
        dsa.PagePool(torch.zeros(4, dtype=torch.int64), 16).c_struct()


def test_binding_refuses_host_tensors(dsa):
    """Nothing is handed to the library unless it lies on a CUDA device."""
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    v = dsa.Verify(i(2, 3), torch.zeros(2, 3, 8))
    with pytest.raises(ValueError):
        dsa.dsa_verify_tree(v, dsa.Tree(3), i(2, 3), i(2), i(2))
    pool = dsa.PagePool(i(8), 4)
    with pytest.raises(ValueError):
        dsa.dsa_reserve_pages(pool, i(2, 3), i(2), 1, i(2))
    with pytest.raises(ValueError):
        dsa.dsa_release_pages(pool, i(2, 3))


def test_references_by_hand():
    # a line of two over two cached tokens, one head: weights from logits (0, ln 3, ln 4)
    q = torch.zeros((2, 1, 2), dtype=torch.float64)
    q[:, 0, 0] = 1.0
    rows = torch.tensor([[[0.0, 0]], [[math.log(3), 0]]], dtype=torch.float64)
    new = torch.tensor([[[math.log(4), 0]], [[0.0, 0]]], dtype=torch.float64)
    vals = torch.tensor([[[1.0, 0]], [[2.0, 0]]], dtype=torch.float64)
    vnew = torch.tensor([[[4.0, 0]], [[8.0, 0]]], dtype=torch.float64)
    out, lse, _, _, count = draft_ref.tree_reference(q, rows, vals, new, vnew, [-1, 0], 2, 0, 2, 1.0)
    assert out[0, 0, 0].item() == pytest.approx((1 + 6 + 16) / 8) and lse[0, 0].item() == pytest.approx(math.log(8))
    assert out[1, 0, 0].item() == pytest.approx((1 + 6 + 16 + 8) / 9) and list(count) == [3, 4]
    out, _, _, _, count = draft_ref.tree_reference(q, rows, vals, new, vnew, [-1, -1], 2, 0, 2, 1.0, window=1)
    assert out[1, 0, 0].item() == 8 and list(count) == [1, 1]
    # rejection: p = (.5, .5), q = (1, 0): token 0 stands below 1/2, else the residual is all on 1
    p, dq = np.array([[0.5, 0.5], [0.25, 0.75]]), np.array([[1.0, 0.0], [0.5, 0.5]])
    assert draft_ref.verify_reference([0, 0], p, dq, [0.3, 0.4], [-1, 0], 2, "sample") == ([0, 1], 1)
    assert draft_ref.verify_reference([0, 0], p, dq, [0.3, 0.6], [-1, 0], 2, "sample") == ([0], 1)
    assert draft_ref.verify_reference([0, 1], p, None, [0.3, 0.6], [-1, 0], 2, "point") == ([0], 0)
    assert draft_ref.verify_reference([0, 1], p, None, None, [-1, 0], 2, "greedy") == ([0], 0)


def test_row_and_page_calls_take_a_trees_problem(dsa, monkeypatch):
    """The problem of a tree call, whose q has a row per node, describes the cache to the calls behind it as well."""
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    cache = torch.zeros((6, 16, 2, 64))
    monkeypatch.setattr(dsa.Problem, "_packed", lambda self, b, hq, d: (b, hq, d))

    def problem(*shape):
        return dsa.Problem(q=torch.zeros(shape), k_cache=cache, v_cache=cache, strides=(2048, 128, 64), seq_len=i(3), prompt_len=i(3),
                           num_kv_heads=2, max_seq_len=32, block_table=i(3, 2), block_size=16, num_blocks=6)
    assert dsa._cache_problem(problem(3, 5, 4, 64)) == dsa._cache_problem(problem(3, 4, 64)) == (3, 4, 64)
    for bad in ((3, 64), (2, 3, 5, 4, 64), (4, 5, 4, 64)):
        with pytest.raises(ValueError):
            dsa._cache_problem(problem(*bad))


def _small(dsa, q, cache, v=None, seq=None, prompt=None):
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    return dsa.Problem(q=q, k_cache=cache, v_cache=cache if v is None else v, strides=(2048, 128, 64), seq_len=i(3) if seq is None else seq,
                       prompt_len=i(3) if prompt is None else prompt, num_kv_heads=2, max_seq_len=32, block_table=i(3, 2), block_size=16,
                       num_blocks=6)


def _every_cache_call(dsa, problem):
    """The calls that take a problem's cache, each as a function."""
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    one, pool = i(1), dsa.PagePool(i(6), 16)
    n = 5
    q = torch.zeros((3, n, 4, 64), dtype=problem.q.dtype)
    tree = dsa.Problem(**{**problem.__dict__, "q": q})
    new = torch.zeros((3, n, 2, 64), dtype=q.dtype)
    yield lambda: dsa.dsa_tree_workspace_size(tree, None, dsa.Tree(n))
    yield lambda: dsa.dsa_tree_step(tree, None, dsa.Tree(n), new, new, torch.zeros_like(q), torch.zeros((3, n, 4)))
    yield lambda: dsa.dsa_compact_kv(problem, i(3, n), i(3))
    yield lambda: dsa.dsa_fork_pages(pool, problem, one, one, one, torch.zeros(16, dtype=torch.uint8))
    yield lambda: dsa.dsa_copy_pages(problem, one, one)


def test_binding_refuses_a_cache_of_another_type(dsa):
    """q's type says how wide the cache's elements are: with another one every address would be off."""
    bf, f32 = torch.zeros((6, 16, 2, 64), dtype=torch.bfloat16), torch.zeros((6, 16, 2, 64))
    for q, k, v in ((torch.float32, bf, bf), (torch.bfloat16, f32, f32), (torch.float32, f32, bf), (torch.bfloat16, f32, bf)):
        for call in _every_cache_call(dsa, _small(dsa, torch.zeros((3, 4, 64), dtype=q), k, v)):
            with pytest.raises(ValueError, match="type"):
                call()


def test_binding_refuses_strided_lengths(dsa):
    """Lengths that are a column of something, or one number for all requests, are not the array that the library reads."""
    cache = torch.zeros((6, 16, 2, 64))
    column, one = torch.zeros((3, 2), dtype=torch.int32)[:, 0], torch.zeros((1,), dtype=torch.int32).expand(3)
    for bad in (column, one):
        for kw in (dict(seq=bad), dict(prompt=bad)):
            for call in _every_cache_call(dsa, _small(dsa, torch.zeros((3, 4, 64)), cache, **kw)):
                with pytest.raises(ValueError, match="contiguous"):
                    call()


def test_sizes_beyond_the_index_arithmetic(dsa):
    """Refused before anything is launched."""
    L, a = dsa._lib, ctypes.addressof
    paged = dict(block_table=FAKE, block_size=16, num_blocks=64, max_blocks=600)
    p = _problem(dsa, batch=1, **paged)
    for keep in (2 ** 31 - 1, 2 ** 31 - 64, 2 ** 30 + 1):
        assert L.dsa_compact_kv(a(p), 1, 0, None, FAKE, FAKE, keep, None, None) == UNSUPPORTED
    # a fork whose copies would be more blocks than a launch has: the plan in front of them is not made either
    pool = dsa.dsa_page_pool(64, 16, FAKE)
    for n, layers in ((2 ** 30, 1), (2 ** 22, 2 ** 16), (2 ** 31 - 1, 1)):
        assert L.dsa_fork_pages(a(pool), a(p), layers, 4096, FAKE, FAKE, n, FAKE, 0x60000, 16 * n, None) == UNSUPPORTED
        assert L.dsa_copy_pages(a(p), layers, 4096, FAKE, FAKE, n, None) == UNSUPPORTED
