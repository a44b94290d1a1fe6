"""Host-only checks of the latent-cache calls: bad arguments are refused before a device is touched, and the plain
references of the GPU tests agree with hand-made values.  No compute call is made here."""
import ctypes
import math

import pytest
import torch

from tests import latent_ref

FAKE = 0x50000
INVALID, UNSUPPORTED, SMALL = -1, -2, -3


@pytest.fixture(scope="module")
def dsa():
    from paper_2609_19702_b200 import build
    build.build()
    from paper_2609_19702_b200 import binding
    return binding


def _latent(dsa, **kw):
    base = dict(batch=64, latent_dim=512, rope_dim=64, dtype=dsa.DSA_BF16, sm_scale=0.1, cache=FAKE, stride_batch=16 * 576, stride_token=576,
                seq_len=FAKE, block_table=FAKE, max_blocks=500, block_size=16, num_blocks=300, max_seq_len=8000)
    base.update(kw)
    x = dsa.dsa_latent()
    for k, v in base.items():
        setattr(x, k, v)
    return x


def _size(dsa, x, heads=16, new=1):
    n = ctypes.c_size_t(0)
    return dsa._lib.dsa_latent_workspace_size(ctypes.addressof(x) if x is not None else None, heads, new, ctypes.byref(n)), n.value


def _step(dsa, x, heads=16, new=1, q=FAKE, c=FAKE, out=FAKE, lse=FAKE, ws=0x60000, n=1 << 40):
    return dsa._lib.dsa_latent_step(ctypes.addressof(x), heads, new, q, c, None, out, lse, ws, n, None)


BAD_LATENTS = [(dict(batch=-1), INVALID), (dict(dtype=7), UNSUPPORTED), (dict(latent_dim=128), UNSUPPORTED), (dict(latent_dim=500), UNSUPPORTED),
               (dict(rope_dim=0), UNSUPPORTED), (dict(rope_dim=72), UNSUPPORTED), (dict(rope_dim=12), UNSUPPORTED), (dict(cache=None), INVALID),
               (dict(cache=FAKE + 8), INVALID), (dict(stride_token=568), INVALID), (dict(stride_token=580), INVALID), (dict(stride_batch=-8), INVALID),
               (dict(stride_batch=12), INVALID), (dict(max_seq_len=-1), INVALID), (dict(block_size=0), INVALID), (dict(num_blocks=0), INVALID),
               (dict(max_blocks=499), INVALID)]


def test_step_refusals(dsa):
    assert _size(dsa, _latent(dsa))[0] == 0
    assert _size(dsa, None)[0] == INVALID
    for kw, rc in BAD_LATENTS + [(dict(sm_scale=0.0), INVALID), (dict(sm_scale=-1.0), INVALID), (dict(sm_scale=math.inf), INVALID),
                                 (dict(sm_scale=math.nan), INVALID), (dict(seq_len=None), INVALID),
                                 (dict(block_table=None, max_seq_len=2 ** 31 - 1), UNSUPPORTED),
                                 (dict(block_table=None, max_seq_len=2 ** 24 + 2 ** 20, batch=1024), UNSUPPORTED)]:     # (a whole request for a block)
        assert _size(dsa, _latent(dsa, **kw))[0] == rc, kw
        assert _step(dsa, _latent(dsa, **kw)) == rc, kw
    assert _size(dsa, _latent(dsa, block_table=None, max_seq_len=2 ** 24 + 2 ** 20))[0] == 0           # (64 requests: cut into smaller pieces)
    x = _latent(dsa)
    for heads, new, rc in [(0, 1, INVALID), (1, 0, INVALID), (1025, 1, UNSUPPORTED), (1, 65, UNSUPPORTED), (1024, 64, 0)]:
        assert _size(dsa, x, heads, new)[0] == rc
    for bad in (dict(q=None), dict(c=None), dict(out=None), dict(lse=None), dict(q=FAKE + 8), dict(c=FAKE + 2), dict(out=FAKE + 4)):
        assert _step(dsa, x, **bad) == INVALID, bad
    need = _size(dsa, x)[1]
    assert need > 0
    assert _step(dsa, x, ws=None) == INVALID
    assert _step(dsa, x, ws=0x60000 + 128) == INVALID
    assert _step(dsa, x, n=need - 1) == SMALL
    assert _step(dsa, _latent(dsa, batch=0)) == 0


def _prompt(dsa, **kw):
    base = dict(batch=2, num_heads=4, nope_dim=128, value_dim=128, rope_dim=64, dtype=dsa.DSA_BF16, sm_scale=0.0, q_tokens=50, kv_tokens=60,
                max_q_len=30, q=FAKE, q_stride_token=4 * 192, q_stride_head=192, k_nope=FAKE, k_stride_token=1024, k_stride_head=256,
                k_rope=FAKE, rope_stride_token=64, v=FAKE, v_stride_token=1024, v_stride_head=256, q_start=FAKE, kv_start=FAKE, causal=1)
    base.update(kw)
    x = dsa.dsa_prompt()
    for k, v in base.items():
        setattr(x, k, v)
    return x


def test_prompt_refusals(dsa):
    call = lambda x, out=FAKE, lse=FAKE: dsa._lib.dsa_latent_prompt(ctypes.addressof(x), out, lse, None)  # noqa: E731
    for kw, rc in [(dict(batch=-1), INVALID), (dict(num_heads=0), INVALID), (dict(num_heads=1025), UNSUPPORTED), (dict(nope_dim=96), UNSUPPORTED),
                   (dict(value_dim=64), UNSUPPORTED), (dict(rope_dim=0), UNSUPPORTED), (dict(rope_dim=68), UNSUPPORTED), (dict(dtype=3), UNSUPPORTED),
                   (dict(sm_scale=-0.5), INVALID), (dict(sm_scale=math.nan), INVALID), (dict(q_tokens=-1), INVALID), (dict(kv_tokens=-1), INVALID),
                   (dict(max_q_len=-1), INVALID), (dict(q=None), INVALID), (dict(k_nope=None), INVALID), (dict(k_rope=None), INVALID),
                   (dict(v=None), INVALID), (dict(q_start=None), INVALID), (dict(q=FAKE + 8), INVALID), (dict(k_nope=FAKE + 2), INVALID),
                   (dict(k_rope=FAKE + 8), INVALID), (dict(v=FAKE + 4), INVALID), (dict(q_stride_token=100), INVALID), (dict(q_stride_token=184), INVALID),
                   (dict(k_stride_head=-8), INVALID), (dict(v_stride_head=4), INVALID), (dict(rope_stride_token=56), INVALID),
                   (dict(v_stride_token=0), INVALID), (dict(kv_tokens=2 ** 25 + 1), UNSUPPORTED)]:
        assert call(_prompt(dsa, **kw)) == rc, kw
    x = _prompt(dsa)
    assert call(x, out=None) == INVALID and call(x, lse=None) == INVALID and call(x, out=FAKE + 8) == INVALID
    for kw in (dict(batch=0), dict(q_tokens=0), dict(max_q_len=0)):
        assert call(_prompt(dsa, **kw)) == 0


def test_map_and_row_refusals(dsa):
    def run_map(start=FAKE, slot=FAKE, **kw):
        base = dict(batch=3, max_tokens=10, count=FAKE, base=None, block_table=FAKE, max_blocks=4, block_size=16, num_blocks=9, max_seq_len=64)
        base.update(kw)
        m = dsa.dsa_token_map()
        for k, v in base.items():
            setattr(m, k, v)
        return dsa._lib.dsa_map_tokens(ctypes.addressof(m), start, slot, None, None, None)

    for kw, rc in [(dict(batch=-1), INVALID), (dict(batch=8193), UNSUPPORTED), (dict(max_tokens=-1), INVALID), (dict(max_seq_len=-1), INVALID),
                   (dict(count=None), INVALID), (dict(start=None), INVALID), (dict(slot=None), INVALID), (dict(slot=FAKE + 4), INVALID),
                   (dict(block_size=0), INVALID), (dict(max_blocks=0), INVALID), (dict(num_blocks=0), INVALID), (dict(max_tokens=2 ** 31 - 1), UNSUPPORTED)]:
        assert run_map(**kw) == rc, kw
    for fn in (dsa._lib.dsa_store_rows, dsa._lib.dsa_gather_rows):
        x = _latent(dsa)
        row = lambda y=x, slot=FAKE, n=5, rows=FAKE, ld=576: fn(ctypes.addressof(y), slot, n, rows, ld, None)  # noqa: E731
        for kw, rc in BAD_LATENTS:
            assert row(_latent(dsa, **kw)) == rc, kw
        assert row(slot=None) == INVALID and row(slot=FAKE + 4) == INVALID and row(rows=None) == INVALID and row(rows=FAKE + 8) == INVALID
        assert row(n=-1) == INVALID and row(ld=568) == INVALID and row(ld=580) == INVALID
        assert row(n=0) == 0 and row(_latent(dsa, batch=0)) == 0
        assert fn(None, FAKE, 1, FAKE, 576, None) == INVALID


def test_binding_refuses(dsa):
    """What only the binding can see: shapes, types, layouts, devices."""
    seq = torch.zeros((2,), dtype=torch.int32)
    cache = torch.zeros((2, 8, 576), dtype=torch.bfloat16)
    lat = dsa.Latent(cache, strides=(8 * 576, 576), seq_len=seq, latent_dim=512, rope_dim=64, max_seq_len=8, sm_scale=0.1)
    q, c = torch.zeros((2, 1, 4, 576), dtype=torch.bfloat16), torch.zeros((2, 1, 576), dtype=torch.bfloat16)
    out, lse = dsa.alloc_latent_outputs(lat, q)
    assert out.shape == (2, 1, 4, 512) and lse.shape == (2, 1, 4)
    for bad in (dict(q=q[:1]), dict(q=q[..., :512]), dict(q=q.float()), dict(q=q.transpose(1, 2)), dict(c_new=c[:, 0]), dict(c_new=c.float()),
                dict(out=out[..., :256]), dict(out=out.float()), dict(lse=lse.double()), dict(lse=lse[0]), dict(new_count=seq[:1]),
                dict(new_count=seq.long())):
        with pytest.raises(ValueError):
            dsa.dsa_latent_step(**{**dict(latent=lat, q=q, c_new=c, out=out, lse=lse), **bad})
    with pytest.raises(ValueError, match="CUDA"):
        dsa.dsa_latent_step(lat, q, c, out, lse)
    lat.seq_len = seq.long()
    with pytest.raises(ValueError):
        dsa.dsa_latent_step(lat, q, c, out, lse)
    lat.seq_len = seq
    lat.block_table = torch.zeros((3, 4), dtype=torch.int32)
    with pytest.raises(ValueError):
        dsa.dsa_latent_step(lat, q, c, out, lse)

    k = torch.zeros((6, 4, 256), dtype=torch.bfloat16)
    pq, kr, qs = torch.zeros((5, 4, 192), dtype=torch.bfloat16), torch.zeros((6, 64), dtype=torch.bfloat16), torch.zeros((3,), dtype=torch.int32)
    good = dict(q=pq, k_nope=k[..., :128], k_rope=kr, v=k[..., 128:], q_start=qs)
    p = dsa.Prompt(**good)
    po, pl = dsa.alloc_prompt_outputs(p)
    assert p.c_struct().nope_dim == 128 and p.c_struct().kv_tokens == 6 and p.c_struct().max_q_len == 5
    for bad in (dict(q=pq[0]), dict(q=pq.float()), dict(k_nope=k[:5, :, :128]), dict(k_nope=k), dict(v=k[:, :2, 128:]), dict(k_rope=kr.float()),
                dict(q_start=qs.long()), dict(kv_start=qs[:2]), dict(k_rope=kr.t().contiguous().t()), dict(v=k.transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises(ValueError):
            dsa.dsa_latent_prompt(dsa.Prompt(**{**good, **bad}), po, pl)
    for o, x in ((po[:4], pl), (po.float(), pl), (po, pl.double()), (po, pl[:, :2])):
        with pytest.raises(ValueError):
            dsa.dsa_latent_prompt(p, o, x)

    i32 = lambda n: torch.zeros((n,), dtype=torch.int32)  # noqa: E731
    slot = torch.zeros((5,), dtype=torch.int64)
    for args in (dict(start=i32(2)), dict(slot=i32(5)), dict(position=i32(4)), dict(request=slot), dict(base=i32(3)), dict(block_table=torch.zeros((3, 4), dtype=torch.int32)),
                 dict(count=torch.zeros((2,), dtype=torch.int64))):
        with pytest.raises(ValueError):
            dsa.dsa_map_tokens(**{**dict(count=i32(2), start=i32(3), slot=slot), **args})
    lat = dsa.Latent(cache, strides=(8 * 576, 576), seq_len=seq, latent_dim=512, rope_dim=64, max_seq_len=8, sm_scale=0.1)
    rows = torch.zeros((5, 576), dtype=torch.bfloat16)
    for s, r in ((slot[:4], rows), (slot.int(), rows), (slot, rows.float()), (slot, rows[:, :570]), (slot, rows[0]), (slot, rows.t().contiguous().t())):
        for fn in (dsa.dsa_store_rows, dsa.dsa_gather_rows):
            with pytest.raises(ValueError):
                fn(lat, s, r)


def test_references_by_hand():
    q = torch.tensor([[[1.0, 0.0]]]).double()
    k = torch.tensor([[[math.log(3.0), 9.0]], [[0.0, -9.0]], [[100.0, 0.0]]]).double()
    out, lse, weight, size, count = latent_ref.attend(q, k, torch.tensor([[[1.0]], [[5.0]], [[7.0]]]).double(), [2], 1.0)
    assert out.item() == pytest.approx(0.75 * 1 + 0.25 * 5) and lse.item() == pytest.approx(math.log(4.0)) and count.item() == 2
    out, lse, tol, _ = latent_ref.prompt_expected(q.expand(2, 1, 2), k[:1, :, :1], k[:1, 0, 1:], torch.ones((1, 1, 1)).double(), True, 1.0, True)
    assert out.flatten().tolist() == [0.0, 1.0] and lse[0, 0] == -math.inf and tol[0].item() == 0.0
    out, lse, _, _ = latent_ref.step_expected(torch.ones((2, 1, 2)).double(), torch.zeros((0, 2)).double(), torch.ones((2, 2)).double(), 1, 1, 1.0, False)
    assert out.flatten().tolist() == [1.0, 0.0] and lse[0, 0].item() == pytest.approx(2.0) and lse[1, 0] == -math.inf
    assert latent_ref.map_expected([2, 0, 3], [1, 5, 0], [[0, 1], [2, 3], [4, -1]], 2, 9, 4, 6) == (
        [0, 2, 2, 5], [1, 2, 8, 9, -1, -1], [1, 2, 0, 1, 2, -1], [0, 0, 2, 2, 2, -1])


def test_size_of_the_workspace(dsa):
    """Follows the batch's shape, never the device's arrays; float32 needs parts only where keys are cut."""
    a, b = _size(dsa, _latent(dsa), 16, 1)[1], _size(dsa, _latent(dsa, max_seq_len=8), 16, 1)[1]
    assert a > 0 and a >= b
    f = lambda **kw: _size(dsa, _latent(dsa, dtype=dsa.DSA_F32, **kw), 16, 1)[1]  # noqa: E731
    assert f() > 0 and f(max_seq_len=8) == 0
