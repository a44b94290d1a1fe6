"""Prompt attention with keys and values expanded per head (dsa_latent_prompt) against a float64 reference."""
import math

import pytest
import torch

from tests import latent_ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def dsa():
    from paper_2609_19702_b200 import binding
    return binding


def run_case(dsa, dtype, heads, d, rope, q_lens, kv_lens=None, causal=True, joint=True, behind=3, max_q=0, seed=0, scale=0.0, change=None):
    g = torch.Generator().manual_seed(seed)
    dt = DT[dtype]
    k_lens = kv_lens if kv_lens is not None else q_lens
    nq, nk = sum(q_lens), sum(k_lens)
    rand = lambda *s: torch.randn(s, generator=g).to(dt)  # noqa: E731
    q = rand(nq + behind, heads, d + rope)
    kv, kr = rand(nk + behind, heads, 2 * d), rand(nk + behind, rope)
    if change:
        change(q, kv, kr)
    kv[nk:], kr[nk:] = math.nan, math.nan                    # nobody's rows
    if kv_lens is None:
        q[nq:] = math.nan
    qs = torch.tensor([0] + list(torch.tensor(q_lens).cumsum(0))).int()
    ks = torch.tensor([0] + list(torch.tensor(k_lens).cumsum(0))).int()
    dkv, dkr, dq = kv.cuda(), kr.cuda(), q.cuda()
    kn, v = (dkv[..., :d], dkv[..., d:]) if joint else (dkv[..., :d].contiguous(), dkv[..., d:].contiguous())
    p = dsa.Prompt(dq, kn, dkr, v, qs.cuda(), None if kv_lens is None else ks.cuda(), max_q_len=max_q or max(q_lens + [1]), sm_scale=scale, causal=causal)
    out, lse = dsa.alloc_prompt_outputs(p)
    out.fill_(7.0), lse.fill_(7.0)
    dsa.dsa_latent_prompt(p, out, lse)
    torch.cuda.synchronize()
    assert dsa.dsa_wait_timeouts() == 0
    at, bt = 0, 0
    used = scale or 1.0 / math.sqrt(d + rope)
    for r, (a, b) in enumerate(zip(q_lens, k_lens)):
        if a:
            k = kv[bt:bt + b].double()
            o, l, tol, ltol = latent_ref.prompt_expected(q[at:at + a].double(), k[..., :d], kr[bt:bt + b].double(), k[..., d:], causal, used, dtype == "bf16")
            top = min(a, max_q or a)
            latent_ref.assert_near(out[at:at + top], o[:top], tol[:top], "out of request %d" % r)
            latent_ref.assert_near(lse[at:at + top], l[:top], ltol[:top], "lse of request %d" % r)
            assert (out[at + top:at + a] == 7.0).all() and (lse[at + top:at + a] == 7.0).all()
        at, bt = at + a, bt + b
    assert (out[nq:] == 7.0).all() and (lse[nq:] == 7.0).all(), "rows behind the last sequence"
    return out, lse


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rope", [(128, 64), (64, 32), (128, 16), (64, 8)])
@pytest.mark.parametrize("q_lens,kv_lens", [
    ([1], None), ([5, 1, 0, 130], None), ([128, 127, 129], None), ([256, 255, 257], None),
    ([1, 1, 1], [1, 300, 0]),                                # single tokens, one of them without any key
    ([10, 200, 3], [10, 333, 129]),                          # behind a cached prefix
    ([20, 140], [7, 13]),                                    # fewer keys than queries: the first ones see nothing
])
def test_prompt(dsa, dtype, d, rope, q_lens, kv_lens):
    run_case(dsa, dtype, 3, d, rope, q_lens, kv_lens)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_lens,kv_lens", [([130, 1, 300], None), ([3, 260], [129, 64]), ([2, 5], [0, 1])])
def test_all_keys(dsa, dtype, q_lens, kv_lens):
    run_case(dsa, dtype, 2, 128, 64, q_lens, kv_lens, causal=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_scale_and_bound(dsa, dtype):
    run_case(dsa, dtype, 2, 128, 64, [70, 200], joint=False)
    run_case(dsa, dtype, 2, 128, 64, [70, 200], scale=0.3)
    run_case(dsa, dtype, 2, 128, 64, [70, 300], max_q=100)   # queries beyond the bound are left out, the others see what they saw
    run_case(dsa, dtype, 1, 128, 64, [33], [400], max_q=33)


@pytest.mark.parametrize("dtype,heads,q_lens,kv_lens", [("bf16", 2, [1500], None), ("bf16", 1, [700, 1200], [2500, 1200]), ("f32", 1, [600], None),
                                                       ("bf16", 1, [3] * 200, None)])
def test_long_and_many(dsa, dtype, heads, q_lens, kv_lens):
    run_case(dsa, dtype, heads, 128, 64, q_lens, kv_lens)


def test_large_scores(dsa):
    """Maxima that keep growing along the sequence: what has been summed is rescaled again and again."""
    for sign in (1.0, -1.0):
        def change(q, kv, kr):
            ramp = sign * torch.linspace(0, 8, kv.shape[0])
            kv[..., :128] = (kv[..., :128].float() + ramp[:, None, None] * q[200, :, :128].float() / 4).bfloat16()
        run_case(dsa, "bf16", 2, 128, 64, [600], change=change)


def test_same_inputs_same_bits(dsa):
    a = run_case(dsa, "bf16", 2, 128, 64, [300, 77])
    for _ in range(3):
        b = run_case(dsa, "bf16", 2, 128, 64, [300, 77])
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
