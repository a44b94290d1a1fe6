"""Layouts of q, k_nope, k_rope and v in a prompt call (dsa_latent_prompt) that their strides describe."""
import math

import pytest
import torch

from tests import latent_ref
from tests.test_gpu_prompt import DT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dsa():
    from paper_2609_19702_b200 import binding
    return binding


def _check(dsa, q, k_nope, k_rope, v, lens, dtype, causal=True):
    start = torch.tensor([0] + lens).cumsum(0).int().cuda()
    p = dsa.Prompt(q, k_nope, k_rope, v, start, max_q_len=max(lens), causal=causal)
    out, lse = dsa.alloc_prompt_outputs(p)
    dsa.dsa_latent_prompt(p, out, lse)
    at = 0
    for n in lens:
        if n:
            x = [t[at:at + n].cpu().double() for t in (q, k_nope, k_rope, v)]
            o, l, tol, ltol = latent_ref.prompt_expected(*x, causal, 1 / math.sqrt(q.shape[2]), dtype == "bf16")
            latent_ref.assert_near(out[at:at + n], o, tol, "out")
            latent_ref.assert_near(lse[at:at + n], l, ltol, "lse")
        at += n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rope", [(128, 64), (64, 24)])
@pytest.mark.parametrize("heads,lens", [(3, [300, 0, 41]), (1, [90]), (5, [1]), (4, [257, 130, 1])])
def test_heads_outside_tokens(dsa, dtype, d, rope, heads, lens):
    """q, k_nope and v with a head's tokens end to end: token strides below head strides; in one of two forms the parts of one
    tensor, with room behind every head and row."""
    g = torch.Generator().manual_seed(heads)
    n = sum(lens)
    rand = lambda *s: torch.randn(s, generator=g).to(DT[dtype]).cuda()  # noqa: E731
    kr = rand(n, rope)
    q, k, v = (rand(heads, n, w).transpose(0, 1) for w in (d + rope, d, d))
    _check(dsa, q, k, kr, v, lens, dtype)
    q = rand(heads, n + 5, d + rope + 8)[:, :n, :d + rope].transpose(0, 1)
    kv = rand(heads, n + 3, 2 * d + 16)[:, :n].transpose(0, 1)
    _check(dsa, q, kv[..., :d], kr, kv[..., d + 16:], lens, dtype, causal=heads != 4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_q_tokens_outside_heads_keys_the_other_way(dsa, dtype):
    g = torch.Generator().manual_seed(2)
    rand = lambda *s: torch.randn(s, generator=g).to(DT[dtype]).cuda()  # noqa: E731
    n, h = 171, 6
    rows = rand(n, 512 + 64)                                 # k_rope where it lies in the rows of a cache
    _check(dsa, rand(n, h, 192), rand(h, n, 128).transpose(0, 1), rows[:, 512:], rand(n, h, 128), [100, 71], dtype)
