"""How the blocks of a prompt call (dsa_latent_prompt) find their work: long runs of requests without a token, very many requests,
bounds of the queries far above what the requests have."""
import pytest
import torch

from tests.test_gpu_prompt import run_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dsa():
    from paper_2609_19702_b200 import binding
    return binding


def test_runs_of_requests_without_a_token(dsa):
    """A running block passes over hundreds of blocks without a query between one item and the next, each time the same."""
    lens = [0] * 3000
    for b, n in ((0, 3), (700, 260), (701, 1), (1999, 40), (2999, 129)):
        lens[b] = n
    first = run_case(dsa, "bf16", 8, 64, 8, lens)
    for _ in range(10):
        again = run_case(dsa, "bf16", 8, 64, 8, lens)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_a_run_longer_than_a_wait_may_take(dsa):
    """A million requests of 1024 heads, hardly any with a token: what a block finds behind seconds of nothing is computed too."""
    lens = [0] * 2 ** 20
    for b, n in ((0, 1), (2 ** 19 + 3, 2), (2 ** 20 - 1, 3)):
        lens[b] = n
    run_case(dsa, "bf16", 1024, 64, 8, lens)
