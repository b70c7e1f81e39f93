"""Sizes of a plan at the ends of their range (no GPU needed)."""
import pytest


@pytest.fixture(scope="module")
def aiq():
    from paper_2512_14090_b200 import build
    build.build()
    from paper_2512_14090_b200 import binding
    return binding


@pytest.mark.parametrize("top_k,e", [(1, 1), (1, 2), (2, 2), (8, 8), (1, 1024), (16, 1024)])
def test_a_plan_of_twice_the_tokens_has_at_most_twice_the_bytes(aiq, top_k, e):
    """Up to 2^30 pairs: blocks of rows stay as wide as they are for half of them."""
    t = 2 ** 30 // top_k
    while t > 4096:
        assert 0 < aiq.aiq_expert_plan_bytes(t, top_k, e) <= 2 * aiq.aiq_expert_plan_bytes(t // 2, top_k, e)
        t //= 2
