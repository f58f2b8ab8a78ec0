"""Choices of cp_shared_prefix_attention's plan that follow from the lengths alone, without a GPU."""
import os

import pytest

import paper_2511_03475_amd as cp


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(cp.LIB_PATH):
        cp.build()
    return cp.load_library()


def plan(sizes, shared, P, E, Hq=8, Hkv=2):
    shape = cp.Shape(len(P), Hq, Hkv, 128, 16, 1 << 20, max((p + e + 15) // 16 for p, e in zip(P, E)), P, E, 0.1)
    sharing = cp.Sharing(sizes, shared)
    return cp.cp_shared_ranges(shape, sharing), cp.cp_shared_workspace_bytes(shape, sharing)


@pytest.mark.parametrize("new", [1, 2, 4])
def test_requests_without_new_tokens_at_the_end_change_nothing(new):
    """64 groups are a launch; what comes behind them is another one, and none at all without a new token."""
    kinds = set()
    for S in range(16, 2500, 48):
        P, E = [S + 300] * 128, [new] * 128
        alone = plan([2] * 64, [S] * 64, P, E)
        kinds.add(alone[0] > 0)
        for tail in (1, 5):
            assert plan([2] * 64 + [tail], [S] * 64 + [16], P + [16] * tail, E + [0] * tail) == alone, S
    assert kinds == {False, True}       # both plans are among them
