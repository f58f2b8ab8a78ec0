"""Groups of cp_shared_prefix_attention anywhere among the 64 requests that are looked at together."""
import numpy as np
import pytest

import paper_2511_03475_amd as cp
from shared_prefix_case import Batch
from test_gpu_shared_prefix import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sizes", [[63, 1, 2, 62, 3], [64, 64, 2], [65, 130, 1, 4], [1, 31, 1, 31, 64, 2], [200], [2] * 63 + [70], [2] * 64, [1] * 66 + [3],
                                   [5] * 13 + [127, 2]])
@pytest.mark.parametrize("own", ["some", "none", "by group"])
@pytest.mark.parametrize("splits", [1, 2])
def test_groups_that_begin_and_end_around_64_requests(sizes, own, splits):
    """Every third group shares nothing, so that groups do not follow each other without a gap."""
    rng = np.random.default_rng(len(sizes))
    n, shared = sum(sizes), [0 if i % 3 == 1 else 16 * (1 + i % 9) for i in range(len(sizes))]
    group = np.repeat(np.arange(len(sizes)), sizes)
    tokens = {"some": rng.integers(0, 40, n), "none": np.zeros(n, int), "by group": np.where(group % 2, rng.integers(0, 40, n), 0)}[own]
    check(Batch(n + splits, 4, 2, sizes, shared, tokens, rng.integers(0, 3, n), splits))


@pytest.mark.parametrize("groups", [2, 33, 64])
def test_results_do_not_depend_on_the_groups_around(groups):
    """The same group in front of others, and between them: bit for bit what it gives alone."""
    from test_gpu_shared_prefix import Device
    rng = np.random.default_rng(groups)
    sizes = rng.integers(1, 5, groups).tolist()
    n = sum(sizes)
    b = Batch(groups, 4, 2, sizes, [96] * groups, [7] * n, [2] * n, 1)
    d = Device(b)
    d.call()
    whole = d.bits().copy()
    for g in (0, groups // 2, groups - 1):
        first, size = sum(sizes[:g]), sizes[g]
        rows = slice(first, first + size)
        one = Batch(0, 4, 2, [size], [96], [7] * size, [2] * size, 1)
        one.q, one.k, one.v = (x[2 * first:2 * (first + size)] for x in (b.q, b.k, b.v))
        one.table, one.width, one.pool, one.pages = b.table[rows], b.width, b.pool, b.pages
        one.set(1)
        e = Device(one)
        assert cp.cp_shared_ranges(one.shape, one.sharing) == 1
        e.call()
        assert (e.bits() == whole[2 * first:2 * (first + size)]).all()
