"""cp_qk_norm_rope where the mean of the squares, or eps, is next to the ends of fp32."""
import pytest

from test_gpu_norm_rope import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("spread,eps", [(1e19, 1e38), (3e19, 1e36), (1e18, 2.0 ** 127), (1e19, 1.9 * 2.0 ** 127), (1.0, 1.9 * 2.0 ** 127), (1e37, 1e38)])
@pytest.mark.parametrize("rotary,interleaved", [(128, False), (64, True)])
def test_large_squares_next_to_a_large_eps(spread, eps, rotary, interleaved):
    c = Case(41, 8, 2, [3, 7], [50, 1], rotary, interleaved, eps=eps, spread=spread)
    c.call()
    c.check()
