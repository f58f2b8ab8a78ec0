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


@pytest.mark.parametrize("spread,eps", [(2.0 ** -66, 2.0 ** -146), (2.0 ** -70, 2.0 ** -140), (2.0 ** -75, 2.0 ** -149), (2.0 ** -63, 2.0 ** -126),
                                        (2.0 ** -66, 1e-30), (2.0 ** -50, 2.0 ** -149), (2.0 ** -45, 2.0 ** -110), (1e-25, 2.0 ** -149)])
@pytest.mark.parametrize("rotary,interleaved", [(128, False), (64, True)])
def test_squares_that_are_no_normal_numbers(spread, eps, rotary, interleaved):
    c = Case(42, 8, 2, [3, 7], [50, 1], rotary, interleaved, eps=eps, spread=spread)
    c.call()
    c.check()
