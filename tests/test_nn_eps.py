"""The norms' eps: what has no root is refused, without a GPU."""
import pytest

from paper_2010_13972_amd import gts
from test_nn_arguments import norm, norm_grad


@pytest.mark.parametrize("eps", [-1e-6, -float("inf"), float("nan")])
@pytest.mark.parametrize("rows", [0, 4])
def test_eps_refused(eps, rows):
    for call in (norm(eps=eps, rows=rows), norm_grad(eps=eps, rows=rows)):
        assert call() == gts.GTS_EINVAL and "eps" in gts.last_error()
