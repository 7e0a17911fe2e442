"""Values of eps that no norm has are refused where they are given."""
import math

import pytest
import torch

from paper_2608_24658_gb300.api import HeadNorm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [0.0, -1e-6, 1e-39, 1e39, math.inf, -math.inf, math.nan])
def test_eps(eps):
    with pytest.raises(ValueError):
        HeadNorm(torch.ones(128, device="cuda", dtype=torch.bfloat16), eps=eps)


@pytest.mark.parametrize("eps", [2.0 ** -126, 1e-6, 1.0, 3.4e38])
def test_eps_of_a_norm(eps):
    assert HeadNorm(torch.ones(128, device="cuda", dtype=torch.bfloat16), eps=eps).eps == eps
