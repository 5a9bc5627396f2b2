"""seed_op_group_norm on the GPU at lengths and values where sums in too few bits or in an unfortunate order would show."""
import numpy as np
import pytest

from paper_1910_06591_amd import seedinf
from tests import ops_reference as ref
from tests.test_gpu_op_norm import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,P,C,G", [(1, 16384, 1280, 1), (1, 65536, 333, 1), (1, 1 << 20, 16, 1), (2, 300000, 24, 3), (1, 1, 4000000, 1), (8, 1728, 32, 2)])
@pytest.mark.parametrize("mean,spread", [(100.02, 0.1), (-3.0, 1.0)])
def test_long_groups_far_from_zero(N, P, C, G, mean, spread):
    """A group of up to 21 million values of one sign: their sum is millions of times a term."""
    import torch
    x = mean + spread * torch.randn(N, P, C, device="cuda", generator=torch.Generator("cuda").manual_seed(P))
    check(x, seedinf.group_norm(x, G), G, None, None, "none")
