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


@pytest.mark.parametrize("dtype,C,G", [("fp32", 1028, 1), ("fp32", 2048, 1), ("fp32", 511, 1), ("bf16", 4096, 1), ("bf16", 4096, 2), ("bf16", 3600, 3), ("fp32", 333, 1)])
def test_slices_of_up_to_512_vectors(dtype, C, G):
    """A row of them that no registers hold: statistics of runs, joined."""
    import torch
    x = (2.0 + torch.randn(3, 500, C, device="cuda", generator=torch.Generator("cuda").manual_seed(C))).to(torch.float32 if dtype == "fp32" else torch.bfloat16)
    w = 1 + 0.1 * torch.randn(C, device="cuda")
    check(x, seedinf.group_norm(x, G, w, activation="silu"), G, w, None, "silu")
