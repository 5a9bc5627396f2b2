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


@pytest.mark.parametrize("P", [(1 << 31) - 1, (1 << 31) - 1030])
def test_the_longest_rows(P):
    """Statistics in 64 bits over a row of 2^31 - 1 points, and its first and last outputs."""
    import torch
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    x = torch.empty(1, P, 1, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(5))
    x += 2
    y = seedinf.group_norm(x, 1, out=torch.zeros_like(x))
    parts = x.view(-1).split(1 << 27)
    mean = sum(float(c.double().sum()) for c in parts) / P
    var = sum(float((c.double() - mean).square().sum()) for c in parts) / P
    for at in (slice(0, 3000), slice(P // 2, P // 2 + 3000), slice(P - 3000, P)):
        want = ((x[0, at, 0].double() - mean) / np.sqrt(var + 1e-5)).cpu().numpy()
        mag = 8 / np.sqrt(var) + np.abs(want)
        assert (np.abs(y[0, at, 0].double().cpu().numpy() - want) <= ref.group_norm_tolerance(want, mag, True)).all()


@pytest.mark.parametrize("N,P,C,G", [(6, 1, 512, 4), (6, 400, 32, 4), (1, 30000, 16, 4), (3, 500, 1028, 1), (1, 40, 8192, 1)])
def test_a_constant_whose_square_overflows(N, P, C, G):
    """No spread, or one of the mean's last bit: what overflows is not multiplied by a weight of zero, and the result is
    finite."""
    import torch
    x = torch.full((N, P, C), 2.0 ** 84, device="cuda")
    y = seedinf.group_norm(x, G, bias=torch.randn(C, device="cuda"))
    assert torch.isfinite(y).all()


@pytest.mark.parametrize("P", [1, 40])
def test_silu_is_good_to_its_last_bits(P):
    """A weight of zero: the result is the bias' silu, for every bias from -110 to 60, to 9 roundings of 2^-24 (two are the
    instructions' for the power and the reciprocal, which are good to a unit, and count twice: 11), or to 2^-118, below which
    it is zero."""
    import torch
    C = 16384
    b = np.linspace(-110, 60, C).astype(np.float32)
    x = torch.randn(2, P, C, device="cuda")
    y = seedinf.group_norm(x, 64, torch.zeros(C, device="cuda"), torch.from_numpy(b).cuda(), activation="silu")
    v = b.astype(np.longdouble)
    want = v / (1 + np.exp(-v))
    err = np.abs(y.cpu().numpy().astype(np.longdouble) - want)
    assert (err <= 11 * ref.U32 * np.abs(want) + 2.0 ** -118).all(), np.max(err / np.maximum(np.abs(want), 1e-35)) / ref.U32
    ends = torch.tensor([[np.inf, -np.inf, np.nan, -1e30, 1e30, 0.0, -0.0, -200.0]], dtype=torch.float32, device="cuda")
    y = seedinf.group_norm(torch.randn(1, 8, device="cuda"), 1, torch.zeros(8, device="cuda"), ends[0], activation="silu")[0]
    assert y[0] == np.inf and torch.isnan(y[1:3]).all() and y[4] == ends[0, 4] and (y[[3, 5, 6, 7]] == 0).all()
