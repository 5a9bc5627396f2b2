"""seed_op_sample on the GPU at values where masses of fewer bits, or differences that leave a type's range, would show."""
import math
from fractions import Fraction

import numpy as np
import pytest

from paper_1910_06591_amd import seedinf
from tests import ops_reference as ref
from tests.test_gpu_op_sample import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [9001, 50001, 1 << 20, 1 << 24])
def test_a_leader_above_equal_choices(V, dtype):
    """One choice far above all others, which are equal: the draw is a quotient.  Its place is off by at most one choice and
    2^-37 of the place (the masses' error); the log-probability by that and half a step of fp32."""
    import torch
    rows = [(gap, u) for gap in (8.0, 14.0, 16.0, 18.0) for u in (0.3, 0.5, 0.9, 0.999, 1 - 2.0 ** -24)]
    x = torch.zeros(len(rows) if V < 1 << 24 else 4, V, device="cuda", dtype=torch.float32 if dtype == "fp32" else torch.bfloat16)
    for some in (rows,) if V < 1 << 24 else (rows[i:i + 4] for i in range(0, len(rows), 4)):
        x[:, 7] = torch.tensor([gap for gap, _ in some], device="cuda")
        token, logprob = seedinf.sample(x, torch.tensor([u for _, u in some], device="cuda"))
        for (gap, u), t, lp in zip(some, token.tolist(), logprob.double().tolist()):
            m = Fraction(math.exp(-gap))
            z = 1 + (V - 1) * m
            place = int((Fraction(float(np.float32(u))) * z - 1) / m) if Fraction(float(np.float32(u))) * z >= 1 else -1      # among the equal ones
            want = 7 if place < 0 else place if place < 7 else place + 1
            assert abs(t - want) <= (1 + place * 2.0 ** -37 if place >= 0 else 0), (gap, u)
            lw = -math.log(z) - (gap if t != 7 else 0)
            assert abs(lp - lw) <= ref.U32 * abs(lw) + 2.0 ** -36, (gap, u)


@pytest.mark.parametrize("V", [200, 9000, 70001])
@pytest.mark.parametrize("t", [1e37, 3e38])
def test_logits_whose_difference_leaves_the_type(V, t):
    """Differences of up to 6e38 at temperatures that they are a few of."""
    import torch
    rng = np.random.default_rng(V)
    R = 16
    x = rng.uniform(-3.3e38, 3.3e38, (R, V)).astype(np.float32)
    x[:4, 1:] = -3.3e38
    x[:4, 0] = 3.3e38
    a = dict(logits=torch.from_numpy(x).cuda(), uniforms=rng.random(R, dtype=np.float32), temperature=np.full(R, t, np.float32))
    check(a)
    check(dict(a, top_p=np.full(R, 0.8, np.float32)))
    check(dict(a, top_k=np.full(R, V // 2, np.int32)))
    check(dict(a, min_p=np.full(R, 0.3, np.float32)))


@pytest.mark.parametrize("V", [3, 18, 64, 300, 9000, 20000])
def test_infinite_logits_at_an_infinite_temperature(V):
    """All finite choices are equal there; beside infinite ones they are none."""
    import torch
    x = torch.linspace(-3, 3, V, device="cuda").repeat(6, 1)
    x[:, 1] = -math.inf
    x[3:, 0] = x[3:, V - 1] = math.inf
    u = torch.tensor([0.0, 0.4, 0.99] * 2, device="cuda")
    token, logprob = seedinf.sample(x, u, temperature=math.inf)
    finite = [0] + list(range(2, V))
    order = [V - 1] + list(range(V - 2, 1, -1)) + [0] if V > 2 else [0]
    want = [order[int(Fraction(float(np.float32(p))) * len(finite))] for p in (0.0, 0.4, 0.99)]
    assert token.tolist() == want + [0, 0, V - 1]
    lw = torch.tensor([-math.log(V - 1)] * 3 + [-math.log(2)] * 3, device="cuda", dtype=torch.float64)
    assert ((logprob.double() - lw).abs() <= ref.U32 * lw.abs() + 1e-11).all()
