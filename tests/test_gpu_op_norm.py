"""seed_op_group_norm on the GPU against 64 bits."""
import numpy as np
import pytest

from paper_1910_06591_amd import seedinf
from tests import ops_reference as ref

pytestmark = pytest.mark.gpu


def make(N, P, C, dtype, seed=0, offset=2.0):
    import torch
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((N, P, C)) * (0.5 + rng.random(C)) + offset * rng.standard_normal(C)
    w, b = (1 + 0.2 * rng.standard_normal(C)).astype(np.float32), (0.2 * rng.standard_normal(C)).astype(np.float32)
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    return torch.from_numpy(x.astype(np.float32)).cuda().to(dt), torch.from_numpy(w).cuda(), torch.from_numpy(b).cuda()


def check(x, y, groups, w, b, act, eps=1e-5):
    host = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
    want, mag = ref.group_norm(host(x), groups, host(w), host(b), eps, act)
    tol = ref.group_norm_tolerance(want, mag, x.element_size() == 2)
    err = np.abs(host(y) - want)
    assert np.isfinite(host(y)).all()
    assert (err <= tol).all(), f"worst {np.max(err / tol):.2f} of the tolerance"


SIZES = [  # N, P, C, G
    (1, 1, 1, 1), (1, 1, 2, 1), (3, 1, 64, 4), (5, 1, 70, 7), (4, 1, 2048, 16), (1000, 1, 128, 128), (2, 1, 8192, 1), (33, 1, 520, 65), (2, 1, 20000, 4),
    (2, 5, 3, 3), (2, 7, 12, 2), (3, 49, 16, 4), (2, 100, 24, 24), (1, 1728, 32, 8), (70, 1728, 32, 8), (300, 432, 64, 1), (3, 1000, 5, 1),
    (1, 40000, 8, 2), (1, 9000, 40, 5), (2, 4097, 320, 32), (1, 100001, 3, 1), (600, 300, 20, 10), (1, 2, 12288, 3), (7, 3, 4100, 100),
    (1, 5000, 260, 130), (65, 700, 130, 13), (2, 33, 10001, 1),
]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("N,P,C,G", SIZES)
def test_sizes(N, P, C, G, dtype):
    x, w, b = make(N, P, C, dtype, seed=N + P)
    y = seedinf.group_norm(x, G, w, b, activation="silu")
    check(x, y, G, w, b, "silu")


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("use_w,use_b", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("N,P,C,G", [(9, 1, 256, 4), (4, 60, 48, 6), (1, 9000, 64, 8)])
def test_parameters(N, P, C, G, use_w, use_b, act):
    x, w, b = make(N, P, C, "fp32")
    w, b = w if use_w else None, b if use_b else None
    check(x, seedinf.group_norm(x, G, w, b, activation=act), G, w, b, act)


@pytest.mark.parametrize("N,P,C,G", [(6, 1, 512, 4), (6, 400, 32, 4), (1, 30000, 16, 4)])
def test_far_from_zero_and_constant(N, P, C, G):
    """A spread that is small beside the mean (the sum of squares minus the squared mean would lose it), and none at all."""
    import torch
    x, w, b = make(N, P, C, "fp32")
    y = x * 0.01 + 100.0
    check(y, seedinf.group_norm(y, G, w, b), G, w, b, "none")
    flat = torch.full_like(x, 3.0)
    got = seedinf.group_norm(flat, G, w, b)
    assert torch.allclose(got, b.expand_as(got), atol=1e-3 * 2 ** -10)     # (a constant's mean is itself: the difference is exactly zero)
    check(x, seedinf.group_norm(x, G, w, b, eps=0.5), G, w, b, "none", eps=0.5)


def test_maps_in_place_and_odd_addresses():
    import torch
    for shape, G in (((3, 9, 12, 32), 8), ((40, 1, 1, 64), 2), ((1, 200, 150, 24), 3)):
        x, w, b = make(shape[0], shape[1] * shape[2], shape[3], "bf16")
        x = x.view(shape)
        want = seedinf.group_norm(x, G, w, b, activation="relu")
        assert want.shape == shape
        flat = torch.empty(x.numel() + 1, dtype=x.dtype, device="cuda")[1:].view(shape)
        odd = torch.empty(2 * shape[3] + 1, device="cuda")[1:]
        odd[:shape[3]], odd[shape[3]:] = w, b
        got = seedinf.group_norm(flat.copy_(x), G, odd[:shape[3]], odd[shape[3]:], activation="relu", out=flat)
        assert got is flat
        check(x.flatten(1, 2), flat.flatten(1, 2), G, w, b, "relu")
        y = x.clone()
        seedinf.group_norm(y, G, w, b, activation="relu", out=y)
        assert torch.equal(y, want)


@pytest.mark.parametrize("N,P,C,G", [(4, 1, 256, 4), (4, 300, 32, 4), (1, 30000, 32, 4)])
def test_a_value_that_is_not_finite_stays_in_its_group(N, P, C, G):
    import torch
    x, w, b = make(N, P, C, "fp32")
    want = seedinf.group_norm(x, G, w, b)
    y = x.clone()
    y[N - 1, P // 2, C // G] = float("inf")
    got = seedinf.group_norm(y, G, w, b).view(N, P, G, -1)
    hit = torch.zeros(N, G, dtype=torch.bool)
    hit[N - 1, 1] = True
    assert torch.equal(got.transpose(1, 2)[~hit], want.view(N, P, G, -1).transpose(1, 2)[~hit])
    assert torch.isnan(got.transpose(1, 2)[hit]).any()


def test_more_than_2_31_elements():
    import torch
    N, P, C = 36000, 1000, 64
    x = torch.empty(N, P, C, dtype=torch.bfloat16, device="cuda")
    part, w, b = make(8, P, C, "bf16")
    x[:] = 0
    x[:4], x[-4:] = part[:4], part[4:]
    got = seedinf.group_norm(x, 4, w, b, out=x)
    check(part[4:], got[-4:], 4, w, b, "none")
    check(part[:4], got[:4], 4, w, b, "none")


def test_graph_and_stream():
    import torch
    for N, P, C, G in ((16, 1, 512, 8), (1, 20000, 64, 8)):
        x, w, b = make(N, P, C, "bf16")
        x2 = make(N, P, C, "bf16", seed=1)[0]
        want = [seedinf.group_norm(v, G, w, b, activation="silu") for v in (x, x2)]
        buf, out = x.clone(), torch.zeros_like(x)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            seedinf.group_norm(buf, G, w, b, activation="silu", out=out)
        for r in range(4):
            buf.copy_((x, x2)[r % 2])
            g.replay()
            eager = seedinf.group_norm(x, G, w, b, activation="silu")
            torch.cuda.synchronize()
            assert torch.equal(out, want[r % 2]) and torch.equal(eager, want[0])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = [seedinf.group_norm(x, G, w, b, activation="silu", stream=side.cuda_stream) for _ in range(3)]
        torch.cuda.synchronize()
        assert all(torch.equal(t, want[0]) for t in got)


def test_nothing_to_do_and_refusals():
    import torch
    w = torch.ones(8, device="cuda")
    assert seedinf.group_norm(torch.empty(0, 5, 8, device="cuda"), 2, w).shape == (0, 5, 8)
    assert seedinf.group_norm(torch.empty(3, 0, 8, device="cuda"), 2, w).shape == (3, 0, 8)
    x = torch.zeros(2, 5, 8, device="cuda")
    for bad in (dict(x=x.half()), dict(x=x.transpose(0, 1)), dict(weight=w[:4]), dict(weight=w.bfloat16()), dict(out=x[:1]), dict(x=x[0, 0])):
        with pytest.raises(TypeError):
            seedinf.group_norm(**dict(dict(x=x, groups=2, weight=w), **bad))
    with pytest.raises(ValueError):
        seedinf.group_norm(x, 2, activation="tanh")
    with pytest.raises(seedinf.SeedError):
        seedinf.group_norm(x, 3)


def test_more_workgroups_than_one_launch_takes():
    """2^21 + 3 rows of 1025 points of one channel, bf16: offsets past 2^32 bytes, and a grid of more than 2^21 workgroups of 512 threads."""
    import torch
    N, P = (1 << 21) + 3, 1025
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GB")
    x = torch.empty(N, P, 1, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(3))
    y = seedinf.group_norm(x, 1, activation="relu")
    for rows in (slice(0, 5), slice((1 << 21) - 4, N)):
        check(x[rows], y[rows], 1, None, None, "relu")
