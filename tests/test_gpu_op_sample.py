"""seed_op_sample on the GPU against 64 bits: the same choices, and their log-probabilities to half a step of fp32."""
import numpy as np
import pytest

from paper_1910_06591_amd import seedinf
from tests import ops_reference as ref

pytestmark = pytest.mark.gpu


def args(R, V, dtype, seed=0, k=None, p=None, m=None, t=True, spread=2.5):
    import torch
    rng = np.random.default_rng(seed)
    x = torch.from_numpy((spread * rng.standard_normal((R, V))).astype(np.float32)).cuda().to(torch.float32 if dtype == "fp32" else torch.bfloat16)
    a = dict(logits=x, uniforms=rng.random(R, dtype=np.float32))
    if t:
        a["temperature"] = np.where(rng.random(R) < 0.1, 0, rng.uniform(0.3, 2.0, R)).astype(np.float32)
    if k is not None:
        a["top_k"] = np.resize(np.int32(k), R)
    if p is not None:
        a["top_p"] = np.resize(np.float32(p), R)
    if m is not None:
        a["min_p"] = np.resize(np.float32(m), R)
    return a


def check(a):
    import torch
    dev = {n: v if isinstance(v, torch.Tensor) else torch.from_numpy(np.ascontiguousarray(v)).cuda() for n, v in a.items()}
    token, logprob = seedinf.sample(**dev)
    want, wlp = ref.sample(dev["logits"].double().cpu().numpy(), *(a.get(n) for n in ("uniforms", "temperature", "top_k", "top_p", "min_p")))
    token, logprob = token.cpu().numpy(), logprob.double().cpu().numpy()
    assert np.array_equal(token, want), np.nonzero(token != want)[0][:10]
    assert np.array_equal(np.isinf(logprob), np.isinf(wlp))
    fine = ~np.isinf(wlp)
    # half a step of fp32; the sums' own error is some 1e-12
    assert (np.abs(logprob - wlp)[fine] <= ref.U32 * np.abs(wlp[fine]) + 1e-11).all()
    return token


SIZES = [(1, 1), (3, 2), (5, 6), (4096, 18), (70, 31), (9, 32), (9, 33), (130, 64), (7, 65), (40, 100), (3, 255), (3, 256), (5, 257), (20, 1000), (4, 4097),
         (3, 32000), (2, 50001), (1, 131072), (1, 200003), (300, 1500)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("R,V", SIZES)
def test_sizes(R, V, dtype):
    check(args(R, V, dtype, seed=V))
    check(args(R, V, dtype, seed=V + 1, k=[1, 5, 50, 0, V, V + 3, -1, V - 1], p=[0.9, 0.3, 1.0, 0.999], m=[0.0, 0.02, 0.3]))
    check(args(R, V, dtype, seed=V + 2, p=[0.95, 0.5, 0.0, 0.01]))
    check(args(R, V, dtype, seed=V + 3, m=[0.05, 1.0, 1.5, 1e-6]))
    check(args(R, V, dtype, seed=V + 4, k=[V // 2, V // 3, 3], t=False))


@pytest.mark.parametrize("V", [7, 40, 300, 5000, 40000])
def test_ties(V):
    """Few distinct values: ties go to the lowest index, also where a filter cuts through them."""
    rng = np.random.default_rng(V)
    import torch
    R = 24
    x = rng.integers(-2, 3, (R, V)).astype(np.float32)
    x[0] = 0.0
    x[1] = np.where(np.arange(V) % 2, 0.0, -0.0)                    # the two zeros are one value
    x[2] = np.finfo(np.float32).min
    x[3, :] = -1e30
    x[3, V // 2] = 0
    a = args(R, V, "fp32", seed=V, k=[3, V // 2, V - 1, 0], p=[0.7, 1.0, 0.2], m=[0.0, 0.5])
    a["logits"] = torch.from_numpy(x).cuda()
    check(a)
    a["temperature"][:] = 1.0
    check({n: a[n] for n in ("logits", "uniforms", "temperature")})
    check({n: a[n] for n in ("logits", "uniforms", "temperature", "top_p")})
    check({n: a[n] for n in ("logits", "uniforms", "temperature", "top_k")})
    check({n: a[n] for n in ("logits", "uniforms", "temperature", "min_p")})


@pytest.mark.parametrize("V", [5, 20, 64, 100, 3000, 40000])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_masks_and_values_that_are_not_finite(V, dtype):
    import torch
    R = 12
    a = args(R, V, dtype, seed=V, k=[0, 2, V], p=[1.0, 0.8])
    a["temperature"][:] = 0.8
    x = a["logits"]
    lowest = float(torch.finfo(x.dtype).min)
    x[0] = -np.inf                                                    # nothing left
    x[1] = float("nan")
    x[2, 1:] = -np.inf                                                # one left
    x[3, :V // 2] = -np.inf
    x[4, 1::2] = lowest                                               # masked by the type's lowest value
    x[5] = lowest
    x[6, V // 2:] = float("nan")
    x[7, V // 3] = np.inf
    x[8, ::2] = np.inf                                                # equal infinities share the mass
    x[9] = np.inf
    x[10] *= 40                                                       # far apart
    token = check(a)
    assert token[0] == -1 and token[1] == -1 and token[2] == 0 and token[7] == V // 3


@pytest.mark.parametrize("V", [18, 200, 9000])
def test_temperatures_and_uniforms_at_their_ends(V):
    import torch
    R = 40
    a = args(R, V, "fp32", seed=V, p=[1.0, 0.9, float("nan"), 2.0, -1.0], k=[0, 4])
    a["temperature"] = np.resize(np.float32([0.0, -1.0, np.nan, 1e-40, 1e-3, 1.0, 50.0, 1e30, np.inf]), R)
    a["uniforms"] = np.resize(np.float32([0.0, 1.0, -0.5, 2.0, np.nan, 1 - 2.0 ** -24, 0.5, 1e-30]), R)
    x = a["logits"]
    x[:, -1] = -np.inf
    check(a)
    # far offsets change nothing
    far = dict(a, logits=x + 1000.0)
    far["logits"] = (x.double() + 1000.0).float()
    check(far)


def test_rows_with_a_stride_and_odd_addresses():
    import torch
    for V in (18, 333, 20000):
        a = args(6, V, "bf16", seed=V, k=[0, 40], p=[0.9])
        wide = torch.zeros(6, V + 7, dtype=torch.bfloat16, device="cuda")
        wide[:, 5:5 + V] = a["logits"]
        want = check(a)
        assert np.array_equal(want, check(dict(a, logits=wide[:, 5:5 + V])))
        one = dict(a, logits=a["logits"][:1].expand(6, V))             # one row of logits, several draws
        check(one)


def test_offsets_past_32_bits():
    import torch
    V, far = 500, 2 ** 31 + 5
    a = args(2, V, "bf16", seed=1, p=[0.9])
    big = torch.empty(far + V, dtype=torch.bfloat16, device="cuda")
    view = big.as_strided((2, V), (far, 1))
    view.copy_(a["logits"])
    assert np.array_equal(check(a), check(dict(a, logits=view)))


def test_numbers_stand_for_every_row():
    import torch
    a = args(50, 300, "fp32", seed=9, t=False)
    u = torch.from_numpy(a["uniforms"]).cuda()
    got = seedinf.sample(a["logits"], u, temperature=0.8, top_k=20, top_p=0.9, min_p=0.05)
    f = lambda v: torch.full((50,), v, device="cuda")  # noqa: E731
    want = seedinf.sample(a["logits"], u, temperature=f(0.8), top_k=torch.full((50,), 20, dtype=torch.int32, device="cuda"), top_p=f(0.9), min_p=f(0.05))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_the_law_of_the_draw():
    """Frequencies over 200000 draws from one row: within 5 standard deviations of the kept probabilities."""
    import torch
    n, V = 200000, 12
    x = torch.linspace(-2, 1, V, device="cuda")
    u = torch.rand(n, device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    token, logprob = seedinf.sample(x.expand(n, V), u, top_k=8)
    prob = torch.softmax(x[4:].double(), 0)
    freq = torch.bincount(token, minlength=V).double() / n
    assert freq[:4].sum() == 0
    assert ((freq[4:] - prob).abs() <= 5 * (prob * (1 - prob) / n).sqrt()).all()
    assert torch.allclose(logprob.double(), torch.log(prob)[token.long() - 4], atol=1e-6)


@pytest.mark.parametrize("R,V", [(64, 18), (3, 3000), (2, 70000)])
def test_graph_and_stream(R, V):
    import torch
    xs = [args(R, V, "fp32", seed=s, k=[50], p=[0.9]) for s in range(2)]
    dev = [{n: v if isinstance(v, torch.Tensor) else torch.from_numpy(v).cuda() for n, v in a.items()} for a in xs]
    want = [seedinf.sample(**d) for d in dev]
    buf = {n: v.clone() for n, v in dev[0].items()}
    token, logprob = torch.zeros_like(want[0][0]), torch.zeros_like(want[0][1])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        seedinf.sample(**buf, token=token, logprob=logprob)
    for r in range(4):
        for n, v in dev[r % 2].items():
            buf[n].copy_(v)
        g.replay()
        eager = seedinf.sample(**dev[0])
        torch.cuda.synchronize()
        assert torch.equal(token, want[r % 2][0]) and torch.equal(logprob, want[r % 2][1]) and torch.equal(eager[0], want[0][0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [seedinf.sample(**dev[i % 2], stream=side.cuda_stream) for i in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(t[0], want[i % 2][0]) for i, t in enumerate(got))


def test_refusals_and_nothing_to_do():
    import torch
    x, u = torch.zeros(4, 10, device="cuda"), torch.zeros(4, device="cuda")
    assert seedinf.sample(x[:0], u[:0])[0].shape == (0,)
    for bad in (dict(logits=x.t()), dict(logits=x.half()), dict(logits=x[0]), dict(uniforms=u[:3]), dict(uniforms=u.double()), dict(top_k=u), dict(top_p=u.cpu()),
                dict(token=torch.zeros(4, device="cuda"))):
        with pytest.raises(TypeError):
            seedinf.sample(**dict(dict(logits=x, uniforms=u), **bad))
    with pytest.raises(seedinf.SeedError):
        seedinf.sample(torch.zeros(4, 0, device="cuda"), u)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("k,p,m", [(None, None, None), (50, None, None), (None, 0.9, None), (None, None, 0.02), (1000, 0.95, 0.001),
                                   (1024, 0.5, None), (1025, 0.99, None), (30000, 0.9, 0.01), (3, 0.0, 1.0)])
def test_long_rows_that_are_not_what_their_beginning_says(k, p, m, dtype):
    """Rising and falling rows, a beginning that is masked, a last choice far above the others, rows that are all but flat,
    masks in most places, temperatures that gather all mass in one choice or spread it over all."""
    import torch
    V = 70001
    rng = np.random.default_rng(9)
    line, noise = np.linspace(-12, 12, V), rng.standard_normal(V)
    rows = [line, -line, noise, noise.copy(), noise.copy(), 1e-3 * noise, np.where(rng.random(V) < 0.999, -np.inf, noise), 300 * noise, 1e-38 * noise]
    rows[3][:40000] = -np.inf
    rows[4][-1] = 500.0
    x = torch.from_numpy(np.repeat(np.stack(rows), 4, 0).astype(np.float32)).cuda().to(torch.float32 if dtype == "fp32" else torch.bfloat16)
    R = x.shape[0]
    a = dict(logits=x, uniforms=rng.random(R, dtype=np.float32), temperature=np.resize(np.float32([1.0, 0.05, 8.0, 1e-38]), R))
    a.update({n: np.resize(f(v), R) for n, v, f in (("top_k", k, np.int32), ("top_p", p, np.float32), ("min_p", m, np.float32)) if v is not None})
    check(a)


def test_sizes_past_32_bits_are_refused():
    """Sizes that a 32-bit field would wrap."""
    import torch
    one = torch.zeros(1, 4, device="cuda")
    with pytest.raises((TypeError, seedinf.SeedError)):
        seedinf.sample(one.expand((1 << 32) + 1, 4), torch.zeros(1, device="cuda"))
    with pytest.raises((TypeError, seedinf.SeedError)):
        seedinf.group_norm(one.expand((1 << 32) + 1, 4), 2)
    with pytest.raises((TypeError, seedinf.SeedError)):
        seedinf.decay_step(*(one[None].expand((1 << 32) + 1, 1, 4) for _ in range(3)), torch.ones(1, device="cuda"))
