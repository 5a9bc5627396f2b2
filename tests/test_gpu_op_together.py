"""The operators together, as a caller composes them: a recurrent core over stored trajectories, its output normalised
head by head, a head's logits, actions; the same agent step by step; and filtered sampling inside the agent's step."""
import ctypes as C

import numpy as np
import pytest

from paper_1910_06591_amd import seedinf, workloads as wl
from tests import ops_reference as ref
from tests.parity import to_device

pytestmark = pytest.mark.gpu


def test_core_norm_and_sampling_as_one_agent():
    import torch
    T, B, H, d, A = 40, 6, 4, 64, 18
    gen = torch.Generator("cuda").manual_seed(0)
    randn = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    proj = randn(T, B, 3 * H * d)                                       # one projection's output: queries, keys, values
    proj[:, :, H * d:2 * H * d] *= d ** -0.5
    q, k, v = (proj[:, :, i * H * d:(i + 1) * H * d].view(T, B, H, d) for i in range(3))
    decay, done = torch.tensor([0.5, 0.9, 0.97, 0.995], device="cuda"), (torch.rand(T, B, device="cuda", generator=gen) < 0.1).to(torch.uint8)
    w, b, head, u = 1 + 0.1 * randn(H * d), 0.1 * randn(H * d), randn(H * d, A) * (H * d) ** -0.5, torch.rand(T, B, device="cuda", generator=gen)
    rule = dict(temperature=0.9, top_k=12, top_p=0.9, min_p=0.01)
    state = randn(B, H, d, d)

    def behind(o):                                                     # [n, H, d] -> actions
        y = seedinf.group_norm(o.reshape(-1, H * d), H, w, b, activation="silu")
        return y, y @ head

    out, last = seedinf.decay_attention(q, k, v, decay, state=state, done=done)
    y, logits = behind(out)
    token, logprob = seedinf.sample(logits, u.view(-1), **rule)

    host = lambda t: t.double().cpu().numpy()  # noqa: E731
    ro, rs, mag, M = ref.decay(host(q), host(k), host(v), host(decay), host(state), host(done))
    tol_o, tol_s = ref.decay_tolerance(ro, mag, rs, M, T, d, False)
    assert (np.abs(host(out) - ro) <= tol_o).all() and (np.abs(host(last) - rs) <= tol_s).all()
    ry, ymag = ref.group_norm(host(out).reshape(T * B, 1, H * d), H, host(w), host(b), 1e-5, "silu")
    assert (np.abs(host(y) - ry[:, 0]) <= ref.group_norm_tolerance(ry, ymag, False)[:, 0]).all()
    n = np.ones(T * B)
    rule32 = [np.float32(v) * np.ones(T * B, np.float32) for v in (0.9, 0.9, 0.01)]
    rt, rl = ref.sample(host(logits), host(u.view(-1)), rule32[0], (12 * n).astype(np.int32), rule32[1], rule32[2])
    assert np.array_equal(token.cpu().numpy(), rt)
    assert (np.abs(host(logprob) - rl) <= ref.U32 * np.abs(rl) + 1e-11).all()

    # the same agent one environment step at a time, the state in place, as a captured graph
    s, bufs = state.clone(), dict(q=q[0].clone(), k=k[0].clone(), v=v[0].clone(), done=done[0].clone())
    ut, tok = u[0].clone(), torch.empty(B, dtype=torch.int32, device="cuda")

    def step():
        o, _ = seedinf.decay_step(bufs["q"], bufs["k"], bufs["v"], decay, state=s, done=bufs["done"], state_out=s)
        yt, lt = behind(o)
        seedinf.sample(lt, ut, token=tok, **rule)
        return yt

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        yt = step()
    s.copy_(state)
    for t in range(T):
        for n_, src in (("q", q), ("k", k), ("v", v), ("done", done)):
            bufs[n_].copy_(src[t])
        ut.copy_(u[t])
        g.replay()
        torch.cuda.synchronize()
        # the step's own roundings: sums of 64 terms in another order
        assert torch.allclose(yt, y.view(T, B, -1)[t], atol=2e-4, rtol=2e-4)
    assert (np.abs(host(s) - rs) <= tol_s).all()


@pytest.mark.parametrize("name,B", [("C1", 9), ("C2", 21), ("C3", 33), ("C4", 5)])
@pytest.mark.parametrize("static", [False, True])
def test_sampling_inside_the_step(name, B, static):
    """The step's action is seed_op_sample's on the step's logits, whatever the arch's own selection; nothing else changes."""
    import torch
    cfg = wl.CONFIGS[name]
    net = seedinf.SeedInfer(seedinf.make_arch(cfg, max_batch=B), wl.make_weights(cfg))
    batch = to_device(wl.make_batch(cfg, B))
    plain = net.step(**batch, static_workspace=static)
    batch["uniforms"] = None
    gen = torch.Generator("cuda").manual_seed(1)
    u = torch.rand(B, device="cuda", generator=gen)
    rule = dict(temperature=0.1 + torch.rand(B, device="cuda", generator=gen), top_k=torch.full((B,), 5, dtype=torch.int32, device="cuda"),
                top_p=torch.full((B,), 0.9, device="cuda"), min_p=torch.full((B,), 0.05, device="cuda"))
    for r in ({}, rule):
        got = net.step(**batch, sample_uniforms=u, static_workspace=static, **r)
        token, _ = seedinf.sample(got["logits"], u, **r)
        torch.cuda.synchronize()
        assert torch.equal(got["action"], token)
        for key in plain:
            assert key == "action" or torch.equal(got[key], plain[key]), key
    net.close()


def test_step_refuses_two_selections_and_accepts_the_shorter_struct():
    import torch
    cfg = wl.CONFIGS["C1"]
    B = 4
    net = seedinf.SeedInfer(seedinf.make_arch(cfg, max_batch=B), wl.make_weights(cfg))
    batch = to_device(wl.make_batch(cfg, B))
    u = torch.rand(B, device="cuda")
    eps = dict(epsilon=u, explore_uniforms=torch.rand(B, 2, device="cuda"))
    none = dict(batch, uniforms=None)
    for bad, text in ((dict(batch, sample_uniforms=u), "uniforms"), (dict(none, sample_uniforms=u, **eps), "epsilon"), (dict(batch, temperature=u), "sample_uniforms"),
                      (dict(batch, top_p=u), "sample_uniforms"), (none, "uniforms")):
        with pytest.raises(seedinf.SeedError) as e:
            net.step(**bad)
        assert e.value.status == 1 and text in e.value.message
    # a caller compiled against the fields up to explore_uniforms: what lies behind them is not looked at
    ext = seedinf.SeedStepExt(seedinf.SeedStepExt.sample_uniforms.offset, None, None, None, 1, 1, 1, 1, 1)
    want = net.step(**batch)
    out = {k: torch.empty_like(v) for k, v in want.items()}
    st, msg = net.step_ext_raw(B, batch["obs"].data_ptr(), None, None, None, None, batch["uniforms"].data_ptr(), ext, out["action"].data_ptr(),
                               out["logits"].data_ptr(), out["value"].data_ptr(), None, None, out["probs"].data_ptr())
    torch.cuda.synchronize()
    assert st == 0, msg
    assert all(torch.equal(out[k], want[k]) for k in want)
    net.close()


def test_step_refuses_sampling_arguments_before_anything_runs():
    """Uniforms that are the actions' own memory, top_k at an odd address: the outputs stay as they were."""
    import torch
    cfg = wl.CONFIGS["C1"]
    B = 4
    net = seedinf.SeedInfer(seedinf.make_arch(cfg, max_batch=B), wl.make_weights(cfg))
    batch = to_device(wl.make_batch(cfg, B))
    out = {k: torch.empty_like(v) for k, v in net.step(**batch).items()}
    for v in out.values():
        v.fill_(7)
    u = torch.rand(B, device="cuda")
    for fields, status in (((out["action"].data_ptr(), None, None, None, None), 4), ((u.data_ptr(), None, u.data_ptr() + 2, None, None), 1)):
        ext = seedinf.SeedStepExt(C.sizeof(seedinf.SeedStepExt), None, None, None, *fields)
        st, _ = net.step_ext_raw(B, batch["obs"].data_ptr(), None, None, None, None, None, ext, out["action"].data_ptr(),
                                 out["logits"].data_ptr(), out["value"].data_ptr(), None, None, out["probs"].data_ptr())
        torch.cuda.synchronize()
        assert st == status
        assert all((v == 7).all() for v in out.values())
    net.close()
