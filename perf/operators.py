"""The stand-alone operators that the library offers beside the agent's step, and the calls they are timed on.

A case is a plain dict; "op" says which operator:

  "decay"   linear attention with a decay for each head (seedinf.decay_attention / seedinf.decay_step): a recurrent
            core whose state is a matrix per head.  steps = 1 is the form for single tokens, one call per
            environment step; steps > 1 is the form for unrolls and prompts, time-major.
              steps, rows, heads, kv_heads, key_dim, value_dim, dtype
              flags   episode flags are given: a flagged row starts from the zero state
              ragged  the rows have lengths of their own
  "norm"    group normalisation with an activation, channels last (seedinf.group_norm)
              rows, points (h * w of a map, 1 for a vector), channels, groups, dtype, act
              affine  with a weight and a bias per channel
  "sample"  sampling with temperature, top-k, top-p and min-p from given uniforms (seedinf.sample)
              rows, choices, dtype, k, p, m (0 = off), and
              masked  a twentieth of the choices is masked with -inf, and now and then a whole row
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
CHUNK = 64


def listed():
    def decay(name, steps, rows, heads, dim, dtype, kv_heads=None, value_dim=None, flags=False, ragged=False):
        return dict(name=name, op="decay", steps=steps, rows=rows, heads=heads, kv_heads=kv_heads or heads, key_dim=dim,
                    value_dim=value_dim or dim, dtype=dtype, flags=flags, ragged=ragged)

    def norm(name, rows, points, channels, groups, dtype, act, affine=True):
        return dict(name=name, op="norm", rows=rows, points=points, channels=channels, groups=groups, dtype=dtype, act=act, affine=affine)

    def sample(name, rows, choices, dtype, k=0, p=0.0, m=0.0, masked=False):
        return dict(name=name, op="sample", rows=rows, choices=choices, dtype=dtype, k=k, p=p, m=m, masked=masked)

    return [
        # a handful of actors, one environment step of a 256-unit core in four heads: latency
        decay("decay_step_b8", 1, 8, 4, 64, "fp32", flags=True),
        # one step of many actors or streams with wide heads: the states are the traffic
        decay("decay_step_b256", 1, 256, 16, 128, "bf16", flags=True),
        # the learner's pass over stored trajectories, episode ends inside them
        decay("decay_unroll_32x128", 32, 128, 4, 64, "fp32", flags=True),
        # prompts of unequal length, queries sharing keys and values in groups of four
        decay("decay_prompts_4x4001", 4001, 4, 16, 128, "bf16", kv_heads=4, ragged=True),
        # one long sequence: few independent states, so the time axis has to be split
        decay("decay_long_32768", 32768, 1, 16, 128, "bf16"),
        # the core's output normalised head by head, a row for each actor
        norm("norm_heads_4096x2048", 4096, 1, 2048, 16, "bf16", "silu"),
        # the first section's maps of a batch of frames
        norm("norm_maps_1024x36x48x32", 1024, 36 * 48, 32, 8, "bf16", "relu"),
        # two large maps with odd sides: few rows, long groups
        norm("norm_wide_2x135x241x320", 2, 135 * 241, 320, 32, "fp32", "silu"),
        # actions of a large batch of actors, each with its own temperature and nucleus
        sample("sample_actions_4096x18", 4096, 18, "fp32", p=0.9),
        # a few streams over a vocabulary: latency
        sample("sample_4x32000", 4, 32000, "fp32", k=50, p=0.95),
        # a serving batch over an odd vocabulary with masked entries
        sample("sample_64x50001", 64, 50001, "bf16", p=0.9, m=0.01, masked=True),
        # a large batch over a large vocabulary, every filter in use
        sample("sample_256x131072", 256, 131072, "fp32", k=1000, p=0.95, m=0.001),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["decay", "decay", "norm", "sample"])
    dtype = rng.choice(["fp32", "bf16"])
    if op == "decay":
        kv = _log(rng, 1, 8)
        heads = kv * rng.choice([1, 1, 2, 4])
        dims = lambda: rng.choice([32, 64, 64, 128, 128, 256, _log(rng, 8, 256)])  # noqa: E731
        dk, dv = dims(), dims()
        # token rows whose products and whose bytes the largest cases allow
        room = min(32768 * 16 * 128 * 128 // (heads * dk * dv), 10 ** 9 // ((heads + kv) * (dk + dv) * 2))
        if rng.random() < 0.35:
            steps, rows = 1, _log(rng, 1, min(512, max(2, 256 * 16 * 128 * 128 // (heads * dk * dv))))
        else:
            steps = _log(rng, 2, min(32768, room // 4))
            rows = _log(rng, 1, max(1, min(256, room // (4 * steps))))
        return dict(op=op, steps=steps, rows=rows, heads=heads, kv_heads=kv, key_dim=dk, value_dim=dv, dtype=dtype,
                    flags=rng.random() < 0.5, ragged=steps > 1 and rng.random() < 0.3)
    if op == "norm":
        groups = rng.choice([1, 4, 8, 16, 32, rng.randint(1, 40)])
        channels = groups * rng.choice([1, 2, 4, 8, 16, 64, 128, rng.randint(1, 64)])
        most = 2 * 135 * 241 * 320 // channels
        points = rng.choice([1 if channels > groups else 2, _log(rng, 2, min(20000, most))])
        rows = _log(rng, 1, max(1, min(8192, most // points)))
        return dict(op=op, rows=rows, points=points, channels=channels, groups=groups, dtype=dtype,
                    act=rng.choice(["none", "relu", "silu"]), affine=rng.random() < 0.7)
    choices = _log(rng, 2, 131072)
    rows = _log(rng, 1, max(1, min(4096, 256 * 131072 // choices)))
    return dict(op=op, rows=rows, choices=choices, dtype=dtype, k=rng.choice([0, 1, 50, _log(rng, 1, choices)]),
                p=rng.choice([0.0, 0.5, 0.9, 0.95]), m=rng.choice([0.0, 0.0, 0.02, 0.1]), masked=rng.random() < 0.3)


def _lengths(case):
    """The rows' lengths: fixed by the case, unequal, the longest the whole of it."""
    T, B = case["steps"], case["rows"]
    return [T - (T * b) // (2 * B) if case["ragged"] else T for b in range(B)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    randn = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)  # noqa: E731
    rand = lambda *shape: torch.rand(*shape, device="cuda", generator=gen)  # noqa: E731
    x = dict(case=case)
    if case["op"] == "decay":
        T, B, H, KV, dk, dv = (case[n] for n in ("steps", "rows", "heads", "kv_heads", "key_dim", "value_dim"))
        x.update(q=randn(T, B, H, dk).to(dtype), k=(randn(T, B, KV, dk) / math.sqrt(dk)).to(dtype), v=randn(T, B, KV, dv).to(dtype))
        # heads forget over horizons from a few steps to hundreds
        x["decay"] = 1 - 2.0 ** (-2 - 7 * (torch.arange(H, device="cuda") + rand(H)) / H)
        x["state"] = 0.5 * randn(B, H, dk, dv)
        x["scale"] = 1.0
        x["done"] = (rand(T, B) < 0.02).to(torch.uint8) if case["flags"] else None
        x["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda") if case["ragged"] else None
        # the buffers such a program keeps: the outputs, and the other half of the state's ping-pong pair
        x["out"], x["state_out"] = torch.zeros(T, B, H, dv, dtype=dtype, device="cuda"), torch.empty_like(x["state"])
        if T == 1:
            x.update({n: x[n][0] for n in ("q", "k", "v", "out")}, done=None if x["done"] is None else x["done"][0])
        return x
    if case["op"] == "norm":
        N, P, C = case["rows"], case["points"], case["channels"]
        # channels of unequal mean and spread, as behind a convolution
        x["x"] = (randn(N, P, C) * (0.5 + rand(C)) + randn(C)).to(dtype)
        x["weight"], x["bias"] = (1 + 0.2 * randn(C), 0.2 * randn(C)) if case["affine"] else (None, None)
        x["out"] = torch.empty_like(x["x"])
        return x
    R, V = case["rows"], case["choices"]
    logits = 2.5 * randn(R, V)
    if case["masked"]:
        logits.masked_fill_((rand(R, V) < 0.05) | (rand(R, 1) < 0.02), -math.inf)
    x["logits"] = logits.to(dtype)
    x["uniforms"] = rand(R)
    # temperatures around one, an eighth of the rows greedy
    x["temperature"] = torch.where(rand(R) < 0.125, 0.0, 0.6 + 0.8 * rand(R))
    x["top_k"] = torch.full((R,), case["k"], dtype=torch.int32, device="cuda") if case["k"] else None
    x["top_p"] = (case["p"] + (1 - case["p"]) * 0.5 * rand(R)) if case["p"] else None
    x["min_p"] = case["m"] * (0.5 + rand(R)) if case["m"] else None
    x["token"], x["logprob"] = torch.empty(R, dtype=torch.int32, device="cuda"), torch.empty(R, device="cuda")
    return x


def run(state):
    op = state["case"]["op"]
    if own:
        from paper_1910_06591_amd import seedinf
        if op == "decay":
            call = seedinf.decay_step if state["case"]["steps"] == 1 else seedinf.decay_attention
            more = {} if state["case"]["steps"] == 1 else {"lengths": state["lengths"]}
            return call(state["q"], state["k"], state["v"], state["decay"], state=state["state"], done=state["done"],
                        scale=state["scale"], out=state["out"], state_out=state["state_out"], **more)
        if op == "norm":
            return seedinf.group_norm(state["x"], state["case"]["groups"], state["weight"], state["bias"], eps=1e-5,
                                      activation=state["case"]["act"], out=state["out"])
        return seedinf.sample(state["logits"], state["uniforms"], temperature=state["temperature"], top_k=state["top_k"],
                              top_p=state["top_p"], min_p=state["min_p"], token=state["token"], logprob=state["logprob"])
    if op == "decay":
        return _decay_step(state) if state["case"]["steps"] == 1 else _decay(state)
    return _norm(state) if op == "norm" else _sample(state)


def _decay_step(s):
    """S' = decay S + k v^T (S = 0 on a flagged row), out = scale q^T S'."""
    groups = s["q"].shape[1] // s["k"].shape[1]
    k, v = (s[n].float().repeat_interleave(groups, 1) for n in "kv")
    S = s["state"] * s["decay"][:, None, None]
    if s["done"] is not None:
        S = S * (s["done"] == 0).float()[:, None, None, None]
    S = S + k[..., :, None] * v[..., None, :]
    out = s["scale"] * (s["q"].float()[..., :, None] * S).sum(-2)
    return out.to(s["q"].dtype), S


def _decay(s):
    """The recurrence in chunks of CHUNK steps: within a chunk the masked product (q k^T * D) v, between chunks the
    states at the chunks' borders as one weighted sum over the chunks' own contributions."""
    T, B, H, dk = s["q"].shape
    dv = s["v"].shape[-1]
    C = min(CHUNK, T)
    N = -(-T // C)
    dev, pad = s["q"].device, N * C - T
    length = s["lengths"][:, None] if s["lengths"] is not None else torch.full((B, 1), T, device=dev)
    t = torch.arange(N * C, device=dev)
    inside = t < length                                                            # [B, NC]

    def chunks(x):                                                                 # [T, B, heads, d] -> [B, H, N, C, d]
        x = torch.nn.functional.pad(x.float(), (0, 0, 0, 0, 0, 0, 0, pad)).permute(1, 2, 0, 3)
        x = (x * inside[:, None, :, None]).repeat_interleave(H // x.shape[1], 1)
        return x.reshape(B, H, N, C, x.shape[-1])

    q, k, v = chunks(s["q"]), chunks(s["k"]), chunks(s["v"])
    n = torch.minimum(t + 1, length)                                               # steps done behind step t
    seg = torch.zeros_like(n)
    if s["done"] is not None:
        seg = torch.cumsum(torch.nn.functional.pad(s["done"].t() != 0, (0, pad)) & inside, 1)
    log2 = torch.log2(s["decay"].double())[None, :, None, None]
    power = lambda steps: torch.exp2(steps * log2)  # noqa: E731
    # within a chunk
    nc, sc = n.view(B, N, C), seg.view(B, N, C)
    lower = torch.tril(torch.ones(C, C, dtype=torch.bool, device=dev))
    same = (sc[..., :, None] == sc[..., None, :]) & lower
    D = torch.where(same[:, None], power((nc[..., :, None] - nc[..., None, :]).clamp_min(0).view(B, 1, N, C * C)).view(B, H, N, C, C).float(), 0.0)
    out = ((q @ k.transpose(-1, -2).contiguous()) * D) @ v
    # what each chunk adds to the state at its end, and the state in front of every chunk and behind the last
    end, eseg = nc[..., -1], sc[..., -1]                                           # [B, N]
    w = torch.where((sc == eseg[..., None])[:, None], power((end[..., None] - nc).view(B, 1, N, C)).float(), 0.0)
    add = ((k * w[..., None]).transpose(-1, -2).contiguous() @ v).reshape(B, H, N, dk * dv)
    zero = torch.zeros(B, 1, dtype=n.dtype, device=dev)
    at, aseg = torch.cat([zero, end], 1), torch.cat([zero, eseg], 1)               # [B, N + 1]
    before = (torch.arange(N + 1, device=dev)[:, None] > torch.arange(N, device=dev)) & (aseg[:, :, None] == eseg[:, None, :])
    W = torch.where(before[:, None], power((at[:, :, None] - end[:, None, :]).clamp_min(0)[:, None]).float(), 0.0)
    first = torch.where((aseg == 0)[:, None], power(at[:, None, :, None])[..., 0].float(), 0.0)
    S = W @ add + first[..., None] * s["state"].reshape(B, H, 1, dk * dv)
    S = S.view(B, H, N + 1, dk, dv)
    reach = torch.where((sc == aseg[:, :-1, None])[:, None], power((nc - at[:, :-1, None]).view(B, 1, N, C)).float(), 0.0)
    out = s["scale"] * (out + reach[..., None] * (q @ S[:, :, :-1]))
    out = out.reshape(B, H, N * C, dv)[:, :, :T].permute(2, 0, 1, 3) * inside[:, :T].t()[:, :, None, None]
    return out.to(s["q"].dtype).contiguous(), S[:, :, -1].contiguous()


def _norm(s):
    """y = act((x - mean) / sqrt(var + eps) * weight + bias), mean and variance over a row's points and a group's channels."""
    N, P, C = s["x"].shape
    x = s["x"].float().view(N, P, s["case"]["groups"], -1)
    x = x - x.mean((1, 3), keepdim=True)
    y = (x * torch.rsqrt(x.square().mean((1, 3), keepdim=True) + 1e-5)).view(N, P, C)
    if s["weight"] is not None:
        y = y * s["weight"] + s["bias"]
    if s["case"]["act"] != "none":
        y = torch.relu(y) if s["case"]["act"] == "relu" else y / (1 + torch.exp(-y))
    return y.to(s["x"].dtype)


def _sample(s):
    """The choices in the order (logit descending, index ascending).  Kept is a prefix: at most top_k of them, the
    shortest prefix that holds top_p of the top-k choices' mass, and only those with at least min_p of the largest
    one's probability.  The choice is the first in that order whose running sum of kept probabilities exceeds the
    uniform; a row without any has the choice -1."""
    x = s["logits"].double()
    V = x.shape[1]
    greedy = ~(s["temperature"] > 0)[:, None]
    top = x.amax(1, keepdim=True)
    empty = top == -math.inf
    z = torch.where(empty, -math.inf, x - top) / torch.where(greedy, 1.0, s["temperature"][:, None].double())
    order, index = torch.sort(x, dim=1, descending=True, stable=True)
    mass = torch.exp(torch.gather(z, 1, index))
    rank = torch.arange(V, device=x.device)
    most = torch.where(greedy, 1, V)
    if s["top_k"] is not None:
        k = s["top_k"][:, None]
        most = torch.where((k > 0) & (k < most), k, most)
    keep = rank < most
    if s["top_p"] is not None:
        p = s["top_p"][:, None].double()
        held = mass * keep
        before = torch.cumsum(held, 1) - held
        keep = keep & ((before < p * held.sum(1, keepdim=True)) | (p >= 1) | (rank == 0))
    if s["min_p"] is not None:
        keep = keep & (mass >= s["min_p"][:, None].double())
    kept = mass * keep
    run = torch.cumsum(kept, 1)
    total = run[:, -1:]
    at = (run <= s["uniforms"][:, None].double() * total).sum(1, keepdim=True).clamp_max(V - 1)
    token = torch.gather(index, 1, at)
    logprob = torch.where(empty, -math.inf, torch.log(torch.gather(kept, 1, at) / total))
    return torch.where(empty, -1, token)[:, 0].to(torch.int32), logprob[:, 0].float()


def work(case):
    """Bytes: every input once, every output once (the states in fp32, in and out).  Flops: what the recurrence, the
    normalisation or one exponential a choice needs."""
    size = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "decay":
        B, H, KV, dk, dv = (case[n] for n in ("rows", "heads", "kv_heads", "key_dim", "value_dim"))
        tokens = sum(_lengths(case))
        rows = tokens * (H * (dk + dv) + KV * (dk + dv)) * size
        return {"bytes": rows + 2 * 4 * B * H * dk * dv + (case["steps"] * B if case["flags"] else 0), "flops": 4.0 * tokens * H * dk * dv}
    if case["op"] == "norm":
        n = case["rows"] * case["points"] * case["channels"]
        return {"bytes": 2 * n * size, "flops": 8.0 * n}
    n = case["rows"] * case["choices"]
    return {"bytes": n * size + 24 * case["rows"], "flops": 4.0 * n}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "decay":
        return _exact_decay(case, s)
    if case["op"] == "norm":
        x = s["x"].double().view(case["rows"], case["points"], case["groups"], -1)
        var, mean = torch.var_mean(x, dim=(1, 3), correction=0, keepdim=True)
        y = ((x - mean) / (var + 1e-5).sqrt()).view(case["rows"], case["points"], case["channels"])
        if s["weight"] is not None:
            y = torch.addcmul(s["bias"].double(), y, s["weight"].double())
        return {"none": lambda v: v, "relu": lambda v: v.clamp_min(0), "silu": lambda v: v * torch.sigmoid(v)}[case["act"]](y)
    return _exact_sample(s)


def _exact_decay(case, s):
    """Step by step."""
    T, group = case["steps"], case["heads"] // case["kv_heads"]
    S, decay = s["state"].double(), s["decay"].double()[:, None, None]
    step = T == 1
    lengths = _lengths(case)
    q, k, v = (s[n][None] if step else s[n] for n in "qkv")
    done = s["done"][None] if step and s["done"] is not None else s["done"]
    out = torch.zeros(T, case["rows"], case["heads"], case["value_dim"], dtype=torch.float64, device=q.device)
    for t in range(T):
        n = sum(t < m for m in lengths)                                  # the lengths descend: the first n rows are alive
        live = S[:n] * decay
        if done is not None:
            live = live * (done[t, :n] == 0).double()[:, None, None, None]
        kt, vt = (a[t, :n].double().repeat_interleave(group, 1) for a in (k, v))
        live = live + kt[..., None] * vt[..., None, :]
        out[t, :n] = s["scale"] * torch.matmul(q[t, :n].double()[..., None, :], live)[..., 0, :]
        S = live if n == len(lengths) else torch.cat([live, S[n:]])
    return (out[0] if step else out), S


def _exact_sample(s):
    """Row by row on the host."""
    import numpy as np
    host = lambda n: None if s[n] is None else s[n].cpu().double().numpy()  # noqa: E731
    logits, u, temp, top_k, top_p, min_p = (host(n) for n in ("logits", "uniforms", "temperature", "top_k", "top_p", "min_p"))
    tokens, logprobs = [], []
    for r, row in enumerate(logits):
        if row.max() == -math.inf:
            tokens.append(-1)
            logprobs.append(-math.inf)
            continue
        if not temp[r] > 0:
            tokens.append(int(np.argmax(row)))
            logprobs.append(0.0)
            continue
        prob = np.exp((row - row.max()) / temp[r])
        order = np.lexsort((np.arange(row.size), -row))
        if top_k is not None and 0 < top_k[r] < row.size:
            order = order[: int(top_k[r])]
        sums = np.cumsum(prob[order])
        most = order.size
        if top_p is not None and top_p[r] < 1:
            most = 1 + int(np.searchsorted(sums[:-1], top_p[r] * sums[-1], side="left"))
        if min_p is not None:
            most = max(1, min(most, int(np.count_nonzero(prob[order] >= min_p[r]))))
        kept = order[:most]
        sums = np.cumsum(prob[kept])
        at = min(int(np.searchsorted(sums, u[r] * sums[-1], side="right")), kept.size - 1)
        tokens.append(int(kept[at]))
        logprobs.append(float(np.log(prob[kept[at]] / sums[-1])))
    return torch.tensor(tokens, dtype=torch.int32), torch.tensor(logprobs, dtype=torch.float64)
