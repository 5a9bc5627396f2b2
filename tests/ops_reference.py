"""Plain 64-bit forms of the stand-alone operators, and how far a result may be from them.

A rounding to a type is off by at most half a step, u = finfo.eps / 2 of the value: 2^-24 in fp32, 2^-8 in bf16."""
import numpy as np

U32, UBF = 2.0 ** -24, 2.0 ** -8


def decay(q, k, v, g, state=None, done=None, lengths=None, scale=1.0):
    """Step by step.  q [T, B, H, dk], k, v [T, B, KV, .]; returns out, state, and the same with every term's absolute
    value (what the roundings of sums are relative to).  out is NaN behind a row's length."""
    q, k, v, g = (np.asarray(x, np.float64) for x in (q, k, v, g))
    T, B, H, dk = q.shape
    dv, grp = v.shape[3], H // k.shape[2]
    k, v = np.repeat(k, grp, 2), np.repeat(v, grp, 2)
    S = np.zeros((B, H, dk, dv)) if state is None else np.array(state, np.float64)
    A = np.abs(S)
    out, mag = np.full((T, B, H, dv), np.nan), np.full((T, B, H, dv), np.nan)
    for b in range(B):
        for t in range(T if lengths is None else min(max(int(lengths[b]), 0), T)):
            if done is not None and done[t, b]:
                S[b], A[b] = 0.0, 0.0
            kv = k[t, b][:, :, None] * v[t, b][:, None, :]
            S[b] = g[:, None, None] * S[b] + kv
            A[b] = np.abs(g)[:, None, None] * A[b] + np.abs(kv)
            out[t, b] = scale * np.einsum("hk,hkv->hv", q[t, b], S[b])
            mag[t, b] = abs(scale) * np.einsum("hk,hkv->hv", np.abs(q[t, b]), A[b])
    return out, S, mag, A


def decay_tolerance(out, mag, S, A, steps, key_dim, bf16):
    """A sum of n fp32 terms is off by at most n u of the sum of their absolute values; a step's term passes `steps`
    additions and multiplications by powers on its way into the state (each power is rounded once more), key_dim more
    into an output, and as many again where scores are summed first.  In bf16 the scores and the state take part as a
    pair of bf16 numbers, whose second is rounded to u u of the value (2^-16 each), and the output is rounded to bf16."""
    n = 2 * steps + 2 * key_dim + 16
    tol_s = (2 * steps + 16) * U32 * A + 1e-37
    tol_o = n * U32 * mag + 1e-37
    if bf16:
        tol_o = tol_o + 2 * UBF * UBF * mag + UBF * np.abs(out)
    return tol_o, tol_s


def group_norm(x, groups, weight=None, bias=None, eps=1e-5, activation="none"):
    """x [N, P, C].  Returns y and the tolerance's magnitude."""
    x = np.asarray(x, np.float64)
    N, P, C = x.shape
    xg = x.reshape(N, P, groups, C // groups)
    mean, var = xg.mean((1, 3), keepdims=True), xg.var((1, 3), keepdims=True)
    rstd = 1 / np.sqrt(var + eps)
    y = ((xg - mean) * rstd).reshape(N, P, C)
    mag = (np.abs(xg).max((1, 3), keepdims=True) * rstd + np.abs((xg - mean) * rstd)).reshape(N, P, C)
    if weight is not None:
        y, mag = y * weight, mag * np.abs(weight)
    if bias is not None:
        y, mag = y + bias, mag + np.abs(bias)
    if activation == "relu":
        y = np.maximum(y, 0)
    elif activation == "silu":
        with np.errstate(over="ignore"):
            y = y / (1 + np.exp(-y))
    return y, mag


def group_norm_tolerance(y, mag, bf16):
    """The mean is off by a few u of the largest |x|, so is every difference to it; the deviation's error is a few u of
    the result (a blocked or shifted sum: its length enters by its logarithm, 32 u are allowed for both); the
    exponential of the activation is good to a few u of its value and of its argument (|y| <= 20 here)."""
    tol = 64 * U32 * mag + 1e-37
    return tol + UBF * np.abs(y) if bf16 else tol


def sample(logits, uniforms, temperature=None, top_k=None, top_p=None, min_p=None):
    """Row by row over the sorted order."""
    logits = np.asarray(logits, np.float64)
    R, V = logits.shape
    tokens, logprobs = np.empty(R, np.int32), np.empty(R)
    for r in range(R):
        x = np.where(np.isnan(logits[r]), -np.inf, logits[r])
        order = np.lexsort((np.arange(V), -x))
        top = x[order[0]]
        if top == -np.inf:
            tokens[r], logprobs[r] = -1, -np.inf
            continue
        temp = 1.0 if temperature is None else float(temperature[r])
        if not temp > 0:
            tokens[r], logprobs[r] = order[0], 0.0
            continue
        z = np.full(V, -np.inf)
        z[x == top] = 0.0
        some = (x != top) & (x != -np.inf)
        z[some] = (x[some] - top) / temp
        m = np.exp(z[order])
        n = V
        if top_k is not None and 0 < top_k[r] < V:
            n = int(top_k[r])
        cum = np.cumsum(m)
        if top_p is not None and top_p[r] < 1:
            n = max(1, min(n, 1 + int(np.count_nonzero(cum[:n - 1] < float(top_p[r]) * cum[n - 1]))))
        if min_p is not None and min_p[r] > 0:
            n = max(1, min(n, int(np.count_nonzero(m >= float(min_p[r])))))
        u = float(uniforms[r])
        u = 0.0 if not u > 0 else min(u, 1 - 2.0 ** -24)
        at = min(int(np.count_nonzero(cum[:n] <= u * cum[n - 1])), n - 1)
        tokens[r], logprobs[r] = order[at], z[order[at]] - np.log(cum[n - 1])
    return tokens, logprobs
