"""Host-only checks of the stand-alone operators' C entry points: exports, sizes of the structs, and every refusal that
is made before anything is enqueued (no device is touched: the pointers are never read)."""
import ctypes as C
import os
import re

import pytest

from paper_1910_06591_amd import seedinf

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, ALIASING = 1, 4
A = 1 << 20                                            # an address: 16-byte aligned, never read


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(seedinf.LIB_PATH):
        seedinf.build_library()
    return seedinf.load_library()


def test_operator_exports_match_header(lib):
    hdr = open(os.path.join(ROOT, "include", "seedinf.h")).read()
    declared = set(re.findall(r"\b(seed_op_[a-z_]+)\s*\(", hdr))
    assert declared == set(seedinf.OP_EXPORTS)
    for name in declared:
        assert getattr(lib, name) is not None


def test_struct_sizes():
    assert C.sizeof(seedinf.SeedDecay) == 4 * 9 + 4 + 8 * 8
    assert C.sizeof(seedinf.SeedStepExt) == 8 * 9
    assert seedinf.SeedStepExt.sample_uniforms.offset == 32


def decay_desc(**kw):
    d = dict(dtype=0, steps=3, rows=2, heads=4, kv_heads=2, key_dim=8, value_dim=16, scale=1.0)
    d.update({k: v for k, v in kw.items() if k in d})
    row_q, row_k, row_v, row_o = d["heads"] * d["key_dim"], d["kv_heads"] * d["key_dim"], d["kv_heads"] * d["value_dim"], d["heads"] * d["value_dim"]
    s = dict(q_step=2 * row_q, q_row=row_q, k_step=2 * row_k, k_row=row_k, v_step=2 * row_v, v_row=row_v, out_step=2 * row_o, out_row=row_o)
    s.update({k: v for k, v in kw.items() if k in s})
    return seedinf.SeedDecay(kw.get("struct_size", C.sizeof(seedinf.SeedDecay)), *d.values(), *s.values())


def decay_call(lib, desc, q=A, k=2 * A, v=3 * A, decay=4 * A, done=None, lengths=None, state=5 * A, out=6 * A, state_out=7 * A, ws=None, n=0):
    st = lib.seed_op_decay(C.byref(desc) if desc is not None else None, q, k, v, decay, done, lengths, state, out, state_out, ws, n, None)
    return st, lib.seed_op_last_error().decode()


@pytest.mark.parametrize("kw,text", [
    (dict(struct_size=8), "struct_size"), (dict(dtype=2), "dtype"), (dict(steps=-1), "steps"), (dict(rows=-1), "rows"),
    (dict(heads=0), "heads"), (dict(kv_heads=0), "kv_heads"), (dict(kv_heads=3), "kv_heads"), (dict(key_dim=0), "key_dim"),
    (dict(key_dim=257), "key_dim"), (dict(value_dim=257), "value_dim"), (dict(q_row=-1), "stride"), (dict(out_step=1 << 50), "stride"),
    (dict(rows=1 << 20), "rows"),
])
def test_decay_refuses_bad_fields(lib, kw, text):
    st, msg = decay_call(lib, decay_desc(**kw))
    assert st == INVALID and text in msg
    assert lib.seed_op_decay_workspace(C.byref(decay_desc(**kw))) == 0


def test_decay_refuses_bad_pointers(lib):
    assert decay_call(lib, None)[0] == INVALID
    assert lib.seed_op_decay_workspace(None) == 0
    for name in ("q", "k", "v", "decay", "out", "state_out"):
        st, msg = decay_call(lib, decay_desc(), **{name: None})
        assert st == INVALID and "required" in msg, name
    for name in ("q", "k", "v", "state", "out", "state_out"):
        st, msg = decay_call(lib, decay_desc(), **{name: A + 2})
        assert st == INVALID and "aligned" in msg, name
    assert decay_call(lib, decay_desc(rows=0), q=None, out=None, state_out=None)[0] == 0       # nothing to do


def test_decay_refuses_overlaps(lib):
    desc = decay_desc()
    for kw in (dict(state_out=5 * A + 16), dict(out=A), dict(out=2 * A), dict(out=3 * A + 4), dict(state_out=A + 16), dict(state_out=6 * A)):
        st, msg = decay_call(lib, desc, **kw)
        assert st == ALIASING and "overlap" in msg, kw
    assert decay_call(lib, decay_desc(out_row=16))[0] == ALIASING                     # out's own rows
    # out as the fourth part of one buffer [steps, rows, q | k | v | out] is no overlap, one element further left is
    row = 32 + 16 + 32 + 64
    part = dict(q_step=2 * row, q_row=row, k_step=2 * row, k_row=row, v_step=2 * row, v_row=row, out_step=2 * row, out_row=row)
    at = dict(q=A, k=A + 4 * 32, v=A + 4 * 48)
    st, msg = decay_call(lib, decay_desc(**part), **at, out=A + 4 * 79)
    assert st == ALIASING, msg
    st, msg = decay_call(lib, decay_desc(**part), **at, out=A + 4 * 80, decay=None)
    assert st == INVALID and "required" in msg                                        # (checked before, so nothing runs)


@pytest.mark.parametrize("kw,text", [
    (dict(dtype=3), "dtype"), (dict(rows=-1), "rows"), (dict(points=-2), "points"), (dict(channels=0), "groups"),
    (dict(groups=0), "groups"), (dict(groups=3), "groups"), (dict(points=1 << 30), "points"), (dict(rows=1 << 23), "rows"),
    (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(act=3), "activation"), (dict(x=None), "required"), (dict(out=None), "required"),
    (dict(x=A + 2), "aligned"), (dict(weight=A + 1), "aligned"),
])
def test_group_norm_refuses(lib, kw, text):
    a = dict(dtype=0, rows=2, points=3, channels=8, groups=2, x=A, weight=3 * A, bias=4 * A, eps=1e-5, act=1, out=2 * A, ws=None, n=0)
    a.update(kw)
    assert lib.seed_op_group_norm(*a.values(), None) == INVALID
    assert text in lib.seed_op_last_error().decode()


def test_group_norm_refuses_overlaps(lib):
    a = dict(dtype=0, rows=2, points=3, channels=8, groups=2, x=A, weight=3 * A, bias=4 * A, eps=1e-5, act=1, out=2 * A, ws=None, n=0)
    for kw in (dict(out=A + 16), dict(weight=2 * A), dict(bias=2 * A + 64)):
        assert lib.seed_op_group_norm(*dict(a, **kw).values(), None) == ALIASING, kw
    assert lib.seed_op_group_norm(*dict(a, rows=0, x=None, out=None).values(), None) == 0
    assert lib.seed_op_group_norm(*dict(a, points=0, x=None, out=None).values(), None) == 0


SAMPLE = dict(dtype=0, rows=2, choices=10, stride=10, logits=A, uniforms=2 * A, temperature=None, top_k=None, top_p=None, min_p=None,
              token=3 * A, logprob=4 * A, ws=None, n=0)


@pytest.mark.parametrize("kw,text", [
    (dict(dtype=-1), "dtype"), (dict(rows=-1), "rows"), (dict(rows=(1 << 21) + 1), "rows"), (dict(choices=0), "choices"),
    (dict(choices=(1 << 24) + 1), "choices"), (dict(stride=-1), "row_stride"), (dict(logits=None), "required"), (dict(uniforms=None), "required"),
    (dict(token=None), "required"), (dict(logits=A + 1), "aligned"), (dict(top_k=A + 2), "aligned"), (dict(token=A + 2), "aligned"),
])
def test_sample_refuses(lib, kw, text):
    assert lib.seed_op_sample(*dict(SAMPLE, **kw).values(), None) == INVALID
    assert text in lib.seed_op_last_error().decode()


def test_sample_refuses_overlaps(lib):
    for kw in (dict(token=A + 4), dict(logprob=A + 64), dict(token=4 * A), dict(top_p=3 * A), dict(uniforms=4 * A)):
        assert lib.seed_op_sample(*dict(SAMPLE, **kw).values(), None) == ALIASING, kw
    assert lib.seed_op_sample(*dict(SAMPLE, rows=0, logits=None, token=None).values(), None) == 0


def test_binding_refuses_host_tensors():
    import torch
    x = torch.zeros(2, 3)
    with pytest.raises(TypeError):
        seedinf.sample(x, torch.zeros(2))
    with pytest.raises(TypeError):
        seedinf.group_norm(x, 1)
    with pytest.raises(TypeError):
        seedinf.decay_attention(x, x, x, x)


@pytest.mark.parametrize("kw", [dict(out=5 * A), dict(out=4 * A), dict(done=6 * A), dict(lengths=6 * A + 64), dict(lengths=7 * A), dict(decay=7 * A + 16), dict(done=7 * A)])
def test_decay_refuses_outputs_over_small_inputs(lib, kw):
    st, msg = decay_call(lib, decay_desc(), **kw)
    assert st == ALIASING and "overlap" in msg
    for name in ("decay", "lengths"):
        st, msg = decay_call(lib, decay_desc(), **{name: A + 2})
        assert st == INVALID and "aligned" in msg, name


@pytest.mark.parametrize("step,row,ok", [(128, 64, True), (64, 4096 * 64, True), (200, 65, True), (64, 64, False), (96, 64, False), (64, 4096 * 64 - 1, False),
                                         (63, 1 << 20, False), (0, 64, False), (127, 64, False)])
def test_decay_refuses_outputs_whose_rows_meet(lib, step, row, ok):
    """4096 steps of 2 rows of 64 elements: which strides keep them apart (accepted ones are refused for the missing workspace, so nothing runs)."""
    desc = decay_desc(steps=4096, rows=2, heads=1, kv_heads=1, key_dim=64, value_dim=64, out_step=step, out_row=row)
    st, msg = decay_call(lib, desc, **FAR)
    assert (st == INVALID and "workspace" in msg) if ok else (st == ALIASING and "rows overlap" in msg)


FAR = dict(q=1 << 30, k=2 << 30, v=3 << 30, out=4 << 30, state=5 << 30, state_out=6 << 30)


def test_workspaces_must_not_overlap(lib):
    desc = decay_desc(steps=4096, rows=1, heads=1, kv_heads=1, key_dim=64, value_dim=64)
    n = lib.seed_op_decay_workspace(C.byref(desc))
    assert n > 0
    far = FAR
    for name, at in far.items():
        st, msg = decay_call(lib, desc, **far, ws=at, n=n)
        assert st == ALIASING and "workspace" in msg, name
    st, msg = decay_call(lib, desc, **far, ws=7 << 30, n=n - 1)
    assert st == INVALID and "workspace" in msg
    sizes = dict(dtype=0, rows=1, points=100000, channels=32, groups=4)
    n = lib.seed_op_group_norm_workspace(*sizes.values())
    assert n > 0
    a = dict(sizes, x=1 << 30, weight=2 << 30, bias=3 << 30, eps=1e-5, act=0, out=4 << 30, ws=None, n=n)
    for name in ("x", "weight", "bias", "out"):
        assert lib.seed_op_group_norm(*dict(a, ws=a[name]).values(), None) == ALIASING, name
    assert lib.seed_op_group_norm(*a.values(), None) == INVALID


def test_the_longest_group_norm_row_is_split(lib):
    """2^31 - 1 points of one channel: rounds past the last point do not wrap."""
    assert lib.seed_op_group_norm_workspace(1, 1, (1 << 31) - 1, 1, 1) > 0


@pytest.mark.parametrize("dtype,channels,groups", [(0, 1028, 1), (0, 2048, 1), (1, 4096, 1), (0, 333, 1), (1, 511, 1)])
def test_group_norm_splits_rows_of_wide_slices(lib, dtype, channels, groups):
    """As many vectors as the splitting kernel has threads, 512: it takes them, and needs a workspace for its statistics."""
    assert lib.seed_op_group_norm_workspace(dtype, 2, 5000, channels, groups) > 0


@pytest.mark.parametrize("steps", [(1 << 31) - 1, (1 << 31) - (1 << 22) + 1, 1 << 30])
def test_the_longest_axis_is_split(lib, steps):
    """512 segments of a state of one number and a pair of factors, whatever is added to the steps to round them up."""
    n = lib.seed_op_decay_workspace(C.byref(decay_desc(steps=steps, rows=1, heads=1, kv_heads=1, key_dim=1, value_dim=1)))
    assert 512 * 8 <= n <= 512 * 12 + 256


@pytest.mark.parametrize("name", ["decay", "done", "lengths"])
def test_decay_workspace_must_not_overlap_small_inputs(lib, name):
    desc = decay_desc(steps=4096, rows=1, heads=1, kv_heads=1, key_dim=64, value_dim=64)
    n = lib.seed_op_decay_workspace(C.byref(desc))
    st, msg = decay_call(lib, desc, **dict(FAR, **{name: 7 << 30}), ws=7 << 30, n=n)
    assert st == ALIASING and "workspace" in msg


@pytest.mark.parametrize("kw", [dict(steps=(1 << 21) + 1, q_step=1 << 43), dict(steps=1 << 30, v_step=1 << 40), dict(steps=1 << 30, out_step=1 << 34), dict(rows=1 << 19, k_row=1 << 44)])
def test_decay_refuses_strides_that_leave_64_bits(lib, kw):
    """Each stride is one that is allowed; the last step or row would lie further on than an address reaches."""
    st, msg = decay_call(lib, decay_desc(**dict(dict(heads=1, kv_heads=1), **kw)), **FAR)
    assert st == INVALID and "stride" in msg


def test_sample_refuses_strides_that_leave_64_bits(lib):
    assert lib.seed_op_sample(*dict(SAMPLE, rows=1 << 21, stride=1 << 44).values(), None) == INVALID
    assert "row_stride" in lib.seed_op_last_error().decode()
