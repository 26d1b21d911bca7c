"""Linear attention with a decay per head: argument checks (CPU) and parity with 64-bit references (GPU).

Tolerances: see dla_reference.near (half a step of the storage type plus float32 sums)."""
import ctypes
import math
import os
import shutil

import pytest


@pytest.fixture(scope="module")
def sdm():
    import paper_2607_07386_gb300 as sdm
    from paper_2607_07386_gb300 import build as B
    if not os.path.exists(sdm.lib_path()):
        if shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"):
            pytest.skip("nvcc not available to build libsdm.so")
        B.build()
    return sdm


# ------------------------------------------------------------------ refusals (nothing is launched)
def _shape(sdm, **kw):
    base = dict(B=2, H=4, T=16, d_k=32, d_v=64, H_k=2, dtype="bf16")
    base.update(kw)
    return sdm.DlaShape.make(**base)


A = 1 << 20      # fake, aligned, far apart device addresses: validation never reads them


def _forward(sdm, shape, **kw):
    p = dict(q=A, k=2 * A, v=3 * A, log_decay=5 * A, state=6 * A, y=7 * A, workspace=64 * A, workspace_nbytes=1 << 40)
    p.update(kw)
    sdm.dla_forward(shape, stream=0, **p)


def test_struct_layout(sdm):
    assert ctypes.sizeof(sdm.DlaShape) == 36 and sdm.DlaShape.scale.offset == 32 and sdm.DlaShape.layout.offset == 28
    assert isinstance(_shape(sdm), sdm.DlaShape) and _shape(sdm).replace(T=5).T == 5


@pytest.mark.parametrize("kw,status", [
    (dict(B=-1), 1), (dict(T=-5), 1), (dict(H=5), 1), (dict(H_k=0), 1), (dict(dtype=7), 1), (dict(layout=2), 1),
    (dict(d_k=0), 1), (dict(d_k=264), 2), (dict(d_v=264), 2), (dict(d_k=12), 2), (dict(d_v=20), 2), (dict(d_k=6, dtype="f32"), 2),
    (dict(B=70000), 2), (dict(B=60000, H=60000, T=1 << 20), 2), (dict(scale=math.inf), 1), (dict(scale=math.nan), 1)])
def test_refused_shapes(sdm, kw, status):
    shape = _shape(sdm, **kw)
    for call in (lambda: _forward(sdm, shape), lambda: sdm.dla_workspace_bytes(shape),
                 lambda: sdm.dla_backward_workspace_bytes(shape)):
        with pytest.raises(sdm.SdmError) as e:
            call()
        assert str(e.value)
    with pytest.raises(sdm.SdmError) as e:
        _forward(sdm, shape)
    assert e.value.status == status


@pytest.mark.parametrize("kw,word", [
    (dict(q=None), "q is NULL"), (dict(state=None), "state is NULL"), (dict(log_decay=None), "log_decay is NULL"),
    (dict(v=3 * A + 8), "v is not 16-byte aligned"), (dict(log_decay=5 * A + 2), "log_decay is not 4-byte aligned"),
    (dict(lengths=9 * A + 2), "lengths is not 4-byte aligned"), (dict(y=3 * A), "y overlaps v"),
    (dict(state=2 * A), "state overlaps k"), (dict(y=6 * A), "overlaps")])
def test_refused_buffers(sdm, kw, word):
    with pytest.raises(sdm.SdmError) as e:
        _forward(sdm, _shape(sdm), **kw)
    assert e.value.status == 1 and word in str(e.value)


def test_step_refusals(sdm):
    args = dict(q=A, k=2 * A, v=3 * A, log_decay=5 * A, state=6 * A, y=7 * A, stream=0)
    with pytest.raises(sdm.SdmError, match="T == 1"):
        sdm.dla_step(_shape(sdm), n_slots=2, **args)
    with pytest.raises(sdm.SdmError, match="n_slots"):
        sdm.dla_step(_shape(sdm, T=1), n_slots=1, **args)
    with pytest.raises(sdm.SdmError, match="n_slots"):
        sdm.dla_step(_shape(sdm, T=1), n_slots=-1, slots=8 * A, **args)


def test_backward_refusals(sdm):
    shape = _shape(sdm)
    names = ("q", "k", "v", "log_decay", "state0", "dy", "dstate", "dq", "dk", "dv", "dstate0")
    base = {n: (i + 1) * A for i, n in enumerate(names)}
    need = sdm.dla_backward_workspace_bytes(shape)
    assert need > 0                                          # shares of the key heads' gradients

    def call(nb=need, ws=64 * A, **kw):
        sdm.dla_backward(shape, workspace=ws, workspace_nbytes=nb, stream=0, **{**base, **kw})

    for kw, word in ((dict(nb=need - 1), "workspace too small"), (dict(ws=64 * A + 16), "256-byte aligned"),
                     (dict(ws=None), "workspace is NULL"), (dict(dq=base["q"]), "dq overlaps q"),
                     (dict(dk=base["dq"]), "overlaps"), (dict(dy=None), "dy is NULL"), (dict(dv=None), "dv is NULL"),
                     (dict(dstate0=base["state0"]), "dstate0 overlaps state0")):
        with pytest.raises(sdm.SdmError) as e:
            call(**kw)
        assert e.value.status == 1 and word in str(e.value)


def test_empty_calls_do_nothing(sdm):
    _forward(sdm, _shape(sdm, T=0))
    _forward(sdm, _shape(sdm, B=0))
    sdm.dla_step(_shape(sdm, T=1, B=0), None, None, None, None, None, None, n_slots=0, stream=0)


@pytest.mark.parametrize("kw", [dict(H=0, H_k=0), dict(H=0, H_k=3), dict(B=0), dict(H=0, H_k=-1, T=0), dict(H=0, H_k=0, d_k=256, d_v=256, T=9000)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_empty_shapes_have_empty_workspaces(sdm, kw, dtype):
    """No sequences or no heads: no bytes, no error, and the calls return."""
    shape = _shape(sdm, dtype=dtype, **kw)
    assert sdm.dla_workspace_bytes(shape) == 0 and sdm.dla_backward_workspace_bytes(shape) == 0
    _forward(sdm, shape, workspace=None, workspace_nbytes=0)
    sdm.dla_backward(shape, *[None] * 11, stream=0)


def test_plan_and_wait_hook_refusals(sdm):
    """sdm_dla_plan is host-only; the hook takes shapes with cut chains and limits from 1 on alone."""
    cut, whole = _shape(sdm, B=10, H=16, H_k=16, T=1000, d_k=64, d_v=128), _shape(sdm)
    assert sdm.dla_plan(cut)["cuts"] > 0 and sdm.dla_plan(whole)["cuts"] == 0
    assert set(sdm.dla_plan(cut, backward=True)) == set(sdm.DLA_PLAN_FIELDS)
    arr = (ctypes.c_int32 * 8)()
    assert sdm.lib().sdm_dla_plan(ctypes.byref(cut), 0, arr, 5) == 1 and "[0, 4]" in sdm.last_error()
    assert sdm.lib().sdm_dla_plan(ctypes.byref(_shape(sdm, T=-1)), 0, arr, 4) == 1
    args = [A, 2 * A, 3 * A, 5 * A, None, 6 * A, 7 * A, 64 * A, 1 << 40]
    for shape, polls, status, word in ((whole, 10, 2, "no chain"), (cut, 0, 1, "wait_polls"), (cut, (1 << 24) + 1, 1, "wait_polls")):
        assert sdm.lib().sdm_test_dla_wait_timeout(ctypes.byref(shape), *args, polls, None) == status and word in sdm.last_error()


# ------------------------------------------------------------------ parity
def _inputs(B, H, Hk, T, dk, dv, dtype, token_major=False, seed=0, device="cuda"):
    import torch
    g = torch.Generator(device=device).manual_seed(seed)
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]

    def rand(*s):
        return torch.randn(s, generator=g, device=device)

    def order(x):
        return x.transpose(1, 2).contiguous() if token_major else x

    q, k = (order((x / x.norm(dim=-1, keepdim=True)).to(dt)) for x in (rand(B, Hk, T, dk), rand(B, Hk, T, dk)))
    s = dict(q=q, k=k, v=order(rand(B, H, T, dv).to(dt)), state=rand(B, H, dk, dv) * 0.3)
    s["log_decay"] = -torch.exp2(-1 - 9 * torch.arange(H, device=device) / max(1, H - 1)).float()
    s["dy"], s["dstate"] = order(rand(B, H, T, dv).to(dt)), rand(B, H, dk, dv) * 0.3
    return s


def _ws(n):
    import torch
    return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") if n else None      # whatever it holds must not matter


def run_forward(sdm, s, shape, lengths=None, **kw):
    import torch
    y, state = torch.full_like(s["v"], math.nan), s["state"].clone()
    sdm.dla_forward(shape, s["q"], s["k"], s["v"], s["log_decay"], state, y, _ws(sdm.dla_workspace_bytes(shape)), lengths=lengths, **kw)
    return y, state


def run_backward(sdm, s, shape, lengths=None, dstate="dstate", **kw):
    import torch
    out = [torch.full_like(s[n], math.nan) for n in ("q", "k", "v", "state")]
    sdm.dla_backward(shape, s["q"], s["k"], s["v"], s["log_decay"], s["state"], s["dy"], s.get(dstate), *out,
                     _ws(sdm.dla_backward_workspace_bytes(shape)), lengths=lengths, **kw)
    return out


CASES = [  # B, H, Hk, T, dk, dv, dtype, layout, lengths
    (1, 1, 1, 1, 32, 32, "f32", "head_major", None),
    (2, 3, 1, 31, 20, 36, "f32", "token_major", None),
    (3, 4, 2, 33, 64, 96, "f32", "head_major", [33, 0, 32]),
    (2, 2, 2, 200, 256, 40, "f32", "head_major", [200, 65]),
    (1, 2, 1, 129, 128, 256, "f32", "token_major", None),
    (1, 1, 1, 1, 128, 128, "bf16", "head_major", None),
    (2, 4, 2, 17, 64, 64, "bf16", "token_major", [17, 1]),
    (2, 2, 1, 64, 128, 128, "bf16", "head_major", None),
    (3, 4, 2, 65, 128, 128, "bf16", "token_major", [65, 64, 1]),
    (4, 2, 2, 320, 64, 128, "bf16", "head_major", [320, 0, 63, 257]),
    (2, 6, 3, 191, 96, 40, "bf16", "token_major", [100, 191]),
    (1, 2, 2, 130, 128, 256, "bf16", "head_major", None),
    (1, 2, 2, 130, 256, 128, "bf16", "head_major", None),
    (1, 2, 1, 1031, 128, 128, "bf16", "token_major", None),
    (2, 1, 1, 777, 8, 8, "bf16", "head_major", [777, 129]),
    (1, 3, 1, 500, 32, 192, "bf16", "head_major", None),
    (2, 20, 20, 150, 160, 32, "bf16", "token_major", None),
    # few chains: the tokens in pieces, some past a sequence's end
    (3, 2, 1, 1100, 128, 128, "bf16", "token_major", [1100, 0, 513]),
    (1, 1, 1, 3000, 64, 64, "bf16", "head_major", None),
    (2, 1, 1, 900, 96, 200, "bf16", "head_major", [300, 897]),
    (1, 1, 1, 700, 40, 64, "f32", "head_major", None),
    (2, 2, 1, 420, 128, 96, "f32", "token_major", [33, 420]),
    # the contraction in two pieces: forwards, backwards, shared key heads
    (1, 2, 1, 200, 136, 72, "bf16", "token_major", None),
    (2, 4, 2, 333, 64, 256, "bf16", "head_major", [0, 330]),
    (1, 1, 1, 1500, 256, 256, "bf16", "head_major", None),
    # where the kernels change: one token, less than a chunk, narrow heads
    (3, 2, 2, 1, 64, 64, "bf16", "head_major", [1, 0, 1]),
    (3, 2, 1, 1, 20, 36, "f32", "head_major", [0, 1, 1]),
    (2, 4, 2, 8, 128, 128, "bf16", "head_major", [8, 3]),
    (2, 2, 1, 63, 64, 64, "bf16", "token_major", [0, 63]),
    (2, 2, 1, 64, 64, 64, "bf16", "head_major", [64, 1]),
    # more chains than SMs: some are cut and hand their state over
    (10, 16, 8, 700, 64, 64, "bf16", "token_major", [700, 0, 699, 64, 1, 300, 65, 512, 700, 130]),
    (4, 15, 5, 830, 128, 136, "bf16", "head_major", None),
    (10, 16, 16, 641, 32, 40, "bf16", "head_major", None),
]


@pytest.mark.gpu
@pytest.mark.parametrize("B,H,Hk,T,dk,dv,dtype,layout,lengths", CASES)
def test_forward_and_backward(sdm, B, H, Hk, T, dk, dv, dtype, layout, lengths):
    import torch
    from dla_reference import dla, dla_grads, near
    tm = layout == "token_major"
    s = _inputs(B, H, Hk, T, dk, dv, dtype, tm)
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    if n is not None:                                        # what lies past a length is never used
        past = torch.arange(T, device="cuda")[None, :] >= n[:, None]
        past = past[:, :, None, None] if tm else past[:, None, :, None]
        dirty = {x: torch.where(past, torch.full_like(s[x], math.nan), s[x]) for x in ("q", "k", "v", "dy")}
    else:
        dirty = {}
    shape = sdm.DlaShape.make(B, H, T, dk, dv, H_k=Hk, dtype=dtype, layout=layout, scale=0.7)
    y, state = run_forward(sdm, {**s, **dirty}, shape, n)
    want_y, want_S = dla(s["q"], s["k"], s["v"], s["log_decay"], s["state"], 0.7, n, tm)
    near(y, want_y, "y")
    near(state, want_S, "state")
    got = run_backward(sdm, {**s, **dirty}, shape, n)
    for name, g, w in zip(("dq", "dk", "dv", "dstate0"), got, dla_grads(*(s[x] for x in ("q", "k", "v", "log_decay", "state")), 0.7, s["dy"], s["dstate"], n, tm)):
        near(g, w, name)
    if n is not None:
        for x, o in (("y", y), ("dq", got[0]), ("dk", got[1]), ("dv", got[2])):
            assert not o[past.expand_as(o)].any(), x + " past the lengths"
    assert sdm.device_status() == 0
    again = run_backward(sdm, {**s, **dirty}, shape, n)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,dk,dv", [("f32", 64, 64), ("bf16", 128, 128), ("bf16", 256, 64)])
def test_decays_from_none_to_all(sdm, dtype, dk, dv):
    """lam = 1 sums everything, lam = 0 keeps one token, and log_decay above 0 grows."""
    import torch
    from dla_reference import dla, dla_grads, near
    s = _inputs(1, 4, 4, 150, dk, dv, dtype)
    s["log_decay"] = torch.tensor([0.0, -math.inf, -200.0, 0.01], device="cuda")
    shape = sdm.DlaShape.make(1, 4, 150, dk, dv, dtype=dtype)
    y, state = run_forward(sdm, s, shape)
    want_y, want_S = dla(s["q"], s["k"], s["v"], s["log_decay"], s["state"], 1.0)
    grads = run_backward(sdm, s, shape)
    want = dla_grads(*(s[x] for x in ("q", "k", "v", "log_decay", "state")), 1.0, s["dy"], s["dstate"])
    for h in range(4):
        near(y[:, h], want_y[:, h], f"y of head {h}")
        near(state[:, h], want_S[:, h], f"state of head {h}")
        for name, a, b in zip(("dq", "dk", "dv", "dstate0"), grads, want):
            near(a[:, h], b[:, h], f"{name} of head {h}")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,dk,dv,T,log_decay", [("f32", 64, 64, 20, 3.0), ("f32", 36, 20, 52, 1.4), ("f32", 200, 64, 20, 3.0),
                                                    ("bf16", 128, 128, 40, 1.5), ("bf16", 64, 64, 100, 0.7), ("bf16", 256, 136, 40, 1.5)])
def test_growth_over_a_partial_chunk(sdm, dtype, dk, dv, T, log_decay):
    """States that grow: the powers of the sequence's tokens fit float32, those of a whole chunk (32 or 64 tokens) need not."""
    import torch
    from dla_reference import dla, dla_grads, near
    s = _inputs(2, 2, 1, T, dk, dv, dtype)
    s["log_decay"] = torch.tensor([log_decay, -0.1], device="cuda")
    n = torch.tensor([T, T // 2], dtype=torch.int32, device="cuda")
    shape = sdm.DlaShape.make(2, 2, T, dk, dv, H_k=1, dtype=dtype)
    y, state = run_forward(sdm, s, shape, n)
    want_y, want_S = dla(s["q"], s["k"], s["v"], s["log_decay"], s["state"], 1.0, n)
    grads = run_backward(sdm, s, shape, n)
    want = dla_grads(*(s[x] for x in ("q", "k", "v", "log_decay", "state")), 1.0, s["dy"], s["dstate"], n)
    for b in range(2):
        for name, g, w in zip(("y", "state", "dq", "dk", "dv", "dstate0"), (y, state, *grads), (want_y, want_S, *want)):
            assert g[b].isfinite().all(), (name, b)
            near(g[b], w[b], f"{name} of sequence {b}")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,dk", [("f32", 64), ("bf16", 128), ("bf16", 256)])
@pytest.mark.parametrize("name", ["q", "k", "v"])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_values_that_are_not_finite_stay_behind(sdm, dtype, dk, name, value):
    """They reach no earlier token's output, and from q no other token's."""
    import torch
    T, t = 300, 171
    s = _inputs(1, 2, 2, T, dk, 128, dtype)
    shape = sdm.DlaShape.make(1, 2, T, dk, 128, dtype=dtype)
    clean, clean_S = run_forward(sdm, s, shape)
    bad = {**s, name: s[name].clone()}
    bad[name][0, 0, t, 5] = value
    y, state = run_forward(sdm, bad, shape)
    assert torch.equal(y[0, 0, :t], clean[0, 0, :t]) and torch.equal(y[0, 1], clean[0, 1]) and torch.equal(state[0, 1], clean_S[0, 1])
    if name == "q":
        assert not y[0, 0, t].isfinite().any()
        assert torch.equal(y[0, 0, t + 1:], clean[0, 0, t + 1:]) and torch.equal(state, clean_S)
    elif name == "v":
        assert not y[0, 0, t:, 5].isfinite().any() and not state[0, 0, :, 5].isfinite().any()
        keep = [c for c in range(128) if c != 5]
        assert torch.equal(y[0, 0][:, keep], clean[0, 0][:, keep]) and torch.equal(state[0, 0][:, keep], clean_S[0, 0][:, keep])
    else:
        assert not y[0, 0, t].isfinite().any() and not state[0, 0, 5].isfinite().any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,B,H,Hk,dk,dv,layout", [("bf16", 3, 4, 2, 128, 128, "head_major"), ("f32", 2, 3, 1, 36, 20, "token_major"),
                                                     ("bf16", 1, 2, 2, 256, 256, "head_major"), ("bf16", 5, 1, 1, 8, 8, "head_major")])
def test_step(sdm, dtype, B, H, Hk, dk, dv, layout):
    import torch
    from dla_reference import dla, near
    tm = layout == "token_major"
    s = _inputs(B, H, Hk, 1, dk, dv, dtype, tm)
    shape = sdm.DlaShape.make(B, H, 1, dk, dv, H_k=Hk, dtype=dtype, layout=layout, scale=0.5)
    want_y, want_S = dla(s["q"], s["k"], s["v"], s["log_decay"], s["state"], 0.5, None, tm)
    y, state = torch.empty_like(s["v"]), s["state"].clone()
    sdm.dla_step(shape, s["q"], s["k"], s["v"], s["log_decay"], state, y)
    near(y, want_y)
    near(state, want_S)
    # rows of a larger cache, one sequence skipped, one slot out of range
    cache = torch.randn((B + 3, H, dk, dv), device="cuda")
    before = cache.clone()
    slots = torch.arange(B + 1, 1, -1, dtype=torch.int32, device="cuda")
    cache[slots.long()] = s["state"]
    expect = cache.clone()
    expect[slots.long()] = state
    if B > 2:
        expect[slots[0].long()], expect[slots[1].long()] = s["state"][0], s["state"][1]
        slots[0], slots[1] = -1, B + 3
    y2 = torch.full_like(y, math.nan)
    sdm.dla_step(shape, s["q"], s["k"], s["v"], s["log_decay"], cache, y2, slots=slots)
    assert torch.equal(cache, expect) and torch.equal(cache[0], before[0])
    assert torch.equal(y2[2 if B > 2 else 0:], y[2 if B > 2 else 0:])
    assert B <= 2 or not y2[:2].any()
    assert sdm.device_status() == (1 if B > 2 else 0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [("f32", 36), ("bf16", 128)])
def test_one_token_is_a_step(sdm, dtype, d):
    """A forward over one token and no lengths gives what a step gives, bit for bit."""
    import torch
    s = _inputs(2, 4, 2, 1, d, d, dtype)
    shape = sdm.DlaShape.make(2, 4, 1, d, d, H_k=2, dtype=dtype, scale=0.7)
    y, state = run_forward(sdm, s, shape)
    y1, state1 = torch.empty_like(y), s["state"].clone()
    sdm.dla_step(shape, s["q"], s["k"], s["v"], s["log_decay"], state1, y1)
    assert torch.equal(y, y1) and torch.equal(state, state1)


@pytest.mark.gpu
def test_one_token_takes_no_workspace(sdm):
    """Where a prompt of that shape would (a contraction in two pieces), one token without lengths does not, and with them does."""
    import torch
    s = _inputs(2, 4, 2, 1, 256, 64, "bf16")
    shape = sdm.DlaShape.make(2, 4, 1, 256, 64, H_k=2, scale=0.7)
    assert sdm.dla_workspace_bytes(shape) > 0
    y, state = torch.empty_like(s["v"]), s["state"].clone()
    sdm.dla_forward(shape, s["q"], s["k"], s["v"], s["log_decay"], state, y)
    want_y, want_S = run_forward(sdm, s, shape)
    assert torch.equal(y, want_y) and torch.equal(state, want_S)
    with pytest.raises(sdm.SdmError, match="workspace is NULL"):
        sdm.dla_forward(shape, s["q"], s["k"], s["v"], s["log_decay"], state, y, lengths=torch.ones(2, dtype=torch.int32, device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prefill_in_pieces_then_tokens(sdm, dtype):
    """A prompt in two calls and the rest token by token gives what one call gives, in whatever pieces."""
    import torch
    from dla_reference import dla, near
    s = _inputs(2, 4, 2, 260, 64, 64, dtype)
    want_y, want_S = dla(s["q"], s["k"], s["v"], s["log_decay"], s["state"], 0.3)
    state, ys = s["state"].clone(), []
    for a, b in [(0, 150), (150, 256)] + [(t, t + 1) for t in range(256, 260)]:
        part = {n: s[n][:, :, a:b].contiguous() for n in ("q", "k", "v")}
        shape = sdm.DlaShape.make(2, 4, b - a, 64, 64, H_k=2, dtype=dtype, scale=0.3)
        y = torch.empty_like(part["v"])
        if b - a > 1:
            sdm.dla_forward(shape, part["q"], part["k"], part["v"], s["log_decay"], state, y, _ws(sdm.dla_workspace_bytes(shape)))
        else:
            sdm.dla_step(shape, part["q"], part["k"], part["v"], s["log_decay"], state, y)
        ys.append(y)
    near(torch.cat(ys, 2), want_y)
    near(state, want_S)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,T", [("f32", 32, 70), ("bf16", 128, 200)])
def test_bad_lengths_are_clamped_and_told(sdm, dtype, d, T):
    import torch
    s = _inputs(3, 2, 2, T, d, d, dtype)
    shape = sdm.DlaShape.make(3, 2, T, d, d, dtype=dtype)
    given = torch.tensor([-4, T + 9, 33], dtype=torch.int32, device="cuda")
    y, state = run_forward(sdm, s, shape, given)
    assert sdm.device_status() == 1
    want = run_forward(sdm, s, shape, given.clamp(0, T))
    assert torch.equal(y, want[0]) and torch.equal(state, want[1]) and sdm.device_status() == 0


@pytest.mark.gpu
def test_backward_without_last_gradient_and_without_tokens(sdm):
    import torch
    from dla_reference import dla_grads, near
    for dtype, d in (("f32", 32), ("bf16", 64)):
        s = _inputs(2, 2, 1, 90, d, d, dtype)
        shape = sdm.DlaShape.make(2, 2, 90, d, d, H_k=1, dtype=dtype)
        got = run_backward(sdm, s, shape, dstate="none")
        want = dla_grads(*(s[x] for x in ("q", "k", "v", "log_decay", "state")), 1.0, s["dy"], None)
        for g, w in zip(got, want):
            near(g, w)
        empty = sdm.DlaShape.make(2, 2, 0, d, d, H_k=1, dtype=dtype)
        e = _inputs(2, 2, 1, 0, d, d, dtype)
        assert torch.equal(run_backward(sdm, e, empty)[3], e["dstate"])
        assert not run_backward(sdm, e, empty, dstate="none")[3].any()


@pytest.mark.gpu
def test_gradient_against_differences(sdm):
    """The loss is linear in each of q, k, v and the state: a difference of two losses is the gradient times the step."""
    import torch
    s = _inputs(1, 2, 1, 100, 32, 32, "f32")
    shape = sdm.DlaShape.make(1, 2, 100, 32, 32, H_k=1, dtype="f32", scale=0.4)
    grads = dict(zip(("q", "k", "v", "state"), run_backward(sdm, s, shape)))

    def loss(**kw):
        y, S = run_forward(sdm, {**s, **kw}, shape)
        return float((y.double() * s["dy"].double()).sum() + (S.double() * s["dstate"].double()).sum())

    base = loss()
    for n, g in grads.items():
        step = torch.randn_like(s[n])
        change = float((g.double() * step.double()).sum())
        scale = float(g.double().norm() * step.double().norm())
        assert abs(loss(**{n: s[n] + step}) - base - change) <= 1e-5 * (scale + abs(base)), n


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,T", [("bf16", 128, 19456), ("bf16", 64, 9001), ("f32", 64, 22000), ("f32", 128, 6001)])
@pytest.mark.parametrize("log_decay", [0.0, -1e-6, -1e-5, -1e-4])
def test_long_memories_over_many_pieces(sdm, dtype, d, T, log_decay):
    """One chain with a slow decay, its tokens in many pieces: each chunk's step of the state, a decay and an addition, is off by at most
    2^-24 of it, and so are n of them in a row, of either sign, by 2^-24 sqrt(n)."""
    import torch
    s = _inputs(1, 1, 1, T, d, d, dtype)
    s["log_decay"] = torch.tensor([log_decay], device="cuda")
    shape = sdm.DlaShape.make(1, 1, T, d, d, dtype=dtype)
    assert sdm.dla_plan(shape)["pieces"] > 10
    _, state = run_forward(sdm, s, shape)
    dstate0 = run_backward(sdm, s, shape)[3]
    ld, at = s["log_decay"].double(), torch.arange(T, device="cuda")
    q, k, v, dy = (s[x][0, 0].double() for x in ("q", "k", "v", "dy"))
    want = torch.exp(ld * T) * s["state"][0, 0].double() + (torch.exp(ld * (T - 1 - at))[:, None] * k).T @ v
    want0 = torch.exp(ld * T) * s["dstate"][0, 0].double() + (torch.exp(ld * (at + 1))[:, None] * q).T @ dy
    limit = 2.0 ** -24 * math.sqrt(T / (64 if dtype == "bf16" else 32))
    for name, a, b in (("state", state, want), ("dstate0", dstate0, want0)):
        assert float((a[0, 0].double() - b).norm() / b.norm()) <= limit, name


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,B,H,d,T", [("f32", 1, 2, 64, 100), ("bf16", 1, 2, 128, 700), ("bf16", 10, 16, 64, 700)])
def test_captured_and_on_another_stream(sdm, dtype, B, H, d, T):
    """A captured forward, backward and step replay with new inputs, while another stream runs the same calls."""
    import torch
    shape, one = sdm.DlaShape.make(B, H, T, d, d, dtype=dtype), sdm.DlaShape.make(B, H, 1, d, d, dtype=dtype)
    s, new = _inputs(B, H, H, T, d, d, dtype), _inputs(B, H, H, T, d, d, dtype, seed=7)
    y, state, ws = torch.empty_like(s["v"]), s["state"].clone(), _ws(sdm.dla_workspace_bytes(shape))
    wb, out = _ws(sdm.dla_backward_workspace_bytes(shape)), [torch.empty_like(s[n]) for n in ("q", "k", "v", "state")]
    tok = [s[n][:, :, :1].contiguous() for n in ("q", "k", "v")]
    y1 = torch.empty_like(tok[2])

    def calls():
        sdm.dla_forward(shape, s["q"], s["k"], s["v"], s["log_decay"], state, y, ws)
        sdm.dla_step(one, *tok, s["log_decay"], state, y1)
        sdm.dla_backward(shape, s["q"], s["k"], s["v"], s["log_decay"], s["state"], s["dy"], s["dstate"], *out, wb)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for n in ("q", "k", "v", "dy", "dstate", "state"):
        s[n].copy_(new[n])
    state.copy_(new["state"])
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    graph.replay()
    with torch.cuda.stream(other):                           # buffers of its own, at the same time
        want_y, want_S = run_forward(sdm, new, shape)
        want = run_backward(sdm, new, shape)
        want_1 = torch.empty_like(y1)
        sdm.dla_step(one, *tok, s["log_decay"], want_S, want_1)
    torch.cuda.synchronize()
    assert torch.equal(y, want_y) and torch.equal(state, want_S) and torch.equal(y1, want_1)
    assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.gpu
def test_cut_chains_give_what_whole_ones_give(sdm):
    """Of ten sequences at once some chains are cut, of five none; the results are the same, bit for bit."""
    import torch
    s = _inputs(10, 16, 16, 1000, 64, 128, "bf16")
    y, state = run_forward(sdm, s, sdm.DlaShape.make(10, 16, 1000, 64, 128, dtype="bf16"))
    for i in (0, 5):
        half = {n: x if n == "log_decay" else x[i:i + 5].contiguous() for n, x in s.items()}
        y5, state5 = run_forward(sdm, half, sdm.DlaShape.make(5, 16, 1000, 64, 128, dtype="bf16"))
        assert torch.equal(y[i:i + 5], y5) and torch.equal(state[i:i + 5], state5)


# Chains that are cut, in the forward, the backward or both: B, H, Hk, T, dk, dv, dtype, layout, lengths, (forward, backward)
CUT = [
    (10, 16, 16, 1000, 64, 128, "bf16", "head_major", None, (True, True)),
    # reversed walks that begin with a partial chunk, and pieces past the end of short sequences
    (10, 16, 8, 1000, 64, 40, "bf16", "token_major", [1000, 0, 999, 64, 1, 300, 65, 512, 961, 130], (True, True)),
    # the long sequence's rest starts while its first piece still runs
    (10, 16, 8, 1000, 32, 32, "bf16", "head_major", [0] * 7 + [1000, 0, 0], (True, True)),
    # a contraction in two pieces, two slices of the state, key heads of three value heads
    (4, 15, 5, 1600, 128, 136, "bf16", "head_major", None, (False, True)),
    (6, 16, 8, 1200, 136, 64, "bf16", "token_major", [1200, 1199, 0, 640, 63, 1111], (True, False)),
    (8, 10, 10, 1400, 136, 72, "bf16", "head_major", None, (True, True)),
]


def test_what_is_cut(sdm):
    """The shapes that stand for cut chains are cut by the rule, so that another constant there does not empty the tests."""
    def cuts(B, H, Hk, T, dk, dv):
        shape = sdm.DlaShape.make(B, H, T, dk, dv, H_k=Hk)
        return tuple(sdm.dla_plan(shape, backward=b)["cuts"] > 0 for b in (False, True))

    for case in CUT:
        assert cuts(*case[:6]) == case[-1], case
    assert cuts(10, 16, 16, 1000, 64, 128) == (True, True) and cuts(5, 16, 16, 1000, 64, 128) == (False, False)      # equal bit for bit, below
    assert cuts(8, 16, 16, 4096, 128, 128) == (False, True)                                      # the 1.4B layer
    for B, H, Hk, T, dk, dv in ((1, 1, 1, 3000, 64, 64), (3, 2, 1, 1100, 128, 128)):             # few chains, in pieces
        assert sdm.dla_plan(sdm.DlaShape.make(B, H, T, dk, dv, H_k=Hk))["pieces"] > 1


@pytest.mark.gpu
@pytest.mark.parametrize("case", CUT)
def test_cut_chains_against_the_definition(sdm, case):
    test_forward_and_backward(sdm, *case[:9])


@pytest.mark.gpu
@pytest.mark.parametrize("lengths", [None, [1000, 0, 999, 64, 1, 300, 65, 512, 961, 130]])
def test_cut_chains_have_the_gradients_of_whole_ones(sdm, lengths):
    """The backward of ten sequences at once, whose chains are cut, and of five, whose chains are not: the same, bit for bit."""
    import torch
    s = _inputs(10, 16, 8, 1000, 64, 128, "bf16")
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    got = run_backward(sdm, s, sdm.DlaShape.make(10, 16, 1000, 64, 128, H_k=8), n)
    for i in (0, 5):
        half = {x: t if x == "log_decay" else t[i:i + 5].contiguous() for x, t in s.items()}
        five = run_backward(sdm, half, sdm.DlaShape.make(5, 16, 1000, 64, 128, H_k=8), None if n is None else n[i:i + 5].contiguous())
        for name, a, b in zip(("dq", "dk", "dv", "dstate0"), got, five):
            assert torch.equal(a[i:i + 5], b), name


@pytest.mark.gpu
@pytest.mark.parametrize("lengths,polls", [(None, 1 << 12), (None, 1), ([0, 1000, 64, 65, 1, 999, 300, 1000, 512, 130], 1)])
def test_a_withheld_state_ends_in_a_status(sdm, lengths, polls):
    """Cut chains whose first piece hands nothing over: the wait runs out, every CTA returns, and the status word says so.  Whole
    chains keep their results, and the next call runs as always."""
    import torch
    B, H, T, dk, dv = 10, 16, 1000, 64, 128
    s = _inputs(B, H, H, T, dk, dv, "bf16")
    shape = sdm.DlaShape.make(B, H, T, dk, dv, dtype="bf16")
    cuts = sdm.dla_plan(shape)["cuts"]
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    want_y, want_S = run_forward(sdm, s, shape, n)
    assert 0 < cuts < B * H and sdm.device_status() == 0
    y, state = torch.zeros_like(want_y), s["state"].clone()
    sdm.test_dla_wait_timeout(shape, s["q"], s["k"], s["v"], s["log_decay"], state, y, _ws(sdm.dla_workspace_bytes(shape)), polls, lengths=n)
    torch.cuda.synchronize()
    code = ctypes.c_int32(0)
    assert sdm.lib().sdm_device_status(ctypes.byref(code), None) == 5 and code.value == 4
    same = [torch.equal(y[b, h], want_y[b, h]) and torch.equal(state[b, h], want_S[b, h]) for b in range(B) for h in range(H)]
    assert sum(same) >= B * H - cuts                         # a cut chain whose tokens end in its first piece may be right, too
    again = run_forward(sdm, s, shape, n)
    assert torch.equal(again[0], want_y) and torch.equal(again[1], want_S) and sdm.device_status() == 0


@pytest.mark.gpu
def test_offsets_past_32_bits(sdm):
    """The last rows of a cache of states whose values number more than 2^31, and of long token rows."""
    import torch
    from dla_reference import dla, near
    H, d = 16, 128
    n = 2 ** 31 // (H * d * d) + 3
    cache = torch.zeros((n, H, d, d), device="cuda")
    s = _inputs(1, H, H, 1, d, d, "bf16")
    cache[n - 1] = s["state"][0]
    y = torch.empty_like(s["v"])
    sdm.dla_step(sdm.DlaShape.make(1, H, 1, d, d), s["q"], s["k"], s["v"], s["log_decay"], cache, y,
                 slots=torch.tensor([n - 1], dtype=torch.int32, device="cuda"))
    want_y, want_S = dla(s["q"], s["k"], s["v"], s["log_decay"], s["state"], 1.0)
    near(y, want_y)
    near(cache[n - 1:], want_S)
    assert not cache[:n - 1:97].any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,layout", [("bf16", "token_major"), ("bf16", "head_major"), ("f32", "token_major")])
def test_long_sequences_past_32_bits(sdm, dtype, layout):
    """A sequence of more than 2^31 values, key heads shared: what its first and its last tokens give, forwards and backwards.  Its
    heads forget within 100 tokens (exp(-50) of a state is left), so that 300 tokens are all that these depend on."""
    import torch
    from dla_reference import dla, dla_grads, near
    H, Hk, d, n, keep = 16, 8, 128, 300, 200
    T, tm = 2 ** 31 // (H * d) + 77, layout == "token_major"
    s = _inputs(1, H, Hk, T, d, d, dtype, tm)
    assert s["v"].numel() > 2 ** 31
    s["log_decay"] = -torch.linspace(0.5, 2.0, H, device="cuda")
    shape = sdm.DlaShape.make(1, H, T, d, d, H_k=Hk, dtype=dtype, layout=layout)
    y, state = run_forward(sdm, s, shape)
    dq, dk, dv, dstate0 = run_backward(sdm, s, shape)
    zero = torch.zeros_like(s["state"])
    for last in (False, True):
        def cut(x, m):
            axis = 1 if tm else 2
            return x.narrow(axis, x.shape[axis] - m if last else 0, m)

        part = {x: cut(s[x], n).contiguous() for x in ("q", "k", "v", "dy")}
        S0, dS = (zero, s["dstate"]) if last else (s["state"], zero)
        want_y, want_S = dla(part["q"], part["k"], part["v"], s["log_decay"], S0, 1.0, None, tm)
        near(cut(y, keep), cut(want_y, keep), f"y, last {last}")
        if last:
            near(state, want_S, "state")
        want = dla_grads(part["q"], part["k"], part["v"], s["log_decay"], S0, 1.0, part["dy"], dS, None, tm)
        for name, a, b in zip(("dq", "dk", "dv"), (dq, dk, dv), want):
            near(cut(a, keep), cut(b, keep), f"{name}, last {last}")
        if not last:
            near(dstate0, want[3], "dstate0")
    assert sdm.device_status() == 0
    del s, y, state, dq, dk, dv
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_sequences_past_32_bits(sdm):
    """The second of two sequences begins past 2^31 values and has few tokens, the first none: what is past the lengths is zero."""
    import torch
    from dla_reference import dla, dla_grads, near
    H, Hk, d, n = 16, 8, 128, 300
    T = 2 ** 31 // (H * d) + 64
    s = _inputs(2, H, Hk, T, d, d, "bf16", True)
    lengths = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    shape = sdm.DlaShape.make(2, H, T, d, d, H_k=Hk, dtype="bf16", layout="token_major")
    y, state = run_forward(sdm, s, shape, lengths)
    grads = run_backward(sdm, s, shape, lengths)
    part = {x: s[x][1:, :n].contiguous() for x in ("q", "k", "v", "dy")}
    want_y, want_S = dla(part["q"], part["k"], part["v"], s["log_decay"], s["state"][1:], 1.0, None, True)
    want = dla_grads(part["q"], part["k"], part["v"], s["log_decay"], s["state"][1:], 1.0, part["dy"], s["dstate"][1:], None, True)
    near(y[1:, :n], want_y, "y")
    near(state[1:], want_S, "state")
    for name, a, b in zip(("dq", "dk", "dv"), grads, want):
        near(a[1:, :n], b, name)
        assert not a[0].any() and not a[1, n:].any(), name
    near(grads[3][1:], want[3], "dstate0")
    assert not y[0].any() and not y[1, n:].any()
    assert torch.equal(state[0], s["state"][0]) and torch.equal(grads[3][0], s["dstate"][0])
    del s, y, state, grads
    torch.cuda.empty_cache()
