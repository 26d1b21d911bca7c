"""Gated delta rule: argument checks (CPU) and parity with 64-bit references (GPU).

Tolerances (relative 2-norm), from the arithmetic: float32 outputs come from float32 sums of at most a
few hundred terms per step, whose errors the decay forgets: 1e-5.  A bf16 output is rounded once
(about 2^-9 in the root mean square) and the tensor-core forms round up to two factors of a product to bf16 on the way:
3 * 2^-9 forward; the gradients multiply up to three rounded factors and round: 4 * 2^-9."""
import ctypes
import math
import os
import shutil

import pytest

TOL_F32, TOL_Y, TOL_GRAD = 1e-5, 3 * 2.0 ** -9, 4 * 2.0 ** -9


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
    return sdm.GdnShape.make(**base)


A = 1 << 20      # fake, aligned, far apart device addresses: validation never reads them


def _forward(sdm, shape, **kw):
    p = dict(q=A, k=2 * A, v=3 * A, alpha=4 * A, beta=5 * A, state=6 * A, y=7 * A, workspace=64 * A, workspace_nbytes=1 << 40)
    p.update(kw)
    sdm.gdn_forward(shape, stream=0, **p)


def test_struct_layout(sdm):
    assert ctypes.sizeof(sdm.GdnShape) == 36 and sdm.GdnShape.scale.offset == 32 and sdm.GdnShape.layout.offset == 28


@pytest.mark.parametrize("kw,status", [
    (dict(B=-1), 1), (dict(T=-5), 1), (dict(H=5), 1), (dict(H_k=0), 1), (dict(dtype=7), 1), (dict(layout=2), 1),
    (dict(d_k=0), 1), (dict(d_k=264), 2), (dict(d_k=12), 2), (dict(d_v=20), 2), (dict(d_k=6, dtype="f32"), 2),
    (dict(B=70000), 2), (dict(scale=math.inf), 1), (dict(scale=math.nan), 1)])
def test_refused_shapes(sdm, kw, status):
    shape = _shape(sdm, **kw)
    for call in (lambda: _forward(sdm, shape), lambda: sdm.gdn_workspace_bytes(shape),
                 lambda: sdm.gdn_backward_workspace_bytes(shape)):
        with pytest.raises(sdm.SdmError) as e:
            call()
        assert str(e.value)
    with pytest.raises(sdm.SdmError) as e:
        _forward(sdm, shape)
    assert e.value.status == status


@pytest.mark.parametrize("kw,word", [
    (dict(q=None), "q is NULL"), (dict(state=None), "state is NULL"), (dict(v=3 * A + 8), "v is not 16-byte aligned"),
    (dict(alpha=4 * A + 1), "alpha is not 2-byte aligned"), (dict(lengths=9 * A + 2), "lengths is not 4-byte aligned"),
    (dict(y=3 * A), "y overlaps v"), (dict(state=2 * A), "state overlaps k"), (dict(y=6 * A), "overlaps")])
def test_refused_buffers(sdm, kw, word):
    with pytest.raises(sdm.SdmError) as e:
        _forward(sdm, _shape(sdm), **kw)
    assert e.value.status == 1 and word in str(e.value)


def test_step_refusals(sdm):
    args = dict(q=A, k=2 * A, v=3 * A, alpha=4 * A, beta=5 * A, state=6 * A, y=7 * A, stream=0)
    with pytest.raises(sdm.SdmError, match="T == 1"):
        sdm.gdn_step(_shape(sdm), n_slots=2, **args)
    with pytest.raises(sdm.SdmError, match="n_slots"):
        sdm.gdn_step(_shape(sdm, T=1), n_slots=1, **args)
    with pytest.raises(sdm.SdmError, match="n_slots"):
        sdm.gdn_step(_shape(sdm, T=1), n_slots=-1, slots=8 * A, **args)


def test_backward_refusals(sdm):
    shape = _shape(sdm)
    names = ("q", "k", "v", "alpha", "beta", "state0", "dy", "dstate", "dq", "dk", "dv", "dalpha", "dbeta", "dstate0")
    base = {n: (i + 1) * A for i, n in enumerate(names)}
    need = sdm.gdn_backward_workspace_bytes(shape)
    assert need > 0

    def call(nb=need, ws=64 * A, **kw):
        sdm.gdn_backward(shape, workspace=ws, workspace_nbytes=nb, stream=0, **{**base, **kw})

    for kw, word in ((dict(nb=need - 1), "workspace too small"), (dict(ws=64 * A + 16), "256-byte aligned"),
                     (dict(ws=None), "workspace is NULL"), (dict(dq=base["q"]), "dq overlaps q"),
                     (dict(dk=base["dq"]), "overlaps"), (dict(dy=None), "dy is NULL"), (dict(dbeta=None), "dbeta is NULL"),
                     (dict(dstate0=base["state0"]), "dstate0 overlaps state0")):
        with pytest.raises(sdm.SdmError) as e:
            call(**kw)
        assert e.value.status == 1 and word in str(e.value)


def test_empty_calls_do_nothing(sdm):
    _forward(sdm, _shape(sdm, T=0))
    _forward(sdm, _shape(sdm, B=0))
    sdm.gdn_step(_shape(sdm, T=1, B=0), None, None, None, None, None, None, None, n_slots=0, stream=0)


def test_host_tensors_are_refused(sdm):
    import torch
    x = torch.zeros(4, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        sdm.gdn_forward(_shape(sdm), x, x, x, x, x, x, x, stream=0)


# ------------------------------------------------------------------ GPU parity
def _inputs(B, H, Hk, T, dk, dv, dtype, layout, seed, mu=3.0, device="cuda"):
    import torch
    g = torch.Generator(device=device).manual_seed(seed)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16

    def rand(*s):
        return torch.randn(s, generator=g, device=device)

    order = (lambda x: x.transpose(1, 2).contiguous()) if layout == "token_major" else (lambda x: x)
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)  # noqa: E731
    x = dict(q=order(unit(rand(B, Hk, T, dk)).to(dt)), k=order(unit(rand(B, Hk, T, dk)).to(dt)),
             v=order(rand(B, H, T, dv).to(dt)), alpha=torch.sigmoid(rand(B, H, T) + mu).to(dt),
             beta=torch.sigmoid(rand(B, H, T)).to(dt), state=rand(B, H, dk, dv) * 0.5)
    x["dy"] = order(rand(B, H, T, dv).to(dt))
    x["dstate"] = rand(B, H, dk, dv) * 0.5
    return x


def _poison(x, lengths, layout, T):
    """NaN and infinities past every sequence's length."""
    import torch
    pad = torch.arange(T, device="cuda")[None, :] >= lengths[:, None]
    for n in ("q", "k", "v", "dy"):
        m = pad[:, :, None, None] if layout == "token_major" else pad[:, None, :, None]
        x[n] = torch.where(m, torch.full_like(x[n], math.nan if n != "v" else math.inf), x[n])
    for n in ("alpha", "beta"):
        x[n] = torch.where(pad[:, None, :], torch.full_like(x[n], math.nan), x[n])


def _ws(n):
    import torch
    return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None


def _run_forward(sdm, x, c, lengths=None, T=None, stream=None):
    import torch
    shape = sdm.GdnShape.make(c["B"], c["H"], c["T"] if T is None else T, c["dk"], c["dv"], H_k=c["Hk"], dtype=c["dtype"],
                              layout=c["layout"], scale=c["dk"] ** -0.5)
    y, S = torch.full_like(x["v"], 7.0), x["state"].clone()
    sdm.gdn_forward(shape, x["q"], x["k"], x["v"], x["alpha"], x["beta"], S, y, _ws(sdm.gdn_workspace_bytes(shape)),
                    lengths=lengths, stream=stream)
    return y, S


def _run_backward(sdm, x, c, lengths=None, dstate=True, dstate0=True):
    import torch
    shape = sdm.GdnShape.make(c["B"], c["H"], c["T"], c["dk"], c["dv"], H_k=c["Hk"], dtype=c["dtype"], layout=c["layout"],
                              scale=c["dk"] ** -0.5)
    g = {n: torch.full_like(x[n], 7.0) for n in ("q", "k", "v", "alpha", "beta", "state")}
    before = x["state"].clone()
    sdm.gdn_backward(shape, x["q"], x["k"], x["v"], x["alpha"], x["beta"], x["state"], x["dy"],
                     x["dstate"] if dstate else None, g["q"], g["k"], g["v"], g["alpha"], g["beta"],
                     g["state"] if dstate0 else None, _ws(sdm.gdn_backward_workspace_bytes(shape)), lengths=lengths)
    assert torch.equal(before, x["state"])
    return g


def case(B=2, H=4, Hk=4, T=65, dk=64, dv=64, dtype="bf16", layout="head_major", lengths=None):
    return dict(B=B, H=H, Hk=Hk, T=T, dk=dk, dv=dv, dtype=dtype, layout=layout, lengths=lengths)


CASES = [
    case(T=1), case(T=2, dtype="f32"), case(T=63), case(T=64), case(T=65, layout="token_major"), case(T=200, dk=128, dv=128),
    case(T=129, dk=128, dv=128, Hk=2, layout="token_major"), case(T=70, dtype="f32", dk=4, dv=4),
    case(T=130, dk=8, dv=8), case(T=97, dk=24, dv=40, Hk=1), case(T=80, dk=96, dv=136, H=3, Hk=1),
    case(T=150, dk=128, dv=192, Hk=2), case(T=66, dk=256, dv=64, B=1), case(T=66, dk=256, dv=72, B=1, dtype="f32"),
    case(T=140, dk=136, dv=128, B=1), case(B=5, T=130, dk=128, dv=128, Hk=2, lengths=[130, 0, 1, 64, 77]),
    case(B=5, T=130, dk=72, dv=56, layout="token_major", lengths=[0, 130, 65, 127, 2]),
    case(B=4, T=90, dk=64, dv=96, dtype="f32", Hk=2, layout="token_major", lengths=[33, 0, 90, 1]),
    case(B=1, H=20, Hk=4, T=300, dk=64, dv=128), case(B=1, H=1, Hk=1, T=513, dk=128, dv=128),
]


def _id(c):
    return "-".join(f"{k}{v}" if not isinstance(v, list) else "ragged" for k, v in c.items() if v is not None)


def _prepared(c, seed):
    import torch
    x = _inputs(c["B"], c["H"], c["Hk"], c["T"], c["dk"], c["dv"], c["dtype"], c["layout"], seed)
    lengths = None
    if c["lengths"] is not None:
        lengths = torch.tensor(c["lengths"], dtype=torch.int32, device="cuda")
        _poison(x, lengths, c["layout"], c["T"])
    return x, lengths


@pytest.mark.gpu
@pytest.mark.parametrize("c", CASES, ids=_id)
def test_forward_parity(sdm, c):
    import torch
    from gdn_reference import gdn, rel
    x, lengths = _prepared(c, 1)
    ry, rS = gdn(x["q"], x["k"], x["v"], x["alpha"], x["beta"], x["state"], c["dk"] ** -0.5, lengths, c["layout"] == "token_major")
    y, S = _run_forward(sdm, x, c, lengths)
    assert sdm.device_status() == 0
    assert rel(S, rS) <= TOL_F32
    assert rel(y, ry) <= (TOL_F32 if c["dtype"] == "f32" else TOL_Y)
    if lengths is not None:
        pad = torch.arange(c["T"], device="cuda")[None, :] >= lengths[:, None]
        m = pad[:, :, None, None] if c["layout"] == "token_major" else pad[:, None, :, None]
        assert (torch.where(m, y, torch.zeros_like(y)) == 0).all()
        gone = lengths == 0
        assert torch.equal(S[gone], x["state"][gone])
    again = _run_forward(sdm, x, c, lengths)
    assert torch.equal(y, again[0]) and torch.equal(S, again[1])


@pytest.mark.gpu
@pytest.mark.parametrize("c", CASES, ids=_id)
def test_backward_parity(sdm, c):
    import torch
    from gdn_reference import gdn_grads, rel
    x, lengths = _prepared(c, 2)
    ref = gdn_grads(x["q"], x["k"], x["v"], x["alpha"], x["beta"], x["state"], c["dk"] ** -0.5, x["dy"], x["dstate"], lengths,
                    c["layout"] == "token_major")
    got = _run_backward(sdm, x, c, lengths)
    assert sdm.device_status() == 0
    for n, r in zip(("q", "k", "v", "alpha", "beta", "state"), ref):
        tol = TOL_F32 if c["dtype"] == "f32" or n == "state" else TOL_GRAD
        assert rel(got[n], r) <= tol, n
    again = _run_backward(sdm, x, c, lengths)
    for n in got:
        assert torch.equal(got[n], again[n]), n


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("what", ["alpha", "beta", "both"])
def test_gates_of_zero_and_one(sdm, dtype, what):
    """Gates of exactly 0 and 1 in every other token, and tiny ones: values and gradients stay right."""
    import torch
    from gdn_reference import gdn, gdn_grads, rel
    c = case(B=1, H=2, Hk=2, T=150, dk=64, dv=64, dtype=dtype)
    x, _ = _prepared(c, 3)
    for n in ("alpha", "beta") if what == "both" else (what,):
        x[n][:, :, ::5] = 0.0
        x[n][:, :, 1::7] = 1.0
        x[n][:, :, 3::11] = 1e-6
    ry, rS = gdn(x["q"], x["k"], x["v"], x["alpha"], x["beta"], x["state"], 0.125)
    y, S = _run_forward(sdm, x, c)
    assert rel(S, rS) <= TOL_F32 and rel(y, ry) <= (TOL_F32 if dtype == "f32" else TOL_Y)
    ref = gdn_grads(x["q"], x["k"], x["v"], x["alpha"], x["beta"], x["state"], 0.125, x["dy"], x["dstate"])
    got = _run_backward(sdm, x, c)
    for n, r in zip(("q", "k", "v", "alpha", "beta", "state"), ref):
        # a state gradient that a gate of zero cut off is a sum of nothing: compared absolutely
        tol = TOL_F32 if dtype == "f32" or n == "state" else TOL_GRAD
        assert rel(got[n], r) <= tol or float(r.norm()) < 1e-20 and float(got[n].double().norm()) < 1e-20, n


@pytest.mark.gpu
def test_backward_against_differences(sdm):
    """Directional derivatives of the 64-bit forward by central differences (step 1e-4: error about 1e-8
    relative plus 1e-12 / 1e-4 of rounding), against the float32 gradients."""
    import torch
    from gdn_reference import F64, gdn
    c = case(B=2, H=4, Hk=2, T=75, dk=16, dv=24, dtype="f32", lengths=[75, 41])
    x, lengths = _prepared(c, 4)
    for n in ("q", "k", "v", "alpha", "beta", "dy"):
        x[n] = torch.nan_to_num(x[n], nan=0.5, posinf=0.5)
    got = _run_backward(sdm, x, c, lengths)
    pad = torch.arange(75, device="cuda")[None, :] >= lengths[:, None]

    def loss(v):
        y, S = gdn(*[v[n] for n in ("q", "k", "v", "alpha", "beta", "state")], 0.25, lengths)
        return (y * x["dy"].to(F64)).sum() + (S * x["dstate"].to(F64)).sum()

    for n in ("q", "k", "v", "alpha", "beta", "state"):
        g = torch.Generator(device="cuda").manual_seed(9)
        d = torch.randn(x[n].shape, generator=g, device="cuda", dtype=F64)
        base = {m: x[m].to(F64) for m in ("q", "k", "v", "alpha", "beta", "state")}
        up = loss({**base, n: base[n] + 1e-4 * d})
        down = loss({**base, n: base[n] - 1e-4 * d})
        want, have = float((up - down) / 2e-4), float((got[n].to(F64) * d).sum())
        assert abs(want - have) <= 2e-5 * float(got[n].to(F64).norm() * d.norm() + abs(want)), n
    assert (got["alpha"].transpose(1, 2)[pad] == 0).all() and (got["q"].transpose(1, 2)[pad] == 0).all()


@pytest.mark.gpu
def test_backward_without_state_gradients(sdm):
    import torch
    c = case(T=70, dk=128, dv=128)
    x, _ = _prepared(c, 5)
    x["dstate"].zero_()
    full = _run_backward(sdm, x, c)
    none = _run_backward(sdm, x, c, dstate=False, dstate0=False)
    for n in ("q", "k", "v", "alpha", "beta"):
        assert torch.equal(full[n], none[n]), n


@pytest.mark.gpu
def test_backward_of_no_tokens(sdm):
    """T = 0: the state's gradient passes through."""
    import torch
    c = case(T=0)
    x, _ = _prepared(c, 6)
    got = _run_backward(sdm, x, c)
    assert torch.equal(got["state"], x["dstate"])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv,H,Hk", [(128, 128, 16, 16), (64, 96, 6, 3), (256, 40, 2, 1), (8, 8, 1, 1)])
def test_step_matches_forward_and_reference(sdm, dtype, dk, dv, H, Hk):
    """Single tokens through the cache give the state and outputs of the reference over the sequence."""
    import torch
    from gdn_reference import gdn, rel
    B, T, n = 5, 6, 9
    c = case(B=B, H=H, Hk=Hk, T=T, dk=dk, dv=dv, dtype=dtype)
    x, _ = _prepared(c, 7)
    ry, rS = gdn(x["q"], x["k"], x["v"], x["alpha"], x["beta"], x["state"], dk ** -0.5)
    slots = torch.tensor([7, 0, 3, 8, 1], dtype=torch.int32, device="cuda")
    cache = torch.full((n, H, dk, dv), 5.0, device="cuda")
    cache[slots.long()] = x["state"]
    shape = sdm.GdnShape.make(B, H, 1, dk, dv, H_k=Hk, dtype=dtype, scale=dk ** -0.5)
    ys = []
    for t in range(T):
        cut = {m: x[m][:, :, t].contiguous() for m in ("q", "k", "v", "alpha", "beta")}
        y = torch.empty((B, H, dv), dtype=x["v"].dtype, device="cuda")
        sdm.gdn_step(shape, cut["q"], cut["k"], cut["v"], cut["alpha"], cut["beta"], cache, y, slots=slots)
        ys.append(y)
    assert sdm.device_status() == 0
    assert rel(cache[slots.long()], rS) <= TOL_F32
    assert rel(torch.stack(ys, 2), ry) <= (TOL_F32 if dtype == "f32" else TOL_Y)
    rest = [i for i in range(n) if i not in slots.tolist()]
    assert (cache[rest] == 5.0).all()


@pytest.mark.gpu
def test_step_skipped_and_bad_slots(sdm):
    import torch
    c = case(B=3, T=1)
    x, _ = _prepared(c, 8)
    shape = sdm.GdnShape.make(3, 4, 1, 64, 64)
    args = [x[m] for m in ("q", "k", "v", "alpha", "beta")]
    state, y = x["state"].clone(), torch.full_like(x["v"], 7.0)
    sdm.gdn_step(shape, *args, state, y, slots=torch.tensor([-1, 2, -7], dtype=torch.int32, device="cuda"))
    assert sdm.device_status() == 0
    assert (y[0] == 0).all() and (y[2] == 0).all() and (y[1] != 0).any()
    assert torch.equal(state[:2], x["state"][:2]) and not torch.equal(state[2], x["state"][2])
    sdm.gdn_step(shape, *args, state, y, slots=torch.tensor([0, 1, 3], dtype=torch.int32, device="cuda"))
    assert sdm.device_status() == 1 and (y[2] == 0).all()


@pytest.mark.gpu
def test_bad_lengths_are_clamped_and_told(sdm):
    import torch
    c = case(B=2, T=70, lengths=None)
    x, _ = _prepared(c, 9)
    y, S = _run_forward(sdm, x, c, torch.tensor([71, -1], dtype=torch.int32, device="cuda"))
    assert sdm.device_status() == 1
    y2, S2 = _run_forward(sdm, x, c, torch.tensor([70, 0], dtype=torch.int32, device="cuda"))
    assert sdm.device_status() == 0
    assert torch.equal(y, y2) and torch.equal(S, S2)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward_in_pieces(sdm, dtype):
    """The state carries a sequence over calls: 200 tokens at once, or 130 + 1 + 69 of them."""
    import torch
    from gdn_reference import gdn, rel
    c = case(B=2, H=2, Hk=2, T=200, dk=128, dv=128, dtype=dtype)
    x, _ = _prepared(c, 10)
    ry, rS = gdn(x["q"], x["k"], x["v"], x["alpha"], x["beta"], x["state"], 128 ** -0.5)
    S, ys = x["state"], []
    for a, b in ((0, 130), (130, 131), (131, 200)):
        part = {n: (x[n][:, :, a:b].contiguous()) for n in ("q", "k", "v", "alpha", "beta")}
        part["state"] = S
        y, S = _run_forward(sdm, part, c, T=b - a)
        ys.append(y)
    assert rel(S, rS) <= TOL_F32
    assert rel(torch.cat(ys, 2), ry) <= (TOL_F32 if dtype == "f32" else TOL_Y)


@pytest.mark.gpu
def test_forward_on_another_stream(sdm):
    import torch
    c = case(T=300, dk=128, dv=128)
    x, _ = _prepared(c, 11)
    y, S = _run_forward(sdm, x, c)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        y2, S2 = _run_forward(sdm, x, c)
    st.synchronize()
    assert torch.equal(y, y2) and torch.equal(S, S2)


@pytest.mark.gpu
def test_offsets_past_32_bits(sdm):
    """A cache whose last state lies past 2^32 bytes (and 2^31 elements)."""
    import torch
    from gdn_reference import gdn, rel
    n, H, dk, dv = 2080, 64, 128, 128
    cache = torch.zeros((n, H, dk, dv), device="cuda")
    c = case(B=1, H=H, Hk=H, T=1, dk=dk, dv=dv)
    x, _ = _prepared(c, 12)
    cache[n - 1] = x["state"][0]
    y = torch.empty_like(x["v"])
    sdm.gdn_step(sdm.GdnShape.make(1, H, 1, dk, dv, scale=1.0), x["q"], x["k"], x["v"], x["alpha"], x["beta"], cache, y,
                 slots=torch.tensor([n - 1], dtype=torch.int32, device="cuda"))
    ry, rS = gdn(x["q"], x["k"], x["v"], x["alpha"], x["beta"], x["state"], 1.0)
    assert rel(cache[n - 1], rS[0]) <= TOL_F32 and rel(y, ry) <= TOL_Y
    assert float(cache[: n - 1].abs().max()) == 0.0


# ------------------------------------------------------------------ correlated keys and slow gates
# Keys and queries of a cosine of rho with each other (a silu before the projection's normalisation, neighbouring tokens),
# alpha = sigmoid(N(mu, 1)), beta = sigmoid(N(bmu, 1)): what a chunk's products cancel down to is far below the products.
REGIMES = [(0.25, 3, 0), (0.64, 8, 4), (0.9, 3, 4), (0.98, 3, 4), (0.98, 8, 0)]


def _correlated(c, rho, mu, bmu, seed):
    import torch
    x, _ = _prepared(c, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1000)

    def rand(*s):
        return torch.randn(s, generator=g, device="cuda")

    unit = lambda t: t / t.norm(dim=-1, keepdim=True)  # noqa: E731
    mean = unit(rand(c["B"], c["Hk"], 1, c["dk"]))
    for n in ("q", "k"):
        x[n] = unit(rho ** 0.5 * mean + (1 - rho) ** 0.5 * unit(rand(c["B"], c["Hk"], c["T"], c["dk"]))).to(x[n].dtype)
    x["alpha"] = torch.sigmoid(rand(c["B"], c["H"], c["T"]) + mu).to(x["alpha"].dtype)
    x["beta"] = torch.sigmoid(rand(c["B"], c["H"], c["T"]) + bmu).to(x["beta"].dtype)
    return x


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dk", [32, 64, 128])
@pytest.mark.parametrize("rho,mu,bmu", REGIMES)
def test_correlated_keys_output(sdm, rho, mu, bmu, dk, dtype):
    """A bf16 y is off by its one rounding, 0.43 * 2^-8 in the root mean square, and what 16 bits of each factor add: 2e-3."""
    from gdn_reference import gdn, rel
    c = case(B=2, H=2, Hk=2, T=320, dk=dk, dv=64, dtype=dtype)
    x = _correlated(c, rho, mu, bmu, 20)
    ry, _ = gdn(x["q"], x["k"], x["v"], x["alpha"], x["beta"], x["state"], dk ** -0.5)
    y, _ = _run_forward(sdm, x, c)
    assert rel(y, ry) <= (TOL_F32 if dtype == "f32" else 2e-3)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dk", [32, 64, 128])
@pytest.mark.parametrize("rho,mu,bmu", REGIMES)
def test_correlated_keys_states(sdm, rho, mu, bmu, dk, dtype):
    """The last state and the first state's gradient, which a chunk's products may take down to a hundredth of where it
    starts, are float32 results all the same."""
    from gdn_reference import gdn, gdn_grads, rel
    c = case(B=2, H=2, Hk=2, T=320, dk=dk, dv=64, dtype=dtype)
    x = _correlated(c, rho, mu, bmu, 21)
    args = [x[n] for n in ("q", "k", "v", "alpha", "beta", "state")]
    assert rel(_run_forward(sdm, x, c)[1], gdn(*args, dk ** -0.5)[1]) <= TOL_F32
    assert rel(_run_backward(sdm, x, c)["state"], gdn_grads(*args, dk ** -0.5, x["dy"], x["dstate"])[-1]) <= TOL_F32


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dk", [32, 64, 128])
@pytest.mark.parametrize("rho,mu,bmu", REGIMES)
def test_correlated_keys_gradients(sdm, rho, mu, bmu, dk, dtype):
    """A bf16 gradient is rounded, 0.43 * 2^-8 in the root mean square, and has up to two once rounded factors (S, D):
    0.74 * 2^-8, and 2^-8 allowed.  dalpha: where the gates forget a chunk's start (mu = 3) its terms, up to a hundred times
    what they cancel down to, have factors of 16 bits: 0.6 * 2^-8 with its rounding; else <D, S> of rounded S and D is in it,
    with one error for all 64 tokens of a chunk, so that a test of few chunks may be off by twice the root mean square:
    1.5 * 2^-8.  In float32 the same terms' sums, a few roundings each: 100 * 2^-22."""
    from gdn_reference import gdn_grads, rel
    c = case(B=2, H=2, Hk=2, T=320, dk=dk, dv=64, dtype=dtype)
    x = _correlated(c, rho, mu, bmu, 22)
    ref = gdn_grads(*[x[n] for n in ("q", "k", "v", "alpha", "beta", "state")], dk ** -0.5, x["dy"], x["dstate"])
    got = _run_backward(sdm, x, c)
    far = {n: rel(got[n], r) for n, r in zip(("q", "k", "v", "alpha", "beta"), ref)}
    for n, f in far.items():
        if dtype == "f32":
            assert f <= (100 * 2.0 ** -22 if n == "alpha" else TOL_F32), far
        else:
            assert f <= (1.0 if n != "alpha" else 0.6 if mu == 3 else 1.5) * 2.0 ** -8, far


# ------------------------------------------------------------------ values that are not finite in a live token
@pytest.mark.gpu
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("c", [
    case(B=2, H=4, Hk=2, T=200, dk=128, dv=136), case(B=2, H=2, Hk=2, T=130, dk=40, dv=64, layout="token_major"),      # chunks of 64
    case(B=2, H=2, Hk=1, T=100, dk=64, dv=40, dtype="f32"),                                                             # chunks of 32
    case(B=2, H=2, Hk=2, T=20, dk=64, dv=64), case(B=1, H=2, Hk=2, T=100, dk=136, dv=64),                               # tokens
    case(B=4, H=16, Hk=16, T=70, dk=16, dv=96, dtype="f32")], ids=_id)
def test_nothing_reaches_earlier_tokens(sdm, c, value):
    """The outputs before the token are those without it, bit for bit, and so are those of other sequences, heads and (for v)
    columns; from it on they are not finite, nor is the state, but for q, which only its own output takes."""
    import torch
    x, _ = _prepared(c, 30)
    clean, S = _run_forward(sdm, x, c)
    tokens = (lambda t: t.transpose(1, 2)) if c["layout"] == "token_major" else (lambda t: t)      # -> [B, heads, T, ...]
    group = c["H"] // c["Hk"]
    mine = (torch.arange(c["H"], device="cuda") // group == 0)[None, :, None, None] & (torch.arange(c["B"], device="cuda") == c["B"] - 1)[:, None, None, None]
    for at in (0, 5, c["T"] // 2 + 3, c["T"] - 1):
        for n in ("q", "k", "v", "alpha", "beta"):
            z = {m: t.clone() for m, t in x.items()}
            if n in ("alpha", "beta"):
                z[n][c["B"] - 1, :group, at] = value
            elif n == "v":
                tokens(z[n])[c["B"] - 1, :group, at, 3] = value
            else:
                tokens(z[n])[c["B"] - 1, 0, at, 3] = value
            y, T = _run_forward(sdm, z, c)
            t = torch.arange(c["T"], device="cuda")[None, None, :, None]
            hit = mine & (t == at if n == "q" else t >= at)
            hit = (hit & (torch.arange(c["dv"], device="cuda") == 3)) if n == "v" else hit.expand(tokens(y).shape)
            left = (mine & (torch.arange(c["dv"], device="cuda") == 3)).expand(S.shape) if n == "v" else (mine & (n != "q")).expand(S.shape)
            assert not torch.isfinite(tokens(y)[hit]).any(), (n, at)
            assert torch.equal(tokens(y)[~hit], tokens(clean)[~hit]), (n, at)
            assert not torch.isfinite(T[left]).any() and torch.equal(T[~left], S[~left]), (n, at)
    assert sdm.device_status() == 0


# ------------------------------------------------------------------ the token recurrence and the forms on either side of it
RECURRENCE = [
    case(B=5, H=16, Hk=16, T=70, dk=64, dv=64, dtype="f32"), case(B=5, H=16, Hk=8, T=96, dk=24, dv=64, dtype="f32", lengths=[96, 0, 1, 64, 33]),
    case(B=5, H=16, Hk=16, T=70, dk=136, dv=72, dtype="f32", layout="token_major", lengths=[31, 70, 32, 0, 69]),
    case(B=5, T=20, dk=64, dv=64, Hk=2, lengths=[20, 0, 1, 16, 17]), case(B=4, T=31, dk=128, dv=40, layout="token_major", lengths=[0, 31, 30, 2]),
    case(B=5, T=70, dk=136, dv=64, Hk=1, lengths=[70, 0, 1, 32, 65]), case(B=3, T=24, dk=16, dv=64, dtype="f32", lengths=[0, 24, 7]),
    case(B=4, T=100, dk=256, dv=24, lengths=[100, 0, 64, 33], layout="token_major"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("c", RECURRENCE, ids=_id)
def test_token_recurrence(sdm, c):
    """float32 above the chunked walk's number of CTAs, bf16 below 32 tokens and above d_k = 128, with and without ragged
    batches whose padding is not finite: outputs, states and gradients."""
    test_forward_parity(sdm, c)
    test_backward_parity(sdm, c)


def test_a_failed_query_is_not_remembered(tmp_path):
    """The register counts of the kernels that split them: asked for again after a failure, once after an answer."""
    import subprocess
    from paper_2607_07386_gb300 import build as B
    try:
        nvcc = B.nvcc()
    except RuntimeError:
        pytest.skip("nvcc not available")
    src = tmp_path / "query.cu"
    src.write_text("""#include "gdn_internal.h"
int main() {
    std::atomic<int> known{0};
    int asked = 0;
    cudaError_t answer = cudaErrorInitializationError;
    auto get = [&](int* n) { ++asked; if (answer == cudaSuccess) *n = 128; return answer; };
    if (sdm::check_registers(128, known, get) != cudaErrorInitializationError) return 1;
    answer = cudaSuccess;
    if (sdm::check_registers(128, known, get) != cudaSuccess || asked != 2) return 2;
    if (sdm::check_registers(128, known, get) != cudaSuccess || asked != 2) return 3;
    return sdm::check_registers(168, known, get) == cudaErrorInvalidConfiguration ? 0 : 4;
}
""")
    exe = tmp_path / "query"
    subprocess.run([nvcc, "-std=c++17", "-I", B.INCLUDE, "-I", B.CSRC, str(src), "-o", str(exe)], check=True, capture_output=True)
    assert subprocess.run([str(exe)]).returncode == 0
