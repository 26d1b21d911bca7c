"""The norms around a block: argument checks (CPU) and parity with 64-bit references (GPU).

Tolerances: see dla_reference.near (half a step of the storage type plus float32 sums)."""
import ctypes
import math

import pytest

from test_dla import A, sdm  # noqa: F401


def _call(sdm, shape=None, **kw):
    p = dict(x=A, y=2 * A, gate=3 * A, res_scale=4 * A, gamma_post=5 * A, gamma_pre=6 * A, h=7 * A, z=8 * A)
    p.update(kw)
    sdm.block_norm(shape or sdm.BlockNormShape.make(16, 64), stream=0, **p)


def _back(sdm, shape=None, **kw):
    names = ("y", "h", "dz", "dh", "dx", "dy", "gate", "res_scale", "gamma_post", "gamma_pre", "dgate", "dres_scale",
             "dgamma_post", "dgamma_pre")
    p = {n: (i + 1) * A for i, n in enumerate(names)}
    p.update(workspace=64 * A, workspace_nbytes=1 << 40)
    p.update(kw)
    sdm.block_norm_backward(shape or sdm.BlockNormShape.make(16, 64), stream=0, **p)


def test_struct_layout(sdm):  # noqa: F811
    assert ctypes.sizeof(sdm.BlockNormShape) == 32 and sdm.BlockNormShape.eps.offset == 24


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), 1), (dict(D=0), 1), (dict(gate_rows=0), 1), (dict(dtype=3), 1), (dict(D=12), 2), (dict(D=16392), 2),
    (dict(D=6, dtype="f32"), 2), (dict(M=1 << 40), 2), (dict(eps=-1e-6), 1), (dict(eps=math.nan), 1), (dict(eps=math.inf), 1)])
def test_refused_shapes(sdm, kw, status):  # noqa: F811
    shape = sdm.BlockNormShape.make(**{**dict(M=16, D=64), **kw})
    for call in (lambda: _call(sdm, shape), lambda: _back(sdm, shape)):
        with pytest.raises(sdm.SdmError) as e:
            call()
        assert e.value.status == status
    with pytest.raises(sdm.SdmError):
        sdm.block_norm_backward_workspace_bytes(shape)


@pytest.mark.parametrize("kw,word", [
    (dict(x=None), "x is NULL"), (dict(h=None), "h is NULL"), (dict(y=None), "gate without y"),
    (dict(y=None, gate=None, res_scale=None, gamma_post=None), "h without y"), (dict(gamma_pre=None), "z without gamma_pre"),
    (dict(z=None), "gamma_pre without z"), (dict(y=None, gate=None, res_scale=None, gamma_post=None, h=None, z=None, gamma_pre=None), "neither"),
    (dict(x=A + 2), "x is not 16-byte aligned"), (dict(res_scale=4 * A + 4), "res_scale is not 16-byte aligned"),
    (dict(h=2 * A), "h overlaps y"), (dict(z=A), "z overlaps x"), (dict(z=7 * A), "overlaps"), (dict(h=A + 16), "h overlaps x")])
def test_refused_buffers(sdm, kw, word):  # noqa: F811
    with pytest.raises(sdm.SdmError) as e:
        _call(sdm, **kw)
    assert e.value.status == 1 and word in str(e.value)


@pytest.mark.parametrize("kw,word", [
    (dict(h=None), "h is NULL"), (dict(dx=None), "dx is NULL"), (dict(dy=None), "dy is NULL"), (dict(dz=None), "gamma_pre without dz"),
    (dict(gate=None), "dgate without gate"), (dict(gamma_post=None), "dgamma_post without"), (dict(res_scale=None), "dres_scale without"),
    (dict(gamma_pre=None), "dgamma_pre without"), (dict(workspace=None), "workspace is NULL"), (dict(workspace=64 * A + 16), "256-byte"),
    (dict(workspace_nbytes=4), "too small"), (dict(dx=3 * A), "overlaps"), (dict(dy=A), "overlaps"), (dict(dgamma_pre=13 * A), "overlaps")])
def test_refused_backward(sdm, kw, word):  # noqa: F811
    with pytest.raises(sdm.SdmError) as e:
        _back(sdm, **kw)
    assert e.value.status == 1 and word in str(e.value)


@pytest.mark.parametrize("rows", [2**40, 2**63 - 1])
def test_gate_of_more_rows_than_there_are(sdm, rows):  # noqa: F811
    """It is one for all of them; its row is still checked."""
    shape = sdm.BlockNormShape.make(16, 64, gate_rows=rows)
    assert sdm.block_norm_backward_workspace_bytes(shape) == sdm.block_norm_backward_workspace_bytes(sdm.BlockNormShape.make(16, 64, gate_rows=16))
    with pytest.raises(sdm.SdmError, match="overlaps"):
        _call(sdm, shape, gate=7 * A + 64)


def test_empty_forward(sdm):  # noqa: F811
    _call(sdm, sdm.BlockNormShape.make(0, 64))


# ------------------------------------------------------------------ parity
def _inputs(M, D, dtype, gate_rows, have, seed=0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    s = dict(x=rand(M, D).to(dt) * 2, dz=rand(M, D).to(dt), dh=rand(M, D).to(dt))
    s["y"] = rand(M, D).to(dt)
    s["gate"] = torch.sigmoid(rand(-(-M // gate_rows), D)).to(dt) if "g" in have else None
    s["res_scale"] = 0.3 + 0.1 * rand(D) if "s" in have else None
    s["gamma_post"] = 1 + 0.2 * rand(D) if "o" in have else None
    s["gamma_pre"] = 1 + 0.2 * rand(D) if "p" in have else None
    return s


VECTORS = ("gate", "res_scale", "gamma_post", "gamma_pre")
CASES = [  # M, D, dtype, gate_rows, which of gate, res_scale, gamma_post, gamma_pre
    (1, 8, "bf16", 1, "gsop"), (1, 4, "f32", 1, "gsop"), (5, 264, "bf16", 2, "gsop"), (33, 256, "bf16", 33, "gsop"), (700, 96, "f32", 3, "gsop"),
    (130, 516, "f32", 1, "gsop"), (67, 2048, "bf16", 30, "gsop"), (9, 4100, "f32", 4, "gsop"), (7, 8200, "bf16", 3, "gsop"), (3, 16384, "bf16", 1, "gsop"),
    (5, 16384, "f32", 5, "gsop"), (4000, 128, "bf16", 1500, "gsop"), (1300, 1032, "bf16", 1300, "gsop"), (64, 512, "bf16", 100, "gp"), (21, 320, "f32", 1, ""),
    (21, 320, "bf16", 1, "p"), (40, 1024, "bf16", 1, "sp"), (40, 1024, "bf16", 7, "go"), (2500, 64, "f32", 2, "gso"), (40, 72, "bf16", 1, "op"),
    (3000, 2048, "bf16", 7, "gsop"), (3001, 1544, "f32", 17, "gsop"), (9000, 256, "bf16", 2, "gp"), (2000, 2048, "f32", 290, "go"),
    (900, 8192, "bf16", 3, "gsop"), (700, 8192, "bf16", 200, "gsop"), (700, 8192, "bf16", 1, "gsop"),
    (1900, 768, "bf16", 30, "gsop"), (1900, 760, "bf16", 1, "gsop"), (1100, 1280, "bf16", 1, "gsop"), (1100, 1256, "bf16", 500, "gsop"),
    (800, 1536, "bf16", 9, "gsop"), (800, 1528, "bf16", 1, "sop"), (900, 2560, "bf16", 1, "gsop"), (900, 2552, "bf16", 77, "gsp"),
    (300, 4096, "f32", 7, "gsop"), (500, 4096, "bf16", 1, "gsop"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("M,D,dtype,gate_rows,have", CASES)
def test_forward_and_backward(sdm, M, D, dtype, gate_rows, have):  # noqa: F811
    import torch
    from dla_reference import F64, block_norm, near
    s = _inputs(M, D, dtype, gate_rows, have)
    eps = 1e-5
    shape = sdm.BlockNormShape.make(M, D, dtype=dtype, gate_rows=gate_rows, eps=eps)
    h, z = torch.full_like(s["x"], math.nan), torch.full_like(s["x"], math.nan) if "p" in have else None
    vec = {n: s[n] for n in VECTORS}
    sdm.block_norm(shape, s["x"], s["y"], h, z, **vec)
    want_h, want_z = block_norm(s["x"], s["y"], *vec.values(), gate_rows, eps, stored=h)
    near(h, want_h, "h")
    if z is not None:
        near(z, want_z, "z")
    # in place, the residual stream gives the same
    x, z2 = s["x"].clone(), None if z is None else torch.empty_like(z)
    sdm.block_norm(shape, x, s["y"], x, z2, **vec)
    assert torch.equal(x, h) and (z is None or torch.equal(z2, z))

    def back(dx=None):
        out = {n: None if s[n] is None else torch.full_like(s[n], math.nan) for n in VECTORS}
        dx, dy = torch.full_like(h, math.nan) if dx is None else dx, torch.full_like(h, math.nan)
        ws = torch.full((sdm.block_norm_backward_workspace_bytes(shape),), 0xFF, dtype=torch.uint8, device="cuda")
        sdm.block_norm_backward(shape, s["y"], h if "p" in have else None, s["dz"] if "p" in have else None,
                                s["dh"] if dx is None else dh_of(dx), dx, dy, **vec, **{"d" + n: o for n, o in out.items()}, workspace=ws)
        return [dx, dy] + [out[n] for n in VECTORS]

    def dh_of(dx):
        return dx if dx is not None and place else s["dh"]

    place = False
    got = back()
    # gradients of h and z where z's norm is of the stored h: the residual stream's own, then through the first half
    hh = h.to(F64).requires_grad_(True)
    live = {n: s[n].to(F64).requires_grad_(True) for n in VECTORS if s[n] is not None}
    a = s["dh"].to(F64)
    want = {}
    if "p" in have:
        _, zz = block_norm(hh, None, None, None, None, live["gamma_pre"], 1, eps)
        dh, want["gamma_pre"] = torch.autograd.grad(zz, (hh, live["gamma_pre"]), s["dz"].to(F64))
        a = a + dh
    yy = s["y"].to(F64).requires_grad_(True)
    first, _ = block_norm(torch.zeros_like(hh), yy, live.get("gate"), live.get("res_scale"), live.get("gamma_post"), None, gate_rows, eps)
    names = [n for n in ("gate", "res_scale", "gamma_post") if n in live]
    grads = torch.autograd.grad(first, [yy] + [live[n] for n in names], a)
    want.update(zip(names, grads[1:]))
    near(got[0], a, "dx")
    near(got[1], grads[0], "dy")
    for n, g in zip(VECTORS, got[2:]):
        if g is not None:
            near(g, want[n], "d" + n)
    assert all(p is None or torch.equal(p, q) for p, q in zip(got, back()))
    place = True                                             # dx over dh
    same = back(s["dh"].clone())
    assert all(p is None or torch.equal(p, q) for p, q in zip(got, same))


@pytest.mark.gpu
def test_one_gate_for_any_number_of_rows(sdm):  # noqa: F811
    import torch
    s, got = _inputs(50, 64, "bf16", 50, "gsop"), []
    for rows in (50, 2**40, 2**63 - 1):
        shape = sdm.BlockNormShape.make(50, 64, gate_rows=rows)
        h, z, dx, dy = (torch.empty_like(s["x"]) for _ in range(4))
        vec = {n: s[n] for n in VECTORS}
        out = {"d" + n: torch.empty_like(s[n]) for n in VECTORS}
        sdm.block_norm(shape, s["x"], s["y"], h, z, **vec)
        ws = torch.empty(sdm.block_norm_backward_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
        sdm.block_norm_backward(shape, s["y"], h, s["dz"], s["dh"], dx, dy, **vec, **out, workspace=ws)
        got.append([h, z, dx, dy, *out.values()])
    assert all(torch.equal(a, b) for g in got[1:] for a, b in zip(got[0], g))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_before_the_first_block(sdm, dtype):  # noqa: F811
    """Without y, z is the norm of x; its backward gives dx and dgamma_pre alone, with and without dh."""
    import torch
    from dla_reference import F64, block_norm, near
    s = _inputs(37, 328, dtype, 1, "p")
    shape = sdm.BlockNormShape.make(37, 328, dtype=dtype)
    z = torch.empty_like(s["x"])
    sdm.block_norm(shape, s["x"], None, None, z, gamma_pre=s["gamma_pre"])
    near(z, block_norm(s["x"], None, None, None, None, s["gamma_pre"], 1, 1e-6)[1])
    x, gamma = s["x"].to(F64).requires_grad_(True), s["gamma_pre"].to(F64).requires_grad_(True)
    want = torch.autograd.grad(block_norm(x, None, None, None, None, gamma, 1, 1e-6)[1], (x, gamma), s["dz"].to(F64))
    ws = torch.empty(sdm.block_norm_backward_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    for dh in (None, s["dh"]):
        dx, dg = torch.empty_like(z), torch.empty_like(s["gamma_pre"])
        sdm.block_norm_backward(shape, None, s["x"], s["dz"], dh, dx, None, gamma_pre=s["gamma_pre"], dgamma_pre=dg, workspace=ws)
        near(dx, want[0] if dh is None else want[0] + dh.to(F64))
        near(dg, want[1])


@pytest.mark.gpu
def test_rows_apart_and_zero_rows(sdm):  # noqa: F811
    """A row that is zero stays zero with eps > 0; NaN and infinity stay in their row; without eps a zero row is NaN alone."""
    import torch
    for dtype, D in (("f32", 132), ("bf16", 1024)):
        s = _inputs(9, D, dtype, 1, "gsop")
        s["x"][2], s["y"][2] = 0, 0
        shape = sdm.BlockNormShape.make(9, D, dtype=dtype)
        vec = {n: s[n] for n in VECTORS}

        def run(eps=1e-6):
            h, z = torch.empty_like(s["x"]), torch.empty_like(s["x"])
            sdm.block_norm(sdm.BlockNormShape.make(9, D, dtype=dtype, eps=eps), s["x"], s["y"], h, z, **vec)
            ws = torch.empty(sdm.block_norm_backward_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
            dx, dy = torch.empty_like(h), torch.empty_like(h)
            sdm.block_norm_backward(sdm.BlockNormShape.make(9, D, dtype=dtype, eps=eps), s["y"], h, s["dz"], s["dh"], dx, dy, **vec, workspace=ws)
            return h, z, dx, dy

        clean = run()
        assert not clean[0][2].any() and not clean[1][2].any() and clean[2].isfinite().all() and clean[3].isfinite().all()
        bare = run(0.0)
        rest = [i for i in range(9) if i != 2]
        assert all(a[rest].isfinite().all() for a in bare) and bare[1][2].isnan().all()
        s["y"][5, 3] = math.inf
        s["x"][7, 4] = math.nan
        bad = run()
        rest = [i for i in range(9) if i not in (5, 7)]
        assert all(torch.equal(a[rest], b[rest]) for a, b in zip(clean, bad))
        assert bad[1][7].isnan().all() and not bad[0][5, 3].isfinite()


@pytest.mark.gpu
def test_empty_backward_zeroes_the_vectors(sdm):  # noqa: F811
    import torch
    shape = sdm.BlockNormShape.make(0, 64)
    none = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    out = [torch.full((64,), 3.0, device="cuda") for _ in range(3)]
    one = torch.ones(64, device="cuda")
    assert sdm.block_norm_backward_workspace_bytes(shape) == 0
    sdm.block_norm_backward(shape, none, none, none, none, none, none, gate=none, res_scale=one, gamma_post=one, gamma_pre=one, dgate=none,
                            dres_scale=out[0], dgamma_post=out[1], dgamma_pre=out[2])
    assert not any(o.any() for o in out)


@pytest.mark.gpu
def test_captured_beside_another_stream(sdm):  # noqa: F811
    import torch
    M, D = 300, 768
    s, new = _inputs(M, D, "bf16", 50, "gsop"), _inputs(M, D, "bf16", 50, "gsop", seed=9)
    shape = sdm.BlockNormShape.make(M, D, gate_rows=50)

    def buffers():
        return ([torch.empty_like(s["x"]) for _ in range(4)], [torch.empty_like(s[n]) for n in VECTORS],
                torch.empty(sdm.block_norm_backward_workspace_bytes(shape), dtype=torch.uint8, device="cuda"))

    def calls(s, out):
        (h, z, dx, dy), v, ws = out
        vec = {n: s[n] for n in VECTORS}
        sdm.block_norm(shape, s["x"], s["y"], h, z, **vec)
        sdm.block_norm_backward(shape, s["y"], h, s["dz"], s["dh"], dx, dy, **vec, **{"d" + n: o for n, o in zip(VECTORS, v)}, workspace=ws)

    one, two = buffers(), buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls(s, one)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(s, one)
    for n, x in new.items():
        s[n].copy_(x)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    graph.replay()
    with torch.cuda.stream(other):
        calls(new, two)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(one[0] + one[1], two[0] + two[1]))


@pytest.mark.gpu
@pytest.mark.parametrize("gate_rows", [1, 4096])
def test_rows_past_32_bits(sdm, gate_rows):  # noqa: F811
    """More than 2^31 values an array: the last rows, the last gate and the vectors' gradients over all of them."""
    import torch
    from dla_reference import block_norm, near, rms_norm
    D, eps, tail = 2048, 1e-5, 61
    M = 2 ** 31 // D + 77
    s = _inputs(M, D, "bf16", gate_rows, "gsop")
    assert s["x"].numel() > 2 ** 31
    vec = {n: s[n] for n in VECTORS}
    shape = sdm.BlockNormShape.make(M, D, dtype="bf16", gate_rows=gate_rows, eps=eps)
    h, z = (torch.full_like(s["x"], math.nan) for _ in range(2))
    sdm.block_norm(shape, s["x"], s["y"], h, z, **vec)
    out = {n: torch.full_like(s[n], math.nan) for n in VECTORS}
    dx, dy = (torch.full_like(s["x"], math.nan) for _ in range(2))
    ws = torch.empty(sdm.block_norm_backward_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    sdm.block_norm_backward(shape, s["y"], h, s["dz"], s["dh"], dx, dy, **vec, **{"d" + n: out[n] for n in VECTORS}, workspace=ws)
    first = M // gate_rows * gate_rows - gate_rows                                       # whole gates up to the end
    rows = slice(first if gate_rows > 1 else M - tail, M)
    gates = s["gate"][first // gate_rows:] if gate_rows > 1 else s["gate"][M - tail:]
    live = {n: vec[n].double().requires_grad_(True) for n in VECTORS if n != "gate"}
    gate, y = gates.double().requires_grad_(True), s["y"][rows].double().requires_grad_(True)
    want_h, _ = block_norm(s["x"][rows], y, gate, live["res_scale"], live["gamma_post"], None, gate_rows, eps)
    near(h[rows], want_h.detach(), "h")
    stored = h[rows].double().requires_grad_(True)
    want_z = rms_norm(stored, live["gamma_pre"], eps)
    near(z[rows], want_z.detach(), "z")
    (pre,) = torch.autograd.grad(want_z, stored, s["dz"][rows].double(), retain_graph=True)
    want_dx = s["dh"][rows].double() + pre
    near(dx[rows], want_dx, "dx")
    want_dy, want_gate = torch.autograd.grad(want_h, (y, gate), want_dx)
    near(dy[rows], want_dy, "dy")
    near(out["gate"][-len(gates):], want_gate, "dgate")
    del y, want_h, want_z, stored, pre, want_dx, want_dy, dx, dy, z, s["x"]
    total = {n: torch.zeros(D, dtype=torch.float64, device="cuda") for n in live}
    for a in range(0, M, 1 << 16):
        b = min(M, a + (1 << 16))
        hh, yy, dz, dh = (t[a:b].double() for t in (h, s["y"], s["dz"], s["dh"]))
        rh, ry = ((t.square().mean(-1, keepdim=True) + eps).rsqrt() for t in (hh, yy))
        dn = dz * vec["gamma_pre"].double()
        g = (dh + rh * (dn - hh * rh * (dn * hh * rh).mean(-1, keepdim=True))) * yy * ry * s["gate"][torch.arange(a, b, device="cuda") // gate_rows].double()
        total["gamma_pre"] += (dz * hh * rh).sum(0)
        total["res_scale"] += (g * vec["gamma_post"].double()).sum(0)
        total["gamma_post"] += (g * vec["res_scale"].double()).sum(0)
    for n in live:
        near(out[n], total[n], "d" + n)
    del s, h, out, vec
    torch.cuda.empty_cache()
