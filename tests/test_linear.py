"""Linear layer with its epilogue and its gradients: argument checks (CPU), parity in 64 bits (GPU).

Tolerances (relative 2-norm): products of bf16 numbers are exact in float32 and their sums over a few
thousand terms are off by about 1e-6, so an output is its one rounding to bf16: at most half of the last
of 8 significant bits, 2^-8.  dx and dW take dz rounded to bf16 as an operand and are rounded; the norms
are over hundreds of independent roundings of at most 2^-8 / sqrt(3) in the root mean square: 2 * 2^-9.
dbias sums unrounded values: 1e-5."""
import ctypes
import os
import shutil

import pytest

TOL, TOL_GRAD, TOL_F32 = 2.0 ** -8, 2 * 2.0 ** -9, 1e-5


@pytest.fixture(scope="module")
def sdm():
    import paper_2607_07386_gb300 as sdm
    from paper_2607_07386_gb300 import build as B
    if not os.path.exists(sdm.lib_path()):
        if shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"):
            pytest.skip("nvcc not available to build libsdm.so")
        B.build()
    return sdm


A = 1 << 24


def _call(sdm, shape, **kw):
    p = dict(x=A, W=2 * A, out=3 * A, workspace=64 * A, workspace_nbytes=1 << 40)
    p.update(kw)
    sdm.linear(shape, stream=0, **p)


def test_struct_layout(sdm):
    assert ctypes.sizeof(sdm.LinearShape) == 24 and sdm.LinearShape.act.offset == 16


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), 1), (dict(N=0), 1), (dict(K=0), 1), (dict(N=12), 2), (dict(K=20), 2), (dict(act=4), 1), (dict(act=-1), 1),
    (dict(M=1 << 24), 2)])
def test_refused_shapes(sdm, kw, status):
    shape = sdm.LinearShape.make(**{**dict(M=64, N=64, K=64), **kw})
    for call in (lambda: _call(sdm, shape), lambda: sdm.linear_workspace_bytes(shape),
                 lambda: sdm.linear_backward_workspace_bytes(shape)):
        with pytest.raises(sdm.SdmError):
            call()
    with pytest.raises(sdm.SdmError) as e:
        _call(sdm, shape)
    assert e.value.status == status


@pytest.mark.parametrize("kw,word", [
    (dict(x=None), "x is NULL"), (dict(W=2 * A + 8), "W is not 16-byte aligned"), (dict(bias=5 * A + 4), "bias is not"),
    (dict(out=A), "out overlaps x"), (dict(pre=3 * A), "overlaps"), (dict(residual=3 * A + 16), "out overlaps residual"),
    (dict(residual=4 * A, pre=4 * A), "overlaps")])
def test_refused_buffers(sdm, kw, word):
    with pytest.raises(sdm.SdmError) as e:
        _call(sdm, sdm.LinearShape.make(64, 64, 64), **kw)
    assert e.value.status == 1 and word in str(e.value)


def test_refused_workspace(sdm):
    shape = sdm.LinearShape.make(64, 64, 4096)
    need = sdm.linear_workspace_bytes(shape)
    assert need > 0
    for kw, word in ((dict(workspace_nbytes=need - 1), "too small"), (dict(workspace=None), "NULL"),
                     (dict(workspace=64 * A + 64), "256-byte")):
        with pytest.raises(sdm.SdmError, match=word):
            _call(sdm, shape, **kw)


def test_backward_refusals(sdm):
    shape = sdm.LinearShape.make(64, 64, 64, act="silu")
    need = sdm.linear_backward_workspace_bytes(shape)
    base = dict(x=A, W=2 * A, pre=3 * A, dout=4 * A, dx=5 * A, dW=6 * A, dbias=7 * A, workspace=64 * A, workspace_nbytes=need)
    for kw, word in ((dict(pre=None), "pre is NULL"), (dict(dout=None), "dout is NULL"), (dict(dx=A), "dx overlaps x"),
                     (dict(dW=5 * A), "overlaps"), (dict(workspace_nbytes=need - 1), "too small")):
        with pytest.raises(sdm.SdmError) as e:
            sdm.linear_backward(shape, stream=0, **{**base, **kw})
        assert e.value.status == 1 and word in str(e.value)


def test_empty_call_does_nothing(sdm):
    _call(sdm, sdm.LinearShape.make(0, 64, 64), x=None, out=None)


# ------------------------------------------------------------------ GPU parity
SIZES = [(1, 8, 8), (2, 40, 2056), (5, 504, 72), (16, 2048, 4104), (17, 64, 64), (100, 136, 8), (128, 256, 64), (129, 264, 200),
         (300, 72, 1032), (1000, 1032, 520), (2500, 1544, 328), (4096, 256, 512)]


def _inputs(M, N, K, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rand(*s):
        return torch.randn(s, generator=g, device="cuda")

    return dict(x=rand(M, K).bfloat16(), W=(rand(N, K) / K ** 0.5).bfloat16(), bias=rand(N), residual=rand(M, N).bfloat16(),
                pre=rand(M, N).bfloat16(), dout=rand(M, N).bfloat16())


def _ws(n):
    import torch
    return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("act,bias,residual,pre", [("none", False, False, False), ("silu", True, True, True),
                                                   ("gelu", True, False, True), ("relu", False, True, False)])
def test_forward_parity(sdm, M, N, K, act, bias, residual, pre):
    import torch
    from gdn_reference import F64, act as f, rel
    t = _inputs(M, N, K, M + N + K)
    z = t["x"].to(F64) @ t["W"].to(F64).mT + (t["bias"].to(F64) if bias else 0)
    want = f(z, act) + (t["residual"].to(F64) if residual else 0)
    shape = sdm.LinearShape.make(M, N, K, act=act)
    out, got = torch.full((M, N), 7.0, dtype=torch.bfloat16, device="cuda"), None
    if pre:
        got = torch.full_like(out, 7.0)
    ws = _ws(sdm.linear_workspace_bytes(shape))
    sdm.linear(shape, t["x"], t["W"], out, bias=t["bias"] if bias else None, residual=t["residual"] if residual else None,
               pre=got, workspace=ws)
    assert sdm.device_status() == 0
    assert rel(out, want) <= TOL
    if pre:
        assert rel(got, z) <= TOL
    if residual:        # in place: the residual's buffer is the output
        inplace = t["residual"].clone()
        sdm.linear(shape, t["x"], t["W"], inplace, bias=t["bias"] if bias else None, residual=inplace, workspace=ws)
        assert torch.equal(inplace, out)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
def test_backward_parity(sdm, M, N, K, act):
    import torch
    from gdn_reference import F64, rel, slope
    t = _inputs(M, N, K, M + N + K + 1)
    dz = t["dout"].to(F64) * slope(t["pre"].to(F64), act)
    shape = sdm.LinearShape.make(M, N, K, act=act)
    dx, dW, db = torch.full_like(t["x"], 7.0), torch.full_like(t["W"], 7.0), torch.full((N,), 7.0, device="cuda")
    ws = _ws(sdm.linear_backward_workspace_bytes(shape))
    sdm.linear_backward(shape, t["x"], t["W"], t["pre"] if act != "none" else None, t["dout"], dx, dW, db, ws)
    assert sdm.device_status() == 0
    assert rel(dx, dz @ t["W"].to(F64)) <= TOL_GRAD
    assert rel(dW, dz.mT @ t["x"].to(F64)) <= TOL_GRAD
    # column sums may cancel: measured against the sums of magnitudes
    assert float((db.to(F64) - dz.sum(0)).abs().max()) <= TOL_F32 * float(dz.abs().sum(0).max())
    dx2, db2 = torch.empty_like(dx), torch.empty_like(db)
    sdm.linear_backward(shape, t["x"], t["W"], t["pre"], t["dout"], dx2, None, None, ws)
    sdm.linear_backward(shape, t["x"], t["W"], t["pre"], t["dout"], None, None, db2, ws)
    assert torch.equal(dx, dx2) and torch.equal(db, db2)


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["relu", "silu", "gelu"])
def test_backward_against_differences(sdm, act):
    """Directional differences of the 64-bit forward in x, W and bias at step 1e-4, with pre as the library
    stores it (rounded to bf16: its slope is off by up to 2^-9 of a slope that changes by O(1))."""
    import torch
    from gdn_reference import F64, act as f
    M, N, K = 200, 72, 136
    t = _inputs(M, N, K, 5)
    shape = sdm.LinearShape.make(M, N, K, act=act)
    out, pre = torch.empty((M, N), dtype=torch.bfloat16, device="cuda"), torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    sdm.linear(shape, t["x"], t["W"], out, bias=t["bias"], pre=pre, workspace=_ws(sdm.linear_workspace_bytes(shape)))
    g = dict(x=torch.empty_like(t["x"]), W=torch.empty_like(t["W"]), bias=torch.empty_like(t["bias"]))
    sdm.linear_backward(shape, t["x"], t["W"], pre, t["dout"], g["x"], g["W"], g["bias"],
                        _ws(sdm.linear_backward_workspace_bytes(shape)))

    def loss(v):
        return (f(v["x"] @ v["W"].mT + v["bias"], act) * t["dout"].to(F64)).sum()

    base = {n: t[n].to(F64) for n in ("x", "W", "bias")}
    for n in base:
        d = g[n].to(F64) / g[n].to(F64).norm()
        want = float(loss({**base, n: base[n] + 1e-4 * d}) - loss({**base, n: base[n] - 1e-4 * d})) / 2e-4
        assert abs(want - float(g[n].to(F64).norm())) <= 4 * 2.0 ** -9 * abs(want), n


@pytest.mark.gpu
def test_backward_of_no_rows(sdm):
    import torch
    shape = sdm.LinearShape.make(0, 64, 32, act="silu")
    e = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    dW, db = torch.full((64, 32), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((64,), 7.0, device="cuda")
    W = torch.ones((64, 32), dtype=torch.bfloat16, device="cuda")
    sdm.linear_backward(shape, torch.empty((0, 32), dtype=torch.bfloat16, device="cuda"), W, e, e, None, dW, db)
    assert (dW == 0).all() and (db == 0).all()


@pytest.mark.gpu
def test_infinities_stay_in_their_rows_and_columns(sdm):
    """A row of x with infinities, NaN in a column of W: other outputs are those without them."""
    import torch
    t = _inputs(200, 136, 72, 6)
    shape = sdm.LinearShape.make(200, 136, 72)
    ws = _ws(sdm.linear_workspace_bytes(shape))
    out, bad = torch.empty((200, 136), dtype=torch.bfloat16, device="cuda"), torch.empty((200, 136), dtype=torch.bfloat16, device="cuda")
    sdm.linear(shape, t["x"], t["W"], out, workspace=ws)
    t["x"][7] = float("inf")
    t["W"][11] = float("nan")
    sdm.linear(shape, t["x"], t["W"], bad, workspace=ws)
    keep_r = torch.arange(200, device="cuda") != 7
    keep_c = torch.arange(136, device="cuda") != 11
    assert torch.equal(out[keep_r][:, keep_c], bad[keep_r][:, keep_c])
    assert torch.isnan(bad[:, 11]).all() and not torch.isfinite(bad[7]).any()


# 128 x 256 tiles in every order of the operands, over more K-blocks than the ring holds, with an odd number of row
# tiles: x W^T at exactly 76 tiles (and two splits), x W^T and dz W at 95 and 133, x W^T and dz^T x at 90 and 95.
WIDE = [(2305, 1024, 520), (2305, 1032, 1544), (1100, 2312, 1032)]


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", WIDE)
def test_wide_tiles(sdm, M, N, K):
    test_forward_parity(sdm, M, N, K, "silu", True, True, True)
    test_backward_parity(sdm, M, N, K, "gelu")


def test_no_load_is_shared_between_ctas():
    """Every rank of a run on several GPUs loads this library, and a caller's matrix may be in another GPU's memory:
    no copy of a source goes to more than one CTA's shared memory."""
    import re
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_07386_gb300", "csrc")
    shared = re.compile("multi" + "cast", re.I)
    names = sorted(n for n in os.listdir(csrc) if n.endswith((".cu", ".cuh", ".h")))
    assert names and [n for n in names if shared.search(open(os.path.join(csrc, n)).read())] == []


@pytest.mark.parametrize("M,N,K", [(64, 64, 64), (64, 72, 64), (4096, 2048, 2048), (64, 4096, 4096), (16, 64, 64), (16, 64, 16)])
def test_only_the_residual_may_be_the_output(sdm, M, N, K):
    """In place over x or W is refused, with the residual there too: tiles, split tiles and up to 16 rows."""
    shape = sdm.LinearShape.make(M, N, K)
    far = dict(x=1 << 40, W=1 << 41, workspace=1 << 42)
    for other in [n for n, same in (("x", N == K), ("W", M == K)) if same]:
        with pytest.raises(sdm.SdmError, match="out overlaps " + other):
            _call(sdm, shape, **{**far, other: 3 * A, "residual": 3 * A})


@pytest.mark.gpu
@pytest.mark.parametrize("M", [5, 200])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
def test_nan_is_not_lost(sdm, act, M):
    """A NaN in a row of x is in every output of the row; one pre-activation's is in its row of dx, its row of dW and its
    dbias, and nowhere else."""
    import torch
    N, K = 72, 136
    t = _inputs(M, N, K, 8)
    t["x"][3, 9] = float("nan")
    shape = sdm.LinearShape.make(M, N, K, act=act)
    out, pre = (torch.empty((M, N), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    sdm.linear(shape, t["x"], t["W"], out, bias=t["bias"], pre=pre, workspace=_ws(sdm.linear_workspace_bytes(shape)))
    row = torch.arange(M, device="cuda") == 3
    assert torch.equal(torch.isnan(out), row[:, None].expand(M, N)) and torch.equal(torch.isnan(pre), torch.isnan(out))
    if act == "none":
        return
    t["x"][3, 9] = 1.0
    t["pre"][3, 11] = float("nan")
    dx, dW, db = torch.empty_like(t["x"]), torch.empty_like(t["W"]), torch.empty((N,), device="cuda")
    sdm.linear_backward(shape, t["x"], t["W"], t["pre"], t["dout"], dx, dW, db, _ws(sdm.linear_backward_workspace_bytes(shape)))
    col = torch.arange(N, device="cuda") == 11
    assert torch.equal(torch.isnan(dx), row[:, None].expand(M, K))
    assert torch.equal(torch.isnan(dW), col[:, None].expand(N, K)) and torch.equal(torch.isnan(db), col)
