"""The norm of many gradients and clipping: argument checks (CPU) and parity with 64-bit references (GPU).

Tolerances: the norm is a float32 square root of sums of at most 32 float32 squares per thread and block, joined in 64 bits:
1e-6.  A clipped value is a product with a factor off by that much, rounded once to its type (half a step)."""
import ctypes
import math

import pytest

from test_dla import A, sdm  # noqa: F401


def _entries(sdm, *rows):
    """(grad, out, n, dtype, out_dtype) rows of raw addresses."""
    from paper_2607_07386_gb300._binding import GradTensor
    return sdm.GradList([GradTensor(*r) for r in rows], None)


def _clip(sdm, rows, max_norm=1.0, stats=50 * A, ws=64 * A, nb=1 << 40, call="grad_clip"):
    getattr(sdm, call)(_entries(sdm, *rows), max_norm, stats, ws, stream=0, workspace_nbytes=nb)


def test_struct_layout(sdm):  # noqa: F811
    from paper_2607_07386_gb300._binding import GradTensor
    assert ctypes.sizeof(GradTensor) == 32 and GradTensor.out_dtype.offset == 28


GOOD = (A, A, 100, 0, 0)


@pytest.mark.parametrize("rows,kw,status,word", [
    ([GOOD], dict(max_norm=-1.0), 1, "max_norm"), ([GOOD], dict(max_norm=math.nan), 1, "max_norm"), ([GOOD], dict(stats=None), 1, "stats is NULL"),
    ([GOOD], dict(stats=50 * A + 2), 1, "stats is not"), ([GOOD], dict(ws=None), 1, "workspace is NULL"), ([GOOD], dict(ws=64 * A + 8), 1, "256-byte"),
    ([GOOD], dict(nb=4), 1, "too small"), ([(A, A, -1, 0, 0)], {}, 1, "n = -1"), ([(A, A, 4, 2, 0)], {}, 1, "dtype"), ([(A, 2 * A, 4, 0, 5)], {}, 1, "dtype"),
    ([(None, A, 4, 0, 0)], {}, 1, "NULL"), ([(A, None, 4, 0, 0)], {}, 1, "NULL"), ([(A + 2, A + 2, 4, 0, 0)], {}, 1, "aligned"),
    ([(A + 1, 2 * A, 4, 1, 1)], {}, 1, "aligned"), ([(A, A, 4, 0, 1)], {}, 1, "in place"), ([GOOD, GOOD], {}, 1, "overlaps"),
    ([GOOD, (A + 396, 3 * A, 4, 0, 0)], {}, 1, "overlaps"), ([(A, 2 * A, 100, 0, 0), (3 * A, 2 * A + 396, 4, 0, 0)], {}, 1, "overlaps"),
    ([(A, A + 4, 100, 0, 0)], {}, 1, "overlaps"), ([GOOD], dict(stats=A + 16), 1, "overlaps"), ([(64 * A, 64 * A, 9, 0, 0)], {}, 1, "workspace"),
    ([(A, 3 * A, 1 << 41, 0, 0)], {}, 2, "2^40")])
def test_refusals(sdm, rows, kw, status, word):  # noqa: F811
    with pytest.raises(sdm.SdmError) as e:
        _clip(sdm, rows, **kw)
    assert e.value.status == status and word in str(e.value)


def test_refused_lists(sdm):  # noqa: F811
    import torch
    for grads, out in (([torch.zeros(3)], None), ([torch.zeros(3, dtype=torch.float64)], None)):
        with pytest.raises(ValueError):
            sdm.GradList.make(grads, out)
    with pytest.raises(sdm.SdmError):
        sdm.grad_workspace_bytes(_entries(sdm, (A, A, -3, 0, 0)))
    many = [((i + 100) * 4096, (i + 100) * 4096, 1024, 0, 0) for i in range(400)]
    many[399] = (100 * 4096, 100 * 4096, 1, 0, 0)            # a long list, its last tensor over its first
    with pytest.raises(sdm.SdmError, match="tensor 399|tensor 0"):
        _clip(sdm, many, stats=1 << 40, ws=1 << 41)


def test_reading_twice_is_allowed(sdm):  # noqa: F811
    """Sizes only: the same gradient twice, out of place and for the norm."""
    assert sdm.grad_workspace_bytes(_entries(sdm, (A, 3 * A, 100, 0, 0), (A, 5 * A, 100, 0, 0))) > 0
    assert sdm.grad_workspace_bytes(_entries(sdm)) == 0


# ------------------------------------------------------------------ parity
def _run(sdm, grads, out, max_norm, call="grad_clip"):
    import torch
    lst = sdm.GradList.make(grads, out)
    stats = torch.full((2,), -1.0, device="cuda")
    n = sdm.grad_workspace_bytes(lst)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") if n else None
    getattr(sdm, call)(lst, max_norm, stats, ws)
    return stats.tolist()


def _norm(grads):
    return math.sqrt(sum(float((g.double() * 2.0 ** -100).square().sum()) for g in grads)) * 2.0 ** 100


def _flat(sizes, types, seed=0, offset=0):
    """Pieces of one buffer per type, so that most begin off 16 bytes."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    out, at = [], dict.fromkeys(set(types), offset)
    flat = {t: torch.randn(sum(n for n, u in zip(sizes, types) if u == t) + offset, generator=g, device="cuda").to(t) for t in at}
    for n, t in zip(sizes, types):
        out.append(flat[t][at[t]:at[t] + n])
        at[t] += n
    return out


SIZES = [1, 3, 0, 8191, 8192, 8193, 16384, 40001, 7, 300000, 2]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_norm_and_clip(sdm, kind, offset):  # noqa: F811
    import torch
    f, b = torch.float32, torch.bfloat16
    types = {"f32": [f], "bf16": [b], "mixed": [f, b, b]}[kind] * len(SIZES)
    grads = _flat(SIZES, types, offset=offset)
    want = _norm(grads)
    kept = [g.clone() for g in grads]
    for limit in (want * 0.01, want * 2, 0.0, math.inf):
        factor = min(1.0, limit / want)
        stats = _run(sdm, grads, None, limit, "grad_norm")
        assert abs(stats[0] - want) <= 1e-6 * want and abs(stats[1] - factor) <= 1e-6 * factor
        assert all(torch.equal(a, c) for a, c in zip(grads, kept))
        for outs in ([torch.full_like(g, math.nan) for g in grads], _flat(SIZES, types[::-1], offset=1),
                     [torch.full(g.shape, math.nan, device="cuda", dtype=f if g.dtype == b else b) for g in grads], None):
            assert _run(sdm, grads, outs, limit) == stats
            for g, o in zip(kept, grads if outs is None else outs):
                half = 2.0 ** -8 if o.dtype == b else 2.0 ** -24
                assert ((o.double() - g.double() * factor).abs() <= (half + 1e-6) * (g.double() * factor).abs()).all()
        for g, c in zip(grads, kept):
            g.copy_(c)


@pytest.mark.gpu
def test_many_tensors_and_repeats(sdm):  # noqa: F811
    """More tensors than one launch takes, between guards that stay; the same result every time; a tensor given twice counts twice."""
    import torch
    sizes = [1 + (37 * i) % 5000 for i in range(700)]
    g = torch.Generator(device="cuda").manual_seed(3)
    flat = torch.randn(sum(sizes) + len(sizes), generator=g, device="cuda").bfloat16()
    grads, at = [], 0
    guard = torch.zeros(flat.numel(), dtype=torch.bool, device="cuda")
    for n in sizes:
        grads.append(flat[at:at + n])
        guard[at + n] = True
        at += n + 1
    before = flat.clone()
    want = _norm(grads)
    first = _run(sdm, grads, None, want / 4, "grad_norm")
    assert abs(first[0] - want) <= 1e-6 * want and all(_run(sdm, grads, None, want / 4, "grad_norm") == first for _ in range(3))
    assert _run(sdm, grads, None, want / 4) == first
    assert torch.equal(flat[guard], before[guard])
    clipped = before[~guard].double() * 0.25
    assert ((flat[~guard].double() - clipped).abs() <= (2.0 ** -8 + 1e-6) * clipped.abs()).all()
    twice = _run(sdm, [grads[5], grads[5]], [torch.empty_like(grads[5]) for _ in range(2)], 1.0)
    assert abs(twice[0] - math.sqrt(2) * _norm([grads[5]])) <= 1e-6 * twice[0]


def _list_sizes(filled, empty):
    """`filled` sizes of up to three blocks' values, with empty tensors at the places given."""
    sizes = [1 + (977 * i) % 20011 if i % 50 == 0 else 1 + (37 * i) % 700 for i in range(filled)]
    for at in sorted(empty):
        sizes.insert(at, 0)
    return sizes


@pytest.mark.gpu
@pytest.mark.parametrize("filled,empty", [(64, []), (65, []), (64, [0, 64, 65]), (960, []), (960, [960, 961, 962]), (961, []), (961, [960]),
                                          (2000, [0, 960, 961, 1922, 2003]), (2881, [])])
@pytest.mark.parametrize("kind", ["f32", "mixed"])
def test_lists_at_and_past_a_launch(sdm, filled, empty, kind):  # noqa: F811
    """A launch takes up to 64 or up to 960 tensors: lists of one, of several, and with empty tensors where one ends.  The
    workspace is as long as asked for and no longer."""
    import torch
    sizes = _list_sizes(filled, empty)
    f, b = torch.float32, torch.bfloat16
    types = [f if kind == "f32" or i % 3 == 0 else b for i in range(len(sizes))]
    grads = _flat(sizes, types, seed=filled)
    kept = [g.clone() for g in grads]
    outs = [torch.full_like(g, math.nan) for g in grads]
    want = _norm([torch.cat([g.double() for g in grads])])
    limit = want / 4
    for out, call in ((None, "grad_norm"), (outs, "grad_clip"), (None, "grad_clip")):
        lst = sdm.GradList.make(grads, out)
        n = sdm.grad_workspace_bytes(lst)
        ws = torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        stats = torch.full((4,), -1.0, device="cuda")
        getattr(sdm, call)(lst, limit, stats[:2], ws, workspace_nbytes=n)
        assert (ws[n:] == 0xA5).all() and (stats[2:] == -1).all()
        norm, factor = stats[:2].tolist()
        assert abs(norm - want) <= 1e-6 * want and abs(factor - 0.25) <= 1e-6 * 0.25
        if call == "grad_norm":
            assert all(torch.equal(g, k) for g, k in zip(grads, kept))
            first = stats.clone()
            continue
        assert torch.equal(stats, first)                     # whichever call, however often
        for t, half in ((f, 2.0 ** -24), (b, 2.0 ** -8)):
            if t not in types:
                continue
            o, g = (torch.cat([x for x, u in zip(xs, types) if u == t]).double() for xs in (grads if out is None else out, kept))
            assert ((o - g * 0.25).abs() <= (half + 1e-6) * (g * 0.25).abs()).all()
    with pytest.raises(sdm.SdmError, match="too small"):
        sdm.grad_clip(lst, limit, stats[:2], ws, workspace_nbytes=n - 1)


@pytest.mark.gpu
@pytest.mark.parametrize("size", [1e38, 1e30, 1e-15, 1e-25, 1e-36])
def test_whole_range_of_values(sdm, size):  # noqa: F811
    """Gradients whose squares float32 does not hold."""
    import torch
    grads = [g * size if i else g * size * 1e-3 for i, g in enumerate(_flat([5, 40], [torch.float32] * 2))]
    grads = [g.clamp(-1e38, 1e38) / 8 for g in grads]
    want = _norm(grads)
    kept = [g.clone() for g in grads]
    stats = _run(sdm, grads, None, want / 3)
    assert abs(stats[0] - want) <= 1e-6 * want and abs(stats[1] - 1 / 3) <= 1e-6
    for a, c in zip(grads, kept):
        assert ((a.double() - c.double() / 3).abs() <= 1e-6 * c.double().abs() + 2.0 ** -149).all()


@pytest.mark.gpu
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("place", [0, 12345])
def test_not_finite(sdm, value, place):  # noqa: F811
    """The norm says so, the factor is NaN, and the gradients are left (or copied) as they are."""
    import torch
    for t in (torch.float32, torch.bfloat16):
        grads = _flat([40000, 17], [t, t])
        grads[0][place] = value
        kept, outs = [g.clone() for g in grads], [torch.empty_like(g) for g in grads]
        for o in (outs, None):
            norm, factor = _run(sdm, grads, o, 1.0)
            assert not math.isfinite(norm) and math.isnan(factor) and math.isnan(norm) == math.isnan(value)
            for a, c in zip(grads if o is None else o, kept):
                assert torch.equal(a.view(torch.int16 if t == torch.bfloat16 else torch.int32), c.view(torch.int16 if t == torch.bfloat16 else torch.int32))


@pytest.mark.gpu
def test_nothing_to_clip(sdm):  # noqa: F811
    import torch
    assert _run(sdm, [], None, 1.0) == [0.0, 1.0]
    assert _run(sdm, [torch.empty(0, device="cuda")], None, 1.0) == [0.0, 1.0]
    zeros = torch.zeros(100, device="cuda")
    assert _run(sdm, [zeros], None, 0.0) == [0.0, 1.0] and not zeros.any()


@pytest.mark.gpu
def test_captured(sdm):  # noqa: F811
    """A captured call holds its list: the host's may go."""
    import torch
    grads = _flat([5000, 123457, 9], [torch.float32, torch.bfloat16, torch.float32])
    outs = [torch.empty_like(g) for g in grads]
    lst = sdm.GradList.make(grads, outs)
    stats, ws = torch.empty(2, device="cuda"), torch.empty(sdm.grad_workspace_bytes(lst), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sdm.grad_clip(lst, 2.0, stats, ws)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sdm.grad_clip(lst, 2.0, stats, ws)
    for i in range(len(grads)):
        lst.array[i].grad, lst.array[i].n = None, 0
    for g in grads:
        g.mul_(0.5)
    want = _norm(grads)
    graph.replay()
    torch.cuda.synchronize()
    assert abs(float(stats[0]) - want) <= 1e-6 * want
    for g, o in zip(grads, outs):
        assert ((o.double() - g.double() * (2 / want)).abs() <= ((2.0 ** -8 if o.dtype == torch.bfloat16 else 2.0 ** -24) + 1e-6) * (g.double() * (2 / want)).abs()).all()


@pytest.mark.gpu
@pytest.mark.parametrize("out", [None, "f32"])
def test_a_tensor_past_32_bits(sdm, out):  # noqa: F811
    """One gradient of more than 2^31 values, off 16 bytes, and a small one behind it; what lies after them stays."""
    import torch
    n = 2 ** 31 + 12345
    g = torch.Generator(device="cuda").manual_seed(1)
    buf = torch.empty(n + 64, dtype=torch.bfloat16, device="cuda")
    for a in range(0, buf.numel(), 1 << 28):
        part = buf[a:a + (1 << 28)]
        part.copy_(torch.randn(part.numel(), generator=g, device="cuda"))
    grads = [buf[3:3 + n], buf[3 + n:20 + n]]
    kept = {a: buf[a:a + 4096].clone() for a in (0, 2 ** 31 - 2048, buf.numel() - 4096)}
    want = math.sqrt(sum(float(buf[3:20 + n][a:a + (1 << 28)].double().square().sum()) for a in range(0, n + 17, 1 << 28)))
    outs = None if out is None else [torch.full((x.numel(),), math.nan, device="cuda") for x in grads]
    norm, factor = _run(sdm, grads, outs, want / 4)
    assert abs(norm - want) <= 1e-6 * want and abs(factor - 0.25) <= 1e-6 * 0.25
    half = 2.0 ** -8 if outs is None else 2.0 ** -24
    for a, before in kept.items():
        end = a + 4096
        lo, hi = max(a, 3), min(end, 3 + n)
        got = buf[lo:hi] if outs is None else outs[0][lo - 3:hi - 3]
        x = before[lo - a:hi - a].double() * 0.25
        assert ((got.double() - x).abs() <= (half + 1e-6) * x.abs()).all(), a
        assert torch.equal(buf[a:lo], before[:lo - a]) and torch.equal(buf[20 + n:][:end - 20 - n], before[20 + n - a:] if end > 20 + n else before[:0])
    last = buf[3 + n:20 + n] if outs is None else outs[1]
    x = kept[buf.numel() - 4096][3 + n - (buf.numel() - 4096):][:17].double() * 0.25
    assert ((last.double() - x).abs() <= (half + 1e-6) * x.abs()).all()
    del buf, grads, outs, last, got
    torch.cuda.empty_cache()
