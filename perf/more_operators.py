"""Linear attention with a decay per head, the norms around a block and gradient clipping: what is timed, and
the operators' plain forms.

Decayed linear attention, per sequence and value head, state S [d_k, d_v], lam_h = exp(log_decay_h):
    S_t = lam_h S_{t-1} + k_t v_t^T,  y_t = scale S_t^T q_t.
Block norm, per row: u = gamma_post y / rms(y);  h = x + res_scale gate u;  z = gamma_pre h / rms(h).
Clipping: norm = sqrt(sum over all tensors of g^2);  g min(1, max_norm / norm).

`own` chooses between the plain forms (elementary torch operations in 32 bits) and the library's
entry points.  Sizes follow synth/configs.py: heads of 64 and 128, 16 heads, d_model = 16 * 128.
"""
import math

import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
CHUNK = 64
EPS = 1e-6


def listed():
    return [
        # one sequence being decoded: the latency of a single small call
        dict(name="step_one", op="step", B=1, H=16, Hk=16, dk=128, dv=128, dtype="bf16", slots=1, layout="head_major"),
        # a serving batch (the decode workload's B and H) over a larger cache of states
        dict(name="step_serving", op="step", B=256, H=16, Hk=16, dk=128, dv=128, dtype="bf16", slots=288,
             layout="head_major"),
        # a padded batch of a few long prompts, key heads shared by two value heads, in the layout that projections write
        dict(name="forward_ragged", op="forward", B=3, H=8, Hk=4, T=6011, dk=128, dv=128, dtype="bf16", ragged=True,
             layout="token_major"),
        # the 1.4B layer's training and prefill shape
        dict(name="forward_layer", op="forward", B=8, H=16, Hk=16, T=4096, dk=128, dv=128, dtype="bf16", ragged=False,
             layout="head_major"),
        # a small fp32 model's training step at odd sizes
        dict(name="backward_f32_odd", op="backward", B=3, H=6, Hk=3, T=333, dk=64, dv=96, dtype="f32", ragged=True,
             layout="head_major"),
        # training of the 1.4B layer
        dict(name="backward_layer", op="backward", B=8, H=16, Hk=16, T=4096, dk=128, dv=128, dtype="bf16",
             ragged=False, layout="head_major"),
        # around a block while one token is decoded
        dict(name="norm_decode", op="norm", M=1, D=2048, dtype="bf16", gate_rows=1, post=True, scale=True, gate=True, pre=True),
        # around a block of the 1.4B model in training or prefill, the gate shared by the tokens of a sequence
        dict(name="norm_layer", op="norm", M=32768, D=2048, dtype="bf16", gate_rows=4096, post=True, scale=True, gate=True,
             pre=True),
        # gradients in a small fp32 model at odd sizes, a gate for every token
        dict(name="norm_backward_odd", op="norm_backward", M=1531, D=1548, dtype="f32", gate_rows=1, post=True, scale=True,
             gate=True, pre=True),
        # gradients around a block of the 1.4B model
        dict(name="norm_backward_layer", op="norm_backward", M=32768, D=2048, dtype="bf16", gate_rows=4096, post=True,
             scale=True, gate=True, pre=True),
        # clipping in a small fp32 model of two layers: many small tensors
        dict(name="clip_small", op="clip", layers=2, H=4, d=64, N=4096, dtype="f32", clips=True),
        # clipping of two layers with a learned initial memory each, whose gradient is fp32; the weights' is bf16
        dict(name="clip_memory", op="clip", layers=2, H=16, d=128, N=65536, dtype="bf16", clips=True),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["step", "forward", "forward", "backward", "backward", "norm", "norm_backward", "clip"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op in ("norm", "norm_backward"):
        c = dict(op=op, M=log(1, 32768), D=8 * log(8, 1024), dtype=dtype, gate_rows=1, post=rng.random() < 0.8,
                 scale=rng.random() < 0.6, gate=rng.random() < 0.7, pre=rng.random() < 0.9)
        while c["M"] * c["D"] * (2 if dtype == "f32" else 1) > 32768 * 2048:
            c["M"] = max(1, c["M"] // 2)
        c["gate_rows"] = rng.choice([1, 1, log(1, c["M"]), c["M"]])
        return c
    if op == "clip":
        c = dict(op=op, layers=log(1, 24), H=rng.choice([1, 3, 4, 8, 16]), d=rng.choice([32, 37, 64, 96, 128]),
                 N=rng.choice([0, 0, 37 * 37, 4096, 65536]), dtype=dtype, clips=rng.random() < 0.75)
        while sum(n * 4 for n, _ in _tensors(c)) > 2 * 16 * 65536 * 128 * 4:
            c["layers"] = max(1, c["layers"] // 2)
            if c["layers"] == 1:
                break
        return c
    Hk = rng.choice([1, 2, 4, 5, 8, 16])
    c = dict(op=op, Hk=Hk, H=Hk * rng.choice([1, 1, 2, 3]), dk=rng.choice([32, 64, 96, 128, 128, 128, 160]),
             dv=rng.choice([32, 64, 96, 128, 128, 128, 192]), dtype=dtype, layout=rng.choice(["head_major", "token_major"]))
    if op == "step":
        c["B"] = log(1, 256)
        while c["B"] * c["H"] * c["dk"] * c["dv"] > 256 * 16 * 128 * 128:
            c["B"] = max(1, c["B"] // 2)
        c["slots"] = c["B"] + rng.randrange(0, 33)
        return c
    c.update(B=log(1, 8), T=log(1, 12000 if dtype == "bf16" else 2048), ragged=rng.random() < 0.5)
    while c["B"] * c["H"] * c["T"] * c["dk"] * c["dv"] > 8 * 16 * 4096 * 128 * 128:
        c["T"] = max(1, c["T"] // 2)
    return c


def _tensors(c):
    """Sizes and types of the gradients of a model's weights: per layer the four projections, the gates' weights, the
    score projections and the initial memory, and what is one-dimensional, the last in 32 bits as the memory."""
    dm, w, out = c["H"] * c["d"], c["dtype"], []
    for _ in range(c["layers"]):
        out += [(dm * dm, w)] * 4 + [(c["H"] * dm, w)] * 2 + [(c["H"], "f32")] * 2 + [(c["d"], "f32"), (dm, "f32"), (dm, "f32")]
        if c["N"]:
            out += [(c["H"] * 2 * math.isqrt(c["N"]) * c["d"], w)] * 2 + [(c["H"] * c["N"] * c["d"], "f32")]
    return out + [(1, "f32")]


def _pieces(flat, c):
    at, out = dict.fromkeys(flat, 0), []
    for n, t in _tensors(c):
        out.append(flat[t][at[t]:at[t] + n])
        at[t] += n
    return out


def work(case):
    c = case
    if c["op"] == "clip":
        size = {"f32": 4, "bf16": 2}
        return {"bytes": sum(2 * n * size[t] for n, t in _tensors(c)), "flops": sum(3 * n for n, _ in _tensors(c))}
    es = 4 if c["dtype"] == "f32" else 2
    if c["op"] in ("norm", "norm_backward"):
        M, D = c["M"], c["D"]
        rows = M * D * es
        gates = -(-M // c["gate_rows"]) * D * es * c["gate"]
        vectors = 4 * D * (c["post"] + c["scale"] + c["pre"])
        if c["op"] == "norm":
            return {"bytes": rows * (3 + c["pre"]) + gates + vectors, "flops": 14 * M * D}
        return {"bytes": rows * (5 + c["pre"]) + 2 * gates + 2 * vectors, "flops": 30 * M * D}
    T = c.get("T", 1)
    tokens = sum(_lengths(c)) if c.get("ragged") else c["B"] * T
    qk, vy = tokens * c["Hk"] * c["dk"] * es, tokens * c["H"] * c["dv"] * es
    state = c["B"] * c["H"] * c["dk"] * c["dv"] * 4
    mul = tokens * c["H"] * c["dk"] * c["dv"]
    pad = (c["B"] * T - tokens) * es                             # zeros past the lengths
    if c["op"] == "backward":        # q, k, v, dy, S_0, dS_T in; dq, dk, dv, dS_0 out
        return {"bytes": 4 * qk + 3 * vy + 3 * state + pad * (2 * c["Hk"] * c["dk"] + c["H"] * c["dv"]), "flops": 12 * mul}
    return {"bytes": 2 * qk + 2 * vy + 2 * state + pad * c["H"] * c["dv"], "flops": 5 * mul}


def _lengths(c):
    """Lengths of a ragged batch, from none of the tokens (five sequences and more) to all of them."""
    B, T = c["B"], c["T"]
    return [T - (T * i * i) // max(1, (B - 1) ** 2 + (B <= 4)) if B > 1 else T - T // 3 for i in range(B)]


def _order(x, c):
    """[B, H, T, d] -> the case's layout."""
    return x.transpose(1, 2).contiguous() if c["layout"] == "token_major" else x.contiguous()


def _inputs(case, seed, device):
    """Every input tensor of a case; sums and norms of the recipe in 32 bits."""
    c = case
    g = torch.Generator(device=device)
    g.manual_seed(seed)

    def rand(*shape):
        return torch.randn(shape, generator=g, device=device, dtype=torch.float32)

    s = {}
    if c["op"] == "clip":
        # the gradients are pieces of one buffer per type, one after the other
        s["flat"] = {t: (rand(sum(n for n, u in _tensors(c) if u == t)) * 0.01).to(DT[t]) for t in sorted({u for _, u in _tensors(c)})}
        s["grads"] = _pieces(s["flat"], c)
        total = 0.01 * math.sqrt(sum(n for n, _ in _tensors(c)))
        s["max_norm"] = total * (0.1 if c["clips"] else 10)
        return s
    dt = DT[c["dtype"]]
    if c["op"] in ("norm", "norm_backward"):
        M, D = c["M"], c["D"]
        s["y"] = (rand(M, D) * 0.7).to(dt)
        s["x"] = (rand(M, D) * 2).to(dt)
        s["gate"] = torch.sigmoid(rand(-(-M // c["gate_rows"]), D)).to(dt) if c["gate"] else None
        s["res_scale"] = 0.3 + 0.1 * rand(D) if c["scale"] else None
        s["gamma_post"] = 1 + 0.1 * rand(D) if c["post"] else None
        s["gamma_pre"] = 1 + 0.1 * rand(D) if c["pre"] else None
        if c["op"] == "norm_backward":                       # the residual stream as the forward left it
            s["h"] = s.pop("x")
            s["dz"] = rand(M, D).to(dt) if c["pre"] else None
            s["dh"] = rand(M, D).to(dt)
        return s
    B, H, Hk, T, dk, dv = c["B"], c["H"], c["Hk"], c.get("T", 1), c["dk"], c["dv"]

    def unit(*shape):
        x = rand(*shape)
        return x / x.square().sum(-1, keepdim=True).sqrt()

    s["q"] = _order(unit(B, Hk, T, dk).to(dt), c)
    s["k"] = _order(unit(B, Hk, T, dk).to(dt), c)
    s["v"] = _order(rand(B, H, T, dv).to(dt), c)
    # memories of 2 to 4096 tokens, spread over the heads
    at = (torch.arange(H, device=device) + torch.rand(H, generator=g, device=device)) / H
    s["log_decay"] = -torch.exp2(-1 - 11 * at)
    n = c["slots"] if c["op"] == "step" else B
    s["state"] = rand(n, H, dk, dv) * 0.3
    s["slots"] = None
    if c["op"] == "step" and c["slots"] > B:
        s["slots"] = torch.randperm(n, generator=g, device=device)[:B].to(torch.int32)
    s["lengths"] = torch.tensor(_lengths(c), dtype=torch.int32, device=device) if c.get("ragged") else None
    if c["op"] == "backward":
        s["dy"] = _order(rand(B, H, T, dv).to(dt), c)
        s["dstate"] = rand(B, H, dk, dv) * 0.3
    return s


def prepare(case, seed):
    s = _inputs(case, seed, "cuda")
    s["case"] = dict(case)
    c = case

    def like(x):
        return None if x is None else torch.empty_like(x)

    if c["op"] == "clip":
        s["to"] = {t: like(x) for t, x in s["flat"].items()}
        s["clipped"] = _pieces(s["to"], c)
        s["stats"] = torch.empty(2, device="cuda")
    elif c["op"] == "norm":
        s["h"], s["z"] = like(s["x"]), like(s["x"]) if c["pre"] else None
    elif c["op"] == "norm_backward":
        s["dx"], s["dy"] = like(s["h"]), like(s["y"])
        for n in ("gate", "res_scale", "gamma_post", "gamma_pre"):
            s["d" + n] = like(s[n])
    else:
        s["y"] = like(s["v"])
        if c["op"] == "backward":
            for n in ("q", "k", "v", "state"):
                s["d" + n + ("0" if n == "state" else "")] = like(s[n])
    return s


# ------------------------------------------------------------------ the framework's calls
def _plan(s):
    """The shape and the workspace, made once and kept with the state as a user's program keeps them."""
    import paper_2607_07386_gb300 as sdm
    c = s["case"]
    if c["op"] == "clip":
        shape = sdm.GradList.make(s["grads"], s["clipped"])
        n = sdm.grad_workspace_bytes(shape)
    elif c["op"] in ("norm", "norm_backward"):
        shape = sdm.BlockNormShape.make(c["M"], c["D"], dtype=c["dtype"], gate_rows=c["gate_rows"], eps=EPS)
        n = sdm.block_norm_backward_workspace_bytes(shape) if c["op"] == "norm_backward" else 0
    else:
        shape = sdm.DlaShape.make(c["B"], c["H"], c.get("T", 1), c["dk"], c["dv"], H_k=c["Hk"], dtype=c["dtype"],
                                  layout=c["layout"], scale=c["dk"] ** -0.5)
        n = {"step": lambda sh: 0, "forward": sdm.dla_workspace_bytes,
             "backward": sdm.dla_backward_workspace_bytes}[c["op"]](shape)
    s["plan"] = (sdm, shape, torch.empty(n, dtype=torch.uint8, device="cuda") if n else None)
    return s["plan"]


def _run_own(s):
    sdm, shape, ws = s.get("plan") or _plan(s)
    op = s["case"]["op"]
    if op == "clip":
        sdm.grad_clip(shape, s["max_norm"], s["stats"], ws)
        return {"stats": s["stats"], **s["to"]}
    if op == "norm":
        sdm.block_norm(shape, s["x"], s["y"], s["h"], s["z"], gate=s["gate"], res_scale=s["res_scale"],
                       gamma_post=s["gamma_post"], gamma_pre=s["gamma_pre"])
        return {"h": s["h"], "z": s["z"]}
    if op == "norm_backward":
        sdm.block_norm_backward(shape, s["y"], s["h"], s["dz"], s["dh"], s["dx"], s["dy"], gate=s["gate"],
                                res_scale=s["res_scale"], gamma_post=s["gamma_post"], gamma_pre=s["gamma_pre"],
                                dgate=s["dgate"], dres_scale=s["dres_scale"], dgamma_post=s["dgamma_post"],
                                dgamma_pre=s["dgamma_pre"], workspace=ws)
        return {n: s[n] for n in ("dx", "dy", "dgate", "dres_scale", "dgamma_post", "dgamma_pre")}
    if op == "step":
        sdm.dla_step(shape, s["q"], s["k"], s["v"], s["log_decay"], s["state"], s["y"], slots=s["slots"])
        return {"y": s["y"], "state": s["state"]}
    if op == "forward":
        sdm.dla_forward(shape, s["q"], s["k"], s["v"], s["log_decay"], s["state"], s["y"], ws, lengths=s["lengths"])
        return {"y": s["y"], "state": s["state"]}
    sdm.dla_backward(shape, s["q"], s["k"], s["v"], s["log_decay"], s["state"], s["dy"], s["dstate"], s["dq"], s["dk"],
                     s["dv"], s["dstate0"], ws, lengths=s["lengths"])
    return {n: s[n] for n in ("dq", "dk", "dv", "dstate0")}


# ------------------------------------------------------------------ plain forms
def _heads(x, c):
    """The case's layout -> [B, H, T, d] in 32 bits, key heads repeated for their value heads."""
    x = x.float()
    x = x.transpose(1, 2) if c["layout"] == "token_major" else x
    return x if x.shape[1] == c["H"] else x.repeat_interleave(c["H"] // c["Hk"], 1)


def _chunks(s, names):
    """The inputs split into chunks [B, H, n, C, d], zero past a sequence's length and past T, and the powers of the
    decay: between two tokens of a chunk (lower), from its start to after a token, from a token to its last live one,
    over its live tokens."""
    c = s["case"]
    T, C = c["T"], CHUNK
    n = -(-T // C)
    ends = s["lengths"].long() if s["lengths"] is not None else torch.full((c["B"],), T, device="cuda")
    live = torch.arange(n * C, device="cuda") < ends[:, None]                     # [B, n C]

    def cut(x):
        y = x.new_zeros((*x.shape[:2], n * C, x.shape[3]))
        y[:, :, :T] = x
        y = torch.where(live[:, None, :, None], y, torch.zeros((), device="cuda"))
        return y.reshape(*x.shape[:2], n, C, x.shape[3])

    g = s["log_decay"].double()[:, None]
    i = torch.arange(C, device="cuda")
    between = torch.tril(torch.exp(g[..., None] * (i[:, None] - i[None, :]).clamp(min=0))).float()     # [H, C, C]
    head = torch.exp(g * (i + 1)).float()                                                              # [H, C]
    count = live.reshape(c["B"], n, C).sum(-1)                                                         # [B, n]
    left = (count[:, None, :, None] - 1 - i).clamp(min=0)                                              # [B, 1, n, C]
    tail = torch.exp(g[None, :, :, None] * left).float()
    over = torch.exp(g[None] * count[:, None, :]).float()                                              # [B, H, n]
    return [cut(_heads(s[x], c)) for x in names], between[None, :, None], head[None, :, None, :, None], tail[..., None], over[..., None, None]


def _back(x, c, dtype, shared=False):
    """[B, H, n, C, d] -> the case's layout and type, summed over the value heads that share a key head."""
    x = x.flatten(2, 3)[:, :, :c["T"]]
    x = x.unflatten(1, (c["Hk"], c["H"] // c["Hk"])).sum(2) if shared else x
    return _order(x, c).to(dtype)


def _states(a, b, over, S, backwards=False):
    """The state before every chunk (after it, walking backwards) and the last one."""
    adds, out = a.mT @ b, [None] * a.shape[2]
    order = range(a.shape[2])
    for n in reversed(order) if backwards else order:
        out[n] = S
        S = over[:, :, n] * S + adds[:, :, n]
    return torch.stack(out, 2), S


def _plain_forward(s):
    c = s["case"]
    (q, k, v), between, head, tail, over = _chunks(s, ("q", "k", "v"))
    S, last = _states(tail * k, v, over, s["state"])
    y = head * (q @ S) + (between * (q @ k.mT)) @ v
    s["state"].copy_(last)
    return {"y": _back(c["dk"] ** -0.5 * y, c, s["v"].dtype), "state": s["state"]}


def _plain_step(s):
    c = s["case"]
    at = s["slots"].long() if s["slots"] is not None else torch.arange(c["B"], device="cuda")
    q, k, v = (_heads(s[n], c)[:, :, 0] for n in ("q", "k", "v"))
    S = torch.exp(s["log_decay"])[None, :, None, None] * s["state"][at] + k[..., None] * v[..., None, :]
    s["state"][at] = S
    y = c["dk"] ** -0.5 * (q[..., None] * S).sum(-2)
    return {"y": _order(y[:, :, None], c).to(s["v"].dtype), "state": s["state"]}


def _plain_backward(s):
    c = s["case"]
    (q, k, v, dy), between, head, tail, over = _chunks(s, ("q", "k", "v", "dy"))
    dy = c["dk"] ** -0.5 * dy
    S, _ = _states(tail * k, v, over, s["state"])
    R, first = _states(head * q, dy, over, s["dstate"], backwards=True)
    P, dP = between * (q @ k.mT), between * (dy @ v.mT)
    dq = head * (dy @ S.mT) + dP @ k
    dk = tail * (v @ R.mT) + dP.mT @ q
    dv = tail * (k @ R) + P.mT @ dy
    dt = s["v"].dtype
    return {"dq": _back(dq, c, dt, True), "dk": _back(dk, c, dt, True), "dv": _back(dv, c, dt), "dstate0": first}


def _rms(x):
    return 1 / (x.square().mean(-1, keepdim=True) + EPS).sqrt()


def _gate_rows(s):
    c = s["case"]
    return s["gate"].float().repeat_interleave(c["gate_rows"], 0)[:c["M"]]


def _plain_norm(s):
    u = s["y"].float()
    if s["gamma_post"] is not None:
        u = u * _rms(u) * s["gamma_post"]
    if s["gate"] is not None:
        u = u * _gate_rows(s)
    if s["res_scale"] is not None:
        u = u * s["res_scale"]
    h = (s["x"].float() + u).to(s["x"].dtype)
    if s["gamma_pre"] is None:
        return {"h": h, "z": None}
    f = h.float()
    return {"h": h, "z": (f * _rms(f) * s["gamma_pre"]).to(h.dtype)}


def _plain_norm_backward(s):
    c, dt = s["case"], s["h"].dtype
    out = dict.fromkeys(("dgate", "dres_scale", "dgamma_post", "dgamma_pre"))
    a = s["dh"].float()
    if s["dz"] is not None:
        h, dz = s["h"].float(), s["dz"].float()
        r = _rms(h)
        n, dn = h * r, dz * s["gamma_pre"]
        out["dgamma_pre"] = (dz * n).sum(0)
        a = a + r * (dn - n * (dn * n).mean(-1, keepdim=True))
    u = y = s["y"].float()
    if s["gamma_post"] is not None:
        r = _rms(y)
        n = y * r
        u = n * s["gamma_post"]
    du = a
    if s["gate"] is not None:
        g = _gate_rows(s)
        d = a * u if s["res_scale"] is None else a * u * s["res_scale"]
        groups, rows = s["gate"].shape[0], c["gate_rows"]
        if groups * rows > c["M"]:
            d = torch.cat([d, d.new_zeros((groups * rows - c["M"], c["D"]))])
        out["dgate"] = d.reshape(groups, rows, c["D"]).sum(1).to(dt)
        du = du * g
    if s["res_scale"] is not None:
        out["dres_scale"] = (du * u).sum(0)
        du = du * s["res_scale"]
    if s["gamma_post"] is not None:
        out["dgamma_post"] = (du * n).sum(0)
        dn = du * s["gamma_post"]
        du = r * (dn - n * (dn * n).mean(-1, keepdim=True))
    return {"dx": a.to(dt), "dy": du.to(dt), **out}


def _plain_clip(s):
    total = sum(g.float().square().sum(dtype=torch.float64) for g in s["grads"])
    norm = total.sqrt().float()
    factor = torch.where(norm > s["max_norm"], s["max_norm"] / norm, torch.ones_like(norm))
    for g, to in zip(s["grads"], s["clipped"]):
        to.copy_(g.float() * factor)
    return {"stats": torch.stack([norm, factor]), **s["to"]}


def run(state):
    if own:
        return _run_own(state)
    return {"step": _plain_step, "forward": _plain_forward, "backward": _plain_backward, "norm": _plain_norm,
            "norm_backward": _plain_norm_backward, "clip": _plain_clip}[state["case"]["op"]](state)


# ------------------------------------------------------------------ definitions in 64 bits
def _exact_attention(c, s):
    """Every pair of tokens at once, one sequence and head after the other."""
    f = torch.float64
    tm, T, G, scale = c["layout"] == "token_major", c.get("T", 1), c["H"] // c["Hk"], c["dk"] ** -0.5
    seq = lambda x, b, h: (x[b, :, h] if tm else x[b, h])  # noqa: E731
    step = c["op"] == "step"
    rows = s["slots"].tolist() if s["slots"] is not None else range(c["B"])
    full = s["state"].to(f)
    names = ("dq", "dk", "dv") if c["op"] == "backward" else ("y",)
    out = {n: torch.zeros(s[{"dq": "q", "dk": "k"}.get(n, "v")].shape, dtype=f, device=full.device) for n in names}
    first = torch.zeros_like(full)
    for b, row in enumerate(rows):
        n = 1 if step else int(s["lengths"][b]) if s["lengths"] is not None else T
        i = torch.arange(n, device=full.device)
        for h in range(c["H"]):
            q, k, v = (seq(s[x], b, hh)[:n].to(f) for x, hh in (("q", h // G), ("k", h // G), ("v", h)))
            ld = s["log_decay"][h].to(f)
            w = torch.where(i[:, None] >= i[None, :], (ld * (i[:, None] - i[None, :]).clamp(min=0)).exp_(), 0)
            since, until = (ld * (i + 1)).exp()[:, None], (ld * (n - 1 - i)).exp()[:, None]
            S0 = full[row, h]
            if c["op"] != "backward":
                seq(out["y"], b, h)[:n] = scale * ((w * torch.einsum("ik,jk->ij", q, k)) @ v + since * (q @ S0))
                full[row, h] = (ld * n).exp() * S0 + torch.einsum("tk,tv->kv", until * k, v)
                continue
            dy, R = scale * seq(s["dy"], b, h)[:n].to(f), s["dstate"][b, h].to(f)
            P, dP = w * torch.einsum("ik,jk->ij", q, k), w * torch.einsum("iv,jv->ij", dy, v)
            seq(out["dq"], b, h // G)[:n] += dP @ k + since * torch.einsum("tv,kv->tk", dy, S0)
            seq(out["dk"], b, h // G)[:n] += torch.einsum("ij,ik->jk", dP, q) + until * torch.einsum("tv,kv->tk", v, R)
            seq(out["dv"], b, h)[:n] = torch.einsum("ij,iv->jv", P, dy) + until * (k @ R)
            first[b, h] = (ld * n).exp() * R + torch.einsum("tk,tv->kv", since * q, dy)
    out.update({"dstate0": first} if c["op"] == "backward" else {"state": full})
    return out


def _exact_norm(c, s):
    """Through torch's differentiation of the definition."""
    f = torch.float64
    t = {n: s[n].to(f) for n in ("y", "gate", "res_scale", "gamma_post", "gamma_pre") if s[n] is not None}
    backward = c["op"] == "norm_backward"
    for x in t.values():
        x.requires_grad_(backward)

    def rms_norm(x, gamma):
        return gamma * x * torch.rsqrt(torch.einsum("md,md->m", x, x)[:, None] / c["D"] + EPS)

    u = rms_norm(t["y"], t["gamma_post"]) if "gamma_post" in t else t["y"]
    if "gate" in t:
        u = u * t["gate"][torch.arange(c["M"], device=u.device) // c["gate_rows"]]
    if "res_scale" in t:
        u = u * t["res_scale"]
    if not backward:
        h = s["x"].to(f) + u
        stored = h.to(s["x"].dtype).to(f)                    # the norm is of what is stored
        return {"h": h, "z": rms_norm(stored, t["gamma_pre"]) if "gamma_pre" in t else None}
    h = s["h"].to(f).requires_grad_(True)
    pre = torch.zeros_like(h)
    out = dict.fromkeys(("dgate", "dres_scale", "dgamma_post", "dgamma_pre"))
    if "gamma_pre" in t:
        pre, out["dgamma_pre"] = torch.autograd.grad(rms_norm(h, t["gamma_pre"]), (h, t["gamma_pre"]), s["dz"].to(f))
    dx = s["dh"].to(f) + pre
    names = [n for n in ("y", "gate", "res_scale", "gamma_post") if n in t]
    if u.requires_grad:
        for n, d in zip(names, torch.autograd.grad(u, [t[n] for n in names], dx)):
            out["d" + n] = d
    return {"dx": dx, **out}


def exact(case, seed):
    c, f = case, torch.float64
    s = _inputs(case, seed, "cuda")
    if c["op"] in ("norm", "norm_backward"):
        out = _exact_norm(c, s)
        order = ("h", "z") if c["op"] == "norm" else ("dx", "dy", "dgate", "dres_scale", "dgamma_post", "dgamma_pre")
        return {n: None if out[n] is None else out[n].detach() for n in order}
    if c["op"] == "clip":
        norm = math.sqrt(sum(float(torch.linalg.vector_norm(g, dtype=f)) ** 2 for g in s["grads"]))
        factor = min(1.0, s["max_norm"] / norm)
        return {"stats": torch.tensor([norm, factor], dtype=f, device="cuda"), **{t: x.to(f) * factor for t, x in s["flat"].items()}}
    return _exact_attention(c, s)
