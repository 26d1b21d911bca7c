"""The gated delta rule and the linear layer around it: what is timed, and the operators' plain forms.

Gated delta rule, per sequence and value head, state S [d_k, d_v]:
    S~ = alpha_t S,  e_t = v_t - S~^T k_t,  S_t = S~ + beta_t k_t e_t^T,  y_t = scale S_t^T q_t.
Linear layer: out = residual + act(x W^T + bias); its backward takes the stored pre-activation.

`own` chooses between the plain forms (elementary torch operations in 32 bits) and the library's
entry points.  Sizes follow synth/configs.py: heads of 64 and 128, 16 heads, d_model = 16 * 128.
"""
import math

import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
CHUNK = 64


def listed():
    return [
        # one sequence being decoded: the latency of a single small call
        dict(name="step_one", op="step", B=1, H=16, Hk=16, dk=128, dv=128, dtype="bf16", slots=1, layout="head_major"),
        # a serving batch (the decode workload's B and H) over a larger cache of states
        dict(name="step_serving", op="step", B=256, H=16, Hk=16, dk=128, dv=128, dtype="bf16", slots=288,
             layout="head_major"),
        # the tiny fp32 workload: one short sequence of one head
        dict(name="forward_tiny_f32", op="forward", B=1, H=1, Hk=1, T=256, dk=64, dv=64, dtype="f32", ragged=False,
             layout="head_major"),
        # a padded batch of prompts of different lengths, key heads shared by two value heads,
        # in the layout that projections write
        dict(name="forward_ragged", op="forward", B=4, H=8, Hk=4, T=2011, dk=128, dv=128, dtype="bf16", ragged=True,
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
        # output projection of a few tokens being decoded, with the residual
        dict(name="linear_decode", op="linear", M=4, N=2048, K=2048, act="none", bias=True, residual=True, pre=False),
        # an up projection at odd sizes, keeping what its backward needs
        dict(name="linear_odd", op="linear", M=1531, N=5448, K=2056, act="gelu", bias=True, residual=False, pre=True),
        # output projection and residual of the 1.4B layer
        dict(name="linear_layer", op="linear", M=32768, N=2048, K=2048, act="silu", bias=True, residual=True, pre=False),
        # gradients of a small projection over a long batch
        dict(name="linear_backward_narrow", op="linear_backward", M=8192, N=504, K=512, act="gelu"),
        # gradients of the 1.4B layer's projection
        dict(name="linear_backward_layer", op="linear_backward", M=32768, N=2048, K=2048, act="silu"),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def eight(lo, hi):
        return 8 * max(1, log(lo, hi) // 8)

    op = rng.choice(["step", "forward", "forward", "backward", "linear", "linear_backward"])
    if op in ("linear", "linear_backward"):
        c = dict(op=op, M=log(1, 32768), N=eight(64, 6144), K=eight(64, 4096), act=rng.choice(["none", "relu", "silu", "gelu"]))
        while c["M"] * c["N"] * c["K"] > 32768 * 2048 * 2048:
            c["M"] = max(1, c["M"] // 2)
        if op == "linear":
            c.update(bias=rng.random() < 0.7, residual=rng.random() < 0.5, pre=rng.random() < 0.5)
        return c
    dtype = rng.choice(["bf16", "bf16", "f32"])
    Hk = rng.choice([1, 2, 4, 5, 8, 16])
    c = dict(op=op, Hk=Hk, H=Hk * rng.choice([1, 1, 2, 3]), dk=rng.choice([32, 64, 96, 128, 128]),
             dv=rng.choice([32, 64, 96, 128, 128, 192]), dtype=dtype, layout=rng.choice(["head_major", "token_major"]))
    if op == "step":
        c["B"] = log(1, 256)
        while c["B"] * c["H"] * c["dk"] * c["dv"] > 256 * 16 * 128 * 128:
            c["B"] = max(1, c["B"] // 2)
        c["slots"] = c["B"] + rng.randrange(0, 33)
        return c
    c.update(B=log(1, 8), T=log(16, 4096 if dtype == "bf16" else 1024), ragged=rng.random() < 0.5)
    while c["B"] * c["H"] * c["T"] * c["dk"] * c["dv"] > 8 * 16 * 4096 * 128 * 128:
        c["T"] = max(16, c["T"] // 2)
    return c


def work(case):
    c = case
    if c["op"] in ("linear", "linear_backward"):
        M, N, K = c["M"], c["N"], c["K"]
        if c["op"] == "linear":
            b = 2 * (M * K + N * K + M * N) + 4 * N * c["bias"] + 2 * M * N * (c["residual"] + c["pre"])
            return {"bytes": b, "flops": 2 * M * N * K}
        gates = 2 * M * N * (1 if c["act"] == "none" else 2)     # dout and, where used, the stored pre-activation
        return {"bytes": 2 * (2 * M * K + 2 * N * K) + gates + 4 * N, "flops": 4 * M * N * K}
    es = 4 if c["dtype"] == "f32" else 2
    T = c.get("T", 1)
    tokens = sum(_lengths(c)) if c.get("ragged") else c["B"] * T
    qk, vy, g = tokens * c["Hk"] * c["dk"] * es, tokens * c["H"] * c["dv"] * es, tokens * c["H"] * es
    state = c["B"] * c["H"] * c["dk"] * c["dv"] * 4
    mul = tokens * c["H"] * c["dk"] * c["dv"]
    if c["op"] == "backward":        # q, k, v, dy, gates, S_0, dS_T in; dq, dk, dv, gate gradients, dS_0 out
        return {"bytes": 4 * qk + 3 * vy + 4 * g + 3 * state, "flops": 20 * mul}
    pad = (c["B"] * T - tokens) * c["H"] * c["dv"] * es          # zeros of y past the lengths
    return {"bytes": 2 * qk + 2 * vy + 2 * g + 2 * state + pad, "flops": 7 * mul}


def _lengths(c):
    """Lengths of a ragged batch, from none of the tokens to all of them."""
    B, T = c["B"], c["T"]
    return [T - (T * i * i) // max(1, (B - 1) ** 2 + (B > 4)) if B > 1 else T - T // 3 for i in range(B)]


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
    if c["op"] in ("linear", "linear_backward"):
        M, N, K = c["M"], c["N"], c["K"]
        s["x"] = rand(M, K).bfloat16()
        s["W"] = (rand(N, K) / math.sqrt(K)).bfloat16()
        s["bias"] = rand(N) * 0.1 if c.get("bias") else None
        s["residual"] = rand(M, N).bfloat16() if c.get("residual") else None
        if c["op"] == "linear_backward":
            s["pre"] = rand(M, N).bfloat16()
            s["dout"] = rand(M, N).bfloat16()
        return s
    B, H, Hk, T, dk, dv, dt = c["B"], c["H"], c["Hk"], c.get("T", 1), c["dk"], c["dv"], DT[c["dtype"]]

    def unit(*shape):
        x = rand(*shape)
        return x / x.square().sum(-1, keepdim=True).sqrt()

    s["q"] = _order(unit(B, Hk, T, dk).to(dt), c)
    s["k"] = _order(unit(B, Hk, T, dk).to(dt), c)
    s["v"] = _order(rand(B, H, T, dv).to(dt), c)
    s["alpha"] = torch.sigmoid(rand(B, H, T) + 4).to(dt)
    s["beta"] = torch.sigmoid(rand(B, H, T)).to(dt)
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
    if c["op"] in ("linear", "linear_backward"):
        if c["op"] == "linear":
            s["out"] = torch.empty((c["M"], c["N"]), dtype=torch.bfloat16, device="cuda")
            s["pre"] = torch.empty_like(s["out"]) if c["pre"] else None
        else:
            s["dx"], s["dW"] = torch.empty_like(s["x"]), torch.empty_like(s["W"])
            s["dbias"] = torch.empty(c["N"], dtype=torch.float32, device="cuda")
        return s
    s["y"] = torch.empty_like(s["v"])
    if c["op"] == "backward":
        for n in ("q", "k", "v", "alpha", "beta", "state"):
            s["d" + n + ("0" if n == "state" else "")] = torch.empty_like(s[n])
    return s


# ------------------------------------------------------------------ the framework's calls
def _plan(s):
    """The shape and the workspace, made once and kept with the state as a user's program keeps them."""
    import paper_2607_07386_gb300 as sdm
    c = s["case"]
    if c["op"] in ("linear", "linear_backward"):
        shape = sdm.LinearShape.make(c["M"], c["N"], c["K"], act=c["act"])
        n = sdm.linear_backward_workspace_bytes(shape) if c["op"] == "linear_backward" else sdm.linear_workspace_bytes(shape)
    else:
        shape = sdm.GdnShape.make(c["B"], c["H"], c.get("T", 1), c["dk"], c["dv"], H_k=c["Hk"], dtype=c["dtype"],
                                  layout=c["layout"], scale=c["dk"] ** -0.5)
        n = {"step": lambda sh: 0, "forward": sdm.gdn_workspace_bytes,
             "backward": sdm.gdn_backward_workspace_bytes}[c["op"]](shape)
    s["plan"] = (sdm, shape, torch.empty(n, dtype=torch.uint8, device="cuda") if n else None)
    return s["plan"]


def _run_own(s):
    sdm, shape, ws = s.get("plan") or _plan(s)
    op = s["case"]["op"]
    if op == "step":
        sdm.gdn_step(shape, s["q"], s["k"], s["v"], s["alpha"], s["beta"], s["state"], s["y"], slots=s["slots"])
        return {"y": s["y"], "state": s["state"]}
    if op == "forward":
        sdm.gdn_forward(shape, s["q"], s["k"], s["v"], s["alpha"], s["beta"], s["state"], s["y"], ws, lengths=s["lengths"])
        return {"y": s["y"], "state": s["state"]}
    if op == "backward":
        sdm.gdn_backward(shape, s["q"], s["k"], s["v"], s["alpha"], s["beta"], s["state"], s["dy"], s["dstate"],
                         s["dq"], s["dk"], s["dv"], s["dalpha"], s["dbeta"], s["dstate0"], ws, lengths=s["lengths"])
        return {n: s[n] for n in ("dq", "dk", "dv", "dalpha", "dbeta", "dstate0")}
    if op == "linear":
        sdm.linear(shape, s["x"], s["W"], s["out"], bias=s["bias"], residual=s["residual"], pre=s["pre"], workspace=ws)
        return {"out": s["out"], "pre": s["pre"]}
    sdm.linear_backward(shape, s["x"], s["W"], s["pre"], s["dout"], s["dx"], s["dW"], s["dbias"], ws)
    return {"dx": s["dx"], "dW": s["dW"], "dbias": s["dbias"]}


# ------------------------------------------------------------------ plain forms
def _heads(x, c):
    """The case's layout -> [B, H, T, d] in 32 bits, key heads repeated for their value heads."""
    x = x.float()
    x = x.transpose(1, 2) if c["layout"] == "token_major" else x
    return x if x.shape[1] == c["H"] else x.repeat_interleave(c["H"] // c["Hk"], 1)


def _chunks(s):
    """q, k, v, alpha, beta (and dy) split into chunks [B, H, n, C, ...]; tokens past a sequence's
    length and past T have q = k = v = dy = 0, alpha = 1 and beta = 0, which changes nothing."""
    c = s["case"]
    T = c["T"]
    n = -(-T // CHUNK)
    live = torch.ones((c["B"], T), dtype=torch.bool, device="cuda")
    if s["lengths"] is not None:
        live = torch.arange(T, device="cuda")[None, :] < s["lengths"][:, None]
    live = live[:, None, :]

    def cut(x, fill):
        x = torch.where(live if x.dim() == 3 else live[..., None], x, torch.full_like(x, fill))
        y = torch.full((*x.shape[:2], n * CHUNK, *x.shape[3:]), fill, dtype=x.dtype, device=x.device)
        y[:, :, :T] = x
        return y.reshape(*x.shape[:2], n, CHUNK, *x.shape[3:])

    names = ("q", "k", "v") + (("dy",) if "dy" in s else ())
    return [cut(_heads(s[x], c), 0.0) for x in names], cut(s["alpha"].float(), 1.0), cut(s["beta"].float(), 0.0)


def _factors(q, k, alpha, beta):
    """Decay products G_ij = prod_{j < l <= i} alpha_l (lower), g_i = prod_{l <= i} alpha_l, the inverse
    (I + L)^-1 of the chunk's unit lower triangle, and k_i.k_j, q_i.k_j."""
    i = torch.arange(CHUNK, device="cuda")
    below = i[:, None] > i[None, :]
    one = torch.ones((), device="cuda")
    G = torch.tril(torch.where(below, alpha[..., :, None], one).cumprod(-2))
    kk, qk = k @ k.mT, q @ k.mT
    X = -torch.tril(beta[..., :, None] * G * kk, -1)
    inv = torch.eye(CHUNK, device="cuda") + X
    for _ in range(5):              # (I - X)^-1 = (I + X)(I + X^2)(I + X^4) ...: X is nilpotent
        X = X @ X
        inv = inv + X @ inv
    return G, alpha.cumprod(-1), inv, kk, qk


def _scan(q, k, v, beta, S, G, g, inv, P):
    """The chunks in order; returns the chunk-initial states, V' = beta e and the reads, unscaled."""
    states, writes, reads = [], [], []
    for n in range(q.shape[2]):
        Q, K, gn = q[:, :, n], k[:, :, n], g[:, :, n, :, None]
        states.append(S)
        w = inv[:, :, n] @ (beta[:, :, n, :, None] * (v[:, :, n] - gn * (K @ S)))
        reads.append(gn * (Q @ S) + P[:, :, n] @ w)
        S = gn[:, :, -1:] * S + (G[:, :, n, -1, :, None] * K).mT @ w
        writes.append(w)
    return states, writes, reads, S


def _back(x, c, dtype):
    """[B, H, n, C, d] -> the case's layout and type."""
    x = x.flatten(2, 3)[:, :, :c["T"]]
    return _order(x, c).to(dtype)


def _shared(x, c):
    """Sums a gradient [B, H, ...] over the value heads that share a key head."""
    return x.unflatten(1, (c["Hk"], c["H"] // c["Hk"])).sum(2)


def _plain_forward(s):
    c = s["case"]
    (q, k, v), alpha, beta = _chunks(s)
    G, g, inv, _, qk = _factors(q, k, alpha, beta)
    _, _, reads, S = _scan(q, k, v, beta, s["state"], G, g, inv, G * qk)
    s["state"].copy_(S)
    return {"y": _back(c["dk"] ** -0.5 * torch.stack(reads, 2), c, s["v"].dtype), "state": s["state"]}


def _plain_step(s):
    c = s["case"]
    at = s["slots"].long() if s["slots"] is not None else torch.arange(c["B"], device="cuda")
    q, k, v = (_heads(s[n], c)[:, :, 0] for n in ("q", "k", "v"))
    S = s["alpha"].float()[..., None] * s["state"][at]
    e = v - (k[..., None] * S).sum(-2)
    S = S + (s["beta"].float() * k)[..., None] * e[..., None, :]
    s["state"][at] = S
    y = c["dk"] ** -0.5 * (q[..., None] * S).sum(-2)
    return {"y": _order(y[:, :, None], c).to(s["v"].dtype), "state": s["state"]}


def _plain_backward(s):
    c = s["case"]
    (q, k, v, dy), alpha, beta = _chunks(s)
    G, g, inv, kk, qk = _factors(q, k, alpha, beta)
    states, writes, _, _ = _scan(q, k, v, beta, s["state"], G, g, inv, G * qk)
    dy = dy * c["dk"] ** -0.5
    P, last = G * qk, G[..., -1, :, None]
    dS, d, ends = s["dstate"], [], []
    for n in reversed(range(q.shape[2])):
        Q, K, gn = q[:, :, n], k[:, :, n], g[:, :, n, :, None]
        ends.insert(0, dS)
        d.insert(0, inv[:, :, n].mT @ (P[:, :, n].mT @ dy[:, :, n] + last[:, :, n] * (K @ dS)))
        dS = gn[:, :, -1:] * dS + Q.mT @ (gn * dy[:, :, n]) - K.mT @ (beta[:, :, n, :, None] * gn * d[0])
    S, dE, d, w = torch.stack(states, 2), torch.stack(ends, 2), torch.stack(d, 2), torch.stack(writes, 2)
    b, gg = beta[..., None], g[..., None]
    yS, dSk, wE = dy @ S.mT, d @ S.mT, w @ dE.mT
    yw, dw = torch.tril(dy @ w.mT), torch.tril(d @ w.mT, -1)
    dq = gg * yS + (G * yw) @ k
    A = b * G * dw
    dk = last * wE - b * gg * dSk + (G * yw).mT @ q - A.mT @ k - A @ k
    e = v - gg * (k @ S) - torch.tril(G * kk, -1) @ w
    dbeta = (d * e).sum(-1)
    # gradient of every product of decays, with the chunk's initial state as column 0 and its end as the last row
    dG = alpha.new_zeros((*alpha.shape[:3], CHUNK + 1, CHUNK + 1))
    dG[..., :-1, 1:] = yw * qk - b * dw * kk
    dG[..., :-1, 0] = (q * yS).sum(-1) - beta * (k * dSk).sum(-1)
    dG[..., -1, 1:] = (k * wE).sum(-1)
    dG[..., -1, 0] = (dE * S).sum((-1, -2))
    tail = torch.cat([G, G[..., -1:, :]], -2).mT                      # [t, i]: prod_{t < l <= i}
    head = torch.cat([g.new_ones((*g.shape[:3], 1, 1)).expand(*g.shape[:3], 1, 1), g[..., :-1, None]], -2)
    head = torch.cat([head, torch.cat([torch.zeros_like(G[..., :1, :]), G[..., :-1, :]], -2)], -1)   # [t, j]: prod_{j < l < t}
    dalpha = ((tail @ dG) * head).sum(-1)
    dt = s["v"].dtype
    live = torch.ones_like(s["alpha"], dtype=torch.bool)
    if s["lengths"] is not None:
        live = live & (torch.arange(c["T"], device="cuda") < s["lengths"][:, None, None])
    zero = torch.zeros((), device="cuda")
    gate = lambda x: torch.where(live, x.flatten(2, 3)[:, :, :c["T"]], zero).to(dt)  # noqa: E731
    return {"dq": _back(_shared(dq, c), c, dt), "dk": _back(_shared(dk, c), c, dt), "dv": _back(b * d, c, dt),
            "dalpha": gate(dalpha), "dbeta": gate(dbeta), "dstate0": dS}


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (0.5 / math.pi) ** 0.5
    return torch.ones_like(z)


def _plain_linear(s):
    z = s["x"].float() @ s["W"].float().mT
    if s["bias"] is not None:
        z = z + s["bias"]
    out = _act(z, s["case"]["act"])
    if s["residual"] is not None:
        out = out + s["residual"].float()
    return {"out": out.bfloat16(), "pre": z.bfloat16() if s["case"]["pre"] else None}


def _plain_linear_backward(s):
    d = s["dout"].float() * _slope(s["pre"].float(), s["case"]["act"])
    return {"dx": (d @ s["W"].float()).bfloat16(), "dW": (d.mT @ s["x"].float()).bfloat16(), "dbias": d.sum(0)}


def run(state):
    if own:
        return _run_own(state)
    return {"step": _plain_step, "forward": _plain_forward, "backward": _plain_backward, "linear": _plain_linear,
            "linear_backward": _plain_linear_backward}[state["case"]["op"]](state)


# ------------------------------------------------------------------ definitions in 64 bits
def _exact_tokens(c, s):
    """Token-by-token recurrence and its reverse, straight from the definition."""
    f = torch.float64
    B, H, T, scale = c["B"], c["H"], c.get("T", 1), c["dk"] ** -0.5
    tm = c["layout"] == "token_major"

    def tok(name, t):
        x = s[name][:, t] if tm else s[name][:, :, t]
        x = x.to(f)
        return x if x.shape[1] == H else x.repeat_interleave(H // c["Hk"], 1)

    at = s["slots"].long() if s["slots"] is not None else None
    S0 = (s["state"][at] if at is not None else s["state"][:B]).to(f)
    ends = s["lengths"].long() if s["lengths"] is not None else torch.full((B,), T, device=S0.device)
    al, be = s["alpha"].to(f), s["beta"].to(f)

    def token(S, t):
        on = (t < ends)[:, None, None, None]
        Sd = al[:, :, t, None, None] * S
        k = tok("k", t)
        e = tok("v", t) - torch.einsum("bhkv,bhk->bhv", Sd, k)
        Sn = Sd + be[:, :, t, None, None] * k[..., None] * e[..., None, :]
        return on, Sd, e, k, torch.where(on, Sn, S)

    if c["op"] != "backward":
        y = torch.zeros(s["v"].shape, dtype=f, device=S0.device)
        S = S0
        for t in range(T):
            on, _, _, _, S = token(S, t)
            r = torch.where(on[..., 0], scale * torch.einsum("bhkv,bhk->bhv", S, tok("q", t)), 0)
            if tm:
                y[:, t] = r
            else:
                y[:, :, t] = r
        full = s["state"].to(f)
        if at is not None:
            full[at] = S
        else:
            full[:B] = S
        return {"y": y, "state": full}

    out = {n: torch.zeros(s[n[1:]].shape, dtype=f, device=S0.device) for n in ("dq", "dk", "dv", "dalpha", "dbeta")}

    def put(name, t, x):
        if x.shape[1] != out[name].shape[2 if tm else 1]:
            x = x.unflatten(1, (c["Hk"], H // c["Hk"])).sum(2)
        if tm:
            out[name][:, t] = x
        else:
            out[name][:, :, t] = x

    span = 64
    marks, S = [], S0
    for t in range(T):
        if t % span == 0:
            marks.append(S)
        S = token(S, t)[-1]
    dS = s["dstate"].to(f)
    for m in reversed(range(len(marks))):
        olds = []
        S = marks.pop()
        for t in range(m * span, min(T, (m + 1) * span)):
            olds.append(S)
            S = token(S, t)[-1]
        for t in reversed(range(m * span, min(T, (m + 1) * span))):
            S = olds.pop()
            on, Sd, e, k, Sn = token(S, t)
            on3 = on[..., 0]
            q, dy, a, b = tok("q", t), tok("dy", t), al[:, :, t], be[:, :, t]
            zero = torch.zeros((), dtype=f, device=S.device)
            put("dq", t, torch.where(on3, scale * torch.einsum("bhkv,bhv->bhk", Sn, dy), zero))
            D = dS + scale * q[..., None] * dy[..., None, :]
            Dk = torch.einsum("bhkv,bhk->bhv", D, k)
            put("dv", t, torch.where(on3, b[..., None] * Dk, zero))
            Dd = D - b[..., None, None] * k[..., None] * Dk[..., None, :]
            put("dk", t, torch.where(on3, b[..., None] * (torch.einsum("bhkv,bhv->bhk", D, e)
                                                          - torch.einsum("bhkv,bhv->bhk", Sd, Dk)), zero))
            out["dbeta"][:, :, t] = torch.where(on3[..., 0], (Dk * e).sum(-1), zero)
            out["dalpha"][:, :, t] = torch.where(on3[..., 0], (Dd * S).sum((-1, -2)), zero)
            dS = torch.where(on, a[..., None, None] * Dd, dS)
    out["dstate0"] = dS
    return out


def exact(case, seed):
    c, f = case, torch.float64
    s = _inputs(case, seed, "cuda")
    if c["op"] not in ("linear", "linear_backward"):
        return _exact_tokens(c, s)
    act = c["act"]
    if c["op"] == "linear":
        z = torch.einsum("mk,nk->mn", s["x"].to(f), s["W"].to(f))
        z = z if s["bias"] is None else z + s["bias"].to(f)
        h = {"none": lambda: z, "relu": lambda: z.clamp(min=0), "silu": lambda: z * torch.sigmoid(z),
             "gelu": lambda: z * torch.special.ndtr(z)}[act]()
        return {"out": h if s["residual"] is None else h + s["residual"].to(f), "pre": z if c["pre"] else None}
    z, d = s["pre"].to(f), s["dout"].to(f)
    sg = torch.sigmoid(z)
    d = d * {"none": lambda: torch.ones_like(z), "relu": lambda: torch.heaviside(z, torch.zeros((), dtype=f, device=z.device)),
             "silu": lambda: sg + z * sg * (1 - sg),
             "gelu": lambda: torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)}[act]()
    return {"dx": torch.einsum("mn,nk->mk", d, s["W"].to(f)), "dW": torch.einsum("mn,mk->nk", d, s["x"].to(f)),
            "dbias": d.sum(0)}
