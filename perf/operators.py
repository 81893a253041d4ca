"""The measured operators: linear attention with a decay for each head (the whole sequence, its
adjoint, one step) and layer normalisation (forward, adjoint), each in a plain form made of
elementary torch operations and through the library's entry points.

Linear attention keeps a matrix S [Dk, Dv] for each head,
    S_t = a_t S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t,   a_t = exp(log_decay),
with one decay for each head or one for each head and step; q and k may have fewer heads than v
(head h reads head h // (H // Hk) of q and k), and sequences of a batch may end early.
"""
from __future__ import annotations

import math

import torch

own = False     # True: `run` calls the library; False: the plain form

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5


# ---- the cases ---------------------------------------------------------------------------

def listed():
    return [
        # the first tokens of a request: latency is all there is
        _attn("forward_short", "forward", B=1, T=24, H=4, Hk=4, Dk=64, Dv=64, type="bf16"),
        # an ordinary batch of windows or prompts
        _attn("forward", "forward", B=2, T=4096, H=16, Hk=16, Dk=128, Dv=128, type="bf16"),
        # one long recording of many sessions laid end to end: a decay for each step, zero where
        # a session starts; keys and queries shared by four heads; continued from a state
        _attn("forward_long", "forward", B=1, T=65536, H=32, Hk=8, Dk=64, Dv=64, type="bf16", per_step=True,
              resets=True, state0=True),
        # odd sizes in float32: recordings of several lengths padded to the longest
        _attn("forward_ragged", "forward", B=5, T=1777, H=6, Hk=3, Dk=40, Dv=72, type="f32", ragged=True, state0=True),
        # the ordinary training step's backward pass, with the gradient of a decay for each step
        _attn("adjoint", "adjoint", B=4, T=4096, H=16, Hk=16, Dk=128, Dv=128, type="bf16", per_step=True),
        # odd sizes in float32, shared keys, recordings of several lengths, states at both ends
        _attn("adjoint_ragged", "adjoint", B=3, T=2500, H=6, Hk=2, Dk=48, Dv=96, type="f32", ragged=True, state0=True),
        # generation of one sequence
        _attn("step_one", "step", B=1, T=1, H=8, Hk=8, Dk=64, Dv=64, type="bf16"),
        # generation of a full batch: the states are all the traffic
        _attn("step_batch", "step", B=256, T=1, H=32, Hk=8, Dk=128, Dv=128, type="bf16", per_step=True),
        # the norm before a layer
        _norm("norm", "norm", rows=32768, G=1, D=2048, type="bf16"),
        # the norm of every head's output, weights of its own for each head
        _norm("norm_heads", "norm", rows=8192, G=16, D=128, type="f16", w32=True),
        # its backward pass at a training step's size
        _norm("norm_adjoint", "norm_adjoint", rows=32768, G=1, D=4096, type="bf16"),
        # a small model's, of an odd width
        _norm("norm_adjoint_odd", "norm_adjoint", rows=701, G=1, D=515, type="f32"),
    ]


def draw(rng):
    """One more case of the ranges above."""
    op = rng.choice(["forward", "forward", "adjoint", "adjoint", "step", "norm", "norm_adjoint"])
    type_ = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op.startswith("norm"):
        D = _log(rng, 16, 16384)
        G = rng.choice([1, 1, rng.randint(2, 16)]) if D <= 512 else 1
        rows = _log(rng, 16, min(65536, max(16, (1 << 26) // (D * G))))
        return _norm(None, op, rows=rows, G=G, D=D, type=type_, w32=rng.random() < 0.5)
    Hk = _log(rng, 1, 16)
    H = Hk * rng.choice([1, 1, 2, 4])
    Dk, Dv = (rng.choice([16, 32, 64, 96, 128, rng.randint(8, 256)]) for _ in range(2))
    if op == "step":
        B = _log(rng, 1, max(1, min(512, (1 << 26) // (H * Dk * Dv))))
        T = 1
    else:
        steps = min(4_000_000_000 // (H * Dk * Dv), 40_000_000 // (H * (Dk + Dv)))     # in the whole batch
        T = _log(rng, 1, min(32768, steps))
        B = min(_log(rng, 1, 16), steps // T)
    # (a single step from no state at all has no gradient of its decay)
    return _attn(None, op, B=B, T=T, H=H, Hk=Hk, Dk=Dk, Dv=Dv, type=type_, per_step=rng.random() < 0.5,
                 ragged=T > 1 and rng.random() < 0.3, state0=T == 1 or rng.random() < 0.4)


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _case(name, c, kw):
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def _attn(name, op, **kw):
    return _case(name, {"op": op, "per_step": False, "resets": False, "ragged": False, "state0": False}, kw)


def _norm(name, op, **kw):
    return _case(name, {"op": op, "w32": False}, kw)


def work(case):
    """Each input read once and each output written once; the products of the recurrence."""
    e = 4 if case["type"] == "f32" else 2
    if case["op"].startswith("norm"):
        n, D, G = case["rows"] * case["G"], case["D"], case["G"]
        if case["op"] == "norm":
            return {"bytes": 2 * n * D * e + 8 * n, "flops": 8 * n * D}
        return {"bytes": 3 * n * D * e + 8 * n + 8 * G * D, "flops": 14 * n * D}
    B, T, H, Hk, Dk, Dv = (case[x] for x in ("B", "T", "H", "Hk", "Dk", "Dv"))
    n, qk, v, s = B * T, B * T * Hk * Dk * e, B * T * H * Dv * e, 4 * B * H * Dk * Dv
    g = 4 * n * H if case["per_step"] else 4 * H
    if case["op"] == "step":
        return {"bytes": 2 * qk + 2 * v + g + 2 * s, "flops": 5 * n * H * Dk * Dv}
    if case["op"] == "forward":
        return {"bytes": 2 * qk + 2 * v + g + s * (2 if case["state0"] else 1), "flops": 4 * n * H * Dk * Dv}
    return {"bytes": 4 * qk + 3 * v + 2 * g + (3 * s if case["state0"] else 0), "flops": 10 * n * H * Dk * Dv}


# ---- inputs --------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    type_ = TYPES[case["type"]]

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, device="cuda", generator=gen).mul_(scale)

    if case["op"].startswith("norm"):
        rows, G, D = case["rows"], case["G"], case["D"]
        shape, wshape = ((rows, G, D), (G, D)) if G > 1 else ((rows, D), (D,))
        wt = torch.float32 if case["w32"] else type_
        # activations with an offset and a scale of their own for each row
        x = (normal(*shape) * torch.exp(normal(*shape[:-1], 1, scale=0.5)) + normal(*shape[:-1], 1, scale=0.5)).to(type_)
        st = {"case": case, "x": x, "w": (1 + normal(*wshape, scale=0.2)).to(wt), "b": normal(*wshape, scale=0.1).to(wt)}
        if case["op"] == "norm_adjoint":
            x64 = x.double() if x.numel() < 1 << 24 else x.float()
            mean = x64.mean(-1)
            var = (x64 - mean[..., None]).square_().mean(-1)
            st.update(g=normal(*shape).to(type_), mean=mean.float(), rstd=(var + EPS).rsqrt().float())
        return st

    B, T, H, Hk, Dk, Dv = (case[x] for x in ("B", "T", "H", "Hk", "Dk", "Dv"))
    st = {"case": case, "scale": Dk ** -0.5, "lengths": None, "state0": None, "g_state": None}
    lead = (B,) if case["op"] == "step" else (B, T)
    st["q"] = normal(*lead, Hk, Dk).to(type_)
    st["k"] = normal(*lead, Hk, Dk, scale=Dk ** -0.5).to(type_)
    st["v"] = normal(*lead, H, Dv).to(type_)
    # memories of 8 steps (the first head) to 500 (the last), a little different for each seed
    memory = torch.logspace(math.log10(8.0), math.log10(500.0), H, device="cuda") * torch.exp(normal(H, scale=0.1))
    if case["per_step"]:
        st["log_decay"] = -torch.exp(normal(*lead, H, scale=0.5)) / memory
        if case["resets"]:      # sessions of some 2048 steps
            start = torch.rand(*lead, 1, device="cuda", generator=gen) < 1 / 2048
            st["log_decay"] = st["log_decay"].masked_fill(start, -math.inf)
    else:
        st["log_decay"] = torch.log1p(-1 / memory)
    if case["ragged"]:
        n = torch.randint(0, T + 1, (B,), device="cuda", generator=gen, dtype=torch.int32)
        n[0] = T
        st["lengths"] = n
    if case["state0"] or case["op"] == "step":
        st["state0"] = normal(B, H, Dk, Dv)
    if case["op"] == "adjoint":
        st["g"] = normal(B, T, H, Dv).to(type_)
        st["g_state"] = normal(B, H, Dk, Dv) if case["state0"] else None
    return st


def run(state):
    op = state["case"]["op"]
    if own:
        return _own(op, state)
    return {"forward": _forward, "adjoint": _adjoint, "step": _step, "norm": _layernorm,
            "norm_adjoint": _layernorm_adjoint}[op](state)


def _own(op, s):
    import paper_2605_12683_amd as D
    if op == "norm":
        r = D.deer_layernorm(s["x"], s["w"], s["b"], eps=EPS)
        return {"y": r["y"], "mean": r["mean"], "rstd": r["rstd"]}
    if op == "norm_adjoint":
        r = D.deer_layernorm_adjoint(s["x"], s["g"], s["mean"], s["rstd"], s["w"])
        return {"x": r["x"], "w": r["grads"]["w"], "b": r["grads"]["b"]}
    kw = {"scale": s["scale"], "lengths": s["lengths"]}
    if op == "forward":
        r = D.deer_linattn(s["q"], s["k"], s["v"], s["log_decay"], state0=s["state0"], want_state=True, **kw)
        return {"o": r["o"], "state": r["state"]}
    if op == "step":
        r = D.deer_linattn_step(s["q"], s["k"], s["v"], s["log_decay"], s["state0"], **kw)
        return {"o": r["o"], "state": r["state"]}
    return D.deer_linattn_adjoint(s["q"], s["k"], s["v"], s["log_decay"], s["g"], state0=s["state0"],
                                  g_state=s["g_state"], **kw)["grads"]


# ---- the plain forms -------------------------------------------------------------------------

CHUNK = 128


def _walk(q, k, v, gate, s0):
    """o_t = S_t^T q_t, S_t = exp(gate_t) S_{t-1} + k_t v_t^T in float32 over [B, H, T, .], and the
    last state: products within chunks of steps, the chunks joined by the decays between them."""
    B, H, T, Dk = k.shape
    Dv = v.shape[-1]
    C = min(CHUNK, T)
    n = -(-T // C)
    pad = n * C - T
    if pad:
        q, k, v = (torch.nn.functional.pad(x, (0, 0, 0, pad)) for x in (q, k, v))
        gate = torch.nn.functional.pad(gate, (0, pad))
    q, k, v = (x.reshape(B, H, n, C, x.shape[-1]) for x in (q, k, v))
    c = gate.double().clamp(min=-200.0).reshape(B, H, n, C).cumsum(-1)
    low = torch.ones(C, C, dtype=torch.bool, device=q.device).tril()
    decay = (c[..., :, None] - c[..., None, :]).masked_fill_(~low, -math.inf).float().exp_()
    o = torch.matmul(torch.matmul(q, k.transpose(-1, -2)).mul_(decay), v)
    del decay
    # states entering each chunk: chunk m's own sum reaches chunk i > m by the decays between
    end = c[..., -1]
    own_sum = torch.matmul((k * (end[..., None] - c).exp().float()[..., None]).transpose(-1, -2), v)
    if s0 is None:
        s0 = torch.zeros(B, H, Dk, Dv, device=q.device)
    pieces = torch.cat([s0[:, :, None], own_sum], 2).reshape(B, H, n + 1, Dk * Dv)
    e = end.cumsum(-1)
    e = torch.nn.functional.pad(e, (1, 0))
    low = torch.ones(n + 1, n + 1, dtype=torch.bool, device=q.device).tril()
    between = (e[..., :, None] - e[..., None, :]).masked_fill_(~low, -math.inf).float().exp_()
    states = torch.matmul(between, pieces).reshape(B, H, n + 1, Dk, Dv)
    o += torch.matmul(q * c.float().exp()[..., None], states[:, :, :n])
    return o.reshape(B, H, n * C, Dv)[:, :, :T], states[:, :, n]


def _heads_first(x, H=None):
    """[B, T, Hk, D] -> float32 [B, H, T, D], shared heads repeated."""
    x = x.float().permute(0, 2, 1, 3)
    return x if H is None else x.repeat_interleave(H // x.shape[1], 1)


def _masked(s):
    """q, k, v (and the cotangent) heads first, the decays [B, H, T], all zero behind a sequence's end."""
    B, T, H, _ = s["v"].shape
    q, k, v = _heads_first(s["q"], H), _heads_first(s["k"], H), _heads_first(s["v"])
    a = s["log_decay"].expand(B, T, H).permute(0, 2, 1)
    g = _heads_first(s["g"]) if "g" in s else None
    if s["lengths"] is None:
        return q, k, v, g, a, None
    out = (torch.arange(T, device=q.device) >= s["lengths"][:, None])[:, None]
    return (q.masked_fill(out[..., None], 0), k.masked_fill(out[..., None], 0), v.masked_fill(out[..., None], 0),
            None if g is None else g.masked_fill(out[..., None], 0), a.masked_fill(out, 0), out)


def _forward(s):
    q, k, v, _, a, _ = _masked(s)
    o, last = _walk(q, k, v, a, s["state0"])
    return {"o": (o * s["scale"]).permute(0, 2, 1, 3).to(s["v"].dtype), "state": last}


def _adjoint(s):
    q, k, v, g, a, out = _masked(s)
    H, Hk, type_ = s["v"].shape[2], s["q"].shape[2], s["v"].dtype
    g = g * s["scale"]
    s0, gs = s["state0"], s["g_state"]
    dq, last = _walk(g, v, k, a, None if s0 is None else s0.transpose(-1, -2))
    # the adjoint state runs backwards: step t's decay is applied on the way from t to t - 1
    back = torch.nn.functional.pad(a[..., 1:], (0, 1)).flip(-1)
    qr, kr, vr, gr = (x.flip(2) for x in (q, k, v, g))
    dv, first = _walk(kr, qr, gr, back, gs)
    dk, _ = _walk(vr, gr, qr, back, None if gs is None else gs.transpose(-1, -2))
    dk, dv = dk.flip(2), dv.flip(2)
    # log decays: what reaches step t or later from before it
    flow = (q.double() * dq - k.double() * dk).sum(-1)
    if gs is not None:
        flow[..., -1] += (last.transpose(-1, -2).double() * gs).sum((-1, -2))
    da = flow.flip(-1).cumsum(-1).flip(-1)
    if out is not None:
        da = da.masked_fill(out, 0)
    da = da.permute(0, 2, 1)

    def shared(x):
        return x.unflatten(1, (Hk, H // Hk)).sum(2).permute(0, 2, 1, 3).to(type_)

    grads = {"q": shared(dq), "k": shared(dk), "v": dv.permute(0, 2, 1, 3).to(type_),
             "log_decay": (da if s["log_decay"].dim() == 3 else da.sum((0, 1))).float()}
    if s0 is not None:
        grads["state0"] = first * a[:, :, 0].exp()[..., None, None]
    return grads


def _step(s):
    H = s["v"].shape[1]
    r = H // s["q"].shape[1]
    q, k = (x.float().repeat_interleave(r, 1) for x in (s["q"], s["k"]))
    a = s["log_decay"].exp().expand(q.shape[:2])
    S = s["state0"]
    S.mul_(a[..., None, None]).add_(k[..., :, None] * s["v"].float()[..., None, :])
    o = (S * q[..., :, None]).sum(-2) * s["scale"]
    return {"o": o.to(s["v"].dtype), "state": S}


def _layernorm(s):
    x = s["x"].float()
    mean = x.mean(-1, keepdim=True)
    d = x - mean
    rstd = (d.square().mean(-1, keepdim=True) + EPS).rsqrt()
    y = d * rstd * s["w"].float() + s["b"].float()
    return {"y": y.to(s["x"].dtype), "mean": mean[..., 0], "rstd": rstd[..., 0]}


def _layernorm_adjoint(s):
    g = s["g"].float()
    xh = (s["x"].float() - s["mean"][..., None]) * s["rstd"][..., None]
    u = g * s["w"].float()
    dx = (u - u.mean(-1, keepdim=True) - xh * (u * xh).mean(-1, keepdim=True)) * s["rstd"][..., None]
    return {"x": dx.to(s["x"].dtype), "w": (g * xh).sum(0), "b": g.sum(0)}


# ---- 64 bits, from the definitions ---------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        x = s["x"].double()
        mean = x.sum(-1) / case["D"]
        var = (x * x).sum(-1) / case["D"] - mean * mean
        rstd = 1 / torch.sqrt(var + EPS)
        y = (x - mean.unsqueeze(-1)) * rstd.unsqueeze(-1) * s["w"].double() + s["b"].double()
        return {"y": y, "mean": mean, "rstd": rstd}
    if case["op"] == "norm_adjoint":
        g, D = s["g"].double(), case["D"]
        rstd = s["rstd"].double().unsqueeze(-1)
        xh = (s["x"].double() - s["mean"].double().unsqueeze(-1)) * rstd
        w, b = (g * xh).sum(0), g.sum(0)
        g *= s["w"].double()
        c1, c2 = g.sum(-1, keepdim=True) / D, torch.linalg.vecdot(g, xh).unsqueeze(-1) / D
        return {"x": rstd * (g - c1 - xh * c2), "w": w, "b": b}
    return _recurrence(case, s)


def _recurrence(case, s):
    """The recurrences step by step; a sequence that has ended keeps its state."""
    B, H, Dk, Dv = (case[x] for x in ("B", "H", "Dk", "Dv"))
    T, r, scale = case["T"], case["H"] // case["Hk"], s["scale"]
    head = torch.arange(H, device="cuda") // r
    step = case["op"] == "step"
    q, k, v = ((x.unsqueeze(1) if step else x).double() for x in (s["q"], s["k"], s["v"]))
    q, k = q[:, :, head], k[:, :, head]
    ld = s["log_decay"].double()
    a = torch.exp(ld.reshape(B, T, H) if ld.dim() > 1 else ld.expand(B, T, H))
    alive = torch.ones(B, T, 1, device="cuda", dtype=torch.float64)
    if s["lengths"] is not None:
        alive = (torch.arange(T, device="cuda")[None, :, None] < s["lengths"][:, None, None]).double()
    a = torch.where(alive > 0, a, torch.ones_like(a))
    q, k, v = (x * alive.unsqueeze(-1) for x in (q, k, v))
    S = torch.zeros(B, H, Dk, Dv, device="cuda", dtype=torch.float64) if s["state0"] is None else s["state0"].double()

    def ahead(S, t):
        return torch.addcmul(S * a[:, t, :, None, None], k[:, t, :, :, None], v[:, t, :, None, :])

    if case["op"] != "adjoint":
        o = torch.empty(B, T, H, Dv, device="cuda", dtype=torch.float64)
        for t in range(T):
            S = ahead(S, t)
            o[:, t] = torch.matmul(q[:, t, :, None, :], S)[:, :, 0]
        o *= scale
        return {"o": o[:, 0] if step else o, "state": S}

    g = s["g"].double() * alive.unsqueeze(-1) * scale
    every = 64
    kept = []
    for t in range(T):
        if t % every == 0:
            kept.append(S)
        S = ahead(S, t)
    R = torch.zeros_like(S) if s["g_state"] is None else s["g_state"].double()
    dq, dk, dv, da = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v), torch.empty_like(a)
    for t0 in reversed(range(0, T, every)):
        S = kept.pop()
        inside = [S]
        for t in range(t0, min(T, t0 + every)):
            S = ahead(S, t)
            inside.append(S)
        for t in reversed(range(t0, min(T, t0 + every))):
            R = torch.addcmul(R, q[:, t, :, :, None], g[:, t, :, None, :])
            dq[:, t] = (inside[t - t0 + 1] * g[:, t, :, None, :]).sum(-1)
            dk[:, t] = (R * v[:, t, :, None, :]).sum(-1)
            dv[:, t] = (R * k[:, t, :, :, None]).sum(-2)
            R = R * a[:, t, :, None, None]
            da[:, t] = (R * inside[t - t0]).sum((-1, -2))
    dq, dk, dv, da = dq * alive.unsqueeze(-1), dk * alive.unsqueeze(-1), dv * alive.unsqueeze(-1), da * alive
    out = {"q": dq.unflatten(2, (case["Hk"], r)).sum(3), "k": dk.unflatten(2, (case["Hk"], r)).sum(3), "v": dv,
           "log_decay": da if case["per_step"] else da.sum((0, 1))}
    if s["state0"] is not None:
        out["state0"] = R
    return out
