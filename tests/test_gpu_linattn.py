"""Linear attention with decays on the GPU (whole sequences, adjoint, single steps) against the
float64 oracle, through the public entry points.

Tolerances, element by element.  Results are sums of products; with A the same sum over absolute
values (the oracle run on |q|, |k|, |v|, ...), an error is at most
    half a step of the result's type |result| + kappa A,
    kappa = 2^-24 (Dk + Dv + 2 * 64 + 4 ceil(T / 64) + 64)  [+ 2^-16 for 16-bit operands]:
every term passes at most Dk (or Dv) + 2 * 64 roundings of float32 sums within a chunk of steps, four
for each chunk its state passes (decay, sum, and those of joining segments of chunks) and fewer than
64 others (decays, exponents, scale, splitting).  For 16-bit operands the decayed scores and the
state enter their second product with 16 bits or more, each term off by 2^-18 twice at most and by
the 2^-18 of the dropped smallest product: 2^-16 holds all three.
The gradient of log_decay at t is z + sum_s (q_s dq_s - k_s dk_s) over at most 1024 steps; the sum of
those terms' absolute values is A_t + 2 sum |k_s dk_s|.  Its terms come from the same products.
"""
import numpy as np
import pytest

from gpu_util import say
from oracle import layers as L

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2605_12683_amd as D  # noqa: E402

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def half_step(t):
    return torch.finfo(t).eps / 2


def make(B, T, H, Hk, Dk, Dv, type_, per_step=False, state=False, lengths=None, seed=0, memory=(3.0, 300.0)):
    rng = np.random.default_rng(seed + 7 * T + 13 * Dk + Dv)
    t = TYPES[type_]

    def n(*shape, dtype=t, scale=1.0):
        return torch.tensor(rng.standard_normal(shape) * scale).to(dtype).cuda()

    mem = np.exp(rng.uniform(np.log(memory[0]), np.log(memory[1]), (B, T, H) if per_step else H))
    c = {"q": n(B, T, Hk, Dk), "k": n(B, T, Hk, Dk, scale=Dk ** -0.5), "v": n(B, T, H, Dv),
         "log_decay": torch.tensor(-1 / mem).float().cuda()}
    kw = {"scale": Dk ** -0.5, "lengths": None if lengths is None else torch.tensor(lengths, dtype=torch.int32).cuda(),
          "state0": n(B, H, Dk, Dv, dtype=torch.float32) if state else None}
    g, gs = n(B, T, H, Dv), n(B, H, Dk, Dv, dtype=torch.float32) if state else None
    return c, kw, g, gs


def kappa(c, state=False):
    """state: of the float32 state, whose sums keep 24 bits whatever the operands' type."""
    T, Dk, Dv = c["v"].shape[1], c["q"].shape[3], c["v"].shape[3]
    k = 2.0 ** -24 * (Dk + Dv + 128 + 4 * -(-T // 64) + 64)
    return k if state or c["v"].dtype == torch.float32 else k + 2.0 ** -16


def near(name, got, ref, absolute, kap):
    # below the type's smallest normal number the step is tiny eps, a rounding is off by half of it
    low = torch.finfo(got.dtype).tiny * half_step(got.dtype) + 1e-37
    got_, tol = f64(got), half_step(got.dtype) * np.abs(ref) + kap * absolute + low
    assert np.isfinite(got_).all(), name
    worst = (np.abs(got_ - ref) / tol).max() if ref.size else 0.0
    assert worst <= 1.0, (name, worst)


def oracle_args(c, kw, absolute=False):
    f = np.abs if absolute else (lambda x: x)
    a = {n: (f(f64(x)) if n != "log_decay" else f64(x)) for n, x in c.items()}
    b = {"scale": abs(kw["scale"]) if absolute else kw["scale"],
         "lengths": None if kw["lengths"] is None else kw["lengths"].cpu().numpy(),
         "state0": None if kw["state0"] is None else f(f64(kw["state0"]))}
    return a, b


def check_forward(c, kw, out=None):
    out = D.deer_linattn(**c, **kw, want_state=True) if out is None else out
    a, b = oracle_args(c, kw)
    o, last = L.linattn(**a, **b)
    a, b = oracle_args(c, kw, True)
    oa, la = L.linattn(**a, **b)
    near("o", out["o"], o, oa, kappa(c))
    near("state", out["state"], last, la, kappa(c, state=True))
    return out


def check_adjoint(c, kw, g, gs, got=None):
    got = D.deer_linattn_adjoint(**c, g=g, **kw, g_state=gs)["grads"] if got is None else got
    a, b = oracle_args(c, kw)
    ref = L.linattn_adjoint(**a, g=f64(g), g_state=f64(gs), **b)
    a, b = oracle_args(c, kw, True)
    ab = L.linattn_adjoint(**a, g=np.abs(f64(g)), g_state=None if gs is None else np.abs(f64(gs)), **b)
    kap = kappa(c)
    for n in ("q", "k", "v"):
        near(n, got[n], ref[n], ab[n], kap)
    if kw["state0"] is not None:
        near("state0", got["state0"], ref["state0"], ab["state0"], kappa(c, state=True))
    # log decays: |terms| from a per-step run of the absolute values
    ld = a["log_decay"]
    B, T, H = c["v"].shape[:3]
    a["log_decay"] = np.broadcast_to(ld, (B, T, H)).copy()
    a["q"], a["k"] = (np.repeat(x, H // x.shape[2], 2) for x in (a["q"], a["k"]))
    per = L.linattn_adjoint(**a, g=np.abs(f64(g)), g_state=None if gs is None else np.abs(f64(gs)), **b)
    flow = (np.abs(a["k"]) * per["k"]).sum(-1)
    absolute = per["log_decay"].copy()
    for t0 in range(0, T, 1024):
        absolute[:, t0:t0 + 1024] += 2 * flow[:, t0:t0 + 1024][:, ::-1].cumsum(1)[:, ::-1]
    if ld.ndim == 1:
        absolute = absolute.sum((0, 1))
    near("log_decay", got["log_decay"], ref["log_decay"], absolute, kap)
    return got


CASES = [
    # B, T, H, Hk, Dk, Dv, type
    (1, 1, 1, 1, 1, 1, "f32"), (2, 1, 2, 1, 64, 64, "bf16"), (1, 2, 1, 1, 3, 5, "f16"),
    (2, 31, 2, 2, 16, 16, "f32"), (1, 32, 2, 1, 33, 17, "bf16"), (2, 33, 1, 1, 32, 32, "f16"),
    (1, 63, 2, 2, 64, 64, "bf16"), (1, 64, 2, 2, 128, 128, "bf16"), (1, 65, 2, 2, 65, 129, "f32"),
    (2, 127, 4, 2, 48, 96, "f32"), (1, 128, 3, 1, 100, 7, "f16"), (1, 129, 1, 1, 256, 256, "bf16"),
    (1, 200, 1, 1, 256, 200, "f32"), (1, 190, 2, 1, 200, 256, "f16"), (3, 257, 4, 4, 40, 72, "bf16"),
    (1, 1023, 2, 1, 24, 24, "f32"), (2, 1024, 1, 1, 16, 8, "bf16"), (1, 1025, 2, 2, 8, 16, "f16"),
    (1, 2100, 2, 1, 64, 64, "bf16"), (1, 2311, 1, 1, 32, 128, "f32"), (40, 70, 8, 8, 16, 16, "bf16"),
]


@pytest.mark.parametrize("B,T,H,Hk,Dk,Dv,type_", CASES)
@pytest.mark.parametrize("per_step", [False, True])
def test_forward_and_adjoint(B, T, H, Hk, Dk, Dv, type_, per_step):
    say("linattn", B, T, H, Hk, Dk, Dv, type_, per_step)
    state = T % 2 == 1
    lengths = None
    if B > 1:
        lengths = np.linspace(T, 0 if B > 2 else max(1, T // 2), B).astype(int)
    c, kw, g, gs = make(B, T, H, Hk, Dk, Dv, type_, per_step, state, lengths)
    check_forward(c, kw)
    check_adjoint(c, kw, g, gs)


@pytest.mark.parametrize("type_", ["f32", "bf16"])
def test_long_sequence(type_):
    """70001 steps of one narrow head (joined from many pieces), and its gradients."""
    c, kw, g, gs = make(1, 70001, 1, 1, 4, 3, type_, True, True, memory=(20.0, 3000.0))
    say("linattn long", type_)
    check_forward(c, kw)
    check_adjoint(c, kw, g, gs)


@pytest.mark.parametrize("type_", ["f32", "bf16", "f16"])
def test_decays_of_every_size(type_):
    """Zero decays (a state that starts anew, twice in a row, at the first and the last step), decays
    of one, decays that vanish at once beside slow ones, growth."""
    c, kw, g, gs = make(2, 150, 4, 2, 20, 36, type_, True, True)
    ld = c["log_decay"]
    ld[0, :, 0] = -torch.inf
    ld[0, [0, 17, 63, 64, 65, 127, 128, 149], 1] = -torch.inf
    ld[0, :, 2] = 0.0
    ld[0, ::3, 3] = -100.0
    ld[1, :40, 0] = -30.0
    ld[1, 40:, 1] = -1e-6
    ld[1, :, 2] = 0.02
    ld[1, 70, 3] = -1e30
    say("linattn decays", type_)
    check_forward(c, kw)
    check_adjoint(c, kw, g, gs)


@pytest.mark.parametrize("type_", ["f32", "bf16"])
def test_decays_of_nothing(type_):
    """Decays of zero, and the first step's from no state, have a gradient of zero exactly; one decay for
    each head that is zero as well."""
    c, kw, g, gs = make(2, 300, 3, 1, 20, 36, type_, True)
    c["log_decay"][0, [40, 64, 200], 1] = -torch.inf
    c["log_decay"][1, 250, 2] = torch.finfo(torch.float32).min
    say("linattn decays of nothing", type_)
    grad = D.deer_linattn_adjoint(**c, g=g, **kw)["grads"]["log_decay"]
    assert (grad[0, [40, 64, 200], 1] == 0).all() and grad[1, 250, 2] == 0 and (grad[:, 0] == 0).all()
    assert (grad != 0).sum() == grad.numel() - 4 - 6
    check_adjoint(c, kw, g, None)
    c["log_decay"] = torch.tensor([-torch.inf, -0.1, -0.2], device="cuda")
    grad = D.deer_linattn_adjoint(**c, g=g, **kw)["grads"]["log_decay"]
    assert grad[0] == 0 and (grad[1:] != 0).all()
    check_adjoint(c, kw, g, None)


@pytest.mark.parametrize("type_", ["f32", "bf16"])
def test_growth(type_):
    """States that grow for a while (by e^0.9 a step for 60 steps, 2^78) and decay again."""
    c, kw, g, gs = make(1, 200, 2, 1, 16, 24, type_, True, True)
    c["log_decay"][0, 30:90, 0] = 0.9
    c["log_decay"][0, 90:150, 0] = -0.8
    c["log_decay"][0, 60:70, 1] = 3.0
    say("linattn growth", type_)
    check_forward(c, kw)
    check_adjoint(c, kw, g, gs)


SEG_CASES = [(1, 1300, 2, 1, 24, 40, "bf16", [1300]), (2, 700, 2, 2, 130, 70, "f32", [700, 257]),
             (3, 640, 1, 1, 64, 64, "f16", [640, 64, 0]), (1, 2500, 1, 1, 96, 256, "bf16", [2111]),
             (2, 1100, 2, 1, 128, 128, "bf16", [1100, 1025]), (1, 200, 1, 1, 40, 31, "f32", [200])]


@pytest.mark.parametrize("B,T,H,Hk,Dk,Dv,type_,lengths", SEG_CASES)
@pytest.mark.parametrize("seg", [64, 128, 320, 1 << 20])
@pytest.mark.parametrize("state", [False, True])
def test_segments(B, T, H, Hk, Dk, Dv, type_, lengths, seg, state, monkeypatch):
    """Segments of every length (and one only), with ends of sequences inside, between and before them."""
    monkeypatch.setenv("DEER_LIN_SEG", str(seg))
    c, kw, g, gs = make(B, T, H, Hk, Dk, Dv, type_, seg == 128, state, lengths)
    say("linattn segments", B, T, H, Hk, Dk, Dv, type_, seg, state)
    check_forward(c, kw)
    check_adjoint(c, kw, g, gs)


@pytest.mark.parametrize("type_", ["f32", "bf16"])
def test_rows_behind_the_end_are_not_read(type_):
    """Lengths from below zero to beyond T; NaN and infinities behind the ends."""
    B, T = 6, 133
    lengths = [-3, 0, 1, 64, 132, 500]
    c, kw, g, gs = make(B, T, 2, 1, 24, 40, type_, True, True, lengths)
    say("linattn lengths", type_)
    for b, n in enumerate(lengths):
        n = max(n, 0)
        for x, bad in ((c["q"], torch.nan), (c["k"], torch.inf), (c["v"], torch.nan), (g, -torch.inf),
                       (c["log_decay"], torch.nan)):
            x[b, n:] = bad
    clean = {n: torch.nan_to_num(x, 0.0, 0.0, 0.0) for n, x in c.items()}
    out = D.deer_linattn(**c, **kw, want_state=True)
    check_forward(clean, kw, out)
    gr = D.deer_linattn_adjoint(**c, g=g, **kw, g_state=gs)["grads"]
    check_adjoint(clean, kw, torch.nan_to_num(g, 0.0, 0.0, 0.0), gs, gr)
    for b, n in enumerate(lengths):
        n = max(n, 0)
        assert not out["o"][b, n:].any()
        assert not any(gr[x][b, n:].any() for x in ("q", "k", "v", "log_decay"))
    assert torch.equal(out["state"][:2], kw["state0"][:2]) and torch.equal(gr["state0"][:2], gs[:2])


@pytest.mark.parametrize("type_,Dk,Dv", [("bf16", 64, 64), ("f32", 31, 48), ("f16", 8, 20)])
def test_views(type_, Dk, Dv):
    """Slices of a fused projection, heads before steps, an odd first element, one row for a batch, a
    last dimension that is not dense: the same results bit for bit as from contiguous copies."""
    B, T, H = 2, 97, 3
    t = TYPES[type_]
    gen = torch.Generator(device="cuda").manual_seed(1)
    say("linattn views", type_)
    fused = torch.randn(B, T, H * (2 * Dk + Dv) + 1, device="cuda", generator=gen).to(t)
    q = fused[..., 1:1 + H * Dk].unflatten(-1, (H, Dk))
    k = fused[..., 1 + H * Dk:1 + 2 * H * Dk].unflatten(-1, (H, Dk))
    v = fused[..., 1 + 2 * H * Dk:].unflatten(-1, (H, Dv))
    swapped = [x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for x in (q, k, v)]
    dense_last = [x.transpose(-1, -2).contiguous().transpose(-1, -2) for x in (q, k, v)]
    shared = [x[:1].expand(B, T, H, x.shape[-1]) for x in (q, k, v)]
    ld = -torch.rand(B, H, T, device="cuda", generator=gen).transpose(1, 2)
    g = torch.randn(B, H, T, Dv, device="cuda", generator=gen).to(t).transpose(1, 2)
    one_step = [x[:, :1].expand(B, T, H, x.shape[-1]) for x in (q, k, v)]
    near_rows = [torch.randn(B, T * 2 + x.shape[-1] + 64, device="cuda", generator=gen).to(t).as_strided(
        (B, T, H, x.shape[-1]), (T * 2 + x.shape[-1] + 64, 2, 16, 1)) for x in (q, k, v)]     # rows that overlap
    for ops in ((q, k, v), swapped, dense_last, shared, one_step, near_rows):
        kw = {"scale": 0.2}
        a = D.deer_linattn(*ops, ld, want_state=True, **kw)
        b = D.deer_linattn(*(x.contiguous() for x in ops), ld.contiguous(), want_state=True, **kw)
        assert torch.equal(a["o"], b["o"]) and torch.equal(a["state"], b["state"])
        a = D.deer_linattn_adjoint(*ops, ld, g, **kw)["grads"]
        b = D.deer_linattn_adjoint(*(x.contiguous() for x in ops), ld.contiguous(), g.contiguous(), **kw)["grads"]
        assert all(torch.equal(a[n], b[n]) for n in a)


@pytest.mark.parametrize("type_,T", [("bf16", 400), ("f32", 200), ("bf16", 1)])
def test_wide_step_strides(type_, T):
    """Tensors with the largest stride of a step that is taken (2^22 elements); one above it is refused."""
    t = TYPES[type_]
    say("linattn wide strides", type_, T)
    B, H, Dk, Dv = 1, 2, 32, 64
    c, kw, g, _ = make(B, T, H, H, Dk, Dv, type_)
    views = {}
    far = torch.empty((T - 1) * (1 << 22) + 1000, dtype=t, device="cuda")
    at = 0
    for n in ("q", "k", "v"):
        views[n] = far.as_strided(c[n].shape, (64, 1 << 22, c[n].shape[3], 1), at)
        views[n].copy_(c[n])
        at += H * c[n].shape[3]
    ref = D.deer_linattn(**c, want_state=True, **kw)
    a = D.deer_linattn(**views, log_decay=c["log_decay"], want_state=True, **kw)
    assert torch.equal(a["o"], ref["o"]) and torch.equal(a["state"], ref["state"])
    ga = D.deer_linattn_adjoint(**views, log_decay=c["log_decay"], g=g, **kw)["grads"]
    gb = D.deer_linattn_adjoint(**c, g=g, **kw)["grads"]
    assert all(torch.equal(ga[n], gb[n]) for n in ga)
    if T > 1:
        wider = {n: far.as_strided((1, 2, *c[n].shape[2:]), (64, (1 << 22) + 8, c[n].shape[3], 1)) for n in ("q", "k", "v")}
        with pytest.raises(D.DeerError, match="stride"):
            D.deer_linattn(**wider, log_decay=c["log_decay"], **kw)


def test_offsets_beyond_32_bits():
    """Two sequences whose rows lie more than 2^32 bytes and 2^31 elements apart."""
    B, T, H, Dk, Dv = 2, 70, 2, 32, 32
    say("linattn far views")
    far = torch.empty((1 << 31) + 100000, dtype=torch.bfloat16, device="cuda")
    c, kw, g, _ = make(B, T, H, H, Dk, Dv, "bf16")
    views = {}
    for i, n in enumerate(("q", "k", "v")):
        x = far.as_strided(c[n].shape, ((1 << 31) + 64, H * 32 * 3, 32, 1), i * H * 32)
        x.copy_(c[n])
        views[n] = x
    a = D.deer_linattn(**views, log_decay=c["log_decay"], want_state=True, **kw)
    b = D.deer_linattn(**c, want_state=True, **kw)
    assert torch.equal(a["o"], b["o"]) and torch.equal(a["state"], b["state"])
    a = D.deer_linattn_adjoint(**views, log_decay=c["log_decay"], g=g, **kw)["grads"]
    b = D.deer_linattn_adjoint(**c, g=g, **kw)["grads"]
    assert all(torch.equal(a[n], b[n]) for n in a)


@pytest.mark.parametrize("B,H,Hk,Dk,Dv,type_,per_step", [
    (1, 1, 1, 1, 1, "f32", False), (1, 8, 8, 64, 64, "bf16", False), (3, 4, 2, 33, 65, "f16", True),
    (2, 2, 1, 256, 256, "f32", True), (5, 3, 3, 100, 30, "bf16", True), (700, 2, 1, 16, 128, "bf16", False)])
def test_step(B, H, Hk, Dk, Dv, type_, per_step):
    """One step against the oracle's; sequences that take none keep their state bit for bit."""
    say("linattn step", B, H, Hk, Dk, Dv, type_, per_step)
    lengths = [i % 3 != 1 for i in range(B)]
    c, kw, _, _ = make(B, 1, H, Hk, Dk, Dv, type_, per_step, True, lengths)
    state = kw["state0"].clone()
    o = torch.full((B, H, Dv), torch.nan, dtype=TYPES[type_], device="cuda")
    x = {n: (y[:, 0] if y.dim() > 1 else y) for n, y in c.items()}
    r = D.deer_linattn_step(**x, state=state, o=o, scale=kw["scale"], lengths=kw["lengths"])
    assert r["o"] is o and r["state"] is state
    check_forward(c, kw, {"o": o[:, None], "state": state})
    for b in range(B):
        if not lengths[b]:
            assert torch.equal(state[b], kw["state0"][b]) and not o[b].any()


@pytest.mark.parametrize("type_", ["f32", "bf16"])
def test_prompt_then_steps(type_):
    """A prompt in two parts (the state continued in place), then single steps, against one call."""
    c, kw, _, _ = make(2, 90, 4, 2, 24, 32, type_, True)
    say("linattn generate", type_)
    state = torch.zeros(2, 4, 24, 32, device="cuda")
    outs = []
    for lo, hi in ((0, 70), (70, 71), (71, 80)):
        part = {n: x[:, lo:hi] for n, x in c.items()}
        r = D.deer_linattn(**part, scale=kw["scale"], state0=state, state=state)
        assert r["state"] is state
        outs.append(r["o"])
    for t in range(80, 90):
        outs.append(D.deer_linattn_step(**{n: x[:, t] for n, x in c.items()}, state=state, scale=kw["scale"])["o"][:, None])
    check_forward(c, kw, {"o": torch.cat(outs, 1), "state": state})


@pytest.mark.parametrize("type_", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("Dk,Dv", [(20, 72), (64, 128), (128, 128), (100, 130)])
@pytest.mark.parametrize("seg", [64, 1 << 20])
def test_many_heads(type_, Dk, Dv, seg, monkeypatch):
    """Enough heads and segments for the wide blocks of every walk (few heads take narrow ones)."""
    monkeypatch.setenv("DEER_LIN_SEG", str(seg))
    B, T = (11, 150) if seg == 64 else (33, 70)
    lengths = np.linspace(T, 0, B).astype(int)
    c, kw, g, gs = make(B, T, 4, 2, Dk, Dv, type_, seg == 64, True, lengths)
    say("linattn many heads", type_, Dk, Dv, seg)
    check_forward(c, kw)
    check_adjoint(c, kw, g, gs)


@pytest.mark.parametrize("B,T,H,Hk,Dk,Dv,type_", [(2, 300, 4, 2, 64, 64, "bf16"), (1, 200, 2, 2, 100, 72, "f32"),
                                                  (2, 130, 3, 1, 32, 128, "f16"), (50, 70, 8, 8, 40, 40, "bf16")])
def test_adjoint_without_decays(B, T, H, Hk, Dk, Dv, type_):
    """The other gradients alone; few heads and many."""
    c, kw, g, gs = make(B, T, H, Hk, Dk, Dv, type_, True, True)
    say("linattn without decays", B, T, H, Dk, Dv, type_)
    full = D.deer_linattn_adjoint(**c, g=g, **kw, g_state=gs)["grads"]
    grads = D.deer_linattn_adjoint(**c, g=g, **kw, g_state=gs, want_decay=False)["grads"]
    assert set(full) - set(grads) == {"log_decay"}
    check_adjoint(c, kw, g, gs, {**grads, "log_decay": full["log_decay"]})


@pytest.mark.parametrize("seg", [64, 320])
def test_state_in_place_over_segments(seg, monkeypatch):
    """state0 overwritten by the state behind the last of 3 or 11 segments, which every block starts from."""
    monkeypatch.setenv("DEER_LIN_SEG", str(seg))
    c, kw, _, _ = make(2, 700, 8, 8, 128, 128, "bf16", state=True, lengths=[700, 300])
    say("linattn in place over segments", seg)
    state = kw["state0"].clone()
    out = D.deer_linattn(**c, **{**kw, "state0": state}, state=state)
    check_forward(c, kw, {"o": out["o"], "state": state})


def test_gradients_against_differences():
    """Directional differences of the GPU's own forward pass: o and the state are linear in each of q,
    k, v and state0 alone; log_decay with a step whose square is below the tolerance."""
    c, kw, g, gs = make(2, 300, 2, 1, 24, 16, "f32", True, True)
    say("linattn differences")
    gr = D.deer_linattn_adjoint(**c, g=g, **kw, g_state=gs)["grads"]
    gen = torch.Generator(device="cuda").manual_seed(4)

    def loss(c, kw):
        r = D.deer_linattn(**c, **kw, want_state=True)
        return float((r["o"].double() * g).sum() + (r["state"].double() * gs).sum())

    for n, e in (("q", 0.5), ("k", 0.5), ("v", 0.5), ("state0", 0.5), ("log_decay", 1e-3)):
        x = kw["state0"] if n == "state0" else c[n]
        d = torch.randn(x.shape, device="cuda", generator=gen)
        vals = []
        for sgn in (1, -1):
            y = x + sgn * e * d
            vals.append(loss(c, {**kw, n: y}) if n == "state0" else loss({**c, n: y}, kw))
        want = float((gr[n].double() * d).sum())
        norm = float(gr[n].double().norm() * d.double().norm())
        # float32 losses of size ~norm: 1e-5 of it; log_decay: e^2 and 1e-7 / e of it
        assert abs((vals[0] - vals[1]) / (2 * e) - want) < (2e-3 if n == "log_decay" else 1e-4) * norm, n


def test_workspace_contents_and_repeats():
    """NaN-poisoned and zero workspaces, and a second call, give the same bits."""
    from paper_2605_12683_amd import _binding as Bnd
    for T, H in ((1500, 2), (700, 1), (5000, 1)):
        c, kw, g, gs = make(1, T, H, 1, 48, 32, "bf16", False, True)
        say("linattn workspace", T, H)
        for op, call in ((Bnd.DEER_OP_SOLVE, lambda ws: D.deer_linattn(**c, **kw, want_state=True, ws=ws)),
                         (Bnd.DEER_OP_ADJOINT, lambda ws: D.deer_linattn_adjoint(**c, g=g, **kw, g_state=gs, ws=ws)["grads"])):
            n = D.deer_linattn_workspace_bytes(1, T, H, 1, 48, 32, op, torch.bfloat16)
            first = call(torch.full((n,), 255, dtype=torch.uint8, device="cuda"))
            ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
            for _ in range(2):
                again = call(ws)
                assert all(torch.equal(first[x], again[x]) for x in first)


def test_streams_and_graphs():
    """On a side stream; captured with other inputs, replayed several times with eager work between."""
    c, kw, g, gs = make(1, 1300, 2, 1, 32, 48, "bf16", True, True)
    say("linattn stream")
    want = (D.deer_linattn(**c, **kw, want_state=True), D.deer_linattn_adjoint(**c, g=g, **kw, g_state=gs)["grads"])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = (D.deer_linattn(**c, **kw, want_state=True), D.deer_linattn_adjoint(**c, g=g, **kw, g_state=gs)["grads"])
    s.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(a[n], b[n]) for n in a)
    say("linattn graph")
    c2 = {n: x.clone() for n, x in c.items()}
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r1 = D.deer_linattn(**c2, **kw, want_state=True)
        r2 = D.deer_linattn_adjoint(**c2, g=g, **kw, g_state=gs)["grads"]
    with torch.cuda.graph(other):
        r3 = D.deer_linattn(**c2, **kw, want_state=True)
    for i in range(3):
        for n in c2:
            c2[n].copy_(c[n] * (1 + i) if n == "v" else c[n])
        graph.replay()
        other.replay()
        torch.cuda.synchronize()
        e = D.deer_linattn(**c2, **kw, want_state=True)
        ea = D.deer_linattn_adjoint(**c2, g=g, **kw, g_state=gs)["grads"]
        assert all(torch.equal(r1[n], e[n]) and torch.equal(r3[n], e[n]) for n in e)
        assert all(torch.equal(r2[n], ea[n]) for n in ea)


def test_refusals():
    c, kw, g, gs = make(2, 8, 2, 1, 4, 4, "bf16", True, True)
    bad = [dict(q=c["q"].float()), dict(k=c["k"][:, :4]), dict(v=c["v"].cpu()), dict(log_decay=c["log_decay"].double()),
           dict(log_decay=c["log_decay"][:, :, :1]), dict(v=c["v"][:, 0]), dict(q=c["q"].int())]
    for x in bad:
        with pytest.raises(ValueError):
            D.deer_linattn(**{**c, **x})
    for x in (dict(lengths=torch.tensor([1, 2])), dict(lengths=torch.tensor([1, 2]).cuda()), dict(state0=gs[:1]),
              dict(state=gs.half()), dict(o=torch.empty_like(c["v"])[:, :4])):
        with pytest.raises(ValueError):
            D.deer_linattn(**c, **x)
    with pytest.raises(ValueError):
        D.deer_linattn_adjoint(**c, g=g.float())
    with pytest.raises(D.DeerError):
        D.deer_linattn(c["q"].repeat(1, 1, 3, 1), c["k"].repeat(1, 1, 3, 1), c["v"], c["log_decay"])   # 2 heads, 3 of q
    with pytest.raises(D.DeerError):
        D.deer_linattn(**c, o=c["v"])
    with pytest.raises(D.DeerError):
        D.deer_linattn(**c, scale=float("nan"))
    with pytest.raises(D.DeerError):
        D.deer_linattn(**c, ws=torch.empty(0, dtype=torch.uint8, device="cuda"))
    for ws in (torch.empty(1 << 20, dtype=torch.uint8), torch.empty(2, 1 << 20, dtype=torch.uint8, device="cuda")[:, ::2]):
        with pytest.raises(ValueError):
            D.deer_linattn(**c, ws=ws)
        with pytest.raises(ValueError):
            D.deer_linattn_adjoint(**c, g=g, ws=ws)
    step = {n: x[:, 0] for n, x in c.items()}
    with pytest.raises(ValueError):
        D.deer_linattn_step(**step, state=gs.transpose(-1, -2))
    with pytest.raises(ValueError):
        D.deer_linattn_step(**step, state=None)
