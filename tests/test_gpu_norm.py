"""Layer normalisation on the GPU, forward and adjoint, against the float64 oracle.

Tolerances, element by element (u = 2^-24, sums of D float32 terms pass at most n = D / 64 + 24
roundings each: no thread or lane adds more than D / 64 terms one after the other, then trees):
  mean: n u avg|x|;  d = x - mean: that and u |d|;  the variance is a mean of squares, relative
  error 2 (relative error of d's norm) + (n + 2) u; rstd half of it and 2 u more.
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
U = 2.0 ** -24


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def make(shape, type_, G=0, w32=False, seed=0, offset=0.5):
    rng = np.random.default_rng(seed + sum(shape))
    t = TYPES[type_]
    wt = torch.float32 if w32 else t
    wshape = shape[-2:] if G else shape[-1:]
    x = torch.tensor(rng.standard_normal(shape) * np.exp(rng.standard_normal((*shape[:-1], 1)) / 2) + offset).to(t).cuda()
    w = torch.tensor(1 + 0.3 * rng.standard_normal(wshape)).to(wt).cuda()
    b = torch.tensor(0.3 * rng.standard_normal(wshape)).to(wt).cuda()
    g = torch.tensor(rng.standard_normal(shape)).to(t).cuda()
    return x, w, b, g


def errors(x, eps):
    """n u, and the errors of mean, d = x - mean (each row) and rstd (relative)."""
    X = f64(x)
    Dn = X.shape[-1]
    nu = (Dn / 64 + 24) * U
    _, mean, rstd = L.layernorm(X, eps=eps)
    em = nu * np.abs(X).mean(-1) + U * np.abs(mean)
    var = 1 / rstd ** 2 - eps
    # ||d + e||^2 - ||d||^2 <= 2 sqrt(var) em + em^2, and the sum's own roundings
    er = 0.5 * ((2 * np.sqrt(np.maximum(var, 0)) * em + em ** 2) * rstd ** 2 + (nu + 4 * U)) + 3 * U
    return nu, mean, rstd, em, er


def check(x, w, b, g, eps, out=None, grads=None, groups=False):
    X = f64(x)
    W = np.ones(X.shape[-1]) if w is None else f64(w)
    out = D.deer_layernorm(x, w, b, eps=eps) if out is None else out
    y, mean, rstd = L.layernorm(X, f64(w), f64(b), eps)
    nu, _, _, em, er = errors(x, eps)
    half = torch.finfo(x.dtype).eps / 2
    low = torch.finfo(x.dtype).tiny * half + 1e-37     # half a step below the smallest normal number
    d = X - mean[..., None]
    ey = np.abs(W) * rstd[..., None] * (em[..., None] + (er[..., None] + 3 * U) * np.abs(d)) + 2 * U * np.abs(y) \
        + (0 if b is None else 2 * U * np.abs(f64(b)))
    assert (np.abs(f64(out["mean"]) - mean) <= em + 1e-37).all()
    assert (np.abs(f64(out["rstd"]) - rstd) <= er * rstd).all()
    assert (np.abs(f64(out["y"]) - y) <= half * np.abs(y) + (1 + half) * ey + low).all()
    if g is None:
        return
    r = D.deer_layernorm_adjoint(x, g, out["mean"], out["rstd"], w) if grads is None else grads
    ref = L.layernorm_adjoint(X, f64(g), f64(w), eps, groups)
    Gv = f64(g)
    xh = d * rstd[..., None]
    exh = rstd[..., None] * em[..., None] + (er[..., None] + 3 * U) * np.abs(xh)
    u = np.abs(Gv * W)
    # each of the three terms, and the factor rstd
    e1 = (nu + 2 * U) * u.mean(-1, keepdims=True)
    c2 = (u * np.abs(xh)).mean(-1, keepdims=True)
    e2 = (u * exh).mean(-1, keepdims=True) + (nu + 4 * U) * c2
    terms = u + u.mean(-1, keepdims=True) + np.abs(xh) * c2
    ex = rstd[..., None] * (4 * U * terms + e1 + np.abs(xh) * e2 + exh * c2 + er[..., None] * terms)
    dx = ref["x"]
    assert (np.abs(f64(r["x"]) - dx) <= half * np.abs(dx) + (1 + half) * ex + low).all()
    tail = xh.shape[-2:] if groups else xh.shape[-1:]
    rows = xh.size // int(np.prod(tail))
    # rows added one after the other in float32 at worst 1024 of them, then float64 or trees
    ns = (min(rows, 1024) + 64) * U
    ew = (np.abs(Gv) * (exh + ns * np.abs(xh))).reshape(-1, *tail).sum(0)
    eb = ns * np.abs(Gv).reshape(-1, *tail).sum(0)
    assert (np.abs(f64(r["grads"]["w"]) - ref["w"]) <= ew + U * np.abs(ref["w"]) + 1e-37).all()
    assert (np.abs(f64(r["grads"]["b"]) - ref["b"]) <= eb + U * np.abs(ref["b"]) + 1e-37).all()


@pytest.mark.parametrize("D_", [1, 2, 3, 7, 8, 31, 64, 65, 100, 128, 255, 256, 515, 1000, 1024, 2048, 2056, 4099, 4096, 8192,
                                16384, 20000, 65536])
@pytest.mark.parametrize("type_", ["f32", "bf16", "f16"])
def test_widths(D_, type_):
    say("layernorm", D_, type_)
    rows = 37 if D_ < 5000 else 5
    x, w, b, g = make((rows, D_), type_, w32=D_ % 2 == 1)
    check(x, w, b, g, 1e-5)


@pytest.mark.parametrize("rows", [1, 2, 3, 5, 255, 1000, 4097])
@pytest.mark.parametrize("type_,D_", [("bf16", 128), ("f32", 33), ("f16", 1024)])
def test_rows(rows, type_, D_):
    say("layernorm rows", rows, type_, D_)
    x, w, b, g = make((rows, D_), type_)
    check(x, w, b, g, 1e-5)


@pytest.mark.parametrize("shape", [(2, 5, 3, 16), (1, 1, 8, 64), (7, 4, 128), (300, 5, 33), (3, 1, 40), (2, 2, 3, 1100)])
@pytest.mark.parametrize("type_", ["f32", "bf16", "f16"])
def test_weights_of_each_head(shape, type_):
    say("layernorm heads", shape, type_)
    x, w, b, g = make(shape, type_, G=shape[-2], w32=True)
    check(x, w, b, g, 1e-6, groups=True)


def test_optional_weights():
    x, w, b, g = make((50, 96), "bf16")
    say("layernorm without weights")
    check(x, None, None, g, 1e-5)
    check(x, w, None, g, 1e-5)
    check(x, None, b, None, 1e-5)
    r = D.deer_layernorm(x, w, b)
    a = D.deer_layernorm_adjoint(x, g, r["mean"], r["rstd"], w, want_grads=False)
    full = D.deer_layernorm_adjoint(x, g, r["mean"], r["rstd"], w)
    assert a["grads"] == {} and torch.equal(a["x"], full["x"])


@pytest.mark.parametrize("type_", ["f32", "bf16"])
def test_large_offset(type_):
    """A mean far above the spread: the variance is no difference of large sums."""
    x, w, b, g = make((40, 700), type_, offset=300.0)
    say("layernorm offset", type_)
    check(x, w, b, g, 1e-5)


def test_special_rows():
    """A constant row (variance 0), rows with a NaN or an infinity: the others are as without them."""
    for D_ in (48, 1000, 9000):
        x, w, b, g = make((9, D_), "f32")
        say("layernorm special rows", D_)
        x[2] = 3.0
        want = D.deer_layernorm(x, w, b)
        wantg = D.deer_layernorm_adjoint(x, g, want["mean"], want["rstd"], w)
        assert torch.equal(want["y"][2], b) and torch.isfinite(wantg["x"]).all()
        y = x.clone()
        y[4, 5], y[6, 0] = torch.nan, torch.inf
        got = D.deer_layernorm(y, w, b)
        gotg = D.deer_layernorm_adjoint(y, g, got["mean"], got["rstd"], w)
        keep = [0, 1, 2, 3, 5, 7, 8]
        assert torch.equal(got["y"][keep], want["y"][keep]) and torch.equal(gotg["x"][keep], wantg["x"][keep])
        assert got["y"][4].isnan().all() and got["y"][6].isnan().any()


@pytest.mark.parametrize("type_,D_", [("bf16", 64), ("f32", 1024), ("f16", 4096), ("bf16", 3000)])
def test_alignment_and_layout(type_, D_):
    """An odd first element and a transposed x: the same bits as from an aligned copy."""
    x, w, b, g = make((12, D_), type_)
    say("layernorm alignment", type_, D_)
    want = D.deer_layernorm(x, w, b)
    wantg = D.deer_layernorm_adjoint(x, g, want["mean"], want["rstd"], w)
    odd = [torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")[1:].view(t.shape).copy_(t) for t in (x, w, b, g)]
    turned = [t.t().contiguous().t() if t.dim() == 2 else t for t in (x, w, b, g)]
    for xx, ww, bb, gg in (odd, turned):
        r = D.deer_layernorm(xx, ww, bb)
        assert all(torch.equal(r[n], want[n]) for n in r)
        a = D.deer_layernorm_adjoint(xx, gg, r["mean"], r["rstd"], ww)
        assert torch.equal(a["x"], wantg["x"]) and all(torch.equal(a["grads"][n], wantg["grads"][n]) for n in a["grads"])


def test_gradients_against_differences():
    x, w, b, g = make((60, 300), "f32")
    say("layernorm differences")
    r = D.deer_layernorm(x, w, b)
    a = D.deer_layernorm_adjoint(x, g, r["mean"], r["rstd"], w)
    gen = torch.Generator(device="cuda").manual_seed(2)

    def loss(x, w, b):
        return float((D.deer_layernorm(x, w, b)["y"].double() * g).sum())

    for i, (grad, e, tol) in enumerate(((a["x"], 1e-2, 1e-3), (a["grads"]["w"], 0.5, 1e-4), (a["grads"]["b"], 0.5, 1e-4))):
        d = torch.randn(grad.shape, device="cuda", generator=gen)
        args = [[x, w, b], [x, w, b]]
        for sgn, ar in zip((1, -1), args):
            ar[i] = ar[i] + sgn * e * d
        diff = (loss(*args[0]) - loss(*args[1])) / (2 * e)
        want = float((grad.double() * d).sum())
        assert abs(diff - want) < tol * float(grad.double().norm() * d.double().norm()), i


def test_streams_graphs_workspace():
    x, w, b, g = make((500, 6, 64), "bf16", G=6)
    say("layernorm stream and graph")
    want = D.deer_layernorm(x, w, b)
    wantg = D.deer_layernorm_adjoint(x, g, want["mean"], want["rstd"], w)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = D.deer_layernorm(x, w, b)
    s.synchronize()
    assert all(torch.equal(got[n], want[n]) for n in got)
    n = D.deer_layernorm_workspace_bytes(3000, 6, 64, torch.bfloat16)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    a = D.deer_layernorm_adjoint(x, g, want["mean"], want["rstd"], w, ws=ws)
    assert torch.equal(a["x"], wantg["x"]) and all(torch.equal(a["grads"][k], wantg["grads"][k]) for k in a["grads"])
    x2 = x.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = D.deer_layernorm(x2, w, b)
        ra = D.deer_layernorm_adjoint(x2, g, r["mean"], r["rstd"], w)
    for i in range(3):
        x2.copy_(x * (i + 1))
        graph.replay()
        torch.cuda.synchronize()
        e = D.deer_layernorm(x2, w, b)
        ea = D.deer_layernorm_adjoint(x2, g, e["mean"], e["rstd"], w)
        assert all(torch.equal(r[n], e[n]) for n in e)
        assert torch.equal(ra["x"], ea["x"]) and all(torch.equal(ra["grads"][k], ea["grads"][k]) for k in ea["grads"])


def test_refusals():
    x, w, b, g = make((6, 4, 10), "bf16", G=4)
    for args in ((x.cpu(), w, b), (x.double(), w, b), (x, w[:3], b), (x, w, b[:, :5]), (x, w.half(), b), (x, w, b.float())):
        with pytest.raises(ValueError):
            D.deer_layernorm(*args)
    with pytest.raises(D.DeerError):
        D.deer_layernorm(x, w, b, eps=-1.0)
    with pytest.raises(D.DeerError):
        D.deer_layernorm(x, w, b, y=x)
    with pytest.raises(D.DeerError):
        D.deer_layernorm(x[:0], w, b)
    r = D.deer_layernorm(x, w, b)
    with pytest.raises(ValueError):
        D.deer_layernorm_adjoint(x, g.float(), r["mean"], r["rstd"], w)
    with pytest.raises(ValueError):
        D.deer_layernorm_adjoint(x, g, r["mean"][:3], r["rstd"], w)
