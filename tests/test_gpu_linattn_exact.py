"""Linear attention on the GPU where float32 arithmetic is exact: operands on a grid so coarse that
every product and every sum of magnitudes has at most 24 bits, decays of one.  However the sums are
ordered, a result is then the exact one rounded once to its type, and is compared bit for bit."""
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
GRID = 2.0 ** -10       # of every result
MOST = 8                # elements of a row that are not zero


def rows(rng, shape, wide):
    """1, 0 or -1, or 7-bit numbers of two sizes (products of 10 to 20 bits of the grid); at most MOST of
    each row are not zero."""
    x = rng.integers(-127, 128, shape) * rng.choice([2.0 ** -5, 2.0 ** -2], shape) if wide else \
        rng.integers(-1, 2, shape).astype(np.float64)
    x[rng.random(shape).argsort(-1) >= MOST] = 0.0
    return x


def rounded(x, type_):
    assert (np.abs(x) < 2.0 ** 24 * GRID).all() and (x == np.rint(x / GRID) * GRID).all()
    return torch.tensor(x).float().to(type_).cuda()       # float32 holds it, so this rounds once


def same(name, got, want):
    off = int((got != want).sum())
    assert off == 0, (name, off, got.numel())


@pytest.mark.parametrize("type_", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,T,H,Hk,Dk,Dv", [(16, 6, 4, 2, 16, 24), (1, 70, 8, 8, 64, 64), (40, 40, 8, 4, 64, 128),
                                            (1, 9, 2, 2, 256, 256), (17, 33, 16, 8, 128, 128)])
@pytest.mark.parametrize("large", ["states", "q and k", "v and g"])
def test_rounded_once(type_, B, T, H, Hk, Dk, Dv, large):
    """States of 20 bits, then scores q k and v g of as many, on their way to outputs of 8, 11 or 24:
    none is rounded in between."""
    say("linattn rounded once", type_, B, T, H, Hk, Dk, Dv, large)
    rng = np.random.default_rng(B + T + Dv)
    q, k = (rows(rng, (B, T, Hk, Dk), large == "q and k") for _ in range(2))
    v, g = (rows(rng, (B, T, H, Dv), large == "v and g") for _ in range(2))
    s0 = gs = None
    if large == "states":
        s0, gs = (rng.integers(-2 ** 19, 2 ** 19, (B, H, Dk, Dv)) * GRID for _ in range(2))
    ld = np.zeros(H)
    t = TYPES[type_]
    dev = {n: torch.tensor(x).to(t).cuda() for n, x in (("q", q), ("k", k), ("v", v))}
    dev["log_decay"] = torch.zeros(H, device="cuda")
    dg = torch.tensor(g).to(t).cuda()
    d0, dgs = (None if x is None else torch.tensor(x).float().cuda() for x in (s0, gs))
    # every sum of magnitudes stays within 24 bits
    mags = [None if x is None else np.abs(x) for x in (q, k, v, g, s0, gs)]
    oa, _ = L.linattn(*mags[:3], ld, state0=mags[4])
    ga = L.linattn_adjoint(*mags[:3], ld, mags[3], state0=mags[4], g_state=mags[5])
    assert all((x < 2.0 ** 24 * GRID).all() for x in (oa, ga["q"], ga["k"], ga["v"]))

    o, last = L.linattn(q, k, v, ld, state0=s0)
    r = D.deer_linattn(**dev, state0=d0, want_state=True)
    same("o", r["o"], rounded(o, t))
    same("state", r["state"], rounded(last, torch.float32))
    ref = L.linattn_adjoint(q, k, v, ld, g, state0=s0, g_state=gs)
    for want_decay in (True, False):
        got = D.deer_linattn_adjoint(**dev, g=dg, state0=d0, g_state=dgs, want_decay=want_decay)["grads"]
        for n in ("q", "k", "v"):
            same(n, got[n], rounded(ref[n], t))
        if s0 is not None:
            same("state0", got["state0"], rounded(ref["state0"], torch.float32))


def odd(rng, top, *shape):
    """Odd whole numbers of either sign in the upper half of 1..top: every bit of the type is used."""
    return (rng.integers(top // 4, top // 2, shape) * 2 + 1) * rng.choice([-1.0, 1.0], shape)


@pytest.mark.parametrize("type_,top", [("bf16", 255), ("f16", 2047)])
@pytest.mark.parametrize("B,H", [(1, 16), (64, 64)])
def test_whole_products(type_, top, B, H):
    """Two steps of one row and column, operands of all their bits, decays of one: scores of 22 bits,
    and the gradient of the second step's decay, which is scale q_2 g_2 k_1 v_1, to the last bit."""
    say("linattn whole products", type_, B, H)
    rng = np.random.default_rng(B)
    scale = 2.0 ** -12
    t = TYPES[type_]
    ld = np.zeros((B, 2, H))
    for pair in (("q", "k"), ("v", "g")):
        x = {n: odd(rng, top, B, 2, H, 1) if n in pair else rng.choice([-1.0, 1.0], (B, 2, H, 1)) for n in "qkvg"}
        dev = {n: torch.tensor(y).to(t).cuda() for n, y in x.items()}
        g = dev.pop("g")
        dev["log_decay"] = torch.zeros(B, 2, H, device="cuda")
        # (sums of at most two products of 22 bits)
        o, last = L.linattn(x["q"], x["k"], x["v"], ld, scale=scale)
        r = D.deer_linattn(**dev, scale=scale, want_state=True)
        ref = L.linattn_adjoint(x["q"], x["k"], x["v"], ld, x["g"], scale=scale)
        got = D.deer_linattn_adjoint(**dev, g=g, scale=scale)["grads"]
        for name, a, want in (("o", r["o"], o), ("state", r["state"], last), *((n, got[n], ref[n]) for n in "qkv"),
                              ("log_decay", got["log_decay"], ref["log_decay"])):
            same(name, a, torch.tensor(want).float().to(a.dtype).cuda())


@pytest.mark.parametrize("seg", [1 << 20, 25024])     # one segment, or eight
@pytest.mark.parametrize("per_step", [False, True])
def test_slow_decays(seg, per_step, monkeypatch):
    """200000 steps that only decay, by e^-5 and e^-0.3 in all: what is left is off by the few roundings at
    the segments' ends, not by one for each of 3125 chunks of steps (2^-25 a chunk, the same way each time,
    would be 1500 half steps). A half step is 2^-24. At each of n segments' ends: the decay's factor (two,
    of a hardware exponential, and one of its exponent), the sum; at the last: the power of two, its
    exponent, a product, and the step that the adjoint adds (four)."""
    monkeypatch.setenv("DEER_LIN_SEG", str(seg))
    say("linattn slow decays", seg, per_step)
    B, T, H, Dk, Dv = 1, 200000, 2, 8, 8
    rng = np.random.default_rng(3)
    ld = np.array([-2.5e-5, -1.5e-6], np.float32)
    s0, gs = (torch.tensor(rng.standard_normal((B, H, Dk, Dv))).float().cuda() for _ in range(2))
    zero = torch.zeros(B, T, H, Dk, device="cuda")
    dec = torch.tensor(ld).cuda()
    args = (zero, zero, zero, dec.expand(B, T, H) if per_step else dec)
    left = torch.tensor(np.exp(ld.astype(np.float64) * T)).cuda()[:, None, None]
    tol = 2.0 ** -24 * (4 * -(-T // seg) + 8)
    state = D.deer_linattn(*args, state0=s0, want_state=True)["state"]
    assert ((state.double() / (s0.double() * left) - 1).abs() <= tol).all()
    back = D.deer_linattn_adjoint(*args, zero, state0=s0, g_state=gs)["grads"]["state0"]
    assert ((back.double() / (gs.double() * left) - 1).abs() <= tol).all()
