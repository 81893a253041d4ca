"""Linear attention with decays above one over whole segments, on the GPU against the float64 oracle:
a segment's product of decays passes float32's range where the state that it multiplies is zero or
tiny, and every state and result lies well inside the range.

Tolerances: those of test_gpu_linattn, and for the decays, whose exponents are large here, one more term.
An exponent e is rounded to 24 bits, which moves exp2(e) by |e| ln 2 2^-24; the exponents that a
term meets add up to at most the growth of 166 (128 steps of e^0.9), the decays elsewhere (memories of
3 steps and more over 64: below 32 a chunk) and the registers' scale (24 a chunk).
"""
import pytest

from gpu_util import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import test_gpu_linattn as A  # noqa: E402


@pytest.mark.parametrize("type_", ["f32", "bf16"])
@pytest.mark.parametrize("T,seg", [(500, 128), (600, 128), (1100, 320)])    # four, five and four segments
def test_growth_over_a_segment(type_, T, seg, monkeypatch):
    """The second segment grows by e^115. Heads 0 and 1: nothing enters it, forwards or backwards; heads 2
    and 3: states of 2^-83 do, and leave it with 2^83."""
    monkeypatch.setenv("DEER_LIN_SEG", str(seg))
    say("linattn growth over a segment", type_, T, seg)
    c, kw, g, _ = A.make(1, T, 4, 4, 24, 40, type_, True, False)
    lo, hi = seg, 2 * seg
    c["log_decay"].clamp_(min=-0.2, max=-0.02)
    c["log_decay"][:, lo:hi] = 0.9 * 128 / seg
    c["k"][:, :hi - 6, :2] = 0
    g[:, lo + 6:, :2] = 0
    c["k"][:, lo:hi, 2:] = 0
    g[:, lo:hi, 2:] = 0
    c["k"][:, :lo, 2:] *= 1e-25
    g[:, hi:, 2:] *= 1e-25
    check(c, kw, g, monkeypatch)


@pytest.mark.parametrize("type_", ["f32", "bf16"])
@pytest.mark.parametrize("T", [500, 900])                                    # four and eight segments
def test_growth_everywhere(type_, T, monkeypatch):
    """One decay above one for each head: the states are zero up to the last 64 steps, backwards up to the
    first."""
    monkeypatch.setenv("DEER_LIN_SEG", "128")
    say("linattn growth everywhere", type_, T)
    c, kw, g, _ = A.make(1, T, 2, 1, 24, 40, type_, False, False)
    c["log_decay"] = torch.tensor([0.9, 0.7], device="cuda")
    c["k"][:, :-64] = 0
    g[:, 64:] = 0
    check(c, kw, g, monkeypatch)


@pytest.mark.parametrize("type_", ["f32", "bf16"])
@pytest.mark.parametrize("seg", [128, 1 << 20])
def test_large_states(type_, seg, monkeypatch):
    """States of up to 2^122 that decay by e^-16 and e^-6 over 64 steps, and products k v as large."""
    monkeypatch.setenv("DEER_LIN_SEG", str(seg))
    say("linattn large states", type_, seg)
    c, kw, g, _ = A.make(1, 300, 2, 1, 8, 40, type_, True, True)
    c["log_decay"].fill_(-0.25)
    c["log_decay"][:, :, 1] = -0.1
    c["k"].clamp_(-1, 1)
    c["v"].clamp_(-2, 2).mul_(2.0 ** 118)
    c["q"].clamp_(-2, 2).mul_(2.0 ** -6)
    g.clamp_(-2, 2).mul_(2.0 ** -6)
    kw["scale"] = 1.0
    kw["state0"].clamp_(-2, 2).mul_(2.0 ** 121)
    check(c, kw, g, monkeypatch)


def check(c, kw, g, monkeypatch):
    plain, extra = A.kappa, 2.0 ** -24 * (166 + (32 + 24) * -(-c["v"].shape[1] // 64))
    monkeypatch.setattr(A, "kappa", lambda c, state=False: plain(c, state) + extra)
    A.check_forward(c, kw)
    A.check_adjoint(c, kw, g, None)
