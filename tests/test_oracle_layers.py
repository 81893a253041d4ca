"""Pins of the layers' oracle: linear attention against its expanded sum, closed forms and central
differences; layer normalisation against torch's double-precision one and its autograd."""
import numpy as np
import pytest

from oracle import layers as L

torch = pytest.importorskip("torch")


def _case(B=2, T=6, H=4, Hk=2, Dk=3, Dv=2, per_step=True, seed=0):
    rng = np.random.default_rng(seed)
    n = rng.standard_normal
    ld = -rng.exponential(0.4, (B, T, H) if per_step else (H,))
    return dict(q=n((B, T, Hk, Dk)), k=n((B, T, Hk, Dk)), v=n((B, T, H, Dv)), log_decay=ld), \
        dict(scale=0.7, lengths=np.array([T, T - 2]), state0=n((B, H, Dk, Dv)))


def test_expanded_sum():
    """o_t = scale (sum_{j<=t} (q_t k_j) a_{j+1} ... a_t v_j + a_1 ... a_t S_0^T q_t)."""
    c, kw = _case()
    o, last = L.linattn(**c, **kw)
    for b in range(2):
        n = kw["lengths"][b]
        for h in range(4):
            a = np.exp(c["log_decay"][b, :, h])
            for t in range(n):
                q = c["q"][b, t, h // 2]
                ref = np.prod(a[:t + 1]) * kw["state0"][b, h].T @ q
                for j in range(t + 1):
                    ref = ref + np.prod(a[j + 1:t + 1]) * (q @ c["k"][b, j, h // 2]) * c["v"][b, j, h]
                assert np.allclose(o[b, t, h], 0.7 * ref, atol=1e-12)
        assert not o[b, n:].any()


def test_state_passes_on_and_zero_decay_starts_anew():
    c, kw = _case(per_step=True)
    kw["lengths"] = None
    o, last = L.linattn(**c, **kw)
    first = {k: x[:, :2] for k, x in c.items()}
    rest = {k: x[:, 2:] for k, x in c.items()}
    o1, s1 = L.linattn(**first, scale=0.7, state0=kw["state0"])
    o2, s2 = L.linattn(**rest, scale=0.7, state0=s1)
    assert np.allclose(np.concatenate([o1, o2], 1), o) and np.allclose(s2, last)
    c["log_decay"][:, 2] = -np.inf
    o, last = L.linattn(**c, **kw)
    o3, s3 = L.linattn(**{k: x[:, 2:] for k, x in c.items()}, scale=0.7)
    assert np.allclose(o[:, 2:], o3) and np.allclose(last, s3)


@pytest.mark.parametrize("per_step", [True, False])
def test_linattn_adjoint_differences(per_step):
    c, kw = _case(per_step=per_step, seed=3)
    rng = np.random.default_rng(9)
    g, gs = rng.standard_normal(c["v"].shape), rng.standard_normal(kw["state0"].shape)

    def loss(c, s0):
        o, last = L.linattn(**c, scale=kw["scale"], lengths=kw["lengths"], state0=s0)
        return (o * g).sum() + (last * gs).sum()

    grads = L.linattn_adjoint(**c, g=g, g_state=gs, **kw)
    e = 1e-6
    for name in ("q", "k", "v", "log_decay", "state0"):
        x = kw["state0"] if name == "state0" else c[name]
        for i in rng.choice(x.size, min(x.size, 12), replace=False):
            at = np.unravel_index(i, x.shape)
            old = x[at]
            x[at] = old + e
            up = loss(c, kw["state0"])
            x[at] = old - e
            down = loss(c, kw["state0"])
            x[at] = old
            assert abs((up - down) / (2 * e) - grads[name][at]) < 1e-6, (name, at)


def test_empty_sequence():
    c, kw = _case()
    kw["lengths"] = np.array([0, 3])
    o, last = L.linattn(**c, **kw)
    assert not o[0].any() and np.array_equal(last[0], kw["state0"][0])
    gs = np.ones_like(kw["state0"])
    gr = L.linattn_adjoint(**c, g=np.ones_like(o), g_state=gs, **kw)
    assert np.array_equal(gr["state0"][0], gs[0]) and not gr["q"][0].any() and not gr["log_decay"][0].any()


@pytest.mark.parametrize("groups", [False, True])
def test_layernorm_against_torch(groups):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 3, 7)) * 3 + 2
    shape = (3, 7) if groups else (7,)
    w, b, g = rng.standard_normal(shape), rng.standard_normal(shape), rng.standard_normal(x.shape)
    xt, wt, bt = (torch.tensor(a, requires_grad=True) for a in (x, w, b))
    yt = torch.nn.functional.layer_norm(xt, (7,), eps=1e-3) * wt + bt
    yt.backward(torch.tensor(g))
    y, mean, rstd = L.layernorm(x, w, b, 1e-3)
    gr = L.layernorm_adjoint(x, g, w, 1e-3, groups)
    assert np.allclose(y, yt.detach().numpy()) and np.allclose(mean, x.mean(-1))
    assert np.allclose(rstd, 1 / np.sqrt(x.var(-1) + 1e-3))
    for name, t in (("x", xt), ("w", wt), ("b", bt)):
        assert np.allclose(gr[name], t.grad.numpy()), name
