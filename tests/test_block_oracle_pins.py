"""Pins of the 64-bit oracle of the gated recurrence and of the norms around a mixer: hand-computed values, and its gradients
against central differences."""
import numpy as np
import pytest

from oracle import block_oracle as bo


def test_recurrence_by_hand():
    half = np.log(0.5)
    x, la = np.array([[[1.0], [2.0], [3.0]]]), np.array([[[half], [-np.inf], [half]]])
    out, h = bo.rec_fwd(x, la, np.array([[4.0]]))
    assert out.ravel().tolist() == [3.0, 2.0, 4.0] and h.ravel().tolist() == [4.0]
    out, h = bo.rec_fwd(x, la, np.array([[4.0]]), coupled=True)
    np.testing.assert_allclose(out.ravel(), [2.5, 2.0, 2.5])
    out, h = bo.rec_fwd(x, la, np.array([[4.0]]), lens=np.array([1]))
    assert out.ravel().tolist() == [3.0, 0.0, 0.0] and h.ravel().tolist() == [3.0]
    out, h = bo.rec_fwd(x, la, np.array([[4.0]]), lens=np.array([0]))
    assert not out.any() and h.ravel().tolist() == [4.0]


def differences(f, x, eps=1e-5):
    """Central differences of f() in every element of x, which f reads."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + eps
        up = f()
        x[i] = keep - eps
        g[i] = (up - f()) / (2 * eps)
        x[i] = keep
    return g


@pytest.mark.parametrize("coupled", [False, True])
@pytest.mark.parametrize("lens", [None, [3, 0, 5]])
def test_recurrence_gradients_by_differences(coupled, lens):
    rng = np.random.default_rng(5)
    B, N, D = 3, 5, 2
    x, la, h = rng.normal(size=(B, N, D)), -np.abs(rng.normal(size=(B, N, D))) - 0.1, rng.normal(size=(B, D))
    dout, dh = rng.normal(size=(B, N, D)), rng.normal(size=(B, D))
    lens = None if lens is None else np.array(lens)

    def loss():
        out, h_out = bo.rec_fwd(x, la, h, lens, coupled)
        return (out * dout).sum() + (h_out * dh).sum()

    dx, dl, dh_in = bo.rec_bwd(x, la, dout, h, lens, dh, coupled)
    for got, var in ((dx, x), (dl, la), (dh_in, h)):
        np.testing.assert_allclose(got, differences(loss, var), rtol=1e-6, atol=1e-8)


def test_norms_by_hand():
    r_out, y = bo.addnorm_fwd(np.array([[1.0, 5.0]]), np.array([[2.0, -2.0]]), np.array([1.0, 0.5]), np.array([2.0, 1.0]), 0.0)
    assert r_out.tolist() == [[3.0, 4.0]]
    np.testing.assert_allclose(y, [[6.0 / np.sqrt(12.5), 4.0 / np.sqrt(12.5)]])
    o = np.array([3.0, 4.0, 0.0, 2.0]).reshape(1, 2, 1, 2)
    got = bo.gatenorm(o, np.array([0.0, 1.0, 2.0, 3.0]).reshape(1, 1, 4), None, 0.0, "identity", "head")["y"].ravel()
    np.testing.assert_allclose(got, [0.0, 4.0 / np.sqrt(12.5), 0.0, 3.0 * 2.0 / np.sqrt(2.0)])
    got = bo.gatenorm(o, None, None, 0.0, "none", "token")["y"].ravel()
    np.testing.assert_allclose(got, np.array([3.0, 4.0, 0.0, 2.0]) / np.sqrt(29.0 / 4.0))


def test_norm_gradients_by_differences():
    rng = np.random.default_rng(6)
    r, x, dy, dr_out = (rng.normal(size=(3, 8)) for _ in range(4))
    scale, w = rng.normal(size=8), rng.normal(size=8)

    def loss():
        r_out, y = bo.addnorm_fwd(r, x, scale, w, 1e-3)
        return (y * dy).sum() + (r_out * dr_out).sum()

    got = bo.addnorm_bwd(r + scale * x, x, scale, w, 1e-3, dy, dr_out)
    for name, var in (("dr", r), ("dx", x), ("dscale", scale), ("dweight", w)):
        np.testing.assert_allclose(got[name], differences(loss, var), rtol=1e-5, atol=1e-7)


@pytest.mark.parametrize("gate", ["none", "identity", "sigmoid", "silu"])
@pytest.mark.parametrize("over", ["head", "token"])
def test_gate_gradients_by_differences(gate, over):
    rng = np.random.default_rng(7)
    B, H, N, D = 2, 3, 2, 4
    o, u, w, dy = rng.normal(size=(B, H, N, D)), rng.normal(size=(B, N, H * D)), rng.normal(size=H * D), rng.normal(size=(B, N, H * D))
    got = bo.gatenorm(o, u, w, 1e-3, gate, over, dy)
    loss = lambda: (bo.gatenorm(o, u, w, 1e-3, gate, over)["y"] * dy).sum()   # noqa: E731
    for name, var in (("do", o), ("dweight", w)) + ((("du", u),) if gate != "none" else ()):
        np.testing.assert_allclose(got[name], differences(loss, var), rtol=1e-5, atol=1e-7)
