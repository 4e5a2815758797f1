"""Pins of the adapters' oracle (CPU): central differences, the dense form of one adapter, rows without an adapter; and of clipping."""
import numpy as np

from oracle import adapter_ref


def draw(seed, T=7, I=6, O=5, R=3, n=3):
    r = np.random.default_rng(seed)
    f = r.standard_normal
    return f((T, I)), f((O, I)), f((n, R, I)), f((n, O, R)), 0.5 + r.random(n), r.integers(-1, n, T), f((T, O))


def test_gradients_against_central_differences():
    x, w, a, b, scale, ids, dout = draw(0)
    g = adapter_ref.adapter_bwd(x, w, a, b, scale, ids, dout)
    loss = lambda: float(np.sum(dout * adapter_ref.adapter_fwd(x, w, a, b, scale, ids)["out"]))
    eps = 1e-5
    for t, d in ((x, g["dx"]), (a, g["da"]), (b, g["db"])):
        for i in np.ndindex(t.shape):
            keep = t[i]
            t[i] = keep + eps
            up = loss()
            t[i] = keep - eps
            down = loss()
            t[i] = keep
            assert abs((up - down) / (2 * eps) - d[i]) < 1e-7


def test_one_adapter_is_a_changed_weight():
    x, w, a, b, scale, _, dout = draw(1)
    ids = np.full(len(x), 2)
    full = w + scale[2] * b[2] @ a[2]
    np.testing.assert_allclose(adapter_ref.adapter_fwd(x, w, a, b, scale, ids)["out"], x @ full.T, rtol=1e-12, atol=1e-12)
    g = adapter_ref.adapter_bwd(x, w, a, b, scale, ids, dout)
    np.testing.assert_allclose(g["dx"], dout @ full, rtol=1e-12, atol=1e-12)
    assert not g["da"][:2].any() and not g["db"][:2].any()


def test_rows_without_an_adapter_take_the_projection_alone():
    x, w, a, b, scale, ids, dout = draw(2)
    out = adapter_ref.adapter_fwd(x, w, a, b, scale, ids)
    bare = ids < 0
    np.testing.assert_allclose(out["out"][bare], (x @ w.T)[bare], rtol=1e-13, atol=1e-13)
    assert not out["hidden"][bare].any()


def test_clip():
    g = [np.array([3.0, 0.0]), np.array([[4.0]])]
    norm, c = adapter_ref.clip(g, 1.0)
    assert norm == 5.0 and abs(np.sqrt(sum(np.sum(v * v) for v in c)) - 1.0) < 1e-6
    norm, c = adapter_ref.clip(g, 6.0)
    assert all(np.array_equal(u, v) for u, v in zip(g, c))
    norm, c = adapter_ref.clip([np.array([np.inf, 1.0])], 1.0)
    assert np.isinf(norm) and np.isnan(c[0][0]) and c[0][1] == 0.0
    assert np.isnan(adapter_ref.clip([np.array([np.nan, 1.0])], 1.0)[1][0][1])
