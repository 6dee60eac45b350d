"""The 64-bit references of what stands around the experts' products (oracle/layer_ref.py), pinned by worked examples and by differences."""
import numpy as np
import pytest

from oracle import layer_ref as R

RNG = np.random.Generator(np.random.Philox(19092))


def test_norm_by_hand():
    y, rho = R.rmsnorm(np.array([[3.0, 4.0, 0.0, 0.0], [0.0, 0.0, 0.0, 0.0]]), np.array([1.0, 2.0, 1.0, 1.0]), 0.25)
    assert rho[0, 0] == pytest.approx(1 / np.sqrt(6.5)) and rho[1, 0] == 2.0
    assert y[0] == pytest.approx(np.array([3.0, 8.0, 0.0, 0.0]) / np.sqrt(6.5)) and (y[1] == 0).all()


def test_scales_by_hand():
    y = np.zeros((1, 300))
    y[0, 5], y[0, 130], y[0, 299] = -896.0, 448.0, 449.0
    assert R.scales(y, "f32").tolist() == [[2.0, 1.0, 449.0 / 448.0]]
    assert R.scales(y, "e8m0").tolist() == [[2.0, 1.0, 2.0]]           # the smallest power of two not below
    assert R.scales(np.zeros((1, 3)), "e8m0").tolist() == [[1.0]]
    assert R.scales(np.full((1, 2), 1e-44), "f32").tolist() == [[2.0 ** -126]]
    assert R.spread(np.array([[2.0, 3.0]]), 130)[0, 126:].tolist() == [2.0, 2.0, 3.0, 3.0]


def test_routing_by_hand():
    logits = np.log(np.array([[1.0, 4.0, 2.0, 1.0]]))
    ids, w = R.route(logits, 2)
    assert ids.tolist() == [[1, 2]] and w == pytest.approx(np.array([[2 / 3, 1 / 3]]))
    ids, w = R.route(logits, 2, renorm=False, scale=8.0)
    assert w == pytest.approx(np.array([[4.0, 2.0]]))
    # a bias decides who is chosen, not the weight; equal choices: the lower index
    ids, w = R.route(logits, 2, bias=np.array([0.5, 0.0, 0.0, 0.5]), renorm=False)
    assert ids.tolist() == [[0, 3]] and w == pytest.approx(np.array([[0.125, 0.125]]))
    # two groups of two: by the maximum the first, by the sum of both the first as well; then only its experts
    assert R.route(logits, 2, groups=2, kept=1)[0].tolist() == [[1, 0]]
    ids, _ = R.route(np.log(np.array([[1.0, 4.0, 3.0, 3.0]])), 1, groups=2, kept=1, top2=True)
    assert ids.tolist() == [[2]]
    # masks
    ids, w = R.route(np.array([[-np.inf, 1.0, np.nan], [-np.inf] * 3]), 2)
    assert ids.tolist() == [[1, -1], [-1, -1]] and w.tolist() == [[1.0, 0.0], [0.0, 0.0]]


def test_order_and_rows_by_hand():
    ids = np.array([[2, 0], [0, -1], [2, 1]])
    rows, row_of = R.experts_order(ids, 3)
    assert rows.tolist() == [0, 2, 3, 5] and row_of.tolist() == [[3, 0], [1, -1], [4, 2]]
    x = np.array([[1.0], [2.0], [3.0]])
    a = R.dispatch(x, row_of, 6, fill=9.0)
    assert a[:, 0].tolist() == [1.0, 2.0, 3.0, 1.0, 3.0, 9.0]
    w = np.array([[0.5, 0.25], [2.0, 7.0], [1.0, 1.0]])
    assert R.combine(a, row_of, w)[:, 0].tolist() == [0.75, 4.0, 6.0]
    d, dw = R.combine_backward(np.array([[1.0], [10.0], [100.0]]), a, row_of, w)
    assert d[:, 0].tolist() == [0.25, 20.0, 100.0, 0.5, 100.0, 0.0] and dw.tolist() == [[1.0, 1.0], [20.0, 0.0], [300.0, 300.0]]


def differences(f, x, step=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[i] = step
        g[i] = (f(x + e) - f(x - e)) / (2 * step)
    return g


def test_gradients_against_differences():
    h, w, g = RNG.standard_normal((3, 9)), RNG.standard_normal(9), RNG.standard_normal((3, 9))
    dx, dw = R.rmsnorm_backward(g, h, w, 1e-3)
    assert dx == pytest.approx(differences(lambda t: (R.rmsnorm(t, w, 1e-3)[0] * g).sum(), h), abs=1e-7)
    assert dw == pytest.approx(differences(lambda t: (R.rmsnorm(h, t, 1e-3)[0] * g).sum(), w), abs=1e-7)
    for kind in ("softmax", "sigmoid"):
        for renorm in (True, False):
            logits, gw = RNG.standard_normal((3, 7)), RNG.standard_normal((3, 3))
            ids = R.route(logits, 3, kind)[0]
            ids[1, 2] = -1
            want = differences(lambda t: (R.route_weights(t, ids, kind, renorm, 1.7) * gw).sum(), logits)
            assert R.route_backward(logits, ids, gw, kind, renorm, 1.7) == pytest.approx(want, abs=1e-7), (kind, renorm)
