"""The oracle of the paged cache against its definition, written another way."""
import numpy as np

from oracle import cache_ref as R


def test_rotation_is_a_complex_product():
    g = np.random.default_rng(1)
    x, a = g.standard_normal((3, 10)), g.uniform(-9, 9, 4)
    y = R.rotate(x, np.cos(a), np.sin(a), "pairs")
    z = (x[:, 0:8:2] + 1j * x[:, 1:8:2]) * np.exp(1j * a)
    assert np.allclose(y[:, 0:8:2], z.real) and np.allclose(y[:, 1:8:2], z.imag) and (y[:, 8:] == x[:, 8:]).all()
    y = R.rotate(x, np.cos(a), np.sin(a), "halves")
    z = (x[:, :4] + 1j * x[:, 4:8]) * np.exp(1j * a)
    assert np.allclose(y[:, :4], z.real) and np.allclose(y[:, 4:8], z.imag) and (y[:, 8:] == x[:, 8:]).all()


def test_attention_over_what_an_append_stored():
    """Relative positions: turned by their positions, scores depend on differences; and the attention of a whole sequence equals a dense one with a triangle's mask."""
    g = np.random.default_rng(2)
    n, Hq, Hkv, D, page, W = 13, 4, 2, 8, 3, 5
    q, k, v = g.standard_normal((n, Hq, D)), g.standard_normal((n, Hkv, D)), g.standard_normal((n, Hkv, D))
    table = np.array([[4, 0, 3, 1, 5]])
    ang = np.arange(15)[:, None] * np.array([[1.0, 0.1, 0.01, 0.001]])
    angles = np.concatenate([np.cos(ang), np.sin(ang)], 1)
    out, ks, vs = R.append(q, k, v, angles, [0, n], [n], table, page, 6, "halves")
    assert sorted(out) == list(range(n)) and len(ks) == n
    kc, vc = np.full((6, page, Hkv, D), np.nan), np.full((6, page, Hkv, D), np.nan)
    for at in ks:
        kc[at], vc[at] = ks[at], vs[at]
    turned = np.stack([out[t] for t in range(n)])
    o, spread, reach, seen = R.attention(turned, kc, vc, [0, n], [n], table, 0.3, True, W)
    i = np.arange(n)
    for h in range(Hq):
        a, b = q[:, h, :4] + 1j * q[:, h, 4:], k[:, h // 2, :4] + 1j * k[:, h // 2, 4:]
        x = 0.3 * np.real(np.einsum("id,jd,ijd->ij", a, b.conj(), np.exp(1j * (i[:, None, None] - i[None, :, None]) * ang[1])))
        x = np.where((i[None] <= i[:, None]) & (i[None] > i[:, None] - W), x, -np.inf)
        w = np.exp(x - x.max(1, keepdims=True))
        assert np.allclose(o[:, h], (w / w.sum(1, keepdims=True)) @ v[:, h // 2])
    assert (seen == np.minimum(i + 1, W)).all() and (spread >= np.abs(o) - 1e-12).all()


def test_places_that_are_none():
    table = np.array([[0, -1, 7]])
    assert R.place(table, 2, 3, 0, 1) == (0, 1) and R.place(table, 2, 3, 0, 2) is None and R.place(table, 2, 3, 0, 4) is None and R.place(table, 2, 3, 0, 6) is None and R.place(table, 2, 3, 0, -1) is None
    z = np.ones((1, 1, 8))
    o, _, _, seen = R.attention(z, np.ones((3, 2, 1, 8)), np.ones((3, 2, 1, 8)), [0, 1], [0], table, 1.0)
    assert (o == 0).all() and seen[0] == 0
