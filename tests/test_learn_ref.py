"""The 64-bit forms that the GPU tests of the learner's operators compare with: worked cases, and
their gradients against central differences."""
import numpy as np
import pytest

import learn_ref as ref


def test_returns_worked_case():
    """Rewards 1, 0, 2, 0, 4 with gamma 1/2, an episode ending at step 2, value 8 afterwards."""
    x = np.array([1.0, 0.0, 2.0, 0.0, 4.0]).reshape(5, 1, 1)
    cut = np.array([[0], [0], [1], [0], [0]])
    out = ref.scan(x, np.array([0.5]), h0=np.array([[8.0]]), cut=cut, reverse=True)
    assert out["y"][0].ravel().tolist() == [1.5, 1.0, 2.0, 4.0, 8.0]


def test_memory_worked_case():
    x = np.array([4.0, 8.0]).reshape(2, 1, 1)
    g = np.zeros((2, 1, 1))
    out = ref.scan(x, g, h0=np.array([[2.0]]), form="gated")
    assert out["y"][0].ravel().tolist() == [3.0, 5.5]
    out = ref.scan(x, g, h0=np.array([[np.nan]]), cut=np.array([[1], [0]]), form="gated")
    assert out["y"][0].ravel().tolist() == [2.0, 5.0]


@pytest.mark.parametrize("form", ["linear", "gated"])
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("columns", [False, True])
def test_scan_gradient_against_differences(form, reverse, columns):
    r = np.random.default_rng(3)
    T, B, D = 6, 2, 3
    x, h0 = r.normal(size=(T, B, D)), r.normal(size=(B, D))
    gate = r.normal(size=(D,) if columns else (T, B, D)) * 0.5
    cut = (r.random((T, B)) < 0.3).astype(int)
    dy, dlast = r.normal(size=(T, B, D)), r.normal(size=(B, D))

    def loss():
        o = ref.scan(x, gate, h0, cut, form, reverse)
        return (o["y"][0] * dy).sum() + (o["last"][0] * dlast).sum()
    out = ref.scan(x, gate, h0, cut, form, reverse, dy, dlast)
    for name, v in (("dx", x), ("dgate", gate), ("dh0", h0)):
        for at in np.ndindex(v.shape):
            old, step = v[at], 1e-5
            v[at] = old + step
            up = loss()
            v[at] = old - step
            down = loss()
            v[at] = old
            # third derivatives are of order one: the difference is off by about step^2
            assert abs((up - down) / (2 * step) - out[name][0][at]) < 1e-8, (name, at)


def test_tokens_worked_case():
    l = np.log(np.array([[1.0, 2.0, 1.0], [0.0, 1.0, 0.0]]) + 1e-300)
    l[1, [0, 2]] = -np.inf
    out = ref.tokens(l, np.array([1, 0]), top=3)
    assert np.allclose(out["logp"][0], [np.log(0.5), -np.inf])
    assert np.allclose(out["entropy"][0], [1.5 * np.log(2.0), 0.0])
    assert out["top_ids"].tolist() == [[1, 0, 2], [1, -1, -1]]


def test_tokens_gradient_against_differences():
    r = np.random.default_rng(4)
    l, ids = r.normal(size=(4, 5)), np.array([0, 4, -1, 2])
    l[3, 1] = -np.inf
    g, gh = r.normal(size=4), r.normal(size=4)

    def loss():
        o = ref.tokens(l, ids)
        return (o["logp"][0] * g).sum() + (o["entropy"][0] * gh).sum()
    d = ref.tokens(l, ids, g, gh)["dlogits"][0]
    for at in np.ndindex(l.shape):
        if not np.isfinite(l[at]):
            assert d[at] == 0
            continue
        old, step = l[at], 1e-5
        l[at] = old + step
        up = loss()
        l[at] = old - step
        down = loss()
        l[at] = old
        assert abs((up - down) / (2 * step) - d[at]) < 1e-8, at


def test_draw_worked_case():
    l = np.log(np.array([[1.0, 2.0, 1.0]] * 5))
    l[4] = [-np.inf, 0.0, -np.inf]
    a, logp = ref.draw(l, np.array([0.0, 0.24, 0.26, 0.76, 0.999]))
    assert a.tolist() == [0, 0, 1, 2, 1]
    assert np.allclose(logp, np.log([0.25, 0.25, 0.5, 0.25, 1.0]))
