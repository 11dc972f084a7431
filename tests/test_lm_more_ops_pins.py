"""CPU pins of the oracle of the norm with the residual, the gated recurrence and the distillation loss (oracle/lm_ops.py):
gradients against central differences, closed forms, what padding and empty rows do."""
import numpy as np
import pytest

from oracle import lm_ops as O


def rng(*seed):
    return np.random.Generator(np.random.PCG64(list(seed)))


def slopes(f, x, h=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[i] = h
        g[i] = (f(x + e) - f(x - e)) / (2 * h)
    return g


@pytest.mark.parametrize("width", [1, 2, 7, 33])
def test_rms_norm_gradients_against_differences(width):
    r = rng(1, width)
    s, gain, dy, dsum = r.normal(size=(3, width)), r.normal(size=width), r.normal(size=(3, width)), r.normal(size=(3, width))
    ds, dg, dsa, dga = O.rms_norm_backward(dy, s, gain, dsum, 1e-3)
    total = lambda s_, g_: (O.rms_norm_forward(s_, g_, 1e-3) * dy).sum() + (s_ * dsum).sum()
    assert abs(slopes(lambda v: total(v, gain), s) - ds).max() < 1e-6
    assert abs(slopes(lambda v: total(s, v), gain) - dg).max() < 1e-6
    assert (dsa + abs(dsum) >= abs(ds) - 1e-12).all() and (dga >= abs(dg) - 1e-12).all()


def test_rms_norm_of_a_row_of_one_size():
    y = O.rms_norm_forward(np.array([[3.0, -3.0, 3.0, 3.0]]), np.ones(4), 1e-12)
    assert np.allclose(y, [[1, -1, 1, 1]])


def test_recurrence_with_a_constant_gate_is_a_geometric_sum():
    T, a = 12, 0.75
    f, z = np.full((T, 1), np.log(3.0)), np.ones((T, 1))
    r = O.recurrence_forward(f, z, None, [0, T], np.array([[2.0]]))
    want = 1.0 + (2.0 - 1.0) * a ** np.arange(1, T + 1)
    assert np.allclose(r["y"][:, 0], want) and np.allclose(r["final"], want[-1])
    assert np.allclose(r["before"][0], 2.0)


@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("state", [False, True])
def test_recurrence_gradients_against_differences(gate, state):
    r = rng(2, gate, state)
    T, C, off = 9, 2, [0, 3, 3, 8]    # a sequence without tokens, and a row of no sequence
    f, z, dy = (r.normal(size=(T, C)) for _ in range(3))
    o = r.normal(size=(T, C)) if gate else None
    h0 = r.normal(size=(3, C)) if state else None
    dfin = r.normal(size=(3, C))

    def total(f_, z_, o_, h_):
        w = O.recurrence_forward(f_, z_, o_, off, h_)
        return (w["y"] * dy).sum() + (w["final"] * dfin).sum()
    w = O.recurrence_forward(f, z, o, off, h0)
    g = O.recurrence_backward(dy, f, z, o, off, w, dfin)
    live = np.arange(T)[:, None] < 8
    assert abs(slopes(lambda v: total(v, z, o, h0), f) - g["df"] * live).max() < 1e-6
    assert abs(slopes(lambda v: total(f, v, o, h0), z) - g["dz"] * live).max() < 1e-6
    if gate:
        assert abs(slopes(lambda v: total(f, z, v, h0), o) - g["do"] * live).max() < 1e-6
    if state:
        assert abs(slopes(lambda v: total(f, z, o, v), h0) - g["dstate"]).max() < 1e-6
        assert np.array_equal(w["final"][1], h0[1]) and np.array_equal(g["dstate"][1], dfin[1])


def test_gates_keep_their_relative_precision():
    f = np.array([-700.0, -40.0, -1.0, 0.0, 1.0, 40.0, 700.0])
    a, b = O.gates(f)
    assert np.allclose(a[:2], np.exp(f[:2]), rtol=1e-14) and np.allclose(b[-2:], np.exp(-f[-2:]), rtol=1e-14)
    assert np.allclose(a, O.sigmoid(f)) and np.array_equal(a, b[::-1])


@pytest.mark.parametrize("tau,mix", [(1.0, 0.0), (2.0, 0.0), (0.5, 0.3), (3.0, 1.0)])
def test_distillation_gradient_against_differences(tau, mix):
    r = rng(3, int(10 * tau), int(10 * mix))
    z, t = 2 * r.normal(size=(5, 11)), 2 * r.normal(size=(5, 4))
    ids = np.array([[3, 1, 9, 0], [3, 3, -1, 10], [-1, 11, -5, 11], [2, 2, 2, 2], [0, 1, 2, 3]])
    t[4, 2] = -np.inf
    labels = np.array([3, 0, 5, -1, 2]) if mix else None
    w = np.array([1.0, 0.5, 2.0, 1.0, 0.0])
    d = O.distill(z, ids, t, tau, labels, mix, w)
    got = slopes(lambda v: (O.distill(v, ids, t, tau, labels, mix, w)["loss"] * w).sum(), z)
    assert abs(got - d["dz"]).max() < 1e-6
    assert not d["dz"][4].any()
    assert abs(d["dz"].sum(1)).max() < 1e-12          # a shift of all logits changes nothing
    if not mix:
        assert d["loss"][2] == 0 and not d["dz"][2].any()   # no entry that counts


def test_distillation_from_the_student_itself_costs_nothing():
    z = rng(4).normal(size=(2, 6))
    d = O.distill(z, np.tile(np.arange(6), (2, 1)), z, 2.0, None, 0.0, np.ones(2))
    assert abs(d["loss"]).max() < 1e-14 and abs(d["dz"]).max() < 1e-14
