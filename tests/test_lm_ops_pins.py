"""CPU pins of the oracle of the language-model operators (oracle/lm_ops.py): gradients against central differences
and the adjoint identity, the 8-bit blocks against their defining properties."""
import numpy as np
import pytest

from oracle import lm_ops as O


def rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def test_embedding_gradient_is_the_adjoint_of_the_lookup():
    r = rng(1)
    W, ids = r.normal(size=(7, 5)), np.array([3, 3, -1, 6, 0, 7, 3], np.int32)
    dy = r.normal(size=(7, 5))
    y = O.embedding_forward(ids, W, 1.5)
    g, a, n = O.embedding_backward(ids, dy, 7, 1.5)
    assert abs((y * dy).sum() - (g * W).sum()) < 1e-12
    assert not y[2].any() and not y[5].any() and n.tolist() == [1, 0, 0, 3, 0, 0, 1]
    assert (a >= abs(g) - 1e-15).all()


@pytest.mark.parametrize("dim,rotary,inter", [(8, 8, False), (8, 8, True), (7, 4, False), (6, 0, False), (5, 2, True), (1, 0, False)])
def test_norm_and_rotation_gradients_against_differences(dim, rotary, inter):
    r = rng(2 + dim + rotary)
    x, gain, dy = r.normal(size=(3, 2, dim)), r.normal(size=dim), r.normal(size=(3, 2, dim))
    pos = np.array([0, 5, 1 << 20])
    f = lambda x_, g_: (O.norm_rope_forward(x_, g_, pos, rotary, 10000.0, inter, 1e-3)[0] * dy).sum()
    dx, dg, _, _ = O.norm_rope_backward(dy, x, gain, pos, rotary, 10000.0, inter, 1e-3)
    h = 1e-6
    for i in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[i] = h
        assert abs((f(x + e, gain) - f(x - e, gain)) / (2 * h) - dx[i]) < 1e-6
    for i in range(dim):
        e = np.zeros(dim)
        e[i] = h
        assert abs((f(x, gain + e) - f(x, gain - e)) / (2 * h) - dg[i]) < 1e-6


def test_rotation_depends_on_the_difference_of_positions_only():
    r = rng(9)
    q, k = r.normal(size=(1, 1, 16)), r.normal(size=(1, 1, 16))
    dots = [(O.rotate(q, [p + 7], 16, 1e4, i) * O.rotate(k, [p], 16, 1e4, i)).sum() for i in (False, True) for p in (0, 11, 1000)]
    assert np.allclose(dots[:3], dots[0], atol=1e-12) and np.allclose(dots[3:], dots[3], atol=1e-12)


def test_stash8_blocks():
    r = rng(3)
    x = r.normal(size=(9, 75)) * np.exp(4 * r.normal(size=(9, 1)))
    x[2, :32] = 0
    x[3, 5] = np.inf
    x[4, 40] = np.nan
    back, codes, e = O.stash8(x)
    assert abs(codes).max() == 127 or abs(codes).max() >= 64
    fine = np.repeat(e != 128, 32, axis=1)[:, :75]
    step = np.ldexp(1.0, np.repeat(e, 32, axis=1)[:, :75])
    assert (abs(back - x)[fine] <= step[fine] / 2).all()
    assert np.isnan(back[3, :32]).all() and np.isnan(back[4, 32:64]).all() and np.isfinite(back[3, 32:]).all()
    assert not back[2, :32].any()
    again, _, _ = O.stash8(np.where(fine, back, 0.0))
    assert np.array_equal(again[fine], back[fine])
    for top, want in ((127.0, 0), (127.0000001, 1), (1.0, -6), (0.9921875, -7), (2.0 ** -140, -126)):
        assert O.stash8(np.full((1, 1), top))[2][0, 0] == want


def test_gelu_derivative_against_differences():
    z = np.linspace(-6, 6, 41)
    g = lambda v: v * O.gelu_parts(v)[0]
    h = 1e-6
    assert np.allclose((g(z + h) - g(z - h)) / (2 * h), sum(O.gelu_parts(z)), atol=1e-8)
