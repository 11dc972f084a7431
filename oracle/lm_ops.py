"""Plain definition (numpy, float64) of the single operators of language-model stages: token embedding, norm and
rotation of queries and keys, activations kept in 8 bits.  Every function also gives the sum of the absolute values that an
entry is added up from where a test's bound needs it."""
import numpy as np
from scipy.special import erfc

BLOCK = 32


# ---------------------------------------------------------------- embedding

def embedding_forward(ids, table, scale):
    y = np.zeros((len(ids), table.shape[1]))
    for t, i in enumerate(ids):
        if 0 <= i < len(table):
            y[t] = scale * table[i]
    return y


def embedding_backward(ids, dy, rows, scale):
    """(gradient, sum of |terms|, number of terms per row)."""
    g, a, n = np.zeros((rows, dy.shape[1])), np.zeros((rows, dy.shape[1])), np.zeros(rows)
    for t, i in enumerate(ids):
        if 0 <= i < rows:
            g[i] += scale * dy[t]
            a[i] += abs(scale * dy[t])
            n[i] += 1
    return g, a, n


# ---------------------------------------------------------------- norm and rotation of heads

def pairs(rotary, interleaved):
    i = np.arange(rotary // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)


def rotate(x, pos, rotary, theta, interleaved, back=False):
    """x [tokens, heads, dim] turned by the tokens' positions."""
    a, b = pairs(rotary, interleaved)
    ang = np.asarray(pos, np.longdouble)[:, None, None] * np.longdouble(theta) ** (-2 * np.arange(rotary // 2, dtype=np.longdouble) / max(rotary, 1))
    c, s = np.cos(ang).astype(np.float64), np.sin(ang).astype(np.float64) * (-1 if back else 1)
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def spread(x, rotary, interleaved):
    """|x_a| + |x_b| at both places of a pair, |x| elsewhere: what a rotated value is made of."""
    a, b = pairs(rotary, interleaved)
    y = abs(x)
    y[..., a] = y[..., b] = abs(x[..., a]) + abs(x[..., b])
    return y


def norm_rope_forward(x, gain, pos, rotary, theta, interleaved, eps):
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    u = x * r * gain
    return rotate(u, pos, rotary, theta, interleaved), spread(u, rotary, interleaved)


def norm_rope_backward(dy, x, gain, pos, rotary, theta, interleaved, eps):
    """(dx, dgain, bound of dx per unit of relative rounding, sum of |terms| of dgain)."""
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    du = rotate(dy, pos, rotary, theta, interleaved, back=True)
    da = spread(dy, rotary, interleaved)
    h, ha = du * gain, da * abs(gain)
    dx = r * (h - x * r * r * (h * x).mean(-1, keepdims=True))
    dxa = r * (ha + abs(x) * r * r * (ha * abs(x)).mean(-1, keepdims=True))
    return dx, (du * x * r).sum((0, 1)), dxa, (da * abs(x) * r).sum((0, 1))


# ---------------------------------------------------------------- 8-bit activations

def stash8(x):
    """(restored values, codes, exponents [rows, blocks])."""
    rows, cols = x.shape
    p = np.zeros((rows, -(-cols // BLOCK) * BLOCK))
    p[:, :cols] = x
    b = p.reshape(rows, -1, BLOCK)
    with np.errstate(invalid="ignore"):
        top = abs(b).max(-1)
    fine = np.isfinite(top)
    m, e = np.frexp(np.where(fine, top, 0.0) / 127.0)   # the least e with top / 127 <= 2^e
    e = np.where(m == 0.5, e - 1, e)
    e = np.clip(np.where(top > 0, e, -126), -126, 121)   # (2^122 times 64 would be no fp32 value)
    step = np.ldexp(1.0, e)[..., None]
    codes = np.where(fine[..., None], np.clip(np.rint(np.where(fine[..., None], b, 0.0) / step), -127, 127), 0.0)
    out = np.where(fine[..., None], codes * step, np.nan)
    return out.reshape(rows, -1)[:, :cols], codes, np.where(fine, e, 128)


def gelu_parts(z):
    """Phi(z) and |z| phi(z) (with its sign: the derivative is their sum)."""
    return 0.5 * erfc(-z / np.sqrt(2.0)), z * np.exp(-0.5 * z * z) / np.sqrt(2.0 * np.pi)
