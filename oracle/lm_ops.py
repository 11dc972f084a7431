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


# ---------------------------------------------------------------- RMS norm between two blocks

def rms_norm_forward(s, gain, eps):
    return s / np.sqrt((s * s).mean(-1, keepdims=True) + eps) * gain


def rms_norm_backward(dy, s, gain, dsum, eps):
    """(ds, dgain, bound of ds without dsum per unit of relative rounding, sum of |terms| of dgain)."""
    r = 1.0 / np.sqrt((s * s).mean(-1, keepdims=True) + eps)
    h = dy * gain
    ds = r * (h - s * r * r * (h * s).mean(-1, keepdims=True)) + dsum
    dsa = r * (abs(h) + abs(s) * r * r * (abs(h) * abs(s)).mean(-1, keepdims=True))
    return ds, (dy * s * r).sum(0), dsa, (abs(dy) * abs(s) * r).sum(0)


# ---------------------------------------------------------------- gated linear recurrence

def sigmoid(x):
    return 0.5 * (1.0 + np.tanh(0.5 * x))


def gates(f):
    """sigmoid(f) and 1 - sigmoid(f), each to its own relative precision."""
    e = np.exp(-abs(f))
    big, small = 1.0 / (1.0 + e), e / (1.0 + e)
    return np.where(f >= 0, big, small), np.where(f >= 0, small, big)


def swish_parts(o):
    """swish, its derivative, and the sum of the derivative's |terms|."""
    s, n = gates(o)
    return o * s, s + o * s * n, s + abs(o) * s * n


def recurrence_forward(f, z, o, offsets, state, step=0.0):
    """Over sequences [offsets[s], offsets[s + 1]) of rows.  Dict of y, h, final; and, where every gate is off by `step[t, c]`
    relative and every operation by `step` too: mag (the sum of |terms| of h), err (how far h may be off)."""
    T, C = f.shape
    a, b = gates(f)
    out = {k: np.zeros((T, C)) for k in ("h", "before", "mag", "mag_before", "err", "err_before")}
    n = len(offsets) - 1
    final = np.zeros((n, C)) if state is None else np.array(state, np.float64)
    final_err = np.zeros((n, C))
    step = np.broadcast_to(step, (T, C))
    for s in range(n):
        h, m, e = final[s].copy(), abs(final[s]), np.zeros(C)
        for t in range(offsets[s], offsets[s + 1]):
            out["before"][t], out["mag_before"][t], out["err_before"][t] = h, m, e
            e = a[t] * e + step[t] * (a[t] * m + b[t] * abs(z[t]))
            h = a[t] * h + b[t] * z[t]
            m = a[t] * m + b[t] * abs(z[t])
            out["h"][t], out["mag"][t], out["err"][t] = h, m, e
        final[s], final_err[s] = h, e
    sw = 1.0 if o is None else swish_parts(o)[0]
    out.update(y=out["h"] * sw, final=final, final_err=final_err)
    return out


def recurrence_backward(dy, f, z, o, offsets, fwd, dfinal, step=0.0):
    """fwd: what recurrence_forward gave.  Dict of df, dz, do, dstate; G, its magnitude and error as above."""
    T, C = f.shape
    a, b = gates(f)
    sw, slope, _ = (1.0, 0.0, 0.0) if o is None else swish_parts(o)
    d = dy * sw
    G, mag, err = np.zeros((T, C)), np.zeros((T, C)), np.zeros((T, C))
    n = len(offsets) - 1
    dstate = np.zeros((n, C)) if dfinal is None else np.array(dfinal, np.float64)
    dstate_err = np.zeros((n, C))
    step = np.broadcast_to(step, (T, C))
    for s in range(n):
        k, m, e = dstate[s].copy(), abs(dstate[s]), np.zeros(C)
        for t in range(offsets[s + 1] - 1, offsets[s] - 1, -1):
            G[t], mag[t], err[t] = d[t] + k, abs(d[t]) + m, e + step[t] * (abs(d[t]) + m)
            k, m, e = a[t] * G[t], a[t] * mag[t], a[t] * (err[t] + step[t] * mag[t])
        dstate[s], dstate_err[s] = k, e
    return dict(df=a * b * (fwd["before"] - z) * G, dz=b * G, do=dy * fwd["h"] * slope, dstate=dstate, dstate_err=dstate_err,
                G=G, mag=mag, err=err)


# ---------------------------------------------------------------- distillation from a teacher's top logits

def distill(z, ids, t, tau, labels, mix, dloss):
    """Of every row: dict of loss, dz; q, q1 (softmax at tau and at 1), p (of every entry), logp, logq, logq1."""
    T, V = z.shape
    with np.errstate(all="ignore"):
        lse = lambda x: np.log(np.exp(x).sum(-1, keepdims=True))   # (of values that are at most 0: a shift is taken off before)
        down = lambda x: x - x.max(-1, keepdims=True)
        logq, logq1 = down(z) / tau - lse(down(z) / tau), down(z) - lse(down(z))
        q, q1 = np.exp(logq), np.exp(logq1)
        loss, dz, p, logp = np.zeros(T), np.zeros((T, V)), np.zeros(ids.shape), np.zeros(ids.shape)
        for r in range(T):
            k = np.flatnonzero((ids[r] >= 0) & (ids[r] < V) & ~(t[r] == -np.inf))
            if len(k) and mix != 1.0:
                x = down(t[r, k]) / tau
                logp[r, k] = x - lse(x)
                p[r, k] = np.exp(logp[r, k])
                on = k[p[r, k] != 0]
                loss[r] += (1 - mix) * tau * tau * (p[r, on] * (logp[r, on] - logq[r, ids[r, on]])).sum()
                dz[r] += (1 - mix) * tau * q[r]
                np.add.at(dz[r], ids[r, k], -(1 - mix) * tau * p[r, k])
            if labels is not None and mix != 0.0 and 0 <= labels[r] < V:
                loss[r] -= mix * logq1[r, labels[r]]
                dz[r] += mix * q1[r]
                dz[r, labels[r]] -= mix
            dz[r] = dz[r] * dloss[r] if dloss[r] != 0 else 0.0
    return dict(loss=loss, dz=dz, q=q, q1=q1, p=p, logp=logp, logq=logq, logq1=logq1)
