"""The norm with the residual, the gated recurrence and the distillation loss (paper_2408_08015_amd.ops) against their definition
in 64 bits.

Bounds: u = 2^-24 is half a step of fp32.  A sum of n terms in any order is off by at most n u times the sum of the terms'
magnitudes, a rounding to bf16 by 2^-8 of the value; what an entry is added up from comes from the oracle."""
import numpy as np
import pytest
import torch

from oracle import lm_ops as O

pytestmark = pytest.mark.gpu

u = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
TINY = 1e-37   # results below fp32's smallest normal number may be cut to 0


@pytest.fixture(scope="module")
def ops():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2408_08015_amd import ops
    return ops


def rng(*seed):
    return np.random.Generator(np.random.PCG64(list(seed)))


def dev(a, dtype="f32"):
    """On the GPU in `dtype`, and the values it holds there in 64 bits."""
    t = torch.from_numpy(np.ascontiguousarray(a)).to("cuda")
    if t.is_floating_point():
        t = t.to(DT[dtype])
        return t, t.double().cpu().numpy()
    return t.to(torch.int32), a


def host(t):
    return t.double().cpu().numpy()


def inside(got, want, bound):
    """|got - want| <= bound, entry by entry; NaN where the definition has NaN and nowhere else."""
    got, bound = host(got), np.broadcast_to(bound, want.shape)
    assert got.shape == want.shape
    assert np.array_equal(np.isnan(got), np.isnan(want))
    with np.errstate(invalid="ignore"):
        bad = np.flatnonzero(~np.isnan(want) & ~((got == want) | (abs(got - want) <= bound)))
    assert bad.size == 0, (bad.size, bad[:5], got.ravel()[bad[:5]], want.ravel()[bad[:5]], bound.ravel()[bad[:5]])


def same(a, b):
    """Equal bits, NaN included."""
    return len(a) == len(b) and all((x is None) == (y is None) and (x is None or torch.equal(torch.nan_to_num(x, 7.0), torch.nan_to_num(y, 7.0))) for x, y in zip(a, b))


# ------------------------------------------------------------------------------------------------ norm and residual

NORM = [(1, 1), (3, 5), (2, 8), (7, 9), (1, 31), (5, 33), (130, 40), (65, 100), (257, 129), (40, 512), (33, 513), (300, 1000), (17, 1024), (9, 1025),
        (12, 1501), (50, 2048), (5, 2049), (21, 4096), (4, 4099), (6, 8192), (3, 8200), (4, 16384), (3, 16383), (3000, 24), (700, 7)]
TYPES = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")]


def norm_data(rows, width, dt, st, seed):
    r = rng(seed, rows, width)
    x, _ = dev(r.normal(size=(rows, width)), dt)
    res, _ = dev(r.normal(size=(rows, width)) * np.exp(r.normal(size=(1, width))) * np.exp(r.normal(size=(rows, 1))), st)
    gain, g = dev(1 + 0.3 * r.normal(size=width))
    return r, x, res, gain, g


@pytest.mark.parametrize("dt,st", TYPES)
@pytest.mark.parametrize("rows,width", NORM)
def test_rms_norm_forward(ops, rows, width, dt, st):
    _, x, res, gain, g = norm_data(rows, width, dt, st, 1)
    eps = float(np.float32(1e-5))
    x0, res0 = x.clone(), res.clone()
    y, s, kept = ops.rms_norm_forward(x, gain, residual=res, eps=1e-5, keep8=True)
    assert torch.equal(x, x0) and torch.equal(res, res0)
    total = host(x) + host(res)
    inside(s, total, abs(total) * (HALF[st] + u) * 1.001)
    # the sum of squares (width terms, halved by the root), the mean, the root and its argument, three products
    bound = lambda want: abs(want) * ((width / 2 + 8) * u * 1.01 + HALF[dt]) + TINY
    want = O.rms_norm_forward(host(s), g, eps)
    inside(y, want, bound(want))
    n = rows * ((width + 31) // 32) * 33
    assert torch.equal(kept.data[:n], ops.stash8_pack(y).data[:n])
    # Without keeping, and in place.  (Rows whose length is no multiple of eight are then read in the tensor's groups, and the squares
    # added up in that order: the bound is the same, the bits need not be.)
    y2, s2, none = ops.rms_norm_forward(x, gain, residual=res, eps=1e-5)
    assert none is None and torch.equal(s2, s) and (width % 8 or torch.equal(y2, y))
    inside(y2, want, bound(want))
    y3, s3, _ = ops.rms_norm_forward(x, gain, residual=res, eps=1e-5, out=x, sum_out=res)
    assert y3 is x and s3 is res and torch.equal(y3, y2) and torch.equal(s3, s)
    if dt == st:   # nothing added
        y4, s4, _ = ops.rms_norm_forward(s, gain, eps=1e-5)
        assert s4 is s and torch.equal(y4, y2)


@pytest.mark.parametrize("dt,st", TYPES)
@pytest.mark.parametrize("rows,width", NORM)
def test_rms_norm_backward(ops, rows, width, dt, st):
    r, _, s, gain, g = norm_data(rows, width, dt, st, 2)
    dy, d = dev(r.normal(size=(rows, width)), dt)
    dsum, dm = dev(r.normal(size=(rows, width)), st)
    eps = float(np.float32(1e-5))
    for more, m in ((dsum, dm), (None, 0.0)):
        dx, ds, dg = ops.rms_norm_backward(dy, s, gain, dsum=more, eps=1e-5)
        want, wg, wa, wga = O.rms_norm_backward(d, host(s), g, m, eps)
        # the two sums over a row (2 width), the norms and the products around them; the sum with dsum
        near = (wa * (2 * width + 24) * u + abs(m) * u) * 1.01 + TINY
        inside(dx, want, near + (abs(want) + near) * HALF[dt])
        inside(ds, want, near + (abs(want) + near) * HALF[st])
        assert (dx is ds) == (dt == st)
        inside(dg, wg, wga * (rows + width / 2 + 16) * u * 1.01 + TINY)
    old, o = dev(r.normal(size=width))
    again = ops.rms_norm_backward(dy, s, gain, eps=1e-5)
    assert same(again, (dx, ds, dg))
    s2, dy2 = s.clone(), dy.clone()
    if dt == st:
        acc = ops.rms_norm_backward(dy, s2, gain, eps=1e-5, out=s2, gain_out=old, accumulate=True)
    else:
        acc = ops.rms_norm_backward(dy2, s2, gain, eps=1e-5, out=dy2, sum_out=s2, gain_out=old, accumulate=True)
    assert torch.equal(acc[0], dx) and torch.equal(acc[1], ds) and acc[2] is old
    inside(old, o + wg, wga * (rows + width / 2 + 16) * u * 1.01 + u * 1.01 * (abs(o) + wga) + TINY)


@pytest.mark.parametrize("dt,st", TYPES)
def test_rms_norm_of_rows_that_are_zero_or_not_finite(ops, dt, st):
    width = 70
    x = torch.zeros(6, width, device="cuda", dtype=DT[dt])
    res = torch.zeros(6, width, device="cuda", dtype=DT[st])
    res[1, 33], res[2, 5], x[3, 7], res[4] = float("nan"), float("inf"), -float("inf"), 1.0
    gain = torch.ones(width, device="cuda")
    y, s, kept = ops.rms_norm_forward(x, gain, residual=res, keep8=True)
    assert not y[0].any() and not y[5].any() and torch.isfinite(y[4]).all()      # a row of zeros: 0, not NaN
    assert y[1].isnan().all()
    for row, at in ((2, 5), (3, 7)):   # the mean is infinite: 0, and NaN where the infinity is
        assert y[row].isnan().sum() == 1 and y[row, at].isnan() and torch.nan_to_num(y[row], 0.0).eq(0).all()
    back = ops.stash8_unpack(kept, torch.float32)
    assert back[1].isnan().all() and back[2, :32].isnan().all() and not back[2, 32:].any() and not back[0].any()
    dy = torch.ones_like(x)
    dx, ds, dg = ops.rms_norm_backward(dy, s, gain)
    assert torch.isfinite(dx[0]).all() and torch.isfinite(dx[4]).all() and dx[1].isnan().all() and dg[0].isnan()


def test_rms_norm_of_no_rows_and_unaligned_rows(ops):
    g = torch.ones(8, device="cuda")
    e = torch.zeros(0, 8, device="cuda")
    y, s, k = ops.rms_norm_forward(e, g, residual=e, keep8=True)
    assert y.shape == s.shape == (0, 8) and ops.stash8_unpack(k).shape == (0, 8)
    dx, _, dg = ops.rms_norm_backward(e, e, g)
    assert dx.shape == (0, 8) and not dg.any()
    one = torch.ones(8, device="cuda")
    assert ops.rms_norm_backward(e, e, g, gain_out=one, accumulate=True)[2].eq(1).all()
    for dt in DT.values():
        big = torch.randn(1 + 40 * 64, device="cuda").to(dt)
        a = big[1:].view(40, 64)
        gain = torch.rand(64, device="cuda")
        out, tot = (torch.empty_like(big)[1:].view(40, 64) for _ in range(2))
        got = ops.rms_norm_forward(a, gain, residual=a, out=out, sum_out=tot)
        want = ops.rms_norm_forward(a.clone(), gain, residual=a.clone())
        assert torch.equal(got[1], want[1]) and torch.equal(got[0], want[0])
        assert same(ops.rms_norm_backward(a, a, gain, dsum=a)[:2], ops.rms_norm_backward(a.clone(), a.clone(), gain, dsum=a.clone())[:2])


@pytest.mark.parametrize("dt,st", TYPES)
@pytest.mark.parametrize("rows,width,off", [(530, 8191, 0), (600, 9001, 0), (2100, 8200, 0), (300, 16384, 1), (290, 9001, 3), (270, 16383, 0)])
def test_rms_norm_of_long_rows(ops, rows, width, off, dt, st):
    """Several rows a block, in every way that rows are read."""
    _, x, res, gain, g = norm_data(rows, width, dt, st, 3)
    if off:
        x, res = (torch.cat([t.new_zeros(off), t.view(-1)])[off:].view(rows, width) for t in (x, res))
    eps = float(np.float32(1e-5))
    y, s, _ = ops.rms_norm_forward(x, gain, residual=res, eps=1e-5)
    total = host(x) + host(res)
    inside(s, total, abs(total) * (HALF[st] + u) * 1.001)
    want = O.rms_norm_forward(host(s), g, eps)
    inside(y, want, abs(want) * ((width / 2 + 8) * u * 1.01 + HALF[dt]) + TINY)
    dx, ds, dg = ops.rms_norm_backward(x, res, gain, dsum=s, eps=1e-5)
    m = host(s)
    want, wg, wa, wga = O.rms_norm_backward(host(x), host(res), g, m, eps)
    near = (wa * (2 * width + 24) * u + abs(m) * u) * 1.01 + TINY
    inside(dx, want, near + (abs(want) + near) * HALF[dt])
    inside(ds, want, near + (abs(want) + near) * HALF[st])
    inside(dg, wg, wga * (rows + width / 2 + 16) * u * 1.01 + TINY)
    assert same(ops.rms_norm_backward(x, res, gain, dsum=s, eps=1e-5), (dx, ds, dg))


# ------------------------------------------------------------------------------------------------ gated recurrence

def period(T, n):
    return dict(period=n), list(range(0, T, n)) + [T]


def ragged(r, T, n, tail=0, head=0):
    cut = np.sort(r.integers(head, T - tail + 1, n - 1))
    off = np.concatenate(([head], cut, [T - tail])).astype(np.int32)
    return dict(offsets=torch.from_numpy(off).cuda()), off.tolist()


REC = [  # tokens, channels, sequences
    (1, 1, ("period", 1)), (3, 2, ("period", 1)), (70, 64, ("period", 1)), (64, 33, ("period", 64)), (64, 128, ("period", 16)), (65, 130, ("period", 65)),
    (200, 7, ("period", 3)), (129, 129, ("period", 50)), (512, 40, ("period", 128)), (700, 65, ("period", 700)), (1000, 31, ("period", 333)),
    (2500, 96, ("period", 2500)), (5000, 3, ("period", 4097)), (1, 5, ("ragged", 1, 0, 0)), (40, 64, ("ragged", 30, 0, 0)), (300, 200, ("ragged", 5, 0, 0)),
    (300, 63, ("ragged", 7, 20, 9)), (1500, 66, ("ragged", 4, 0, 0)), (1500, 20, ("ragged", 200, 300, 130)), (4200, 48, ("ragged", 3, 1, 0)),
    (260, 16, ("ragged", 600, 0, 0)), (2304, 34, ("ragged", 2, 2000, 0)),
    (60, 65, ("ragged", 63, 3, 2)), (60, 33, ("ragged", 64, 5, 0)), (128, 40, ("ragged", 200, 10, 10)), (128, 9, ("ragged", 20, 0, 100)),
    (4200, 1000, ("period", 1)), (9, 5, ("ragged", 3, 4, 5)), (100, 200, ("ragged", 12, 0, 1)),
]


def rec_data(T, C, how, dt, gate, state, layout, seed):
    r = rng(seed, T, C, gate, state)
    kw, off = period(T, how[1]) if how[0] == "period" else ragged(r, T, *how[1:])
    p = r.normal(size=(T, 3, C))
    p[:, 0] = 2 * p[:, 0] + np.linspace(-3, 9, C)   # channels that forget at once and channels that keep
    if layout == "packed":
        t, v = dev(p, dt)
        parts = [t[:, i] for i in range(3)]
    else:
        parts, v = [dev(p[:, i], dt)[0] for i in range(3)], dev(p, dt)[1]
    h0 = dev(r.normal(size=(len(off) - 1, C))) if state else (None, None)
    if not gate:
        parts[2] = None
    return r, kw, off, parts, [v[:, 0], v[:, 1], v[:, 2] if gate else None], h0


def gate_steps(f, dt):
    # a gate: the exponent's rounding and that of its constant (2 |f| u; added behind the exponential in the fp32 form), exponential,
    # sum, reciprocal and product one to two steps each; a step of the recurrence: product and sum; joining: below
    return ((2 * abs(f) if dt == "bf16" else 0) + 16) * u


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("gate,state,layout", [(True, True, "packed"), (True, False, "apart"), (False, True, "apart"), (False, False, "packed")])
@pytest.mark.parametrize("T,C,how", REC)
def test_recurrence(ops, T, C, how, dt, gate, state, layout):
    r, kw, off, (f, z, o), (vf, vz, vo), (h0, v0) = rec_data(T, C, how, dt, gate, state, layout, 3)
    n = len(off) - 1
    live = np.zeros((T, 1), bool)
    live[off[0]:off[-1]] = True
    steps = gate_steps(vf, dt)
    w = O.recurrence_forward(vf, vz, vo, off, v0, steps)
    # maps of tokens, wavefronts, blocks and groups are joined on the way: at most 8 + 16 + 2 roundings at a place, and again behind
    # every group, where they fade with the state
    err = w["err"] + 64 * u * w["mag"]
    filled = torch.full((T, C), 3.0, device="cuda", dtype=DT[dt])
    y, final, saved = ops.recurrence_forward(f, z, o=o, state=h0, final=True, saved=True, out=filled, **kw)
    k = 0.0 if vo is None else gate_steps(vo, dt) + 4 * u
    sw = 1.0 if vo is None else abs(O.swish_parts(vo)[0])
    near = sw * err + abs(w["y"]) * k
    inside(y, np.where(live, w["y"], 3.0), np.where(live, (near + (abs(w["y"]) + near) * HALF[dt]) * 1.01 + TINY, 0.0))   # other rows stay
    last = np.array([max(off[i + 1] - 1, 0) for i in range(n)])
    some = np.array([off[i + 1] > off[i] for i in range(n)])[:, None]
    inside(final, w["final"], np.where(some, err[last] * 1.01 + TINY, 0.0))
    again = ops.recurrence_forward(f, z, o=o, state=h0, final=True, saved=True, **kw)
    assert torch.equal(again[0][live[:, 0]], y[live[:, 0]]) and torch.equal(again[1], final)
    if state:   # states in place
        moved = h0.clone()
        assert ops.recurrence_forward(f, z, o=o, state=moved, final=moved, **kw)[1] is moved and torch.equal(moved, final)

    dy, d = dev(r.normal(size=(T, C)), dt)
    dfin, df_ = dev(r.normal(size=(n, C))) if state else (None, None)
    b = O.recurrence_backward(d, vf, vz, vo, off, w, df_, steps + (0 if vo is None else gate_steps(vo, dt) + 4 * u))
    out = [torch.full((T, C), 3.0, device="cuda", dtype=DT[dt]) for _ in range(3 if gate else 2)]
    df, dz, do, dstate = ops.recurrence_backward(dy, f, z, saved, o=o, state=h0, dfinal=dfin, dstate=True, out=out, **kw)
    ga, gb = O.gates(vf)
    gerr = b["err"] + 64 * u * b["mag"]
    rounded = lambda want, e: np.where(live, (e + (abs(want) + e) * HALF[dt]) * 1.01 + TINY, 0.0)
    at = lambda want: np.where(live, want, 3.0)
    inside(dz, at(b["dz"]), rounded(b["dz"], gb * (gerr + b["mag"] * (steps + 2 * u))))
    hz = w["mag_before"] + abs(vz)
    herr = w["err_before"] + 64 * u * w["mag_before"] + u * hz
    inside(df, at(b["df"]), rounded(b["df"], ga * gb * (herr * (b["mag"] + gerr) + hz * (gerr + b["mag"] * (2 * steps + 4 * u)))))
    if gate:
        _, _, sa = O.swish_parts(vo)
        inside(do, at(b["do"]), rounded(b["do"], abs(d) * sa * (err + (w["mag"] + err) * (2 * gate_steps(vo, dt) + 6 * u))))
    first = np.array([min(off[i], T - 1) for i in range(n)])
    inside(dstate, b["dstate"], np.where(some, ga[first] * (gerr + b["mag"] * (steps + 2 * u))[first] * 1.01 + TINY, 0.0))
    # the same bits again; in place of the inputs, in the packed projection where they lie in one
    two = ops.recurrence_backward(dy, f, z, saved, o=o, state=h0, dfinal=dfin, dstate=True, **kw)
    rows = torch.from_numpy(live[:, 0]).cuda()
    assert all(p is None or torch.equal(p[rows], q[rows]) for p, q in zip(two[:3], (df, dz, do))) and torch.equal(two[3], dstate)
    if state:   # the states' gradients in place
        moved = dfin.clone()
        assert ops.recurrence_backward(dy, f, z, saved, o=o, state=h0, dfinal=moved, dstate=moved, **kw)[3] is moved and torch.equal(moved, dstate)
    three = ops.recurrence_backward(dy, f, z, saved, o=o, state=h0, dfinal=dfin, out=[t for t in (f, z, o) if t is not None], **kw)
    assert three[0] is f and all(p is None or torch.equal(p[rows], q[rows]) for p, q in zip(three[:3], (df, dz, do)))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_recurrence_token_by_token_and_in_segments(ops, dt):
    """A text at once, token by token and in segments, with the state carried on: within the bounds of each, the same values."""
    T, C, n = 150, 72, 5   # five texts of 150 tokens
    r, _, _, (f, z, o), (vf, vz, vo), _ = rec_data(n * T, C, ("period", T), dt, True, False, "apart", 4)
    off = list(range(0, n * T + 1, T))
    w = O.recurrence_forward(vf, vz, vo, off, None, gate_steps(vf, dt))
    err = w["err"] + 64 * u * w["mag"]
    near = abs(O.swish_parts(vo)[0]) * err + abs(w["y"]) * (gate_steps(vo, dt) + 4 * u)
    bound = (near + (abs(w["y"]) + near) * HALF[dt]) * 1.01 + TINY
    rows = lambda t, a, b: t.view(n, T, C)[:, a:b].reshape(-1, C)
    for step in (1, 40):
        state = torch.zeros(n, C, device="cuda")
        got = []
        for a in range(0, T, step):
            b = min(a + step, T)
            y, state, _ = ops.recurrence_forward(rows(f, a, b), rows(z, a, b), o=rows(o, a, b), period=b - a, state=state, final=state)
            got.append(y.view(n, b - a, C))
        inside(torch.cat(got, 1).view(n * T, C), w["y"], bound)
        inside(state, w["final"], err[np.array(off[1:]) - 1] * 1.01 + TINY)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("how", ["period", "ragged"])
def test_recurrence_keeps_what_is_not_finite_in_its_sequence(ops, dt, how):
    """NaN and infinities in one sequence, in its state, its gates and its gradients: the others' results do not change by a bit."""
    T, C, n = 1400, 70, 7
    g = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    f, z, o, dy = (rnd(T, C).to(DT[dt]) for _ in range(4))
    h0, dfin = rnd(n, C), rnd(n, C)
    off = [0, 200, 400, 400, 611, 993, 1397, 1400] if how == "ragged" else list(range(0, T + 1, 200))
    kw = dict(offsets=torch.tensor(off, dtype=torch.int32, device="cuda")) if how == "ragged" else dict(period=200)

    def both():
        y, fin, saved = ops.recurrence_forward(f, z, o=o, state=h0, final=True, saved=True, **kw)
        return (y, fin) + ops.recurrence_backward(dy, f, z, saved, o=o, state=h0, dfinal=dfin, dstate=True, **kw)
    clean = both()
    assert all(torch.isfinite(t).all() for t in clean)
    s = 4 if how == "ragged" else 3
    a, b = off[s], off[s + 1]
    f[a + 3, 5], f[a + 70, 6], z[a + 1, 7], o[b - 1, 8], dy[b - 2, 9] = [float("nan")] * 5
    z[a + 100, 10], h0[s, 11], dfin[s, 12] = float("inf"), -float("inf"), float("nan")
    f[a + 9, 13], f[a + 10, 14] = float("inf"), -float("inf")   # gates of exactly 1 and 0
    f[b - 1, 15], f[a, 16] = float("nan"), float("nan")
    got = both()
    others = torch.ones(T, dtype=torch.bool, device="cuda")
    others[a:b] = False
    which = torch.ones(n, dtype=torch.bool, device="cuda")
    which[s] = False
    for p, q in zip(got, clean):
        keep = others if p.shape[0] == T else which
        assert torch.equal(p[keep], q[keep])
    assert got[0][a + 2, 5].isfinite() and got[0][a + 3:b, 5].isnan().all() and got[1][s, 5].isnan()
    assert got[0][a:b, 13].isfinite().all() and got[0][a:b, 14].isfinite().all()
    assert torch.isnan(got[2][a:b - 1, 12]).any() and torch.isnan(got[5][s, 12])


def test_recurrence_forgets_and_keeps_at_the_ends_of_the_gate(ops):
    """f = -inf: the state is the candidate; f = +inf: it stays as it is, over any number of blocks."""
    T, C = 5000, 5
    z = torch.randn(T, C, device="cuda")
    h0 = torch.randn(1, C, device="cuda")
    f = torch.full((T, C), float("inf"), device="cuda")
    y, fin, saved = ops.recurrence_forward(f, z, period=T, state=h0, final=True, saved=True)
    assert torch.equal(y, h0.expand(T, C)) and torch.equal(fin, h0)
    dy = torch.ones(T, C, device="cuda")
    df, dz, _, ds = ops.recurrence_backward(dy, f, z, saved, period=T, state=h0, dstate=True)
    assert not df.any() and not dz.any() and torch.equal(ds, torch.full_like(ds, T))
    y, fin, saved = ops.recurrence_forward(-f, z, period=T, state=h0, final=True, saved=True)
    assert torch.equal(y, z) and torch.equal(fin[0], z[-1])
    df, dz, _, ds = ops.recurrence_backward(dy, -f, z, saved, period=T, state=h0, dstate=True)
    assert not df.any() and torch.equal(dz, dy) and not ds.any()


def test_recurrence_of_no_tokens_and_broadcast_rows(ops):
    e = torch.zeros(0, 6, device="cuda")
    h0 = torch.randn(3, 6, device="cuda")
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    y, fin, saved = ops.recurrence_forward(e, e, offsets=off, state=h0, final=True, saved=True)
    assert y.shape == (0, 6) and torch.equal(fin, h0) and saved.shape == (0, 6)
    df, dz, do, ds = ops.recurrence_backward(e, e, e, saved, offsets=off, state=h0, dfinal=h0, dstate=True)
    assert df.shape == (0, 6) and do is None and torch.equal(ds, h0)
    assert not ops.recurrence_forward(e, e, offsets=off, final=True)[1].any()
    assert ops.recurrence_forward(e, e, period=4, final=True)[1].shape == (0, 6)
    x = torch.randn(90, 6, device="cuda")
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full((90, 6), 2.0, device="cuda")
    assert ops.recurrence_forward(x, x, offsets=none, out=out)[0].eq(2).all()      # no sequences at all: nothing is written
    f = torch.randn(1, 6, device="cuda").expand(500, 6)      # one row for all tokens
    z = torch.randn(500, 6, device="cuda")
    for a, b in zip(ops.recurrence_forward(f, z, period=500, saved=True), ops.recurrence_forward(f.contiguous(), z, period=500, saved=True)):
        assert a is b is None or torch.equal(a, b)


def test_recurrence_rows_of_odd_strides_and_addresses(ops):
    for dt in DT.values():
        g = torch.Generator(device="cuda").manual_seed(6)
        T, C = 333, 67
        big = torch.randn(1 + T * 211, generator=g, device="cuda").to(dt)
        rows = big[1:].view(T, 211)
        f, z, o = rows[:, :C], rows[:, C:2 * C], rows[:, 140:140 + C]
        a = ops.recurrence_forward(f, z, o=o, period=111, final=True, saved=True)
        c = [t.clone() for t in (f, z, o)]
        b = ops.recurrence_forward(c[0], c[1], o=c[2], period=111, final=True, saved=True)
        assert same(a, b)
        dy = torch.randn(T, 70, generator=g, device="cuda").to(dt)[:, 1:C + 1]
        want = ops.recurrence_backward(dy.clone(), *c[:2], b[2], o=c[2], period=111, dstate=True)
        left = rows.clone()
        got = ops.recurrence_backward(dy, f, z, a[2], o=o, period=111, dstate=True, out=(f, z, o))
        assert same(got, want)
        for lo, hi in ((2 * C, 140), (140 + C, 211)):        # what lies between the parts stays
            assert torch.equal(rows[:, lo:hi], left[:, lo:hi])


# ------------------------------------------------------------------------------------------------ distillation

DISTILL = [  # rows, vocab, entries, temperature, label weight, room behind a row
    (1, 1, 1, 1.0, 0.0, 0), (2, 7, 3, 2.0, 0.5, 0), (3, 8, 8, 0.5, 0.0, 3), (5, 33, 40, 1.0, 0.3, 0), (9, 100, 1, 3.0, 1.0, 0), (4, 511, 17, 1.5, 0.0, 1),
    (6, 512, 64, 2.0, 0.1, 0), (3, 4096, 65, 1.0, 0.0, 0), (2, 4097, 200, 4.0, 0.5, 7), (2, 30011, 1024, 0.7, 0.2, 5), (3, 65536, 128, 1.0, 0.5, 0), (2, 131072, 64, 2.0, 0.5, 0),
    (2, 131077, 9, 2.0, 0.5, 3), (2, 250001, 50, 1.0, 0.0, 7), (40, 16391, 33, 4.0, 0.4, 0),
    # (rows of a wavefront each, with as many entries as those take and one more; and rows that are just too long)
    (11, 1999, 256, 1.5, 0.3, 1), (11, 1999, 257, 1.0, 0.0, 1), (7, 2049, 256, 2.0, 0.5, 0), (6, 4096, 255, 4.0, 0.2, 0), (300, 130, 20, 1.0, 0.4, 6),
    # (more rows than are cut into slices: kept in registers whole, or the first part of them)
    (80, 9001, 8, 1.0, 0.0, 0), (65, 20000, 30, 4.0, 0.5, 1), (70, 33000, 12, 1.5, 0.2, 0), (66, 131077, 40, 2.0, 0.5, 3),
    # (a part of the rows in shared memory, less and a little more than fits there; fp32, then bf16)
    (65, 36001, 11, 2.0, 0.5, 0), (65, 45007, 30, 1.5, 0.2, 0), (65, 53256, 16, 1.0, 0.0, 0),
    (66, 69633, 30, 4.0, 0.5, 0), (65, 98313, 16, 1.5, 0.2, 0), (65, 106505, 9, 2.0, 0.3, 2),
]


def distill_data(T, V, K, mix, room, dt, tt, seed):
    r = rng(seed, T, V, K)
    base = torch.zeros(T, V + room, device="cuda", dtype=DT[dt])
    z = base[:, :V]
    z.copy_(torch.from_numpy(3 * r.normal(size=(T, V))))
    t, tv = dev(3 * r.normal(size=(T, K)), tt)
    ids = r.integers(-2, V + 2, (T, K))
    ids[:, : K // 3] = r.integers(0, min(V, 5), (T, K // 3))   # places that stand several times
    if T > 2:
        ids[1] = -1                                            # no entry that counts
    if T > 3:
        tv[3, :] = -np.inf
        t[3] = -float("inf")
    labels = r.integers(0, V, T)
    labels[0] = max(int(ids[0, 0]), 0)
    if T > 4:
        labels[2], labels[4] = -1, V
    w = r.normal(size=T).astype(np.float32)
    if T > 1:
        w[-1] = 0.0
    return r, base, z, host(z), ids, t, tv, (labels if mix else None), w


def distill_bounds(want, z, t, ids, tau, labels, mix, w, dt):
    """(bounds of loss, dz) from the oracle's parts."""
    T, V = z.shape
    K = ids.shape[1]
    top = z.max(1, keepdims=True)
    far, far1 = (top - z) / tau, top - z
    sums = V / 256 + 64          # a thread's own values with their rescalings, then the block's
    eq, e1 = 4 * far + 6, 4 * far1 + 6
    rq = (eq + (want["q"] * eq).sum(1, keepdims=True) + sums) * u      # a softmax value: its exponential, and the sum's
    r1 = (e1 + (want["q1"] * e1).sum(1, keepdims=True) + sums) * u
    tf = np.where(np.isfinite(t), abs(t - np.where(np.isfinite(t), t, -1e30).max(1, keepdims=True)), 0.0) / tau
    rp = (2 * (4 * tf + 8) + K) * u
    loss, dz = np.zeros(T), np.zeros((T, V))
    for r in range(T):
        k = np.flatnonzero((ids[r] >= 0) & (ids[r] < V))
        p, lq = want["p"][r, k], want["logq"][r, ids[r, k]]
        loss[r] = (1 - mix) * tau * tau * (p * ((abs(want["logp"][r, k]) + abs(lq)) * (rp[r, k] + (K + 12) * u) + rp[r, k] +
                                                rq[r].max() + (far[r, ids[r, k]] + abs(np.log(V)) + 12) * 4 * u)).sum()
        np.add.at(dz[r], ids[r, k], (1 - mix) * tau * p * (rp[r, k] + K * u))
        if labels is not None and 0 <= labels[r] < V:
            loss[r] += mix * (r1[r].max() + (far1[r, labels[r]] + np.log(V) + 12) * 4 * u)
            dz[r, labels[r]] += 4 * mix * u
    rate, m = (1 - mix) * tau, (mix if labels is not None else 0.0)
    dz += rate * want["q"] * (rq + 6 * u) + m * want["q1"] * (r1 + 6 * u)
    dz = (dz + 4 * u * (rate * want["q"] + m * want["q1"])) * abs(w[:, None]) + abs(want["dz"]) * 8 * u
    return loss * 1.01 + TINY, (dz + (abs(want["dz"]) + dz) * HALF[dt]) * 1.01 + TINY


@pytest.mark.parametrize("dt,tt", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("T,V,K,tau,mix,room", DISTILL)
def test_distill(ops, T, V, K, tau, mix, room, dt, tt):
    r, base, z, v, ids, t, tv, labels, w = distill_data(T, V, K, mix, room, dt, tt, 7)
    tau32, mix32 = float(np.float32(tau)), float(np.float32(mix))
    want = O.distill(v, ids, tv, tau32, labels, mix32, w.astype(np.float64))
    bl, bz = distill_bounds(want, v, tv, ids, tau32, labels, mix32, w, dt)
    wd, idd = dev(w)[0], dev(ids)[0]
    kw = dict(temperature=tau, labels=None if labels is None else dev(labels)[0], label_weight=mix)
    loss, stats = ops.distill_forward(z, idd, t, **kw)
    inside(loss, want["loss"], bl)
    top = v.max(1)
    assert np.array_equal(host(stats)[:, 0], top)
    for col, at, on in ((1, tau32, True), (2, 1.0, labels is not None)):
        e = np.exp((v - top[:, None]) / at)
        s = e.sum(1)
        inside(stats[:, col], s if on else np.zeros(T), (e * (4 * (top[:, None] - v) / at + 6)).sum(1) * u + s * (V / 256 + 64) * u)
    dz = ops.distill_backward(wd, z, idd, t, stats, **kw)
    inside(dz, want["dz"], bz)
    assert not dz[host(wd) == 0].any()
    loss2, dz2 = ops.distill_step(wd, z, idd, t, **kw)
    inside(loss2, want["loss"], bl)
    inside(dz2, want["dz"], bz)
    assert same(ops.distill_step(wd, z, idd, t, **kw), (loss2, dz2)) and same(ops.distill_forward(z, idd, t, **kw), (loss, stats))
    # in place, what lies behind the rows stays; and into rows of another stride
    if room:
        base[:, V:] = 5.0
    wide = torch.full((T, V + 9), 4.0, device="cuda", dtype=DT[dt])
    assert torch.equal(ops.distill_step(wd, z, idd, t, out=wide[:, :V], **kw)[1], dz2) and wide[:, V:].eq(4).all()
    keep = z.clone()
    got = ops.distill_step(wd, z, idd, t, out=z, **kw)
    assert got[1] is z and torch.equal(z, dz2) and torch.equal(got[0], loss2) and base[:, V:].eq(5).all()
    z.copy_(keep)
    ops.distill_backward(wd, z, idd, t, stats, out=z, **kw)
    assert torch.equal(z, dz) and base[:, V:].eq(5).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_distill_of_logits_at_the_ends_of_the_range(ops, dt):
    """Masked logits (-inf and the type's lowest value), large ones, NaN in rows that do not count."""
    V = 600
    low = torch.finfo(DT[dt]).min
    z = torch.randn(8, V, device="cuda").to(DT[dt])
    z[0, 100:] = -float("inf")
    z[1, 100:] = low
    z[2] = low
    z[3] += 5000.0
    z[4, 7] = float("nan")
    z[5, 7] = float("inf")
    z[6] = -float("inf")
    z[7] = float("nan")
    ids = torch.tensor([[1, 50, 99]], dtype=torch.int32, device="cuda").repeat(8, 1)
    t = torch.tensor([[3.0, low, -float("inf")]], device="cuda").repeat(8, 1)
    w = torch.ones(8, device="cuda")
    w[7] = 0.0
    labels = torch.zeros(8, dtype=torch.int32, device="cuda")
    for tau in (1.0, 2.0):
        v = host(z)
        want = O.distill(v, ids.cpu().numpy(), host(t), tau, labels.cpu().numpy(), 0.5, host(w))
        loss, dz = ops.distill_step(w, z, ids, t, temperature=tau, labels=labels, label_weight=0.5)
        back = ops.distill_backward(w, z, ids, t, ops.distill_forward(z, ids, t, temperature=tau, labels=labels, label_weight=0.5)[1],
                                    temperature=tau, labels=labels, label_weight=0.5)
        for g in (dz, back):
            got = host(g)
            assert np.array_equal(np.isnan(got), np.isnan(want["dz"]))
            fine = [0, 1, 2, 3, 7]
            assert np.allclose(got[fine], want["dz"][fine], rtol=2e-2 if dt == "bf16" else 1e-4, atol=1e-6)
            assert not got[7].any()
        assert np.allclose(host(loss)[[0, 1, 3]], want["loss"][[0, 1, 3]], rtol=1e-5)
        assert np.isnan(host(loss)[[4, 5, 6, 7]]).all()


def test_distill_of_a_gradient_that_only_the_entries_have(ops):
    """Softmax values times dloss that round to 0: the entries' places still get dloss (q - p), here -dloss."""
    z = torch.zeros(1, 64, device="cuda")
    ids, t = torch.tensor([[5]], dtype=torch.int32, device="cuda"), torch.zeros(1, 1, device="cuda")
    w = torch.full((1,), 2e-37, device="cuda")
    dz = ops.distill_backward(w, z, ids, t, torch.tensor([[0.0, 2.0 ** 30, 0.0]], device="cuda"))   # (the sum of 2^30 equal logits)
    assert dz[0, 5] == -w[0] and dz.abs().sum() == w[0]


def test_distill_of_no_rows(ops):
    e = torch.zeros(0, 40, device="cuda")
    ids, t, w = torch.zeros(0, 3, dtype=torch.int32, device="cuda"), torch.zeros(0, 3, device="cuda"), torch.zeros(0, device="cuda")
    loss, stats = ops.distill_forward(e, ids, t)
    assert loss.shape == (0,) and stats.shape == (0, 3)
    assert ops.distill_backward(w, e, ids, t, stats).shape == (0, 40) and ops.distill_step(w, e, ids, t)[1].shape == (0, 40)


def test_distill_of_more_rows_than_a_launch_takes(ops):
    """The rows behind the 2^22nd are a launch of their own."""
    g = torch.Generator(device="cuda").manual_seed(12)
    T, V = (1 << 22) + 37, 9
    z = torch.randn(T, V, generator=g, device="cuda")
    ids = torch.randint(-1, V, (T, 3), generator=g, device="cuda", dtype=torch.int32)
    t, w = torch.randn(T, 3, generator=g, device="cuda"), torch.rand(T, generator=g, device="cuda")
    loss, dz = ops.distill_step(w, z, ids, t)
    stats = ops.distill_forward(z, ids, t)[1]
    for a, b in ((0, 50), ((1 << 22) - 20, T)):
        s = slice(a, b)
        want = ops.distill_step(w[s], z[s].clone(), ids[s], t[s])
        assert torch.equal(loss[s], want[0]) and torch.equal(dz[s], want[1])
    # two ways to the same gradient, |dloss| <= 1 and softmax values at most 1: each is off by at most the exponential (4 (|z - max|) + 6,
    # here below 60), its sum and the teacher's p (64 and 2 x (4 x 12 + 8) + 3) in steps of u
    assert (ops.distill_backward(w, z, ids, t, stats) - dz).abs().max() <= 2 * (60 + 64 + 115) * u and bool(loss.isfinite().all())


# ------------------------------------------------------------------------------------------------ together

def stage(ops, D, V, K, g):
    """A recurrent stage and its loss: lookup, norm (kept in 8 bits), projection, recurrence, projection, norm with the residual,
    logits, distillation; and back.  Products are plain ones of torch in fp32.  Returns (inputs, step)."""
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    T = 420
    p = dict(ids=torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32), table=0.5 * rnd(V, D), g1=1 + 0.1 * rnd(D), g2=1 + 0.1 * rnd(D),
             win=rnd(3 * D, D) / D ** 0.5, wout=rnd(D, D) / D ** 0.5, head=rnd(V, D) / D ** 0.5,
             off=torch.tensor([0, 100, 100, 333, T], dtype=torch.int32, device="cuda"), state=rnd(4, D),
             tid=torch.randint(0, V, (T, K), generator=g, device="cuda", dtype=torch.int32), t=rnd(T, K), w=torch.rand(T, generator=g, device="cuda") / T,
             lab=torch.randint(-1, V, (T,), generator=g, device="cuda", dtype=torch.int32))

    def step():
        x = ops.embedding_forward(p["ids"], p["table"])
        n1, s1, _ = ops.rms_norm_forward(x, p["g1"])
        proj = n1 @ p["win"].t()
        f, z, o = proj[:, :D], proj[:, D:2 * D], proj[:, 2 * D:]
        # (rows of no sequence are not written)
        y, fin, saved = ops.recurrence_forward(f, z, o=o, offsets=p["off"], state=p["state"], final=True, saved=True, out=torch.zeros_like(x))
        n2, s2, kept = ops.rms_norm_forward(y @ p["wout"].t(), p["g2"], residual=s1, keep8=True)
        logits = n2 @ p["head"].t()
        loss, dl = ops.distill_step(p["w"], logits, p["tid"], p["t"], temperature=2.0, labels=p["lab"], label_weight=0.3, out=logits)
        dhead, _ = ops.linear_wgrad_stash8(dl.bfloat16(), kept, bias=False)
        dm, _, dg2 = ops.rms_norm_backward(dl @ p["head"], s2, p["g2"])
        dwout = dm.t() @ y
        dproj = torch.zeros_like(proj)
        _, _, _, dstate = ops.recurrence_backward(dm @ p["wout"], f, z, saved, o=o, offsets=p["off"], state=p["state"], dfinal=fin, dstate=True,
                                                  out=(dproj[:, :D], dproj[:, D:2 * D], dproj[:, 2 * D:]))
        dwin = dproj.t() @ n1
        dx, _, dg1 = ops.rms_norm_backward(dproj @ p["win"], s1, p["g1"], dsum=dm)
        return loss, fin, ops.embedding_backward(p["ids"], dx, V), dg1, dwin, dstate, dwout, dg2, dhead
    return p, step


def test_a_recurrent_stage_against_autograd(ops):
    """The run of operators as a stage uses them, against torch's automatic differentiation in 64 bits on the CPU."""
    D, V, K = 48, 200, 9
    p, step = stage(ops, D, V, K, torch.Generator(device="cuda").manual_seed(8))
    loss, fin, dtable, dg1, dwin, dstate, dwout, dg2, dhead = step()
    c = {k: v.cpu() for k, v in p.items()}
    leaf = {k: c[k].double().requires_grad_() for k in ("table", "g1", "win", "state", "wout", "g2", "head")}
    rms = lambda s, g: s / torch.sqrt((s * s).mean(-1, keepdim=True) + 1e-6) * g
    x = leaf["table"][c["ids"].long()]
    f, z, o = (rms(x, leaf["g1"]) @ leaf["win"].t()).split(D, 1)
    a, ys, ends = torch.sigmoid(f), [], []
    off = c["off"].tolist()
    for s in range(4):
        h = leaf["state"][s]
        for t in range(off[s], off[s + 1]):
            h = a[t] * h + (1 - a[t]) * z[t]
            ys.append(h)
        ends.append(h)
    y = torch.stack(ys) * o * torch.sigmoid(o)
    logits = rms(y @ leaf["wout"].t() + x, leaf["g2"]) @ leaf["head"].t()
    q, q1 = torch.log_softmax(logits / 2, 1), torch.log_softmax(logits, 1)
    lp = torch.log_softmax(c["t"].double() / 2, 1)
    L = 0.7 * 4 * (lp.exp() * (lp - q.gather(1, c["tid"].long()))).sum(1)
    lab = c["lab"].long()
    L = L - 0.3 * torch.where(lab >= 0, q1.gather(1, lab.clamp(min=0)[:, None])[:, 0], 0.0)
    final = torch.stack(ends)
    ((L * c["w"].double()).sum() + (final * fin.cpu().double()).sum()).backward()
    rel = lambda g, w: ((g.cpu().double() - w).norm() / w.norm()).item()
    # fp32 chains of products of up to 200 terms: a few 1e-6; the head's gradient is formed from bf16 dy (2^-9 rms and less) and
    # inputs in 8 bits (uniform steps of up to 1/127 of a block's largest value, at most four sizes of a normal value: 0.9 %)
    assert rel(loss, L.detach()) < 1e-5 and rel(fin, final.detach()) < 1e-5
    for got, name in ((dtable, "table"), (dg1, "g1"), (dwin, "win"), (dstate, "state"), (dwout, "wout"), (dg2, "g2")):
        assert rel(got, leaf[name].grad) < 5e-5, name
    assert rel(dhead, leaf["head"].grad) < 2e-2


def test_operators_on_another_stream_and_in_replayed_graphs(ops):
    """The run on a stream of the caller's, and captured into two graphs that are replayed in turn with eager work and new inputs
    in between: equal bits everywhere."""
    D, V, K = 130, 300, 7
    g = torch.Generator(device="cuda").manual_seed(9)
    p, step = stage(ops, D, V, K, g)
    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert same(want, got)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            res = step()
        graphs.append((graph, res))
    for n in range(4):
        p["ids"].copy_(torch.randint(0, V, p["ids"].shape, generator=g, device="cuda", dtype=torch.int32))
        p["state"].copy_(torch.randn(4, D, generator=g, device="cuda"))
        p["off"].copy_(torch.tensor([0, 10 + 50 * n, 300, 300, 420 - n], dtype=torch.int32))
        for graph, res in graphs:
            graph.replay()
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        for _, res in graphs:
            assert same(res, want), n


def test_in_place_and_with_a_workspace_of_the_callers(ops):
    """Outputs on every input that the interface allows, and a workspace that is larger than needed, full of other calls' words and
    taken by several of them: the bits of outputs of their own."""
    g = torch.Generator(device="cuda").manual_seed(13)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
    ws = torch.full((1 << 22,), 0xAB, dtype=torch.uint8, device="cuda")
    for rows, width in ((70, 1000), (41, 1501), (37, 5000)):
        x, r, dsum, gain = rnd(rows, width), rnd(rows, width), rnd(rows, width), torch.rand(width, generator=g, device="cuda")
        y, s, _ = ops.rms_norm_forward(x, gain, residual=r)
        for into in ("x", "r"):
            a, b = x.clone(), r.clone()
            got = ops.rms_norm_forward(a, gain, residual=b, **(dict(out=b, sum_out=a) if into == "x" else dict(out=a, sum_out=b)))
            assert torch.equal(got[0], y) and torch.equal(got[1], s)
        want = ops.rms_norm_backward(x, s, gain, dsum=dsum)
        for n in range(3):
            three = [x.clone(), s.clone(), dsum.clone()]
            got = ops.rms_norm_backward(three[0], three[1], gain, dsum=three[2], out=three[n], workspace=ws)
            assert got[0] is three[n] and same(got, want)
        s32, d32 = s.float(), dsum.float()
        want = ops.rms_norm_backward(x, s32, gain, dsum=d32)
        for n in range(2):
            two = [s32.clone(), d32.clone()]
            got = ops.rms_norm_backward(x, two[0], gain, dsum=two[1], sum_out=two[n], workspace=ws)
            assert got[1] is two[n] and same(got, want)
    for T, C, kw in ((1700, 130, dict(period=1700)), (300, 66, dict(period=100)), (129, 31, dict(period=1)),
                     (900, 65, dict(offsets=torch.tensor([0, 5, 400, 400, 900], dtype=torch.int32, device="cuda")))):
        n = 4 if "offsets" in kw else -(-T // kw["period"])
        data, dy = [rnd(T, C) for _ in range(3)], rnd(T, C)
        h0 = torch.randn(n, C, generator=g, device="cuda")
        f, z, o = data
        want = ops.recurrence_forward(f, z, o=o, state=h0, final=True, saved=True, **kw)
        for k in range(3):
            d = [t.clone() for t in data]
            got = ops.recurrence_forward(d[0], d[1], o=d[2], state=h0, final=True, saved=True, out=d[k], workspace=ws, **kw)
            assert got[0] is d[k] and same(got, want)
        back = ops.recurrence_backward(dy, f, z, want[2], o=o, state=h0, dfinal=want[1], dstate=True, **kw)
        for k in range(3):
            d, e = [t.clone() for t in data], dy.clone()
            out = d[:k] + [e] + d[k + 1:]        # one of the gradients in place of dy, the others of their inputs
            assert same(ops.recurrence_backward(e, d[0], d[1], want[2], o=d[2], state=h0, dfinal=want[1], dstate=True, out=out, workspace=ws, **kw), back)
    z, ids = 2 * rnd(5, 40000), torch.randint(0, 40000, (5, 9), generator=g, device="cuda", dtype=torch.int32)
    t, w = torch.randn(5, 9, generator=g, device="cuda"), torch.rand(5, generator=g, device="cuda")
    want = ops.distill_step(w, z, ids, t)
    got = ops.distill_step(w, z, ids, t, out=z, workspace=ws)
    assert got[1] is z and same(got, want)


def test_two_recurrences_at_once(ops):
    """Two long chains on two streams, a workspace each: both end, with the bits of each alone."""
    g = torch.Generator(device="cuda").manual_seed(10)
    T, C = 40000, 640
    data = [[torch.randn(T, C, generator=g, device="cuda").bfloat16() for _ in range(4)] for _ in range(2)]

    def run(f, z, o, dy):
        y, fin, saved = ops.recurrence_forward(f, z, o=o, period=T, final=True, saved=True)
        return (y, fin) + ops.recurrence_backward(dy, f, z, saved, o=o, period=T)[:3]
    want = [run(*d) for d in data]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for s, d in zip(streams, data):
        with torch.cuda.stream(s):
            got.append(run(*d))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert same(a, b)


# ------------------------------------------------------------------------------------------------ more than 2^31 values

def test_rows_behind_2_to_the_31st_value(ops):
    """Rows at the end of tensors of more than 2^31 values: the bits of the same rows in a small tensor."""
    g = torch.Generator(device="cuda").manual_seed(11)
    rows, width = (1 << 31) // 4096 + 600, 4096
    x = torch.zeros(rows, width, device="cuda", dtype=torch.bfloat16)
    end = torch.randn(500, width, generator=g, device="cuda").bfloat16()
    x[-500:] = end
    gain = torch.rand(width, generator=g, device="cuda")
    y, s, kept = ops.rms_norm_forward(x, gain, residual=x, keep8=True)
    y0, s0, k0 = ops.rms_norm_forward(end, gain, residual=end, keep8=True)
    assert torch.equal(y[-500:], y0) and torch.equal(s[-500:], s0)
    assert torch.equal(kept.data[rows * width - 500 * width: rows * width], k0.data[:500 * width])
    dx = ops.rms_norm_backward(y, s, gain, dsum=s, out=y)[0]
    assert torch.equal(dx[-500:], ops.rms_norm_backward(y0, s0, gain, dsum=s0)[0])
    del y, s, kept, dx
    T = rows // 128 * 128
    f = x[:T]
    state = torch.ones(T // 128, width, device="cuda")
    y, fin, saved = ops.recurrence_forward(f, f, period=128, state=state, final=True, saved=True)
    y0, fin0, saved0 = ops.recurrence_forward(f[-512:].clone(), f[-512:].clone(), period=128, state=state[:4], final=True, saved=True)
    assert torch.equal(y[-512:], y0) and torch.equal(fin[-4:], fin0)
    df, dz = ops.recurrence_backward(y, f, f, saved, period=128, state=state, out=(y, torch.empty_like(f)))[:2]
    want = ops.recurrence_backward(y0, f[-512:].clone(), f[-512:].clone(), saved0, period=128, state=state[:4])
    assert torch.equal(df[-512:], want[0]) and torch.equal(dz[-512:], want[1])
    del y, fin, saved, df, dz
    z = x.view(-1)[: (1 << 31) + 3 * 100003].view(-1)[: ((1 << 31) // 100003 + 2) * 100003].view(-1, 100003)
    z[-2:] = 3 * torch.randn(2, 100003, generator=g, device="cuda").bfloat16()
    n = z.shape[0]
    ids = torch.randint(0, 100003, (n, 6), generator=g, device="cuda", dtype=torch.int32)
    t, w = torch.randn(n, 6, generator=g, device="cuda"), torch.ones(n, device="cuda")
    small = ops.distill_step(w[-2:], z[-2:].clone(), ids[-2:], t[-2:])
    loss, dz = ops.distill_step(w, z, ids, t, out=z)
    assert torch.equal(loss[-2:], small[0]) and torch.equal(dz[-2:], small[1])
