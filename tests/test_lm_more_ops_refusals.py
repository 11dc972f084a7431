"""CPU: what the norm with the residual, the gated recurrence and the distillation loss refuse, before anything is launched."""
import ctypes as C

import pytest
import torch

import paper_2408_08015_amd as A
from paper_2408_08015_amd import ops

EINVAL = -1
P = 1 << 20           # addresses that are never read: the calls below are refused
FAR = [P + (i << 24) for i in range(16)]
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    A.load_library()
    return ops._lib()


def refused(lib, name, *args):
    st = getattr(lib, "asteroid_" + name)(*args)
    msg = lib.asteroid_last_error().decode()
    assert st == EINVAL and name in msg, (name, args, st, msg)
    return msg


def each(ok, bad):
    for at, values in bad.items():
        for v in values:
            yield [v if i == at else a for i, a in enumerate(ok)]


def norm(**kw):
    c = dict(rows=8, width=40, dtype=1, sum_dtype=0, eps=1e-6)
    c.update(kw)
    return ops.ast_norm_cfg(*[c[n] for n, _ in ops.ast_norm_cfg._fields_])


BAD_NORM = [None] + [norm(**k) for k in (dict(rows=-1), dict(rows=1 << 31), dict(width=0), dict(width=16385), dict(dtype=2), dict(sum_dtype=3),
                                         dict(dtype=0, sum_dtype=1), dict(eps=0.0), dict(eps=1e-40), dict(eps=NAN), dict(eps=INF), dict(eps=-1.0))]


def test_rms_norm_refusals(lib):
    x, r, g, y, s, k = FAR[:6]
    ok = [norm(), x, r, g, y, s, k, None]
    for a in each(ok, {0: BAD_NORM, 1: [None, x + 1], 2: [None, r + 2], 3: [None, g + 2], 4: [None, y + 1], 5: [None, s + 2], 6: [k + 8]}):
        refused(lib, "rms_norm_forward", *a)
    refused(lib, "rms_norm_forward", norm(), x, None, g, y, None, None, None)          # an fp32 sum of bf16 rows alone
    for a in each(ok, {4: [s, s + 8 * 40 * 4 - 2, s - 8 * 40 * 2 + 2, k], 5: [k, k + 4]}):
        assert "overlap" in refused(lib, "rms_norm_forward", *a)
    assert lib.asteroid_rms_norm_forward(norm(rows=0), None, None, None, None, None, None, None) == 0
    n = C.c_size_t()
    for c in BAD_NORM:
        refused(lib, "rms_norm_backward_workspace", c, C.byref(n))
    refused(lib, "rms_norm_backward_workspace", norm(), None)
    assert lib.asteroid_rms_norm_backward_workspace(norm(), C.byref(n)) == 0 and n.value > 0
    dy, s, g, ds0, dx, ds, dg, ws = FAR[:8]
    ok = [norm(), dy, s, g, ds0, dx, ds, dg, 0, ws, n.value, None]
    for a in each(ok, {0: BAD_NORM, 1: [None, dy + 1], 2: [None, s + 2], 3: [None, g + 2], 4: [ds0 + 2], 5: [dx + 1], 6: [ds + 2], 7: [None, dg + 2],
                       9: [None, ws + 8], 10: [n.value - 1]}):
        refused(lib, "rms_norm_backward", *a)
    refused(lib, "rms_norm_backward", norm(), dy, s, g, ds0, None, None, dg, 0, ws, n.value, None)
    for a in each(ok, {5: [ds, ds + 8 * 40 * 4 - 2, dg], 7: [dx, ds + 4]}):
        assert "overlap" in refused(lib, "rms_norm_backward", *a)


def rows(dev=P, stride=40):
    return ops.ast_rows(dev, stride)


def rec(**kw):
    c = dict(tokens=300, channels=40, dtype=1, offsets_dev=P, sequences=3, period=0)
    c.update(kw)
    return ops.ast_recurrence_cfg(*[c[n] for n, _ in ops.ast_recurrence_cfg._fields_])


BAD_REC = [None] + [rec(**k) for k in (dict(tokens=-1), dict(tokens=1 << 31), dict(channels=0), dict(channels=(1 << 20) + 1), dict(dtype=2),
                                       dict(tokens=1 << 30, channels=17), dict(tokens=(1 << 28) + 1, channels=64), dict(offsets_dev=P + 2), dict(sequences=-1),
                                       dict(sequences=(1 << 31) - 1), dict(offsets_dev=None), dict(offsets_dev=None, period=-1),
                                       dict(offsets_dev=None, period=1 << 31))]
BAD_ROWS = [None, rows(None), rows(P + 1), rows(stride=-1), rows(stride=(1 << 40) + 1)]


def test_recurrence_refusals(lib):
    n = C.c_size_t()
    for c in BAD_REC:
        refused(lib, "recurrence_workspace", c, C.byref(n))
    refused(lib, "recurrence_workspace", rec(), None)
    assert lib.asteroid_recurrence_workspace(rec(), C.byref(n)) == 0 and n.value > 300 * 4
    f, z, o, st, y, fin, sav, ws, dy, df, dz, do, dst = FAR[:13]
    R = rows
    ok = [rec(), R(f), R(z), R(o), st, y, fin, sav, ws, n.value, None]
    bad = [r for r in BAD_ROWS if r is not None]
    for a in each(ok, {0: BAD_REC, 1: BAD_ROWS, 2: BAD_ROWS, 3: bad, 4: [st + 2], 5: [None, y + 1], 6: [fin + 2], 7: [sav + 2], 8: [None, ws + 8],
                       9: [n.value - 1]}):
        refused(lib, "recurrence_forward", *a)
    for a in each(ok, {6: [y, y + 300 * 40 * 2 - 4, sav, sav + 4], 7: [y + 4, fin + 3 * 40 * 4 - 4]}):
        assert "overlap" in refused(lib, "recurrence_forward", *a)
    ok = [rec(), R(dy), R(f), R(z), R(o), st, sav, fin, R(df), R(dz), R(do), dst, ws, n.value, None]
    short = [R(df, 39), R(df, 0)]
    for a in each(ok, {0: BAD_REC, 1: BAD_ROWS, 2: BAD_ROWS, 3: BAD_ROWS, 4: BAD_ROWS, 5: [st + 2], 6: [None, sav + 2], 7: [fin + 2],
                       8: BAD_ROWS + short, 9: BAD_ROWS + short, 10: BAD_ROWS + short, 11: [dst + 2], 12: [None, ws + 8], 13: [n.value - 1]}):
        refused(lib, "recurrence_backward", *a)
    # gradients in one packed tensor lie side by side; on each other they are refused
    packed = [R(df + 80 * i, 120) for i in range(3)]
    for a, b in ((0, 2 * 39), (0, -2 * 39), (120 * 2, 2), (0, 0)):
        m = [packed[0], R(df + a + b, 120), packed[2]]
        assert "overlap" in refused(lib, "recurrence_backward", *(ok[:8] + m + ok[11:]))
    assert "overlap" in refused(lib, "recurrence_backward", *(ok[:8] + [packed[0], packed[1], R(df + 80, 240)] + ok[11:]))
    assert "overlap" in refused(lib, "recurrence_backward", *(ok[:8] + [packed[0], packed[1], packed[1]] + ok[11:]))


def test_recurrence_workspace_is_none_where_sequences_begin_with_every_block(lib):
    n = C.c_size_t()
    for tokens, period, some in ((4096, 64, False), (4096, 1, False), (60, 60, False), (4096, 4096, True), (4096, 48, True)):
        assert lib.asteroid_recurrence_workspace(rec(tokens=tokens, offsets_dev=None, period=period), C.byref(n)) == 0
        assert (n.value > 0) == some, (tokens, period, n.value)
    assert lib.asteroid_recurrence_workspace(rec(tokens=0), C.byref(n)) == 0 and n.value == 0


def dist(**kw):
    c = dict(rows=4, vocab=50, logits_stride=64, dtype=1, entries=7, teacher_dtype=0, temperature=2.0, label_weight=0.5, labels_dev=P)
    c.update(kw)
    return ops.ast_distill_cfg(*[c[n] for n, _ in ops.ast_distill_cfg._fields_])


BAD_DIST = [None] + [dist(**k) for k in (dict(rows=-1), dict(rows=1 << 31), dict(vocab=0), dict(vocab=(1 << 30) + 1, logits_stride=1 << 31),
                                         dict(logits_stride=49), dict(logits_stride=(1 << 31) + 1), dict(dtype=2), dict(entries=0), dict(entries=1025),
                                         dict(teacher_dtype=5), dict(temperature=0.0), dict(temperature=1e-30), dict(temperature=1e20), dict(temperature=-1.0), dict(temperature=NAN),
                                         dict(temperature=INF), dict(label_weight=-0.1), dict(label_weight=1.1), dict(label_weight=NAN),
                                         dict(labels_dev=None), dict(labels_dev=P + 1))]


def test_distill_refusals(lib):
    z, ids, t, loss, st, w, dz, ws = FAR[:8]
    n = C.c_size_t()
    for c in BAD_DIST:
        refused(lib, "distill_step_workspace", c, C.byref(n))
    refused(lib, "distill_step_workspace", dist(), None)
    assert lib.asteroid_distill_step_workspace(dist(), C.byref(n)) == 0 and n.value == 0
    few = dist(vocab=40000, logits_stride=40000)      # few long rows are cut into slices
    assert lib.asteroid_distill_step_workspace(few, C.byref(n)) == 0 and n.value > 0
    ok = [dist(), z, ids, t, loss, st, None]
    for a in each(ok, {0: BAD_DIST, 1: [None, z + 1], 2: [None, ids + 2], 3: [None, t + 2], 4: [None, loss + 2, st, st + 44], 5: [None, st + 2]}):
        refused(lib, "distill_forward", *a)
    for a in each([few, w, z, ids, t, loss, dz, 40000, ws, n.value, None], {8: [None, ws + 8], 9: [n.value - 1]}):
        refused(lib, "distill_step", *a)
    ok = [dist(), w, z, ids, t, st, dz, 50, None]
    for a in each(ok, {0: BAD_DIST, 1: [None, w + 2], 2: [None, z + 1], 3: [None, ids + 2], 4: [None, t + 2], 5: [None, st + 2], 6: [None, dz + 1, z],
                       7: [49, (1 << 31) + 1]}):
        refused(lib, "distill_backward", *a)
    ok = [dist(), w, z, ids, t, loss, dz, 50, None, 0, None]
    for a in each(ok, {0: BAD_DIST, 1: [None, w + 2], 2: [None, z + 1], 3: [None, ids + 2], 4: [None, t + 2], 5: [None, loss + 2, dz, dz + 64],
                       6: [None, dz + 1, z], 7: [49, (1 << 31) + 1]}):
        refused(lib, "distill_step", *a)
    c = dist(rows=0)
    assert lib.asteroid_distill_forward(c, None, None, None, None, None, None) == 0
    assert lib.asteroid_distill_backward(c, None, None, None, None, None, None, 0, None) == 0
    assert lib.asteroid_distill_step(c, None, None, None, None, None, None, 0, None, 0, None) == 0


def test_tensors_are_checked():
    f, i, h = torch.zeros, torch.int32, torch.bfloat16
    g = f(8)
    with pytest.raises(ValueError, match="GPU"):
        ops.rms_norm_forward(f(3, 8), g)
    for args, kw, what in (((f(8), g), {}, "matrix"), ((f(3, 8), f(7)), {}, "shape"), ((f(3, 8, dtype=torch.float16), g), {}, "float32 or"),
                           ((f(3, 8), g), dict(residual=f(3, 7)), "shape"), ((f(3, 8), g), dict(residual=f(3, 8, dtype=h)), "must be a tensor of"),
                           ((f(8, 3).t(), g), {}, "contiguous"), ((f(3, 8), g), dict(sum_out=f(3, 8)), "no sum"),
                           ((f(3, 8, dtype=h), g), dict(residual=f(3, 8), sum_out=f(3, 8, dtype=h)), "sum_out"),
                           ((f(3, 8), g), dict(out=f(3, 8, dtype=h)), "out"), ((f(3, 8), g), dict(kept_out=f(3)), "Stash8"),
                           ((f(3, 8), g), dict(kept_out=ops.Stash8(4, 8, "cpu")), "keeps")):
        with pytest.raises(ValueError, match=what):
            ops.rms_norm_forward(*args, **kw)
    for args, kw, what in (((f(3, 8), f(3, 8, dtype=h), g), {}, "s must"), ((f(3, 8), f(3, 7), g), {}, "shape"), ((f(3, 8), f(3, 8), g), dict(accumulate=True), "accumulate"),
                           ((f(3, 8), f(3, 8), g), dict(dsum=f(3, 8, dtype=h)), "dsum"), ((f(3, 8), f(3, 8), g), dict(out=f(3, 8), sum_out=f(3, 8)), "one tensor"),
                           ((f(3, 8), f(3, 8), g), dict(gain_out=f(9)), "gain_out"), ((f(3, 8), f(3, 8), g), {}, "GPU")):
        with pytest.raises(ValueError, match=what):
            ops.rms_norm_backward(*args, **kw)
    a = f(5, 8)
    for args, kw, what in (((a, a), {}, "period"), ((a, a), dict(period=0), "period"), ((a, a), dict(period=(1 << 32) + 1), "period"), ((a, f(5, 7)), dict(period=5), "z must"),
                           ((a, a), dict(period=5, o=f(5, 8, dtype=h)), "o must"), ((f(8, 5).t(), a), dict(period=5), "unit stride"),
                           ((a, a), dict(offsets=f(3)), "offsets"), ((a, a), dict(offsets=f(0, dtype=i)), "one number more"),
                           ((a, a), dict(period=2, state=f(2, 8)), "state"), ((a, a), dict(period=5, final=f(1, 8, dtype=h)), "final"),
                           ((a, a), dict(period=5, saved=f(2, 8)), "saved"), ((a, a), dict(period=5, out=f(5, 9)), "out"), ((a, a), dict(period=5), "GPU")):
        with pytest.raises(ValueError, match=what):
            ops.recurrence_forward(*args, **kw)
    s = f(1, 8)
    for args, kw, what in (((a, a, a, f(2, 8)), dict(period=5), "saved"), ((f(4, 8), a, a, s), dict(period=5), "dy must"), ((a, a, a, s), dict(period=5, out=(a, a, a)), "gradient of o"),
                           ((a, a, a, s), dict(period=5, o=a, out=(a, a)), "gradient of o"), ((a, a, a, s), dict(period=5, dstate=f(2, 8)), "dstate"),
                           ((a, a, a, s), dict(period=5, out=(a, f(8, 5).t())), "unit stride")):
        with pytest.raises(ValueError, match=what):
            ops.recurrence_backward(*args, **kw)
    z, ids, t = f(4, 50), f(4, 7, dtype=i), f(4, 7)
    for args, kw, what in (((f(50), ids, t), {}, "logits"), ((z, f(4, 7), t), {}, "ids"), ((z, f(3, 7, dtype=i), t), {}, "shape"), ((z, ids, f(4, 6)), {}, "teacher"),
                           ((z, ids, t), dict(labels=f(4)), "labels"), ((z, ids, t), dict(labels=f(3, dtype=i)), "labels"), ((f(50, 4).t(), ids, t), {}, "unit stride"),
                           ((z, ids, t), dict(out=f(5)), "out"), ((z, ids, t), dict(stats_out=f(4, 2)), "stats_out"), ((z, ids, t), {}, "GPU")):
        with pytest.raises(ValueError, match=what):
            ops.distill_forward(*args, **kw)
    with pytest.raises(ValueError, match="dloss"):
        ops.distill_step(f(3), z, ids, t)
    with pytest.raises(ValueError, match="out"):
        ops.distill_step(f(4), z, ids, t, out=f(4, 50, dtype=h))
    with pytest.raises(ValueError, match="stats"):
        ops.distill_backward(f(4), z, ids, t, f(4, 2))


def test_states_that_are_read_are_tensors():
    """True asks for a tensor to be made; that is for results only."""
    a, s = torch.zeros(5, 8), torch.zeros(1, 8)
    with pytest.raises(ValueError, match="state must be a tensor"):
        ops.recurrence_forward(a, a, period=5, state=True)
    for kw in (dict(state=True), dict(dfinal=True)):
        with pytest.raises(ValueError, match="must be a tensor"):
            ops.recurrence_backward(a, a, a, s, period=5, **kw)
