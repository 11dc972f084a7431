"""CPU: tensors of one call of the norm with the residual, the gated recurrence and the distillation loss that lie on each other
are refused, before anything is launched, except where the interface allows it; and numbers that it has no room for."""
import ctypes as C

import pytest
import torch

import paper_2408_08015_amd as A
from paper_2408_08015_amd import ops

EINVAL = -1
FAR = [(1 << 40) + (i << 32) for i in range(16)]   # addresses that are never read: every call below is refused


@pytest.fixture(scope="module")
def lib():
    A.load_library()
    return ops._lib()


def refused(lib, name, *args):
    st = getattr(lib, "asteroid_" + name)(*args)
    msg = lib.asteroid_last_error().decode()
    assert st == EINVAL and name in msg, (name, args, st, msg)
    return msg


# ------------------------------------------------------------------------------------------------ recurrence

R = ops.ast_rows


def rec(tokens=300, channels=40, dtype=1, offsets=FAR[15], sequences=3, period=0):
    return ops.ast_recurrence_cfg(tokens, channels, dtype, offsets, sequences, period)


def recurrence_backward(lib, cfg, **at):
    """The message of the refused call; what `at` does not give lies apart.  (Without its workspace it would be refused last.)"""
    c = cfg.channels
    a = {n: R(FAR[i], c) for i, n in enumerate(("dy", "f", "z", "o", "df", "dz", "do"))}
    a.update(state=FAR[7], saved=FAR[8], dfinal=FAR[9], dstate=FAR[10], ws=None, size=0)
    a.update(at)
    return refused(lib, "recurrence_backward", cfg, a["dy"], a["f"], a["z"], a["o"], a["state"], a["saved"], a["dfinal"], a["df"], a["dz"], a["do"],
                   a["dstate"], a["ws"], a["size"], None)


def test_gradients_of_the_recurrence_whose_extent_passes_64_bits(lib):
    """The rows of dz begin at df's second row; (tokens - 1) * stride * 2 bytes is 2^64."""
    big = rec(tokens=(1 << 23) + 1)
    for other in ("dz", "do"):
        assert "outputs overlap" in recurrence_backward(lib, big, df=R(FAR[4], 1 << 40), **{other: R(FAR[4] + (2 << 40), 1 << 40)})


def test_gradients_of_the_recurrence_beside_each_other(lib):
    """Parts of one packed tensor, and rows behind another's last one, are no overlap; one value on another is."""
    e, c, T = 2, 40, 300
    p = FAR[4]
    for dz, fine in ((R(p + 80 * e, 120), True), (R(p + 39 * e, 120), False), (R(p - 40 * e, 120), True), (R(p - 39 * e, 120), False),
                     (R(p + T * 120 * e, 120), True), (R(p + (T - 1) * 120 * e, 120), False), (R(p + ((T - 1) * 120 + 40) * e, 120), True),
                     (R(p - T * 120 * e, 120), True), (R(p - (T - 1) * 120 * e, 120), False), (R(p - (T * 120 - 81) * e, 120), False),
                     (R(p + ((T - 1) * 120 + 40) * e, 40), True), (R(p + ((T - 1) * 120 + 39) * e, 40), False)):
        assert ("workspace" if fine else "outputs overlap") in recurrence_backward(lib, rec(tokens=T, channels=c), df=R(p, 120), dz=dz), (dz.dev - p, dz.stride)


def test_gradients_of_the_recurrence_on_other_tensors(lib):
    """Blocks read the inputs, states and offsets of their own tokens while others write: only the same rows may be shared."""
    e, c, T, n = 2, 40, 300, 3
    packed = {k: R(FAR[1] + i * c * e, 3 * c) for i, k in enumerate(("f", "z", "o"))}
    need = C.c_size_t()
    assert lib.asteroid_recurrence_workspace(rec(), need) == 0 and need.value > 0
    ok = [{}, dict(df=R(FAR[1], c), dz=R(FAR[2], c), do=R(FAR[3], c)), dict(df=R(FAR[0], c)), dict(df=R(FAR[2], c), dz=R(FAR[1], c)),
          dict(packed, df=packed["f"], dz=packed["z"], do=packed["o"]), dict(packed, df=packed["o"]), dict(packed, df=R(FAR[1] + T * 3 * c * e, 3 * c)),
          dict(dstate=FAR[9]), dict(dstate=FAR[7]), dict(dstate=FAR[9] + n * c * 4), dict(state=None, dfinal=None, dstate=None)]
    for a in ok:
        assert "workspace is missing" in recurrence_backward(lib, rec(), **a), a
    for a in (dict(dstate=FAR[4]), dict(dstate=FAR[5] + T * c * e - 4), dict(dstate=FAR[6] - n * c * 4 + 4)):
        assert "outputs overlap" in recurrence_backward(lib, rec(), **a), a
    for a in (dict(dstate=FAR[0]), dict(dstate=FAR[1]), dict(dstate=FAR[2]), dict(dstate=FAR[3] + T * c * e - 4), dict(dstate=FAR[8]), dict(dstate=FAR[9] + 4),
              dict(dstate=FAR[9] + c * 4), dict(dstate=FAR[7] - c * 4), dict(dstate=FAR[15]), dict(dstate=FAR[15] + 4 * n),
              dict(df=R(FAR[0] + e, c)), dict(dz=R(FAR[1] + c * e, c)), dict(do=R(FAR[3] + e, c)), dict(df=R(FAR[1], c + 1)), dict(f=R(FAR[4], 0)),
              dict(packed, df=R(FAR[1] + e, 3 * c)), dict(packed, df=R(FAR[1] + 3 * c * e, 3 * c)), dict(packed, df=R(FAR[1], c)),
              dict(df=R(FAR[7], c)), dict(dz=R(FAR[8], c)), dict(do=R(FAR[9], c)), dict(df=R(FAR[15], c))):
        assert "an output and an input" in recurrence_backward(lib, rec(), **a), a
    for at in range(11):
        a = dict(ws=FAR[at], size=need.value)
        assert "workspace overlaps" in recurrence_backward(lib, rec(), **a), at


def recurrence_forward(lib, cfg, **at):
    c = cfg.channels
    a = {n: R(FAR[i], c) for i, n in enumerate(("f", "z", "o"))}
    a.update(state=FAR[3], y=FAR[4], final=FAR[5], saved=FAR[6], ws=None, size=0)
    a.update(at)
    return refused(lib, "recurrence_forward", cfg, a["f"], a["z"], a["o"], a["state"], a["y"], a["final"], a["saved"], a["ws"], a["size"], None)


def test_results_of_the_recurrence_on_other_tensors(lib):
    e, c, T, n = 2, 40, 300, 3
    need = C.c_size_t()
    assert lib.asteroid_recurrence_workspace(rec(), need) == 0 and need.value > 0
    wide = R(FAR[0], 3 * c)
    for a in ({}, dict(y=FAR[0]), dict(y=FAR[2]), dict(final=FAR[3]), dict(final=FAR[3] + n * c * 4), dict(state=None, final=None, saved=None, o=None),
              dict(f=wide, z=R(FAR[0] + c * e, 3 * c), y=FAR[0] + T * 3 * c * e)):
        assert "workspace is missing" in recurrence_forward(lib, rec(), **a), a
    for a in (dict(y=FAR[0] + e), dict(y=FAR[1] - T * c * e + e), dict(f=wide, y=FAR[0]), dict(f=R(FAR[0], 0), y=FAR[0]), dict(f=wide, y=FAR[0] + (T - 1) * 3 * c * e),
              dict(y=FAR[3]), dict(y=FAR[15]), dict(final=FAR[3] + 4), dict(final=FAR[3] + c * 4), dict(final=FAR[1]), dict(final=FAR[15]),
              dict(saved=FAR[0]), dict(saved=FAR[1]), dict(saved=FAR[2] + T * c * e - 4), dict(saved=FAR[3]), dict(saved=FAR[15] + 4 * n)):
        assert "an output and an input" in recurrence_forward(lib, rec(), **a), a
    # of no tokens, states are passed on
    assert "an output and an input" in recurrence_forward(lib, rec(tokens=0), final=FAR[3] + 4)
    for at in range(7):
        assert "workspace overlaps" in recurrence_forward(lib, rec(), ws=FAR[at], size=need.value), at


# ------------------------------------------------------------------------------------------------ distillation

def dist(rows=4, vocab=40000, stride=40000, dtype=1, entries=7, teacher=0, labels=FAR[15]):
    return ops.ast_distill_cfg(rows, vocab, stride, dtype, entries, teacher, 2.0, 0.5 if labels else 0.0, labels)


def distill_step(lib, cfg, **at):
    a = dict(dloss=FAR[0], z=FAR[1], ids=FAR[2], t=FAR[3], loss=FAR[4], dz=FAR[5], stride=cfg.logits_stride, ws=None, size=0)
    a.update(at)
    return refused(lib, "distill_step", cfg, a["dloss"], a["z"], a["ids"], a["t"], a["loss"], a["dz"], a["stride"], a["ws"], a["size"], None)


def test_gradient_of_the_logits_on_other_tensors(lib):
    """Few rows are cut into slices, whose blocks read logits while others write: only the same rows may be shared."""
    e, T, V = 2, 4, 40000
    side = dict(cfg=dist(stride=2 * V), dz=FAR[1] + V * e)        # the gradient beside the logits in the same rows
    for a in ({}, dict(dz=FAR[1]), side, dict(side, dz=FAR[1] - V * e), dict(dz=FAR[1] + T * V * e), dict(cfg=dist(labels=None))):
        a = dict(dict(cfg=dist()), **a)
        assert "workspace is missing" in distill_step(lib, **a), a
    on = [dict(dz=FAR[1] + e), dict(dz=FAR[1] - e), dict(dz=FAR[1] + V * e), dict(side, dz=FAR[1] + (V - 1) * e), dict(dz=FAR[1] + 2 * e, stride=V + 8),
          dict(dz=FAR[0]), dict(dz=FAR[2]), dict(dz=FAR[3] + 4 * 7 * T - e), dict(dz=FAR[15]), dict(dz=FAR[15] - T * V * e + e)]
    for a in on:
        a = dict(dict(cfg=dist()), **a)
        assert "an output and an input" in distill_step(lib, **a), a
        cfg, dz, stride = a["cfg"], a["dz"], a.get("stride", a["cfg"].logits_stride)
        assert "an output and an input" in refused(lib, "distill_backward", cfg, FAR[0], FAR[1], FAR[2], FAR[3], FAR[6], dz, stride, None), a
    assert "an output and an input" in refused(lib, "distill_backward", dist(), FAR[0], FAR[1], FAR[2], FAR[3], FAR[6], FAR[6] + 12 * T - e, V, None)
    assert "an output and an input" in distill_step(lib, dist(rows=(1 << 31) - 1, vocab=1 << 30, stride=1 << 31, dtype=0), dz=FAR[1] + 4, stride=1 << 31)


def test_loss_on_other_tensors(lib):
    """One that lies on dloss, for instance: of a row in slices, the first writes it while others still read dloss."""
    e, T, V = 2, 4, 40000
    need = C.c_size_t()
    assert lib.asteroid_distill_step_workspace(dist(), need) == 0 and need.value > 0
    assert "workspace is missing" in distill_step(lib, dist(), loss=FAR[0] + 4 * T)
    for a in (FAR[0], FAR[0] + 4, FAR[0] - 4 * T + 4, FAR[1], FAR[1] + T * V * e - 4, FAR[2], FAR[3] + 4 * 7 * T - 4, FAR[15]):
        assert "an output and an input" in distill_step(lib, dist(), loss=a), a - FAR[0]
        if a not in (FAR[0], FAR[0] + 4, FAR[0] - 4 * T + 4):
            for loss, stats in ((a, FAR[6]), (FAR[6], a)):
                assert "an output and an input" in refused(lib, "distill_forward", dist(), FAR[1], FAR[2], FAR[3], loss, stats, None), a - FAR[0]
    for at in (0, 1, 2, 3, 4, 5, 15):
        assert "workspace overlaps" in distill_step(lib, dist(), ws=FAR[at], size=need.value), at


# ------------------------------------------------------------------------------------------------ norm and residual

def norm(dtype=1, sum_dtype=0):
    return ops.ast_norm_cfg(8, 40, dtype, sum_dtype, 1e-6)


def test_gradients_of_the_norm_on_other_tensors(lib):
    """A block's rows of another type, or shifted, are other blocks' rows."""
    n, need = 8 * 40, C.c_size_t()
    assert lib.asteroid_rms_norm_backward_workspace(norm(), need) == 0 and need.value > 0

    def call(cfg, ws=None, size=0, **at):
        a = dict(dy=FAR[0], s=FAR[1], gain=FAR[2], dsum=FAR[3], dx=FAR[4], ds=FAR[5], dgain=FAR[6])
        a.update(at)
        return refused(lib, "rms_norm_backward", cfg, a["dy"], a["s"], a["gain"], a["dsum"], a["dx"], a["ds"], a["dgain"], 0, ws, size, None)
    for cfg, a in ((norm(), {}), (norm(), dict(dx=FAR[0], ds=FAR[1])), (norm(), dict(ds=FAR[3])), (norm(), dict(dgain=FAR[2])), (norm(1, 1), dict(dx=FAR[1], ds=FAR[0])),
                   (norm(0, 0), dict(dx=FAR[3], ds=None)), (norm(), dict(dx=FAR[0] + 2 * n)), (norm(), dict(dsum=None, dx=None))):
        assert "workspace is missing" in call(cfg, **a), a
    for cfg, a in ((norm(), dict(dx=FAR[1])), (norm(), dict(dx=FAR[3])), (norm(), dict(ds=FAR[0])), (norm(1, 1), dict(dx=FAR[0] + 2)), (norm(0, 0), dict(ds=FAR[3] - 4 * n + 4)),
                   (norm(), dict(dx=FAR[2])), (norm(), dict(ds=FAR[2] + 4 * 39)), (norm(), dict(dgain=FAR[2] + 4)), (norm(), dict(dgain=FAR[0])), (norm(), dict(dgain=FAR[1])),
                   (norm(), dict(dgain=FAR[3] + 4 * n - 4))):
        assert "an output and an input" in call(cfg, **a), a
    for at in range(7):
        assert "workspace overlaps" in call(norm(), ws=FAR[at], size=need.value), at


def test_results_of_the_norm_on_other_tensors(lib):
    n = 8 * 40

    def call(cfg, **at):
        a = dict(x=FAR[0], r=FAR[1], gain=FAR[2], y=FAR[3], s=FAR[4], kept=FAR[5])
        a.update(at)
        return refused(lib, "rms_norm_forward", cfg, a["x"], a["r"], a["gain"], a["y"], a["s"], a["kept"], None)
    for cfg, a in ((norm(), dict(y=FAR[1])), (norm(), dict(s=FAR[0])), (norm(1, 1), dict(y=FAR[1] + 2)), (norm(0, 0), dict(s=FAR[0] + 4 * n - 4)), (norm(), dict(y=FAR[0] - 2)),
                   (norm(), dict(y=FAR[2])), (norm(), dict(s=FAR[2])), (norm(), dict(kept=FAR[2])), (norm(), dict(kept=FAR[0])), (norm(), dict(kept=FAR[1] + 16))):
        assert "an output and an input" in call(cfg, **a), a


# ------------------------------------------------------------------------------------------------ numbers without room

def test_entries_that_the_interface_has_no_room_for(lib):
    n = (1 << 32) + 7
    with pytest.raises(ValueError, match="entries"):
        ops.distill_step_workspace(4, 40000, n)
    ids, t, z = torch.zeros(0, n, dtype=torch.int32), torch.zeros(0, n), torch.zeros(0, 50)
    for call in (lambda: ops.distill_forward(z, ids, t), lambda: ops.distill_step(torch.zeros(0), z, ids, t),
                 lambda: ops.distill_backward(torch.zeros(0), z, ids, t, torch.zeros(0, 3))):
        with pytest.raises(ValueError, match="entries"):
            call()
