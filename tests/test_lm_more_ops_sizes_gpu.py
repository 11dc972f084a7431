"""The norm with the residual, the gated recurrence and the distillation loss (paper_2408_08015_amd.ops) at sizes where a block has
more than one run of rows, where a lane has two channels, and with outputs in place of further inputs."""
import pytest
import torch

import test_lm_more_ops_gpu as G   # (the comparisons with the definition in 64 bits, and their bounds)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2408_08015_amd import ops
    return ops


# tokens, channels, lengths (0: by period), period: alone, by a few offsets, by many, as a chain, in wide blocks
@pytest.mark.parametrize("T,C,off,period", [(90, 33, [0, 7, 7, 60, 90], 0), (300, 65, list(range(0, 290, 4)) + [290, 290], 0), (700, 40, None, 700),
                                            (700, 40, None, 128), (129, 8, None, 1)])
def test_gradient_of_the_states_in_place_of_them(ops, T, C, off, period):
    g = torch.Generator(device="cuda").manual_seed(T)
    f, z, o, dy = (torch.randn(T, C, generator=g, device="cuda") for _ in range(4))
    kw = dict(offsets=torch.tensor(off, dtype=torch.int32, device="cuda")) if off else dict(period=period)
    n = len(off) - 1 if off else -(-T // period)
    h0, dfin = (torch.randn(n, C, generator=g, device="cuda") for _ in range(2))
    _, _, saved = ops.recurrence_forward(f, z, o=o, state=h0, saved=True, **kw)
    out = lambda: [torch.zeros(T, C, device="cuda") for _ in range(3)]   # (rows of no sequence are not written)
    for d in (dfin, None):
        want = ops.recurrence_backward(dy, f, z, saved, o=o, state=h0, dfinal=d, dstate=True, out=out(), **kw)
        moved = h0.clone()
        got = ops.recurrence_backward(dy, f, z, saved, o=o, state=moved, dfinal=d, dstate=moved, out=out(), **kw)
        assert got[3] is moved and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_of_the_gain_in_place_of_it(ops, accumulate):
    g = torch.Generator(device="cuda").manual_seed(3)
    dy, s = (torch.randn(500, 257, generator=g, device="cuda").bfloat16() for _ in range(2))
    gain = torch.rand(257, generator=g, device="cuda")
    want = ops.rms_norm_backward(dy, s, gain, gain_out=gain.clone(), accumulate=accumulate)
    got = ops.rms_norm_backward(dy, s, gain, gain_out=gain, accumulate=accumulate)
    assert got[2] is gain and torch.equal(got[2], want[2]) and torch.equal(got[0], want[0])


# ------------------------------------------------------------------------------------------------ several rows a group of lanes

# A launch has at most 2048 blocks forward (1024 backward) of 256 threads, or of 512 where rows are read in the tensor's groups, and a row of up to
# 512 values takes the power of two of lanes that holds a group of eight each, one of up to 1024 values 64 lanes, a longer one the block.
LOOPS = [(70000, 40), (140000, 41), (9000, 512), (17000, 513), (9000, 1024), (2500, 1504), (2500, 1501), (2300, 3001), (4096, 512), (40000, 100)]


def rows_at_once(width, blocks):
    lanes = 1 if width <= 8 else 1 << ((min(width, 512) + 14) // 8 - 1).bit_length()
    return blocks * (1 if width > 1024 else 512 // min(lanes, 64) if width % 8 else 256 // min(lanes, 64))


@pytest.mark.parametrize("dt,st", G.TYPES)
@pytest.mark.parametrize("rows,width", LOOPS[:8])
def test_norm_of_more_rows_than_a_launch_takes_at_once(ops, rows, width, dt, st):
    assert rows > rows_at_once(width, 2048)
    G.test_rms_norm_forward(ops, rows, width, dt, st)


@pytest.mark.parametrize("dt,st", G.TYPES)
@pytest.mark.parametrize("rows,width", LOOPS)
def test_gradient_of_the_norm_of_more_rows_than_a_launch_takes_at_once(ops, rows, width, dt, st):
    """The gain's gradient is a sum over a lane's own rows, then over the others'; also in place, and added to what is there."""
    assert rows > (rows_at_once(width, 512 if width <= 1024 else 1024))
    G.test_rms_norm_backward(ops, rows, width, dt, st)


@pytest.mark.parametrize("dt,st", G.TYPES)
@pytest.mark.parametrize("rows,width,off", [(70000, 40, 1), (9000, 512, 3), (9000, 1024, 1), (2500, 1501, 5), (9000, 700, 1)])
def test_norm_of_many_rows_from_odd_addresses(ops, rows, width, off, dt, st):
    G.test_rms_norm_of_long_rows(ops, rows, width, off, dt, st)


# ------------------------------------------------------------------------------------------------ two channels a lane

# bf16 calls of at least 1024 blocks of 128 tokens and channels: the last block column of one channel, of two, of some, full; a lane's pair
# that is half a row; one chain, uneven sequences with empty ones and rows of none, sequences that need no chain
PAIRS = [(65600, 129, ("period", 65600), True, True, "packed"), (65600, 129, ("ragged", 90, 70, 300), True, True, "apart"),
         (131100, 2, ("period", 50000), False, True, "apart"), (131100, 3, ("ragged", 2000, 5, 1), True, False, "packed"),
         (43700, 258, ("period", 64), True, True, "apart"), (43700, 300, ("period", 128), False, False, "packed"),
         (22000, 641, ("ragged", 61, 0, 0), True, True, "packed"), (33000, 512, ("ragged", 7, 129, 0), False, True, "packed")]


def takes_pairs(T, C):
    return -(-T // 128) * -(-C // 128) >= 1024


@pytest.mark.parametrize("T,C,how,gate,state,layout", PAIRS)
def test_recurrence_of_two_channels_a_lane(ops, T, C, how, gate, state, layout):
    assert takes_pairs(T, C)
    G.test_recurrence(ops, T, C, how, "bf16", gate, state, layout)


@pytest.mark.parametrize("how", ["period", "ragged"])
def test_recurrence_of_two_channels_a_lane_keeps_what_is_not_finite(ops, how):
    """NaN and infinities in one sequence, in its states, its gates and its gradients, in a lane's first and second channel: no other
    sequence's results change by a bit, nor do the other channels' in that one."""
    T, C = 65600, 129
    assert takes_pairs(T, C)
    g = torch.Generator(device="cuda").manual_seed(15)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    f, z, o, dy = (rnd(T, C).bfloat16() for _ in range(4))
    off = [0, 20000, 20000, 20100, 36001, 36003, 65600] if how == "ragged" else [0, 20000, 40000, 60000, 65600]
    n = len(off) - 1
    kw = dict(offsets=torch.tensor(off, dtype=torch.int32, device="cuda")) if how == "ragged" else dict(period=20000)
    h0, dfin = rnd(n, C), rnd(n, C)

    def both():
        y, fin, saved = ops.recurrence_forward(f, z, o=o, state=h0, final=True, saved=True, **kw)
        return (y, fin) + ops.recurrence_backward(dy, f, z, saved, o=o, state=h0, dfinal=dfin, dstate=True, **kw)
    clean = both()
    assert all(torch.isfinite(t).all() for t in clean)
    s = 3 if how == "ragged" else 1
    a, b = off[s], off[s + 1]
    nan, inf = float("nan"), float("inf")
    f[a, 2], f[a + 5000, 5], f[b - 1, 128], z[a + 1, 8], o[b - 2, 11], dy[a + 9, 14] = [nan] * 6
    z[a + 130, 17], h0[s, 20], dfin[s, 23], f[a + 7, 26], f[a + 8, 29] = inf, -inf, nan, inf, -inf
    touched = torch.tensor([2, 5, 128, 8, 11, 14, 17, 20, 23, 26, 29], device="cuda")
    got = both()
    for p, q in zip(got, clean):
        rows = torch.arange(p.shape[0], device="cuda")
        own = ((rows >= a) & (rows < b) if p.shape[0] == T else rows == s)[:, None]
        cols = torch.zeros(C, dtype=torch.bool, device="cuda").index_fill(0, touched, True)[None]
        assert torch.equal(torch.where(own & cols, 0.0, p), torch.where(own & cols, 0.0, q))
    assert got[0][a:a + 5000, 5].isfinite().all() and got[0][a + 5000:b, 5].isnan().all() and got[1][s, 5].isnan()
    assert got[0][a:b, 26].isfinite().all() and got[0][a:b, 29].isfinite().all()
    assert got[2][a:b, 23].isnan().any() and got[5][s, 23].isnan()
