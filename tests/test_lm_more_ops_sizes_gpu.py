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
