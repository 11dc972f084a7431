"""CPU: what the single operators of language-model stages refuse, before anything is launched."""
import ctypes as C

import pytest
import torch

import paper_2408_08015_amd as A
from paper_2408_08015_amd import ops

EINVAL = -1
P = 1 << 20   # an address that is never read: the calls below are refused


@pytest.fixture(scope="module")
def lib():
    A.load_library()
    return ops._lib()


def refused(lib, name, *args):
    st = getattr(lib, "asteroid_" + name)(*args)
    msg = lib.asteroid_last_error().decode()
    assert st == EINVAL and name in msg, (name, args, st, msg)


def test_embedding_refusals(lib):
    ok = [P, 8, P, 0, 100, 16, 1.0, P, 0, None]
    for at, bad in ((0, None), (0, P + 1), (1, -1), (1, 1 << 31), (2, None), (2, P + 2), (3, 2), (4, 0), (4, 1 << 31), (5, 0), (5, (1 << 20) + 1),
                    (7, None), (7, P + 1), (8, -1)):
        refused(lib, "embedding_forward", *[bad if i == at else a for i, a in enumerate(ok)])
    assert lib.asteroid_embedding_forward(None, 0, None, 0, 100, 16, 1.0, None, 0, None) == 0   # no tokens: nothing to do
    n = C.c_size_t()
    refused(lib, "embedding_backward_workspace", 8, 100, 16, None)
    refused(lib, "embedding_backward_workspace", 8, 0, 16, C.byref(n))
    for scale in (float("inf"), float("-inf"), float("nan")):   # (0 times it would not be 0 for ids outside the table)
        refused(lib, "embedding_forward", P, 8, P, 0, 100, 16, scale, P, 0, None)
        refused(lib, "embedding_backward", P, 8, P, 0, 100, 16, scale, 0, P, P, 1 << 30, None)
    assert lib.asteroid_embedding_backward_workspace(8, 100, 16, C.byref(n)) == 0
    ok = [P, 8, P, 0, 100, 16, 1.0, 0, P, P, n.value, None]
    for at, bad in ((0, None), (1, -1), (2, None), (2, P + 2), (3, 7), (4, 0), (5, 0), (8, None), (8, P + 2), (9, None), (9, P + 4), (10, n.value - 1)):
        refused(lib, "embedding_backward", *[bad if i == at else a for i, a in enumerate(ok)])


def heads(**kw):
    h = dict(dev=P, token_stride=512, head_stride=64, heads=8)
    h.update(kw)
    return ops.ast_heads(h["dev"], h["token_stride"], h["head_stride"], h["heads"])


def cfg(**kw):
    c = dict(tokens=4, dtype=1, head_dim=64, rotary=64, interleaved=0, eps=1e-6, theta=1e4, positions_dev=P, period=0)
    c.update(kw)
    return ops.ast_qk_cfg(*[c[f] for f, _ in ops.ast_qk_cfg._fields_])


BAD_CFG = [dict(tokens=-1), dict(tokens=1 << 31), dict(dtype=2), dict(head_dim=0), dict(head_dim=257), dict(rotary=63), dict(rotary=66),
           dict(rotary=-2), dict(eps=0.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(theta=0.0), dict(theta=float("nan")),
           dict(positions_dev=P + 2), dict(positions_dev=None), dict(positions_dev=None, period=-3)]
BAD_IN = [dict(dev=None), dict(dev=P + 1), dict(token_stride=-1), dict(token_stride=1 << 31), dict(head_stride=-64),
          dict(head_stride=(1 << 40) + 1), dict(heads=0), dict(heads=65536)]
BAD_OUT = BAD_IN + [dict(heads=7), dict(head_stride=63), dict(token_stride=511), dict(token_stride=0), dict(head_stride=0)]


def test_qk_norm_rope_refusals(lib):
    fwd = lambda c, q, k, yq, yk, g=P, h=P: refused(lib, "qk_norm_rope_forward", c, q, k, g, h, yq, yk, None)
    for bad in BAD_CFG:
        fwd(cfg(**bad), heads(), heads(), heads(), heads())
    fwd(None, heads(), heads(), heads(), heads())
    for bad in BAD_IN:
        fwd(cfg(), heads(**bad), heads(), heads(), heads())
        fwd(cfg(), heads(), heads(**bad), heads(), heads())
    for bad in BAD_OUT:
        fwd(cfg(), heads(), heads(), heads(**bad), heads())
        fwd(cfg(), heads(), heads(), heads(), heads(**bad))
    for i in range(4):
        fwd(cfg(), *[None if j == i else heads() for j in range(4)])
    for g, h in ((None, P), (P, None), (P + 2, P), (P, P + 2)):
        fwd(cfg(), heads(), heads(), heads(), heads(), g, h)
    n = C.c_size_t()
    refused(lib, "qk_norm_rope_backward_workspace", cfg(), 8, 8, None)
    refused(lib, "qk_norm_rope_backward_workspace", cfg(), 0, 8, C.byref(n))
    refused(lib, "qk_norm_rope_backward_workspace", None, 8, 8, C.byref(n))
    assert lib.asteroid_qk_norm_rope_backward_workspace(cfg(), 8, 8, C.byref(n)) == 0 and n.value > 0

    def bwd(c, t, g=(P, P, P, P), ws=P, nb=None):
        refused(lib, "qk_norm_rope_backward", c, t[0], t[1], t[2], t[3], g[0], g[1], t[4], t[5], g[2], g[3], 0, ws, n.value if nb is None else nb, None)
    good = [heads() for _ in range(6)]
    for bad in BAD_CFG:
        bwd(cfg(**bad), good)
    for i in range(6):
        bwd(cfg(), [None if j == i else h for j, h in enumerate(good)])
        for bad in (BAD_OUT if i > 3 else BAD_IN + [dict(heads=7)]):
            bwd(cfg(), [heads(**bad) if j == i else h for j, h in enumerate(good)])
    for i in range(4):
        bwd(cfg(), good, [None if j == i else P for j in range(4)])
    bwd(cfg(), good, ws=None)
    bwd(cfg(), good, ws=P + 8)
    bwd(cfg(), good, nb=n.value - 1)


def test_stash8_refusals(lib):
    n = C.c_size_t()
    for r, c in ((-1, 8), (1 << 31, 8), (8, 0), (8, (1 << 20) + 1), ((1 << 31) - 1, 1 << 10)):
        refused(lib, "stash8_bytes", r, c, C.byref(n))
        refused(lib, "stash8_pack", P, 0, r, c, P, None)
        refused(lib, "stash8_unpack", P, r, c, P, 0, None)
        refused(lib, "gelu_backward_stash8", P, 0, P, r, c, P, None)
        refused(lib, "linear_wgrad_stash8_workspace", r, c, 8, C.byref(n))
        refused(lib, "linear_wgrad_stash8", P, P, r, c, 8, P, P, 0, P, 1 << 40, None)
    refused(lib, "stash8_bytes", 8, 8, None)
    for x, dt, s in ((None, 0, P), (P, 3, P), (P + 2, 0, P), (P + 1, 1, P), (P, 0, None), (P, 0, P + 8)):
        refused(lib, "stash8_pack", x, dt, 8, 8, s, None)
        refused(lib, "stash8_unpack", s, 8, 8, x, dt, None)
        refused(lib, "gelu_backward_stash8", x, dt, s, 8, 8, P, None)
    refused(lib, "gelu_backward_stash8", P, 0, P, 8, 8, None, None)
    refused(lib, "linear_wgrad_stash8_workspace", 8, 8, 0, C.byref(n))
    refused(lib, "linear_wgrad_stash8_workspace", 8, 1 << 20, 1 << 20, C.byref(n))
    refused(lib, "linear_wgrad_stash8_workspace", 8, 8, 8, None)
    assert lib.asteroid_linear_wgrad_stash8_workspace(4096, 512, 512, C.byref(n)) == 0 and n.value > 0
    ok = [P, P, 4096, 512, 512, P, P, 0, P, n.value, None]
    for at, bad in ((0, None), (0, P + 1), (1, None), (1, P + 8), (5, None), (5, P + 2), (6, P + 2), (8, None), (8, P + 8), (9, n.value - 1)):
        refused(lib, "linear_wgrad_stash8", *[bad if i == at else a for i, a in enumerate(ok)])


def test_every_share_of_a_weight_gradient_has_rows(lib):
    """Shares are whole steps of 64 rows; as many as have any."""
    n = C.c_size_t()
    for cin, cout in ((40, 300), (128, 128), (512, 192), (2816, 31), (2048, 512)):
        for rows in list(range(250, 1200, 13)) + [2049, 4097, 5732, 8645, 8787, 10099, 16384, 100003]:
            assert lib.asteroid_linear_wgrad_stash8_workspace(rows, cin, cout, C.byref(n)) == 0
            shares, rest = divmod(n.value, 4 * (cin + 1) * cout)
            assert rest == 0 and shares != 1
            if shares:
                per = -(-rows // shares)
                assert (shares - 1) * (-(-per // 64) * 64) < rows, (rows, cin, cout, shares)


def test_tensors_are_checked():
    f, i = torch.zeros, torch.int32
    with pytest.raises(ValueError, match="GPU"):
        ops.embedding_forward(f(3, dtype=i), f(4, 8))
    with pytest.raises(ValueError, match="int32"):
        ops.embedding_forward(f(3, dtype=torch.int64), f(4, 8))
    with pytest.raises(ValueError, match="contiguous"):
        ops.embedding_forward(f(3, dtype=i), f(8, 4).t())
    with pytest.raises(ValueError, match="shape"):
        ops.embedding_forward(f(3, dtype=i), f(4, 8), out=f(3, 7))
    with pytest.raises(ValueError, match="float32 or torch.bfloat16"):
        ops.embedding_forward(f(3, dtype=i), f(4, 8), dtype=torch.float16)
    with pytest.raises(ValueError, match="not torch.bfloat16"):
        ops.embedding_forward(f(3, dtype=i), f(4, 8), dtype=torch.bfloat16, out=f(3, 8))
    with pytest.raises(ValueError, match="float32 or torch.bfloat16"):
        ops.embedding_backward(f(3, dtype=i), f(3, 8, dtype=torch.float16), 4)
    with pytest.raises(ValueError, match="shape"):
        ops.embedding_backward(f(3, dtype=i), f(2, 8), 4)
    with pytest.raises(ValueError, match="accumulate"):
        ops.embedding_backward(f(3, dtype=i), f(3, 8), 4, accumulate=True)
    g = f(8)
    with pytest.raises(ValueError, match="period"):
        ops.qk_norm_rope_forward(f(3, 2, 8), f(3, 2, 8), g, g)
    with pytest.raises(ValueError, match="k must be"):
        ops.qk_norm_rope_forward(f(3, 2, 8), f(4, 2, 8), g, g, period=3)
    with pytest.raises(ValueError, match="unit stride"):
        ops.qk_norm_rope_forward(f(3, 8, 2).transpose(1, 2), f(3, 2, 8), g, g, period=3)
    with pytest.raises(ValueError, match="positions"):
        ops.qk_norm_rope_forward(f(3, 2, 8), f(3, 2, 8), g, g, positions=f(2, dtype=i))
    with pytest.raises(ValueError, match="accumulate"):
        ops.qk_norm_rope_backward(*[f(3, 2, 8)] * 4, g, g, period=3, accumulate=True)
    with pytest.raises(ValueError, match="Stash8"):
        ops.stash8_unpack(f(8))
    with pytest.raises(ValueError, match="matrix"):
        ops.stash8_pack(f(8))
    s = ops.Stash8(4, 40, "cpu")
    assert s.data.numel() == 4 * 64 + 8 + 8 == ops.stash8_bytes(4, 40)
    with pytest.raises(ValueError, match="keeps"):
        ops.stash8_pack(f(4, 41), out=s)
    with pytest.raises(ValueError, match="rows"):
        ops.linear_wgrad_stash8(f(5, 8, dtype=torch.bfloat16), s)
    with pytest.raises(ValueError, match="bfloat16"):
        ops.linear_wgrad_stash8(f(4, 8), s)
    with pytest.raises(ValueError, match="workspace"):
        ops.Stash8(4, 40, "cpu", data=f(10, dtype=torch.uint8))


def test_numbers_that_the_c_interface_has_no_room_for():
    q, g = torch.zeros(3, 2, 8), torch.zeros(8)
    with pytest.raises(ValueError, match="period"):
        ops.qk_norm_rope_forward(q, q, g, g, period=(1 << 32) + 3)
    with pytest.raises(ValueError, match="rotary"):
        ops.qk_norm_rope_forward(q, q, g, g, period=3, rotary=(1 << 32) + 8)


def test_outputs_that_lie_on_each_other(lib):
    """Two writers of one place: gradients of a gain that queries and keys share, one tensor for both results, dW over db."""
    n = C.c_size_t()
    assert lib.asteroid_qk_norm_rope_backward_workspace(cfg(), 8, 8, C.byref(n)) == 0
    h, far = heads(), heads(dev=P + (1 << 20))
    bwd = lambda dq, dk, g, w: refused(lib, "qk_norm_rope_backward", cfg(), h, h, h, h, P, P, dq, dk, g, w, 1, P, n.value, None)
    for by in (0, 4, 252, -252):
        bwd(h, far, P + 1024, P + 1024 + by)
        assert "gains" in lib.asteroid_last_error().decode()
    bwd(h, h, P, P + 256)
    assert "one tensor" in lib.asteroid_last_error().decode()
    refused(lib, "qk_norm_rope_forward", cfg(), h, h, P, P, far, far, None)
    assert "one tensor" in lib.asteroid_last_error().decode()
    assert lib.asteroid_linear_wgrad_stash8_workspace(64, 40, 24, C.byref(n)) == 0
    for by in (0, 4 * 40 * 24 - 4, -4 * 23):
        refused(lib, "linear_wgrad_stash8", P, P, 64, 40, 24, P + 4096, P + 4096 + by, 0, P, 1 << 30, None)
        assert "overlap" in lib.asteroid_last_error().decode()
