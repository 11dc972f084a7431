"""The single operators of language-model stages (paper_2408_08015_amd.ops) against their definition in 64 bits.

Bounds: u = 2^-24 is half a step of fp32.  A sum of n terms in any order is off by at most n u times the sum of the terms'
magnitudes, a rounding to bf16 by 2^-8 of the value; what an entry is added up from comes from the oracle."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import lm_ops as O

pytestmark = pytest.mark.gpu

u = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


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
    return t, a


def host(t):
    return t.double().cpu().numpy()


def inside(got, want, bound):
    """|got - want| <= bound, entry by entry; NaN where the definition has NaN and nowhere else."""
    got, bound = host(got), np.broadcast_to(bound, want.shape)
    assert got.shape == want.shape
    assert np.array_equal(np.isnan(got), np.isnan(want))
    bad = np.flatnonzero(~np.isnan(want) & ~(abs(got - want) <= bound))
    assert bad.size == 0, (bad.size, bad[:5], got.ravel()[bad[:5]], want.ravel()[bad[:5]], bound.ravel()[bad[:5]])


# ------------------------------------------------------------------------------------------------ embedding

IDS = {
    "text": lambda r, T, V: (np.exp(r.uniform(0, np.log(V + 1.0), T)).astype(np.int64) - 1).clip(0, V - 1),
    "one": lambda r, T, V: np.full(T, V - 1),
    "none": lambda r, T, V: np.full(T, -1),
    "mixed": lambda r, T, V: r.choice([-1, 0, V - 1, V, V + 1, -2**31, 2**31 - 1, V // 2], T),
    "each": lambda r, T, V: r.permutation(np.arange(T) % V),
}
EMBED = [(1, 1, 1, "one"), (1, 1000, 512, "text"), (2, 5, 3, "mixed"), (64, 300, 8, "text"), (65, 300, 33, "text"), (300, 7, 520, "mixed"),
         (257, 257, 100, "each"), (2048, 513, 64, "text"), (1000, 40, 1021, "one"), (500, 40, 16, "none"), (4097, 3000, 24, "text"),
         (9000, 70000, 9, "text"), (12289, 4, 40, "mixed"), (20000, 1 << 20, 2, "text"), (33000, 100, 12, "text")]


@pytest.mark.parametrize("table_t,out_t", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("T,V,D,kind", EMBED)
def test_embedding_forward(ops, T, V, D, kind, table_t, out_t):
    r = rng(1, T, V, D)
    ids = IDS[kind](r, T, V).astype(np.int32)
    table, W = dev(r.normal(size=(V, D)), table_t)
    y = ops.embedding_forward(dev(ids)[0], table, scale=1.7, dtype=DT[out_t])
    want = O.embedding_forward(ids, W, float(np.float32(1.7)))
    inside(y, want, abs(want) * (u + HALF[out_t]) * 1.001)


@pytest.mark.parametrize("table_t,out_t", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("T,V,D", [(9000, 5003, 1024), (9001, 5003, 1021), (9000, 700, 1026), (1000003, 300, 9), (1100001, 50, 8), (300007, 64, 28)])
def test_embedding_forward_of_many_values(ops, T, V, D, table_t, out_t):
    """Four groups of eight a thread, rows at 16-byte addresses and not."""
    from paper_2408_08015_amd import lib_path
    assert C.CDLL(lib_path()).ast_embedding_fwd_choice(C.c_int64(T), C.c_int64(D)) == 4
    g = torch.Generator(device="cuda").manual_seed(T + D)
    table = torch.randn(V, D, generator=g, device="cuda").to(DT[table_t])
    ids = torch.randint(-V // 8, V + V // 8, (T,), generator=g, device="cuda", dtype=torch.int32)
    ids[-1], ids[0] = V - 1, 0
    y = ops.embedding_forward(ids, table, scale=1.7, dtype=DT[out_t])
    live = (ids >= 0) & (ids < V)
    want = table.double()[ids.long().clamp(0, V - 1)] * float(np.float32(1.7)) * live.unsqueeze(1)
    assert ((y.double() - want).abs() <= want.abs() * (u + HALF[out_t]) * 1.001).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,D,kind", EMBED)
def test_embedding_backward(ops, T, V, D, kind, dt):
    r = rng(2, T, V, D)
    ids = IDS[kind](r, T, V).astype(np.int32)
    dy, g = dev(r.normal(size=(T, D)), dt)
    want, terms, n = O.embedding_backward(ids, g, V, float(np.float32(0.3)))
    bound = (n[:, None] + 2) * u * terms * 1.001
    out = torch.full((V, D), float("nan"), device="cuda")
    got = ops.embedding_backward(dev(ids)[0], dy, V, scale=0.3, out=out)
    assert got is out
    inside(got, want, bound)
    again = ops.embedding_backward(dev(ids)[0], dy, V, scale=0.3)
    assert torch.equal(got, again)                      # equal calls give equal bits
    old = r.normal(size=(V, D)).astype(np.float32)
    acc = ops.embedding_backward(dev(ids)[0], dy, V, scale=0.3, out=dev(old)[0], accumulate=True)
    inside(acc, old + want, bound + u * 1.001 * (abs(old) + terms))
    still = n == 0
    assert np.array_equal(host(acc)[still], old[still].astype(np.float64))   # rows without a token stay


@pytest.mark.parametrize("D", [513, 516, 519, 520, 1025, 1031])
def test_embedding_rows_that_end_just_behind_a_share_of_the_columns(ops, D):
    """A block's last columns may be a few only: every column has one writer all the same, which adding needs."""
    r = rng(11, D)
    T, V = 700, 90
    ids = IDS["text"](r, T, V).astype(np.int32)
    dy, g = dev(r.normal(size=(T, D)), "bf16")
    want, terms, n = O.embedding_backward(ids, g, V, 1.0)
    bound = (n[:, None] + 2) * u * terms * 1.001
    inside(ops.embedding_backward(dev(ids)[0], dy, V), want, bound)
    old = r.normal(size=(V, D)).astype(np.float32)
    for _ in range(3):
        acc = ops.embedding_backward(dev(ids)[0], dy, V, out=dev(old)[0], accumulate=True)
        inside(acc, old + want, bound + u * 1.001 * (abs(old) + terms))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("D", [9, 15, 63, 127, 519, 526, 1021, 1535])
def test_embedding_adds_a_tokens_gradient_to_every_column_once(ops, D, dt):
    """Rows that do not end with a lane's eight columns, every row of the table inside a chunk, at a chunk's end and across
    chunks; small whole numbers, so the sums are exact."""
    r = rng(14, D)
    for T, V in ((700, 311), (3000, 40), (20000, 3001)):
        ids = r.integers(0, V, T)
        dy = r.integers(-4, 5, (T, D))
        old = r.integers(-100, 101, (V, D))
        want = old.copy()
        np.add.at(want, ids, 2 * dy)
        got = dev(old.astype(np.float32))[0]
        for n in range(2):
            ops.embedding_backward(dev(ids.astype(np.int32))[0], dev(dy.astype(np.float32), dt)[0], V, scale=2.0, out=got, accumulate=True)
            assert np.array_equal(host(got), old + (n + 1) * (want - old)), (T, V, n)


@pytest.mark.parametrize("T,step", [(64, 1), (4096, 1), (16384, 3), (20480, 1), (32768, 40), (65536, 100), (262144, 1)])
@pytest.mark.parametrize("D", [3, 8, 13])
def test_embedding_adds_the_tokens_of_an_id_in_their_order(ops, T, step, D):
    """Every id four times, so that no run of sorted tokens crosses a chunk: the fp32 sums from the first token to the last, bit
    for bit, which needs an order that is stable among equal ids."""
    r = rng(15, T, D)
    ids = r.permutation(np.repeat(np.arange(T // 4) * step, 4))
    dy = (r.normal(size=(T, D)) * np.exp(4 * r.normal(size=(T, 1)))).astype(np.float32)
    V = T // 4 * step
    got = ops.embedding_backward(dev(ids.astype(np.int32))[0], dev(dy)[0], V).cpu().numpy()
    a = dy[np.argsort(ids, kind="stable")].reshape(T // 4, 4, D)
    want = np.zeros((V, D), np.float32)
    want[::step] = ((a[:, 0] + a[:, 1]) + a[:, 2]) + a[:, 3]
    assert np.array_equal(got, want)


def test_embedding_of_no_tokens(ops):
    ids = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert ops.embedding_forward(ids, torch.ones(3, 4, device="cuda")).shape == (0, 4)
    dy = torch.zeros(0, 4, device="cuda")
    assert not ops.embedding_backward(ids, dy, 3).any()
    out = torch.ones(3, 4, device="cuda")
    assert ops.embedding_backward(ids, dy, 3, out=out, accumulate=True).eq(1).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("D", [5, 64])
def test_embedding_tensors_that_are_not_16_byte_aligned(ops, dt, D):
    r = rng(3, D)
    T, V = 130, 50
    ids = IDS["text"](r, T, V).astype(np.int32)
    skew = lambda a, t: dev(np.concatenate((np.zeros(1, a.dtype), a.ravel())), t)[0][1:].view(a.shape)
    table, dy = r.normal(size=(V, D)).astype(np.float32), r.normal(size=(T, D)).astype(np.float32)
    i0, t0, d0 = dev(ids)[0], dev(table, dt)[0], dev(dy, dt)[0]
    i1, t1, d1 = skew(ids, "f32"), skew(table, dt), skew(dy, dt)
    assert t1.data_ptr() % 16 and d1.data_ptr() % 16
    assert torch.equal(ops.embedding_forward(i0, t0), ops.embedding_forward(i1, t1))
    out = torch.zeros(V * D + 1, device="cuda")[1:].view(V, D)
    assert torch.equal(ops.embedding_backward(i0, d0, V), ops.embedding_backward(i1, d1, V, out=out))


# ------------------------------------------------------------------------------------------------ queries and keys

QK = [  # tokens, query heads, key heads, head_dim, rotary, interleaved, dtype
    (1, 1, 1, 64, 64, False, "bf16"), (1, 3, 2, 64, 64, True, "bf16"), (37, 8, 8, 64, 64, False, "bf16"), (130, 4, 1, 128, 128, False, "bf16"),
    (65, 6, 2, 256, 256, False, "bf16"), (65, 6, 2, 256, 256, True, "f32"), (33, 5, 3, 96, 96, False, "bf16"), (33, 5, 3, 80, 32, False, "bf16"),
    (50, 2, 2, 80, 40, True, "f32"), (50, 2, 2, 80, 40, False, "bf16"), (19, 7, 1, 40, 40, True, "bf16"), (19, 7, 1, 24, 24, True, "bf16"), (19, 300, 1, 8, 8, False, "f32"),
    (21, 3, 2, 63, 62, False, "bf16"), (21, 3, 2, 63, 20, True, "f32"), (21, 2, 2, 2, 2, False, "f32"), (21, 2, 2, 1, 0, False, "bf16"),
    (40, 2, 1, 64, 0, False, "bf16"), (40, 2, 1, 199, 0, True, "f32"), (17, 2, 2, 255, 254, True, "bf16"), (2500, 2, 1, 64, 32, False, "f32"),
    (9000, 1, 1, 16, 16, False, "bf16"),
]


def qk_case(T, hq, hk, d, dt, seed, packed):
    r = rng(4, T, hq, hk, d, seed)
    heads = hq + 2 * hk if packed else hq + hk
    x, v = dev(r.normal(size=(T, heads, d)) * np.exp(r.normal(size=(T, heads, 1))), dt)
    q, k = x[:, :hq], x[:, hq:hq + hk]
    if not packed:
        q, k = q.contiguous(), k.contiguous()
    gains = [dev(1 + 0.3 * r.normal(size=d)) for _ in range(2)]
    pos = r.integers(-5, 1 << 20, T).astype(np.int32)
    return q, k, v[:, :hq], v[:, hq:hq + hk], gains, pos, r


def forward_bound(want, parts, d, dt):
    # relative roundings of a value: the sum of squares (d terms, halved by the root) and the root d / 2 + 4, norm and gain 3,
    # cos and sin 6 (half a turn rounded to fp32: pi / 2 u, and 2 ulp), the rotation 3
    return parts * (d / 2 + 16) * u * 1.01 + abs(want) * HALF[dt] * 1.001


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("T,hq,hk,d,rot,inter,dt", QK)
def test_qk_norm_rope_forward(ops, T, hq, hk, d, rot, inter, dt, packed):
    q, k, fq, fk, gains, pos, _ = qk_case(T, hq, hk, d, dt, rot, packed)
    kw = dict(rotary=rot, interleaved=inter, theta=10000.0, eps=1e-5)
    y = ops.qk_norm_rope_forward(q, k, gains[0][0], gains[1][0], positions=dev(pos)[0], **kw)
    for got, x, g in ((y[0], fq, gains[0][1]), (y[1], fk, gains[1][1])):
        want, parts = O.norm_rope_forward(x, g, pos, rot, 10000.0, inter, float(np.float32(1e-5)))
        inside(got, want, forward_bound(want, parts, d, dt))
    # in place, and positions that count up inside sequences of 16
    q2, k2 = q.clone(), k.clone()
    z = ops.qk_norm_rope_forward(q2, k2, gains[0][0], gains[1][0], positions=dev(pos)[0], out=(q2, k2), **kw)
    assert z[0] is q2 and torch.equal(q2, y[0]) and torch.equal(k2, y[1])
    a = ops.qk_norm_rope_forward(q, k, gains[0][0], gains[1][0], period=16, **kw)
    b = ops.qk_norm_rope_forward(q, k, gains[0][0], gains[1][0], positions=dev((np.arange(T) % 16).astype(np.int32))[0], **kw)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("T,hq,hk,d,rot,inter,dt", QK)
def test_qk_norm_rope_backward(ops, T, hq, hk, d, rot, inter, dt, packed):
    q, k, fq, fk, gains, pos, r = qk_case(T, hq, hk, d, dt, rot + 1, packed)
    dyq, gyq = dev(r.normal(size=(T, hq, d)), dt)
    dyk, gyk = dev(r.normal(size=(T, hk, d)), dt)
    args = (q, k, gains[0][0], gains[1][0])
    kw = dict(positions=dev(pos)[0], rotary=rot, interleaved=inter, theta=10000.0, eps=1e-5)
    got = ops.qk_norm_rope_backward(dyq, dyk, *args, **kw)
    old = [dev(r.normal(size=d)) for _ in range(2)]
    in_place = (dyq.clone(), dyk.clone())
    acc = ops.qk_norm_rope_backward(*in_place, *args, out=in_place, gain_out=[o[0].clone() for o in old], accumulate=True, **kw)
    for w, (x, dy, g) in enumerate(((fq, gyq, gains[0][1]), (fk, gyk, gains[1][1]))):
        dx, dg, dxa, dga = O.norm_rope_backward(dy, x, g, pos, rot, 10000.0, inter, float(np.float32(1e-5)))
        # the two sums over a head (2 d), the norms and the products around them, cos and sin (as forward)
        inside(got[w], dx, dxa * (2 * d + 40) * u * 1.01 + abs(dx) * HALF[dt] * 1.001)
        n = x.shape[0] * x.shape[1]
        bound = dga * (n + d / 2 + 24) * u * 1.01
        inside(got[2 + w], dg, bound)
        inside(acc[2 + w], old[w][1] + dg, bound + u * 1.01 * (abs(old[w][1]) + dga))
        assert torch.equal(acc[w], got[w])
    assert all(torch.equal(a, b) for a, b in zip(got, ops.qk_norm_rope_backward(dyq, dyk, *args, **kw)))


def test_qk_norm_rope_zero_rows_and_no_tokens(ops):
    g = torch.ones(64, device="cuda")
    q = torch.zeros(5, 2, 64, device="cuda", dtype=torch.bfloat16)
    y = ops.qk_norm_rope_forward(q, q.clone(), g, g, period=5)
    assert not y[0].any() and not y[1].any()            # a head of zeros: 0, not NaN
    dy = torch.ones_like(q)
    dq, dk, dgq, dgk = ops.qk_norm_rope_backward(dy, dy, q, q, g, g, period=5)
    assert torch.isfinite(dq).all() and not dgq.any()
    e = q[:0]
    assert ops.qk_norm_rope_forward(e, e, g, g, period=1)[0].shape == (0, 2, 64)
    r = ops.qk_norm_rope_backward(e, e, e, e, g, g, period=1)
    assert not r[2].any() and not r[3].any()


def test_qk_norm_rope_tokens_inside_heads(ops):
    """Heads outermost (another order of strides), odd strides and an unaligned start."""
    r = rng(5)
    T, H, d = 45, 3, 64
    x, f = dev(r.normal(size=(T, H, d)), "bf16")
    g = [dev(1 + 0.1 * r.normal(size=d)) for _ in range(2)]
    base = ops.qk_norm_rope_forward(x, x.clone(), g[0][0], g[1][0], period=T)
    outer = x.permute(1, 0, 2).contiguous().permute(1, 0, 2)
    room = torch.zeros(T * H * 65 + 1, device="cuda", dtype=torch.bfloat16)
    odd = room[1:].view(T, H, 65)[:, :, :64]
    odd.copy_(x)
    for q in (outer, odd):
        want, parts = O.norm_rope_forward(f, g[0][1], np.arange(T), d, 10000.0, False, float(np.float32(1e-6)))
        y = ops.qk_norm_rope_forward(q, q, g[0][0], g[1][0], period=T)
        inside(y[0], want, forward_bound(want, parts, d, "bf16"))
        assert (y[0].float() - base[0].float()).abs().max() <= 2.0 ** -7 * base[0].float().abs().max()
    out = (torch.zeros(H, T, d, device="cuda", dtype=torch.bfloat16).permute(1, 0, 2), torch.zeros_like(x))
    y = ops.qk_norm_rope_forward(x, x, g[0][0], g[1][0], period=T, out=out)
    assert torch.equal(y[0], base[0]) and torch.equal(y[1], base[1])


def test_qk_norm_rope_broadcast_gradients_and_one_head_for_all(ops):
    """Inputs whose tokens or heads lie on top of each other (strides of zero)."""
    r = rng(12)
    T, H, d = 70, 4, 64
    x = dev(r.normal(size=(T, 1, d)), "bf16")[0]
    one = dev(r.normal(size=(1, 1, d)), "bf16")[0]
    g = [dev(1 + 0.1 * r.normal(size=d))[0] for _ in range(2)]
    for q, dy in ((x.expand(T, H, d), one.expand(T, H, d)), (x.expand(T, H, d), torch.ones_like(one).expand(T, H, d))):
        a = ops.qk_norm_rope_backward(dy, dy, q, q, g[0], g[1], period=T)
        b = ops.qk_norm_rope_backward(dy.contiguous(), dy.contiguous(), q.contiguous(), q.contiguous(), g[0], g[1], period=T)
        assert all(torch.equal(m, n) for m, n in zip(a, b))
        assert torch.equal(ops.qk_norm_rope_forward(q, q, g[0], g[1], period=T)[0],
                           ops.qk_norm_rope_forward(q.contiguous(), q, g[0], g[1], period=T)[0])


# ------------------------------------------------------------------------------------------------ 8-bit activations

SHAPES = [(1, 1), (1, 32), (3, 31), (5, 33), (2, 64), (7, 1500), (130, 40), (257, 129), (1000, 512), (63, 2048), (4096, 24), (1, 4099)]


def activations(r, rows, cols, kind):
    x = r.normal(size=(rows, cols)) * np.exp(r.normal(size=(1, cols)))
    if kind == "extreme":      # zeros, the type's smallest and largest values, ties between two steps
        x *= np.exp2(r.integers(-140, 120, size=(rows, 1)).astype(np.float64))
        x[r.random(x.shape) < 0.2] = 0
        x[::3] = np.rint(x[::3] / abs(x[::3]).max() * 254) / 2
        x[::7] = np.sign(x[::7]) * 3.38e38
        x[1::5] = 0
    if kind == "broken":
        x[r.random(x.shape) < 0.02] = np.nan
        x[r.random(x.shape) < 0.02] = -np.inf
    return x


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["plain", "extreme", "broken"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_stash8_is_exact(ops, rows, cols, kind, dt):
    x, f = dev(activations(rng(6, rows, cols), rows, cols, kind).astype(np.float32), dt)
    want, codes, e = O.stash8(f)
    s = ops.stash8_pack(x)
    for out in (torch.float32, torch.bfloat16):
        inside(ops.stash8_unpack(s, out), want, 0.0)
    pitch = (cols + 31) // 32 * 32
    raw = s.data.cpu().numpy()
    assert np.array_equal(raw[:rows * pitch].view(np.int8).reshape(codes.shape), codes)
    assert np.array_equal(raw[rows * pitch:rows * pitch // 32 * 33].astype(int) - 127, e.ravel())
    again = ops.stash8_pack(ops.stash8_unpack(s, torch.float32))
    inside(ops.stash8_unpack(again, torch.float32), want, 0.0)


def test_stash8_from_an_unaligned_matrix_and_of_no_rows(ops):
    x = torch.randn(1 + 50 * 77, device="cuda")
    a, b = x[1:].view(50, 77), x[1:].clone().view(50, 77)
    assert torch.equal(ops.stash8_pack(a).data[:50 * 96], ops.stash8_pack(b).data[:50 * 96])
    out = torch.zeros(1 + 50 * 77, device="cuda", dtype=torch.bfloat16)[1:].view(50, 77)
    assert torch.equal(ops.stash8_unpack(ops.stash8_pack(a), out=out), ops.stash8_unpack(ops.stash8_pack(b)))
    s = ops.stash8_pack(torch.zeros(0, 40, device="cuda"))
    assert ops.stash8_unpack(s).shape == (0, 40)
    dw, db = ops.linear_wgrad_stash8(torch.zeros(0, 8, device="cuda", dtype=torch.bfloat16), s)
    assert dw.shape == (8, 40) and not dw.any() and not db.any()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["plain", "broken"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_gelu_backward_stash8(ops, rows, cols, kind, dt):
    r = rng(7, rows, cols)
    z, f = dev(2 * activations(r, rows, cols, kind).astype(np.float32), dt)
    dy, g = dev(r.normal(size=(rows, cols)), dt)
    zz = O.stash8(f)[0]
    phi, slope = O.gelu_parts(zz)
    want = g * (phi + slope)
    # Phi: argument (z^2 relative), a few ulp, and in the bf16 form 3e-7; phi: its exponent z^2 / 2 rounded
    bound = abs(g) * ((phi + abs(slope)) * (24 + 6 * zz * zz) * u + (3.1e-7 if dt == "bf16" else 0)) + abs(want) * HALF[dt] * 1.001 + 1e-37
    s = ops.stash8_pack(z)
    got = ops.gelu_backward_stash8(dy, s)
    inside(got, want, bound)
    same = dy.clone()
    assert torch.equal(torch.nan_to_num(ops.gelu_backward_stash8(same, s, out=same), 9.0), torch.nan_to_num(got, 9.0))


WGRAD = [(1, 1, 1), (1, 40, 8), (31, 33, 7), (33, 64, 130), (256, 129, 127), (300, 513, 65), (1000, 128, 128), (2049, 96, 200),
         (513, 1000, 24), (4097, 40, 300), (700, 2048, 3), (12000, 24, 17)]


@pytest.mark.parametrize("rows,cin,cout", WGRAD)
def test_linear_wgrad_stash8(ops, rows, cin, cout):
    r = rng(8, rows, cin, cout)
    x, f = dev(activations(r, rows, cin, "plain"), "bf16")
    dy, g = dev(r.normal(size=(rows, cout)), "bf16")
    s = ops.stash8_pack(x)
    xx = O.stash8(f)[0]
    # products are exact; a sum of `rows` terms, where a matrix instruction may cut a step instead of rounding it (2 u)
    want, bound = g.T @ xx, (abs(g).T @ abs(xx)) * (2 * rows + 4) * u
    wb, bb = g.sum(0), abs(g).sum(0) * (rows + 4) * u
    dw, db = ops.linear_wgrad_stash8(dy, s)
    inside(dw, want, bound)
    inside(db, wb, bb)
    again = ops.linear_wgrad_stash8(dy, s)
    assert torch.equal(dw, again[0]) and torch.equal(db, again[1])
    old, oldb = dev(r.normal(size=(cout, cin)))[0], dev(r.normal(size=cout))[0]
    ow, ob = host(old), host(oldb)
    acc = ops.linear_wgrad_stash8(dy, s, out=old, bias_out=oldb, accumulate=True)
    inside(acc[0], ow + want, bound + 1.01 * u * (abs(ow) + abs(g).T @ abs(xx)))
    inside(acc[1], ob + wb, bb + 1.01 * u * (abs(ob) + abs(g).sum(0)))
    only, none = ops.linear_wgrad_stash8(dy, s, bias=False)
    assert none is None and torch.equal(only, dw)


@pytest.mark.parametrize("rows,cin,cout,shares", [
    (64, 4096, 4096, 1), (257, 4096, 4096, 1), (1000, 4096, 4096, 1), (257, 4096, 4093, 1), (1000, 4096, 4093, 1), (2111, 4000, 3999, 1),
    (1000, 4095, 4096, 1), (4862, 1430, 1024, 8), (4862, 1430, 1019, 8)])
def test_linear_wgrad_stash8_in_the_large_tile(ops, rows, cin, cout, shares):
    """Rows of dy at 16-byte addresses and not, dW written by the product itself and from shares, with and without adding."""
    from paper_2408_08015_amd import lib_path
    pick = (C.c_int * 2)()
    C.CDLL(lib_path()).ast_stash8_wgrad_choice(C.c_int64(rows), C.c_int64(cin), C.c_int64(cout), pick)
    assert tuple(pick) == (256, shares)
    gen = torch.Generator(device="cuda").manual_seed(rows + cin + cout)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    s = ops.stash8_pack((rnd(rows, cin) * torch.exp(rnd(cin))).bfloat16())
    xx = ops.stash8_unpack(s, torch.float32).double()
    dy = rnd(rows, cout).bfloat16()
    g = dy.double()
    want, terms = torch.mm(g.t(), xx), torch.mm(g.abs().t(), xx.abs())
    wb, tb = g.sum(0), g.abs().sum(0)
    # as in test_linear_wgrad_stash8
    near = lambda got, want, bound: bool(((got.double() - want).abs() <= bound).all())
    dw, db = ops.linear_wgrad_stash8(dy, s)
    assert near(dw, want, terms * ((2 * rows + 4) * u)) and near(db, wb, tb * ((rows + 4) * u))
    old, oldb = rnd(cout, cin), rnd(cout)
    acc, accb = ops.linear_wgrad_stash8(dy, s, out=old.clone(), bias_out=oldb.clone(), accumulate=True)
    assert near(acc, old.double() + want, terms * ((2 * rows + 4) * u) + 1.01 * u * (old.double().abs() + terms))
    assert near(accb, oldb.double() + wb, tb * ((rows + 4) * u) + 1.01 * u * (oldb.double().abs() + tb))
    only, none = ops.linear_wgrad_stash8(dy, s, bias=False)
    assert none is None and torch.equal(only, dw)


def test_linear_wgrad_stash8_at_the_ends_of_the_range(ops):
    """Inputs of the largest and smallest sizes that are kept, dy small enough that the products are finite."""
    r = rng(13)
    rows, cin, cout = 90, 96, 40
    x = r.normal(size=(rows, cin))
    x[:, :32] = np.sign(x[:, :32]) * 3.38e38
    x[:, 32:64] *= 2.0 ** -120
    xt, f = dev(x.astype(np.float32), "bf16")
    dy, g = dev(r.normal(size=(rows, cout)) * 2.0 ** -10, "bf16")
    xx = O.stash8(f)[0]
    dw, db = ops.linear_wgrad_stash8(dy, ops.stash8_pack(xt))
    inside(dw, g.T @ xx, (abs(g).T @ abs(xx)) * (2 * rows + 4) * u + 2.0 ** -149 * rows)


def test_linear_wgrad_stash8_keeps_what_is_not_finite_in_its_column(ops):
    r = rng(9)
    x = r.normal(size=(400, 200))
    x[77, 33] = np.nan
    dy = r.normal(size=(400, 50))
    dy[5, 4] = np.inf
    xt, dt = dev(x, "bf16")[0], dev(dy, "bf16")[0]
    dw = host(ops.linear_wgrad_stash8(dt, ops.stash8_pack(xt))[0])
    bad = ~np.isfinite(dw)
    want = np.zeros_like(bad)
    want[:, 32:64] = True     # the block of the NaN
    want[4] = True            # the output of the infinity
    assert np.array_equal(bad, want)


# ------------------------------------------------------------------------------------------------ together

def test_operators_on_another_stream_and_in_a_replayed_graph(ops):
    """Embedding, heads, kept activations and all gradients as one chain: on a stream of the caller's, and captured and
    replayed with the program's own work and new inputs between the replays; equal bits everywhere."""
    T, V, H, d, N = 700, 900, 4, 64, 96
    D = H * d
    g = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    ids = torch.randint(-1, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    table, dy = rnd(V, D), rnd(T, N).bfloat16()
    gq, gk = 1 + 0.1 * rnd(d), 1 + 0.1 * rnd(d)

    def chain():
        x = ops.embedding_forward(ids, table, scale=2.0, dtype=torch.bfloat16)
        q, k = ops.qk_norm_rope_forward(x.view(T, H, d), x.view(T, H, d), gq, gk, period=100)
        s = ops.stash8_pack(x)
        dw, db = ops.linear_wgrad_stash8(dy, s)
        dx = ops.gelu_backward_stash8(q.reshape(T, D), s)
        dq, dk, dgq, dgk = ops.qk_norm_rope_backward(dx.view(T, H, d), k, x.view(T, H, d), x.view(T, H, d), gq, gk, period=100)
        return x, q, k, dw, db, dx, dq, dk, dgq, dgk, ops.embedding_backward(ids, dq.view(T, D), V, scale=2.0)

    want = [t.clone() for t in chain()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = chain()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graphs = []
    for _ in range(2):   # two graphs, replayed in turn
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            res = chain()
        graphs.append((graph, res))
    for step in range(3):
        ids.copy_(torch.randint(-1, V, (T,), generator=g, device="cuda", dtype=torch.int32))
        table.copy_(rnd(V, D))
        for graph, res in graphs:
            graph.replay()
        want = [t.clone() for t in chain()]
        torch.cuda.synchronize()
        for _, res in graphs:
            assert all(torch.equal(a, b) for a, b in zip(want, res)), step


# ------------------------------------------------------------------------------------------------ more than 2^31 values

def at_the_ends(rows, shape, seed, n=500):
    """bf16 zeros [rows, *shape] with n random rows at each end."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.zeros(rows, *shape, device="cuda", dtype=torch.bfloat16)
    for part in (t[:n], t[-n:]):
        part.copy_(torch.randn(part.shape, generator=g, device="cuda"))
    return t


def test_embedding_of_more_than_2_31_values(ops):
    V, D = (1 << 21) + 5, 1032
    table = at_the_ends(V, (D,), 1)
    ids = torch.tensor([V - 1, 0, V, 1 << 20, V - 2, -1, V - 1], device="cuda", dtype=torch.int32)
    want = table[ids.long().clamp(0, V - 1)]
    want[[2, 5]] = 0
    assert torch.equal(ops.embedding_forward(ids, table), want)
    dy = table[-len(ids):].contiguous()
    del table
    out = ops.embedding_backward(ids, dy, V, out=torch.full((V, D), float("nan"), device="cuda"))
    f = dy.float()
    assert torch.equal(out[V - 1], f[0] + f[6]) and torch.equal(out[0], f[1]) and torch.equal(out[1 << 20], f[3])
    assert torch.equal(out[V - 2], f[4])
    out[[0, 1 << 20, V - 2, V - 1]] = 0
    assert not out.any()
    del out
    # as many tokens, nearly all of one id (a run through thousands of chunks): small whole numbers, so the sums are exact
    dy = torch.ones(V, D, device="cuda", dtype=torch.bfloat16)
    dy[-1], dy[-2] = 5, 7
    ids = torch.full((V,), 3, device="cuda", dtype=torch.int32)
    ids[-1], ids[0] = 7, -1
    got = ops.embedding_backward(ids, dy, 9)
    assert got[7].eq(5).all() and got[3].eq(V - 3 + 7).all() and got[[0, 1, 2, 4, 5, 6, 8]].eq(0).all()
    y = ops.embedding_forward(ids, got.bfloat16())
    assert y[-1].eq(5).all() and y[0].eq(0).all() and torch.equal(y[-2], got[3].bfloat16())


def test_qk_norm_rope_of_more_than_2_31_values(ops):
    T, H, d, n = (1 << 20) + 3, 16, 128, 500
    q, k = at_the_ends(T, (H, d), 2), at_the_ends(T, (1, d), 3)
    g = torch.Generator(device="cuda").manual_seed(4)
    gq, gk = 1 + 0.1 * torch.randn(2, d, generator=g, device="cuda")
    pos = torch.arange(T, device="cuda", dtype=torch.int32) * 3
    yq, yk = ops.qk_norm_rope_forward(q, k, gq, gk, positions=pos)
    ends = (slice(0, n), slice(T - n, T))
    for e in ends:
        a, b = ops.qk_norm_rope_forward(q[e], k[e], gq, gk, positions=pos[e])
        assert torch.equal(a, yq[e]) and torch.equal(b, yk[e])
    assert not yq[n:-n].any() and not yk[n:-n].any()
    dq, dk, dgq, dgk = ops.qk_norm_rope_backward(yq, yk, q, k, gq, gk, positions=pos, out=(yq.clone(), yk.clone()))
    sums = [0, 0]
    for e in ends:
        a, b, ga, gb = ops.qk_norm_rope_backward(yq[e], yk[e], q[e], k[e], gq, gk, positions=pos[e])
        assert torch.equal(a, dq[e]) and torch.equal(b, dk[e])
        sums = [sums[0] + ga.double(), sums[1] + gb.double()]
    # Both runs add the same terms du n in different orders, 2 n H of a place, u each.  dy is the result, so |du| is at most
    # the largest gain times the norm of n's pair (1 + 2^-8 for its rounding): the terms' magnitudes add up to at most that
    # gain times the pair's sum of n^2, which the gradients of the pair, sums of gain n^2 up to 2^-7 of it, give.
    for got, want, gain, heads in ((dgq, sums[0], gq, H), (dgk, sums[1], gk, 1)):
        terms = 1.05 * (want + want.roll(d // 2)) * gain.max() / gain.min()
        assert (want > 0).all() and ((got - want).abs() <= 2 * (2 * n * heads + 4) * u * terms).all()


def test_kept_activations_of_more_than_2_31_values(ops):
    rows, cin, cout, n = (1 << 21) + 67, 1032, 1040, 500
    x, dy = at_the_ends(rows, (cin,), 5), at_the_ends(rows, (cin,), 6)
    s = ops.stash8_pack(x)
    back = ops.stash8_unpack(s)
    dz = ops.gelu_backward_stash8(dy, s)
    assert not back[n:-n].any() and not dz[n:-n].any()
    for e in (slice(0, n), slice(rows - n, rows)):
        part = ops.stash8_pack(x[e])
        assert torch.equal(ops.stash8_unpack(part), back[e])
        assert torch.equal(ops.gelu_backward_stash8(dy[e], part), dz[e])
    del x, dy, dz
    dy = at_the_ends(rows, (cout,), 7)
    dw, db = ops.linear_wgrad_stash8(dy, s)
    a, b = (torch.cat([t[:n], t[-n:]]).double().cpu() for t in (dy, back))
    # 2 n terms that are not zero, each sum of them as in test_linear_wgrad_stash8
    inside(dw, (a.t() @ b).numpy(), (a.abs().t() @ b.abs()).numpy() * (4 * n + 4) * u)
    inside(db, a.sum(0).numpy(), a.abs().sum(0).numpy() * (2 * n + 4) * u)
