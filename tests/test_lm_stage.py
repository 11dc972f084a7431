"""CPU: stages with token embeddings, normalised and rotated queries and keys, and activations kept in 8 bits - the oracle
against differences, the plan's byte counts and refusals."""
import numpy as np
import pytest

import paper_2408_08015_amd as A
from asteroid_workloads import configs as C
from asteroid_workloads import gen
from oracle import OracleStage


def plan(cfg, K=1, **kw):
    a = dict(layers=cfg.layers, in_shape=cfg.in_shape, dtype=cfg.dtype, layout=cfg.layout, grad=cfg.needs_input_grad)
    a.update(kw)
    return A.plan_memory(a["layers"], cfg.B, cfg.M, K, a["in_shape"], a["dtype"], a["layout"], a["grad"])


def small(**kw):
    a = dict(B=2, M=2, S=32, d=128, heads=2, ffn=256, nlayers=2, rows=300)
    a.update(kw)
    return C.lm_stage(**a)


def test_oracle_gradients_against_differences():
    cfg = small(B=1, M=1, S=8, d=16, heads=2, ffn=24, nlayers=1, rows=11, keep8=False)
    inp = gen.make_inputs(cfg, randomize_affine=True)
    assert inp["x"].dtype == np.int32 and inp["x"].shape == (1, 8)
    st = OracleStage(cfg.layers, 1, 1, cfg.in_shape, cfg.layout, False)
    r = np.random.Generator(np.random.PCG64(1))
    w = inp["params"].astype(np.float64) + 0.2 * r.normal(size=inp["params"].size)
    dy = r.normal(size=inp["dy"].shape)

    def f(v):
        st.set_params(v)
        y, _ = st.forward(0, inp["x"])
        st.stash.clear()
        return (y * dy).sum()

    st.set_params(w)
    st.forward(0, inp["x"])
    st.backward(0, dy)
    G, h = st.G.copy(), 1e-6
    names = {s[1] for s in gen.param_specs(cfg.layers)}
    assert {"table", "q_gain", "k_gain"} <= names and gen.num_params(cfg.layers) == st.nparams
    for i in r.choice(st.nparams, 150, replace=False).tolist() + list(range(st.nparams - 20, st.nparams)):
        e = np.zeros_like(w)
        e[i] = h
        assert abs((f(w + e) - f(w - e)) / (2 * h) - G[i]) < 1e-5 * max(1.0, abs(G[i])), i


def test_kept_activations_leave_the_stash():
    """Per token and layer of width d, in bytes: what is kept in 8 bits takes 33/32 instead of 2."""
    full, kept = small(keep8=False), small(keep8=True)
    m0, m1 = plan(full), plan(kept)
    tokens, d, ffn, layers = 2 * 32, 128, 256, 2
    assert m0[0] == m1[0] and m0[1] == m1[1]
    saved = layers * tokens * (2 * d + 2 * ffn) * (2 - 33 / 32)   # inputs of both blocks, GELU's input and output
    assert abs((m0[2] - m1[2]) - saved) <= 256 * 8 * layers      # buffers are laid out in steps of 256 bytes
    assert plan(kept, K=2) == m1
    deep, one = plan(small(nlayers=6, keep8=True)), plan(small(nlayers=1, keep8=True))
    assert deep[2] - m1[2] == 4 * (m1[2] - one[2])


def test_a_shortcut_branch_keeps_the_blocks_input():
    """The input of a shortcut branch is the block's: its 8-bit form has room of its own, once."""
    L = lambda a, b: [dict(C.linear(64, 64), keep8=0), C.simple("res_begin"), dict(C.linear(64, 64), keep8=a), C.simple("res_swap"),
                      dict(C.linear(64, 64), keep8=b), C.simple("res_add")]
    cfg = small()
    act = [plan(cfg, layers=L(a, b), in_shape=(32, 64), grad=True)[2] for a, b in ((0, 0), (0, 1), (1, 0), (1, 1))]
    room = 2 * 32 * 64 * 33 // 32
    assert act[1] == act[2] == act[3] and room <= act[1] - act[0] <= room + 256


@pytest.mark.parametrize("d,n,B,act", [(512, 2, 32, 0), (512, 3, 24, 0), (256, 4, 32, 0), (1024, 2, 8, 0), (512, 2, 32, 1), (768, 3, 8, 1), (448, 2, 36, 0)])
def test_a_stage_that_fits_the_static_array_fits_it_with_kept_inputs(d, n, B, act):
    """What only a forward pass uses does not count, and the weight gradients take fewer shares where theirs would not fit."""
    L = lambda k: sum([[dict(C.linear(d, d), keep8=k)] + ([dict(C.simple("gelu"), keep8=k)] if act else []) for _ in range(n)], [])
    ws = [A.plan_memory(L(k), B, 1, 1, (128, d), "bf16", "bsd", True)[3] for k in (0, 1)]
    # tensors of a forward pass that are alive together: a layer's input and output, and the value in front of a GELU
    passing = B * 128 * d * 2 * ((2 if act or n > 2 else 1) + act * (n > 2))
    assert ws[0] <= 32 << 20 and ws[1] - passing <= 32 << 20


def test_the_profiler_cuts_behind_the_embedding():
    from paper_2408_08015_amd import profiler
    cfg = small(nlayers=1)
    units = profiler.split_units(cfg.layers)
    assert units[0] == (0, 1) and len(units) == 3
    assert profiler._out_shape(cfg.layers[:1], cfg.in_shape) == (32, 128)


def test_token_ids_are_int32():
    """An int64 tensor, torch's own integer type, would be read as pairs of ids."""
    import torch
    cfg = small()
    st = A.Stage.__new__(A.Stage)     # (checked before anything is asked of the library)
    st.layers, st.B, st.in_shape, st.lib = cfg.layers, cfg.B, cfg.in_shape, None
    for ids in (torch.zeros(2, 32, dtype=torch.int64), torch.zeros(2, 32), torch.zeros(2, 31, dtype=torch.int32),
                torch.zeros(2, 64, dtype=torch.int32)[:, ::2], torch.zeros(4, 32, dtype=torch.int32)):
        with pytest.raises(ValueError, match="int32"):
            st.forward(0, ids)


def test_refusals():
    cfg = small(nlayers=1)

    def no(layers=None, status=-1, **kw):
        with pytest.raises(A.AsteroidError) as e:
            plan(cfg, layers=cfg.layers if layers is None else layers, **kw)
        assert e.value.status == status, e.value

    def with_layer(i, **kw):
        L = [dict(l) for l in cfg.layers]
        L[i].update(kw)
        return L

    no(grad=True)                                        # ids have no gradient
    no(in_shape=(32, 128))                               # one id a position
    no(dtype="f32", status=-5)
    no(layout="nhwc", in_shape=(1, 32, 1), status=-5)
    no([dict(kind="layernorm", d=128, eps=1e-5)] + cfg.layers, in_shape=(32, 128))   # not the first layer
    for bad in (dict(rows=0), dict(rows=-1), dict(rows=2**31 - 1), dict(d=4), dict(d=132), dict(scale=float("nan"))):
        no(with_layer(0, **bad))
    mha = 2
    for bad in (dict(qk_norm=2), dict(rotary=63), dict(rotary=66), dict(rotary=-2), dict(theta=0), dict(eps=0.0), dict(eps=-1.0),
                dict(eps=float("nan")), dict(interleaved=2), dict(keep8=3)):
        no(with_layer(mha, **bad))
    assert plan(cfg, layers=with_layer(mha, rotary=0, theta=0))      # norms alone need no theta
    no(with_layer(6, keep8=2))
    no(with_layer(7, keep8=-1))
    L = [dict(kind="global_avgpool"), dict(C.linear(8, 4), keep8=1)]
    no(L, status=-5, dtype="f32", layout="nchw", in_shape=(8, 4, 4), grad=True)


def test_numbers_that_a_description_has_no_room_for():
    cfg = small(nlayers=1)

    def with_layer(i, **kw):
        return plan(cfg, layers=[dict(l, **kw) if j == i else l for j, l in enumerate(cfg.layers)])

    mha = 2
    for i, bad in ((0, dict(rows=2**32 + 300)), (0, dict(d=2**32 + 128)), (mha, dict(theta=2**32 + 10000)), (mha, dict(theta=0.5)),
                   (mha, dict(theta=10000.5)), (mha, dict(rotary=2**32))):
        with pytest.raises(ValueError, match="32 bits"):
            with_layer(i, **bad)
    assert with_layer(mha, theta=10000.0) == plan(cfg)


def plan_described(arr, cfg, in_shape, needs_input_grad=1):
    """asteroid_stage_plan_memory of C descriptions: its status, and the four byte counts."""
    import ctypes
    from paper_2408_08015_amd import binding as Bd
    lib = A.load_library()
    out = [ctypes.c_size_t() for _ in range(4)]
    c = Bd._marshal_cfg(cfg.B, cfg.M, 1, in_shape, cfg.dtype, cfg.layout, needs_input_grad)
    return lib.asteroid_stage_plan_memory(arr, len(arr), ctypes.byref(c), *[ctypes.byref(o) for o in out]), [o.value for o in out]


@pytest.mark.parametrize("junk", [1, 2, -1, 1 << 30])
def test_descriptions_that_leave_the_entries_behind_their_own_unset(junk):
    """p beyond what a kind had, and eps of an attention, were never looked at: a description that leaves them as they come means
    the plain layer still.  With AST_LAYER_MORE they count."""
    from paper_2408_08015_amd import binding as Bd
    cfg = C.cfg5(B=2, M=2, S=32, d=128, heads=2, ffn=256, nlayers=1)
    layers = cfg.layers + [dict(kind="gelu")]
    own = {"linear": 3, "mha": 2, "gelu": 0}
    zeroed = plan_described(Bd._marshal_layers(layers), cfg, cfg.in_shape)
    arr = Bd._marshal_layers(layers)
    for a, L in zip(arr, layers):
        for i in range(own.get(L["kind"], 8), 8):
            a.p[i] = junk
        if L["kind"] in own:
            a.eps = float("nan")
    assert zeroed[0] == 0 and plan_described(arr, cfg, cfg.in_shape) == zeroed
    for a, L in zip(arr, layers):   # counted: no layer takes these
        b = Bd._marshal_layers(layers)
        if L["kind"] in own and junk != 1 or L["kind"] == "mha":
            i = [x is L for x in layers].index(True)
            b[i] = a
            b[i].kind += Bd.LAYER_MORE
            assert plan_described(b, cfg, cfg.in_shape)[0] == -1, L
    b = Bd._marshal_layers(layers)
    b[[L["kind"] for L in layers].index("layernorm")].kind += Bd.LAYER_MORE
    assert plan_described(b, cfg, cfg.in_shape)[0] == -1
    kept = Bd._marshal_layers([dict(L, keep8=1) for L in layers])
    st, mem = plan_described(kept, cfg, cfg.in_shape)
    assert st == 0 and mem[2] < zeroed[1][2]


def test_what_was_planned_before_is_planned_the_same():
    """Layers without the new entries keep their byte counts."""
    cfg = C.cfg5(B=2, M=2, S=32, d=128, heads=2, ffn=256, nlayers=1)
    mod, opt, act, _ = plan(cfg)
    assert opt == 4 * gen.num_params(cfg.layers)
    t = 2 * 32
    # x, qkv, o, the sums and outputs around both LayerNorms, z, h in bf16; log-sum-exp, LayerNorm statistics
    want = t * 2 * (128 + 3 * 128 + 128 + 128 + 128 + 256 + 256 + 128) + 2 * 2 * 32 * 4 + 2 * 2 * t * 4
    assert want <= act <= want + 256 * 16
