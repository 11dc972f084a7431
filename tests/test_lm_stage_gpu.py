"""GPU: stages with token embeddings, normalised and rotated queries and keys, and activations kept in 8 bits: against the oracle
(the bf16 bar of the other stages, 2e-2 per tensor), bit-identical however the round is run, and layer by layer against what
the single operators give."""
import numpy as np
import pytest

import harness
from asteroid_workloads import configs as C
from asteroid_workloads import gen

pytestmark = pytest.mark.gpu

TOL = 2e-2   # rel-L2 of bf16 stages


@pytest.fixture(scope="module")
def A():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2408_08015_amd as A
    return A


def small(**kw):
    a = dict(B=2, M=3, S=64, d=128, heads=2, ffn=256, nlayers=2, rows=300)
    a.update(kw)
    return C.lm_stage(**a)


def encoder(layers, B=2, M=2, S=32, d=128, seed=77):
    return C.StageConfig("layers", layers, B, M, (S, d), "bf16", "bsd", True, seed, init="normal0.02")


def check(cfg, inp=None):
    inp = inp or gen.make_inputs(cfg, randomize_affine=True)
    ora, _ = harness.run_oracle(cfg, inp, rounds=1)
    hip, _, _ = harness.run_hip(cfg, inp, rounds=1)
    h, o = hip[0], ora[0]
    assert harness.rel_l2(h["y"], o["y"]) <= TOL
    if cfg.needs_input_grad:
        assert harness.rel_l2(h["dx"], o["dx"]) <= TOL
    rms = float(np.sqrt(np.mean(np.square(o["G"]))))
    errs = [(n,) + harness.grad_error(a, b, rms) for (n, a), (_, b) in
            zip(harness.split_params(cfg.layers, h["G"]), harness.split_params(cfg.layers, o["G"]))]
    worst = max(errs, key=lambda t: t[1])
    print(cfg.name, "y", harness.rel_l2(h["y"], o["y"]), "worst G", worst, "floored", [n for n, _, f in errs if f])
    assert worst[1] <= TOL, errs
    for (n, a), (_, b) in zip(harness.split_params(cfg.layers, h["W"]), harness.split_params(cfg.layers, o["W"])):
        assert harness.rel_l2(a, b) <= TOL, n
    return h


@pytest.mark.parametrize("keep8", [False, True])
@pytest.mark.parametrize("kw", [dict(), dict(B=1, M=2, S=32, d=512, heads=8, ffn=2048, nlayers=1, rows=5000),
                                dict(B=3, M=2, S=32, d=512, heads=8, ffn=2048, nlayers=2, rows=500)])   # one launch for all kept inputs
def test_language_model_stage(A, kw, keep8):
    check(small(keep8=keep8, **kw))


@pytest.mark.parametrize("mha", [dict(qk_norm=1, eps=1e-6), dict(qk_norm=1, rotary=32, theta=500, eps=1e-6),
                                 dict(qk_norm=1, rotary=64, theta=10000, interleaved=1, eps=1e-5), dict(keep8=1),
                                 dict(qk_norm=1, rotary=64, theta=10000, eps=1e-6, keep8=1)])
def test_attention_variants(A, mha):
    L = [C.simple("res_begin"), dict(kind="mha", d=128, heads=2, **mha), C.simple("res_add"), dict(kind="layernorm", d=128, eps=1e-5)]
    check(encoder(L))
    check(encoder(L[1:2]))     # alone: the layer's input is the stage's, its output the caller's


@pytest.mark.parametrize("layers", [
    lambda: [dict(C.linear(128, 64), keep8=1)],
    lambda: [dict(C.linear(128, 200, bias=False), keep8=1), dict(kind="layernorm", d=200, eps=1e-5)],
    lambda: [C.linear(128, 64), dict(C.simple("gelu"), keep8=1)],                                     # the stage's output
    lambda: [C.linear(128, 64), dict(C.simple("gelu"), keep8=1), dict(C.linear(64, 96), keep8=1)],
    lambda: [dict(kind="layernorm", d=128, eps=1e-5), dict(C.simple("gelu"), keep8=1), C.linear(128, 64)],   # GELU of its own
    lambda: [C.linear(128, 64), C.simple("relu"), dict(C.linear(64, 64), keep8=1)],       # ReLU's backward needs the input too
    lambda: [C.simple("res_begin"), dict(C.linear(128, 128), keep8=1), C.simple("res_swap"), C.linear(128, 128), C.simple("res_add")],
    lambda: [C.simple("res_begin"), C.linear(128, 128), C.simple("res_swap"), dict(C.linear(128, 128), keep8=1), C.simple("res_add")],
    lambda: [C.linear(128, 96), C.simple("res_begin"), dict(C.linear(96, 96), keep8=1), C.simple("res_swap"),
             dict(C.linear(96, 96), keep8=1), C.simple("res_add")],      # both branches keep the block's input
    lambda: [C.simple("res_begin"), dict(C.linear(128, 128), keep8=1), C.simple("gelu"), dict(C.linear(128, 128), keep8=1), C.simple("res_add")],
])
def test_layers_with_kept_inputs(A, layers):
    check(encoder(layers()))
    check(encoder(layers(), B=1, M=1, S=1))
    check(encoder(layers(), B=3, M=1, S=17))


@pytest.mark.parametrize("cin,c,hw", [(16, 24, 9), (8, 40, 12), (32, 64, 7)])
def test_a_kept_gelu_between_convolutions(A, cin, c, hw):
    """Images: a row is a pixel's channels."""
    kept = dict(C.simple("gelu"), keep8=1)
    for layers in ([C.conv(cin, c, 3, 1, 1, bias=True), kept, C.conv(c, cin, 3, 1, 1, bias=True)], [kept, C.conv(cin, c, 3, 1, 1, bias=True)]):
        check(C.StageConfig("images", layers, 3, 2, (cin, hw, hw), "bf16", "nhwc", True, 78, init="normal0.02"))


@pytest.mark.parametrize("kw", [dict(), dict(B=1, S=32, d=512, heads=8, ffn=2048, rows=100)])
@pytest.mark.parametrize("K", [1, 2, 3])
def test_bit_identical_however_it_runs(A, K, kw):
    cfg = small(**kw)
    inp = gen.make_inputs(cfg, randomize_affine=True)
    ref, _, mem = harness.run_hip(cfg, inp, K=1, rounds=2)
    assert mem[3] <= 32 << 20
    for kw in (dict(), dict(static_backward=True), dict(forward_stream=True), dict(forward_stream=True, static_backward=True)):
        got, _, _ = harness.run_hip(cfg, inp, K=K, rounds=2, **kw)
        for r in range(2):
            for k in ("y", "G", "W"):
                assert np.array_equal(ref[r][k], got[r][k]), (K, kw, r, k)


@pytest.mark.parametrize("layers", [
    lambda: [dict(C.linear(512, 512), keep8=1), dict(C.linear(512, 512), keep8=1)],
    lambda: [dict(C.linear(512, 512), keep8=1), dict(C.simple("gelu"), keep8=1), dict(C.linear(512, 512), keep8=1)],
])
def test_static_backward_of_a_stage_whose_shares_were_brought_down(A, layers):
    cfg = encoder(layers(), B=32, M=2, S=128, d=512)
    inp = gen.make_inputs(cfg, randomize_affine=True)
    ref, _, _ = harness.run_hip(cfg, inp, K=1, rounds=2)
    for kw in (dict(), dict(forward_stream=True)):
        got, _, _ = harness.run_hip(cfg, inp, K=2, rounds=2, static_backward=True, **kw)
        for r in range(2):
            for k in ("y", "dx", "G", "W"):
                assert np.array_equal(ref[r][k], got[r][k]), (kw, r, k)
    check(cfg, inp)


@pytest.mark.parametrize("layers", [
    # both branches of a block, products without a bias, and a GELU in front of a kept product and behind one
    lambda: [dict(C.linear(512, 768), keep8=1), C.simple("res_begin"), dict(C.linear(768, 768), keep8=1), C.simple("gelu"),
             dict(C.linear(768, 768, bias=False), keep8=1), C.simple("res_swap"), dict(C.linear(768, 768), keep8=1), C.simple("res_add"),
             dict(kind="layernorm", d=768, eps=1e-5), dict(C.linear(768, 1024), keep8=1), dict(C.simple("gelu"), keep8=1),
             dict(C.linear(1024, 520), keep8=1), dict(kind="layernorm", d=520, eps=1e-5)],
    # the last product's upstream gradient is the caller's: a product of its own beside the launch
    lambda: [dict(C.linear(512, 1536), keep8=1), C.simple("relu"), dict(C.linear(1536, 1000), keep8=1), C.simple("res_begin"),
             dict(C.linear(1000, 1000), keep8=1), C.simple("res_add"), dict(C.linear(1000, 512), keep8=1)],
])
def test_one_launch_for_kept_inputs(A, layers):
    """More than 192 tiles of 128 x 128, so that the weight gradients are one launch; rows that end inside a step."""
    cfg = encoder(layers(), B=3, M=2, S=37, d=512)
    inp = gen.make_inputs(cfg, randomize_affine=True)
    check(cfg, inp)
    ref, _, _ = harness.run_hip(cfg, inp, K=1, rounds=2)
    for kw in (dict(), dict(static_backward=True), dict(forward_stream=True)):
        got, _, _ = harness.run_hip(cfg, inp, K=2, rounds=2, **kw)
        for r in range(2):
            for k in ("y", "dx", "G", "W"):
                assert np.array_equal(ref[r][k], got[r][k]), (kw, r, k)
    import torch
    st = A.Stage(cfg.layers, cfg.B, 1, 1, cfg.in_shape, cfg.dtype, cfg.layout, True, stream=torch.cuda.current_stream().cuda_stream)
    x, dy = torch.from_numpy(inp["x"][:3]).cuda().bfloat16(), torch.from_numpy(inp["dy"][:3]).cuda().bfloat16()
    st.forward(0, x, None, torch.zeros_like(dy))
    st.profile_begin()
    st.backward(0, dy, torch.zeros_like(x))
    assert st.profile_end()["stash8_wgrad_group_kernel"][0] == 1
    st.close()


def test_results_over_an_input_that_is_kept_in_8_bits_only(A):
    """The caller's x is read as it lies: y may take its place where x has been read by then, and is refused where not."""
    import torch
    k = dict(C.linear(128, 128), keep8=1)
    for layers, ok in (([k], False), ([C.simple("res_begin"), k, C.simple("res_add")], False),
                       ([C.simple("res_begin"), k, C.simple("gelu"), k, C.simple("res_add")], False),
                       ([k, C.simple("gelu")], False), ([k, dict(kind="layernorm", d=128, eps=1e-5)], True), ([k, k], True),
                       ([k, C.simple("relu")], True), ([C.linear(128, 128)], True)):
        cfg = encoder(layers, M=1)
        inp = gen.make_inputs(cfg, randomize_affine=True)
        ref, _, _ = harness.run_hip(cfg, inp, rounds=1)
        st = A.Stage(cfg.layers, cfg.B, 1, 1, cfg.in_shape, cfg.dtype, cfg.layout, True, stream=torch.cuda.current_stream().cuda_stream)
        st.set_params(inp["params"])
        room = torch.zeros(3 * inp["x"].size, device="cuda", dtype=torch.bfloat16)
        n = inp["x"].size
        x = room[n:2 * n].view(inp["x"].shape)
        x.copy_(torch.from_numpy(inp["x"]))
        dy, dx = torch.from_numpy(inp["dy"]).cuda().bfloat16(), torch.zeros_like(x)
        if ok:
            st.forward(0, x, None, x)
            y = x
        else:
            for at in (n, 1024, 2 * n - 1024):
                with pytest.raises(A.AsteroidError, match="overlap") as e:
                    st.forward(0, x, None, room[at:at + n])
                assert e.value.status == -1
            y = room[2 * n:].view(x.shape)
            st.forward(0, x, None, y)
        st.backward(0, dy, dx)
        torch.cuda.synchronize()
        assert np.array_equal(y.float().cpu().numpy(), ref[0]["y"]) and np.array_equal(dx.float().cpu().numpy(), ref[0]["dx"])
        assert np.array_equal(st.get_grads(), ref[0]["G"])
        st.close()


def test_keeping_changes_nothing_but_the_gradients_it_forms(A):
    """Forward pass and input gradient of dense layers are those of the stage without it, bit for bit; the flagged weight
    gradients are the operator's on the same tensors."""
    import torch
    from paper_2408_08015_amd import ops
    L = lambda k: [dict(C.linear(128, 96), keep8=k), dict(kind="layernorm", d=96, eps=1e-5), dict(C.linear(96, 40), keep8=k)]
    a, b = encoder(L(0), M=1), encoder(L(1), M=1)
    inp = gen.make_inputs(a, randomize_affine=True)
    x0, _, m0 = harness.run_hip(a, inp, rounds=1)
    x1, _, m1 = harness.run_hip(b, inp, rounds=1)
    assert np.array_equal(x0[0]["y"], x1[0]["y"]) and np.array_equal(x0[0]["dx"], x1[0]["dx"])
    assert m1[2] < m0[2]
    G = dict(harness.split_params(b.layers, x1[0]["G"]))
    dy = torch.from_numpy(inp["dy"]).cuda().bfloat16().reshape(-1, 40)
    # the last layer's input, as the forward pass of the first two layers gives it
    c = encoder(L(0)[:2], M=1)
    n = gen.num_params(c.layers)
    x2, _, _ = harness.run_hip(c, dict(x=inp["x"], dy=np.zeros((2, 32, 96), np.float32), params=inp["params"][:n]), rounds=1)
    h = torch.from_numpy(x2[0]["y"]).cuda().bfloat16().reshape(-1, 96)
    dw, db = ops.linear_wgrad_stash8(dy, ops.stash8_pack(h))
    assert np.array_equal(dw.cpu().numpy().ravel(), G["L2.weight"]) and np.array_equal(db.cpu().numpy(), G["L2.bias"])


def test_embedding_gradient_is_exact_up_to_its_sums(A):
    """A stage that is the embedding alone: y rounded once, G the sums of dy over every id's tokens, over the micro-batches."""
    cfg = C.StageConfig("embedding", [dict(kind="embedding", rows=50, d=64, scale=8.0)], 4, 3, (16, 1), "bf16", "bsd", False, 5)
    inp = gen.make_inputs(cfg)
    ora, _ = harness.run_oracle(cfg, inp, rounds=1)
    hip, _, _ = harness.run_hip(cfg, inp, rounds=1)
    assert np.array_equal(hip[0]["y"], ora[0]["y"].astype(np.float32))
    terms = np.zeros((50, 64))
    for i, g in zip(inp["x"].ravel(), inp["dy"].reshape(-1, 64)):
        if i >= 0:
            terms[i] += abs(8.0 * g)
    n = 4 * 16 * 3 + 4
    assert (abs(hip[0]["G"] - ora[0]["G"]).reshape(50, 64) <= n * 2.0 ** -24 * terms).all()
    unseen = ~np.isin(np.arange(50), inp["x"])
    assert not hip[0]["G"].reshape(50, 64)[unseen].any()


def test_a_round_as_a_graph(A):
    """A whole round recorded and replayed with new ids in between; every replay against the eager round."""
    import torch
    cfg = small(M=2)
    inp = gen.make_inputs(cfg, randomize_affine=True)
    B, M = cfg.B, cfg.M
    side = torch.cuda.Stream()
    runs = []
    for _ in range(2):      # one stage that is recorded, one that runs the same rounds eagerly
        st = A.Stage(cfg.layers, B, M, 1, cfg.in_shape, cfg.dtype, cfg.layout, False, stream=side.cuda_stream)
        st.set_params(inp["params"])
        xs = [torch.from_numpy(inp["x"][m * B:(m + 1) * B].copy()).cuda() for m in range(M)]
        dys = [torch.from_numpy(inp["dy"][m * B:(m + 1) * B].copy()).cuda().bfloat16() for m in range(M)]
        runs.append((st, xs, dys, [torch.zeros_like(d) for d in dys]))

    def rnd(run):
        st, xs, dys, ys = run
        for m in range(M):
            st.forward(m, xs[m], None, ys[m])
            st.backward(m, dys[m])
        st.step(0.01, 0.9)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            rnd(runs[0])
    r = np.random.Generator(np.random.PCG64(9))
    for step in range(3):
        ids = [torch.from_numpy(r.integers(-1, cfg.layers[0]["rows"], (B, cfg.in_shape[0])).astype(np.int32)) for _ in range(M)]
        for run in runs:
            for m in range(M):
                run[1][m].copy_(ids[m])
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
            rnd(runs[1])
        torch.cuda.synchronize()
        for a, b in zip(runs[0][3], runs[1][3]):
            assert torch.equal(a, b), step
        assert np.array_equal(runs[0][0].get_params(), runs[1][0].get_params()), step
    for run in runs:
        run[0].close()


def test_profiler_times_the_embedding(A):
    from paper_2408_08015_amd import profiler
    cfg = small(nlayers=1)
    for lo, hi in profiler.split_units(cfg.layers)[:2]:
        tf, tb = profiler.time_unit(cfg.layers[lo:hi], cfg.in_shape if lo == 0 else (64, 128), 2, "bf16", "bsd", lo > 0, reps=2, warmup=1)
        assert tf > 0 and tb > 0
