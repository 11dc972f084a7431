"""More operators of a language model's pipeline stages that are timed, and what they compute in plain form.

norm        RMS norm between two blocks with the residual's addition; forward also with the result in 8 bits (blocks of
            32 channels with one power-of-two scale), and backward with the gain's gradient.
recurrence  the gated linear recurrence h = sigmoid(f) h' + (1 - sigmoid(f)) z, y = h swish(o), over sequences of
            tokens: one token of each (step), a forward pass (fwd), a forward and a backward pass (train).
distill     the loss of the last stage from a teacher's top logits, mixed with that of a label: the loss alone (fwd), the
            gradient from the statistics that the forward pass left (bwd), loss and gradient at once (train).

A case names the operator (`op`), its direction or use (`dir`) and the sizes.
"""
import math

import torch

own = False

BLOCK = 32   # channels of a token that share a scale
EPS = 1e-6


# ---------------------------------------------------------------------------------------------- cases

def _norm(d, T, C, dtype="bf16", stream="bf16", residual=True, keep8=False):
    return dict(op="norm", dir=d, T=T, C=C, dtype=dtype, stream=stream, residual=residual, keep8=keep8)


def _recurrence(d, T, C, period=0, lengths=0, dtype="bf16", gate=True, state=False, packed=True):
    """Sequences of `period` tokens, or `lengths` of them that share the tokens unevenly."""
    return dict(op="recurrence", dir=d, T=T, C=C, period=period, lengths=lengths, dtype=dtype, gate=gate, state=state, packed=packed)


def _distill(d, T, V, K, dtype="bf16", teacher="bf16", tau=2.0, mix=0.0, room=0):
    return dict(op="distill", dir=d, T=T, V=V, K=K, dtype=dtype, teacher=teacher, tau=tau, mix=mix, room=room)


def listed():
    return [
        # One sequence of the transformer stage (128 tokens of 512), as a profiler's smallest call: latency alone.
        dict(_norm("fwd", 128, 512), name="norm_fwd_one_sequence"),
        # A large micro-batch in front of a wide layer: an fp32 residual stream, the result also kept for the weight gradient.
        dict(_norm("fwd", 16384, 2048, stream="f32", keep8=True), name="norm_fwd_kept"),
        # One micro-batch of the transformer stage, backward: 32 sequences of 128 tokens.
        dict(_norm("bwd", 4096, 512), name="norm_bwd_stage"),
        # Rows that divide by nothing, bf16 layers on an fp32 stream.
        dict(_norm("bwd", 12289, 1501, stream="f32"), name="norm_bwd_ragged"),
        # One more token of each of 64 texts: what a sampled answer takes per token.
        dict(_recurrence("step", 64, 1024, period=1, state=True), name="recurrence_step"),
        # A long text as one sequence: a chain of tokens through the whole call.
        dict(_recurrence("fwd", 65536, 1024, period=65536), name="recurrence_fwd_long"),
        # One micro-batch of the transformer stage's size, forward and backward.
        dict(_recurrence("train", 4096, 512, period=128), name="recurrence_train_stage"),
        # Texts of any length one behind the other, fp32, an odd number of channels, states carried in and out.
        dict(_recurrence("train", 20011, 777, lengths=61, dtype="f32", state=True, packed=False), name="recurrence_train_ragged_f32"),
        # The loss of one sequence over the vocabulary of the language-model stage.
        dict(_distill("fwd", 128, 32768, 32), name="distill_fwd_one_sequence"),
        # The gradient of a micro-batch in a backward pass of its own, an odd vocabulary in padded rows, with labels.
        dict(_distill("bwd", 2001, 50021, 100, tau=1.5, mix=0.3, room=27), name="distill_bwd_padded"),
        # Loss and gradient of a micro-batch of the language-model stage, fp32 logits.
        dict(_distill("train", 4096, 32768, 64, dtype="f32", teacher="f32", tau=1.0), name="distill_train_stage_f32"),
        # A large vocabulary with labels: two temperatures in one pass, logits that fill a good part of a cache.
        dict(_distill("train", 4096, 131072, 64, mix=0.5), name="distill_train_large_vocabulary"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm_fwd", "norm_bwd", "step", "fwd", "train", "train", "distill_fwd", "distill_bwd", "distill_train"])
    if kind.startswith("norm"):
        C = rng.choice([_log(rng, 8, 8192), 8 * _log(rng, 4, 1024)])
        dtype, stream = rng.choice([("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
        residual = rng.random() < 0.8 or stream != dtype
        return _norm(kind[-3:], _log(rng, 1, min(65536, (1 << 25) // C)), C, dtype=dtype, stream=stream, residual=residual,
                     keep8=kind == "norm_fwd" and rng.random() < 0.5)
    if kind in ("step", "fwd", "train"):
        C = rng.choice([_log(rng, 32, 4096), 32 * _log(rng, 1, 128)])
        how = dict(dtype=rng.choice(["f32", "bf16", "bf16"]), gate=rng.random() < 0.7, state=rng.random() < 0.5, packed=rng.random() < 0.6)
        if kind == "step":
            how["state"] = True
            return _recurrence("step", _log(rng, 1, 512), C, period=1, **how)
        T = _log(rng, 1, min(65536, (1 << 25) // C))
        if rng.random() < 0.5:
            return _recurrence(kind, T, C, lengths=_log(rng, 1, max(2, T // 8)), **how)
        return _recurrence(kind, T, C, period=rng.choice([T, max(1, T // _log(rng, 1, 64)), _log(rng, 1, T + 1)]), **how)
    V = rng.choice([_log(rng, 500, 131072), 64 * _log(rng, 8, 2048)])
    T = _log(rng, 1, min(8192, (1 << 28) // V))
    return _distill(kind[8:], T, V, _log(rng, 1, 256), dtype=rng.choice(["f32", "bf16", "bf16"]), teacher=rng.choice(["f32", "bf16"]),
                    tau=rng.choice([1.0, 1.0, 2.0, 0.7, 4.0]), mix=rng.choice([0.0, 0.0, 0.5, 0.1]), room=rng.choice([0, 0, -V % 64]))


# ---------------------------------------------------------------------------------------------- inputs

def _dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _stream(g, T, C):
    """A residual stream: channels of different sizes, a few of them much larger."""
    x = _randn(g, T, C)
    x *= torch.exp(0.5 * _randn(g, C))
    x[:, ::97] *= 12.0
    return x


def _rows(g, T, V, room, dtype, scale):
    """A matrix [T, V] in rows of V + room."""
    t = torch.zeros(T, V + room, device="cuda", dtype=dtype)[:, :V]
    t.copy_(_randn(g, T, V).mul_(scale))
    return t


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    T = case["T"]
    if case["op"] == "norm":
        C, dt, st = case["C"], _dt(case["dtype"]), _dt(case["stream"])
        s["gain"] = 1.0 + 0.2 * _randn(g, C)
        if case["dir"] == "fwd":
            s["x"] = _randn(g, T, C).to(dt)
            s["r"] = _stream(g, T, C).to(st) if case["residual"] else None
        else:
            s["s"] = _stream(g, T, C).to(st)
            s["dy"] = (1e-2 * _randn(g, T, C)).to(dt)
            s["dsum"] = (1e-2 * _randn(g, T, C)).to(st) if case["residual"] else None
    elif case["op"] == "recurrence":
        C, dt, parts = case["C"], _dt(case["dtype"]), 3 if case["gate"] else 2
        p = _randn(g, T, parts, C)   # the projection: forget gate, candidate, output gate
        p[:, 0] = 1.5 * p[:, 0] + torch.linspace(0.0, 5.0, C, device="cuda")   # channels that keep for one token up to some hundreds
        p = p.to(dt)
        part = [p[:, i] if case["packed"] else p[:, i].contiguous() for i in range(parts)]
        s["f"], s["z"], s["o"] = part[0], part[1], part[2] if case["gate"] else None
        s["offsets"] = None
        n = -(-T // case["period"]) if case["period"] else case["lengths"]
        if case["lengths"]:   # lengths of zero among them
            cut = torch.randint(0, T + 1, (n - 1,), generator=g, device="cuda").sort().values
            s["offsets"] = torch.cat((cut.new_zeros(1), cut, cut.new_full((1,), T))).to(torch.int32)
        s["n"] = n
        s["state"] = _randn(g, n, C) if case["state"] else None
        if case["dir"] == "train":
            s["dy"] = (1e-2 * _randn(g, T, C)).to(dt)
            s["dfinal"] = 1e-2 * _randn(g, n, C) if case["state"] else None
    else:
        V, K = case["V"], case["K"]
        z = _rows(g, T, V, case["room"], torch.float32, 2.5)
        # the teacher's largest logits in falling order, at places that the student has begun to favour
        first = torch.randint(0, V, (T, 1), generator=g, device="cuda")
        ids = (first + torch.arange(K, device="cuda") * (V // K)) % V
        t = (12.0 - 8.0 * torch.rand(T, K, generator=g, device="cuda")).sort(1, descending=True).values
        z.scatter_add_(1, ids, 0.6 * t)
        some = torch.randint(1, K + 1, (T, 1), generator=g, device="cuda")   # a tenth of the rows have fewer entries
        few = torch.rand(T, 1, generator=g, device="cuda") < 0.1
        ids = torch.where(few & (torch.arange(K, device="cuda") >= some), torch.full_like(ids, -1), ids)
        s["ids"], s["t"] = ids.to(torch.int32).contiguous(), t.to(_dt(case["teacher"]))
        s["z"] = torch.empty(T, V + case["room"], device="cuda", dtype=_dt(case["dtype"]))[:, :V].copy_(z)
        s["labels"] = None
        if case["mix"]:
            s["labels"] = torch.where(torch.rand(T, generator=g, device="cuda") < 0.5, ids[:, 0],
                                      torch.randint(0, V, (T,), generator=g, device="cuda")).to(torch.int32)
        w = (torch.rand(T, generator=g, device="cuda") >= 0.05).float()   # tokens that do not count
        s["dloss"] = w / w.sum().clamp_(min=1.0)
        if case["dir"] == "bwd":   # what the forward pass left of every row: its largest logit, and the sums
            f = s["z"].float()
            top = f.amax(1, keepdim=True)
            s["stats"] = torch.cat((top, torch.exp((f - top) / case["tau"]).sum(1, keepdim=True),
                                    torch.exp(f - top).sum(1, keepdim=True)), 1)
    return s


# ---------------------------------------------------------------------------------------------- one pass

def run(state):
    s = state
    if own:
        return _run_own(s)
    if s["op"] == "norm":
        return _norm_fwd_plain(s) if s["dir"] == "fwd" else _norm_bwd_plain(s)
    if s["op"] == "recurrence":
        return _recurrence_plain(s)
    return _distill_plain(s)


def _run_own(s):
    from paper_2408_08015_amd import ops
    if s["op"] == "norm":
        if s["dir"] == "fwd":
            y, total, kept = ops.rms_norm_forward(s["x"], s["gain"], residual=s["r"], eps=EPS, keep8=s["keep8"])
            return y, total, ops.stash8_unpack(kept, torch.bfloat16) if s["keep8"] else None
        return ops.rms_norm_backward(s["dy"], s["s"], s["gain"], dsum=s["dsum"], eps=EPS)
    if s["op"] == "recurrence":
        kw = dict(o=s["o"], offsets=s["offsets"], period=s["period"], state=s["state"])
        carry = s["state"] is not None
        y, final, saved = ops.recurrence_forward(s["f"], s["z"], final=carry, saved=s["dir"] == "train", **kw)
        if s["dir"] != "train":
            return y, final
        return (y, final) + ops.recurrence_backward(s["dy"], s["f"], s["z"], saved, dfinal=s["dfinal"], dstate=carry, **kw)
    kw = dict(temperature=s["tau"], labels=s["labels"], label_weight=s["mix"])
    if s["dir"] == "fwd":
        return ops.distill_forward(s["z"], s["ids"], s["t"], **kw)
    if s["dir"] == "bwd":
        return ops.distill_backward(s["dloss"], s["z"], s["ids"], s["t"], s["stats"], **kw)
    return ops.distill_step(s["dloss"], s["z"], s["ids"], s["t"], **kw)


def _norm_fwd_plain(s):
    x, r = s["x"], s["r"]
    total = x if r is None else (x.float() + r.float()).to(r.dtype)
    f = total.float()
    y = (f * torch.rsqrt((f * f).mean(-1, keepdim=True) + EPS) * s["gain"]).to(x.dtype)
    return y, total, _through8(y) if s["keep8"] else None


def _norm_bwd_plain(s):
    f, dy = s["s"].float(), s["dy"].float()
    rstd = torch.rsqrt((f * f).mean(-1, keepdim=True) + EPS)
    n = f * rstd
    h = dy * s["gain"]
    ds = rstd * (h - n * (h * n).mean(-1, keepdim=True))
    if s["dsum"] is not None:
        ds = ds + s["dsum"].float()
    return ds.to(s["dy"].dtype), ds.to(s["s"].dtype), (dy * n).sum(0)


def _pow2(e):
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _through8(x):
    """x in 8 bits and back: the least power of two by which a block's values stay within 127, and the values in its
    steps, rounded to nearest even."""
    T, C = x.shape
    f = torch.nn.functional.pad(x.float(), (0, -C % BLOCK)).view(T, -1, BLOCK)
    m, e = torch.frexp(f.abs().amax(-1, keepdim=True))
    e = (e - 7 + (m > 127.0 / 128.0).to(e.dtype)).clamp_(min=-126)
    e = torch.where(m == 0, torch.full_like(e, -126), e)
    return (torch.round(f * _pow2(-e)) * _pow2(e)).flatten(1)[:, :C].to(torch.bfloat16)   # (exact: seven bits and a sign)


def _sequences(s):
    """(sequence of every token, first token of every sequence, tokens in front of its end)."""
    T = s["T"]
    t = torch.arange(T, device="cuda")
    if s["offsets"] is None:
        begin = torch.arange(s["n"], device="cuda") * s["period"]
        end = (begin + s["period"]).clamp(max=T)
        return t // s["period"], begin, end
    o = s["offsets"].long()
    return torch.searchsorted(o, t, right=True) - 1, o[:-1], o[1:]


def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t along the first axis, h_{-1} = 0: maps of 1, 2, 4, ... tokens joined."""
    step = 1
    while step < a.shape[0]:
        b = torch.cat((b[:step], b[step:] + a[step:] * b[:-step]))
        a = torch.cat((a[:step], a[step:] * a[:-step]))
        step *= 2
    return b


def _recurrence_plain(s):
    f, z = s["f"].float(), s["z"].float()
    seq, begin, end = _sequences(s)
    some = end > begin
    first, last = begin[some], end[some] - 1
    a, b = torch.sigmoid(f), torch.sigmoid(-f)
    into = torch.zeros_like(f) if s["state"] is None else torch.zeros_like(f).index_copy_(0, first, s["state"][some])
    cut = a.index_fill(0, first, 0.0)
    h = _scan(cut, b * z + a * into)
    gate = torch.ones_like(h) if s["o"] is None else s["o"].float() * torch.sigmoid(s["o"].float())
    y = (h * gate).to(s["f"].dtype)
    final = None if s["state"] is None else torch.where(some[:, None], h[(end - 1).clamp(min=0)], s["state"])
    if s["dir"] != "train":
        return y, final
    dy = s["dy"].float()
    before = into.clone()   # h of the token in front
    before[1:] += h[:-1] * (seq[1:] == seq[:-1])[:, None]
    g = dy * gate
    if s["dfinal"] is not None:
        g = g.index_add(0, last, s["dfinal"][some])
    back = torch.cat((cut[1:], torch.zeros_like(cut[:1])))   # what reaches a token from the next one
    G = _scan(back.flip(0), g.flip(0)).flip(0)
    df, dz = G * (before - z) * a * b, G * b
    do = None
    if s["o"] is not None:
        o = s["o"].float()
        sg = torch.sigmoid(o)
        do = (dy * h * (sg + o * sg * torch.sigmoid(-o))).to(s["f"].dtype)
    dstate = None if s["state"] is None else s["dfinal"].index_copy(0, some.nonzero().flatten(), (a * G)[first])
    return y, final, df.to(s["f"].dtype), dz.to(s["f"].dtype), do, dstate


def _distill_plain(s):
    z, tau, mix = s["z"].float(), s["tau"], s["mix"]
    ids = s["ids"].long()
    live = ids >= 0
    at = torch.where(live, ids, torch.zeros_like(ids))
    t = torch.where(live, s["t"].float() / tau, torch.full_like(at, -math.inf, dtype=torch.float32))
    t = t - t.amax(1, keepdim=True)
    p = torch.exp(t)
    total = p.sum(1, keepdim=True)
    logp = torch.where(live, t - torch.log(total), torch.zeros_like(t))
    p = p / total
    top = z.amax(1, keepdim=True)
    e = torch.exp((z - top) / tau)
    sums = e.sum(1, keepdim=True)
    sums1 = torch.exp(z - top).sum(1, keepdim=True) if mix else None
    if s["dir"] != "bwd":
        logq = (z.gather(1, at) - top) / tau - torch.log(sums)
        loss = (1.0 - mix) * tau * tau * (p * (logp - logq)).sum(1)
        if mix:
            loss = loss - mix * ((z.gather(1, s["labels"].long()[:, None]) - top) - torch.log(sums1))[:, 0]
        if s["dir"] == "fwd":
            return loss, torch.cat((top, sums, sums1 if mix else torch.zeros_like(sums)), 1)
    d = (1.0 - mix) * tau * (e / sums).scatter_add_(1, at, -p)
    if mix:
        d = d + mix * (torch.exp(z - top) / sums1).scatter_add_(1, s["labels"].long()[:, None], torch.full_like(sums1, -1.0))
    d = (d * s["dloss"][:, None]).to(s["z"].dtype)
    return d if s["dir"] == "bwd" else (loss, d)


# ---------------------------------------------------------------------------------------------- sizes and definition

def work(case):
    size = {"f32": 4, "bf16": 2}
    T, e = case["T"], size[case["dtype"]]
    if case["op"] == "norm":
        C, st = case["C"], size[case["stream"]]
        n = T * C
        if case["dir"] == "fwd":   # x and y; the stream in and out; 8 bits with their scales, and restored
            return {"bytes": 2 * n * e + (2 * n * st if case["residual"] else 0) + 4 * C + (3 * n + n // BLOCK if case["keep8"] else 0),
                    "flops": 6 * n}
        return {"bytes": 2 * n * e + n * st + (n * st if case["residual"] else 0) + (n * st if st != e else 0) + 8 * C, "flops": 12 * n}
    if case["op"] == "recurrence":
        n = T * case["C"]
        parts = 3 if case["gate"] else 2
        k = -(-T // case["period"]) if case["period"] else case["lengths"]
        states = 4 * k * case["C"] if case["state"] else 0
        if case["dir"] != "train":
            return {"bytes": (parts + 1) * n * e + 2 * states, "flops": 14 * n}
        return {"bytes": (2 * parts + 2) * n * e + 4 * states, "flops": 40 * n}
    n, small = T * case["V"], T * case["K"] * (4 + size[case["teacher"]]) + 20 * T
    exps = 4 if case["mix"] and case["tau"] != 1.0 else 2
    if case["dir"] == "fwd":
        return {"bytes": n * e + small, "flops": exps * n}
    return {"bytes": 2 * n * e + small, "flops": 3 * exps * n}


def exact(case, seed):
    """The operators' definitions in 64 bits."""
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _norm_exact(case, s)
    if case["op"] == "recurrence":
        return _recurrence_exact(case, s)
    return _distill_exact(case, s)


def _norm_exact(case, s):
    if case["dir"] == "bwd":
        x, h = s["s"].double(), s["dy"].double() * s["gain"].double()
        size = torch.sqrt(torch.linalg.vector_norm(x, dim=1, keepdim=True) ** 2 / case["C"] + EPS)
        d = h / size - x * ((h * x).sum(1, keepdim=True) / (case["C"] * size ** 3))
        if case["residual"]:
            d += s["dsum"].double()
        return d, d, torch.einsum("tc,tc->c", s["dy"].double(), x / size)
    x = s["x"].double()
    if case["residual"]:
        x = (x + s["r"].double()).to(s["r"].dtype).double()   # the sum has the stream's type
    y = x / torch.sqrt(torch.linalg.vector_norm(x, dim=1, keepdim=True) ** 2 / case["C"] + EPS) * s["gain"].double()
    if not case["keep8"]:
        return y, x, None
    b = y.to(s["x"].dtype).double()   # what is kept is the result as it is written
    b = torch.cat((b, b.new_zeros(case["T"], -case["C"] % BLOCK)), 1).view(case["T"], -1, BLOCK)
    big = b.abs().max(-1, keepdim=True).values
    step = torch.full_like(big, -126.0)
    guess = torch.floor(torch.log2(torch.where(big > 0, big, torch.ones_like(big)))) - 7.0
    for e in (guess, guess + 1.0, guess + 2.0):   # the least exponent that holds the block
        step = torch.where(big > 127.0 * torch.exp2(step), torch.maximum(step, e), step)
    return y, x, (torch.round(b / torch.exp2(step)) * torch.exp2(step)).view(case["T"], -1)[:, :case["C"]]


def _recurrence_exact(case, s):
    """Token by token, the sequences side by side where they have one length."""
    T, n, C = case["T"], s["n"], case["C"]
    f, z = s["f"].double(), s["z"].double()
    keep, new = 1.0 / (1.0 + torch.exp(-f)), 1.0 / (1.0 + torch.exp(f))
    ends = ([min(T, (i + 1) * case["period"]) for i in range(n)] if case["period"] else s["offsets"].tolist()[1:])
    begins = [0] + ends[:-1]
    start = [None if s["state"] is None else s["state"][i].double() for i in range(n)]
    zero = torch.zeros(C, device="cuda", dtype=torch.float64)
    h = torch.empty_like(f)
    if case["period"] and case["period"] * n == T and n > 1:
        k = lambda x: x.view(n, case["period"], C)
        cur = s["state"].double() if s["state"] is not None else torch.zeros(n, C, device="cuda", dtype=torch.float64)
        for t in range(case["period"]):
            cur = k(keep)[:, t] * cur + k(new)[:, t] * k(z)[:, t]
            k(h)[:, t] = cur
    else:
        drive = new * z
        for i in range(n):
            cur = zero if start[i] is None else start[i]
            for t in range(begins[i], ends[i]):
                cur = torch.addcmul(drive[t], keep[t], cur)
                h[t] = cur
    gate = 1.0 if s["o"] is None else s["o"].double() / (1.0 + torch.exp(-s["o"].double()))
    y = h * gate
    at = torch.tensor([max(e - 1, 0) for e in ends], device="cuda")
    empty = torch.tensor([e == b for b, e in zip(begins, ends)], device="cuda")[:, None]
    final = None if s["state"] is None else torch.where(empty, s["state"].double(), h[at])
    if case["dir"] != "train":
        return y, final
    dy = s["dy"].double()
    G = dy * gate
    dstate = None if s["state"] is None else s["dfinal"].double().clone()
    prev = torch.cat((zero[None], h[:-1]))
    for i in range(n):
        b, e = begins[i], ends[i]
        if b == e:
            continue
        prev[b] = zero if start[i] is None else start[i]
        if s["dfinal"] is not None:
            G[e - 1] += s["dfinal"][i].double()
        if case["period"] and case["period"] * n == T and n > 1:
            continue
        for t in range(e - 2, b - 1, -1):
            G[t].addcmul_(keep[t + 1], G[t + 1])
    if case["period"] and case["period"] * n == T and n > 1:
        for t in range(case["period"] - 2, -1, -1):
            G.view(n, -1, C)[:, t] += keep.view(n, -1, C)[:, t + 1] * G.view(n, -1, C)[:, t + 1]
    if dstate is not None:
        live = (~empty[:, 0]).nonzero().flatten()
        where = torch.tensor(begins, device="cuda")[live]
        dstate[live] = keep[where] * G[where]
    do = None
    if s["o"] is not None:
        o = s["o"].double()
        sg = 1.0 / (1.0 + torch.exp(-o))
        do = dy * h * sg * (1.0 + o * (1.0 - sg))
    return y, final, G * (prev - z) * keep * new, G * new, do, dstate


def _distill_exact(case, s):
    z, tau, mix = s["z"].double(), case["tau"], case["mix"]
    rows, places = (s["ids"] >= 0).nonzero(as_tuple=True)
    v = s["ids"][rows, places].long()
    t = torch.full(s["t"].shape, -math.inf, device="cuda", dtype=torch.float64)
    t[rows, places] = s["t"][rows, places].double() / tau
    logp = t - torch.logsumexp(t, 1, keepdim=True)
    p = logp.exp()
    logq = z / tau
    logq -= torch.logsumexp(logq, 1, keepdim=True)
    rate = (1.0 - mix) * tau
    out = []
    if mix:
        label = s["labels"].long()
        every = torch.arange(case["T"], device="cuda")
        logq1 = z - torch.logsumexp(z, 1, keepdim=True)
    if case["dir"] != "bwd":
        loss = torch.zeros(case["T"], device="cuda", dtype=torch.float64)
        loss.index_add_(0, rows, rate * tau * p[rows, places] * (logp[rows, places] - logq[rows, v]))
        if mix:
            loss -= mix * logq1[every, label]
        out.append(loss)
    if case["dir"] == "fwd":
        top = z.max(1).values
        ones = torch.logsumexp(z - top[:, None], 1).exp() if mix else torch.zeros_like(top)
        out.append(torch.stack((top, torch.logsumexp((z - top[:, None]) / tau, 1).exp(), ones), 1))
    else:
        d = logq.exp_().mul_(rate)
        d.index_put_((rows, v), -rate * p[rows, places], accumulate=True)
        if mix:
            d += mix * logq1.exp_()
            d[every, label] -= mix
        out.append(d.mul_(s["dloss"].double()[:, None]))
    return out[0] if len(out) == 1 else tuple(out)
