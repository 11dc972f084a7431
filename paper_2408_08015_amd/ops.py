"""The single operators of language-model stages on torch tensors (include/asteroid_ops.h; same names, argument
marshalling only).

Every call checks its tensors, enqueues on the current torch stream of their device and returns at once.  Outputs
and workspaces that are not passed are allocated from torch's caching allocator (a workspace is the call's own, so
calls on two streams, or captured into two graphs, never share one).  Tensors are contiguous unless stated."""
import ctypes as C

import torch

from .binding import _check, load_library

_DT = {torch.float32: 0, torch.bfloat16: 1}
_F32, _I32 = (torch.float32,), (torch.int32,)


class ast_heads(C.Structure):
    _fields_ = [("dev", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64), ("heads", C.c_int32)]


class ast_qk_cfg(C.Structure):
    _fields_ = [("tokens", C.c_int64), ("dtype", C.c_int32), ("head_dim", C.c_int32), ("rotary", C.c_int32),
                ("interleaved", C.c_int32), ("eps", C.c_float), ("theta", C.c_double),
                ("positions_dev", C.c_void_p), ("period", C.c_int32)]


class ast_norm_cfg(C.Structure):
    _fields_ = [("rows", C.c_int64), ("width", C.c_int64), ("dtype", C.c_int32), ("sum_dtype", C.c_int32), ("eps", C.c_float)]


class ast_rows(C.Structure):
    _fields_ = [("dev", C.c_void_p), ("stride", C.c_int64)]


class ast_recurrence_cfg(C.Structure):
    _fields_ = [("tokens", C.c_int64), ("channels", C.c_int64), ("dtype", C.c_int32), ("offsets_dev", C.c_void_p),
                ("sequences", C.c_int64), ("period", C.c_int64)]


class ast_distill_cfg(C.Structure):
    _fields_ = [("rows", C.c_int64), ("vocab", C.c_int64), ("logits_stride", C.c_int64), ("dtype", C.c_int32),
                ("entries", C.c_int32), ("teacher_dtype", C.c_int32), ("temperature", C.c_float), ("label_weight", C.c_float),
                ("labels_dev", C.c_void_p)]


RECURRENCE_CHUNK = 64   # AST_RECURRENCE_CHUNK

_LIB = None


def _lib():
    global _LIB
    if _LIB is None:
        lib = load_library()
        vp, i32, i64, f32, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
        szp, hp, qp = C.POINTER(sz), C.POINTER(ast_heads), C.POINTER(ast_qk_cfg)
        np_, rp, sp, dp = (C.POINTER(t) for t in (ast_norm_cfg, ast_recurrence_cfg, ast_rows, ast_distill_cfg))
        for name, types in {
            "embedding_forward": [vp, i64, vp, i32, i64, i64, f32, vp, i32, vp],
            "embedding_backward_workspace": [i64, i64, i64, szp],
            "embedding_backward": [vp, i64, vp, i32, i64, i64, f32, i32, vp, vp, sz, vp],
            "qk_norm_rope_forward": [qp, hp, hp, vp, vp, hp, hp, vp],
            "qk_norm_rope_backward_workspace": [qp, i32, i32, szp],
            "qk_norm_rope_backward": [qp, hp, hp, hp, hp, vp, vp, hp, hp, vp, vp, i32, vp, sz, vp],
            "stash8_bytes": [i64, i64, szp],
            "stash8_pack": [vp, i32, i64, i64, vp, vp],
            "stash8_unpack": [vp, i64, i64, vp, i32, vp],
            "linear_wgrad_stash8_workspace": [i64, i64, i64, szp],
            "linear_wgrad_stash8": [vp, vp, i64, i64, i64, vp, vp, i32, vp, sz, vp],
            "gelu_backward_stash8": [vp, i32, vp, i64, i64, vp, vp],
            "rms_norm_forward": [np_, vp, vp, vp, vp, vp, vp, vp],
            "rms_norm_backward_workspace": [np_, szp],
            "rms_norm_backward": [np_, vp, vp, vp, vp, vp, vp, vp, i32, vp, sz, vp],
            "recurrence_workspace": [rp, szp],
            "recurrence_forward": [rp, sp, sp, sp, vp, vp, vp, vp, vp, sz, vp],
            "recurrence_backward": [rp, sp, sp, sp, sp, vp, vp, vp, sp, sp, sp, vp, vp, sz, vp],
            "distill_forward": [dp, vp, vp, vp, vp, vp, vp],
            "distill_backward": [dp, vp, vp, vp, vp, vp, vp, i64, vp],
            "distill_step_workspace": [dp, szp],
            "distill_step": [dp, vp, vp, vp, vp, vp, vp, i64, vp, sz, vp],
        }.items():
            getattr(lib, "asteroid_" + name).argtypes = types
        _LIB = lib
    return _LIB


# the handle of a device's current stream (without a Stream object around it, where torch offers that)
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda d: torch.cuda.current_stream(d).cuda_stream)
_current = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _device(t, *others):
    """The GPU that holds the tensors."""
    d = t.get_device()
    if d < 0:
        raise ValueError("tensors must be on a GPU, got %s" % t.device)
    for o in others:
        if o is not None and o.get_device() != d:
            raise ValueError("tensors on different devices: %s and %s" % (t.device, o.device))
    return d


def _call(d, fn, *args):
    """fn(*args, stream) with device d current (the calls launch on the current one) and its current stream."""
    if _current() == d:
        st = fn(*args, _stream(d))
    else:
        with torch.cuda.device(d):
            st = fn(*args, _stream(d))
    if st:
        _check(_LIB, st)


def _is(t, name, dtypes, shape):
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes:
        raise ValueError("%s must be a tensor of %s" % (name, " or ".join(str(d) for d in dtypes)))
    if t.shape != shape:
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t


def _matrix(t, name, dtypes=(torch.float32, torch.bfloat16)):
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError("%s must be a matrix" % name)
    return _is(t, name, dtypes, t.shape)


def _vector_i32(t, name, n=None):
    if not isinstance(t, torch.Tensor) or t.dim() != 1:
        raise ValueError("%s must be a vector" % name)
    return _is(t, name, _I32, t.shape if n is None else (n,))


def _empty(n, device):
    return torch.empty(max(int(n), 1), dtype=torch.uint8, device=device)


def _workspace(given, need, device):
    if given is None:
        return _empty(need, device)
    if given.dtype != torch.uint8 or not given.is_contiguous() or given.numel() < need or given.device != device:
        raise ValueError("the workspace must be a contiguous uint8 tensor of at least %d bytes on %s" % (need, device))
    return given


# ------------------------------------------------------------------------------------------------ embedding

def embedding_forward(ids, table, scale=1.0, dtype=None, out=None):
    """scale * table[ids] [tokens, width] in `dtype` (the table's, if not given); 0 for ids outside the table.
    ids int32 [tokens]; table float32 or bfloat16 [rows, width]."""
    _vector_i32(ids, "ids")
    _matrix(table, "table")
    T, (V, D) = ids.shape[0], table.shape
    if out is None:
        out = torch.empty((T, D), dtype=dtype or table.dtype, device=table.device)
    _is(out, "out", tuple(_DT), (T, D))
    if dtype not in (None, out.dtype):
        raise ValueError("out is %s, not %s" % (out.dtype, dtype))
    lib = _lib()
    _call(_device(table, ids, out), lib.asteroid_embedding_forward, ids.data_ptr(), T, table.data_ptr(), _DT[table.dtype],
          V, D, scale, out.data_ptr(), _DT[out.dtype])
    return out


def embedding_backward_workspace(tokens, rows, width):
    """Bytes of workspace that embedding_backward takes."""
    n = C.c_size_t()
    lib = _lib()
    _check(lib, lib.asteroid_embedding_backward_workspace(tokens, rows, width, C.byref(n)))
    return n.value


def embedding_backward(ids, dy, rows, scale=1.0, out=None, accumulate=False, workspace=None):
    """The table's gradient, float32 [rows, width]: scale * the sum of dy over the tokens of each id.  accumulate:
    added to `out` (which has to be given), rows without a token stay as they are."""
    _vector_i32(ids, "ids")
    _matrix(dy, "dy")
    T, D = dy.shape
    _vector_i32(ids, "ids", T)
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs the tensor to add to")
        out = torch.empty((rows, D), dtype=torch.float32, device=dy.device)
    _is(out, "out", _F32, (rows, D))
    lib = _lib()
    d = _device(dy, ids, out)
    ws = _workspace(workspace, embedding_backward_workspace(T, rows, D), dy.device)
    _call(d, lib.asteroid_embedding_backward, ids.data_ptr(), T, dy.data_ptr(), _DT[dy.dtype], rows, D, scale,
          bool(accumulate), out.data_ptr(), ws.data_ptr(), ws.numel())
    return out


# ------------------------------------------------------------------------------------------------ queries and keys

def _heads(t, name, T, d, dtype):
    shape = t.shape if isinstance(t, torch.Tensor) else ()
    if len(shape) != 3 or t.dtype != dtype or shape[0] != T or shape[2] != d:
        raise ValueError("%s must be a %s tensor [%d, heads, %d]" % (name, dtype, T, d))
    ts, hs, unit = t.stride()
    if unit != 1 and d > 1:
        raise ValueError("%s must have unit stride inside a head" % name)
    return ast_heads(t.data_ptr(), ts, hs, shape[1])


def _qk_cfg(q, positions, period, rotary, theta, interleaved, eps):
    if not isinstance(q, torch.Tensor) or q.dim() != 3 or q.dtype not in _DT:
        raise ValueError("q must be a float32 or bfloat16 tensor [tokens, heads, head_dim]")
    T, _, d = q.shape
    if positions is not None:
        _vector_i32(positions, "positions", T)
    elif not 1 <= period < 1 << 31:   # (ctypes would cut it off)
        raise ValueError("positions, or the period of the sequences (below 2^31), must be given")
    if rotary is not None and not -1 << 31 <= rotary < 1 << 31:
        raise ValueError("rotary must lie in [0, head_dim]")
    return ast_qk_cfg(T, _DT[q.dtype], d, d // 2 * 2 if rotary is None else rotary, int(bool(interleaved)), eps, theta,
                      None if positions is None else positions.data_ptr(), period)


def qk_norm_rope_forward(q, k, q_gain, k_gain, positions=None, period=0, rotary=None, theta=10000.0, interleaved=False,
                         eps=1e-6, out=None):
    """RMS norm of every head with a gain, then the rotation by the token's position: (yq, yk).
    q [tokens, heads, head_dim], k [tokens, other heads, head_dim], any strides between tokens and heads; gains
    float32 [head_dim]; positions int32 [tokens], or `period`: token t stands at t % period.  rotary: leading values
    of a head that turn (all of them if not given), in pairs of (i, i + rotary / 2), or interleaved (2i, 2i + 1).
    out: a pair of tensors, (q, k) itself allowed."""
    cfg = _qk_cfg(q, positions, period, rotary, theta, interleaved, eps)
    T, d = q.shape[0], q.shape[2]
    yq, yk = out if out is not None else (torch.empty(q.shape, dtype=q.dtype, device=q.device),
                                          torch.empty(k.shape, dtype=q.dtype, device=q.device))
    _is(q_gain, "q_gain", _F32, (d,))
    _is(k_gain, "k_gain", _F32, (d,))
    a = [_heads(t, n, T, d, q.dtype) for t, n in ((q, "q"), (k, "k"), (yq, "yq"), (yk, "yk"))]
    lib = _lib()
    _call(_device(q, k, yq, yk, q_gain, k_gain, positions), lib.asteroid_qk_norm_rope_forward, cfg, a[0], a[1],
          q_gain.data_ptr(), k_gain.data_ptr(), a[2], a[3])
    return yq, yk


def _qk_workspace(cfg):
    n = C.c_size_t()
    lib = _lib()
    _check(lib, lib.asteroid_qk_norm_rope_backward_workspace(cfg, 1, 1, n))
    return n.value


def qk_norm_rope_backward_workspace(tokens, head_dim):
    """Bytes of workspace that qk_norm_rope_backward takes."""
    return _qk_workspace(ast_qk_cfg(tokens, 0, head_dim, 0, 0, 1.0, 1.0, None, 1))


def qk_norm_rope_backward(dyq, dyk, q, k, q_gain, k_gain, positions=None, period=0, rotary=None, theta=10000.0,
                          interleaved=False, eps=1e-6, out=None, gain_out=None, accumulate=False, workspace=None):
    """(dq, dk, dq_gain, dk_gain) of qk_norm_rope_forward with the same arguments; q, k are its inputs.
    out: (dq, dk), (dyq, dyk) itself allowed.  gain_out: (dq_gain, dk_gain); accumulate: added to them."""
    cfg = _qk_cfg(q, positions, period, rotary, theta, interleaved, eps)
    T, d = q.shape[0], q.shape[2]
    dq, dk = out if out is not None else (torch.empty(q.shape, dtype=q.dtype, device=q.device),
                                          torch.empty(k.shape, dtype=q.dtype, device=q.device))
    if gain_out is None:
        if accumulate:
            raise ValueError("accumulate needs the tensors to add to")
        gain_out = torch.empty((2, d), dtype=torch.float32, device=q.device).unbind(0)
    gq, gk = gain_out
    for t, n in ((q_gain, "q_gain"), (k_gain, "k_gain"), (gq, "dq_gain"), (gk, "dk_gain")):
        _is(t, n, _F32, (d,))
    a = [_heads(t, n, T, d, q.dtype) for t, n in ((dyq, "dyq"), (dyk, "dyk"), (q, "q"), (k, "k"), (dq, "dq"), (dk, "dk"))]
    lib = _lib()
    on = _device(q, k, dyq, dyk, dq, dk, q_gain, k_gain, gq, gk, positions)
    ws = _workspace(workspace, _qk_workspace(cfg), q.device)
    _call(on, lib.asteroid_qk_norm_rope_backward, cfg, a[0], a[1], a[2], a[3], q_gain.data_ptr(), k_gain.data_ptr(), a[4], a[5],
          gq.data_ptr(), gk.data_ptr(), bool(accumulate), ws.data_ptr(), ws.numel())
    return dq, dk, gq, gk


# ------------------------------------------------------------------------------------------------ 8-bit activations

class Stash8:
    """A matrix [rows, cols] kept in 8 bits (`data`, a uint8 tensor in the layout of asteroid_ops.h)."""
    __slots__ = ("data", "rows", "cols")

    def __init__(self, rows, cols, device=None, data=None):
        if data is None and device is None:
            raise ValueError("a device, or the tensor to keep the values in, must be given")
        self.data = _workspace(data, stash8_bytes(rows, cols), device if data is None else data.device)
        self.rows, self.cols = rows, cols


def stash8_bytes(rows, cols):
    """Bytes of the buffer that keeps a matrix [rows, cols]."""
    n = C.c_size_t()
    lib = _lib()
    _check(lib, lib.asteroid_stash8_bytes(rows, cols, C.byref(n)))
    return n.value


def _stash(s):
    if not isinstance(s, Stash8):
        raise ValueError("a Stash8 is expected")
    return s


def stash8_pack(x, out=None):
    """x float32 or bfloat16 [rows, cols] in 8 bits: blocks of 32 values of a row share a power of two."""
    _matrix(x, "x")
    s = Stash8(x.shape[0], x.shape[1], x.device) if out is None else _stash(out)
    if (s.rows, s.cols) != tuple(x.shape):
        raise ValueError("the stash keeps [%d, %d], x is %s" % (s.rows, s.cols, tuple(x.shape)))
    lib = _lib()
    _call(_device(x, s.data), lib.asteroid_stash8_pack, x.data_ptr(), _DT[x.dtype], s.rows, s.cols, s.data.data_ptr())
    return s


def stash8_unpack(stash, dtype=torch.bfloat16, out=None):
    """The values that the stash stands for, exact in float32 and bfloat16."""
    s = _stash(stash)
    if out is None:
        out = torch.empty((s.rows, s.cols), dtype=dtype, device=s.data.device)
    _is(out, "out", tuple(_DT), (s.rows, s.cols))
    lib = _lib()
    _call(_device(s.data, out), lib.asteroid_stash8_unpack, s.data.data_ptr(), s.rows, s.cols, out.data_ptr(), _DT[out.dtype])
    return out


def linear_wgrad_stash8_workspace(rows, inputs, outputs):
    """Bytes of workspace that linear_wgrad_stash8 takes."""
    n = C.c_size_t()
    lib = _lib()
    _check(lib, lib.asteroid_linear_wgrad_stash8_workspace(rows, inputs, outputs, C.byref(n)))
    return n.value


def linear_wgrad_stash8(dy, stash, bias=True, out=None, bias_out=None, accumulate=False, workspace=None):
    """(dW [outputs, inputs], db [outputs]) of a dense layer y = x W^T + b, float32, from dy bfloat16 [rows, outputs]
    and the kept x [rows, inputs]; db is None where bias is false.  accumulate: added to out and bias_out."""
    s = _stash(stash)
    _matrix(dy, "dy", (torch.bfloat16,))
    if dy.shape[0] != s.rows:
        raise ValueError("dy has %d rows, the stash %d" % (dy.shape[0], s.rows))
    N, K = dy.shape[1], s.cols
    if accumulate and (out is None or (bias and bias_out is None)):
        raise ValueError("accumulate needs the tensors to add to")
    if out is None:
        out = torch.empty((N, K), dtype=torch.float32, device=dy.device)
    _is(out, "out", _F32, (N, K))
    db = None
    if bias:
        db = torch.empty((N,), dtype=torch.float32, device=dy.device) if bias_out is None else bias_out
        _is(db, "bias_out", _F32, (N,))
    lib = _lib()
    d = _device(dy, s.data, out, db)
    ws = _workspace(workspace, linear_wgrad_stash8_workspace(s.rows, K, N), dy.device)
    _call(d, lib.asteroid_linear_wgrad_stash8, dy.data_ptr(), s.data.data_ptr(), s.rows, K, N, out.data_ptr(),
          None if db is None else db.data_ptr(), bool(accumulate), ws.data_ptr(), ws.numel())
    return out, db


def gelu_backward_stash8(dy, stash, out=None):
    """dy * GELU'(z) for the kept pre-activation z [rows, cols]; dy float32 or bfloat16, `out` may be dy."""
    s = _stash(stash)
    _is(dy, "dy", tuple(_DT), (s.rows, s.cols))
    if out is None:
        out = torch.empty_like(dy)
    _is(out, "out", (dy.dtype,), (s.rows, s.cols))
    lib = _lib()
    _call(_device(dy, s.data, out), lib.asteroid_gelu_backward_stash8, dy.data_ptr(), _DT[dy.dtype], s.data.data_ptr(), s.rows,
          s.cols, out.data_ptr())
    return out


# ------------------------------------------------------------------------------------------------ RMS norm and residual

def _ptr(t):
    return None if t is None else t.data_ptr()


def rms_norm_forward(x, gain, residual=None, eps=1e-6, keep8=False, out=None, sum_out=None, kept_out=None):
    """(y, s, kept): s = x + residual in the residual's type (x itself without one), y = s / sqrt(mean s^2 + eps) * gain
    in x's type, kept = y in 8 bits (a Stash8; None unless keep8).  x float32 or bfloat16 [rows, width], residual of the same
    shape in x's type or float32, gain float32 [width].  out may be x, sum_out the residual."""
    _matrix(x, "x")
    _is(gain, "gain", _F32, (x.shape[1],))
    if residual is not None:
        _is(residual, "residual", (x.dtype, torch.float32), x.shape)
        if sum_out is None:
            sum_out = torch.empty_like(residual)
        else:
            _is(sum_out, "sum_out", (residual.dtype,), x.shape)
    elif sum_out is not None:
        raise ValueError("without a residual there is no sum to write")
    if out is None:
        out = torch.empty_like(x)
    else:
        _is(out, "out", (x.dtype,), x.shape)
    kept = None
    if keep8 or kept_out is not None:
        kept = Stash8(x.shape[0], x.shape[1], x.device) if kept_out is None else _stash(kept_out)
        if (kept.rows, kept.cols) != tuple(x.shape):
            raise ValueError("the stash keeps [%d, %d], x is %s" % (kept.rows, kept.cols, tuple(x.shape)))
    sums = x if residual is None else sum_out
    lib = _lib()
    cfg = ast_norm_cfg(x.shape[0], x.shape[1], _DT[x.dtype], _DT[sums.dtype], eps)
    _call(_device(x, gain, residual, out, sum_out, None if kept is None else kept.data), lib.asteroid_rms_norm_forward, cfg,
          x.data_ptr(), _ptr(residual), gain.data_ptr(), out.data_ptr(), _ptr(sum_out), None if kept is None else kept.data.data_ptr())
    return out, sums, kept


def _norm_workspace(cfg):
    n = C.c_size_t()
    lib = _lib()
    _check(lib, lib.asteroid_rms_norm_backward_workspace(cfg, n))
    return n.value


def rms_norm_backward_workspace(rows, width):
    """Bytes of workspace that rms_norm_backward takes."""
    return _norm_workspace(ast_norm_cfg(rows, width, 0, 0, 1.0))


def rms_norm_backward(dy, s, gain, dsum=None, eps=1e-6, out=None, sum_out=None, gain_out=None, accumulate=False, workspace=None):
    """(dx, ds, dgain) of rms_norm_forward: the gradient of x and the residual in dy's type and in that of s (one tensor
    where these are the same), and the gain's, float32.  s is the sum that the forward pass returned, dsum (of s's
    type) the gradient that reaches it from further on.  out may be dy, sum_out may be dsum or s.  accumulate: added to gain_out."""
    _matrix(dy, "dy")
    _is(s, "s", (dy.dtype, torch.float32), dy.shape)
    _is(gain, "gain", _F32, (dy.shape[1],))
    if dsum is not None:
        _is(dsum, "dsum", (s.dtype,), dy.shape)
    one = s.dtype == dy.dtype
    if one and out is not None and sum_out is not None and out is not sum_out:
        raise ValueError("out and sum_out are one tensor where the types are the same")
    if one and out is None:
        out = sum_out
    if out is None:
        out = torch.empty_like(dy)
    else:
        _is(out, "out", (dy.dtype,), dy.shape)
    if one:
        sum_out = out
    elif sum_out is None:
        sum_out = torch.empty_like(s)
    else:
        _is(sum_out, "sum_out", (s.dtype,), dy.shape)
    if gain_out is None:
        if accumulate:
            raise ValueError("accumulate needs the tensor to add to")
        gain_out = torch.empty_like(gain)
    else:
        _is(gain_out, "gain_out", _F32, gain.shape)
    cfg = ast_norm_cfg(dy.shape[0], dy.shape[1], _DT[dy.dtype], _DT[s.dtype], eps)
    lib = _lib()
    d = _device(dy, s, gain, dsum, out, sum_out, gain_out)
    ws = _workspace(workspace, _norm_workspace(cfg), dy.device)
    _call(d, lib.asteroid_rms_norm_backward, cfg, dy.data_ptr(), s.data_ptr(), gain.data_ptr(), _ptr(dsum), out.data_ptr(),
          None if one else sum_out.data_ptr(), gain_out.data_ptr(), bool(accumulate), ws.data_ptr(), ws.numel())
    return out, sum_out, gain_out


# ------------------------------------------------------------------------------------------------ gated recurrence

def _tokens(t, name, shape, dtype):
    """A matrix [tokens, channels] in rows of any stride, as the C calls take it."""
    if not isinstance(t, torch.Tensor) or t.shape != shape or t.dtype != dtype:
        raise ValueError("%s must be a %s tensor %s" % (name, dtype, tuple(shape)))
    step, unit = t.stride()
    if unit != 1 and shape[1] > 1:
        raise ValueError("%s must have unit stride inside a row" % name)
    return ast_rows(t.data_ptr(), step if shape[0] > 1 else shape[1])


def _recurrence_inputs(f, z, o, offsets, period):
    """The call's cfg, its sequences, and f, z, o as the C calls take them."""
    if not isinstance(f, torch.Tensor) or f.dim() != 2 or f.dtype not in _DT:
        raise ValueError("f must be a float32 or bfloat16 tensor [tokens, channels]")
    shape, dtype = f.shape, f.dtype
    rows = _tokens(f, "f", shape, dtype), _tokens(z, "z", shape, dtype), None if o is None else _tokens(o, "o", shape, dtype)
    T, D = shape
    if offsets is not None:
        _vector_i32(offsets, "offsets")
        n = offsets.shape[0] - 1
        if n < 0:
            raise ValueError("offsets must hold one number more than there are sequences")
        return ast_recurrence_cfg(T, D, _DT[dtype], offsets.data_ptr(), n, 0), n, rows
    if not 1 <= period < 1 << 31:
        raise ValueError("offsets, or the period of the sequences (below 2^31), must be given")
    return ast_recurrence_cfg(T, D, _DT[dtype], None, 0, period), -(-T // period), rows


def _state(t, name, n, f):
    """None or a tensor [sequences, channels] to read from."""
    return None if t is None else _is(t, name, _F32, (n, f.shape[1]))


def _states(t, name, n, f, like=None):
    """None, a tensor [sequences, channels], or (True) one that is made here (as `like`, which has been checked, where there is one)."""
    if t is None or t is False:
        return None
    if t is True and like is not None:
        return torch.empty_like(like)
    shape = (n, f.shape[1])
    return torch.empty(shape, dtype=torch.float32, device=f.device) if t is True else _is(t, name, _F32, shape)


def _workspace_of(fn, cfg, given, device):
    """The workspace and its size, which `fn` says; none where the call takes none."""
    n = C.c_size_t()
    st = fn(cfg, n)
    if st:
        _check(_LIB, st)
    if not n.value:
        return None, 0
    ws = _workspace(given, n.value, device)
    return ws.data_ptr(), ws.numel()


def recurrence_workspace(tokens, channels, dtype, offsets=False, period=0):
    """Bytes of workspace that recurrence_forward and recurrence_backward take (offsets: whether they are given)."""
    n = C.c_size_t()
    lib = _lib()
    _check(lib, lib.asteroid_recurrence_workspace(ast_recurrence_cfg(tokens, channels, _DT[dtype], 4 if offsets else None, 0, period), n))
    return n.value


def recurrence_forward(f, z, o=None, offsets=None, period=0, state=None, final=None, saved=None, out=None, workspace=None):
    """(y, final, saved): h_t = a_t h_{t-1} + (1 - a_t) z_t with a = sigmoid(f), y = h * o sigmoid(o) (h without o).
    f, z, o float32 or bfloat16 [tokens, channels] with unit stride inside a row; sequences one behind the other: offsets int32
    [sequences + 1], or `period` tokens each.  state float32 [sequences, channels]: in front of every sequence (0 if not given).
    final: True or a tensor (state itself allowed) to receive the states behind them.  saved: True or a float32 tensor
    [tokens / 64 rounded up, channels] for recurrence_backward.  y is dense; rows of no sequence are not written."""
    cfg, n, a = _recurrence_inputs(f, z, o, offsets, period)
    state = _state(state, "state", n, f)
    final = _states(final, "final", n, f, state)
    saved = _states(saved, "saved", -(-f.shape[0] // RECURRENCE_CHUNK), f)
    if out is None:
        out = torch.empty_like(f, memory_format=torch.contiguous_format)
    else:
        _is(out, "out", (f.dtype,), f.shape)
    lib = _lib()
    d = _device(f, z, o, offsets, state, final, saved, out)
    ws, size = _workspace_of(lib.asteroid_recurrence_workspace, cfg, workspace, f.device)
    _call(d, lib.asteroid_recurrence_forward, cfg, a[0], a[1], a[2], _ptr(state), out.data_ptr(), _ptr(final), _ptr(saved), ws, size)
    return out, final, saved


def recurrence_backward(dy, f, z, saved, o=None, offsets=None, period=0, state=None, dfinal=None, dstate=None, out=None,
                        workspace=None):
    """(df, dz, do, dstate) of recurrence_forward with the same arguments; saved is what it left.  dfinal float32
    [sequences, channels]: the gradient of final (0 if not given).  dstate: True or a tensor (dfinal or state allowed) to receive the gradient
    of state.
    out: (df, dz, do), rows with any stride; (f, z, o) themselves allowed.  do is None where o is."""
    cfg, n, a = _recurrence_inputs(f, z, o, offsets, period)
    _is(saved, "saved", _F32, (-(-f.shape[0] // RECURRENCE_CHUNK), f.shape[1]))
    state = _state(state, "state", n, f)
    dfinal = _state(dfinal, "dfinal", n, f)
    dstate = _states(dstate, "dstate", n, f, state)
    shape, dtype = f.shape, f.dtype
    b = [_tokens(dy, "dy", shape, dtype)]
    if out is None:
        out = torch.empty((2 if o is None else 3,) + tuple(shape), dtype=dtype, device=f.device).unbind(0)
        b += [ast_rows(g.data_ptr(), shape[1]) for g in out]
    df, dz, do = (tuple(out) + (None,))[:3]
    if (do is None) != (o is None):
        raise ValueError("out holds the gradient of o where o is given, and only there")
    if len(b) == 1:
        b += [_tokens(g, name, shape, dtype) for g, name in ((df, "df"), (dz, "dz"), (do, "do")) if g is not None]
    if do is None:
        b.append(None)
    lib = _lib()
    d = _device(f, z, o, dy, saved, offsets, state, dfinal, dstate, df, dz, do)
    ws, size = _workspace_of(lib.asteroid_recurrence_workspace, cfg, workspace, f.device)
    _call(d, lib.asteroid_recurrence_backward, cfg, b[0], a[0], a[1], a[2], _ptr(state), saved.data_ptr(), _ptr(dfinal), b[1], b[2],
          b[3], _ptr(dstate), ws, size)
    return df, dz, do, dstate


# ------------------------------------------------------------------------------------------------ distillation

def _distill_cfg(logits, ids, teacher, temperature, labels, label_weight):
    if not isinstance(logits, torch.Tensor) or logits.dim() != 2 or logits.dtype not in _DT:
        raise ValueError("logits must be a float32 or bfloat16 tensor [rows, vocab]")
    T, V = logits.shape
    if not isinstance(ids, torch.Tensor) or ids.dim() != 2:
        raise ValueError("ids must be a matrix")
    _is(ids, "ids", _I32, (T, ids.shape[1]))
    _is(teacher, "teacher", tuple(_DT), ids.shape)
    if labels is not None:
        _vector_i32(labels, "labels", T)
    return ast_distill_cfg(T, V, _vocab_rows(logits, "logits"), _DT[logits.dtype], _entries(ids.shape[1]), _DT[teacher.dtype], temperature,
                           label_weight, None if labels is None else labels.data_ptr())


def _entries(n):
    if not -1 << 31 <= n < 1 << 31:   # (ctypes would cut it off)
        raise ValueError("entries must lie in [1, 1024], got %d" % n)
    return n


def _vocab_rows(t, name):
    if t.stride(1) != 1 and t.shape[1] > 1:
        raise ValueError("%s must have unit stride inside a row" % name)
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _gradient_of(logits, out, dloss):
    _is(dloss, "dloss", _F32, (logits.shape[0],))
    if out is None:
        T, V = logits.shape
        step = logits.stride(0) if T > 1 and 0 < logits.stride(0) - V < 64 else V   # rows padded a little stay so
        if step == V:
            return torch.empty_like(logits, memory_format=torch.contiguous_format), V
        out = torch.empty((T, step), dtype=logits.dtype, device=logits.device)[:, :V]
    if not isinstance(out, torch.Tensor) or out.shape != logits.shape or out.dtype != logits.dtype:
        raise ValueError("out must be a %s tensor %s" % (logits.dtype, tuple(logits.shape)))
    return out, _vocab_rows(out, "out")


def distill_forward(logits, ids, teacher, temperature=1.0, labels=None, label_weight=0.0, out=None, stats_out=None):
    """(loss [rows], stats [rows, 3]), float32: (1 - l) T^2 KL(p || q) + l CE(label) of every row, p the softmax of the
    teacher's logits [rows, entries] / T over the entries whose ids lie in the vocabulary, q that of the student's / T.
    logits float32 or bfloat16 [rows, vocab] with unit stride inside a row, ids int32 [rows, entries], labels int32 [rows].
    stats is for distill_backward."""
    cfg = _distill_cfg(logits, ids, teacher, temperature, labels, label_weight)
    T = logits.shape[0]
    if out is None:
        out = torch.empty((T,), dtype=torch.float32, device=logits.device)
    else:
        _is(out, "out", _F32, (T,))
    if stats_out is None:
        stats_out = torch.empty((T, 3), dtype=torch.float32, device=logits.device)
    else:
        _is(stats_out, "stats_out", _F32, (T, 3))
    lib = _lib()
    _call(_device(logits, ids, teacher, labels, out, stats_out), lib.asteroid_distill_forward, cfg, logits.data_ptr(), ids.data_ptr(),
          teacher.data_ptr(), out.data_ptr(), stats_out.data_ptr())
    return out, stats_out


def distill_backward(dloss, logits, ids, teacher, stats, temperature=1.0, labels=None, label_weight=0.0, out=None):
    """The logits' gradient for dloss float32 [rows]; stats is what distill_forward left.  out may be logits (made here,
    its rows are padded as those of logits are, where that is by fewer than 64 values)."""
    cfg = _distill_cfg(logits, ids, teacher, temperature, labels, label_weight)
    _is(stats, "stats", _F32, (logits.shape[0], 3))
    out, stride = _gradient_of(logits, out, dloss)
    lib = _lib()
    _call(_device(logits, ids, teacher, labels, stats, dloss, out), lib.asteroid_distill_backward, cfg, dloss.data_ptr(),
          logits.data_ptr(), ids.data_ptr(), teacher.data_ptr(), stats.data_ptr(), out.data_ptr(), stride)
    return out


def distill_step_workspace(rows, vocab, entries):
    """Bytes of workspace that distill_step takes."""
    n = C.c_size_t()
    lib = _lib()
    _check(lib, lib.asteroid_distill_step_workspace(ast_distill_cfg(rows, vocab, vocab, 0, _entries(entries), 0, 1.0, 0.0, None), n))
    return n.value


def distill_step(dloss, logits, ids, teacher, temperature=1.0, labels=None, label_weight=0.0, out=None, loss_out=None, workspace=None):
    """(loss, the logits' gradient) at once, where dloss is known beforehand.  out may be logits."""
    cfg = _distill_cfg(logits, ids, teacher, temperature, labels, label_weight)
    out, stride = _gradient_of(logits, out, dloss)
    if loss_out is None:
        loss_out = torch.empty_like(dloss)
    else:
        _is(loss_out, "loss_out", _F32, (logits.shape[0],))
    lib = _lib()
    d = _device(logits, ids, teacher, labels, dloss, loss_out, out)
    ws, size = _workspace_of(lib.asteroid_distill_step_workspace, cfg, workspace, logits.device)
    _call(d, lib.asteroid_distill_step, cfg, dloss.data_ptr(), logits.data_ptr(), ids.data_ptr(), teacher.data_ptr(), loss_out.data_ptr(),
          out.data_ptr(), stride, ws, size)
    return loss_out, out
