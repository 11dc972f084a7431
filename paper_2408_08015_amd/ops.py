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


_LIB = None


def _lib():
    global _LIB
    if _LIB is None:
        lib = load_library()
        vp, i32, i64, f32, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
        szp, hp, qp = C.POINTER(sz), C.POINTER(ast_heads), C.POINTER(ast_qk_cfg)
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
        }.items():
            getattr(lib, "asteroid_" + name).argtypes = types
        _LIB = lib
    return _LIB


# the handle of a device's current stream (without a Stream object around it, where torch offers that)
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda d: torch.cuda.current_stream(d).cuda_stream)


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
    if torch.cuda.current_device() == d:
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
