"""Operators of token sequence models on torch tensors: marshalling for the entry points of include/snn.h that take a snn_launch.

Every call queues its kernels on the current stream of its tensors' device and returns; results and workspace are tensors of torch's
allocator, so calls may be captured into a graph like torch's own.  Arguments that do not fit raise before anything is queued
(TypeError: element types, ValueError: shapes, strides and devices, SnnError: what the library refuses).  No element of a result may be
one of another tensor of the call, but where it is said so.  Gradients come from the backward calls: nothing is recorded for torch.autograd,
and results have no history even where an argument requires a gradient.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple

SNN_F32, SNN_BF16 = 0, 1
GLR_INTERVAL = 128  # steps between the states that snn_glr_forward keeps
DELTA_INTERVAL = 256  # and snn_delta_forward
PACK_BLOCK = 32     # elements of a row that share a step in 8 bits


class snn_launch(C.Structure):
    _fields_ = [("device", C.c_int32), ("stream", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class snn_glr(C.Structure):
    _fields_ = [("T", C.c_int32), ("batch", C.c_int32), ("n", C.c_int32), ("dtype", C.c_int32), ("ld_z", C.c_int64),
                ("ld_x", C.c_int64), ("ld_h", C.c_int64), ("ld_dz", C.c_int64), ("ld_dx", C.c_int64), ("lengths", C.c_void_p)]


class snn_packed(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("exps", C.c_void_p), ("ld", C.c_int64), ("ld_exps", C.c_int64)]


class snn_vocab(C.Structure):
    _fields_ = [("rows", C.c_int32), ("d", C.c_int32), ("vocab", C.c_int32), ("dtype", C.c_int32), ("ld_h", C.c_int64),
                ("ld_w", C.c_int64)]


class snn_delta(C.Structure):
    _fields_ = [("T", C.c_int32), ("batch", C.c_int32), ("heads", C.c_int32), ("key_heads", C.c_int32), ("dk", C.c_int32), ("dv", C.c_int32),
                ("dtype", C.c_int32), ("scale", C.c_float), ("ld_q", C.c_int64), ("ld_k", C.c_int64), ("ld_v", C.c_int64), ("ld_o", C.c_int64),
                ("ld_dq", C.c_int64), ("ld_dk", C.c_int64), ("ld_dv", C.c_int64), ("lengths", C.c_void_p)]


class snn_norm(C.Structure):
    _fields_ = [("rows", C.c_int64), ("n", C.c_int32), ("dtype", C.c_int32), ("eps", C.c_float), ("ld_x", C.c_int64),
                ("ld_residual", C.c_int64), ("ld_total", C.c_int64), ("ld_y", C.c_int64), ("ld_dtotal", C.c_int64), ("ld_dx", C.c_int64)]


class snn_adamw(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("weight_decay", C.c_double),
                ("step", C.c_int64), ("step_on_device", C.c_void_p), ("grad_scale", C.c_void_p)]


class snn_adamw_tensor(C.Structure):
    _fields_ = [("p", C.c_void_p), ("g", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p), ("m_exps", C.c_void_p), ("v_exps", C.c_void_p),
                ("copy", C.c_void_p), ("n", C.c_int64), ("dtype_p", C.c_int32), ("dtype_g", C.c_int32)]


class Packed(NamedTuple):
    """Rows in 8 bits, as snn_pack gives them: codes int8 [..., n], exps uint8 [..., ceil(n / 32)]."""
    codes: object
    exps: object


def declare(L):
    vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    at, glr, vocab, packed = (C.POINTER(t) for t in (snn_launch, snn_glr, snn_vocab, snn_packed))
    L.snn_launch_error.argtypes = []
    L.snn_launch_error.restype = C.c_char_p
    L.snn_glr_workspace.argtypes = [glr]
    L.snn_glr_workspace.restype = C.c_size_t
    L.snn_vocab_workspace.argtypes = [vocab, i32]
    L.snn_vocab_workspace.restype = C.c_size_t
    L.snn_glr_forward.argtypes = [at, glr] + [vp] * 6
    L.snn_glr_backward.argtypes = [at, glr] + [vp] * 8
    L.snn_glr_backward_packed.argtypes = [at, glr, packed, packed] + [vp] * 6
    L.snn_pack.argtypes = L.snn_unpack.argtypes = [at, C.c_int, i64, i32, i64] + [vp] * 3
    L.snn_vocab_loss.argtypes = [at, vocab] + [vp] * 5
    L.snn_vocab_loss_grad.argtypes = [at, vocab] + [vp] * 7
    norm, adamw, delta = C.POINTER(snn_norm), C.POINTER(snn_adamw), C.POINTER(snn_delta)
    L.snn_delta_workspace.argtypes = [delta, i32]
    L.snn_delta_workspace.restype = C.c_size_t
    L.snn_delta_forward.argtypes = [at, delta] + [vp] * 9
    L.snn_delta_backward.argtypes = [at, delta] + [vp] * 14
    L.snn_norm_workspace.argtypes = [norm]
    L.snn_norm_workspace.restype = C.c_size_t
    L.snn_norm_forward.argtypes = [at, norm] + [vp] * 5
    L.snn_norm_forward_packed.argtypes = L.snn_norm_backward.argtypes = [at, norm] + [vp] * 6
    L.snn_adamw_workspace.argtypes = [adamw]
    L.snn_adamw_workspace.restype = C.c_size_t
    L.snn_adamw_step.argtypes = [at, adamw, C.POINTER(snn_adamw_tensor), i64]
    for name in ("snn_glr_forward", "snn_glr_backward", "snn_glr_backward_packed", "snn_pack", "snn_unpack", "snn_vocab_loss",
                 "snn_vocab_loss_grad", "snn_norm_forward", "snn_norm_forward_packed", "snn_norm_backward", "snn_adamw_step", "snn_delta_forward",
                 "snn_delta_backward"):
        getattr(L, name).restype = C.c_int


_functions = {}  # entry points, by name


def _entry(name):
    f = _functions.get(name)
    if f is None:
        from . import lib
        f = _functions[name] = getattr(lib(), name)
    return f


def _run(name, *args):
    st = _entry(name)(*args)
    if st:
        from . import SnnError
        raise SnnError(st, _entry("snn_launch_error")().decode())


def _type(x, name):
    import torch
    if x.dtype == torch.bfloat16:
        return SNN_BF16
    if x.dtype != torch.float32:
        raise TypeError(f"{name} must be float32 or bfloat16, got {x.dtype}")
    return SNN_F32


def _same(x, name, dtype, shape, device):
    """x has this type and shape and is on this device."""
    if x.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {x.dtype}")
    if tuple(x.shape) != tuple(shape):
        raise ValueError(f"{name} must be {tuple(shape)}, got {tuple(x.shape)}")
    if x.device != device:
        raise ValueError(f"{name} is on {x.device}, not on {device}")
    return x


def _packed_rows(x, name):
    if not x.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return x


def _ld(x, name):
    """Elements between consecutive rows of [..., n], if every row follows the one before at the same distance."""
    if x.is_contiguous():
        return x.shape[-1]
    ld = None
    rows = 1
    if x.shape[-1] > 1 and x.stride(-1) != 1:
        raise ValueError(f"{name}: the elements of a row must be consecutive")
    for size, stride in zip(reversed(x.shape[:-1]), reversed(x.stride()[:-1])):
        if size > 1:
            if ld is None:
                if stride % rows:
                    raise ValueError(f"{name}: its rows must be equally far apart")
                ld = stride // rows
            if stride != ld * rows or ld < x.shape[-1]:
                raise ValueError(f"{name}: its rows must be equally far apart")
        rows *= size
    return x.shape[-1] if ld is None else ld


def _launch(device, work=0):
    """Where a call runs, and its workspace (to be held until the call has returned)."""
    import torch
    if device.type != "cuda":
        raise ValueError(f"the operators run on a GPU, got tensors on {device}")
    stream = torch._C._cuda_getCurrentRawStream(device.index)  # (torch.cuda.current_stream makes an object first)
    if not work:
        return snn_launch(device.index, stream, None, 0), None
    space = torch.empty(work, dtype=torch.uint8, device=device)
    return snn_launch(device.index, stream, space.data_ptr(), work), space


def _at(x):
    return None if x is None else x.data_ptr()


def _sequences(x, name):
    if x.dim() != 3:
        raise ValueError(f"{name} must be [T][batch][n], got {tuple(x.shape)}")
    return tuple(x.shape)


def _out(x, name, like):
    """x as the result `name`, or a new tensor for it."""
    import torch
    if x is None:
        return torch.empty_like(like, memory_format=torch.contiguous_format)
    return _same(x, name, like.dtype, like.shape, like.device)


def _glr_shape(dtype, T, batch, n, lds, lengths, device):
    import torch
    if lengths is not None:
        _packed_rows(_same(lengths, "lengths", torch.int32, (batch,), device), "lengths")
    return snn_glr(T, batch, n, dtype, *lds, _at(lengths))


def snn_glr_forward(z, x, h0=None, lengths=None, keep=False, h=None, h_last=None):
    """h_t = a_t h_{t-1} + (1 - a_t) x_t with a = sigmoid(z), over [T][batch][n] from the state h0 [batch][n] (float32; None: zeros).

    Returns h, the last state and, with keep, the states that snn_glr_backward needs (else None).  h and h_last: tensors for the results;
    h_last may be h0 itself, a state that is updated in place."""
    import torch
    T, batch, n = _sequences(z, "z")
    dtype, device = _type(z, "z"), z.device
    _same(x, "x", z.dtype, z.shape, device)
    if h0 is not None:
        _packed_rows(_same(h0, "h0", torch.float32, (batch, n), device), "h0")
    h = _out(h, "h", z)
    p = _glr_shape(dtype, T, batch, n, (_ld(z, "z"), _ld(x, "x"), _ld(h, "h"), 0, 0), lengths, device)
    at, space = _launch(device, _entry("snn_glr_workspace")(C.byref(p)))
    if h_last is None:
        h_last = torch.empty((batch, n), dtype=torch.float32, device=device)
    else:
        _packed_rows(_same(h_last, "h_last", torch.float32, (batch, n), device), "h_last")
    kept = torch.empty((-(-T // GLR_INTERVAL), batch, n), dtype=torch.float32, device=device) if keep else None
    _run("snn_glr_forward", C.byref(at), C.byref(p), _at(z), _at(x), _at(h0), _at(h), _at(h_last), _at(kept))
    return h, h_last, kept


def snn_glr_backward(z, x, kept, dh, dh_last=None, lengths=None, dz=None, dx=None):
    """Gradients of z, x and h0 from those of h (and of the last state).  z and x: the forward pass's, or both Packed.
    dz and dx: tensors for the results (the halves of a projection's gradient, say)."""
    import torch
    T, batch, n = _sequences(dh, "dh")
    dtype, device = _type(dh, "dh"), dh.device
    packed = isinstance(z, Packed)
    if packed != isinstance(x, Packed):
        raise TypeError("z and x must be tensors both, or Packed both")
    _packed_rows(_same(kept, "kept", torch.float32, (-(-T // GLR_INTERVAL), batch, n), device), "kept")
    if dh_last is not None:
        _packed_rows(_same(dh_last, "dh_last", torch.float32, (batch, n), device), "dh_last")
    if packed:
        for name, v in (("z", z), ("x", x)):
            _same(v.codes, f"the codes of {name}", torch.int8, (T, batch, n), device)
            _same(v.exps, f"the exponents of {name}", torch.uint8, (T, batch, -(-n // PACK_BLOCK)), device)
        inputs = [C.byref(snn_packed(_at(v.codes), _at(v.exps), _ld(v.codes, f"the codes of {name}"), _ld(v.exps, f"the exponents of {name}")))
                  for name, v in (("z", z), ("x", x))]
        lds = (0, 0)
    else:
        _same(z, "z", dh.dtype, dh.shape, device)
        _same(x, "x", dh.dtype, dh.shape, device)
        inputs, lds = [_at(z), _at(x)], (_ld(z, "z"), _ld(x, "x"))
    dz, dx = _out(dz, "dz", dh), _out(dx, "dx", dh)
    dh0 = torch.empty((batch, n), dtype=torch.float32, device=device)
    p = _glr_shape(dtype, T, batch, n, (*lds, _ld(dh, "dh"), _ld(dz, "dz"), _ld(dx, "dx")), lengths, device)
    at, space = _launch(device, _entry("snn_glr_workspace")(C.byref(p)))
    _run("snn_glr_backward_packed" if packed else "snn_glr_backward", C.byref(at), C.byref(p), *inputs, _at(kept), _at(dh), _at(dh_last),
         _at(dz), _at(dx), _at(dh0))
    return dz, dx, dh0


def snn_pack(x):
    """Rows [..., n] in 8 bits: blocks of 32 elements of a row share a power of two as their step."""
    import torch
    dtype, n = _type(x, "x"), x.shape[-1] if x.dim() else 0
    if n < 1:
        raise ValueError(f"x must be rows of at least one element, got {tuple(x.shape)}")
    at, _ = _launch(x.device)
    codes = torch.empty(x.shape, dtype=torch.int8, device=x.device)
    exps = torch.empty((*x.shape[:-1], -(-n // PACK_BLOCK)), dtype=torch.uint8, device=x.device)
    _run("snn_pack", C.byref(at), dtype, x.numel() // n, n, _ld(x, "x"), _at(x), _at(codes), _at(exps))
    return Packed(codes, exps)


def snn_unpack(packed, dtype=None):
    """The values of rows in 8 bits, as float32 (or bfloat16)."""
    import torch
    codes, exps = packed
    n = codes.shape[-1] if codes.dim() else 0
    if n < 1:
        raise ValueError(f"the codes must be rows of at least one element, got {tuple(codes.shape)}")
    _packed_rows(_same(codes, "the codes", torch.int8, codes.shape, codes.device), "the codes")
    _packed_rows(_same(exps, "the exponents", torch.uint8, (*codes.shape[:-1], -(-n // PACK_BLOCK)), codes.device), "the exponents")
    x = torch.empty(codes.shape, dtype=torch.float32 if dtype is None else dtype, device=codes.device)
    kind = _type(x, "the values")
    at, _ = _launch(codes.device)
    _run("snn_unpack", C.byref(at), kind, codes.numel() // n, n, n, _at(codes), _at(exps), _at(x))
    return x


def _vocab_shape(h, w, targets):
    import torch
    dtype = _type(h, "h")
    if h.dim() != 2 or w.dim() != 2:
        raise ValueError(f"h must be [rows][d] and w [vocab][d], got {tuple(h.shape)} and {tuple(w.shape)}")
    _same(w, "w", h.dtype, (w.shape[0], h.shape[1]), h.device)
    _packed_rows(_same(targets, "targets", torch.int32, (h.shape[0],), h.device), "targets")
    return snn_vocab(h.shape[0], h.shape[1], w.shape[0], dtype, _ld(h, "h"), _ld(w, "w"))


def snn_vocab_loss(h, w, targets):
    """Softmax cross entropy of rows h [rows][d] against w [vocab][d]; a target outside 0..vocab-1 makes a row without a loss.

    Returns the losses [rows] (float32) and the state [rows][3] that snn_vocab_loss_grad takes."""
    import torch
    p = _vocab_shape(h, w, targets)
    at, space = _launch(h.device, _entry("snn_vocab_workspace")(C.byref(p), 0))
    loss = torch.empty(p.rows, dtype=torch.float32, device=h.device)
    state = torch.empty((p.rows, 3), dtype=torch.float32, device=h.device)
    _run("snn_vocab_loss", C.byref(at), C.byref(p), _at(h), _at(w), _at(targets), _at(loss), _at(state))
    return loss, state


def snn_vocab_loss_grad(h, w, targets, state, dloss=None):
    """Gradients of h and w from those of the losses, dloss [rows] (float32; None: of the mean over the rows that have a target)."""
    import torch
    p = _vocab_shape(h, w, targets)
    _packed_rows(_same(state, "state", torch.float32, (p.rows, 3), h.device), "state")
    if dloss is not None:
        _packed_rows(_same(dloss, "dloss", torch.float32, (p.rows,), h.device), "dloss")
    at, space = _launch(h.device, _entry("snn_vocab_workspace")(C.byref(p), 1))
    dh = torch.empty((p.rows, p.d), dtype=h.dtype, device=h.device)
    dw = torch.empty((p.vocab, p.d), dtype=h.dtype, device=h.device)
    _run("snn_vocab_loss_grad", C.byref(at), C.byref(p), _at(h), _at(w), _at(targets), _at(state), _at(dloss), _at(dh), _at(dw))
    return dh, dw


def _ld_heads(x, name):
    """Elements between consecutive rows of [T][batch][heads][d], a row being all its heads one after the other."""
    T, batch, heads, d = x.shape
    if x.is_contiguous():
        return heads * d
    if (d > 1 and x.stride(3) != 1) or (heads > 1 and x.stride(2) != d):
        raise ValueError(f"{name}: the heads of a row must follow one another")
    return _ld(x.as_strided((T, batch, heads * d), (x.stride(0), x.stride(1), 1)), name)


def _delta_shape(q, k, v, g, beta, lengths, scale):
    import torch
    if q.dim() != 4 or v.dim() != 4:
        raise ValueError(f"q, k must be [T][batch][key_heads][dk] and v [T][batch][heads][dv], got {tuple(q.shape)} and {tuple(v.shape)}")
    (T, batch, key_heads, dk), (heads, dv), dtype, device = q.shape, v.shape[2:], _type(q, "q"), q.device
    _same(k, "k", q.dtype, q.shape, device)
    _same(v, "v", q.dtype, (T, batch, heads, dv), device)
    _packed_rows(_same(g, "g", torch.float32, (T, batch, heads), device), "g")
    _packed_rows(_same(beta, "beta", torch.float32, (T, batch, heads), device), "beta")
    if lengths is not None:
        _packed_rows(_same(lengths, "lengths", torch.int32, (batch,), device), "lengths")
    return snn_delta(T, batch, heads, key_heads, dk, dv, dtype, dk ** -0.5 if scale is None and dk else scale or 0.0, _ld_heads(q, "q"), _ld_heads(k, "k"),
                     _ld_heads(v, "v"), 0, 0, 0, 0, _at(lengths)), (batch, heads, dk, dv)


def snn_delta_forward(q, k, v, g, beta, s0=None, lengths=None, scale=None, keep=False, o=None, s_last=None):
    """S_t = exp(g_t) S_{t-1} + k_t u_t^T with u_t = beta_t (v_t - exp(g_t) S_{t-1}^T k_t), and o_t = scale S_t^T q_t, over q, k [T][batch][key_heads][dk],
    v [T][batch][heads][dv], g, beta [T][batch][heads] (float32) from the state s0 [batch][heads][dk][dv] (float32; None: zeros).
    scale: 1 / sqrt(dk) unless given; consecutive heads share queries and keys where there are more of them than of keys.

    Returns o, the last state and, with keep, the states that snn_delta_backward needs (else None).  o and s_last: tensors for the results;
    s_last may be s0 itself, a state that is updated in place, and o may be v."""
    import torch
    p, state = _delta_shape(q, k, v, g, beta, lengths, scale)
    device = q.device
    if s0 is not None:
        _packed_rows(_same(s0, "s0", torch.float32, state, device), "s0")
    o = _out(o, "o", v)
    p.ld_o = _ld_heads(o, "o")
    at, space = _launch(device, _entry("snn_delta_workspace")(C.byref(p), 0))
    if s_last is None:
        s_last = torch.empty(state, dtype=torch.float32, device=device)
    else:
        _packed_rows(_same(s_last, "s_last", torch.float32, state, device), "s_last")
    kept = torch.empty((-(-p.T // DELTA_INTERVAL), *state), dtype=torch.float32, device=device) if keep else None
    _run("snn_delta_forward", C.byref(at), C.byref(p), _at(q), _at(k), _at(v), _at(g), _at(beta), _at(s0), _at(o), _at(s_last), _at(kept))
    return o, s_last, kept


def snn_delta_backward(q, k, v, g, beta, kept, do, ds_last=None, lengths=None, scale=None, dq=None, dk=None, dv=None):
    """Gradients of q, k, v, g, beta and s0 from those of o (and of the last state); q to beta, lengths and scale as the forward pass had them.
    dq, dk and dv: tensors for the results (the parts of a projection's gradient, say), which may be q, k and v themselves."""
    import torch
    p, state = _delta_shape(q, k, v, g, beta, lengths, scale)
    device = q.device
    _packed_rows(_same(kept, "kept", torch.float32, (-(-p.T // DELTA_INTERVAL), *state), device), "kept")
    _same(do, "do", v.dtype, v.shape, device)
    if ds_last is not None:
        _packed_rows(_same(ds_last, "ds_last", torch.float32, state, device), "ds_last")
    dq, dk, dv = _out(dq, "dq", q), _out(dk, "dk", k), _out(dv, "dv", v)
    p.ld_o, p.ld_dq, p.ld_dk, p.ld_dv = _ld_heads(do, "do"), _ld_heads(dq, "dq"), _ld_heads(dk, "dk"), _ld_heads(dv, "dv")
    dg, dbeta = torch.empty_like(g), torch.empty_like(beta)
    ds0 = torch.empty(state, dtype=torch.float32, device=device)
    at, space = _launch(device, _entry("snn_delta_workspace")(C.byref(p), 1))
    _run("snn_delta_backward", C.byref(at), C.byref(p), _at(q), _at(k), _at(v), _at(g), _at(beta), _at(kept), _at(do), _at(ds_last), _at(dq), _at(dk), _at(dv),
         _at(dg), _at(dbeta), _at(ds0))
    return dq, dk, dv, dg, dbeta, ds0


def _rows(x, name):
    n = x.shape[-1] if x.dim() else 0
    if n < 1:
        raise ValueError(f"{name} must be rows of at least one element, got {tuple(x.shape)}")
    return x.numel() // n, n


def snn_norm_forward(x, w=None, residual=None, eps=1e-6, packed=False, y=None, total=None):
    """y = w s / sqrt(mean(s^2) + eps) for rows s = x + residual (or x) [..., n]; w [n] (None: ones).

    Returns y (packed: as Packed, in 8 bits) and s, which is what snn_norm_backward takes: x itself without a residual.  y and total: tensors
    for the results; total may be x or residual itself, a sum that is updated in place, and so may y."""
    import torch
    dtype, device, (rows, n) = _type(x, "x"), x.device, _rows(x, "x")
    if w is not None:
        _packed_rows(_same(w, "w", x.dtype, (n,), device), "w")
    ld_r = ld_total = 0
    if residual is None:
        if total is not None:
            raise ValueError("total without a residual: it would be x")
    else:
        ld_r = _ld(_same(residual, "residual", x.dtype, x.shape, device), "residual")
        total = _out(total, "total", x)
        ld_total = _ld(total, "total")
    at, _ = _launch(device)
    if packed:
        if y is not None:
            raise ValueError("y in 8 bits is a new Packed")
        y = Packed(torch.empty(x.shape, dtype=torch.int8, device=device),
                   torch.empty((*x.shape[:-1], -(-n // PACK_BLOCK)), dtype=torch.uint8, device=device))
        to, ld_y = (_at(y.codes), _at(y.exps)), 0
    else:
        y = _out(y, "y", x)
        to, ld_y = (_at(y),), _ld(y, "y")
    p = snn_norm(rows, n, dtype, eps, _ld(x, "x"), ld_r, ld_total, ld_y, 0, 0)
    _run("snn_norm_forward_packed" if packed else "snn_norm_forward", C.byref(at), C.byref(p), _at(x), _at(residual), _at(w), _at(total), *to)
    return y, x if residual is None else total


def snn_norm_backward(total, w, dy, dtotal=None, eps=1e-6, dx=None):
    """Gradients of x (and of the residual: the same) and of w (None without one) from those of y and, if given, of s = total itself.
    dx: a tensor for the result, which may be total, dy or dtotal itself."""
    import torch
    dtype, device, (rows, n) = _type(total, "total"), total.device, _rows(total, "total")
    _same(dy, "dy", total.dtype, total.shape, device)
    if w is not None:
        _packed_rows(_same(w, "w", total.dtype, (n,), device), "w")
    ld_dtotal = 0
    if dtotal is not None:
        ld_dtotal = _ld(_same(dtotal, "dtotal", total.dtype, total.shape, device), "dtotal")
    dx = _out(dx, "dx", total)
    dw = None if w is None else torch.empty((n,), dtype=total.dtype, device=device)
    p = snn_norm(rows, n, dtype, eps, 0, 0, _ld(total, "total"), _ld(dy, "dy"), ld_dtotal, _ld(dx, "dx"))
    at, space = _launch(device, _entry("snn_norm_workspace")(C.byref(p)) if w is not None else 0)
    _run("snn_norm_backward", C.byref(at), C.byref(p), _at(total), _at(w), _at(dy), _at(dtotal), _at(dx), _at(dw))
    return dx, dw


class AdamwPlan:
    """Tensors that snn_adamw_step moves, with their moments: params, m, v, copies as snn_adamw_plan was given them."""

    def __init__(self, params, m, v, copies, tensors, device):
        self.params, self.m, self.v, self.copies, self.tensors, self.device = params, m, v, copies, tensors, device
        self.held = [y for x in (*params, *m, *v, *copies) if x is not None for y in (x if isinstance(x, Packed) else (x,))]
        # (the memory that `tensors` points at stays, also where a tensor is given other memory)
        self.memory = [x.detach() for x in self.held]
        self.addresses = [x.data_ptr() for x in self.held]

    def names(self):
        """What each of `held` is called."""
        for name, xs in (("params", self.params), ("m", self.m), ("v", self.v), ("copies", self.copies)):
            for i, x in enumerate(xs):
                if isinstance(x, Packed):
                    yield f"the codes of {name}[{i}]"
                    yield f"the exponents of {name}[{i}]"
                elif x is not None:
                    yield f"{name}[{i}]"


def snn_adamw_moments(params, bits=32):
    """m and v of tensors that have not been moved yet: zeros, float32 in their shapes, or (bits=8) Packed: codes in their shapes, an
    exponent for 32 elements.  Each of the two is one array for all, of which the tensors' parts are views."""
    import torch
    if bits not in (8, 32):
        raise ValueError(f"moments of 8 or 32 bits, not {bits}")
    params = list(params)
    counts = [p.numel() for p in params]
    blocks = [-(-n // PACK_BLOCK) for n in counts]

    def views(dtype, sizes):
        whole = torch.zeros(sum(sizes), dtype=dtype, device=params[0].device if params else None)
        return whole.split(sizes) if sizes else []

    def moment():
        values = views(torch.float32 if bits == 32 else torch.int8, [PACK_BLOCK * k for k in blocks])
        values = [x[:n].view(p.shape) for x, n, p in zip(values, counts, params)]
        return values if bits == 32 else [Packed(x, e) for x, e in zip(values, views(torch.uint8, blocks))]

    return moment(), moment()


def snn_adamw_plan(params, m, v, copies=None):
    """What snn_adamw_step needs of its tensors, once for all steps: params (float32 or bfloat16, contiguous), their moments (snn_adamw_moments,
    or tensors like those) and, if wanted, copies in bfloat16 of params in float32 (None in the list: no copy of that one).
    The tensors are held, and changed in place by each step; where any of them has been given other memory since (x.data = ...), a step
    raises: that needs a new plan."""
    import torch
    params, m, v = list(params), list(m), list(v)
    copies = [None] * len(params) if copies is None else list(copies)
    if not len(params) == len(m) == len(v) == len(copies):
        raise ValueError(f"{len(params)} params, {len(m)} m, {len(v)} v, {len(copies)} copies")
    tensors = (snn_adamw_tensor * len(params))()
    for i, (p, a, b, c, t) in enumerate(zip(params, m, v, copies, tensors)):
        kind, device = _type(p, f"params[{i}]"), params[0].device
        _packed_rows(_same(p, f"params[{i}]", p.dtype, p.shape, device), f"params[{i}]")
        if isinstance(a, Packed) != isinstance(b, Packed):
            raise TypeError(f"m[{i}] and v[{i}] must be tensors both, or Packed both")
        for name, x in (("m", a), ("v", b)):
            if isinstance(x, Packed):
                if x.codes.numel() != p.numel():
                    raise ValueError(f"the codes of {name}[{i}] must be as many as params[{i}] has elements")
                _packed_rows(_same(x.codes, f"the codes of {name}[{i}]", torch.int8, x.codes.shape, device), f"the codes of {name}[{i}]")
                _packed_rows(_same(x.exps, f"the exponents of {name}[{i}]", torch.uint8, (-(-p.numel() // PACK_BLOCK),), device),
                             f"the exponents of {name}[{i}]")
            else:
                _packed_rows(_same(x, f"{name}[{i}]", torch.float32, p.shape, device), f"{name}[{i}]")
        if isinstance(a, Packed):
            t.m, t.m_exps, t.v, t.v_exps = _at(a.codes), _at(a.exps), _at(b.codes), _at(b.exps)
        else:
            t.m, t.v = _at(a), _at(b)
        if c is not None:
            if p.dtype != torch.float32:
                raise TypeError(f"copies[{i}] is of params in {p.dtype}: only float32 has copies")
            t.copy = _at(_packed_rows(_same(c, f"copies[{i}]", torch.bfloat16, p.shape, device), f"copies[{i}]"))
        t.p, t.n, t.dtype_p = _at(p), p.numel(), kind
    return AdamwPlan(params, m, v, copies, tensors, params[0].device if params else None)


def snn_adamw_step(plan, grads, step, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, grad_scale=None):
    """One step of AdamW: params, moments and copies of the plan change in place.  grads: a gradient (float32 or bfloat16, contiguous) for each of
    params.  step: 1, 2, ..., or an int32 tensor [1] on the device with the number of steps taken, which the call counts up (a step in a
    graph, which keeps lr and the other numbers as they were when it was captured).  grad_scale: float32 [1] that the gradients are multiplied by first.  A plan is for one call at a time."""
    import torch
    grads = list(grads)
    if len(grads) != len(plan.params):
        raise ValueError(f"{len(grads)} grads for {len(plan.params)} params")
    if not grads:
        return
    device = plan.device
    now = list(map(torch.Tensor.data_ptr, plan.held))
    if now != plan.addresses:
        name = next(name for name, a, b in zip(plan.names(), now, plan.addresses) if a != b)
        raise ValueError(f"{name} has other memory than when the plan was made")
    kinds = {torch.float32: SNN_F32, torch.bfloat16: SNN_BF16}
    for i, (g, p, t) in enumerate(zip(grads, plan.params, plan.tensors)):
        kind = kinds.get(g.dtype)
        if kind is None:
            raise TypeError(f"grads[{i}] must be float32 or bfloat16, got {g.dtype}")
        t.dtype_g = kind
        if g.shape != p.shape or g.device != device or not g.is_contiguous():
            _packed_rows(_same(g, f"grads[{i}]", g.dtype, p.shape, device), f"grads[{i}]")
        t.g = g.data_ptr()
    how = snn_adamw(lr, betas[0], betas[1], eps, weight_decay, 0, None, None)
    if isinstance(step, torch.Tensor):
        how.step_on_device = _at(_same(step, "step", torch.int32, (1,), device))
    else:
        how.step = step
    if grad_scale is not None:
        how.grad_scale = _at(_same(grad_scale, "grad_scale", torch.float32, (1,), device))
    at, space = _launch(device, _entry("snn_adamw_workspace")(C.byref(how)))
    _run("snn_adamw_step", C.byref(at), C.byref(how), plan.tensors, len(grads))
