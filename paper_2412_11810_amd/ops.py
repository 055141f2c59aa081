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
    for name in ("snn_glr_forward", "snn_glr_backward", "snn_glr_backward_packed", "snn_pack", "snn_unpack", "snn_vocab_loss",
                 "snn_vocab_loss_grad"):
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
