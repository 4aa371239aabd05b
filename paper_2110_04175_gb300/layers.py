"""Layer operators of n workers' models on one GPU, with 8-bit activation checkpoints.

The binding of ``include/relaylayers.h``: the functions have the C names, take
torch tensors on the current CUDA device, write into the outputs that they are
given, and enqueue on ``stream`` (default: torch's current stream).  Activations
are ``[n][tokens][d]`` (worker, token, feature) in bf16, fp16 or fp32 with the
features next to one another and any strides otherwise; weights and their
gradients are fp32 and may be views of the workers' model rows.

Unlike the C calls, these see the tensors' types, sizes and devices: a tensor
that does not fit raises ValueError, and the library's own refusals RelayError.
A tensor that another stream still uses has to be kept, as with any torch call,
by the caller (``Tensor.record_stream``).
"""
from __future__ import annotations

import ctypes
import struct

from ._native import RelayError, _check, _load, _stream

RELAY_BF16, RELAY_FP16, RELAY_FP32 = 0, 1, 2
RELAY_NORM_MAX_D = 32768


_pack_rows = struct.Struct("=qqq").pack  # relay_rows, as bytes: a fifth of the time of a ctypes.Structure

_vp, _i32, _i64, _f32, _rows_p = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_char_p
_SHAPE = [_i32, _i32, _i64, _i64]  # type, n, tokens, d
_SIGNATURES = {
    "relay_checkpoint_pitch": (_i64, [_i64]),
    "relay_checkpoint_pack": (ctypes.c_int, _SHAPE + [_rows_p, _vp, _vp, _vp]),
    "relay_checkpoint_unpack": (ctypes.c_int, _SHAPE + [_vp, _vp, _rows_p, _vp]),
    "relay_rms_norm": (ctypes.c_int, _SHAPE + [_rows_p, _rows_p, _vp, _i64, _f32, _rows_p, _rows_p, _vp, _vp, _vp,
                                               _vp]),
    "relay_rms_norm_backward_workspace": (_i64, [_i32, _i64, _i64]),
    "relay_rms_norm_backward": (ctypes.c_int, _SHAPE + [_rows_p, _rows_p, _vp, _i64, _vp, _rows_p, _vp, _vp, _vp,
                                                        _rows_p, _vp, _i64, _vp, _i64, _vp]),
    "relay_gated": (ctypes.c_int, _SHAPE + [_rows_p, _rows_p, _rows_p, _vp, _vp, _vp, _vp, _vp]),
    "relay_gated_backward": (ctypes.c_int, _SHAPE + [_rows_p, _rows_p, _rows_p, _vp, _vp, _vp, _vp, _rows_p, _rows_p,
                                                     _vp, _vp, _vp]),
    "relay_weight_grad_workspace": (_i64, [_i32, _i32, _i64, _i64, _i64, _rows_p]),
    "relay_weight_grad": (ctypes.c_int, [_i32, _i32, _i64, _i64, _i64, _rows_p, _vp, _vp, _vp, _i64, _vp, _vp, _i64,
                                         _i64, _vp, _i64, _vp]),
    "relay_block_norm": (ctypes.c_int, _SHAPE + [_rows_p, _rows_p, _rows_p, _vp, _i64, _vp, _i64, _vp, _i64, _f32, _rows_p,
                                                 _rows_p, _vp, _vp, _vp, _vp]),
    "relay_block_norm_backward_workspace": (_i64, [_i32, _i64, _i64]),
    "relay_block_norm_backward": (ctypes.c_int, _SHAPE + [_rows_p] * 5 + [_vp, _i64] * 3 + [_vp, _vp] + [_rows_p] * 3 +
                                  [_vp, _i64] * 3 + [_vp, _i64, _vp]),
    "relay_orthogonalise_workspace": (_i64, [_i32, _i64, _i64]),
    "relay_orthogonalise": (ctypes.c_int, [_i32, _i64, _i64, _vp, _i64, _i64, _i32, _f32, _f32, _vp, _i64, _i64, _vp, _i64,
                                           _vp]),
    "relay_recurrence_workspace": (_i64, [_i32, _i64, _i64]),
    "relay_recurrence": (ctypes.c_int, _SHAPE + [_rows_p, _rows_p, _vp, _i64, _vp, _vp, _rows_p, _vp, _i64, _vp, _i64,
                                                 _vp]),
    "relay_recurrence_backward": (ctypes.c_int, _SHAPE + [_rows_p, _rows_p, _rows_p, _rows_p, _vp, _i64, _vp, _i64, _vp,
                                                          _vp, _rows_p, _rows_p, _vp, _i64, _vp, _i64, _vp]),
}

_lib = None
torch = None  # the module, and the types' numbers, once a call needs them (importing the package does not)
_TYPES: dict = {}


def _library():
    """The library with these calls' signatures set."""
    global _lib, torch
    lib = _load()
    if lib is not _lib:
        import torch as module
        torch = module
        _TYPES.update({torch.bfloat16: RELAY_BF16, torch.float16: RELAY_FP16, torch.float32: RELAY_FP32})
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return lib


# ------------------------------------------------------------------ arguments


def _refuse(name, t, what):
    got = f"{t.dtype} {tuple(t.shape)} on {t.device}" if isinstance(t, torch.Tensor) else repr(t)
    raise ValueError(f"{name}: {what}, not {got}")


def _on_device(name, t, dtype):
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype:
        _refuse(name, t, f"a {dtype} tensor is needed")
    if not t.is_cuda or t.get_device() != torch._C._cuda_getDevice():
        _refuse(name, t, "a tensor on the current CUDA device is needed")


def _shape_of(name, t):
    """(type, n, tokens, d) of an activation that sets the call's sizes."""
    if not isinstance(t, torch.Tensor) or t.dtype not in _TYPES or t.dim() != 3:
        _refuse(name, t, "a bf16, fp16 or fp32 tensor [n][tokens][d] is needed")
    return (_TYPES[t.dtype], *t.shape)


def _rows(name, t, dtype, shape):
    """relay_rows of an activation of the call's type and shape; None for None."""
    if t is None:
        return None
    _on_device(name, t, dtype)
    if t.shape != shape:
        _refuse(name, t, f"the shape {tuple(shape)} is needed")
    worker, token, one = t.stride()
    if one != 1 and shape[2] > 1:
        _refuse(name, t, f"features next to one another are needed (strides {t.stride()})")
    return _pack_rows(t.data_ptr(), worker, token)


def _weights(name, t, n, d):
    """(pointer, stride from worker to worker) of fp32 [n][d] values."""
    _on_device(name, t, torch.float32)
    if t.shape != (n, d):
        _refuse(name, t, f"the shape {(n, d)} is needed")
    worker, one = t.stride()
    if one != 1 and d > 1:
        _refuse(name, t, f"values next to one another are needed (strides {t.stride()})")
    return t.data_ptr(), worker


def _state(name, t, n, d):
    """The same of a state that may be left out."""
    return (None, 0) if t is None else _weights(name, t, n, d)


def _plain(name, t, dtype, shape):
    """Pointer of a contiguous tensor; None for None."""
    if t is None:
        return None
    _on_device(name, t, dtype)
    if t.shape != shape or not t.is_contiguous():
        _refuse(name, t, f"a contiguous tensor of shape {tuple(shape)} is needed")
    return t.data_ptr()


def _held(name, ckpt, n, tokens, d):
    """(codes, scales) pointers of an ActivationCheckpoint or a (codes, scales) pair; Nones for None."""
    if ckpt is None:
        return None, None
    if isinstance(ckpt, ActivationCheckpoint):
        if ckpt.d != d:
            raise ValueError(f"{name}: a checkpoint of {d} features is needed, not of {ckpt.d}")
        ckpt = ckpt.codes, ckpt.scales
    pitch = -(-d // 128) * 128
    return (_plain(name + " codes", ckpt[0], torch.int8, (n, tokens, pitch)),
            _plain(name + " scales", ckpt[1], torch.uint8, (n, tokens, pitch // 32)))


def _workspace(name, t):
    if not isinstance(t, torch.Tensor) or not t.is_contiguous():
        _refuse(name, t, "a contiguous tensor is needed")
    _on_device(name, t, t.dtype)
    return t.data_ptr() or None, t.numel() * t.element_size()


def _bytes(size, what):
    size = int(size)
    if size < 0:
        raise RelayError(size, what)
    return size


# ------------------------------------------------------------------ the calls


def relay_checkpoint_pitch(d: int) -> int:
    """Codes per row of a checkpoint of d features (scale bytes: a 32nd of it)."""
    return _bytes(_library().relay_checkpoint_pitch(int(d)), "relay_checkpoint_pitch")


class ActivationCheckpoint:
    """Device buffers of one activation [n][tokens][d] held in 8 bits: ``codes``
    (int8 [n][tokens][pitch]) and ``scales`` (uint8 [n][tokens][pitch / 32]),
    33/32 byte a feature.  Calls that take a checkpoint also take the pair."""

    def __init__(self, n: int, tokens: int, d: int, device="cuda"):
        pitch = relay_checkpoint_pitch(d)  # (loads torch)
        self.n, self.tokens, self.d = n, tokens, d
        self.codes = torch.empty(n, tokens, pitch, dtype=torch.int8, device=device)
        self.scales = torch.empty(n, tokens, pitch // 32, dtype=torch.uint8, device=device)

    def pack(self, x, stream=None):
        """Puts x away."""
        relay_checkpoint_pack(x, self, stream)
        return self

    def unpack(self, dtype=None, stream=None):
        """A new tensor of the values held (bf16 unless a type is given)."""
        out = torch.empty(self.n, self.tokens, self.d, dtype=dtype or torch.bfloat16, device=self.codes.device)
        relay_checkpoint_unpack(self, out, stream)
        return out


def relay_checkpoint_pack(x, checkpoint, stream=None):
    """x to 8 bits."""
    lib = _library()
    shape = type_, n, tokens, d = _shape_of("x", x)
    _check(lib.relay_checkpoint_pack(*shape, _rows("x", x, x.dtype, x.shape),
                                            *_held("checkpoint", checkpoint, n, tokens, d), _stream(stream)),
           "relay_checkpoint_pack")


def relay_checkpoint_unpack(checkpoint, out, stream=None):
    """8 bits to `out` (exact in bf16 and fp32)."""
    lib = _library()
    shape = type_, n, tokens, d = _shape_of("out", out)
    _check(lib.relay_checkpoint_unpack(*shape, *_held("checkpoint", checkpoint, n, tokens, d),
                                              _rows("out", out, out.dtype, out.shape), _stream(stream)),
           "relay_checkpoint_unpack")


def relay_rms_norm(x, weight, y, eps: float, residual=None, total=None, rstd=None, checkpoint=None, stream=None):
    """total = x + residual; y = total rstd weight with rstd = 1 / sqrt(mean(total^2) + eps).

    weight: fp32 [n][d].  total, rstd (fp32 [n][tokens]) and checkpoint (total rstd in
    8 bits: what relay_rms_norm_backward and, with the weight as column_scale,
    relay_weight_grad read) are written where given.  total may be x or residual itself."""
    lib = _library()
    shape = type_, n, tokens, d = _shape_of("x", x)
    dt, sh = x.dtype, x.shape
    _check(lib.relay_rms_norm(*shape, _rows("x", x, dt, sh), _rows("residual", residual, dt, sh),
                                     *_weights("weight", weight, n, d), eps, _rows("total", total, dt, sh),
                                     _rows("y", y, dt, sh), _plain("rstd", rstd, torch.float32, (n, tokens)),
                                     *_held("checkpoint", checkpoint, n, tokens, d), _stream(stream)),
           "relay_rms_norm")


def relay_rms_norm_backward_workspace(n: int, tokens: int, d: int) -> int:
    """Bytes of workspace for relay_rms_norm_backward."""
    return _bytes(_library().relay_rms_norm_backward_workspace(n, tokens, d), "relay_rms_norm_backward_workspace")


def relay_rms_norm_backward(dy, weight, rstd, dx, dweight, workspace, total=None, checkpoint=None, dtotal=None,
                            lengths=None, stream=None):
    """dx (the gradient of x and of the residual) and dweight (fp32 [n][d], overwritten).

    The normalised rows come from `checkpoint`, or from `total` and rstd.  dtotal: the
    gradient that reaches the sum past the norm.  lengths (int32 [n]): the rows of each
    worker that count."""
    lib = _library()
    shape = type_, n, tokens, d = _shape_of("dy", dy)
    dt, sh = dy.dtype, dy.shape
    _check(lib.relay_rms_norm_backward(
        *shape, _rows("dy", dy, dt, sh), _rows("dtotal", dtotal, dt, sh), *_weights("weight", weight, n, d),
        _plain("rstd", rstd, torch.float32, (n, tokens)), _rows("total", total, dt, sh),
        *_held("checkpoint", checkpoint, n, tokens, d), _plain("lengths", lengths, torch.int32, (n,)),
        _rows("dx", dx, dt, sh), *_weights("dweight", dweight, n, d), *_workspace("workspace", workspace),
        _stream(stream)), "relay_rms_norm_backward")


def relay_gated(gate, up, out, gate_checkpoint=None, up_checkpoint=None, stream=None):
    """out = gate sigma(gate) up; gate and up in 8 bits too where their checkpoints are given."""
    lib = _library()
    shape = type_, n, tokens, d = _shape_of("gate", gate)
    dt, sh = gate.dtype, gate.shape
    _check(lib.relay_gated(*shape, _rows("gate", gate, dt, sh), _rows("up", up, dt, sh),
                                  _rows("out", out, dt, sh), *_held("gate_checkpoint", gate_checkpoint, n, tokens, d),
                                  *_held("up_checkpoint", up_checkpoint, n, tokens, d), _stream(stream)),
           "relay_gated")


def relay_gated_backward(dout, dgate, dup, gate=None, up=None, gate_checkpoint=None, up_checkpoint=None,
                         out_checkpoint=None, stream=None):
    """The gradients of gate and up, from those rows or from both checkpoints; the
    activation formed again from them, in 8 bits, where out_checkpoint is given."""
    lib = _library()
    shape = type_, n, tokens, d = _shape_of("dout", dout)
    dt, sh = dout.dtype, dout.shape
    _check(lib.relay_gated_backward(
        *shape, _rows("dout", dout, dt, sh), _rows("gate", gate, dt, sh), _rows("up", up, dt, sh),
        *_held("gate_checkpoint", gate_checkpoint, n, tokens, d),
        *_held("up_checkpoint", up_checkpoint, n, tokens, d), _rows("dgate", dgate, dt, sh),
        _rows("dup", dup, dt, sh), *_held("out_checkpoint", out_checkpoint, n, tokens, d), _stream(stream)),
        "relay_gated_backward")


def relay_weight_grad_workspace(n: int, tokens: int, outputs: int, inputs: int, dy=None) -> int:
    """Bytes of workspace for relay_weight_grad: for the tensor dy, or without one enough
    for any type and strides and for fewer tokens too.  Rows that are not bf16 on 16-byte
    boundaries are copied into it as bf16 terms; for those that are it is 0, or the split
    sums of few outputs."""
    lib = _library()
    if dy is None:
        return _bytes(lib.relay_weight_grad_workspace(RELAY_FP32, n, tokens, outputs, inputs, None),
                      "relay_weight_grad_workspace")
    type_, *_ = _shape_of("dy", dy)
    return _bytes(lib.relay_weight_grad_workspace(type_, n, tokens, outputs, inputs,
                                                  _rows("dy", dy, dy.dtype, (n, tokens, outputs))),
                  "relay_weight_grad_workspace")


def relay_weight_grad(dy, checkpoint, dweight, workspace, column_scale=None, lengths=None, stream=None):
    """dweight[i][o][k] = column_scale[i][k] sum_t dy[i][t][o] xhat[i][t][k], overwritten
    (fp32 [n][outputs][inputs], a view of any strides with the inputs next to one another);
    xhat: the layer's inputs, in 8 bits."""
    lib = _library()
    type_, n, tokens, outputs = _shape_of("dy", dy)
    if not isinstance(dweight, torch.Tensor) or dweight.dim() != 3:
        _refuse("dweight", dweight, "an fp32 tensor [n][outputs][inputs] is needed")
    inputs = dweight.shape[2]
    _rows("dweight", dweight, torch.float32, (n, outputs, inputs))
    worker_stride, row_stride, _ = dweight.stride()
    scale, scale_stride = (None, 0) if column_scale is None else _weights("column_scale", column_scale, n, inputs)
    _check(lib.relay_weight_grad(
        type_, n, tokens, outputs, inputs, _rows("dy", dy, dy.dtype, dy.shape),
        *_held("checkpoint", checkpoint, n, tokens, inputs), scale, scale_stride,
        _plain("lengths", lengths, torch.int32, (n,)), dweight.data_ptr(), worker_stride, row_stride,
        *_workspace("workspace", workspace), _stream(stream)), "relay_weight_grad")


def relay_block_norm(x, residual, post, pre, total, y, eps: float, gate=None, scale=None, rstd=None, checkpoint=None,
                     stream=None):
    """From one block to the next: total = scale residual + sigma(gate) norm(x) post; y = norm(total) pre.

    post, pre, scale: fp32 [n][d]; without gate or scale they are 1.  total (the sum, which may be
    x or residual itself, or None), rstd (fp32 [2][n][tokens]: the two norms' factors, what
    relay_block_norm_backward reads) and checkpoint (norm(total) in 8 bits: with pre as
    column_scale what relay_weight_grad reads) are written where given."""
    lib = _library()
    shape = type_, n, tokens, d = _shape_of("x", x)
    dt, sh = x.dtype, x.shape
    _check(lib.relay_block_norm(
        *shape, _rows("x", x, dt, sh), _rows("gate", gate, dt, sh), _rows("residual", residual, dt, sh),
        *_weights("post", post, n, d), *_weights("pre", pre, n, d), *_state("scale", scale, n, d), eps,
        _rows("total", total, dt, sh), _rows("y", y, dt, sh), _plain("rstd", rstd, torch.float32, (2, n, tokens)),
        *_held("checkpoint", checkpoint, n, tokens, d), _stream(stream)), "relay_block_norm")


def relay_block_norm_backward_workspace(n: int, tokens: int, d: int) -> int:
    """Bytes of workspace for relay_block_norm_backward."""
    return _bytes(_library().relay_block_norm_backward_workspace(n, tokens, d), "relay_block_norm_backward_workspace")


def relay_block_norm_backward(dy, x, residual, post, pre, rstd, dx, dresidual, dpost, dpre, workspace, gate=None, scale=None,
                              dtotal=None, dgate=None, dscale=None, lengths=None, stream=None):
    """The gradients of relay_block_norm: dx, dresidual and (with a gate) dgate, and dpost, dpre
    and, where given, dscale (fp32 [n][d], overwritten).  dtotal: the gradient that reaches the
    sum past the second norm.  lengths (int32 [n]): the rows of each worker that count."""
    lib = _library()
    shape = type_, n, tokens, d = _shape_of("dy", dy)
    dt, sh = dy.dtype, dy.shape
    _check(lib.relay_block_norm_backward(
        *shape, _rows("dy", dy, dt, sh), _rows("dtotal", dtotal, dt, sh), _rows("x", x, dt, sh), _rows("gate", gate, dt, sh),
        _rows("residual", residual, dt, sh), *_weights("post", post, n, d), *_weights("pre", pre, n, d),
        *_state("scale", scale, n, d), _plain("rstd", rstd, torch.float32, (2, n, tokens)),
        _plain("lengths", lengths, torch.int32, (n,)), _rows("dx", dx, dt, sh), _rows("dgate", dgate, dt, sh),
        _rows("dresidual", dresidual, dt, sh), *_weights("dpost", dpost, n, d), *_weights("dpre", dpre, n, d),
        *_state("dscale", dscale, n, d), *_workspace("workspace", workspace), _stream(stream)), "relay_block_norm_backward")


def relay_recurrence_workspace(n: int, tokens: int, d: int) -> int:
    """Bytes of workspace for relay_recurrence and relay_recurrence_backward (0 for most shapes)."""
    return _bytes(_library().relay_recurrence_workspace(n, tokens, d), "relay_recurrence_workspace")


def relay_recurrence(gate, value, out, workspace, initial=None, last=None, begins=None, lengths=None, stream=None):
    """out_t = f_t out_{t-1} + (1 - f_t) value_t along the tokens, f = sigma(gate).

    initial, last: the states (fp32 [n][d]) before the first and behind the last token; the same
    tensor may be both.  begins (uint8 [n][tokens]): not 0 where a sequence begins, which takes
    nothing from before it.  lengths (int32 [n]): the rows of each worker that count; the others
    get 0 and leave the state as it is."""
    lib = _library()
    shape = type_, n, tokens, d = _shape_of("gate", gate)
    dt, sh = gate.dtype, gate.shape
    _check(lib.relay_recurrence(
        *shape, _rows("gate", gate, dt, sh), _rows("value", value, dt, sh), *_state("initial", initial, n, d),
        _plain("begins", begins, torch.uint8, (n, tokens)), _plain("lengths", lengths, torch.int32, (n,)),
        _rows("out", out, dt, sh), *_state("last", last, n, d), *_workspace("workspace", workspace), _stream(stream)),
        "relay_recurrence")


def relay_recurrence_backward(dout, gate, value, out, dgate, dvalue, workspace, initial=None, dlast=None, dinitial=None,
                              begins=None, lengths=None, stream=None):
    """The gradients of gate and value from the rows of the forward pass, and, where dinitial
    (fp32 [n][d]) is given, of the state before the first token.  dlast: the gradient that
    reaches the last state."""
    lib = _library()
    shape = type_, n, tokens, d = _shape_of("dout", dout)
    dt, sh = dout.dtype, dout.shape
    _check(lib.relay_recurrence_backward(
        *shape, _rows("dout", dout, dt, sh), _rows("gate", gate, dt, sh), _rows("value", value, dt, sh),
        _rows("out", out, dt, sh), *_state("initial", initial, n, d), *_state("dlast", dlast, n, d),
        _plain("begins", begins, torch.uint8, (n, tokens)), _plain("lengths", lengths, torch.int32, (n,)),
        _rows("dgate", dgate, dt, sh), _rows("dvalue", dvalue, dt, sh), *_state("dinitial", dinitial, n, d),
        *_workspace("workspace", workspace), _stream(stream)), "relay_recurrence_backward")


def relay_orthogonalise_workspace(n: int, rows: int, columns: int) -> int:
    """Bytes of workspace for relay_orthogonalise."""
    return _bytes(_library().relay_orthogonalise_workspace(n, rows, columns), "relay_orthogonalise_workspace")


def relay_orthogonalise(update, out, workspace, steps: int = 5, eps: float = 1e-7, scale: float = 1.0, stream=None):
    """out = scale times `update` (fp32 [n][rows][columns], views of any strides with the columns next
    to one another) made nearly orthogonal, each matrix by itself, by Newton-Schulz steps from
    update / (|update| + eps).  out may be update itself."""
    lib = _library()
    for name, t in (("update", update), ("out", out)):
        if not isinstance(t, torch.Tensor) or t.dim() != 3:
            _refuse(name, t, "an fp32 tensor [n][rows][columns] is needed")
    n, rows, columns = update.shape
    _rows("update", update, torch.float32, update.shape)
    _rows("out", out, torch.float32, update.shape)
    _check(lib.relay_orthogonalise(n, rows, columns, update.data_ptr(), *update.stride()[:2], steps, eps, scale, out.data_ptr(),
                                   *out.stride()[:2], *_workspace("workspace", workspace), _stream(stream)),
           "relay_orthogonalise")
