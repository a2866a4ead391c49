"""Operators around the expert layer (declared in include/moe_ovl.h): the norm in front of it, the router, the gated
activation and the 8-bit integer product, by the names that the C interface gives them.

Every tensor is the caller's, outputs and workspaces too; nothing is allocated and nothing is waited for.  What the C
side cannot see of a tensor -- its shape, type, device and the order of its columns -- is checked here, and a tensor
that does not fit raises MoeOvlError with ERR_INVALID_ARG before anything is launched.  Work goes to the current stream
of the tensors' device, or to `stream`; tensors used on a stream that is not the current one are recorded on it.

Nothing is recorded for autograd: outputs carry no gradient, and the two gradients are called by hand or from the backward of a
torch.autograd.Function (whose forward runs with gradients off).  An input that requires a gradient while they are on gets a warning.
"""
from __future__ import annotations

import ctypes as C
import struct
import warnings

import torch

from . import binding as B
from .binding import MoeOvlError

DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
SCORE_SOFTMAX, SCORE_SIGMOID = 0, 1
SCORES = {"softmax": SCORE_SOFTMAX, "sigmoid": SCORE_SIGMOID}
FLAG_QUANT_MATMUL_TEST_NO_LOADS = 1
MAX_ROW, MAX_ROUTED, MAX_TOP_K, MAX_QUANT_K = 32768, 1024, 32, 131056

_u32, _i32, _i64, _f32, _ptr = C.c_uint32, C.c_int32, C.c_int64, C.c_float, C.c_void_p


def _struct(name, text):
    """The C structure that `text` spells out, and in `pack` the same layout as bytes: a call builds its arguments with that,
    which takes a third of the time of filling the structure."""
    kinds = {"u": _u32, "i": _i32, "l": _i64, "f": _f32, "p": _ptr, "z": C.c_size_t}
    codes = {"u": "I", "i": "i", "l": "q", "f": "f", "p": "P", "z": "N"}
    fields = [(f, part[0]) for part in text.split(";") for f in part[1:].replace(",", " ").split()]
    t = type(name, (C.Structure,), {"_fields_": [(f, kinds[k]) for f, k in fields]})
    packer = struct.Struct("@" + "".join(codes[k] for _, k in fields) + "0q")
    assert packer.size == C.sizeof(t)
    t.pack = packer.pack
    t.bytes = packer.size
    return t


NormArgs = _struct("NormArgs", "u struct_size;i device,rows,d,dtype,weight_dtype;f eps;u flags;"
                   "p x,residual,weight,residual_out,y,q,scale,rstd;l x_stride,residual_stride,residual_out_stride,y_stride,q_stride;p stream")
NormBackwardArgs = _struct("NormBackwardArgs", "u struct_size;i device,rows,d,dtype,weight_dtype;p dy,h,weight,rstd,d_residual,dx,dweight,workspace;"
                           "z workspace_bytes;l dy_stride,h_stride,d_residual_stride,dx_stride;p stream")
SwigluArgs = _struct("SwigluArgs", "u struct_size;i device,rows,f,dtype;u flags;p gate_up,q,scale;l gate_up_stride,q_stride;p stream")
RouteArgs = _struct("RouteArgs", "u struct_size;i device,rows,num_experts,top_k,dtype,score,num_groups,top_groups,group_best,renormalise;f gate_scale;"
                    "p logits,bias,expert,gate,counts;l logits_stride;p stream")
RouteBackwardArgs = _struct("RouteBackwardArgs", "u struct_size;i device,rows,num_experts,top_k,dtype,score,renormalise;f gate_scale;u flags;"
                            "p logits,expert,dgate,dlogits;l logits_stride,dlogits_stride;p stream")
QuantMatmulArgs = _struct("QuantMatmulArgs", "u struct_size;i device,rows,n,k,num_experts,out_dtype,wait_timeout_us;u flags;"
                          "p a,a_scale,b,b_scale,expert_counts,out,status;l a_stride,b_stride,out_stride;p stream")


def _refuse(where: str, what: str):
    raise MoeOvlError(B.ERR_INVALID_ARG, f"{where}: {what}")


def _device(where, t) -> int:
    device = t.get_device() if isinstance(t, torch.Tensor) else -1
    if device < 0:
        _refuse(where, "tensors have to be on a CUDA device")
    return device


def _dtype(where, name, t) -> int:
    d = DTYPES.get(t.dtype)
    if d is None:
        _refuse(where, f"{name} has to be bfloat16, float16 or float32, not {t.dtype}")
    return d


def _matrix(where, name, t, shape, dtype, device) -> int:
    """Row stride of a tensor of two dimensions whose columns lie next to each other."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device:
        _refuse(where, f"{name} has to be {list(shape)} {dtype} on cuda:{device}, not {list(t.shape)} {t.dtype} on {t.device}")
    s0, s1 = t.stride()
    if s1 == 1 and s0 >= shape[1]:
        return s0
    rows, cols = shape
    if (s1 != 1 and cols > 1) or s0 < 0:
        _refuse(where, f"{name}: the columns of a row have to lie next to each other (strides {t.stride()})")
    if rows > 1 and s0 < cols:
        _refuse(where, f"{name}: rows must not overlap (strides {t.stride()})")
    return s0


def _vector(where, name, t, shape, dtype, device) -> None:
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device or not t.is_contiguous():
        _refuse(where, f"{name} has to be a contiguous {list(shape)} {dtype} on cuda:{device}, not {list(t.shape)} {t.dtype} on {t.device}")


def _gradient_lost(where: str) -> None:
    if torch.is_grad_enabled():
        warnings.warn(f"{where} records nothing for autograd: an input requires a gradient that the outputs will not carry (call it under torch.no_grad() "
                      "and take the gradient with the operator's own backward call, where it has one)", stacklevel=3)


def _at(t) -> int:
    return 0 if t is None else t.data_ptr()


def _stream(device: int, stream, *tensors) -> int:
    current = torch._C._cuda_getCurrentRawStream(device)
    if stream is None or stream.cuda_stream == current:
        return current
    if stream.device_index != device:
        _refuse("stream", f"it belongs to cuda:{stream.device_index}, the tensors to cuda:{device}")
    for t in tensors:
        if t is not None:
            t.record_stream(stream)
    return stream.cuda_stream


def _done(rc: int, where: str) -> None:
    if rc != B.OK:
        raise MoeOvlError(rc, where)


def _call(where: str, function, kind, *values) -> None:
    try:
        args = kind.pack(kind.bytes, *values)
    except struct.error as e:           # a number that its field does not hold
        _refuse(where, str(e))
    _done(function(args), where)


def moe_ovl_add_norm(*, x, weight, eps: float = 1e-6, residual=None, residual_out=None, y=None, q=None, scale=None, rstd=None,
                     stream=None) -> None:
    """RMS norm of x + residual, rounded to x's type: h -> residual_out; h * rstd * weight -> y and / or, in 8 bits with a
    scale per row, q and scale; rstd for the backward pass."""
    where = "moe_ovl_add_norm"
    dev, dt = _device(where, x), _dtype(where, "x", x)
    if x.dim() != 2:
        _refuse(where, "x has to be [rows, d]")
    shape, kind, wkind = x.shape, x.dtype, weight.dtype
    rows, d = shape
    sx = _matrix(where, "x", x, shape, kind, dev)
    if wkind is not kind and wkind is not torch.float32:
        _refuse(where, f"weight has to be {kind} or float32, not {wkind}")
    _vector(where, "weight", weight, (d,), wkind, dev)
    sr = _matrix(where, "residual", residual, shape, kind, dev) if residual is not None else 0
    so = _matrix(where, "residual_out", residual_out, shape, kind, dev) if residual_out is not None else 0
    sy = _matrix(where, "y", y, shape, kind, dev) if y is not None else 0
    sq = _matrix(where, "q", q, shape, torch.int8, dev) if q is not None else 0
    if x.requires_grad or weight.requires_grad or (residual is not None and residual.requires_grad):
        _gradient_lost(where)
    if scale is not None:
        _vector(where, "scale", scale, (rows,), torch.float32, dev)
    if rstd is not None:
        _vector(where, "rstd", rstd, (rows,), torch.float32, dev)
    _call(where, B.load().moe_ovl_add_norm, NormArgs, dev, rows, d, dt, DTYPES[wkind], eps, 0, x.data_ptr(), _at(residual), weight.data_ptr(),
          _at(residual_out), _at(y), _at(q), _at(scale), _at(rstd), sx, sr, so, sy, sq,
          _stream(dev, stream, x, weight, residual, residual_out, y, q, scale, rstd))


def moe_ovl_add_norm_workspace_bytes(rows: int, d: int) -> int:
    n = C.c_size_t(0)
    _done(B.load().moe_ovl_add_norm_workspace_bytes(int(rows), int(d), C.byref(n)), "moe_ovl_add_norm_workspace_bytes")
    return int(n.value)


def moe_ovl_add_norm_backward(*, dy, h, weight, rstd, dx, dweight=None, d_residual=None, workspace=None, stream=None) -> None:
    """Gradient of moe_ovl_add_norm: dx (of x and of residual alike, with what arrives at residual_out added) and dweight.
    `h` is what the forward pass normalised; dweight needs a workspace of moe_ovl_add_norm_workspace_bytes bytes."""
    where = "moe_ovl_add_norm_backward"
    dev, dt = _device(where, dy), _dtype(where, "dy", dy)
    if dy.dim() != 2:
        _refuse(where, "dy has to be [rows, d]")
    shape = dy.shape
    rows, d = shape
    sy = _matrix(where, "dy", dy, shape, dy.dtype, dev)
    sh = _matrix(where, "h", h, shape, dy.dtype, dev)
    sx = _matrix(where, "dx", dx, shape, dy.dtype, dev)
    sr = _matrix(where, "d_residual", d_residual, shape, dy.dtype, dev) if d_residual is not None else 0
    if weight.dtype is not dy.dtype and weight.dtype is not torch.float32:
        _refuse(where, f"weight has to be {dy.dtype} or float32, not {weight.dtype}")
    _vector(where, "weight", weight, (d,), weight.dtype, dev)
    _vector(where, "rstd", rstd, (rows,), torch.float32, dev)
    if dweight is not None:
        _vector(where, "dweight", dweight, (d,), torch.float32, dev)
    nbytes = 0
    if workspace is not None:
        if not workspace.is_cuda or workspace.device.index != dev or not workspace.is_contiguous():
            _refuse(where, f"workspace has to be contiguous on cuda:{dev}")
        nbytes = workspace.numel() * workspace.element_size()
    _call(where, B.load().moe_ovl_add_norm_backward, NormBackwardArgs, dev, rows, d, dt, DTYPES[weight.dtype], dy.data_ptr(), h.data_ptr(),
          weight.data_ptr(), rstd.data_ptr(), _at(d_residual), dx.data_ptr(), _at(dweight), _at(workspace), nbytes, sy, sh, sr, sx,
          _stream(dev, stream, dy, h, weight, rstd, d_residual, dx, dweight, workspace))


def moe_ovl_swiglu_quant(*, gate_up, q, scale, stream=None) -> None:
    """silu(gate) * up of [rows, 2F] (gate in the first F columns) in 8 bits with a scale per row."""
    where = "moe_ovl_swiglu_quant"
    dev, dt = _device(where, gate_up), _dtype(where, "gate_up", gate_up)
    if gate_up.dim() != 2 or gate_up.shape[1] % 2:
        _refuse(where, "gate_up has to be [rows, 2F]")
    rows, f = gate_up.shape[0], gate_up.shape[1] // 2
    sg = _matrix(where, "gate_up", gate_up, gate_up.shape, gate_up.dtype, dev)
    sq = _matrix(where, "q", q, (rows, f), torch.int8, dev)
    _vector(where, "scale", scale, (rows,), torch.float32, dev)
    if gate_up.requires_grad:
        _gradient_lost(where)
    _call(where, B.load().moe_ovl_swiglu_quant, SwigluArgs, dev, rows, f, dt, 0, gate_up.data_ptr(), q.data_ptr(), scale.data_ptr(), sg, sq,
          _stream(dev, stream, gate_up, q, scale))


def moe_ovl_route(*, logits, expert, gate, counts=None, bias=None, score: int = SCORE_SOFTMAX, num_groups: int = 1, top_groups: int = 1,
                  group_best: int = 1, renormalise: bool = True, gate_scale: float = 1.0, stream=None) -> None:
    """The top experts of every row of logits and their gates; top_k is expert.shape[1].  counts[e]: how often e was chosen."""
    where = "moe_ovl_route"
    dev, dt = _device(where, logits), _dtype(where, "logits", logits)
    if logits.dim() != 2 or expert.dim() != 2:
        _refuse(where, "logits have to be [rows, experts], expert [rows, top_k]")
    rows, e = logits.shape
    k = expert.shape[1]
    sl = _matrix(where, "logits", logits, logits.shape, logits.dtype, dev)
    _vector(where, "expert", expert, (rows, k), torch.int32, dev)
    _vector(where, "gate", gate, expert.shape, torch.float32, dev)
    if bias is not None:
        _vector(where, "bias", bias, (e,), torch.float32, dev)
    if counts is not None:
        _vector(where, "counts", counts, (e,), torch.int32, dev)
    if logits.requires_grad:
        _gradient_lost(where)
    _call(where, B.load().moe_ovl_route, RouteArgs, dev, rows, e, k, dt, score, num_groups, top_groups, group_best, 1 if renormalise else 0, gate_scale,
          logits.data_ptr(), _at(bias), expert.data_ptr(), gate.data_ptr(), _at(counts), sl, _stream(dev, stream, logits, expert, gate, bias, counts))


def moe_ovl_route_backward(*, logits, expert, dgate, dlogits, score: int = SCORE_SOFTMAX, renormalise: bool = True, gate_scale: float = 1.0,
                           stream=None) -> None:
    """dlogits from the gradient of the gates, the choice held fixed."""
    where = "moe_ovl_route_backward"
    dev, dt = _device(where, logits), _dtype(where, "logits", logits)
    if logits.dim() != 2 or expert.dim() != 2:
        _refuse(where, "logits have to be [rows, experts], expert [rows, top_k]")
    rows, e = logits.shape
    k = expert.shape[1]
    sl = _matrix(where, "logits", logits, logits.shape, logits.dtype, dev)
    so = _matrix(where, "dlogits", dlogits, logits.shape, logits.dtype, dev)
    _vector(where, "expert", expert, (rows, k), torch.int32, dev)
    _vector(where, "dgate", dgate, expert.shape, torch.float32, dev)
    _call(where, B.load().moe_ovl_route_backward, RouteBackwardArgs, dev, rows, e, k, dt, score, 1 if renormalise else 0, gate_scale, 0,
          logits.data_ptr(), expert.data_ptr(), dgate.data_ptr(), dlogits.data_ptr(), sl, so, _stream(dev, stream, logits, expert, dgate, dlogits))


def moe_ovl_quant_matmul(*, a, a_scale, b, b_scale, out, status, expert_counts=None, wait_timeout_us: int = 0, flags: int = 0,
                         stream=None) -> None:
    """out = (a @ b^T) * a_scale[:, None] * b_scale in 8-bit integers.  b is [n, k] (or [1, n, k]), or with expert_counts [experts, n, k]
    and the rows of a are grouped by expert.  `status`: 4 int32 that the caller clears once (torch.zeros)."""
    where = "moe_ovl_quant_matmul"
    dev = _device(where, a)
    if a.dim() != 2 or b.dim() not in (2, 3):
        _refuse(where, "a has to be [rows, k], b [n, k] or [experts, n, k]")
    rows, k = a.shape
    experts = 0
    if expert_counts is not None:
        if b.dim() != 3:
            _refuse(where, "with expert_counts b has to be [experts, n, k]")
        experts = b.shape[0]
        if experts < 1:
            _refuse(where, "b has no experts")
        _vector(where, "expert_counts", expert_counts, (experts,), torch.int32, dev)
    elif b.dim() == 3 and b.shape[0] != 1:
        _refuse(where, "several experts need expert_counts")
    n = b.shape[-2]
    sa = _matrix(where, "a", a, a.shape, torch.int8, dev)
    if b.shape[-1] != k or b.dtype is not torch.int8 or b.get_device() != dev or b.stride(-1) != 1:
        _refuse(where, f"b has to be [..., {n}, {k}] int8 on cuda:{dev} with its columns next to each other")
    sb = b.stride(0) if n == 1 and experts > 1 else b.stride(-2)        # one channel each: the experts are the rows
    if sb < k or (experts > 1 and b.stride(0) != n * sb):
        _refuse(where, "the rows of b have to lie at one distance, across experts too")
    dt = _dtype(where, "out", out)
    so = _matrix(where, "out", out, (rows, n), out.dtype, dev)
    _vector(where, "a_scale", a_scale, (rows,), torch.float32, dev)
    _vector(where, "b_scale", b_scale, b.shape[:-1], torch.float32, dev)
    _vector(where, "status", status, (4,), torch.int32, dev)
    if a_scale.requires_grad or b_scale.requires_grad:
        _gradient_lost(where)
    _call(where, B.load().moe_ovl_quant_matmul, QuantMatmulArgs, dev, rows, n, k, experts, dt, wait_timeout_us, flags, a.data_ptr(), a_scale.data_ptr(),
          b.data_ptr(), b_scale.data_ptr(), _at(expert_counts), out.data_ptr(), status.data_ptr(), sa, sb, so,
          _stream(dev, stream, a, a_scale, b, b_scale, expert_counts, out, status))
