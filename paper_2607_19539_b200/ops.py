"""Operators around the expert layer (declared in include/moe_ovl.h): the norm in front of it, the router, the gated
activation and the 8-bit integer product; experts in 8-bit floats with a scale per block; the experts' products with their
gradients, the gradients' norm and clipping.  They go by the names that the C interface gives them.

Every tensor is the caller's, outputs and workspaces too; nothing is allocated and nothing is waited for.  What the C
side cannot see of a tensor -- its shape, type, device and the order of its columns -- is checked here, and a tensor
that does not fit raises MoeOvlError with ERR_INVALID_ARG before anything is launched.  Work goes to the current stream
of the tensors' device, or to `stream`; tensors used on a stream that is not the current one are recorded on it.

Nothing is recorded for autograd: outputs carry no gradient, and the gradients are called by hand or from the backward of a
torch.autograd.Function (whose forward runs with gradients off).  An input that requires a gradient while they are on gets a warning.
"""
from __future__ import annotations

import ctypes as C
import struct
import warnings
from array import array
from operator import attrgetter

import torch

from . import binding as B
from .binding import MoeOvlError

DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
SCORE_SOFTMAX, SCORE_SIGMOID = 0, 1
SCORES = {"softmax": SCORE_SOFTMAX, "sigmoid": SCORE_SIGMOID}
FLAG_QUANT_MATMUL_TEST_NO_LOADS = 1
FLAG_MATMUL_TEST_NO_LOADS = 1
MAX_ROW, MAX_ROUTED, MAX_TOP_K, MAX_QUANT_K = 32768, 1024, 32, 131056
MAX_GROUPS, MAX_MATMUL, MAX_TENSORS = 1024, 16777216, 65536
BLOCK = 128             # values of K that share a scale of moe_ovl_block_matmul
FLOAT8 = torch.float8_e4m3fn

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

GroupedMatmulArgs = _struct("GroupedMatmulArgs", "u struct_size;i device,rows,n,k,num_experts,dtype,out_dtype,transposed,wait_timeout_us;u flags;"
                            "p a,b,expert_counts,out,status;l a_stride,b_stride,b_expert_stride,out_stride;p stream")
GroupedMatmulBackwardArgs = _struct("GroupedMatmulBackwardArgs", "u struct_size;i device,rows,n,k,num_experts,dtype,out_dtype,accumulate,wait_timeout_us;u flags;"
                                    "p dy,x,expert_counts,dweight,status,workspace;z workspace_bytes;l dy_stride,x_stride,dweight_stride,dweight_expert_stride;"
                                    "p stream")
BlockQuantArgs = _struct("BlockQuantArgs", "u struct_size;i device,depth,rows,k,dtype,gated,tiles;u flags;p x,q,scale;l x_stride,q_stride,x_far,q_far;p stream")
BlockMatmulArgs = _struct("BlockMatmulArgs", "u struct_size;i device,rows,n,k,num_experts,out_dtype,wait_timeout_us;u flags;"
                          "p a,a_scale,b,b_scale,expert_counts,out,status;l a_stride,b_stride,b_expert_stride,out_stride;p stream")
GradsArgs = _struct("GradsArgs", "u struct_size;i device,num_tensors;u flags;p grads,out,sizes,dtypes,norm;f max_norm,eps;p workspace;z workspace_bytes;p stream")


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


def _matrices(where, name, t, shape, dtype, device):
    """Strides between rows and between matrices of a tensor of three dimensions (or of two: one matrix) whose columns lie next to each other."""
    depth, rows, cols = shape
    if (t.shape != shape and (depth != 1 or t.shape != shape[1:])) or t.dtype is not dtype or t.get_device() != device:
        _refuse(where, f"{name} has to be {list(shape)} {dtype} on cuda:{device}, not {list(t.shape)} {t.dtype} on {t.device}")
    strides = t.stride()
    far, s0, s1 = strides if len(strides) == 3 else (0, *strides)
    if (s1 != 1 and cols > 1) or s0 < 0:
        _refuse(where, f"{name}: the columns of a row have to lie next to each other (strides {strides})")
    if rows > 1 and s0 < cols:
        _refuse(where, f"{name}: rows must not overlap (strides {strides})")
    return s0, far


def _apart(where, name, shape, row_stride, far) -> None:
    """Refuses matrices that are written and would overlap: either matrices lie behind each other or their rows interleave."""
    depth, rows, cols = shape
    if depth < 2 or rows * cols == 0:
        return
    if far >= (rows - 1) * row_stride + cols or (far >= cols and (rows == 1 or row_stride >= (depth - 1) * far + cols)):
        return
    _refuse(where, f"{name}: the matrices of the experts must not overlap")


def _experts(where, name, t, expert_counts, device) -> int:
    if expert_counts is None:
        if t.dim() == 3 and t.shape[0] != 1:
            _refuse(where, "several experts need expert_counts")
        return 0
    if t.dim() != 3 or t.shape[0] < 1:
        _refuse(where, f"with expert_counts {name} has to have three dimensions, the experts first")
    _vector(where, "expert_counts", expert_counts, (t.shape[0],), torch.int32, device)
    return t.shape[0]


def _workspace(where, workspace, device) -> int:
    if workspace.get_device() != device or not workspace.is_contiguous():
        _refuse(where, f"workspace has to be contiguous on cuda:{device}")
    return workspace.numel() * workspace.element_size()


def moe_ovl_grouped_matmul(*, a, b, out, status, expert_counts=None, transposed: bool = False, wait_timeout_us: int = 0, flags: int = 0, stream=None) -> None:
    """out = a @ b^T in 16-bit floats, rows of a grouped by expert: b [experts, n, k], or with `transposed` a @ b, b [experts, k, n].  Without expert_counts
    b is one matrix.  The gradient of a is moe_ovl_grouped_matmul(a=dout, b=b, transposed=not transposed)."""
    where = "moe_ovl_grouped_matmul"
    dev = _device(where, a)
    if a.dim() != 2 or b.dim() not in (2, 3) or out.dim() != 2:
        _refuse(where, "a has to be [rows, k], b [n, k] or [experts, n, k], out [rows, n]")
    if a.dtype not in (torch.bfloat16, torch.float16):
        _refuse(where, f"a has to be bfloat16 or float16, not {a.dtype}")
    if out.dtype is not a.dtype and out.dtype is not torch.float32:
        _refuse(where, f"out has to be {a.dtype} or float32, not {out.dtype}")
    rows, k = a.shape
    experts = _experts(where, "b", b, expert_counts, dev)
    n = b.shape[-1] if transposed else b.shape[-2]
    sa = _matrix(where, "a", a, a.shape, a.dtype, dev)
    sb, far = _matrices(where, "b", b, (max(experts, 1), k, n) if transposed else (max(experts, 1), n, k), a.dtype, dev)
    so = _matrix(where, "out", out, (rows, n), out.dtype, dev)
    _vector(where, "status", status, (4,), torch.int32, dev)
    if a.requires_grad or b.requires_grad:
        _gradient_lost(where)
    _call(where, B.load().moe_ovl_grouped_matmul, GroupedMatmulArgs, dev, rows, n, k, experts, DTYPES[a.dtype], DTYPES[out.dtype], 1 if transposed else 0,
          wait_timeout_us, flags, a.data_ptr(), b.data_ptr(), _at(expert_counts), out.data_ptr(), status.data_ptr(), sa, sb, far, so,
          _stream(dev, stream, a, b, expert_counts, out, status))


def moe_ovl_grouped_matmul_workspace_bytes(num_experts: int) -> int:
    n = C.c_size_t(0)
    _done(B.load().moe_ovl_grouped_matmul_workspace_bytes(int(num_experts), C.byref(n)), "moe_ovl_grouped_matmul_workspace_bytes")
    return int(n.value)


def moe_ovl_grouped_matmul_backward(*, dy, x, dweight, status, workspace, expert_counts=None, accumulate: bool = False, wait_timeout_us: int = 0,
                                    flags: int = 0, stream=None) -> None:
    """dweight[e] = dy_e^T @ x_e over the rows of each expert, or added to what dweight holds.  The workspace has
    moe_ovl_grouped_matmul_workspace_bytes bytes."""
    where = "moe_ovl_grouped_matmul_backward"
    dev = _device(where, dy)
    if dy.dim() != 2 or x.dim() != 2 or dweight.dim() not in (2, 3):
        _refuse(where, "dy has to be [rows, n], x [rows, k], dweight [n, k] or [experts, n, k]")
    if dy.dtype not in (torch.bfloat16, torch.float16):
        _refuse(where, f"dy has to be bfloat16 or float16, not {dy.dtype}")
    if dweight.dtype is not dy.dtype and dweight.dtype is not torch.float32:
        _refuse(where, f"dweight has to be {dy.dtype} or float32, not {dweight.dtype}")
    rows, n = dy.shape
    k = x.shape[1]
    experts = _experts(where, "dweight", dweight, expert_counts, dev)
    shape = (max(experts, 1), n, k)
    sy = _matrix(where, "dy", dy, dy.shape, dy.dtype, dev)
    sx = _matrix(where, "x", x, (rows, k), dy.dtype, dev)
    sw, far = _matrices(where, "dweight", dweight, shape, dweight.dtype, dev)
    _apart(where, "dweight", shape, sw, far)
    _vector(where, "status", status, (4,), torch.int32, dev)
    nbytes = _workspace(where, workspace, dev)
    _call(where, B.load().moe_ovl_grouped_matmul_backward, GroupedMatmulBackwardArgs, dev, rows, n, k, experts, DTYPES[dy.dtype], DTYPES[dweight.dtype],
          1 if accumulate else 0, wait_timeout_us, flags, dy.data_ptr(), x.data_ptr(), _at(expert_counts), dweight.data_ptr(), status.data_ptr(),
          workspace.data_ptr(), nbytes, sy, sx, sw, far, _stream(dev, stream, dy, x, expert_counts, dweight, status, workspace))


def moe_ovl_block_quant(*, x, q, scale, gated: bool = False, tiles: bool = False, stream=None) -> None:
    """x in 8-bit floats with a scale for each 128 values of a row (or with `tiles` for each 128 x 128 of a matrix, x [n, k] or [experts, n, k]).  With `gated`
    x is [rows, 2k] and silu(gate) * up is what becomes 8 bits, gate in the first k columns."""
    where = "moe_ovl_block_quant"
    dev, dt = _device(where, x), _dtype(where, "x", x)
    if x.dim() != 2 and not (tiles and x.dim() == 3):
        _refuse(where, "x has to be [rows, k], or with tiles [n, k] or [experts, n, k]")
    if gated and (tiles or x.shape[1] % 2):
        _refuse(where, "with gated x has to be [rows, 2k], and tiles cannot be asked for")
    depth, rows, k = x.shape[0] if x.dim() == 3 else 1, x.shape[-2], x.shape[-1] // 2 if gated else x.shape[-1]
    if k < 1 or depth < 1:
        _refuse(where, f"x has no values: {list(x.shape)}")
    sx, x_far = _matrices(where, "x", x, (depth, rows, x.shape[-1]), x.dtype, dev)
    if q.dim() != x.dim():
        _refuse(where, f"q has to have {x.dim()} dimensions as x")
    sq, q_far = _matrices(where, "q", q, (depth, rows, k), FLOAT8, dev)
    _apart(where, "q", (depth, rows, k), sq, q_far)
    blocks = -(-k // BLOCK)
    _vector(where, "scale", scale, (*x.shape[:-2], -(-rows // BLOCK), blocks) if tiles else (rows, blocks), torch.float32, dev)
    if x.requires_grad:
        _gradient_lost(where)
    _call(where, B.load().moe_ovl_block_quant, BlockQuantArgs, dev, depth, rows, k, dt, 1 if gated else 0, 1 if tiles else 0, 0, x.data_ptr(), q.data_ptr(),
          scale.data_ptr(), sx, sq, x_far, q_far, _stream(dev, stream, x, q, scale))


def moe_ovl_block_matmul(*, a, a_scale, b, b_scale, out, status, expert_counts=None, wait_timeout_us: int = 0, flags: int = 0, stream=None) -> None:
    """out = a @ b^T in 8-bit floats, a with a scale per row and 128 values, b with one per 128 x 128 (as moe_ovl_block_quant gives them).  b is [n, k], or
    with expert_counts [experts, n, k] and the rows of a are grouped by expert."""
    where = "moe_ovl_block_matmul"
    dev = _device(where, a)
    if a.dim() != 2 or b.dim() not in (2, 3) or out.dim() != 2:
        _refuse(where, "a has to be [rows, k], b [n, k] or [experts, n, k], out [rows, n]")
    rows, k = a.shape
    experts = _experts(where, "b", b, expert_counts, dev)
    n, blocks = b.shape[-2], -(-k // BLOCK)
    sa = _matrix(where, "a", a, a.shape, FLOAT8, dev)
    sb, far = _matrices(where, "b", b, (max(experts, 1), n, k), FLOAT8, dev)
    dt = _dtype(where, "out", out)
    so = _matrix(where, "out", out, (rows, n), out.dtype, dev)
    _vector(where, "a_scale", a_scale, (rows, blocks), torch.float32, dev)
    _vector(where, "b_scale", b_scale, (*b.shape[:-2], -(-n // BLOCK), blocks), torch.float32, dev)
    _vector(where, "status", status, (4,), torch.int32, dev)
    if a_scale.requires_grad or b_scale.requires_grad:
        _gradient_lost(where)
    _call(where, B.load().moe_ovl_block_matmul, BlockMatmulArgs, dev, rows, n, k, experts, dt, wait_timeout_us, flags, a.data_ptr(), a_scale.data_ptr(),
          b.data_ptr(), b_scale.data_ptr(), _at(expert_counts), out.data_ptr(), status.data_ptr(), sa, sb, far, so,
          _stream(dev, stream, a, a_scale, b, b_scale, expert_counts, out, status))


def _dense(t) -> bool:
    """Whether a tensor's values fill a stretch of memory, in whatever order."""
    if t.is_contiguous():
        return True
    size = 1
    for stride, n in sorted((s, n) for s, n in zip(t.stride(), t.shape) if n != 1):
        if stride != size:
            return False
        size *= n
    return True


_dtype_of, _shape_of = attrgetter("dtype"), attrgetter("shape")


def _tensor_list(where, name, tensors, device):
    """Addresses, sizes and types of a list of tensors as arrays, and whether all are contiguous."""
    if not all(isinstance(t, torch.Tensor) for t in tensors):
        _refuse(where, f"{name} has to be a list of tensors")
    if any(d != device for d in map(torch.Tensor.get_device, tensors)):
        _refuse(where, f"every tensor of {name} has to be on cuda:{device}, not {[str(t.device) for t in tensors if t.get_device() != device][0]}")
    contiguous = all(map(torch.Tensor.is_contiguous, tensors))
    if not contiguous:
        for t in tensors:
            if not _dense(t):
                _refuse(where, f"the tensors of {name} have to fill the memory that they span (strides {t.stride()} of {list(t.shape)})")
    kinds = [DTYPES.get(t, -1) for t in map(_dtype_of, tensors)]
    if -1 in kinds:
        _refuse(where, f"every tensor of {name} has to be bfloat16, float16 or float32, not {tensors[kinds.index(-1)].dtype}")
    at, sizes = list(map(torch.Tensor.data_ptr, tensors)), list(map(torch.Tensor.numel, tensors))
    real = at if 0 not in sizes else [a for a, n in zip(at, sizes) if n]
    if len(set(real)) != len(real):
        _refuse(where, f"a tensor is twice in {name}")
    return array("Q", at), array("q", sizes), array("i", kinds), contiguous


def moe_ovl_grad_norm_workspace_bytes(num_tensors: int) -> int:
    n = C.c_size_t(0)
    _done(B.load().moe_ovl_grad_norm_workspace_bytes(int(num_tensors), C.byref(n)), "moe_ovl_grad_norm_workspace_bytes")
    return int(n.value)


def moe_ovl_grad_norm(*, grads, norm, workspace, stream=None) -> None:
    """norm[0] = the square root of the sum of the squares of all values of a list of tensors.  The workspace has moe_ovl_grad_norm_workspace_bytes
    bytes.  Ranks that hold different gradients combine their norms (the root of the sum of squares) before moe_ovl_clip_grads."""
    where = "moe_ovl_grad_norm"
    dev, grads = _device(where, norm), list(grads)
    at, sizes, dtypes, _ = _tensor_list(where, "grads", grads, dev)
    _vector(where, "norm", norm, (1,), torch.float32, dev)
    nbytes = _workspace(where, workspace, dev)
    _call(where, B.load().moe_ovl_grad_norm, GradsArgs, dev, len(grads), 0, _host(at), 0, _host(sizes), _host(dtypes), norm.data_ptr(), 0.0, 0.0,
          workspace.data_ptr(), nbytes, _stream(dev, stream, *grads, norm, workspace))


def moe_ovl_clip_grads(*, grads, norm, max_norm: float, eps: float = 1e-6, out=None, stream=None) -> None:
    """Every value of a list of tensors times min(1, max_norm / (norm[0] + eps)), where it lies or into the tensors of `out`."""
    where = "moe_ovl_clip_grads"
    dev, grads = _device(where, norm), list(grads)
    at, sizes, dtypes, plain = _tensor_list(where, "grads", grads, dev)
    to = None
    if out is not None:
        out = list(out)
        if len(out) != len(grads):
            _refuse(where, f"out has {len(out)} tensors, grads {len(grads)}")
        to, _, kinds, as_plain = _tensor_list(where, "out", out, dev)
        if not plain or not as_plain or kinds != dtypes or list(map(_shape_of, out)) != list(map(_shape_of, grads)):
            for g, o in zip(grads, out):
                if o.shape != g.shape or o.dtype is not g.dtype or any(s != z for s, z, n in zip(o.stride(), g.stride(), g.shape) if n != 1):
                    _refuse(where, f"a tensor of out has to be {list(g.shape)} {g.dtype} with strides {g.stride()}, not {list(o.shape)} {o.dtype} with {o.stride()}")
    _vector(where, "norm", norm, (1,), torch.float32, dev)
    _call(where, B.load().moe_ovl_clip_grads, GradsArgs, dev, len(grads), 0, _host(at), 0 if to is None else _host(to), _host(sizes), _host(dtypes), norm.data_ptr(),
          max_norm, eps, 0, 0, _stream(dev, stream, *grads, norm, *(out or ())))


def _host(a) -> int:
    return a.buffer_info()[0]
