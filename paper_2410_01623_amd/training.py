"""The operators around the optimizer step, by the names of their C entry points (include/fira.h): embedding lookup, layer norm
and root-mean-square norm, each with its gradient, and the norm and clipping of a list of gradients.

As in `fira`, this is argument marshalling: tensors become pointers, sizes and leading dimensions, everything is computed by
libfira.so, and there is no fallback.  All tensors are on one GPU, bf16 or fp32.  `stream` is the torch stream to enqueue on (default: the
current one of that GPU); the caller orders it after whatever made the inputs, and keeps tensors of another stream until it has passed
the call.  Results and workspaces that are not given are allocated on that stream.  Of a tensor with more than two dimensions all but
the last are its rows.  An input whose rows cannot be told from one leading dimension (an expanded or permuted view) is copied first; a
result given by the caller has to be such a matrix, and must not overlap an input.  What the library refuses raises fira.FiraError with its status, and so does a
tensor that does not fit the others.

Autograd does not see these calls: their results carry no graph, whether or not an input requires a gradient, and gradients are what
the *_gradient calls return (examples/train_small_lm.py has them as torch.autograd.Function)."""
from __future__ import annotations

import contextlib
import ctypes
import functools
from typing import Optional, Sequence, Tuple

import torch

from . import fira
from .fira import FiraError, FIRA_BF16, FIRA_ERR_DTYPE, FIRA_ERR_INVALID_ARG, FIRA_ERR_SHAPE, FIRA_F32, FIRA_I32, FIRA_I64

_DTYPE = {torch.float32: FIRA_F32, torch.bfloat16: FIRA_BF16}
_IDS = {torch.int32: FIRA_I32, torch.int64: FIRA_I64}


def _refuse(status: int, message: str):
    raise FiraError(status, message)


def _dtype(dtype: torch.dtype, name: str) -> int:
    dt = _DTYPE.get(dtype)
    if dt is None:
        _refuse(FIRA_ERR_DTYPE, f"{name} is neither bf16 nor fp32")
    return dt


def _device(*tensors) -> torch.device:
    dev = tensors[0].device
    if dev.type != "cuda":
        _refuse(FIRA_ERR_INVALID_ARG, "tensors are not on a GPU")
    for t in tensors[1:]:
        if t is not None and t.device != dev:
            _refuse(FIRA_ERR_INVALID_ARG, f"tensors on {dev} and {t.device}")
    return dev


@contextlib.contextmanager
def _device_and_stream(dev, stream):
    with torch.cuda.device(dev), (torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext()):
        yield


def _elsewhere(dev: torch.device, stream: Optional[torch.cuda.Stream]):
    """None if the call belongs on the current device and its current stream (entering them costs as much as a launch), else what to call again in."""
    if stream is None and dev.index == torch.cuda.current_device():
        return None
    if stream is not None and stream.device != dev:
        _refuse(FIRA_ERR_INVALID_ARG, f"tensors on {dev}, stream on {stream.device}")
    return _device_and_stream(dev, stream)


def _stream(dev: torch.device) -> int:
    """Handle of the current stream, without a torch.cuda.Stream made for it where torch can do so."""
    return _raw_stream(dev.index)


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _ld(t: torch.Tensor) -> Optional[int]:
    """Leading dimension of t seen as rows of its last dimension, or None if it has no such."""
    shape, strides = t.shape, t.stride()
    cols = shape[-1]
    if t.is_contiguous():
        return cols
    if cols > 1 and strides[-1] != 1:
        return None
    ld = None
    need = None            # stride that the next dimension outwards has to have
    for size, stride in zip(reversed(shape[:-1]), reversed(strides[:-1])):
        if size == 1:
            continue
        if need is None:
            ld = stride
        elif stride != need:
            return None
        need = stride * size
    if ld is None:
        return cols
    return ld if ld >= cols else None


def _input(t: torch.Tensor) -> Tuple[torch.Tensor, int]:
    ld = _ld(t)
    if ld is None:
        t = t.contiguous()
        ld = t.shape[-1]
    return t, ld


def _result(given: Optional[torch.Tensor], shape, dtype, dev, name: str, like: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, int]:
    """A result and its leading dimension; like: a tensor of its shape, type and device, if there is one."""
    if given is None:
        if like is not None and like.is_contiguous():
            return torch.empty_like(like), shape[-1]
        return torch.empty(shape, dtype=dtype, device=dev), shape[-1]
    if tuple(given.shape) != tuple(shape):
        _refuse(FIRA_ERR_SHAPE, f"{name} is {tuple(given.shape)}, not {tuple(shape)}")
    if given.dtype != dtype:
        _refuse(FIRA_ERR_DTYPE, f"{name} is {given.dtype}, not {dtype}")
    ld = _ld(given)
    if ld is None:
        _refuse(FIRA_ERR_SHAPE, f"{name} has no single leading dimension")
    return given, ld


def _vector(t: Optional[torch.Tensor], n: int, name: str) -> Optional[int]:
    if t is None:
        return None
    if t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        _refuse(FIRA_ERR_SHAPE, f"{name} is not a dense vector of {n}")
    return t.data_ptr()


def _workspace(given: Optional[torch.Tensor], need: int, dev) -> torch.Tensor:
    if given is not None:
        if given.device != dev or given.dtype != torch.uint8 or not given.is_contiguous():
            _refuse(FIRA_ERR_INVALID_ARG, f"workspace is not a dense byte tensor on {dev}")
        return given
    if need == fira.FIRA_UNUSED_WORKSPACE_BYTES:
        return _unused_workspace(dev)
    return torch.empty(need, dtype=torch.uint8, device=dev)


@functools.lru_cache(maxsize=None)
def _unused_workspace(dev) -> torch.Tensor:
    """What calls are given that want a workspace but do not touch it."""
    return torch.empty(fira.FIRA_UNUSED_WORKSPACE_BYTES, dtype=torch.uint8, device=dev)


def _ids(ids: torch.Tensor) -> torch.Tensor:
    if ids.dtype not in _IDS:
        _refuse(FIRA_ERR_DTYPE, "ids are neither int32 nor int64")
    return ids.contiguous()


def _check(status: int):
    if status:
        fira._check(fira.load_library(), None, status)


def fira_embed_lookup(table: torch.Tensor, ids: torch.Tensor, *, scale: float = 1.0, dtype: Optional[torch.dtype] = None,
                      out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """scale * table[ids], of shape ids.shape + (width,) and type `dtype` (default: out's, else the table's).  ids (int32 or int64) outside the
    table, such as -1 for padding, give zeros."""
    lib = fira.load_library()
    if table.dim() != 2:
        _refuse(FIRA_ERR_SHAPE, "the table is no matrix")
    dev = _device(table, ids, out)
    dtype = dtype or (out.dtype if out is not None else table.dtype)
    dt, rdt = _dtype(table.dtype, "table"), _dtype(dtype, "result")
    elsewhere = _elsewhere(dev, stream)
    if elsewhere is not None:
        with elsewhere:
            return fira_embed_lookup(table, ids, scale=scale, dtype=dtype, out=out)
    ids = _ids(ids)
    table, ld = _input(table)
    rows, dim = table.shape
    out, ld_out = _result(out, (*ids.shape, dim), dtype, dev, "out")
    d = fira.fira_embed_desc(rows, dim, ld, dt, rdt, _IDS[ids.dtype], scale)
    _check(lib.fira_embed_lookup(d, table.data_ptr(), ids.data_ptr(), ids.numel(), out.data_ptr(), ld_out, _stream(dev)))
    return out


def fira_embed_gradient(dout: torch.Tensor, ids: torch.Tensor, rows: int, *, scale: float = 1.0, dtype: Optional[torch.dtype] = None,
                        out: Optional[torch.Tensor] = None, accumulate: bool = False, workspace: Optional[torch.Tensor] = None,
                        stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Gradient of fira_embed_lookup's table of `rows` rows: dout is the gradient of its result (ids.shape + (width,)).  The result has type `dtype`
    (default: out's, else dout's).  accumulate adds to `out`."""
    lib = fira.load_library()
    dev = _device(dout, ids, out)
    dtype = dtype or (out.dtype if out is not None else dout.dtype)
    dt, rdt = _dtype(dtype, "result"), _dtype(dout.dtype, "dout")
    if dout.dim() < 1 or dout.shape[:-1] != ids.shape:
        _refuse(FIRA_ERR_SHAPE, f"dout is {tuple(dout.shape)} for ids of {tuple(ids.shape)}")
    if accumulate and out is None:
        _refuse(FIRA_ERR_INVALID_ARG, "accumulate without out")
    elsewhere = _elsewhere(dev, stream)
    if elsewhere is not None:
        with elsewhere:
            return fira_embed_gradient(dout, ids, rows, scale=scale, dtype=dtype, out=out, accumulate=accumulate, workspace=workspace)
    ids = _ids(ids)
    dout, ld_dout = _input(dout)
    dim, count = dout.shape[-1], ids.numel()
    d = fira.fira_embed_desc(rows, dim, dim, dt, rdt, _IDS[ids.dtype], scale)
    need = lib.fira_embed_gradient_workspace_bytes(d, count)
    if not need:                                         # refused: before anything of such a size is allocated
        _check(lib.fira_embed_gradient(d, None, ld_dout, None, count, None, 0, None, 0, None))
    out, d.ld = _result(out, (rows, dim), dtype, dev, "out")
    workspace = _workspace(workspace, need, dev)
    _check(lib.fira_embed_gradient(d, dout.data_ptr(), ld_dout, ids.data_ptr(), count, out.data_ptr(), bool(accumulate),
                                   workspace.data_ptr(), workspace.numel(), _stream(dev)))
    return out


def fira_layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, *, eps: float = 1e-5,
                    rms: bool = False, out: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor], torch.Tensor]:
    """Layer norm (rms: root-mean-square norm) over x's last dimension -> (y, mean, rstd); y is of x's type, mean (None with rms) and rstd are
    fp32 of shape x.shape[:-1], for fira_layer_norm_gradient.  weight and bias, of one type, default to ones and zeros."""
    lib = fira.load_library()
    if x.dim() < 1:
        _refuse(FIRA_ERR_SHAPE, "x has no dimension")
    dev = _device(x, weight, bias, out)
    dt = _dtype(x.dtype, "x")
    pdt = _param_dtype(dt, weight, bias)
    elsewhere = _elsewhere(dev, stream)
    if elsewhere is not None:
        with elsewhere:
            return fira_layer_norm(x, weight, bias, eps=eps, rms=rms, out=out)
    x, ld_x = _input(x)
    dim = x.shape[-1]
    out, ld_y = _result(out, x.shape, x.dtype, dev, "out", like=x)
    rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=dev)
    mean = None if rms else torch.empty_like(rstd)
    d = fira.fira_layer_norm_desc(rstd.numel(), dim, dt, pdt, fira.FIRA_RMS_NORM if rms else fira.FIRA_LAYER_NORM, eps)
    _check(lib.fira_layer_norm(d, x.data_ptr(), ld_x, _vector(weight, dim, "weight"), _vector(bias, dim, "bias"), out.data_ptr(), ld_y,
                               None if rms else mean.data_ptr(), rstd.data_ptr(), _stream(dev)))
    return out, mean, rstd


def _param_dtype(default: int, *params) -> int:
    given = None
    for p in params:
        if p is not None:
            dt = _dtype(p.dtype, "parameter")
            if given is not None and dt != given:
                _refuse(FIRA_ERR_DTYPE, "parameters of two types")
            given = dt
    return default if given is None else given


def fira_layer_norm_gradient(dy: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor], mean: Optional[torch.Tensor], rstd: torch.Tensor, *,
                             rms: bool = False, bias: bool = True, param_dtype: Optional[torch.dtype] = None, dx: Optional[torch.Tensor] = None,
                             dweight: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None, accumulate: bool = False,
                             workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """Gradients of fira_layer_norm -> (dx, dweight, dbias); dbias is None without `bias`.  mean and rstd are the forward pass's.  dweight and dbias
    are of weight's type (without weight: param_dtype, default x's).  accumulate adds them to what the given dweight and dbias hold, rounding to
    their type each time: to add up a bf16 weight's gradients in fp32, give weight.float(), whose values are the same."""
    lib = fira.load_library()
    if x.dim() < 1 or dy.shape != x.shape:
        _refuse(FIRA_ERR_SHAPE, f"dy is {tuple(dy.shape)} for x of {tuple(x.shape)}")
    dev = _device(x, dy, weight, mean, rstd, dx, dweight, dbias)
    dt = _dtype(x.dtype, "x")
    if dy.dtype != x.dtype:
        _refuse(FIRA_ERR_DTYPE, "dy is not of x's type")
    ptype = weight.dtype if weight is not None else param_dtype or (dweight.dtype if dweight is not None else x.dtype)
    pdt = _dtype(ptype, "parameter")
    if not rms and mean is None:
        _refuse(FIRA_ERR_INVALID_ARG, "a layer norm's gradient needs its mean")
    for t, name in ((rstd, "rstd"), (None if rms else mean, "mean")):
        if t is not None and (t.dtype != torch.float32 or t.shape != x.shape[:-1] or not t.is_contiguous()):
            _refuse(FIRA_ERR_SHAPE, f"{name} is not a dense fp32 tensor of {tuple(x.shape[:-1])}")
    if accumulate and (dweight is None or (bias and dbias is None)):
        _refuse(FIRA_ERR_INVALID_ARG, "accumulate without dweight and dbias")
    elsewhere = _elsewhere(dev, stream)
    if elsewhere is not None:
        with elsewhere:
            return fira_layer_norm_gradient(dy, x, weight, mean, rstd, rms=rms, bias=bias, param_dtype=ptype, dx=dx, dweight=dweight, dbias=dbias,
                                            accumulate=accumulate, workspace=workspace)
    x, ld_x = _input(x)
    dy, ld_dy = _input(dy)
    dim = x.shape[-1]
    dx, ld_dx = _result(dx, x.shape, x.dtype, dev, "dx", like=x)
    dweight, _ = _result(dweight, (dim,), ptype, dev, "dweight", like=weight)
    if bias:
        dbias, _ = _result(dbias, (dim,), ptype, dev, "dbias", like=dweight)
    else:
        dbias = None
    d = fira.fira_layer_norm_desc(rstd.numel(), dim, dt, pdt, fira.FIRA_RMS_NORM if rms else fira.FIRA_LAYER_NORM, 0.0)
    workspace = _workspace(workspace, lib.fira_layer_norm_gradient_workspace_bytes(d), dev)
    _check(lib.fira_layer_norm_gradient(d, dy.data_ptr(), ld_dy, x.data_ptr(), ld_x, _vector(weight, dim, "weight"),
                                        None if rms else mean.data_ptr(), rstd.data_ptr(), dx.data_ptr(), ld_dx, _vector(dweight, dim, "dweight"),
                                        _vector(dbias, dim, "dbias"), bool(accumulate), workspace.data_ptr(), workspace.numel(), _stream(dev)))
    return dx, dweight, dbias


class GradientList:
    """Gradients that are measured and clipped together, marshalled once: any tensors of bf16 and fp32 on one GPU that can be seen as
    matrices.  outs, one per gradient and of its shape, take the clipped gradients in their own type; without them clipping is in place.  A list
    holds no device memory but the tensors it was given: the workspace is allocated on the stream of each call, so that a list may be used on any
    stream, and dropped while its calls are still at work if the tensors are kept."""

    def __init__(self, grads: Sequence[torch.Tensor], outs: Optional[Sequence[torch.Tensor]] = None, device: Optional[torch.device] = None):
        self.lib = fira.load_library()
        grads = list(grads)
        if not grads and device is None:
            _refuse(FIRA_ERR_INVALID_ARG, "an empty list needs a device")
        self.device = _device(*(grads or [torch.empty(0, device=device)]), *(outs or ()))
        if outs is not None and len(outs) != len(grads):
            _refuse(FIRA_ERR_INVALID_ARG, f"{len(outs)} results for {len(grads)} gradients")
        n = self.count = len(grads)
        self.descs = (fira.fira_gradient_desc * n)()
        for i, g in enumerate(grads):
            o = outs[i] if outs is not None else g
            if o.shape != g.shape:
                _refuse(FIRA_ERR_SHAPE, f"result {i} is {tuple(o.shape)}, not {tuple(g.shape)}")
            (rows, cols, ld), (_, _, ld_out) = self._matrix(g, f"gradient {i}"), self._matrix(o, f"result {i}")
            self.descs[i] = fira.fira_gradient_desc(rows, cols, ld, _dtype(g.dtype, f"gradient {i}"), _dtype(o.dtype, f"result {i}"), ld_out)
        pointers = ctypes.c_void_p * n
        self.G = pointers(*[g.data_ptr() for g in grads])
        self.outs = pointers(*[o.data_ptr() for o in outs]) if outs is not None else None
        self.bytes = self.lib.fira_gradient_workspace_bytes(self.descs, n)
        self._keep = (grads, list(outs) if outs is not None else None)

    @staticmethod
    def _matrix(t: torch.Tensor, name: str) -> Tuple[int, int, int]:
        if t.dim() == 0:
            return 1, 1, 1
        ld = _ld(t)
        if ld is None:
            _refuse(FIRA_ERR_SHAPE, f"{name} has no single leading dimension")
        cols = t.shape[-1]
        return (t.numel() // cols if cols else 0), cols, ld

    def _result_and_workspace(self) -> Tuple[torch.Tensor, torch.Tensor]:
        return torch.empty((), dtype=torch.float32, device=self.device), torch.empty(self.bytes, dtype=torch.uint8, device=self.device)

    def fira_gradient_norm(self, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """The norm of all gradients together, an fp32 scalar on the GPU."""
        elsewhere = _elsewhere(self.device, stream)
        if elsewhere is not None:
            with elsewhere:
                return self.fira_gradient_norm()
        norm, workspace = self._result_and_workspace()
        _check(self.lib.fira_gradient_norm(self.descs, self.count, self.G, norm.data_ptr(), workspace.data_ptr(), self.bytes, _stream(self.device)))
        return norm

    def fira_clip_gradients(self, max_norm: float, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """Scales all gradients by min(1, max_norm / norm) -> the norm before, an fp32 scalar on the GPU.  A norm that is not finite leaves
        them as they are."""
        elsewhere = _elsewhere(self.device, stream)
        if elsewhere is not None:
            with elsewhere:
                return self.fira_clip_gradients(max_norm)
        norm, workspace = self._result_and_workspace()
        _check(self.lib.fira_clip_gradients(self.descs, self.count, self.G, self.outs, max_norm, norm.data_ptr(), workspace.data_ptr(),
                                            self.bytes, _stream(self.device)))
        return norm
