"""The operators around the optimizer step, by the names of their C entry points (include/fira.h): embedding lookup, layer norm
and root-mean-square norm, each with its gradient, the norm and clipping of a list of gradients, AdamW over a list
of tensors, rotary positions, and the block norm (what stands between two blocks on the residual stream) with its gradient.

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
import math
from typing import NamedTuple, Optional, Sequence, Tuple

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


class BlockNorm(NamedTuple):
    """What fira_block_norm gives: the stream after the block, its norm, and both norms' statistics (None where there is no such)."""
    residual: torch.Tensor
    y: Optional[torch.Tensor]
    mean: Optional[torch.Tensor]
    rstd: Optional[torch.Tensor]
    post_mean: Optional[torch.Tensor]
    post_rstd: Optional[torch.Tensor]


class BlockNormGradients(NamedTuple):
    """What fira_block_norm_gradient gives; None for vectors that are not there."""
    dx: torch.Tensor
    dblock: torch.Tensor
    dweight: Optional[torch.Tensor]
    dbias: Optional[torch.Tensor]
    dgate: Optional[torch.Tensor]
    dpost_weight: Optional[torch.Tensor]
    dpost_bias: Optional[torch.Tensor]


def _block_desc(x, block, gate, weight, bias, post_weight, post_bias, norm, post, eps, post_eps, residual_scale, block_scale):
    """Checks what both calls have in common -> (descriptor, pointers of the vectors, their type or None)."""
    shape = x.shape
    if block.shape != shape:
        _refuse(FIRA_ERR_SHAPE, f"the block is {tuple(block.shape)} for a stream of {tuple(shape)}")
    dt = _dtype(x.dtype, "stream")
    if block.dtype != x.dtype:
        _refuse(FIRA_ERR_DTYPE, "the block is not of the stream's type")
    if norm == fira.FIRA_NO_NORM and (weight is not None or bias is not None):
        _refuse(FIRA_ERR_INVALID_ARG, "weight or bias without a norm")
    if post == fira.FIRA_NO_NORM and (post_weight is not None or post_bias is not None):
        _refuse(FIRA_ERR_INVALID_ARG, "post_weight or post_bias without a post norm")
    dim = shape[-1]
    pdt = _param_dtype(dt, gate, weight, bias, post_weight, post_bias)
    at = fira.fira_block_norm_params(_vector(gate, dim, "gate"), _vector(weight, dim, "weight"), _vector(bias, dim, "bias"), _vector(post_weight, dim, "post_weight"),
                                     _vector(post_bias, dim, "post_bias"))
    return fira.fira_block_norm_desc(x.numel() // dim if dim else 0, dim, dt, pdt, norm, post, eps, post_eps, residual_scale, block_scale), at


def _pointer(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _statistics(x, kind, dev):
    """-> (mean, rstd) of a norm, uninitialised; None for what it has not"""
    if kind == fira.FIRA_NO_NORM:
        return None, None
    rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=dev)
    return torch.empty_like(rstd) if kind == fira.FIRA_LAYER_NORM else None, rstd


def _check_statistics(x, kind, mean, rstd, name):
    """-> (mean, rstd) as the library wants them"""
    if kind == fira.FIRA_NO_NORM:
        return None, None
    if kind != fira.FIRA_LAYER_NORM:
        mean = None
    for t, wanted in ((rstd, True), (mean, kind == fira.FIRA_LAYER_NORM)):
        if wanted and (t is None or t.dtype != torch.float32 or t.shape != x.shape[:-1] or not t.is_contiguous()):
            _refuse(FIRA_ERR_SHAPE, f"the {name}'s statistics are not dense fp32 tensors of {tuple(x.shape[:-1])}")
    return mean, rstd


def _vector_gradient(given, wanted, like, dim, dtype, dev, accumulate, name):
    if not wanted:
        if given is not None:
            _refuse(FIRA_ERR_INVALID_ARG, f"{name} of a vector that is not there")
        return None
    if given is None:
        if accumulate:
            _refuse(FIRA_ERR_INVALID_ARG, f"accumulate without {name}")
        return torch.empty(dim, dtype=dtype, device=dev) if like is None else torch.empty_like(like)
    if given.shape != (dim,) or given.dtype != dtype or not given.is_contiguous():
        _refuse(FIRA_ERR_SHAPE, f"{name} is not a dense vector of {dim} of {dtype}")
    return given


def fira_block_norm(x: torch.Tensor, block: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, *, gate: Optional[torch.Tensor] = None,
                    post_weight: Optional[torch.Tensor] = None, post_bias: Optional[torch.Tensor] = None, norm: int = fira.FIRA_RMS_NORM, post: int = fira.FIRA_NO_NORM,
                    eps: float = 1e-5, post_eps: Optional[float] = None, residual_scale: float = 1.0, block_scale: float = 1.0, out: Optional[torch.Tensor] = None,
                    y_out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> BlockNorm:
    """The stream after a block, r = residual_scale x + block_scale gate post_norm(block), and the next block's norm of it, over the last dimension.
    norm and post: FIRA_LAYER_NORM, FIRA_RMS_NORM or FIRA_NO_NORM; without a norm, y is None, without a post norm the block goes as it is.
    The vectors, of one type, default to ones (gate, weights) and zeros (biases).  out and y_out take r and y.  post_eps defaults to eps."""
    lib = fira.load_library()
    if x.dim() < 1:
        _refuse(FIRA_ERR_SHAPE, "x has no dimension")
    dev = _device(x, block, gate, weight, bias, post_weight, post_bias, out, y_out)
    d, at = _block_desc(x, block, gate, weight, bias, post_weight, post_bias, norm, post, eps, eps if post_eps is None else post_eps, residual_scale, block_scale)
    if norm == fira.FIRA_NO_NORM and y_out is not None:
        _refuse(FIRA_ERR_INVALID_ARG, "y_out without a norm")
    elsewhere = _elsewhere(dev, stream)
    if elsewhere is not None:
        with elsewhere:
            return fira_block_norm(x, block, weight, bias, gate=gate, post_weight=post_weight, post_bias=post_bias, norm=norm, post=post, eps=eps, post_eps=post_eps,
                                   residual_scale=residual_scale, block_scale=block_scale, out=out, y_out=y_out)
    x, ld_x = _input(x)
    block, ld_block = _input(block)
    out, ld_r = _result(out, x.shape, x.dtype, dev, "out", like=x)
    y, ld_y = (None, 0) if norm == fira.FIRA_NO_NORM else _result(y_out, x.shape, x.dtype, dev, "y_out", like=x)
    mean, rstd = _statistics(x, norm, dev)
    post_mean, post_rstd = _statistics(x, post, dev)
    _check(lib.fira_block_norm(d, x.data_ptr(), ld_x, block.data_ptr(), ld_block, at, out.data_ptr(), ld_r, _pointer(y), ld_y, _pointer(mean), _pointer(rstd), _pointer(post_mean),
                               _pointer(post_rstd), _stream(dev)))
    return BlockNorm(out, y, mean, rstd, post_mean, post_rstd)


def fira_block_norm_gradient(dresidual: Optional[torch.Tensor], dy: Optional[torch.Tensor], residual: torch.Tensor, block: torch.Tensor, weight: Optional[torch.Tensor] = None,
                             mean: Optional[torch.Tensor] = None, rstd: Optional[torch.Tensor] = None, *, gate: Optional[torch.Tensor] = None,
                             post_weight: Optional[torch.Tensor] = None, post_bias: Optional[torch.Tensor] = None, post_mean: Optional[torch.Tensor] = None,
                             post_rstd: Optional[torch.Tensor] = None, bias: bool = False, norm: int = fira.FIRA_RMS_NORM, post: int = fira.FIRA_NO_NORM,
                             residual_scale: float = 1.0, block_scale: float = 1.0, dx: Optional[torch.Tensor] = None, dblock: Optional[torch.Tensor] = None,
                             dweight: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None, dgate: Optional[torch.Tensor] = None,
                             dpost_weight: Optional[torch.Tensor] = None, dpost_bias: Optional[torch.Tensor] = None, accumulate: bool = False,
                             workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> BlockNormGradients:
    """Gradients of fira_block_norm from those of its residual (None: nothing else uses it) and y (None without a norm).  residual and the statistics are
    what it gave, the vectors and scales what it was given.  The gradients of the vectors that are there, and with `bias` the norm's, have the vectors' type (bias alone:
    dbias's, default the stream's); accumulate adds them to what those given hold."""
    lib = fira.load_library()
    if residual.dim() < 1:
        _refuse(FIRA_ERR_SHAPE, "residual has no dimension")
    dev = _device(residual, block, dresidual, dy, gate, weight, post_weight, post_bias, mean, rstd, post_mean, post_rstd, dx, dblock, dweight, dbias, dgate, dpost_weight, dpost_bias)
    d, at = _block_desc(residual, block, gate, weight, None, post_weight, post_bias, norm, post, 0.0, 0.0, residual_scale, block_scale)
    for t, name in ((dresidual, "dresidual"), (dy, "dy")):
        if t is not None and (t.shape != residual.shape or t.dtype != residual.dtype):
            _refuse(FIRA_ERR_SHAPE, f"{name} is {tuple(t.shape)} of {t.dtype} for a stream of {tuple(residual.shape)} of {residual.dtype}")
    if (dy is None) != (norm == fira.FIRA_NO_NORM):
        _refuse(FIRA_ERR_INVALID_ARG, "dy without a norm, or a norm without dy")
    if bias and norm == fira.FIRA_NO_NORM:
        _refuse(FIRA_ERR_INVALID_ARG, "bias without a norm")
    mean, rstd = _check_statistics(residual, norm, mean, rstd, "norm")
    post_mean, post_rstd = _check_statistics(residual, post, post_mean, post_rstd, "post norm")
    if gate is None and weight is None and post_weight is None and post_bias is None and dbias is not None:
        d.param_dtype = _dtype(dbias.dtype, "parameter")
    elsewhere = _elsewhere(dev, stream)
    if elsewhere is not None:
        with elsewhere:
            return fira_block_norm_gradient(dresidual, dy, residual, block, weight, mean, rstd, gate=gate, post_weight=post_weight, post_bias=post_bias, post_mean=post_mean,
                                            post_rstd=post_rstd, bias=bias, norm=norm, post=post, residual_scale=residual_scale, block_scale=block_scale, dx=dx, dblock=dblock,
                                            dweight=dweight, dbias=dbias, dgate=dgate, dpost_weight=dpost_weight, dpost_bias=dpost_bias, accumulate=accumulate,
                                            workspace=workspace)
    residual, ld_r = _input(residual)
    block, ld_b = _input(block)
    dresidual, ld_dr = (None, 0) if dresidual is None else _input(dresidual)
    dy, ld_dy = (None, 0) if dy is None else _input(dy)
    dx, ld_dx = _result(dx, residual.shape, residual.dtype, dev, "dx", like=residual)
    dblock, ld_db = _result(dblock, residual.shape, residual.dtype, dev, "dblock", like=residual)
    dim, ptype = residual.shape[-1], torch.float32 if d.param_dtype == FIRA_F32 else torch.bfloat16
    dgate = _vector_gradient(dgate, gate is not None, gate, dim, ptype, dev, accumulate, "dgate")
    dweight = _vector_gradient(dweight, weight is not None, weight, dim, ptype, dev, accumulate, "dweight")
    dbias = _vector_gradient(dbias, bias, weight, dim, ptype, dev, accumulate, "dbias")
    dpost_weight = _vector_gradient(dpost_weight, post_weight is not None, post_weight, dim, ptype, dev, accumulate, "dpost_weight")
    dpost_bias = _vector_gradient(dpost_bias, post_bias is not None, post_bias, dim, ptype, dev, accumulate, "dpost_bias")
    to = fira.fira_block_norm_params(_pointer(dgate), _pointer(dweight), _pointer(dbias), _pointer(dpost_weight), _pointer(dpost_bias))
    workspace = _workspace(workspace, lib.fira_block_norm_gradient_workspace_bytes(d), dev)
    _check(lib.fira_block_norm_gradient(d, _pointer(dresidual), ld_dr, _pointer(dy), ld_dy, residual.data_ptr(), ld_r, block.data_ptr(), ld_b, at, _pointer(mean), _pointer(rstd),
                                        _pointer(post_mean), _pointer(post_rstd), dx.data_ptr(), ld_dx, dblock.data_ptr(), ld_db, to, bool(accumulate), workspace.data_ptr(),
                                        workspace.numel(), _stream(dev)))
    return BlockNormGradients(dx, dblock, dweight, dbias, dgate, dpost_weight, dpost_bias)


def fira_rotary_frequencies(rotated: int, base: float = 10000.0, *, context: int = fira.FIRA_ROTARY_PLAIN, factor: float = 1.0, trained: float = 4096.0,
                            low: float = 1.0, high: float = 32.0, device="cuda") -> Tuple[torch.Tensor, float]:
    """-> (angles of one position, rotated / 2 fp64 values on `device`, and a scale) for fira_rotary; context: FIRA_ROTARY_PLAIN, or
    FIRA_ROTARY_LINEAR or FIRA_ROTARY_BY_PARTS for one `factor` times as long as the trained one.  The scale is 0.1 ln(factor) + 1 by parts, else 1: queries and keys times
    it make the scores larger, as models expect that were trained so; for one that was not, take the frequencies alone."""
    lib = fira.load_library()
    f, scale = (ctypes.c_double * min(max(1, rotated // 2), 1 << 15))(), ctypes.c_double()       # (more is refused)
    _check(lib.fira_rotary_frequencies(rotated, base, context, factor, trained, low, high, f, scale))
    return torch.tensor(list(f), dtype=torch.float64, device=device), scale.value


def fira_rotary(q: torch.Tensor, k: Optional[torch.Tensor], positions: Optional[torch.Tensor], frequencies: torch.Tensor, *, interleaved: bool = False,
                scale: float = 1.0, q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None,
                stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Turns queries and keys (k may be None) of shape (..., length, heads, dim), each with heads of its own, by their positions -> (q, k).  The first
    2 * len(frequencies) values of a head are turned, the rest copied; frequencies: fp64, as fira_rotary_frequencies makes them.  positions: int32 or int64 of shape
    (..., length) or (length,), or None: 0, 1, ... in every sequence.  q_out and k_out may be q and k themselves.  Any strides will do where a head's
    values are neighbours and the leading dimensions can be seen as one, as in parts of one buffer of queries, keys and values; other inputs are copied first."""
    return _rotary("fira_rotary", q, k, positions, frequencies, interleaved, scale, q_out, k_out, stream)


def fira_rotary_gradient(dq: torch.Tensor, dk: Optional[torch.Tensor], positions: Optional[torch.Tensor], frequencies: torch.Tensor, *, interleaved: bool = False,
                         scale: float = 1.0, q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None,
                         stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Gradients of fira_rotary's q and k from those of its results, with the arguments of that call."""
    return _rotary("fira_rotary_gradient", dq, dk, positions, frequencies, interleaved, scale, q_out, k_out, stream)


def _heads(t: torch.Tensor):
    """Strides of sequences, tokens and heads of t, or None if it has no such."""
    shape, strides = t.shape, t.stride()
    if strides[-1] != 1 and shape[-1] > 1:
        return None
    if len(shape) == 4:
        return strides[:3]
    batch = 0
    need = None            # stride that the next dimension outwards has to have
    for size, stride in zip(reversed(shape[:-3]), reversed(strides[:-3])):
        if size == 1:
            continue
        if need is None:
            batch = stride
        elif stride != need:
            return None
        need = stride * size
    return batch, strides[-3], strides[-2]


_ONE_OR_TWO = [None, fira.fira_rotary_heads * 1, fira.fira_rotary_heads * 2]


def _rotary(name, q, k, positions, frequencies, interleaved, scale, q_out, k_out, stream):
    lib = fira.load_library()
    shape = q.shape
    if k is None and k_out is not None:
        _refuse(FIRA_ERR_INVALID_ARG, "k_out without k")
    if len(shape) < 3 or (k is not None and (k.dim() < 3 or k.shape[:-2] != shape[:-2] or k.shape[-1] != shape[-1])):
        _refuse(FIRA_ERR_SHAPE, f"queries are {tuple(shape)}, keys {None if k is None else tuple(k.shape)}")
    dev = _device(q, k, positions, frequencies, q_out, k_out)
    dt = _dtype(q.dtype, "q")
    if k is not None and k.dtype != q.dtype:
        _refuse(FIRA_ERR_DTYPE, "k is not of q's type")
    if frequencies.dtype != torch.float64 or frequencies.dim() != 1 or not frequencies.is_contiguous():
        _refuse(FIRA_ERR_DTYPE, "frequencies are not a dense fp64 vector")
    length = shape[-3]
    stride = 0
    if positions is not None:
        if positions.dtype not in _IDS:
            _refuse(FIRA_ERR_DTYPE, "positions are neither int32 nor int64")
        if positions.shape != shape[:-2] and positions.shape != (length,):
            _refuse(FIRA_ERR_SHAPE, f"positions are {tuple(positions.shape)} for tokens of {tuple(shape[:-2])}")
        stride = length if positions.dim() > 1 else 0
    elsewhere = _elsewhere(dev, stream)
    if elsewhere is not None:
        with elsewhere:
            return _rotary(name, q, k, positions, frequencies, interleaved, scale, q_out, k_out, None)
    if positions is not None:
        positions = positions.contiguous()
    q, q_out, heads = _turned(q, q_out)
    if k is None:
        h = _ONE_OR_TWO[1](heads)
    else:
        k, k_out, more = _turned(k, k_out)
        h = _ONE_OR_TWO[2](heads, more)
    batch = shape[0] if len(shape) == 4 else math.prod(shape[:-3])
    d = fira.fira_rotary_desc(batch, length, shape[-1], 2 * frequencies.shape[0], dt, interleaved and 1 or 0, FIRA_I64 if positions is None else _IDS[positions.dtype], stride, scale)
    _check(getattr(lib, name)(d, h, len(h), frequencies.data_ptr(), None if positions is None else positions.data_ptr(), _stream(dev)))
    return q_out, k_out


def _turned(x, out):
    """-> (x, copied if it has to be, its result, the descriptor of both)"""
    at = _heads(x)
    if at is None:
        x = x.contiguous()
        at = _heads(x)
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        to = _heads(out) if not at[0] or not x.is_contiguous() else at
    else:
        if out.shape != x.shape or out.dtype != x.dtype:
            _refuse(FIRA_ERR_SHAPE, f"a result is {tuple(out.shape)} of {out.dtype}, not {tuple(x.shape)} of {x.dtype}")
        to = _heads(out)
        if to is None:
            _refuse(FIRA_ERR_SHAPE, "a result has no strides of sequences, tokens and heads")
    return x, out, fira.fira_rotary_heads(x.data_ptr(), out.data_ptr(), x.shape[-2], *at, *to)


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


_STATES = {torch.float32: fira.FIRA_STATE_F32, torch.float8_e4m3fn: fira.FIRA_STATE_E4M3}


class AdamWList:
    """Tensors that take AdamW steps together, marshalled once: parameters and gradients of bf16 and fp32 (a gradient's type need not be its
    parameter's) on one GPU that can be seen as matrices, and their states.  weight_decay: of all, or one for each.  state: torch.float32 or
    torch.float8_e4m3fn, of all or one for each; the latter's m and sqrt(v) are codes, to be multiplied with the scale of their 256 values, and
    are rounded at random by seeds (default: the place in the list).

    m, v, m_scale, v_scale (lists; the scales of a float32 state are None) and t (two int64: the steps taken, and a value of the call's) are a
    checkpoint.  Lists that are not given begin at zero, on the stream that is current then; states that are given have the type that they have,
    whatever `state` says.  The states may be dropped with the list while its calls are still at work, on whatever stream that is; parameters and
    gradients are kept by their owner, and everything by that of a captured step."""

    def __init__(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], *, weight_decay=0.0, state=torch.float32,
                 m: Optional[Sequence[torch.Tensor]] = None, v: Optional[Sequence[torch.Tensor]] = None, m_scale: Optional[Sequence[Optional[torch.Tensor]]] = None,
                 v_scale: Optional[Sequence[Optional[torch.Tensor]]] = None, t: Optional[torch.Tensor] = None, seeds: Optional[Sequence[int]] = None,
                 device: Optional[torch.device] = None):
        self.lib = fira.load_library()
        params, grads = list(params), list(grads)
        if not params and device is None:
            _refuse(FIRA_ERR_INVALID_ARG, "an empty list needs a device")
        if (m is None) != (v is None) or (m_scale is None) != (v_scale is None) or (m is None and m_scale is not None) or (m is not None and any(x is None for x in (*m, *v))):
            _refuse(FIRA_ERR_INVALID_ARG, "states that are given in part")
        n = self.count = len(params)
        each = lambda x: list(x) if isinstance(x, (list, tuple)) else [x] * n  # noqa: E731
        decays, states, seeds = each(weight_decay), each(state) if m is None else [x.dtype for x in m], list(range(n)) if seeds is None else list(seeds)
        for given, name in ((grads, "gradients"), (decays, "weight decays"), (states, "states"), (seeds, "seeds"), (states if v is None else v, "states v"),
                            (states if m_scale is None else m_scale, "scales of m"), (states if v_scale is None else v_scale, "scales of v")):
            if given is None or len(given) != n:
                _refuse(FIRA_ERR_INVALID_ARG, f"{None if given is None else len(given)} {name} for {n} tensors")
        for i, x in enumerate(states):
            if x not in _STATES:
                _refuse(FIRA_ERR_DTYPE, f"state {i} is neither float32 nor float8_e4m3fn")
        if m_scale is not None and any(x is torch.float8_e4m3fn and None in (a, b) for x, a, b in zip(states, map(_pointer, m_scale), map(_pointer, v_scale))):
            _refuse(FIRA_ERR_INVALID_ARG, "8-bit states that are given in part, without a scale")
        self.device = dev = _device(*(params or [torch.empty(0, device=device)]), *grads)
        self.descs = (fira.fira_adamw_desc * n)()
        for i, (p, g) in enumerate(zip(params, grads)):
            if p.shape != g.shape:
                _refuse(FIRA_ERR_SHAPE, f"gradient {i} is {tuple(g.shape)}, not {tuple(p.shape)}")
            (rows, cols, ld_w), (_, _, ld_g) = GradientList._matrix(p, f"tensor {i}"), GradientList._matrix(g, f"gradient {i}")
            self.descs[i] = fira.fira_adamw_desc(rows, cols, ld_w, ld_g, _dtype(p.dtype, f"tensor {i}"), _dtype(g.dtype, f"gradient {i}"), _STATES[states[i]],
                                                 seeds[i] & 0xffffffff, decays[i])
        sizes, scales = [p.numel() for p in params], [self.lib.fira_adamw_scales(self.descs[i]) for i in range(n)]
        self.m, self.v = ([self._state(x, i, sizes[i], states[i], name) for i, x in enumerate(given or [None] * n)] for given, name in ((m, "m"), (v, "v")))
        if m is not None and any(s is torch.float8_e4m3fn for s in states) and (m_scale is None or v_scale is None):
            _refuse(FIRA_ERR_INVALID_ARG, "8-bit states without their scales")
        self.m_scale, self.v_scale = ([self._state(x, i, scales[i], torch.float32, name) if states[i] is not torch.float32 else None
                                       for i, x in enumerate(given or [None] * n)] for given, name in ((m_scale, "m_scale"), (v_scale, "v_scale")))
        self.t = self._state(t, 0, 2, torch.int64, "t")
        for given, name in ((params, "tensor"), ((*self.m, *self.v, *self.m_scale, *self.v_scale, self.t), "state or scale")):
            places = [x.data_ptr() for x in given if x is not None and x.numel()]
            if len(set(places)) < len(places):
                _refuse(FIRA_ERR_INVALID_ARG, f"a {name} is listed twice")
        pointers = ctypes.c_void_p * n
        self.W, self.G = pointers(*[p.data_ptr() for p in params]), pointers(*[g.data_ptr() for g in grads])
        at = lambda x: None if x is None else x.data_ptr()  # noqa: E731
        self.states = (fira.fira_adamw_state * n)(*[fira.fira_adamw_state(*map(at, x)) for x in zip(self.m, self.v, self.m_scale, self.v_scale)])
        self._keep = (params, grads)
        self._streams = set()                              # on which the states are known to be in use

    def _state(self, given, i: int, size: int, dtype, name: str) -> torch.Tensor:
        if given is None:
            return torch.zeros(size, dtype=torch.uint8 if dtype is torch.float8_e4m3fn else dtype, device=self.device).view(dtype)
        if given.dtype != dtype or given.numel() != size or not given.is_contiguous():
            _refuse(FIRA_ERR_SHAPE, f"{name} of tensor {i} is not {size} dense values of {dtype}")
        if given.device != self.device:
            _refuse(FIRA_ERR_INVALID_ARG, f"tensors on {self.device} and {given.device}")
        return given

    def fira_adamw_step(self, lr, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, *, norm: Optional[torch.Tensor] = None,
                        max_norm: float = float("inf"), stream: Optional[torch.cuda.Stream] = None):
        """One step of all tensors, in place.  lr: a number, or an fp32 scalar on the GPU, which a captured step reads again.  norm: the gradients' norm, an
        fp32 scalar on the GPU (GradientList.fira_gradient_norm), by which they are cut to max_norm on their way in."""
        given = lr if isinstance(lr, torch.Tensor) else None
        for x, name in ((given, "lr"), (norm, "norm")):
            if x is not None and (x.device != self.device or x.dtype != torch.float32 or x.numel() != 1):
                _refuse(FIRA_ERR_INVALID_ARG, f"{name} is not an fp32 scalar on {self.device}")
        elsewhere = _elsewhere(self.device, stream)
        if elsewhere is not None:
            with elsewhere:
                return self.fira_adamw_step(lr, beta1, beta2, eps, norm=norm, max_norm=max_norm)
        q = _stream(self.device)
        if q not in self._streams and not torch.cuda.is_current_stream_capturing():
            for x in (*self.m, *self.v, *self.m_scale, *self.v_scale, self.t):
                if x is not None:
                    x.record_stream(torch.cuda.current_stream())
            self._streams.add(q)
        hp = fira.fira_adamw_hparams(0.0 if given is not None else lr, beta1, beta2, eps, max_norm)
        _check(self.lib.fira_adamw_step(self.descs, self.count, hp, self.W, self.G, self.states, self.t.data_ptr(), None if given is None else given.data_ptr(),
                                        None if norm is None else norm.data_ptr(), q))
