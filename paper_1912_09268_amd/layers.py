"""The operators that make per-layer gradients, on torch tensors: embedding lookup and its gradient, and activation
checkpoints in 8 bits with what the backward pass makes of them.

Arguments are checked (ValueError) and handed to the library, in native code where the extension module is there; memory and streams are torch's.  Every call runs on
the tensors' device and on torch's current stream there, and does not wait for it.  A tensor made on another stream
needs that stream's work to be waited for, and Tensor.record_stream where it is freed early, as with any other call.

The operators are the backward pass, and autograd knows nothing of them: results have no graph.  So that no gradient is lost without
a word, tensors that require grad are refused in grad mode; under torch.no_grad(), in an autograd.Function and detached they are
taken.  Tensors that a call has written count as changed: autograd refuses to go on with one that it has saved before.

    h = layers.embed([word, position, token_type], [ids, places, types])          # bf16, from binary32 weights
    u = torch.empty_like(z)
    kept = layers.act_store(z, kind="gelu", y=u)                                  # z in 8 bits, u = gelu(z)
    ...
    layers.act_backward(kept, du, kind="gelu", dx=dz)                             # dz = du * gelu'(z)
    layers.act_linear_grad(dz, kept_input, grad_of_w, db=grad_of_b)
    layers.embed_grad(dh, ids, grad_of_word)

The gradients may be the very tensors that the merged-gradient calls read: `DeviceModel.grads` holds 16-bit gradients as
raw bits, so view them, e.g. `dm.grads[w][i].view(torch.bfloat16).view(rows, dim)`."""
from __future__ import annotations

from typing import NamedTuple, Optional, Sequence, Union

import torch

from . import layers_binding as B

try:
    from . import _layers_calls as _native
    B._native = _native
    B._announce()
except ImportError:             # not built for this Python and torch: every call goes the plain way
    class _native:
        embed = embed_grad = act_store = act_backward = act_linear_grad = staticmethod(lambda *args: NotImplemented)

_DTYPES = {torch.float32: B.F32, torch.bfloat16: B.BF16, torch.float16: B.F16}
_ID_TYPES = {torch.int32: B.I32, torch.int64: B.I64}
KINDS = {"identity": B.IDENTITY, "gelu": B.GELU, "gelu_tanh": B.GELU_TANH, "silu": B.SILU}


class Act8(NamedTuple):
    """A checkpoint: q int8 [tokens, ld] and scale float32 [groups of 128 tokens, ld]; it stands for q * scale on its first
    `channels` columns."""
    q: torch.Tensor
    scale: torch.Tensor
    channels: int


def _fail(message: str):
    raise ValueError(message)


def _matrix(t: torch.Tensor, name: str, rows: Optional[int], cols: Optional[int], dtypes=_DTYPES) -> int:
    """Checks a matrix and returns the distance of its rows."""
    if t.dtype not in dtypes:
        _fail(f"{name} has type {t.dtype}")
    if t.dim() != 2 or (rows is not None and t.shape[0] != rows) or (cols is not None and t.shape[1] != cols):
        _fail(f"{name} has shape {tuple(t.shape)}, wanted ({'any' if rows is None else rows}, {'any' if cols is None else cols})")
    row, col = t.stride()
    if (t.shape[1] > 1 and col != 1) or (t.shape[0] > 1 and row < t.shape[1]):
        _fail(f"{name}: elements of a row must follow each other and rows must not overlap, strides are {t.stride()}")
    return row if t.shape[0] > 1 else t.shape[1]


def _flat(t: torch.Tensor, name: str, tokens: int, dim: int) -> torch.Tensor:
    """A tensor of a row for each token, whatever its shape, as a matrix."""
    if t.dim() == 2:
        return t
    try:
        return t.view(tokens, dim)
    except RuntimeError:
        _fail(f"{name} has shape {tuple(t.shape)} and strides {t.stride()}: no {tokens} rows of {dim} at one distance")


def _device(*tensors) -> torch.device:
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        _fail("autograd follows a tensor, and the operators have no graph: call them without grad mode, or detach it")
    if any(t is not None and t.is_neg() for t in tensors):
        _fail("the memory of a tensor holds its values negated: take its resolve_neg()")
    device = tensors[0].device
    if device.type != "cuda":
        _fail(f"tensors must be on the GPU, not on {device}")
    for t in tensors[1:]:
        if t is not None and t.device != device:
            _fail(f"tensors are on {device} and on {t.device}")
    return device


def _written(*tensors) -> None:
    """Raises the versions of tensors that a call has written, so that autograd notices where it has saved one of them."""
    for t in tensors:
        if t is not None and not t.is_inference():
            torch.autograd.graph.increment_version(t)


class _on:
    """The device's current stream as a handle, with the device current: free of charge where it is already."""
    __slots__ = ("device", "guard")

    def __init__(self, device: torch.device):
        self.device, self.guard = device, None

    def __enter__(self) -> int:
        if torch.cuda.current_device() != self.device.index:
            self.guard = torch.cuda.device(self.device)
            self.guard.__enter__()
        return torch.cuda.current_stream(self.device).cuda_stream

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


def _workspace(given: Optional[torch.Tensor], nbytes: int, device: torch.device) -> torch.Tensor:
    if given is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    if given.device != device or not given.is_contiguous() or given.numel() * given.element_size() < nbytes or given.data_ptr() % 256:
        _fail(f"the workspace must be contiguous, on {device}, aligned to 256 bytes and of {nbytes} bytes or more")
    return given


def _kind(kind: str) -> int:
    if kind not in KINDS:
        _fail(f"unknown kind {kind!r}; choose from {tuple(KINDS)}")
    return KINDS[kind]


Tensors = Union[torch.Tensor, Sequence[torch.Tensor]]


def embed(tables: Tensors, ids: Tensors, scales: Optional[Sequence[float]] = None, out: Optional[torch.Tensor] = None,
          dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """out[t] = sum over k of scales[k] * tables[k][ids[k][t]], summed in binary32 in that order and rounded once.

    One to four tables [rows, dim] of one type, as many integer id tensors (contiguous, of one shape; ids outside a table
    stand for no row), `out` [tokens, dim] or the ids' shape + [dim]; without it a new tensor of `dtype`."""
    tables = [tables] if isinstance(tables, torch.Tensor) else tables
    ids = [ids] if isinstance(ids, torch.Tensor) else ids
    scales = [1.0] * len(tables) if scales is None else scales
    if out is not None and _native.embed(tables, ids, scales, out) is None:
        return out
    if not 1 <= len(tables) <= B.MAX_TABLES or len(ids) != len(tables) or len(scales) != len(tables):
        _fail(f"one to {B.MAX_TABLES} tables with ids and a scale each")
    device = _device(*tables, *ids, out)
    first, shape = tables[0], ids[0].shape
    tokens, dim = ids[0].numel(), first.shape[-1]
    rows = []
    for table, i, scale in zip(tables, ids, scales):
        if table.dtype != first.dtype:
            _fail("the tables must be of one type")
        if i.dtype not in _ID_TYPES or i.shape != shape or not i.is_contiguous():
            _fail("ids must be contiguous int32 or int64 tensors of one shape")
        stride = _matrix(table, "a table", None, dim)
        rows.append(B.Table(table.data_ptr(), i.data_ptr(), table.shape[0], stride, scale, _ID_TYPES[i.dtype]))
    if out is None:
        out = torch.empty(*shape, dim, dtype=dtype, device=device)
    if out.shape != (*shape, dim) and out.shape != (tokens, dim):
        _fail(f"out has shape {tuple(out.shape)}, wanted {(*shape, dim)}")
    flat = _flat(out, "out", tokens, dim)
    out_stride = _matrix(flat, "out", tokens, dim)
    with _on(device) as stream:
        B.embed(rows, _DTYPES[first.dtype], tokens, dim, flat.data_ptr(), out_stride, _DTYPES[out.dtype], stream)
    _written(out)
    return out


def embed_grad(dy: torch.Tensor, ids: torch.Tensor, grad: torch.Tensor, scale: float = 1.0, padding_row: int = -1,
               accumulate: bool = False, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """grad[r] = scale * sum of dy[t] over the tokens with ids[t] == r, for every row of grad [rows, dim]; added to grad where
    `accumulate`.  dy [tokens, dim]; tokens of `padding_row` and ids outside the table count for nothing.
    `workspace`: device memory of layers_binding.embed_grad_workspace(tokens, rows, dim) bytes to use; None takes torch's."""
    if _native.embed_grad(dy, ids, grad, scale, padding_row, accumulate, workspace) is None:
        return grad
    device = _device(dy, ids, grad, workspace)
    if ids.dtype not in _ID_TYPES or not ids.is_contiguous():
        _fail("ids must be a contiguous int32 or int64 tensor")
    tokens = ids.numel()
    grad_stride = _matrix(grad, "grad", None, None)
    rows, dim = grad.shape
    dy = _flat(dy, "dy", tokens, dim)
    dy_stride = _matrix(dy, "dy", tokens, dim)
    with _on(device) as stream:
        space = _workspace(workspace, B.embed_grad_workspace(tokens, rows, dim), device)
        B.embed_grad(ids.data_ptr(), _ID_TYPES[ids.dtype], tokens, dy.data_ptr(), dy_stride, _DTYPES[dy.dtype], scale, padding_row, accumulate,
                     grad.data_ptr(), rows, dim, grad_stride, _DTYPES[grad.dtype], space.data_ptr(), space.numel() * space.element_size(), stream)
    _written(grad)
    return grad


def act_empty(tokens: int, channels: int, device="cuda") -> Act8:
    """Memory for the checkpoint of a [tokens, channels] activation."""
    ld, groups = B.act_dims(tokens, channels)
    return Act8(torch.empty(tokens, ld, dtype=torch.int8, device=device), torch.empty(groups, ld, device=device), channels)


def _act(act: Act8):
    """Checks a checkpoint -> (tokens, ld)."""
    q, scale, channels = act
    if q.dim() != 2 or q.dtype != torch.int8 or scale.dtype != torch.float32 or not q.is_contiguous() or not scale.is_contiguous():
        _fail("a checkpoint is a contiguous int8 and a contiguous float32 matrix")
    tokens, ld = q.shape
    if scale.shape != ((tokens + B.ACT_GROUP - 1) // B.ACT_GROUP, ld) or not 0 <= channels <= ld or ld % 16:
        _fail(f"q {tuple(q.shape)}, scale {tuple(scale.shape)} and {channels} channels do not make a checkpoint")
    return tokens, ld


def _address(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.data_ptr()


def act_store(x: torch.Tensor, act: Optional[Act8] = None, kind: str = "identity", y: Optional[torch.Tensor] = None) -> Act8:
    """x [tokens, channels] in 8 bits, into `act` (or new memory), which is returned; and y = f(x) in the same pass where `y` is
    given (x's type).  A group with an infinity or NaN is held as NaN."""
    if act is not None and _native.act_store(x, act.q, act.scale, act.channels, KINDS.get(kind), y) is None:
        return act
    x_stride = _matrix(x, "x", None, None)
    tokens, channels = x.shape
    if act is None:
        act = act_empty(tokens, channels, x.device)
    device = _device(x, act.q, act.scale, y)
    rows, ld = _act(act)
    if rows != tokens or act.channels != channels:
        _fail(f"x has shape {tuple(x.shape)}, the checkpoint is of {(rows, act.channels)}")
    y_stride = 0
    if y is not None:
        y_stride = _matrix(y, "y", tokens, channels, (x.dtype,))
    with _on(device) as stream:
        B.act_store(x.data_ptr(), x_stride, _DTYPES[x.dtype], tokens, channels, _kind(kind), act.q.data_ptr(), act.scale.data_ptr(), ld,
                    _address(y), y_stride, stream)
    _written(act.q, act.scale, y)
    return act


def act_backward(act: Act8, dy: Optional[torch.Tensor] = None, kind: str = "identity", dx: Optional[torch.Tensor] = None,
                 y: Optional[torch.Tensor] = None):
    """dx = dy * f'(x) and, where `y` is given, y = f(x), for the x that `act` holds.  dy, dx and y are [tokens, channels] of one
    type.  With dy and without dx, dx is a new tensor.  Without dy, only y.  Returns dx, or y without dy."""
    if _native.act_backward(act.q, act.scale, act.channels, dy, KINDS.get(kind), dx, y) is None:
        return y if dy is None else dx
    tokens, ld = _act(act)
    if dy is None and (dx is not None or y is None):
        _fail("dx takes a dy, and without dy there must be a y")
    one = dy if dy is not None else y
    if dy is not None and dx is None:
        dx = torch.empty(tokens, act.channels, dtype=dy.dtype, device=dy.device)
    device = _device(act.q, act.scale, dy, dx, y)
    strides = [0 if t is None else _matrix(t, name, tokens, act.channels, (one.dtype,)) for t, name in ((dy, "dy"), (dx, "dx"), (y, "y"))]
    if one.dtype not in _DTYPES:
        _fail(f"dy has type {one.dtype}")
    with _on(device) as stream:
        B.act_backward(act.q.data_ptr(), act.scale.data_ptr(), ld, tokens, act.channels, _kind(kind), _address(dy), strides[0],
                       _address(dx), strides[1], _address(y), strides[2], _DTYPES[one.dtype], stream)
    _written(dx, y)
    return y if dy is None else dx


def act_linear_grad(dy: torch.Tensor, act: Act8, dw: torch.Tensor, db: Optional[torch.Tensor] = None, accumulate: bool = False,
                    workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dw [outputs, channels] = dy^T x and, where `db` [outputs] is given, db = dy's column sums, for the x that `act` holds and
    dy [tokens, outputs]; added to what is there where `accumulate`.  dw and db are of one type.
    `workspace`: device memory of layers_binding.act_linear_grad_workspace(tokens, channels, outputs) bytes; None takes torch's."""
    if _native.act_linear_grad(dy, act.q, act.scale, act.channels, dw, db, accumulate, workspace) is None:
        return dw
    tokens, ld = _act(act)
    device = _device(dy, act.q, act.scale, dw, db, workspace)
    dy_stride = _matrix(dy, "dy", tokens, None)
    outputs = dy.shape[1]
    dw_stride = _matrix(dw, "dw", outputs, act.channels)
    if db is not None and (db.dtype != dw.dtype or db.shape != (outputs,) or (outputs > 1 and db.stride(0) != 1)):
        _fail(f"db must be a contiguous tensor of {outputs} elements of dw's type")
    with _on(device) as stream:
        space = _workspace(workspace, B.act_linear_grad_workspace(tokens, act.channels, outputs), device)
        B.act_linear_grad(act.q.data_ptr(), act.scale.data_ptr(), ld, tokens, act.channels, dy.data_ptr(), dy_stride, _DTYPES[dy.dtype], outputs,
                          accumulate, dw.data_ptr(), dw_stride, _address(db), _DTYPES[dw.dtype], space.data_ptr(),
                          space.numel() * space.element_size(), stream)
    _written(dw, db)
    return dw
