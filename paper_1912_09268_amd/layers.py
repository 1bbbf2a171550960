"""The operators that make per-layer gradients, on torch tensors: embedding lookup and its gradient, activation
checkpoints in 8 bits with what the backward pass makes of them, and what lies between and behind the linear layers of a language
model: root-mean-square norm, a gated linear recurrence over the tokens, and the loss against labels and a teacher's top logits.

Arguments are checked (ValueError) and handed to the library, in native code where the extension module is there; memory and streams are torch's.  Every call runs on
the tensors' device and on torch's current stream there, and does not wait for it.  A tensor made on another stream
needs that stream's work to be waited for, and Tensor.record_stream where it is freed early, as with any other call.

The operators are the backward pass, and autograd knows nothing of them: results have no graph.  So that no gradient is lost without
a word, tensors that require grad are refused in grad mode; under torch.no_grad(), in an autograd.Function and detached they are
taken.  Dual tensors of forward-mode autograd are refused, too: their tangents would be lost.  Tensors that a call has written count as changed:
autograd refuses to go on with one that it has saved before.

A call that is given its outputs (y, and h with a residual; dh; dgate and dx; loss; out, act, dx) costs some 3 us of the host.  One that makes them, and
one on [sequences, 1, channels] tensors that are not contiguous, has its arguments taken apart in Python: 15 to 24 us.

An output of norm, recur, their ways back and distill may lie over an input as a whole where a line says so; every other overlap of what a call
writes with its other tensors is refused.

    h = layers.embed([word, position, token_type], [ids, places, types])          # bf16, from binary32 weights
    u = torch.empty_like(z)
    kept = layers.act_store(z, kind="gelu", y=u)                                  # z in 8 bits, u = gelu(z)
    ...
    layers.act_backward(kept, du, kind="gelu", dx=dz)                             # dz = du * gelu'(z)
    layers.act_linear_grad(dz, kept_input, grad_of_w, db=grad_of_b)
    layers.embed_grad(dh, ids, grad_of_word)

    y, h = layers.norm(branch, weight, residual=stream, kept=kept)                # h = stream + branch, y = h / rms(h) * weight
    layers.act_linear_grad(dz, kept.linear, grad_of_w)                            # of the linear layer that y goes into
    layers.norm_backward(kept, dy, weight, dres=dstream, dh=dstream, dw=grad_of_weight)
    y = layers.recur(gate, x, states=states)                                      # [sequences, length, channels]
    dgate, dx = layers.recur_backward(gate, x, states, dy)
    loss = layers.distill(logits, top_ids, top_logits, labels=labels, temperature=2.0, dlogits=logits)

The gradients may be the very tensors that the merged-gradient calls read: `DeviceModel.grads` holds 16-bit gradients as
raw bits, so view them, e.g. `dm.grads[w][i].view(torch.bfloat16).view(rows, dim)`."""
from __future__ import annotations

from typing import NamedTuple, Optional, Sequence, Union

import torch
from torch.autograd import forward_ad

from . import layers_binding as B

try:
    from . import _layers_calls as _native
    B._native = _native
    B._announce()
except ImportError:             # not built for this Python and torch: every call goes the plain way
    class _native:
        embed = embed_grad = act_store = act_backward = act_linear_grad = staticmethod(lambda *args: NotImplemented)
        norm = norm_backward = recur = recur_backward = distill = staticmethod(lambda *args: NotImplemented)

_DTYPES = {torch.float32: B.F32, torch.bfloat16: B.BF16, torch.float16: B.F16}
_ID_TYPES = {torch.int32: B.I32, torch.int64: B.I64}
KINDS = {"identity": B.IDENTITY, "gelu": B.GELU, "gelu_tanh": B.GELU_TANH, "silu": B.SILU}
RECUR_KINDS = {"free": B.FREE, "convex": B.CONVEX, "unit": B.UNIT}


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
    if forward_ad._current_level >= 0 and any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        _fail("forward-mode autograd follows a tensor, and the operators have no tangents: take its primal")
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


def _span(t: torch.Tensor):
    """A tensor's memory: address, rows, bytes of a row, bytes from one row to the next."""
    size, width = t.element_size(), t.shape[-1]
    rows = t.numel() // width
    step = next((stride for n, stride in zip(t.shape[-2::-1], t.stride()[-2::-1]) if n > 1), width)
    return t.data_ptr(), rows, width * size, step * size


def _share(a: torch.Tensor, b: torch.Tensor) -> bool:
    """Whether matrices share memory, as the library sees it (csrc/spans.h)."""
    if a.numel() == 0 or b.numel() == 0:
        return False
    (p, rows, width, step), (q, q_rows, q_width, q_step) = _span(a), _span(b)
    behind = q - p
    if behind >= (rows - 1) * step + width or -behind >= (q_rows - 1) * q_step + q_width:
        return False
    if rows > 1 and q_rows > 1 and step != q_step:
        return True
    step = step if rows > 1 else q_step if q_rows > 1 else 1
    return max(1 - rows, (-q_width - behind) // step + 1) <= min(q_rows - 1, -((behind - width) // step) - 1)


def _why(writes: dict, reads: dict) -> None:
    """Behind a call that the library refuses: a ValueError that names tensors over each other, where that is the reason."""
    writes, reads = ({name: t for name, t in of.items() if t is not None} for of in (writes, reads))
    names = list(writes)
    for i, name in enumerate(names):
        for other in names[i + 1:]:
            if _share(writes[name], writes[other]):
                _fail(f"{name} and {other} are written and share memory")
        for other, t in reads.items():
            if _share(writes[name], t) and _span(writes[name]) != _span(t):
                _fail(f"{name} is written and shares memory with {other}")


class _on:
    """The device's current stream as a handle, with the device current: free of charge where it is already.  A refusal of the library is
    explained where tensors that the call writes lie over others."""
    __slots__ = ("device", "guard", "writes", "reads")

    def __init__(self, device: torch.device, writes: dict = {}, reads: dict = {}):
        self.device, self.guard, self.writes, self.reads = device, None, writes, reads

    def __enter__(self) -> int:
        if torch.cuda.current_device() != self.device.index:
            self.guard = torch.cuda.device(self.device)
            self.guard.__enter__()
        return torch.cuda.current_stream(self.device).cuda_stream

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)
        if isinstance(exc[1], B.MgwfbpError) and exc[1].status == -1:
            _why(self.writes, self.reads)


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
    return Act8(torch.empty(tokens, ld, dtype=torch.int8, device=device), torch.empty(groups, ld, dtype=torch.float32, device=device), channels)


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


class Norm8(NamedTuple):
    """What norm keeps: `act`, the normed values before the weight in 8 bits; `rstd` float32 [tokens]; and `linear`, what the next linear layer
    sees, values times weight: the same q with scales of its own."""
    act: Act8
    rstd: torch.Tensor
    linear: Act8


def norm_empty(tokens: int, channels: int, device="cuda") -> Norm8:
    """Memory for what norm keeps of [tokens, channels]."""
    act = act_empty(tokens, channels, device)
    return Norm8(act, torch.empty(tokens, dtype=torch.float32, device=device), Act8(act.q, torch.empty_like(act.scale), channels))


def _kept(kept: Norm8):
    """Checks what norm keeps -> (tokens, ld)."""
    act, rstd, linear = kept
    tokens, ld = _act(act)
    if linear.q.data_ptr() != act.q.data_ptr() or linear.channels != act.channels or _act(linear) != (tokens, ld):
        _fail("the two checkpoints of a norm have one q")
    _vector(rstd, "rstd", tokens, (torch.float32,))
    return tokens, ld


def _kept_names(kept: Optional[Norm8]) -> dict:
    return {} if kept is None else {"kept.rstd": kept.rstd, "kept.act.q": kept.act.q, "kept.act.scale": kept.act.scale, "kept.linear.scale": kept.linear.scale}


def _vector(t: Optional[torch.Tensor], name: str, n: int, dtypes=_DTYPES) -> int:
    """Checks a contiguous vector, which may be left out, and returns its address."""
    if t is None:
        return 0
    if t.dtype not in dtypes or t.shape != (n,) or not t.is_contiguous():
        _fail(f"{name} must be a contiguous tensor of {n} elements of {' or '.join(str(d) for d in dtypes)}, not {tuple(t.shape)} of {t.dtype}")
    return t.data_ptr()


def _code(t: Optional[torch.Tensor], of=_DTYPES) -> int:
    return 0 if t is None else of[t.dtype]


def _same_place(a: torch.Tensor, b: Optional[torch.Tensor]) -> bool:
    return b is not None and a.data_ptr() == b.data_ptr()


def norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None,
         h: Optional[torch.Tensor] = None, kept: Optional[Norm8] = None, eps: float = 1e-6):
    """h = x + residual and y = h / sqrt(mean(h^2) + eps) * weight over the channels of x [tokens, channels]; returns (y, h).

    weight [channels] (None: 1).  residual, and h with it, are of x's type or float32; None for h makes a new tensor; without a residual h is x.  y is of x's type.
    h and y may each lie over residual or x (y not over an x that is kept).  `kept` (norm_empty) takes what norm_backward and the next layer's act_linear_grad need."""
    if y is not None and (residual is None) == (h is None) and isinstance(eps, float):
        act, rstd, linear = (None, None, None) if kept is None else kept
        if kept is None or (linear.q is act.q and linear.channels == act.channels):
            if _native.norm(x, weight, residual, y, h, act and act.q, act and act.scale, act and act.channels, rstd, linear and linear.scale, eps) is None:
                return y, x if residual is None else h
    x_stride = _matrix(x, "x", None, None)
    tokens, channels = x.shape
    if y is None:
        y = torch.empty(tokens, channels, dtype=x.dtype, device=x.device)
    if residual is None and h is not None:
        _fail("without a residual h is x itself")
    if residual is not None and h is None:
        h = torch.empty(tokens, channels, dtype=residual.dtype, device=x.device)
    memory = () if kept is None else (kept.act.q, kept.act.scale, kept.rstd, kept.linear.scale)
    device = _device(x, weight, residual, y, h, *memory)
    w = _vector(weight, "weight", channels)
    y_stride = _matrix(y, "y", tokens, channels, (x.dtype,))
    stream_type, res_stride, h_stride = x.dtype, 0, 0
    if residual is not None:
        stream_type = residual.dtype
        res_stride = _matrix(residual, "residual", tokens, channels, (x.dtype, torch.float32))
        h_stride = _matrix(h, "h", tokens, channels, (stream_type,))
        if _same_place(h, residual) and h_stride != res_stride:
            _fail("h over residual must have its strides")
    if tokens and channels and (_same_place(y, h) if h is not None else kept is not None and _same_place(y, x)):
        _fail("y must be other memory than h, and than an x that is kept in 8 bits")
    ld = 0
    if kept is not None:
        rows, ld = _kept(kept)
        if rows != tokens or kept.act.channels != channels:
            _fail(f"x has shape {tuple(x.shape)}, what is kept is of {(rows, kept.act.channels)}")
    with _on(device, dict(h=h, y=y, **_kept_names(kept)), dict(x=x, residual=residual, weight=weight)) as stream:
        B.norm(x.data_ptr(), x_stride, _DTYPES[x.dtype], _address(residual), res_stride, _DTYPES[stream_type], tokens, channels, w, _code(weight), float(eps),
               _address(h), h_stride, y.data_ptr(), y_stride, *((m.data_ptr() for m in (kept.rstd, kept.act.q, kept.act.scale, kept.linear.scale)) if kept else (0, 0, 0, 0)),
               ld, stream)
    _written(y, h, *memory)
    return y, x if residual is None else h


def norm_backward(kept: Norm8, dy: torch.Tensor, weight: Optional[torch.Tensor] = None, dres: Optional[torch.Tensor] = None,
                  dh: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None, dw: Optional[torch.Tensor] = None, accumulate: bool = False,
                  workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient of norm's h, from the gradient dy [tokens, channels] of its y and what it has kept, plus `dres`, what flows into h by itself;
    that is the gradient of x and of residual.  Where given, `dx` gets it in dy's type, too, and `dw` [channels] the weight's gradient (added to
    what is there where `accumulate`).  dres and dh are of dy's type or float32, None makes a new tensor; dh and dx may each lie over dres or dy.
    `workspace`: device memory of layers_binding.norm_backward_workspace(tokens, channels) bytes; None takes torch's.  Returns dh."""
    if dh is not None and kept.linear.q is kept.act.q:
        if _native.norm_backward(kept.act.q, kept.act.scale, kept.act.channels, kept.rstd, dy, weight, dres, dh, dx, dw, accumulate, workspace) is None:
            return dh
    tokens, ld = _kept(kept)
    channels = kept.act.channels
    if dh is None:
        dh = torch.empty(tokens, channels, dtype=dy.dtype if dres is None else dres.dtype, device=dy.device)
    device = _device(dy, kept.act.q, kept.act.scale, kept.rstd, weight, dres, dh, dx, dw, workspace)
    dy_stride = _matrix(dy, "dy", tokens, channels)
    dh_stride = _matrix(dh, "dh", tokens, channels, (dy.dtype, torch.float32))
    dres_stride = 0 if dres is None else _matrix(dres, "dres", tokens, channels, (dh.dtype,))
    dx_stride = 0 if dx is None else _matrix(dx, "dx", tokens, channels, (dy.dtype,))
    if _same_place(dh, dres) and dh_stride != dres_stride:
        _fail("dh over dres must have its strides")
    w, to = _vector(weight, "weight", channels), _vector(dw, "dw", channels)
    with _on(device, dict(dh=dh, dx=dx, dw=dw, workspace=workspace), dict(dy=dy, dres=dres, weight=weight, **_kept_names(kept))) as stream:
        space = _workspace(workspace, B.norm_backward_workspace(tokens, channels), device)
        B.norm_backward(kept.act.q.data_ptr(), kept.act.scale.data_ptr(), ld, kept.rstd.data_ptr(), tokens, channels, w, _code(weight), dy.data_ptr(), dy_stride,
                        _DTYPES[dy.dtype], _address(dres), dres_stride, dh.data_ptr(), dh_stride, _DTYPES[dh.dtype], _address(dx), dx_stride, accumulate, to,
                        _code(dw), space.data_ptr(), space.numel() * space.element_size(), stream)
    _written(dh, dx, dw)
    return dh


def _sequences(t: torch.Tensor, offsets: Optional[torch.Tensor]):
    """Checks the shape of a tensor of tokens -> (sequences, tokens, channels)."""
    if offsets is None:
        if t.dim() not in (2, 3):
            _fail(f"tokens are [length, channels], or [sequences, length, channels]: not {tuple(t.shape)}")
        count = 1 if t.dim() == 2 else t.shape[0]
        tokens = t.shape[0] if t.dim() == 2 else t.shape[0] * t.shape[1]
        return B.Sequences(count, tokens, 0, 0), tokens, t.shape[-1]
    if t.dim() != 2:
        _fail(f"tokens with offsets are [tokens, channels]: not {tuple(t.shape)}")
    if offsets.dtype not in _ID_TYPES or offsets.dim() != 1 or offsets.numel() == 0 or not offsets.is_contiguous():
        _fail("offsets must be a contiguous int32 or int64 tensor of one element more than there are sequences")
    return B.Sequences(offsets.numel() - 1, t.shape[0], offsets.data_ptr(), _ID_TYPES[offsets.dtype]), t.shape[0], t.shape[1]


def _tokens(t: torch.Tensor, name: str, like: torch.Tensor, tokens: int, channels: int):
    """Checks a tensor of tokens of `like`'s shape and type -> (address, distance of its rows)."""
    if t.shape != like.shape:
        _fail(f"{name} has shape {tuple(t.shape)}, wanted {tuple(like.shape)}")
    if t.numel() == 0:
        if t.dtype != like.dtype:
            _fail(f"{name} has type {t.dtype}")
        return t.data_ptr(), channels
    flat = _flat(t, name, tokens, channels)
    return flat.data_ptr(), _matrix(flat, name, tokens, channels, (like.dtype,))


def _states(t: Optional[torch.Tensor], name: str, rows: int, channels: int) -> int:
    if t is None:
        return 0
    if t.dtype != torch.float32 or t.shape != (rows, channels) or not t.is_contiguous():
        _fail(f"{name} must be a contiguous float32 tensor of shape {(rows, channels)}, not {tuple(t.shape)} of {t.dtype}")
    return t.data_ptr()


def _recur_kind(kind: str) -> int:
    if kind not in RECUR_KINDS:
        _fail(f"unknown kind {kind!r}; choose from {tuple(RECUR_KINDS)}")
    return RECUR_KINDS[kind]


def recur_empty(gate: torch.Tensor, offsets: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Memory for the states that recur keeps for recur_backward: one for every 128 tokens of a sequence, or of all where there are offsets."""
    sequences, _, channels = _sequences(gate, offsets)
    return torch.empty(B.recur_states(sequences), channels, dtype=torch.float32, device=gate.device)


def recur(gate: torch.Tensor, x: torch.Tensor, kind: str = "convex", first: Optional[torch.Tensor] = None, offsets: Optional[torch.Tensor] = None,
          y: Optional[torch.Tensor] = None, last: Optional[torch.Tensor] = None, states: Optional[torch.Tensor] = None,
          workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y[t] = h[t] = a[t] * h[t-1] + c * x[t] with a = sigmoid(gate), for every channel by itself; c is 1 ("free"), 1 - a ("convex") or
    sqrt(1 - a^2) ("unit").

    gate, x and y are of one type: [length, channels], [sequences, length, channels], or with `offsets` [sequences + 1] sequences one behind the other
    in [tokens, channels], offsets[s] .. offsets[s+1]-1 being sequence s (rows behind the last one are left as they are; a new y has zeros there).
    y may lie over gate or x.
    h is float32: `first` [sequences, channels] goes in (None: 0) and `last`, which may be first where there are no offsets, comes out.  `states`
    (recur_empty) takes what recur_backward needs.  `workspace`: device memory of layers_binding.recur_workspace bytes; None takes torch's."""
    if y is not None and _native.recur(gate, x, RECUR_KINDS.get(kind), first, offsets, y, last, states, workspace) is None:
        return y
    sequences, tokens, channels = _sequences(gate, offsets)
    if y is None:
        y = (torch.empty if offsets is None else torch.zeros)(gate.shape, dtype=gate.dtype, device=gate.device)
    device = _device(gate, x, first, offsets, y, last, states, workspace)
    if gate.dtype not in _DTYPES:
        _fail(f"gate has type {gate.dtype}")
    sides = [_tokens(t, name, gate, tokens, channels) for t, name in ((gate, "gate"), (x, "x"), (y, "y"))]
    first_at, last_at = (_states(t, name, sequences.n_sequences, channels) for t, name in ((first, "first"), (last, "last")))
    if offsets is not None and first_at and first_at == last_at:
        _fail("last over first takes sequences of one length")
    states_at = _states(states, "states", B.recur_states(sequences), channels)
    with _on(device, dict(y=y, last=last, states=states, workspace=workspace), dict(gate=gate, x=x, first=first, offsets=offsets)) as stream:
        space = _workspace(workspace, B.recur_workspace(sequences, channels, _DTYPES[gate.dtype]), device)
        B.recur(sequences, channels, _recur_kind(kind), _DTYPES[gate.dtype], *sides[0], *sides[1], first_at, *sides[2], last_at, states_at, space.data_ptr(),
                space.numel() * space.element_size(), stream)
    _written(y, last, states)
    return y


def recur_backward(gate: torch.Tensor, x: torch.Tensor, states: torch.Tensor, dy: torch.Tensor, kind: str = "convex", first: Optional[torch.Tensor] = None,
                   offsets: Optional[torch.Tensor] = None, dlast: Optional[torch.Tensor] = None, dgate: Optional[torch.Tensor] = None,
                   dx: Optional[torch.Tensor] = None, dfirst: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Gradients of recur's gate and x, and of `first` where `dfirst` is given, from those of its y and, where given, of `last`; gate, x, kind, first and offsets as
    they were, `states` as recur has written them.  Returns (dgate, dx); rows behind the last sequence are left as they are (new tensors have zeros there).
    dgate and dx may each lie over gate, x or dy."""
    if dgate is not None and dx is not None and _native.recur_backward(gate, x, states, dy, RECUR_KINDS.get(kind), first, offsets, dlast, dgate, dx, dfirst, workspace) is None:
        return dgate, dx
    sequences, tokens, channels = _sequences(gate, offsets)
    fresh = torch.empty if offsets is None else torch.zeros
    dgate = fresh(gate.shape, dtype=gate.dtype, device=gate.device) if dgate is None else dgate
    dx = fresh(gate.shape, dtype=gate.dtype, device=gate.device) if dx is None else dx
    device = _device(gate, x, states, dy, first, offsets, dlast, dgate, dx, dfirst, workspace)
    if gate.dtype not in _DTYPES:
        _fail(f"gate has type {gate.dtype}")
    sides = [_tokens(t, name, gate, tokens, channels) for t, name in ((gate, "gate"), (x, "x"), (dy, "dy"), (dgate, "dgate"), (dx, "dx"))]
    first_at, dlast_at, dfirst_at = (_states(t, name, sequences.n_sequences, channels) for t, name in ((first, "first"), (dlast, "dlast"), (dfirst, "dfirst")))
    if dlast_at and dlast_at == dfirst_at:
        _fail("dfirst must be other memory than dlast")
    states_at = _states(states, "states", B.recur_states(sequences), channels)
    with _on(device, dict(dgate=dgate, dx=dx, dfirst=dfirst, workspace=workspace),
             dict(gate=gate, x=x, dy=dy, first=first, dlast=dlast, states=states, offsets=offsets)) as stream:
        space = _workspace(workspace, B.recur_workspace(sequences, channels, _DTYPES[gate.dtype]), device)
        B.recur_backward(sequences, channels, _recur_kind(kind), _DTYPES[gate.dtype], *sides[0], *sides[1], first_at, states_at, *sides[2], dlast_at, *sides[3],
                         *sides[4], dfirst_at, space.data_ptr(), space.numel() * space.element_size(), stream)
    _written(dgate, dx, dfirst)
    return dgate, dx


def distill(logits: torch.Tensor, ids: Optional[torch.Tensor] = None, teacher: Optional[torch.Tensor] = None, labels: Optional[torch.Tensor] = None,
            temperature: float = 1.0, label_weight: float = 1.0, teacher_weight: float = 1.0, row_weight: Optional[torch.Tensor] = None,
            loss: Optional[torch.Tensor] = None, dlogits: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The loss of every row of logits [tokens, vocabulary], and its gradient where `dlogits` is given (of logits' type; it may be logits):

      row_weight * (label_weight * cross_entropy(logits, labels)
                    + teacher_weight * temperature^2 * KL(p, softmax(logits / temperature))),  p = softmax(teacher / temperature)

    labels [tokens] (integers, contiguous; one outside the vocabulary: none) and the teacher's top logits `teacher` [tokens, top] with their `ids`; either may be
    left out (labels alone: cross entropy).  An id outside the vocabulary or a logit of -inf is no entry.  row_weight float32 [tokens] (None: 1).
    Rows with weight 0, and those with neither label nor entry, have loss 0 and gradient 0 whatever is in them.  Where entries cover the vocabulary, the
    divergence nears 0 as the temperature grows, and the loss is what binary32 leaves of a difference: 1e-6 of it at 4, 2e-4 at 64, 6 % at 1024.
    `workspace`: device memory of layers_binding.distill_workspace(tokens, vocabulary, top) bytes; None takes torch's.  Returns `loss`, float32 [tokens]."""
    if loss is not None and _native.distill(logits, ids, teacher, labels, temperature, label_weight, teacher_weight, row_weight, loss, dlogits, workspace) is None:
        return loss
    stride = _matrix(logits, "logits", None, None)
    tokens, vocabulary = logits.shape
    if loss is None:
        loss = torch.empty(tokens, dtype=torch.float32, device=logits.device)
    device = _device(logits, ids, teacher, labels, row_weight, loss, dlogits, workspace)
    if vocabulary < 1 or (ids is None) != (teacher is None):
        _fail("a vocabulary of one logit or more, and ids and teacher together")
    top, ids_stride, teacher_stride = 0, 0, 0
    if ids is not None:
        ids_stride = _matrix(ids, "ids", tokens, None, _ID_TYPES)
        top = ids.shape[1]
        teacher_stride = _matrix(teacher, "teacher", tokens, top)
        if top > B.MAX_TOP:
            _fail(f"{top} entries of the teacher, at most {B.MAX_TOP}")
    labels_at, weight_at, loss_at = (_vector(labels, "labels", tokens, _ID_TYPES), _vector(row_weight, "row_weight", tokens, (torch.float32,)),
                                     _vector(loss, "loss", tokens, (torch.float32,)))
    dz_stride = 0
    if dlogits is not None:
        dz_stride = _matrix(dlogits, "dlogits", tokens, vocabulary, (logits.dtype,))
        if _same_place(dlogits, logits) and dz_stride != stride:
            _fail("dlogits over logits must have its strides")
    if tokens and row_weight is not None and _same_place(loss, row_weight):
        _fail("loss must be other memory than row_weight")
    with _on(device, dict(loss=loss, dlogits=dlogits, workspace=workspace), dict(logits=logits, labels=labels, ids=ids, teacher=teacher, row_weight=row_weight)) as stream:
        space = _workspace(workspace, B.distill_workspace(tokens, vocabulary, top), device)
        B.distill(logits.data_ptr(), stride, _DTYPES[logits.dtype], tokens, vocabulary, labels_at, _code(labels, _ID_TYPES), _address(ids), ids_stride,
                  _code(ids, _ID_TYPES), _address(teacher), teacher_stride, _code(teacher), top, temperature, label_weight, teacher_weight, weight_at, loss_at,
                  _address(dlogits), dz_stride, space.data_ptr(), space.numel() * space.element_size(), stream)
    _written(loss, dlogits)
    return loss
