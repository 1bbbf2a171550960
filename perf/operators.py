"""Performance cases of the operators that make a training step's per-layer gradients: embedding lookup and its gradient,
and activation checkpoints held in 8 bits with their use in the backward pass.

  embed            out = sum over tables of scale * table[ids]; an id outside the table stands for no row
  embed_grad       the gradient of one table: every row's tokens summed, rows without tokens zero
  act_store        x into 8 bits with a scale for each channel and group of 128 tokens, and f(x) in the same pass
  act_backward     dy * f'(x^) and f(x^) from the 8 bits
  act_linear_grad  weight and bias gradient of a linear layer from its output's gradient and its input's 8 bits

Sizes are those of the transformer encoder (hidden 1024, feed-forward 4096, vocabulary 30522, 512 positions, batches of
8 x 512 tokens) and of the VGG-16 classifier (25088 to 4096, batch 32) in workloads.py, and general ones around them.
`exact` restates every operator in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
GROUP = 128                              # tokens that share a channel's scale
LARGEST = 2 * 32775 * 1024 * 4096        # multiplications and additions of the largest listed case
MOST_BYTES = 1.9e9                       # bytes of the longest listed case


def listed():
    return [
        # one new token of a sequence, word + position + type: latency
        {"name": "embed one token", "op": "embed", "tokens": 1, "dim": 1024, "rows": 30522, "tables": 3, "table": "f32",
         "out": "bf16", "ids": "i64", "holes": 0.0},
        # the encoder's input: 8 x 512 tokens, word + position + type from binary32 master weights
        {"name": "embed a batch", "op": "embed", "tokens": 4096, "dim": 1024, "rows": 30522, "tables": 3, "table": "f32",
         "out": "bf16", "ids": "i64", "holes": 0.0},
        # the encoder's word table, its largest gradient tensor: few tokens, many rows, frequent words
        {"name": "embed_grad words", "op": "embed_grad", "tokens": 4096, "dim": 1024, "rows": 30522, "dy": "bf16",
         "grad": "bf16", "ids": "i64", "spread": "words", "holes": 0.0},
        # its token-type table: all tokens in two rows
        {"name": "embed_grad types", "op": "embed_grad", "tokens": 4096, "dim": 1024, "rows": 2, "dy": "bf16",
         "grad": "bf16", "ids": "i64", "spread": "even", "holes": 0.0},
        # a long, ragged batch with padded places, binary32
        {"name": "embed_grad long", "op": "embed_grad", "tokens": 65543, "dim": 1024, "rows": 30522, "dy": "f32",
         "grad": "f32", "ids": "i32", "spread": "words", "holes": 0.1},
        # the feed-forward layer's inner activation: checkpoint and GELU in one pass
        {"name": "act_store gelu", "op": "act_store", "tokens": 4096, "channels": 4096, "dtype": "bf16", "kind": "gelu"},
        # odd sizes, binary32, checkpoint alone
        {"name": "act_store odd", "op": "act_store", "tokens": 1003, "channels": 1001, "dtype": "f32", "kind": "identity"},
        # back through the GELU of the encoder's feed-forward layer
        {"name": "act_backward gelu", "op": "act_backward", "tokens": 4096, "channels": 4096, "dtype": "bf16",
         "kind": "gelu", "y": False},
        # a long batch, gradient and recomputed activation together
        {"name": "act_backward long", "op": "act_backward", "tokens": 65536, "channels": 4096, "dtype": "f16",
         "kind": "gelu_tanh", "y": True},
        # VGG-16's first classifier layer, batch 32, binary32: the weight gradient's bytes count
        {"name": "act_linear_grad classifier", "op": "act_linear_grad", "tokens": 32, "channels": 25088, "outputs": 4096,
         "dy": "f32", "grad": "f32", "bias": True},
        # the encoder's feed-forward layer
        {"name": "act_linear_grad ffn", "op": "act_linear_grad", "tokens": 4096, "channels": 1024, "outputs": 4096,
         "dy": "bf16", "grad": "bf16", "bias": True},
        # the same layer on a long, ragged batch in binary16
        {"name": "act_linear_grad long", "op": "act_linear_grad", "tokens": 32775, "channels": 1024, "outputs": 4096,
         "dy": "f16", "grad": "f16", "bias": True},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A channel count: every third as it falls, the others multiples of 8 or 64, as layers have them."""
    n, step = _log(rng, lo, hi), rng.choice((1, 8, 64))
    return max(step, n // step * step)


def draw(rng):
    op = rng.choice(("embed", "embed_grad", "act_store", "act_backward", "act_linear_grad"))
    types = ("f32", "bf16", "f16")
    while True:
        if op == "embed":
            case = {"op": op, "tokens": _log(rng, 1, 65536), "dim": _width(rng, 8, 4096), "rows": _log(rng, 2, 100000),
                    "tables": rng.randint(1, 3), "table": rng.choice(types), "out": rng.choice(types),
                    "ids": rng.choice(("i32", "i64")), "holes": rng.choice((0.0, 0.2))}
        elif op == "embed_grad":
            dy = rng.choice(types)
            case = {"op": op, "tokens": _log(rng, 1, 65536), "dim": _width(rng, 8, 4096), "rows": _log(rng, 2, 60000),
                    "dy": dy, "grad": rng.choice((dy, "f32")), "ids": rng.choice(("i32", "i64")),
                    "spread": rng.choice(("words", "even")), "holes": rng.choice((0.0, 0.2))}
        elif op == "act_store":
            case = {"op": op, "tokens": _log(rng, 1, 65536), "channels": _width(rng, 8, 8192), "dtype": rng.choice(types),
                    "kind": rng.choice(("identity", "gelu", "gelu_tanh", "silu"))}
        elif op == "act_backward":
            case = {"op": op, "tokens": _log(rng, 1, 65536), "channels": _width(rng, 8, 8192), "dtype": rng.choice(types),
                    "kind": rng.choice(("gelu", "gelu_tanh", "silu")), "y": rng.random() < 0.5}
        else:
            dy = rng.choice(types)
            case = {"op": op, "tokens": _log(rng, 1, 65536), "channels": _width(rng, 8, 25088),
                    "outputs": _width(rng, 8, 8192), "dy": dy, "grad": rng.choice((dy, "f32")),
                    "bias": rng.random() < 0.7}
        cost = work(case)
        if cost["bytes"] <= MOST_BYTES and cost["flops"] <= LARGEST and 3072 not in case.values():
            return case


# ---- inputs --------------------------------------------------------------------------------------------------------

def _ids(gen, tokens, rows, kind, spread, holes):
    """Token numbers: "words" have the frequency of words (one over the rank), "even" are even; holes are padded places."""
    u = torch.rand(tokens, generator=gen, device="cuda", dtype=torch.float64)
    ids = (torch.exp(u * math.log(rows + 1.0)) - 1.0) if spread == "words" else u * rows
    ids = ids.long().clamp_(0, rows - 1)
    if spread == "words":                # ranks in no order, as a vocabulary has them
        ids = torch.randperm(rows, generator=gen, device="cuda")[ids]
    if holes > 0:
        ids[torch.rand(tokens, generator=gen, device="cuda") < holes] = -1
    return ids.to(torch.int32 if kind == "i32" else torch.int64)


def _normal(gen, shape, dtype, sigma):
    x = torch.empty(shape, dtype=DTYPES[dtype], device="cuda")
    return x.normal_(0.0, sigma, generator=gen)


def _activation(gen, tokens, channels, dtype):
    """Activations: every channel has a size of its own, and a few are far larger than the others."""
    size = torch.exp(0.5 * torch.randn(channels, generator=gen, device="cuda"))
    size[torch.rand(channels, generator=gen, device="cuda") < 0.01] *= 20.0
    return _normal(gen, (tokens, channels), dtype, 1.0).mul_(size.to(DTYPES[dtype]))


def _groups(tokens):
    return (tokens + GROUP - 1) // GROUP


def _padded(channels):
    return (channels + 15) // 16 * 16    # rows of a checkpoint begin on 16 bytes


def _code(x):
    """x in 8 bits: (q, scale), rows padded with zeros; elementary operations in 32 bits."""
    tokens, channels = x.shape
    groups = _groups(tokens)
    amax = x.abs().float()
    amax = torch.cat([amax, amax.new_zeros(groups * GROUP - tokens, channels)]).view(groups, GROUP, channels).amax(1)
    scale = torch.where(amax < math.inf, amax.clamp(min=2.0 ** -100) * (1.0 / 127.0), math.nan)
    q = torch.round(x.float() * scale.reciprocal().repeat_interleave(GROUP, 0)[:tokens]).clamp(-127, 127).to(torch.int8)
    pad = _padded(channels) - channels
    return torch.nn.functional.pad(q, (0, pad)), torch.nn.functional.pad(scale, (0, pad))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, tokens = case["op"], case["tokens"]
    state = {"case": case}
    if op == "embed":
        sizes = [case["rows"], 512, 2][:case["tables"]]
        state["tables"] = [_normal(gen, (n, case["dim"]), case["table"], 0.02) for n in sizes]
        state["scales"] = [math.sqrt(case["dim"]), 1.0, 1.0][:case["tables"]]
        ids = [_ids(gen, tokens, case["rows"], case["ids"], "words", case["holes"]),
               torch.arange(tokens, device="cuda").remainder(512).to(torch.int32 if case["ids"] == "i32" else torch.int64),
               _ids(gen, tokens, 2, case["ids"], "even", 0.0)]
        state["ids"] = ids[:case["tables"]]
        state["out"] = torch.empty(tokens, case["dim"], dtype=DTYPES[case["out"]], device="cuda")
    elif op == "embed_grad":
        state["ids"] = _ids(gen, tokens, case["rows"], case["ids"], case["spread"], case["holes"])
        state["dy"] = _normal(gen, (tokens, case["dim"]), case["dy"], 1e-3)
        state["scale"] = math.sqrt(case["dim"])
        state["grad"] = torch.empty(case["rows"], case["dim"], dtype=DTYPES[case["grad"]], device="cuda")
    elif op == "act_store":
        channels = case["channels"]
        state["x"] = _activation(gen, tokens, channels, case["dtype"])
        state["q"] = torch.empty(tokens, _padded(channels), dtype=torch.int8, device="cuda")
        state["scale"] = torch.empty(_groups(tokens), _padded(channels), device="cuda")
        state["y"] = torch.empty_like(state["x"]) if case["kind"] != "identity" else None
    else:
        state["q"], state["scale"] = _code(_activation(gen, tokens, case["channels"], "bf16"))
        if op == "act_backward":
            state["dy"] = _normal(gen, (tokens, case["channels"]), case["dtype"], 1e-3)
            state["dx"] = torch.empty_like(state["dy"])
            state["y"] = torch.empty_like(state["dy"]) if case["y"] else None
        else:
            state["dy"] = _normal(gen, (tokens, case["outputs"]), case["dy"], 1e-3)
            state["dw"] = torch.empty(case["outputs"], case["channels"], dtype=DTYPES[case["grad"]], device="cuda")
            state["db"] = torch.empty(case["outputs"], dtype=DTYPES[case["grad"]], device="cuda") if case["bias"] else None
    return state


# ---- one pass ------------------------------------------------------------------------------------------------------

def _gelu(x):
    return 0.5 * x * (1.0 + torch.erf(x * math.sqrt(0.5)))


def _gelu_slope(x):
    return 0.5 * (1.0 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) * (1.0 / math.sqrt(2.0 * math.pi))


_TANH_A, _TANH_B = math.sqrt(2.0 / math.pi), 0.044715


def _gelu_tanh(x):
    return 0.5 * x * (1.0 + torch.tanh(_TANH_A * (x + _TANH_B * x * x * x)))


def _gelu_tanh_slope(x):
    t = torch.tanh(_TANH_A * (x + _TANH_B * x * x * x))
    return 0.5 * (1.0 + t) + 0.5 * x * (1.0 - t * t) * _TANH_A * (1.0 + 3.0 * _TANH_B * x * x)


def _silu(x):
    return x / (1.0 + torch.exp(-x))


def _silu_slope(x):
    s = 1.0 / (1.0 + torch.exp(-x))
    return s * (1.0 + x * (1.0 - s))


VALUE = {"identity": lambda x: x, "gelu": _gelu, "gelu_tanh": _gelu_tanh, "silu": _silu}
SLOPE = {"gelu": _gelu_slope, "gelu_tanh": _gelu_tanh_slope, "silu": _silu_slope}


def _decoded(q, scale, tokens, channels):
    return q[:, :channels].to(scale.dtype) * scale[:, :channels].repeat_interleave(GROUP, 0)[:tokens]


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    from paper_1912_09268_amd import layers
    case = state["case"]
    op = case["op"]
    if op == "embed":
        return layers.embed(state["tables"], state["ids"], scales=state["scales"], out=state["out"])
    if op == "embed_grad":
        return layers.embed_grad(state["dy"], state["ids"], state["grad"], scale=state["scale"])
    if op == "act_store":
        act = layers.Act8(state["q"], state["scale"], case["channels"])
        layers.act_store(state["x"], act, kind=case["kind"], y=state["y"])
        return [act.q[:, :case["channels"]], act.scale[:, :case["channels"]], state["y"]]
    act = layers.Act8(state["q"], state["scale"], case["channels"])
    if op == "act_backward":
        layers.act_backward(act, state["dy"], kind=case["kind"], dx=state["dx"], y=state["y"])
        return [state["dx"], state["y"]]
    layers.act_linear_grad(state["dy"], act, state["dw"], db=state["db"])
    return [state["dw"], state["db"]]


def _picked(table, ids, scale):
    here = (ids >= 0) & (ids < table.shape[0])
    return torch.where(here[:, None], table[ids.long().clamp(0, table.shape[0] - 1)].float() * scale, 0.0)


def _run_plain(state):
    case = state["case"]
    op, tokens = case["op"], case["tokens"]
    if op == "embed":
        rows = [_picked(t, i, s) for t, i, s in zip(state["tables"], state["ids"], state["scales"])]
        return sum(rows[1:], rows[0]).to(state["out"].dtype)
    if op == "embed_grad":
        ids = state["ids"].long()
        rows = case["rows"]
        at = torch.where((ids >= 0) & (ids < rows), ids, rows)                  # padded places go to a row of their own
        total = torch.zeros(rows + 1, case["dim"], device="cuda").index_add_(0, at, state["dy"].float())[:rows]
        return (total * state["scale"]).to(state["grad"].dtype)
    if op == "act_store":
        q, scale = _code(state["x"])
        y = None if state["y"] is None else VALUE[case["kind"]](state["x"].float()).to(state["x"].dtype)
        return [q[:, :case["channels"]], scale[:, :case["channels"]], y]
    x = _decoded(state["q"], state["scale"], tokens, case["channels"])
    if op == "act_backward":
        dx = (state["dy"].float() * SLOPE[case["kind"]](x)).to(state["dy"].dtype)
        return [dx, VALUE[case["kind"]](x).to(state["dy"].dtype) if case["y"] else None]
    dy = state["dy"].float()
    dw = dy.t() @ x
    db = dy.sum(0) if case["bias"] else None
    return [dw.to(state["dw"].dtype), None if db is None else db.to(state["dw"].dtype)]


# ---- cost and definition -------------------------------------------------------------------------------------------

def work(case):
    op, tokens = case["op"], case["tokens"]
    if op == "embed":
        places, per_id = tokens * case["dim"], 4 if case["ids"] == "i32" else 8
        rows = sum(min(tokens, n) for n in [case["rows"], 512, 2][:case["tables"]])
        return {"bytes": tokens * per_id * case["tables"] + rows * case["dim"] * SIZE[case["table"]] + places * SIZE[case["out"]],
                "flops": 2 * places * case["tables"]}
    if op == "embed_grad":
        places, per_id = tokens * case["dim"], 4 if case["ids"] == "i32" else 8
        return {"bytes": tokens * per_id + places * SIZE[case["dy"]] + case["rows"] * case["dim"] * SIZE[case["grad"]],
                "flops": 2 * places}
    places, scales = tokens * case["channels"], 4 * _groups(tokens) * case["channels"]
    if op == "act_store":
        size = SIZE[case["dtype"]]
        return {"bytes": places * (size + 1 + (size if case["kind"] != "identity" else 0)) + scales, "flops": 4 * places}
    if op == "act_backward":
        return {"bytes": places * (1 + SIZE[case["dtype"]] * (3 if case["y"] else 2)) + scales, "flops": 16 * places}
    weights = case["outputs"] * case["channels"] * SIZE[case["grad"]]
    return {"bytes": places + scales + tokens * case["outputs"] * SIZE[case["dy"]] + weights,
            "flops": 2 * places * case["outputs"]}


def exact(case, seed):
    """Every operator's definition in 64 bits.  The 8-bit numbers of act_store are whole and have no such value."""
    state = prepare(case, seed)
    op, tokens, f64 = case["op"], case["tokens"], torch.float64
    if op == "embed":
        out = torch.zeros(tokens, case["dim"], dtype=f64, device="cuda")
        for table, ids, scale in zip(state["tables"], state["ids"], state["scales"]):
            at = torch.nonzero((ids >= 0) & (ids < table.shape[0])).squeeze(1)
            out[at] += scale * table[ids[at].long()].to(f64)
        return out
    if op == "embed_grad":
        at = torch.nonzero((state["ids"] >= 0) & (state["ids"] < case["rows"])).squeeze(1)
        at = at[torch.argsort(state["ids"][at].long(), stable=True)]
        rows, counts = torch.unique_consecutive(state["ids"][at].long(), return_counts=True)
        grad = torch.zeros(case["rows"], case["dim"], dtype=f64, device="cuda")
        if rows.numel():
            run_of = torch.repeat_interleave(torch.arange(rows.numel(), device="cuda"), counts)
            sums = torch.zeros(rows.numel(), case["dim"], dtype=f64, device="cuda")
            sums.index_add_(0, run_of, state["dy"][at].to(f64))
            grad[rows] = state["scale"] * sums
        return grad
    if op == "act_store":
        x = state["x"].to(f64)
        whole = torch.zeros(_groups(tokens) * GROUP, case["channels"], dtype=f64, device="cuda")
        whole[:tokens] = x.abs()
        scale = whole.view(-1, GROUP, case["channels"]).amax(1).clamp(min=2.0 ** -100) / 127.0
        return [None, scale, None if state["y"] is None else _exact_value(case["kind"], x)]
    group = torch.arange(tokens, device="cuda") // GROUP
    x = state["q"][:, :case["channels"]].to(f64) * state["scale"].to(f64)[group, :case["channels"]]
    dy = state["dy"].to(f64)
    if op == "act_backward":
        dx = dy * _exact_slope(case["kind"], x)
        return [dx, _exact_value(case["kind"], x) if case["y"] else None]
    dw, db = torch.matmul(x.t(), dy).t(), dy.sum(0) if case["bias"] else None
    return [dw.contiguous(), db]


def _exact_value(kind, x):
    if kind == "gelu":
        return x * 0.5 * torch.erfc(-x / math.sqrt(2.0))
    if kind == "gelu_tanh":              # (1 + tanh u) / 2 is the logistic function of 2 u
        return x * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (x + 0.044715 * x ** 3))
    return x * torch.sigmoid(x)


def _exact_slope(kind, x):
    if kind == "gelu":
        return 0.5 * torch.erfc(-x / math.sqrt(2.0)) + x * torch.exp(-x * x / 2.0) / math.sqrt(2.0 * math.pi)
    if kind == "gelu_tanh":
        s = torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (x + 0.044715 * x ** 3))
        return s + x * 2.0 * s * (1.0 - s) * math.sqrt(2.0 / math.pi) * (1.0 + 3 * 0.044715 * x * x)
    s = torch.sigmoid(x)
    return s + x * s * (1.0 - s)
