"""What the operators that make per-layer gradients refuse: at the C entry points (checked before anything touches a GPU) and
on torch tensors."""
import ctypes as C
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_1912_09268_amd import layers_binding as B
from paper_1912_09268_amd import layers

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 12                       # an aligned address that no refused call looks at


def _refused(fn, *args):
    with pytest.raises(B.MgwfbpError) as e:
        fn(*args)
    assert e.value.status == -1


def _table(**kw):
    d = dict(d_rows=P, d_ids=P, n_rows=10, row_stride=64, scale=1.0, id_type=B.I64)
    d.update(kw)
    return B.Table(*d.values())


def test_embed_refuses():
    good = dict(tables=[_table()], table_dtype=B.F32, n_tokens=5, dim=64, d_out=P, out_stride=64, out_dtype=B.BF16)

    def refused(**kw):
        _refused(B.embed, *{**good, **kw}.values())

    refused(tables=[])
    refused(tables=[_table()] * 5)
    refused(table_dtype=3)
    refused(out_dtype=-1)
    refused(n_tokens=-1)
    refused(n_tokens=2 ** 26 + 1)
    refused(dim=-1)
    refused(dim=2 ** 23 + 1)
    refused(d_out=0)
    refused(d_out=P + 1)
    refused(out_stride=63)
    refused(out_stride=2 ** 41)
    for bad in (dict(d_rows=0), dict(d_ids=0), dict(d_rows=P + 2), dict(d_ids=P + 4), dict(n_rows=-1), dict(row_stride=63), dict(id_type=2),
                dict(n_rows=2 ** 40, row_stride=2 ** 40)):
        refused(tables=[_table(), _table(**bad)])
    status = B.lib().mgwfbp_embed(None, 1, B.F32, 5, 64, P, 64, B.F32, None)
    assert status == -1
    # nothing to do is no error, whatever the addresses
    B.embed([_table(d_rows=0, d_ids=0)], B.F32, 0, 64, 0, 64, B.F32)
    B.embed([_table(d_rows=0, d_ids=0, row_stride=0)], B.F32, 5, 0, 0, 0, B.F32)


def test_embed_grad_refuses():
    good = dict(d_ids=P, id_type=B.I64, n_tokens=1000, d_dy=P, dy_stride=64, dy_dtype=B.BF16, scale=1.0, padding_row=-1, accumulate=False,
                d_grad=P, n_rows=10, dim=64, grad_stride=64, grad_dtype=B.F32, d_workspace=P, workspace_bytes=1 << 30)

    def refused(**kw):
        _refused(B.embed_grad, *{**good, **kw}.values())

    for bad in (dict(d_ids=0), dict(d_ids=P + 4), dict(id_type=7), dict(n_tokens=-1), dict(n_tokens=2 ** 26 + 1), dict(d_dy=0), dict(d_dy=P + 1),
                dict(dy_stride=63), dict(dy_dtype=3), dict(d_grad=0), dict(d_grad=P + 2), dict(n_rows=-1), dict(n_rows=2 ** 31 - 1), dict(dim=-1),
                dict(dim=2 ** 23 + 1), dict(grad_stride=63), dict(grad_dtype=-1), dict(d_workspace=0), dict(d_workspace=P + 128),
                dict(workspace_bytes=B.embed_grad_workspace(1000, 10, 64) - 1)):
        refused(**bad)
    B.embed_grad(*{**good, "n_rows": 0, "d_grad": 0}.values())
    B.embed_grad(*{**good, "n_tokens": 0, "accumulate": True, "d_ids": 0, "d_dy": 0, "d_workspace": 0, "workspace_bytes": 0}.values())
    assert B.lib().mgwfbp_embed_grad_workspace(1, 1, 1, None) == -1
    _refused(B.embed_grad_workspace, -1, 1, 1)
    assert B.embed_grad_workspace(0, 0, 0) == 0
    assert B.embed_grad_workspace(100000, 50000, 1024) > 2 * 4 * 100000


def test_act_calls_refuse():
    store = dict(d_x=P, x_stride=20, dtype=B.BF16, n_tokens=9, n_channels=20, kind=B.GELU, d_q=P, d_scale=P, ld=32, d_y=P, y_stride=20)
    for bad in (dict(d_x=0), dict(d_x=P + 1), dict(x_stride=19), dict(dtype=5), dict(n_tokens=-1), dict(n_tokens=2 ** 26 + 1), dict(n_channels=-1),
                dict(n_channels=2 ** 23 + 1), dict(kind=4), dict(kind=-1), dict(d_q=0), dict(d_q=P + 8), dict(d_scale=0), dict(d_scale=P + 4),
                dict(ld=16), dict(ld=40), dict(d_y=P + 1), dict(y_stride=19)):
        _refused(B.act_store, *{**store, **bad}.values())
    B.act_store(*{**store, "n_tokens": 0, "d_x": 0, "d_q": 0, "d_scale": 0}.values())
    back = dict(d_q=P, d_scale=P, ld=32, n_tokens=9, n_channels=20, kind=B.SILU, d_dy=P, dy_stride=20, d_dx=P, dx_stride=20, d_y=P, y_stride=20, dtype=B.F16)
    for bad in (dict(d_q=0), dict(d_q=P + 4), dict(d_scale=0), dict(ld=31), dict(ld=16), dict(n_tokens=-1), dict(n_channels=-1), dict(kind=9), dict(d_dy=0), dict(d_dx=0),
                dict(d_dy=0, d_dx=0, d_y=0), dict(dy_stride=19), dict(dx_stride=19), dict(y_stride=19), dict(d_dy=P + 1), dict(dtype=3)):
        _refused(B.act_backward, *{**back, **bad}.values())
    grad = dict(d_q=P, d_scale=P, ld=32, n_tokens=9, n_channels=20, d_dy=P, dy_stride=7, dy_dtype=B.F32, n_outputs=7, accumulate=False, d_dw=P, dw_stride=20,
                d_db=P, grad_dtype=B.F32, d_workspace=P, workspace_bytes=1 << 30)
    for bad in (dict(d_q=0), dict(d_scale=P + 4), dict(ld=16), dict(ld=33), dict(n_tokens=-1), dict(n_tokens=2 ** 23 + 1), dict(n_channels=-1), dict(d_dy=0), dict(d_dy=P + 2),
                dict(dy_stride=6), dict(dy_dtype=3), dict(n_outputs=-1), dict(d_dw=0), dict(d_dw=P + 2), dict(dw_stride=19), dict(d_db=P + 1), dict(grad_dtype=4),
                dict(n_tokens=4096, d_workspace=0), dict(n_tokens=4096, d_workspace=P + 64),          # split over the tokens: it takes one
                dict(n_tokens=4096, workspace_bytes=B.act_linear_grad_workspace(4096, 20, 7) - 1), dict(n_channels=2 ** 23, n_outputs=2 ** 23, ld=2 ** 23)):
        _refused(B.act_linear_grad, *{**grad, **bad}.values())
    B.act_linear_grad(*{**grad, "n_outputs": 0, "d_dy": 0, "d_dw": 0, "d_db": 0}.values())
    _refused(B.act_dims, -1, 4)
    _refused(B.act_linear_grad_workspace, 1, 1, -1)
    assert B.act_dims(129, 17) == (32, 2) and B.act_dims(0, 0) == (0, 0)
    assert B.lib().mgwfbp_act_linear_grad_workspace(1, 1, 1, None) == -1
    assert B.lib().mgwfbp_act_dims(1, 1, None, None) == 0


def test_the_structure_of_a_table_is_the_headers():
    assert C.sizeof(B.Table) == 40 and B.Table.scale.offset == 32 and B.ACT_GROUP == 128


@pytest.mark.parametrize("call", [
    lambda: layers.embed(torch.zeros(3, 4), torch.zeros(2, dtype=torch.int64)),                              # not on a GPU
    lambda: layers.embed([], []),
    lambda: layers.embed([torch.zeros(3, 4)] * 5, [torch.zeros(2, dtype=torch.int64)] * 5),
    lambda: layers.embed([torch.zeros(3, 4)], [torch.zeros(2, dtype=torch.int64)] * 2),
    lambda: layers.embed_grad(torch.zeros(2, 4), torch.zeros(2, dtype=torch.int64), torch.zeros(3, 4)),
    lambda: layers.act_store(torch.zeros(2, 4, dtype=torch.float64)),
    lambda: layers.act_store(torch.zeros(2, 4, 4)),
    lambda: layers.act_store(torch.zeros(4, 2).t()),
    lambda: layers.act_store(torch.zeros(4, 2), layers.act_empty(4, 2, "cpu"), y=torch.zeros(4, 2)),
    lambda: layers.act_backward(layers.act_empty(4, 2, "cpu")),
    lambda: layers.act_backward(layers.act_empty(4, 2, "cpu"), dx=torch.zeros(4, 2)),
    lambda: layers.act_backward(layers.Act8(torch.zeros(4, 20, dtype=torch.int8), torch.zeros(1, 20), 2), torch.zeros(4, 2)),
    lambda: layers.act_backward(layers.Act8(torch.zeros(200, 16, dtype=torch.int8), torch.zeros(1, 16), 2), torch.zeros(200, 2)),
    lambda: layers.act_backward(layers.Act8(torch.zeros(4, 16, dtype=torch.int8), torch.zeros(1, 16), 17), torch.zeros(4, 17)),
    lambda: layers.act_linear_grad(torch.zeros(4, 3), layers.act_empty(4, 2, "cpu"), torch.zeros(3, 2)),
])
def test_tensors_that_are_refused(call):
    with pytest.raises(ValueError):
        call()


def test_header_library_and_binding_agree(tmp_path):
    """The entry points that the header declares are those that the binding knows and the library exports, and the header is C99."""
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "mgwfbp_layers.h")).read(), flags=re.S)
    declared = sorted(set(re.findall(r"\b(mgwfbp_[a-z0-9_]+)\s*\(", text)))
    assert declared == sorted(B._SIGNATURES)
    handle = C.CDLL(B.library_path())
    assert all(hasattr(handle, name) for name in declared)
    if shutil.which("gcc"):
        source = tmp_path / "client.c"
        source.write_text('#include "mgwfbp_layers.h"\nint main(void) { return mgwfbp_act_dims(1, 1, 0, 0); }\n')
        lib = B.library_path()
        r = subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), str(source), "-o",
                            str(tmp_path / "client"), lib, "-Wl,-rpath," + os.path.dirname(lib), "-Wl,-rpath,/opt/rocm/lib",
                            "-Wl,--allow-shlib-undefined"], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        assert subprocess.run([str(tmp_path / "client")], timeout=60).returncode == 0


def test_a_missing_library_fails_loudly(monkeypatch):
    monkeypatch.setenv("MGWFBP_LAYERS_LIBRARY", "/nonexistent/libmgwfbp_layers.so")
    monkeypatch.setattr(B, "_LIB", None)
    with pytest.raises(B.MgwfbpError):
        B.embed([_table()], B.F32, 5, 64, P, 64, B.F32)
