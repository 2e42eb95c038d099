"""Host-side checks of the layer operators that need no GPU: symbols, layouts, and refusals before anything is enqueued."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

import paper_2508_16905_amd as ta
from paper_2508_16905_amd import binding as B
from paper_2508_16905_amd.build import build_library

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = {"triaccel_linear_args": B.LinearArgs, "triaccel_linear_backward_args": B.LinearBackwardArgs, "triaccel_gated_args": B.GatedArgs,
           "triaccel_gated_backward_args": B.GatedBackwardArgs, "triaccel_residual_norm_args": B.ResidualNormArgs,
           "triaccel_residual_norm_backward_args": B.ResidualNormBackwardArgs, "triaccel_dropout_args": B.DropoutArgs,
           "triaccel_dropout_spec": B.DropoutSpec, "triaccel_norm_spec": B.NormSpec}


@pytest.fixture(scope="module")
def lib():
    build_library(force=False)
    return ta.load_library()


def test_every_declared_symbol_is_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "triaccel_layers.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(triaccel_[a-z0-9_]+)\s*\(", text)))
    assert sorted(B.LAYER_EXPORTS) == names
    for name in names:
        assert hasattr(lib, name), name


def test_ctypes_layout_matches_the_header(tmp_path):
    fields = [(s, f) for s, c in STRUCTS.items() for f, _ in c._fields_]
    text = '#include <stdio.h>\n#include <stddef.h>\n#include "triaccel_layers.h"\nint main(void){\n'
    text += "".join(f'printf("%zu\\n", sizeof({s}));\n' for s in STRUCTS)
    text += "".join(f'printf("%zu\\n", offsetof({s}, {"in" if f == "in_" else f}));\n' for s, f in fields)
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text(text + "return 0;}\n")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [C.sizeof(c) for c in STRUCTS.values()] + [getattr(STRUCTS[s], f).offset for s, f in fields]


ADDRESS = 0x100000  # of nothing: no refused call reads it


def linear(**kw):
    a = B.LinearArgs(struct_size=C.sizeof(B.LinearArgs), dtype=B.BF16, rows=4, in_=16, out=8, x=ADDRESS, ldx=16, weight=ADDRESS, ldw=16, y=ADDRESS, ldy=8,
                     scale=1.0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def norm(**kw):
    a = B.ResidualNormArgs(struct_size=C.sizeof(B.ResidualNormArgs), dtype=B.BF16, rows=4, cols=16, residual=ADDRESS, ldr=16, scale=1.0)
    a.norm = B.NormSpec(1, B.FP32, None, None, 1e-6, 0)
    a.y, a.ldy = ADDRESS, 16
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("code,change", [
    (-1, dict(struct_size=8)), (-1, dict(rows=-1)), (-1, dict(in_=0)), (-1, dict(out=0)), (-1, dict(rows=1 << 31)), (-1, dict(ldx=15)), (-1, dict(ldw=8)),
    (-1, dict(ldy=7)), (-1, dict(act=5)), (-1, dict(act=-1)), (-1, dict(scale=float("nan"))), (-1, dict(scale=float("inf"))),
    (-1, dict(drop=B.DropoutSpec(1.0, 0, 0, None))), (-1, dict(drop=B.DropoutSpec(-0.1, 0, 0, None))), (-1, dict(drop=B.DropoutSpec(float("nan"), 0, 0, None))),
    (-2, dict(dtype=3)), (-2, dict(bias=ADDRESS, bias_dtype=7)), (-4, dict(x=None)), (-4, dict(weight=None)), (-4, dict(y=None)),
    (-5, dict(x=ADDRESS + 1)), (-5, dict(pre=ADDRESS + 1, ldpre=8)), (-5, dict(drop=B.DropoutSpec(0.5, 0, 0, ADDRESS + 4))),
    (-1, dict(residual=ADDRESS, ldr=7)), (-1, dict(rows=64, in_=1 << 20, ldx=1 << 20, ldw=1 << 20)),  # the last: no workspace for a long k
])
def test_linear_refuses(lib, code, change):
    assert lib.triaccel_linear(C.byref(linear(**change)), None) == code
    assert lib.triaccel_last_error() != b""


@pytest.mark.parametrize("code,change", [
    (-1, dict(cols=16385, ldr=16385, ldy=16385)), (-1, dict(norm=B.NormSpec(3, B.FP32, None, None, 1e-6, 0))),
    (-1, dict(norm=B.NormSpec(1, B.FP32, None, None, 0.0, 0))), (-2, dict(norm=B.NormSpec(1, 9, ADDRESS, None, 1e-6, 0))),
    (-5, dict(norm=B.NormSpec(1, B.FP32, ADDRESS + 2, None, 1e-6, 0))), (-4, dict(y=None)), (-4, dict(block=ADDRESS, ldb=16)),
    (-1, dict(rows_per_gate=-1)), (-1, dict(gate=ADDRESS, gate_dtype=B.FP32, rows_per_gate=2, ldgate=15)), (-1, dict(scale=float("nan"))),
])
def test_residual_norm_refuses(lib, code, change):
    assert lib.triaccel_residual_norm(C.byref(norm(**change)), None) == code


def test_other_refusals(lib):
    a = B.GatedArgs(struct_size=C.sizeof(B.GatedArgs), dtype=B.BF16, rows=4, in_=16, out=8, x=ADDRESS, ldx=16, w_gate=ADDRESS, w_up=ADDRESS, ldw=16, h=ADDRESS,
                    ldh=8, act=2)
    for code, change in ((-4, dict(w_up=None)), (-4, dict(b_gate=ADDRESS, bias_dtype=2)), (-4, dict(gate=ADDRESS, ldg=8)), (-1, dict(act=0)),
                         (-1, dict(out=1 << 30))):
        b = B.GatedArgs.from_buffer_copy(a)
        for k, v in change.items():
            setattr(b, k, v)
        assert lib.triaccel_gated(C.byref(b), None) == code, change
    g = B.GatedBackwardArgs(struct_size=C.sizeof(B.GatedBackwardArgs), dtype=B.BF16, rows=4, in_=16, out=8, dh=ADDRESS, lddh=8, x=ADDRESS, ldx=16,
                            w_gate=ADDRESS, w_up=ADDRESS, ldw=16, gate=ADDRESS, up=ADDRESS, ldg=8, dx=ADDRESS, lddx=16, dweight_dtype=1, act=2)
    for code, change in ((-1, {}), (-2, dict(dweight_dtype=0)), (-4, dict(dw_gate=ADDRESS, lddw=16)), (-4, dict(db_up=ADDRESS)), (-4, dict(gate=None))):
        b = B.GatedBackwardArgs.from_buffer_copy(g)
        for k, v in change.items():
            setattr(b, k, v)
        assert lib.triaccel_gated_backward(C.byref(b), None) == code, change   # the first: no workspace
    n = B.ResidualNormBackwardArgs(struct_size=C.sizeof(B.ResidualNormBackwardArgs), dtype=B.BF16, rows=4, cols=16, residual=ADDRESS, ldr=16, dresidual=ADDRESS,
                                   lddr=16, dvec_dtype=2, scale=1.0)
    for code, change in ((-1, dict(dnorm_weight=ADDRESS)), (-4, dict(dblock=ADDRESS, lddb=16)), (-4, dict(dgate=ADDRESS)),
                         (-1, dict(dpost_bias=ADDRESS, block=ADDRESS, ldb=16)), (-5, dict(dresidual=ADDRESS + 1))):
        b = B.ResidualNormBackwardArgs.from_buffer_copy(n)
        for k, v in change.items():
            setattr(b, k, v)
        assert lib.triaccel_residual_norm_backward(C.byref(b), None) == code, change
    d = B.DropoutArgs(struct_size=C.sizeof(B.DropoutArgs), dtype=B.BF16, rows=4, cols=16, x=ADDRESS, ldx=16, y=ADDRESS, ldy=16, scale=1.0,
                      drop=B.DropoutSpec(0.5, 1, 2, None))
    for code, change in ((-1, dict(cols=0)), (-4, dict(y=None)), (-1, dict(ldy=3)), (-2, dict(dtype=-1)), (-1, dict(drop=B.DropoutSpec(1.5, 0, 0, None)))):
        b = B.DropoutArgs.from_buffer_copy(d)
        for k, v in change.items():
            setattr(b, k, v)
        assert lib.triaccel_dropout(C.byref(b), None) == code, change
    for call, _ in B._LAYER_CALLS.items():
        assert getattr(lib, call)(None, None) == -4


def test_no_rows_enqueue_nothing(lib):
    assert lib.triaccel_linear(C.byref(linear(rows=0, x=None, y=None)), None) == 0
    assert lib.triaccel_residual_norm(C.byref(norm(rows=0, residual=None, y=None)), None) == 0


def test_workspaces_grow_with_what_they_hold(lib):
    a = B.LinearBackwardArgs(struct_size=C.sizeof(B.LinearBackwardArgs), dtype=B.BF16, rows=100, in_=64, out=50, dweight_dtype=B.BF16, scale=1.0)
    assert lib.triaccel_linear_backward_workspace(C.byref(a)) == 0
    a.dx, a.act = ADDRESS, 2
    assert lib.triaccel_linear_backward_workspace(C.byref(a)) >= 100 * 56 * 2   # dz, whose rows are whole 16-byte units
    a.dtype = 9
    assert lib.triaccel_linear_backward_workspace(C.byref(a)) == -2


def test_the_wrapper_refuses_tensors_of_the_host():
    with pytest.raises(ValueError):
        ta.linear(torch.ones(2, 4), torch.ones(3, 4))


@pytest.mark.parametrize("rows_per_gate", [1 << 31, 1 << 62, -(1 << 62)])
def test_groups_of_rows_past_the_sizes_are_refused(lib, rows_per_gate):
    assert lib.triaccel_residual_norm(C.byref(norm(gate=ADDRESS, gate_dtype=B.FP32, ldgate=16, rows_per_gate=rows_per_gate)), None) == -1
    a = B.ResidualNormBackwardArgs(struct_size=C.sizeof(B.ResidualNormBackwardArgs), dtype=B.BF16, rows=4, cols=16, residual=ADDRESS, ldr=16, dvec_dtype=2,
                                   scale=1.0, rows_per_gate=rows_per_gate)
    assert lib.triaccel_residual_norm_backward_workspace(C.byref(a)) == -1


def test_dropout_of_more_rows_than_a_launch_has(lib):
    d = B.DropoutArgs(struct_size=C.sizeof(B.DropoutArgs), dtype=B.BF16, rows=(1 << 25) + 1, cols=16, x=ADDRESS, ldx=24, y=ADDRESS, ldy=16, scale=1.0,
                      drop=B.DropoutSpec(0.5, 1, 2, None))
    assert lib.triaccel_dropout(C.byref(d), None) == -1
