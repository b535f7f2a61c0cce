"""The host side of the row operators (csrc/row_ops.cu) without a device: what is refused before a launch, over the stand-in for the CUDA
runtime (host_path/), and the binding's own checks and struct layouts."""
import ctypes as C
import os
import subprocess
from types import SimpleNamespace

import pytest
import torch

from paper_2507_19131_b200 import binding as mq
from paper_2507_19131_b200 import build as mq_build

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
OK, INVALID, UNSUPPORTED, SMALL, INTERNAL = 0, -1, -2, -3, -6
F32, BF16, F16 = 0, 1, 2
NONE, LAYER, RMS = 0, 1, 2
AT = 0x7000_0000_0000                     # made-up device addresses, 1 MiB apart


class Matrix(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("row_stride", C.c_int64), ("block_rows", C.c_int),
                ("scale", C.c_void_p), ("scale_row_stride", C.c_int64), ("scale_col_stride", C.c_int64)]


class NormS(C.Structure):
    _fields_ = [("kind", C.c_int), ("gamma", C.c_void_p), ("beta", C.c_void_p), ("eps", C.c_float)]


class Params(C.Structure):
    _fields_ = [("rows", C.c_int64), ("dim", C.c_int), ("x_dtype", C.c_int), ("y_dtype", C.c_int), ("gate_dtype", C.c_int),
                ("x", C.c_void_p), ("x_stride", C.c_int64), ("y", C.c_void_p), ("y_stride", C.c_int64),
                ("gate", C.c_void_p), ("gate_stride", C.c_int64), ("rows_per_gate", C.c_int64), ("scale", C.c_float),
                ("post", NormS), ("pre", NormS), ("x_out", C.c_void_p), ("x_out_stride", C.c_int64), ("h", C.c_void_p), ("h_stride", C.c_int64),
                ("pow2", C.c_int)]


class Grads(C.Structure):
    _fields_ = [("dx_out", C.c_void_p), ("dx_out_stride", C.c_int64), ("dh", C.c_void_p), ("dh_stride", C.c_int64),
                ("dx", C.c_void_p), ("dx_stride", C.c_int64), ("dy", C.c_void_p), ("dy_stride", C.c_int64),
                ("dgate", C.c_void_p), ("dgate_stride", C.c_int64),
                ("dpost_gamma", C.c_void_p), ("dpost_beta", C.c_void_p), ("dpre_gamma", C.c_void_p), ("dpre_beta", C.c_void_p)]


def test_struct_layouts_are_those_of_the_header(tmp_path):
    """The C compiler's offsets, those of the ctypes structs above, and the binding's packed formats."""
    lines = []
    for name, s in (("mixaq_fp8_matrix", Matrix), ("mixaq_norm", NormS), ("mixaq_residual_norm_params", Params), ("mixaq_residual_norm_grads", Grads)):
        lines += [f'printf("%zu\\n", offsetof({name}, {f[0]}));' for f in s._fields_] + [f'printf("%zu\\n", sizeof({name}));']
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "mixaq.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0; }\n")
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(tmp_path / "layout"), str(src)])
    got = [int(v) for v in subprocess.check_output([str(tmp_path / "layout")]).split()]
    want = []
    for s in (Matrix, NormS, Params, Grads):
        want += [getattr(s, f[0]).offset for f in s._fields_] + [C.sizeof(s)]
    assert got == want
    assert mq._FP8_MATRIX.size == C.sizeof(Matrix) and mq._NORM_PARAMS.size == C.sizeof(Params) and mq._NORM_GRADS.size == C.sizeof(Grads)
    values = list(range(1, 9))
    m = Matrix.from_buffer_copy(mq._FP8_MATRIX.pack(*values))
    assert [getattr(m, f[0]) for f in Matrix._fields_] == values
    flat = mq._NORM_PARAMS.unpack(bytes(Params(1, 2, 0, 1, 2, 6, 7, 8, 9, 10, 11, 12, 13.0, NormS(1, 15, 16, 17.0), NormS(2, 19, 20, 21.0), 22, 23, 24, 25, 1)))
    assert flat == (1, 2, 0, 1, 2, 6, 7, 8, 9, 10, 11, 12, 13.0, 1, 15, 16, 17.0, 2, 19, 20, 21.0, 22, 23, 24, 25, 1)
    assert mq._NORM_GRADS.unpack(bytes(Grads(*range(1, 15)))) == tuple(range(1, 15))


@pytest.fixture(scope="module")
def L(tmp_path_factory):
    if not os.path.exists(NVCC):
        pytest.skip("no nvcc")
    out = str(tmp_path_factory.mktemp("row_ops_host") / "libhost.so")
    flags = [f for f in mq_build.NVCC_FLAGS if f not in ("-O3", "-lineinfo")]
    fake = os.path.join(HERE, "host_path")
    subprocess.check_call([NVCC] + flags + ["-cudart", "none", "-Xlinker", "-Bsymbolic", "-o", out] +
                          [os.path.join(mq_build.CSRC, f) for f in ("mixaq.cu", "merge_static.cu", "row_ops.cu")] +
                          [os.path.join(fake, f) for f in ("fake_launch.cu", "fake_row_ops.cu", "fake_runtime.cpp")] + ["-ldl"])
    lib = C.CDLL(out)
    lib.mixaq_last_error.restype = C.c_char_p
    lib.mixaq_residual_norm_backward_workspace_bytes.restype = C.c_size_t
    ptr, i64 = C.c_void_p, C.c_int64
    lib.mixaq_fp8_quantize.argtypes = [ptr, ptr, C.c_int, i64, i64, i64, C.c_int, C.c_int, ptr, ptr]
    lib.mixaq_fp8_matmul.argtypes = [ptr, ptr, ptr, ptr, ptr, C.c_int, i64, ptr]
    lib.mixaq_residual_norm_forward.argtypes = [ptr, ptr, ptr, ptr]
    lib.mixaq_residual_norm_backward.argtypes = [ptr, ptr, ptr, ptr, C.c_size_t, ptr]
    return lib


@pytest.fixture
def ctx(L):
    h = C.c_void_p()
    assert L.mixaq_create(C.byref(h), 0) == 0
    yield h
    assert L.mixaq_destroy(h) == 0


def launches(L, ctx):
    return L.mixaq_last_launch_count(ctx)


def matrix(rows=10, cols=100, **kw):
    m = Matrix(AT, rows, cols, -(-cols // 16) * 16, 1, AT + (1 << 20), 1, rows)
    for k, v in kw.items():
        setattr(m, k, v)
    return m


BAD_MATRICES = [
    (dict(codes=None), INVALID), (dict(codes=AT + 8), INVALID), (dict(scale=None), INVALID), (dict(scale=AT + 2), INVALID),
    (dict(row_stride=104), INVALID), (dict(row_stride=96), INVALID), (dict(block_rows=64), INVALID), (dict(block_rows=0), INVALID),
    (dict(scale_row_stride=-1), INVALID), (dict(scale_col_stride=-1), INVALID),
    (dict(row_stride=1 << 41), UNSUPPORTED), (dict(scale_row_stride=1 << 41), UNSUPPORTED),
]


@pytest.mark.parametrize("change,status", BAD_MATRICES)
def test_bad_matrices_are_refused_everywhere(L, ctx, change, status):
    m, good = matrix(**change), matrix()
    assert L.mixaq_fp8_quantize(ctx, AT, F32, 10, 100, 100, 0, 0, C.byref(m), None) == status
    assert L.mixaq_fp8_matmul(ctx, C.byref(m), C.byref(good), None, AT, F32, 100, None) == status
    assert L.mixaq_fp8_matmul(ctx, C.byref(good), C.byref(m), None, AT, F32, 100, None) == status
    p = params(h=None)
    assert L.mixaq_residual_norm_forward(ctx, C.byref(p), C.byref(matrix(10, 100, **change)), None) != OK
    assert launches(L, ctx) == 0 and L.mixaq_last_error(ctx)


def test_quantize_refusals(L, ctx):
    def call(x=AT, dtype=F32, rows=10, cols=100, stride=100, transpose=0, out=None):
        return L.mixaq_fp8_quantize(ctx, x, dtype, rows, cols, stride, transpose, 0, C.byref(out or matrix()), None)
    assert call() == OK and launches(L, ctx) == 1
    assert call(x=AT + 4) == OK                                        # elements' alignment is enough
    assert L.mixaq_fp8_quantize(None, AT, F32, 10, 100, 100, 0, 0, C.byref(matrix()), None) == INVALID
    assert L.mixaq_fp8_quantize(ctx, AT, F32, 10, 100, 100, 0, 0, None, None) == INVALID
    for kw in (dict(x=None), dict(x=AT + 2), dict(x=AT + 1, dtype=BF16), dict(dtype=3), dict(rows=-1), dict(cols=-1), dict(stride=99), dict(rows=9),
               dict(cols=99), dict(transpose=1), dict(out=matrix(100, 10))):
        assert call(**kw) == INVALID, kw
    assert call(transpose=1, out=matrix(100, 10)) == OK
    assert call(rows=1 << 31, out=matrix(1 << 31, 100)) == UNSUPPORTED
    assert call(rows=(1 << 31) - 300, cols=256, stride=256, out=matrix((1 << 31) - 300, 256)) == UNSUPPORTED      # blocks beyond 31 bits
    assert call(rows=0, out=matrix(0, 100)) == OK and launches(L, ctx) == 0
    assert call(cols=0, stride=0, out=matrix(10, 0)) == OK and launches(L, ctx) == 0
    # scales of an output that share a place
    for rs, cs in ((0, 1), (1, 0), (1, 9), (1, 1), (1, 5)):
        assert call(cols=300, stride=300, out=matrix(10, 300, scale_row_stride=rs, scale_col_stride=cs)) == INVALID, (rs, cs)
    for rs, cs in ((1, 10), (3, 1), (5, 1), (1, 11), (2, 20)):
        assert call(cols=300, stride=300, out=matrix(10, 300, scale_row_stride=rs, scale_col_stride=cs)) == OK, (rs, cs)


def test_matmul_refusals(L, ctx):
    def call(a=None, w=None, bias=None, y=AT + (8 << 20), dtype=BF16, stride=7):
        return L.mixaq_fp8_matmul(ctx, C.byref(a or matrix()), C.byref(w or matrix(7)), bias, y, dtype, stride, None)
    assert call() == OK and launches(L, ctx) == 1
    last = C.c_long.in_dll(L, "last_matmul")
    assert last is not None
    assert call(a=matrix(scale_row_stride=0, scale_col_stride=0)) == OK        # one scale for all: fine as an input
    for kw in (dict(y=None), dict(y=AT + 1), dict(y=AT + 2, dtype=F32), dict(bias=AT + 2), dict(dtype=7), dict(stride=6), dict(w=matrix(7, 116)),
               dict(a=matrix(10, 0)), dict(a=matrix(-1))):
        assert call(**kw) == INVALID, kw
    assert call(stride=1 << 40) == UNSUPPORTED
    assert call(a=matrix((1 << 31) - 300), w=matrix((1 << 31) - 300), stride=1 << 31) == UNSUPPORTED
    assert call(a=matrix(0)) == OK and launches(L, ctx) == 0
    assert call(w=matrix(0), stride=0) == OK and launches(L, ctx) == 0
    C.c_int.in_dll(L, "fail_matmul").value = 1
    assert call() == INTERNAL
    C.c_int.in_dll(L, "fail_matmul").value = 0


def params(**kw):
    p = Params(10, 100, F32, BF16, BF16, AT, 100, AT + (1 << 20), 100, AT + (2 << 20), 100, 10, 1.0, NormS(LAYER, AT, AT, 1e-5),
               NormS(RMS, AT, None, 1e-5), AT + (3 << 20), 100, AT + (4 << 20), 100, 0)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


COMMON_BAD = [
    (dict(rows=-1), INVALID), (dict(dim=0), INVALID), (dict(dim=16385), UNSUPPORTED), (dict(rows=1 << 31), UNSUPPORTED),
    (dict(x_dtype=5), INVALID), (dict(y_dtype=-1), INVALID), (dict(x_dtype=F16), INVALID), (dict(x_dtype=BF16, y_dtype=F32), INVALID),
    (dict(post=NormS(3, AT, AT, 1e-5)), INVALID), (dict(pre=NormS(RMS, AT + 2, None, 1e-5)), INVALID), (dict(pre=NormS(RMS, AT, None, 0.0)), INVALID),
    (dict(post=NormS(LAYER, AT, AT, -1.0)), INVALID), (dict(post=NormS(LAYER, AT, AT, float("nan"))), INVALID), (dict(post=NormS(LAYER, AT, AT, float("inf"))), INVALID),
    (dict(gate_dtype=F16), INVALID), (dict(rows_per_gate=0), INVALID), (dict(gate_stride=-1), INVALID), (dict(gate=AT + 1), INVALID),
    (dict(y=None), INVALID),                                             # with its gate and post norm still there
]


@pytest.mark.parametrize("change,status", COMMON_BAD)
def test_bad_norm_arguments_are_refused_forward_and_backward(L, ctx, change, status):
    p = params(**change)
    assert L.mixaq_residual_norm_forward(ctx, C.byref(p), None, None) == status
    g = grads()
    assert L.mixaq_residual_norm_backward(ctx, C.byref(p), C.byref(g), AT, 1 << 30, None) == status
    assert launches(L, ctx) == 0


def test_norm_forward_refusals(L, ctx):
    def call(fp8=None, **kw):
        return L.mixaq_residual_norm_forward(ctx, C.byref(params(**kw)), C.byref(fp8) if fp8 is not None else None, None)
    assert call() == OK and launches(L, ctx) == 1
    assert L.mixaq_residual_norm_forward(ctx, None, None, None) == INVALID and L.mixaq_residual_norm_forward(None, None, None, None) == INVALID
    none = NormS(NONE, None, None, 0.0)
    for kw in (dict(h=None), dict(x=None), dict(x_out=None), dict(x=AT + 2), dict(y=AT + 1), dict(x_stride=99), dict(y_stride=99), dict(x_out_stride=99),
               dict(h_stride=99), dict(h=AT + 1), dict(pre=none), dict(x_out=AT, x_out_stride=104), dict(h=AT + (1 << 20), h_stride=104), dict(h=AT),
               dict(h=AT + (3 << 20)), dict(x_out=AT + (1 << 20)),
               dict(y=None, gate=None, post=none), dict(y=None, gate=None, post=none, x_out=None, h=None, pre=none)):
        assert call(**kw) == INVALID, kw
    assert call(fp8=matrix(10, 100)) == INVALID                         # h as well
    for bad in (matrix(9, 100), matrix(10, 101), matrix(10, 100, block_rows=128)):
        assert call(fp8=bad, h=None) == INVALID
    assert call(fp8=matrix(10, 100), h=None) == OK
    assert call(x_out=AT) == OK and call(h=AT + (1 << 20)) == OK          # in place
    assert call(y=None, gate=None, post=none, x_out=None) == OK
    assert call(gate_dtype=F32) == OK and call(gate=None) == OK and call(pre=none, h=None) == OK
    assert call(rows=0) == OK and launches(L, ctx) == 0
    assert call(rows_per_gate=1 << 40) == OK
    # a sequence longer than the batch is a gate per channel
    last = (C.c_long * 16).in_dll(L, "last_norm")
    assert last[0] == 10


def grads(**kw):
    g = Grads(AT + (5 << 20), 100, AT + (6 << 20), 100, AT + (7 << 20), 100, AT + (8 << 20), 100, AT + (9 << 20), 100, AT, AT + 4096, AT + 8192, AT + 12288)
    for k, v in kw.items():
        setattr(g, k, v)
    return g


def test_norm_backward_refusals(L, ctx):
    def call(ws=AT + (20 << 20), ws_bytes=1 << 20, p=None, **kw):
        q = params(**(p or {}))
        return L.mixaq_residual_norm_backward(ctx, C.byref(q), C.byref(grads(**kw)), ws, ws_bytes, None)
    assert call() == OK and launches(L, ctx) == 1
    assert L.mixaq_residual_norm_backward(ctx, C.byref(params()), None, AT, 1 << 20, None) == INVALID
    none = NormS(NONE, None, None, 0.0)
    for kw in (dict(ws=None), dict(ws=AT + 64), dict(dx_out=None, dh=None), dict(dx=AT + 2), dict(dy=AT + 1), dict(dgate=AT + 2), dict(dpre_gamma=AT + 2),
               dict(dx_stride=99), dict(dh_stride=99), dict(dgate_stride=99), dict(dx=AT), dict(dx=AT + (1 << 20)), dict(dx=AT + (5 << 20), dx_stride=104),
               dict(dy=AT + (6 << 20), dy_stride=104), dict(dy=AT + (5 << 20)), dict(dx=AT + (8 << 20)), dict(p=dict(x=None)),
               dict(p=dict(pre=none)), dict(p=dict(post=none)), dict(p=dict(gate=None)), dict(p=dict(y=None, gate=None, post=none))):
        assert call(**kw) == INVALID, kw
    need = L.mixaq_residual_norm_backward_workspace_bytes(C.byref(params()))
    assert call(ws_bytes=need) == OK and call(ws_bytes=need - 1) == SMALL
    per_sequence = params(rows_per_gate=3)
    assert L.mixaq_residual_norm_backward_workspace_bytes(C.byref(per_sequence)) > need
    assert call(dx=AT + (5 << 20)) == OK and call(dy=AT + (6 << 20)) == OK and call(dy=AT + (1 << 20)) == OK      # in place
    assert call(dh=None) == OK and call(dh=None, p=dict(x=None)) == OK and call(dx_out=None) == OK
    assert call(dx=None, dy=None, dgate=None, dpost_gamma=None, dpost_beta=None, dpre_gamma=None, dpre_beta=None) == OK
    assert call(p=dict(rows=0)) == OK and launches(L, ctx) == 0
    assert L.mixaq_residual_norm_backward_workspace_bytes(None) == 0
    assert L.mixaq_residual_norm_backward_workspace_bytes(C.byref(params(dim=0))) == 0
    many = dict(rows=(1 << 31) - 300, dim=16384, rows_per_gate=2, x_stride=16384, y_stride=16384, gate_stride=16384)
    assert call(ws_bytes=1 << 60, p=many, dx_out_stride=16384, dh_stride=16384, dx_stride=16384, dy_stride=16384, dgate_stride=16384) == UNSUPPORTED


# ---- the binding's own checks (they come before any call of the library) ---------------------------------------------------------
CPU = SimpleNamespace(device=torch.device("cpu"), h=None)


def fp8(rows, cols, block_rows=1, device="cpu"):
    return mq.Fp8Matrix.empty(rows, cols, block_rows, device)


@pytest.mark.parametrize("rows,cols,block_rows", [(1, 1, 1), (5, 130, 1), (300, 17, 128), (0, 64, 1)])
def test_room_for_a_matrix(rows, cols, block_rows):
    m = fp8(rows, cols, block_rows)
    assert m.shape == (rows, cols) and m.codes.stride(0) % 16 == 0 and m.scale.shape == (-(-rows // block_rows), -(-cols // 128))
    v = mq._FP8_MATRIX.unpack(m.pack(CPU))
    assert v[1:5] == (rows, cols, -(-cols // 16) * 16, block_rows) and v[6:] == m.scale.stride()
    m.codes.view(torch.uint8).fill_(0x38)                                 # 1.0
    m.scale.fill_(0.5)
    assert torch.equal(m.values(), torch.full((rows, cols), 0.5))


def test_bad_matrices_are_refused_by_the_binding():
    good = fp8(5, 130)
    bad = [mq.Fp8Matrix(good.codes, good.scale, 2), mq.Fp8Matrix(good.codes.view(torch.uint8), good.scale), mq.Fp8Matrix(good.codes, good.scale.double()),
           mq.Fp8Matrix(good.codes, good.scale[:4]), mq.Fp8Matrix(good.codes, good.scale, 128), mq.Fp8Matrix(good.codes.t(), good.scale.t()),
           mq.Fp8Matrix(good.codes[0], good.scale), mq.Fp8Matrix(good.codes.to("meta"), good.scale)]
    for m in bad:
        with pytest.raises(mq.MixaqError) as e:
            m.pack(CPU)
        assert e.value.status == -1


def test_bad_calls_are_refused_by_the_binding():
    x, a, w = torch.zeros(4, 32), fp8(4, 32), fp8(3, 32)
    norm = mq.Norm("rms", torch.ones(32))
    bad = [
        lambda: mq.fp8_quantize(CPU, x[0]), lambda: mq.fp8_quantize(CPU, x.double()), lambda: mq.fp8_quantize(CPU, x.t()),
        lambda: mq.fp8_quantize(CPU, x, block_rows=64), lambda: mq.fp8_quantize(CPU, x, 128, out=a), lambda: mq.fp8_quantize(CPU, torch.zeros(1, 32).expand(4, 32)),
        lambda: mq.fp8_matmul(CPU, a, w, out_dtype=torch.int32), lambda: mq.fp8_matmul(CPU, a, w, y=torch.zeros(4, 4)), lambda: mq.fp8_matmul(CPU, a, w, bias=torch.zeros(4)),
        lambda: mq.fp8_matmul(CPU, a, w, bias=torch.zeros(3).double()), lambda: mq.fp8_matmul(CPU, a, w, y=torch.zeros(4, 3, dtype=torch.float64)),
        lambda: mq.Norm("batch"), lambda: mq.residual_norm_forward(CPU, x, fp8=True), lambda: mq.residual_norm_forward(CPU, x, h=x),
        lambda: mq.residual_norm_forward(CPU, x, x_out=x, pre=norm), lambda: mq.residual_norm_forward(CPU, x, torch.zeros(4, 31), pre=norm),
        lambda: mq.residual_norm_forward(CPU, x, x.bfloat16(), pre=mq.Norm("rms", torch.ones(31))), lambda: mq.residual_norm_forward(CPU, x, x, gate=torch.ones(3, 32)),
        lambda: mq.residual_norm_forward(CPU, x, x, gate=torch.ones(2, 32), rows_per_gate=1), lambda: mq.residual_norm_forward(CPU, x, x, gate=torch.ones(32).half()),
        lambda: mq.residual_norm_forward(CPU, x, x, gate=torch.ones(2, 32), rows_per_gate=0), lambda: mq.residual_norm_forward(CPU, x, x, h_dtype=torch.float16, pre=norm),
        lambda: mq.residual_norm_backward(CPU, None), lambda: mq.residual_norm_backward(CPU, x, dh=x), lambda: mq.residual_norm_backward(CPU, None, dx_out=x, dh=x, pre=norm),
        lambda: mq.residual_norm_backward(CPU, x, dx_out=x, dh=torch.zeros(4, 31), pre=norm),
    ]
    for call in bad:
        with pytest.raises(mq.MixaqError):
            call()
