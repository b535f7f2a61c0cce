"""What the row operators' entry points hand to their launchers (csrc/row_ops.cu over the stand-in for the CUDA runtime): every argument, and
the number of rows of a gate, by which the kernels divide in 32 bits."""
import ctypes as C

import pytest

from test_row_ops_host import AT, BF16, F16, F32, LAYER, NONE, OK, L, NormS, ctx, grads, matrix, params  # noqa: F401 (fixtures)


def struct(name, text):
    kinds = {"p": C.c_void_p, "l": C.c_long, "i": C.c_int, "f": C.c_float, "b": C.c_bool}
    return type(name, (C.Structure,), {"_fields_": [(f[2:], kinds[f[0]]) for f in text.split()]})


# as in csrc/kernels.h
Quant = struct("Quant", "p:x i:dtype l:rows l:cols l:row_stride b:transpose b:pow2 i:block_rows p:codes l:code_stride p:scale l:srs l:scs")
Operand = struct("Operand", "p:codes l:rows l:stride i:block_rows p:scale l:srs l:scs")
Spec = struct("Spec", "i:kind p:gamma p:beta f:eps")
Grad = struct("Grad", "p:dx_out l:dx_out_stride p:dh l:dh_stride p:dx l:dx_stride p:dy l:dy_stride p:dgate l:dgate_stride "
              "p:dpost_gamma p:dpost_beta p:dpre_gamma p:dpre_beta p:workspace")


class Matmul(C.Structure):
    _fields_ = [("a", Operand), ("w", Operand), ("K", C.c_long), ("bias", C.c_void_p), ("y", C.c_void_p), ("y_dtype", C.c_int), ("y_stride", C.c_long),
                ("status", C.c_void_p)]


class Norm(C.Structure):
    _fields_ = [("rows", C.c_long), ("dim", C.c_int), ("x_dtype", C.c_int), ("y_dtype", C.c_int), ("x", C.c_void_p), ("x_stride", C.c_long),
                ("y", C.c_void_p), ("y_stride", C.c_long), ("gate", C.c_void_p), ("gate_stride", C.c_long), ("rows_per_gate", C.c_long),
                ("gate_f32", C.c_bool), ("scale", C.c_float), ("post", Spec), ("pre", Spec), ("x_out", C.c_void_p), ("x_out_stride", C.c_long),
                ("h", C.c_void_p), ("h_stride", C.c_long), ("codes", C.c_void_p), ("code_stride", C.c_long), ("h_scale", C.c_void_p),
                ("srs", C.c_long), ("scs", C.c_long), ("pow2", C.c_bool)]


def values(s):
    return tuple(values(getattr(s, f[0])) if isinstance(getattr(s, f[0]), C.Structure) else getattr(s, f[0]) for f in s._fields_)


def test_quantize_hands_its_arguments_on(L, ctx):
    m = matrix(200, 100, row_stride=256, block_rows=128, scale_row_stride=3, scale_col_stride=9)
    assert L.mixaq_fp8_quantize(ctx, AT + 512, F16, 100, 200, 333, 1, 1, C.byref(m), None) == OK
    assert values(Quant.in_dll(L, "last_quantize")) == (AT + 512, F16, 100, 200, 333, True, True, 128, m.codes, 256, m.scale, 3, 9)
    assert L.mixaq_fp8_quantize(ctx, AT, F32, 10, 100, 100, 0, 0, C.byref(matrix()), None) == OK
    assert values(Quant.in_dll(L, "last_quantize")) == (AT, F32, 10, 100, 100, False, False, 1, AT, 112, AT + (1 << 20), 1, 10)


def test_matmul_hands_its_arguments_on(L, ctx):
    a = matrix(10, 300, row_stride=512, scale_row_stride=0, scale_col_stride=7)
    w = matrix(70, 300, block_rows=128, codes=AT + (2 << 20), scale=AT + (3 << 20), scale_row_stride=5, scale_col_stride=1)
    assert L.mixaq_fp8_matmul(ctx, C.byref(a), C.byref(w), AT + 64, AT + (8 << 20), BF16, 71, None) == OK
    got = Matmul.in_dll(L, "last_matmul")
    assert values(got)[:-1] == ((AT, 10, 512, 1, AT + (1 << 20), 0, 7), (AT + (2 << 20), 70, 304, 128, AT + (3 << 20), 5, 1), 300, AT + 64,
                                AT + (8 << 20), BF16, 71)
    assert got.status                                       # the context's status word
    assert L.mixaq_fp8_matmul(ctx, C.byref(a), C.byref(w), None, AT + (8 << 20), F32, 1 << 33, None) == OK
    got = Matmul.in_dll(L, "last_matmul")
    assert got.bias is None and got.y_dtype == F32 and got.y_stride == 1 << 33


def test_norms_hand_their_arguments_on(L, ctx):
    p = params(rows=10, x_stride=101, y_stride=102, gate_stride=103, rows_per_gate=4, scale=0.25, x_out_stride=104, h_stride=105, gate_dtype=F32)
    common = (10, 100, F32, BF16, p.x, 101, p.y, 102, p.gate, 103, 4, True, 0.25, values(p.post), values(p.pre))
    assert L.mixaq_residual_norm_forward(ctx, C.byref(p), None, None) == OK
    assert values(Norm.in_dll(L, "last_norm")) == common + (p.x_out, 104, p.h, 105, None, 0, None, 0, 0, False)
    p.h, p.pow2, p.gate_dtype = None, 1, BF16
    m = matrix(10, 100, scale_row_stride=2, scale_col_stride=40)
    assert L.mixaq_residual_norm_forward(ctx, C.byref(p), C.byref(m), None) == OK
    got = Norm.in_dll(L, "last_norm")
    assert not got.gate_f32 and values(got)[-8:] == (None, 105, m.codes, 112, m.scale, 2, 40, True)
    g = grads(dx_out_stride=110, dh_stride=111, dx_stride=112, dy_stride=113, dgate_stride=114)
    p.gate_dtype = F32
    assert L.mixaq_residual_norm_backward(ctx, C.byref(p), C.byref(g), AT + (20 << 20), 1 << 20, None) == OK
    assert values(Norm.in_dll(L, "last_norm"))[:len(common)] == common
    assert values(Grad.in_dll(L, "last_grads")) == values(g) + (AT + (20 << 20),)


@pytest.mark.parametrize("per,want", [(1, 1), (9, 9), (10, 10), (11, 10), ((1 << 32) - 1, 10), (1 << 32, 10), (1 << 40, 10), ((1 << 63) - 1, 10)])
def test_a_sequence_longer_than_the_batch_is_the_batch(L, ctx, per, want):
    """The kernels divide a row's number by rows_per_gate in 32 bits: it never reaches them above the number of rows."""
    p = params(rows=10, rows_per_gate=per)
    assert L.mixaq_residual_norm_forward(ctx, C.byref(p), None, None) == OK
    assert Norm.in_dll(L, "last_norm").rows_per_gate == want
    assert L.mixaq_residual_norm_backward(ctx, C.byref(p), C.byref(grads()), AT + (20 << 20), 1 << 20, None) == OK
    assert Norm.in_dll(L, "last_norm").rows_per_gate == want


def test_without_a_gate_the_batch_is_one_sequence(L, ctx):
    p = params(rows=10, gate=None, rows_per_gate=0, post=NormS(NONE, None, None, 0.0), pre=NormS(LAYER, AT, None, 1e-5))
    assert L.mixaq_residual_norm_forward(ctx, C.byref(p), None, None) == OK
    assert Norm.in_dll(L, "last_norm").rows_per_gate == 10
