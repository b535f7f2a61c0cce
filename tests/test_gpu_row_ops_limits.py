"""The row operators on the GPU where the first set of tests does not go: scales of the product at both ends of binary32's range, and
gradients written over what they are made from.  Tolerances are counted as in test_gpu_row_ops.py, whose definitions these tests share."""
import pytest
import torch

from paper_2507_19131_b200 import binding as mq
from test_gpu_row_ops import E4M3, TYPES, U, Case, codes_of, ctx, g, matmul_reference, normal, rounding, within  # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu

# every width of tile, parts of a cluster, single CTAs, pairs of CTAs; a k-block that is not full
SHAPES = [(40, 300, 1100), (300, 520, 1000), (1000, 64, 5000), (9, 4096, 2100), (5000, 4300, 700)]


def check_far(ctx, a, w, dtype="f32"):
    want, mag = matmul_reference(a, w, None)
    blocks = -(-a.codes.shape[1] // 128)
    chain = 128 + blocks + 2 + 8
    # a block's scaled addition below the smallest normal number is off by half of 2^-149
    within(mq.fp8_matmul(ctx, a, w, out_dtype=TYPES[dtype]), want, chain * U * mag + blocks * 2.0 ** -150 + rounding(TYPES[dtype], want), "matmul")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("w_rows", [1, 128])
@pytest.mark.parametrize("a_exp,w_exp,size", [
    (-64, -64, 60.0),                   # the scales' product is subnormal, the results are not
    (-60, -80, 60.0),                   # it is zero
    (70, -119, 2.0 ** -7),              # a block's sum times the column's scale is subnormal
    (-110, 119, 60.0),                  # that product passes the largest number
    (119, -110, 60.0),
])
def test_scales_far_from_one(ctx, g, dtype, m, n, k, w_rows, a_exp, w_exp, size):
    a, w = codes_of(g, m, k, 1), codes_of(g, n, k, w_rows, "rows")
    if size != 60.0:
        for q in (a, w):
            q.codes.copy_((normal(g, *q.codes.shape) * size).to(E4M3))
    a.scale, w.scale = a.scale * 2.0 ** a_exp, w.scale * 2.0 ** w_exp
    check_far(ctx, a, w, dtype)


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("w_rows", [1, 128])
def test_scales_of_all_sizes_in_one_product(ctx, g, m, n, k, w_rows):
    a, w = codes_of(g, m, k, 1), codes_of(g, n, k, w_rows, "rows")
    for q in (a, w):
        q.scale = q.scale * torch.exp2(torch.randint(-75, 51, q.scale.shape, generator=g, device="cuda").float())
    check_far(ctx, a, w)


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("w_rows", [1, 128])
def test_sums_of_zero_under_scales_whose_product_is_infinite(ctx, g, m, n, k, w_rows):
    """Zero where all codes are zeros, infinity elsewhere (all products are positive, so nothing cancels)."""
    a, w = codes_of(g, m, k, 1), codes_of(g, n, k, w_rows, "rows")
    for q in (a, w):
        q.codes.copy_(((normal(g, *q.codes.shape).abs() * 60).clamp(1, 448)).to(E4M3))
        q.codes[::3] = torch.zeros((), device="cuda").to(E4M3)
    a.scale, w.scale = torch.full_like(a.scale, 1e25), torch.full_like(w.scale, 1e15)
    y = mq.fp8_matmul(ctx, a, w, out_dtype=torch.float32)
    want = torch.full((m, n), torch.inf, device="cuda")
    want[::3] = 0
    want[:, ::3] = 0
    assert torch.equal(y, want)


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("w_rows", [1, 128])
def test_far_scales_change_their_own_outputs_only(ctx, g, m, n, k, w_rows):
    a, w = codes_of(g, m, k, 1), codes_of(g, n, k, w_rows, "rows")
    y = mq.fp8_matmul(ctx, a, w, out_dtype=torch.float32)
    a.scale, w.scale = a.scale.clone(), w.scale.clone()
    a.scale[5] = 2.0 ** -120
    w.scale[0] = 2.0 ** -120
    z = mq.fp8_matmul(ctx, a, w, out_dtype=torch.float32)
    rows = torch.arange(m, device="cuda") != 5
    assert torch.equal(y[rows][:, w_rows:], z[rows][:, w_rows:])
    check_far(ctx, a, w)


# ---- gradients over what they are made from ------------------------------------------------------------------------------------
def backward_into(ctx, c, x, y, dx_out, dh, dx, dy):
    """mixaq_residual_norm_backward through the C interface, dx and dy at given places; returns the parameters' gradients."""
    rows, dim = c.rows, c.dim
    def place(t):
        return t.data_ptr(), t.stride(0)
    gate = mq._gate_fields(ctx, c.gate, c.per, rows, dim, c.yt)
    dgate = torch.full((gate[4], dim), torch.nan, device="cuda")
    sums = torch.full((4, dim), torch.nan, device="cuda")
    p = mq._NORM_PARAMS.pack(rows, dim, mq._DTYPES[c.xt], mq._DTYPES[c.yt], gate[1], *place(x), *place(y), gate[0], gate[2], gate[3], c.scale,
                             *mq._norm_fields(ctx, c.post, dim, "post"), *mq._norm_fields(ctx, c.pre, dim, "pre"), 0, 0, 0, 0, 0)
    at = mq._NORM_GRADS.pack(*place(dx_out), *place(dh), *place(dx), *place(dy), dgate.data_ptr(), dim, *(s.data_ptr() for s in sums))
    work = torch.empty(mq.lib().mixaq_residual_norm_backward_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    ctx.check(mq.lib().mixaq_residual_norm_backward(ctx.h, p, at, work.data_ptr(), work.numel(), mq._stream()), "residual_norm_backward")
    return dgate, sums


@pytest.mark.parametrize("xt,yt", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("rows,dim,pad,odd", [(1, 96, 0, 0), (3000, 96, 0, 0), (1037, 257, 3, 1), (1037, 1001, 0, 1), (1037, 2048, 8, 8), (1037, 4096, 0, 0), (901, 3001, 1, 3),
                                              (301, 8192, 0, 0), (301, 8191, 5, 1), (200, 16384, 0, 0), (160, 16383, 0, 0)])
def test_gradients_in_place(ctx, g, xt, yt, rows, dim, pad, odd):
    """dx over dx_out, dy over dh or over y: the same bits as apart, and nothing beside the rows written."""
    c = Case(g, rows, dim, xt, yt, "rms", "layer", "sequence", 5, 0.5, pad=pad, odd=odd)
    dx_out, dh = c.rows_of(c.xt), c.rows_of(c.yt)
    dx_out.copy_(normal(g, rows, dim))
    dh.copy_(normal(g, rows, dim) * 0.5)

    def copy(t):
        u = c.rows_of(t.dtype)
        u.copy_(t)
        return u
    dx, dy = c.rows_of(c.xt), c.rows_of(c.yt)
    want = backward_into(ctx, c, c.x, c.y, dx_out, dh, dx, dy)
    assert not any(bool(torch.isnan(t).any()) for t in (dx, dy, want[0], want[1][[0, 2, 3]]))
    for over in ("dh", "y"):
        x1, y1, dxo1, dh1 = copy(c.x), copy(c.y), copy(dx_out), copy(dh)
        dy1 = dh1 if over == "dh" else y1
        got = backward_into(ctx, c, x1, y1, dxo1, dh1, dxo1, dy1)
        assert torch.equal(dxo1, dx) and torch.equal(dy1, dy) and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert torch.equal(x1, c.x) and torch.equal(dh1 if over == "y" else y1, dh if over == "y" else c.y)
        for t in (dxo1, dy1):
            beside = torch.ones(t.untyped_storage().nbytes() // t.element_size(), dtype=torch.bool, device="cuda")
            torch.as_strided(beside, t.shape, t.stride(), t.storage_offset()).fill_(False)
            assert bool(torch.isnan(torch.as_strided(t, beside.shape, (1,), 0)[beside]).all())


@pytest.mark.parametrize("per", [601, (1 << 32) - 1, 1 << 32, 1 << 40])
def test_a_sequence_longer_than_the_batch(ctx, g, per):
    c = Case(g, 600, 264, "f32", "bf16", "rms", "layer", "channel")
    dx_out, dh = normal(g, 600, 264), normal(g, 600, 264).bfloat16()
    want = mq.residual_norm_forward(ctx, c.x, c.y, **c.args)
    grads = mq.residual_norm_backward(ctx, want.x, c.y, dx_out=dx_out, dh=dh, **c.args)
    c.args["rows_per_gate"] = per
    got = mq.residual_norm_forward(ctx, c.x, c.y, **c.args)
    assert torch.equal(got.x, want.x) and torch.equal(got.h, want.h)
    for name, value in vars(mq.residual_norm_backward(ctx, want.x, c.y, dx_out=dx_out, dh=dh, **c.args)).items():
        assert value is None or torch.equal(value, getattr(grads, name)), name
