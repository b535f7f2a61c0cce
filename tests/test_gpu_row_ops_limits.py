"""The row operators on the GPU where the first set of tests does not go: scales of the product at both ends of binary32's range.
Tolerances are counted as in test_gpu_row_ops.py, whose definitions these tests share."""
import pytest
import torch

from paper_2507_19131_b200 import binding as mq
from test_gpu_row_ops import E4M3, TYPES, U, codes_of, ctx, g, matmul_reference, normal, rounding, within  # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu

# parts of a cluster, single CTAs, pairs of CTAs; a k-block that is not full
SHAPES = [(40, 300, 1100), (300, 520, 1000), (1000, 64, 5000), (5000, 4300, 700)]


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
