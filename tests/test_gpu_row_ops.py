"""The row operators on the GPU against their definitions in 64 bits: quantizer and product of e4m3 codes with block scales, norms at a
sublayer's border (forward and backward), and a run of them together.

Tolerances.  u = 2^-24 is half a step of binary32; eps(t) / 2 half a step of an output's type.  A sum of n terms in binary32, in any order,
is off by at most (n - 1) u times the sum of the terms' magnitudes; sums that are added in parts of a thread, a warp and a CTA take at most
the longest chain of additions in the place of n.  Every tolerance below is such a count times u times the magnitudes that go in, plus the
rounding of the output."""
import math

import pytest
import torch

from paper_2507_19131_b200 import binding as mq

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
E4M3 = torch.float8_e4m3fn
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def ctx():
    c = mq.Context(0)
    yield c
    torch.cuda.synchronize()
    assert c.device_status() == 0
    c.close()


@pytest.fixture
def g():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    return gen


def normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def rounding(t, want):
    """The rounding to type t: half a step, eps / 2 of a normal value.  Below the smallest normal number the steps stay what they are there
    (2^-24 in float16), so the magnitude counts as at least that."""
    return torch.finfo(t).eps / 2 * want.abs().clamp(min=torch.finfo(t).tiny)


def within(got, want, tol, what=""):
    """|got - want| <= tol everywhere, with the same infinities and NaN."""
    got = got.double()
    assert got.shape == want.shape, what
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), what
    over = ((got - want).abs() - tol)[fine]
    assert over.numel() == 0 or float(over.max()) <= 0.0, f"{what}: {float(over.max())} over the tolerance"


# ---- quantizer --------------------------------------------------------------------------------------------------------------
def quantize_reference(x, block_rows, pow2):
    """Codes (as binary32 values) and scales, in the quantizer's own operations: binary32 quotients and one product."""
    rows, cols = x.shape
    rb, cb = -(-rows // block_rows), -(-cols // 128)
    p = torch.zeros((rb * block_rows, cb * 128), device=x.device)
    p[:rows, :cols] = x.float()
    p = p.view(rb, block_rows, cb, 128)
    amax = p.abs().amax(dim=(1, 3))
    amax = torch.where(torch.isfinite(amax), amax, torch.nan)
    scale = amax / torch.full_like(amax, 448.0)
    if pow2:
        exact = amax.double() / torch.full_like(amax, 448.0, dtype=torch.float64)
        m, e = torch.frexp(exact)
        scale = torch.where(exact > 0, torch.ldexp(torch.where(m == 0.5, 0.5, 1.0).double() + 0 * exact, e), exact).float()
    scale = scale.clamp(min=2.0 ** -126)
    q = (p * (1.0 / scale)[:, None, :, None]).clamp(-448, 448).to(E4M3).float()
    return q.view(rb * block_rows, cb * 128)[:rows, :cols], scale


def same(a, b):
    """Equal, with NaN in the same places."""
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 4096), (3, 130), (49, 96), (128, 128), (129, 257), (1000, 1001), (257, 16)])
@pytest.mark.parametrize("block_rows,transpose,pow2", [(1, False, False), (1, True, False), (128, False, False), (128, True, True), (1, False, True)])
def test_quantizer_is_its_definition_bit_for_bit(ctx, g, dtype, rows, cols, block_rows, transpose, pow2):
    x = normal(g, rows, cols) * torch.exp2(normal(g, rows, 1) * 4)
    x = x.to(TYPES[dtype])
    q = mq.fp8_quantize(ctx, x, block_rows, transpose, pow2)
    codes, scale = quantize_reference(x.t() if transpose else x, block_rows, pow2)
    assert same(q.scale, scale) and same(q.codes.float(), codes)


@pytest.mark.parametrize("block_rows,transpose", [(1, False), (1, True), (128, False), (128, True)])
@pytest.mark.parametrize("pow2", [False, True])
def test_quantizer_at_the_ends_of_the_range(ctx, g, block_rows, transpose, pow2):
    """Zeros, subnormals, values at a power of two times 448 and beside it, the largest, infinities and NaN: in blocks of their own."""
    x = torch.zeros(256, 1280, device="cuda")
    x[:, 128:256] = 2.0 ** -149
    x[:, 256:384] = normal(g, 256, 128) * 2.0 ** -140
    x[:, 384:512] = torch.where(torch.arange(128, device="cuda") == 5, 448.0, 1.0)
    x[:, 512:640] = torch.where(torch.arange(128, device="cuda") == 9, math.nextafter(448.0, 1e9), 1.0)       # (448 in binary32)
    x[:, 640:768] = torch.nextafter(torch.tensor(448.0), torch.tensor(1e9)).cuda()
    x[:, 768:896] = 3.4e38 * torch.sign(normal(g, 256, 128))
    x[7, 900] = math.inf
    x[200, 1030] = -math.inf
    x[130, 1160] = math.nan
    if transpose:
        x = x.t().contiguous()
    q = mq.fp8_quantize(ctx, x, block_rows, transpose, pow2)
    codes, scale = quantize_reference(x.t() if transpose else x, block_rows, pow2)
    assert same(q.scale, scale) and same(q.codes.float(), codes)
    assert torch.isnan(scale).any() and not torch.isnan(scale).all()
    if pow2:
        s = q.scale[torch.isfinite(q.scale)]
        assert torch.equal(torch.frexp(s).mantissa, torch.full_like(s, 0.5))


@pytest.mark.parametrize("transpose", [False, True])
def test_quantizer_with_strides_and_what_lies_beside(ctx, g, transpose):
    """Rows at odd addresses with a stride, scales in row order, the output's padding and neighbours left as they were."""
    store = normal(g, 70, 333).half()
    x = store[3:67, 5:306]                                         # 64 x 301, rows not aligned
    r, c = (301, 64) if transpose else (64, 301)
    buf = torch.full((r + 2, 320), 0x55, dtype=torch.uint8, device="cuda")
    scale = torch.full((r + 2, 5), 77.0, device="cuda")
    out = mq.Fp8Matrix(buf.view(E4M3)[1:r + 1, :c], scale[1:r + 1, :-(-c // 128)], 1)
    mq.fp8_quantize(ctx, x, 1, transpose, out=out)
    codes, want = quantize_reference(x.t() if transpose else x, 1, False)
    assert torch.equal(out.codes.float(), codes) and torch.equal(out.scale, want)
    assert int((buf[0] != 0x55).sum()) == 0 and int((buf[-1] != 0x55).sum()) == 0 and int((buf[:, c:] != 0x55).sum()) == 0
    assert float((scale[0] - 77).abs().max()) == 0 and float((scale[-1] - 77).abs().max()) == 0 and float((scale[:, -(-c // 128):] - 77).abs().max()) == 0


# ---- product ----------------------------------------------------------------------------------------------------------------
def codes_of(g, rows, cols, block_rows, order="cols"):
    """Normal codes; the padding behind the rows is NaN, which nothing may read."""
    ld = -(-cols // 16) * 16 + 16
    buf = torch.full((rows + 1, ld), 0x7F, dtype=torch.uint8, device="cuda").view(E4M3)
    buf[:rows, :cols] = (normal(g, rows, cols) * 60).clamp(-448, 448).to(E4M3)
    rb, cb = -(-rows // block_rows), -(-cols // 128)
    s = torch.exp2(normal(g, rb, cb)) * 0.01
    return mq.Fp8Matrix(buf[:rows, :cols], s.t().contiguous().t() if order == "cols" else s, block_rows)


def matmul_reference(a, w, bias):
    """y and the tolerance's magnitudes in 64 bits."""
    def values(m):
        rows, cols = m.codes.shape
        s = m.scale.double().repeat_interleave(m.block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :cols]
        return m.codes.double() * s
    va, vw = values(a), values(w)
    y, mag = va @ vw.t(), va.abs() @ vw.abs().t()
    if bias is not None:
        y, mag = y + bias.double(), mag + bias.double().abs()
    return y, mag


def check_matmul(ctx, a, w, bias, dtype, y=None):
    got = mq.fp8_matmul(ctx, a, w, bias, TYPES[dtype], y=y)
    want, mag = matmul_reference(a, w, bias)
    # 128 products of a block (exact) in a row, then one scaled addition a block, two roundings of the scales, up to 8 parts, the bias
    chain = 128 + -(-a.codes.shape[1] // 128) + 2 + 8 + 1
    within(got, want, chain * U * mag + rounding(TYPES[dtype], want), "matmul")
    return got


@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 32, 16), (1, 1000, 4096), (7, 33, 129), (49, 288, 96), (64, 4096, 512), (128, 128, 128), (129, 130, 131),
                                   (200, 256, 4100), (300, 520, 1000), (513, 1030, 260), (2048, 2100, 384), (1000, 64, 10000)])
@pytest.mark.parametrize("w_block_rows", [1, 128])
@pytest.mark.parametrize("dtype", TYPES)
def test_matmul(ctx, g, m, n, k, w_block_rows, dtype):
    check_matmul(ctx, codes_of(g, m, k, 1), codes_of(g, n, k, w_block_rows, "rows"), normal(g, n) if n % 2 == 0 else None, dtype)


@pytest.mark.parametrize("m,n,k", [(300, 700, 300), (5000, 4300, 700)])
@pytest.mark.parametrize("a_rows,a_order,w_rows,w_order", [(1, "rows", 128, "cols"), (128, "rows", 128, "rows"), (128, "cols", 1, "cols"), (1, "cols", 1, "rows")])
def test_matmul_with_every_kind_of_scale(ctx, g, m, n, k, a_rows, a_order, w_rows, w_order):
    check_matmul(ctx, codes_of(g, m, k, a_rows, a_order), codes_of(g, n, k, w_rows, w_order), None, "f32")


def test_matmul_with_one_scale_for_a_whole_matrix(ctx, g):
    a, w = codes_of(g, 100, 300, 1), codes_of(g, 200, 300, 128)
    a.scale = torch.full((1, 1), 0.25, device="cuda").expand(100, 3)
    check_matmul(ctx, a, w, None, "f32")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n", [(70, 45), (300, 515)])
def test_matmul_writes_its_own_rows_only(ctx, g, dtype, m, n):
    buf = torch.full((m + 2, n + 9), 5.0, dtype=TYPES[dtype], device="cuda")
    y = buf[1:m + 1, 3:n + 3]                                      # rows at odd addresses
    check_matmul(ctx, codes_of(g, m, 200, 1), codes_of(g, n, 200, 128), None, dtype, y=y)
    buf[1:m + 1, 3:n + 3] = 5.0
    assert float((buf.float() - 5.0).abs().max()) == 0.0


@pytest.mark.parametrize("m", [3, 700])
def test_a_value_that_is_none_shows_in_its_row_alone(ctx, g, m):
    x = normal(g, m, 700)
    x[2, 650] = math.inf
    a, w = mq.fp8_quantize(ctx, x), codes_of(g, 300, 700, 128)
    y = mq.fp8_matmul(ctx, a, w, out_dtype=torch.float32)
    assert bool(torch.isnan(y[2]).all()) and not bool(torch.isnan(y[torch.arange(m, device="cuda") != 2]).any())


def test_empty_and_repeated_calls(ctx, g):
    w = codes_of(g, 300, 200, 128)
    assert mq.fp8_matmul(ctx, mq.Fp8Matrix.empty(0, 200, 1, "cuda"), w).shape == (0, 300)
    assert ctx.launch_count() == 0
    assert mq.fp8_quantize(ctx, torch.zeros(0, 64, device="cuda")).shape == (0, 64) and ctx.launch_count() == 0
    for m in (40, 300, 4000):                                      # parts of a cluster, one CTA a tile, pairs
        a = codes_of(g, m, 200, 1)
        first = mq.fp8_matmul(ctx, a, w)
        assert ctx.launch_count() == 1
        for _ in range(3):
            assert torch.equal(first, mq.fp8_matmul(ctx, a, w))


# ---- norms ------------------------------------------------------------------------------------------------------------------
class Case:
    def __init__(self, g, rows, dim, xt="f32", yt="f32", post="layer", pre="rms", gate="channel", per=None, scale=0.7, gate_f32=False, pad=0, odd=0, mean=0.3):
        def rows_of(t, n=rows):
            """A matrix whose rows are `pad` elements apart, starting `odd` elements into its storage; what lies beside is NaN."""
            buf = torch.full((n * (dim + pad) + odd + 1,), math.nan, dtype=t, device="cuda")
            return torch.as_strided(buf, (n, dim), (dim + pad, 1), odd)
        self.rows, self.dim, self.scale, self.xt, self.yt = rows, dim, scale, TYPES[xt], TYPES[yt]
        self.x, self.y = rows_of(self.xt), rows_of(self.yt)
        self.x.copy_(normal(g, rows, dim) + mean)
        self.y.copy_(normal(g, rows, dim) * 2 - mean)
        self.per = {"": None, "channel": None, "sequence": per, "token": 1}[gate]
        gates = {"": 0, "channel": 1, "sequence": -(-rows // (per or 1)), "token": rows}[gate]
        self.gate = None
        if gates:
            gt = torch.float32 if gate_f32 else self.yt
            self.gate = rows_of(gt, gates)
            self.gate.copy_(normal(g, gates, dim) * 0.3 + 0.5)
        def norm(kind):
            return mq.Norm(kind, normal(g, dim) * 0.1 + 1, normal(g, dim) * 0.1 if kind == "layer" else None, 1e-5) if kind else None
        self.post, self.pre = norm(post), norm(pre)
        self.rows_of = rows_of
        self.which = torch.arange(rows, device="cuda") // (rows if gate == "channel" else self.per or 1)
        self.args = dict(gate=self.gate, rows_per_gate=self.per, scale=scale, post=self.post, pre=self.pre)

    def gate64(self):
        return torch.ones((), dtype=torch.float64, device="cuda") if self.gate is None else self.gate.double()[self.which]


def norm_reference(v, norm):
    """The normalised rows, the reciprocal deviation, the result, and how far a binary32 computation may be off it.
    Sums over a row are chains of at most 40 additions (32 of a thread, a warp's and a CTA's steps): the mean is off by 40 u mean|v|, a
    deviation d by that and u |d|, the variance by 42 u of itself and twice the mean's error times mean|d| (which is at most the
    standard deviation), so the normalised value by the relative (42 / 2 + 4) u and the mean's error times rstd, twice."""
    if norm is None:
        return v, None, v, torch.zeros_like(v)
    mean = v.mean(1, keepdim=True) if norm.kind == "layer" else torch.zeros_like(v[:, :1])
    d = v - mean
    rstd = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + norm.eps)
    n = d * rstd
    out = n * norm.gamma.double()
    off = (25 * n.abs() + 2 * 40 * v.abs().mean(1, keepdim=True) * rstd * (1 + n.abs()) * (norm.kind == "layer")) * U
    tol = (off + 3 * U * n.abs()) * norm.gamma.double().abs()
    if norm.beta is not None:
        out = out + norm.beta.double()
        tol = tol + U * norm.beta.double().abs()
    return n, rstd, out, tol + U * out.abs()


def check_forward(ctx, c, fp8=False, pow2=False, got=None, x=None, y=None):
    x0, y0 = (c.x if x is None else x).double(), (c.y if y is None else y).double()
    r = got or mq.residual_norm_forward(ctx, c.x, c.y, fp8=fp8, pow2=pow2, **c.args)
    _, _, out, tol = norm_reference(y0, c.post)
    factor = c.gate64() * c.scale
    want = x0 + factor * out
    within(r.x, want, factor.abs() * (tol + 2 * U * out.abs()) + U * want.abs() + rounding(c.xt, want), "x")
    if c.pre is None:
        assert r.h is None
        return r
    _, _, h, htol = norm_reference(r.x.double(), c.pre)             # of the rounded sum that the call returned
    if not fp8:
        within(r.h, h, htol + rounding(c.yt, h), "h")
        return r
    blocks = -(-c.dim // 128)
    pad = torch.zeros((c.rows, blocks * 128), dtype=torch.float64, device="cuda")
    pad[:, :c.dim] = h.abs()
    tpad = torch.zeros_like(pad)
    tpad[:, :c.dim] = htol
    want = (pad.view(c.rows, blocks, 128).amax(2) / 448).clamp(min=2.0 ** -126)
    stol = tpad.view(c.rows, blocks, 128).amax(2) / 448 + 2 * U * want
    s = r.h.scale.double()
    if pow2:
        assert torch.equal(torch.frexp(r.h.scale).mantissa, torch.full_like(r.h.scale, 0.5))
        assert bool((s >= want - stol).all()) and bool((s < 2 * (want + stol)).all())
    else:
        within(r.h.scale, want, stol, "h scale")
    each = s.repeat_interleave(128, 1)[:, :c.dim]
    # half a step of e4m3: 2^-4 of a normal code, 2^-10 of the scale below 2^-6; the product with the rounded reciprocal twice u
    within(r.h.codes.double() * each, h, htol + (2.0 ** -4 + 3 * U) * h.abs() + 2.0 ** -10 * each, "h codes")
    return r


@pytest.mark.parametrize("xt,yt", [("f32", "f32"), ("f32", "bf16"), ("f32", "f16"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("rows,dim", [(1, 1), (1, 4096), (3, 31), (5, 96), (49, 256), (600, 257), (20, 512), (7000, 64), (33, 768), (2000, 1024), (9, 1001), (1300, 2048), (5, 4095), (1500, 4096),
                                      (4, 5000), (700, 8192), (3, 16384), (500, 16383)])
def test_norm_forward_types_and_widths(ctx, g, xt, yt, rows, dim):
    c = Case(g, rows, dim, xt, yt)
    check_forward(ctx, c)
    check_forward(ctx, c, fp8=True, pow2=rows % 2 == 1)


@pytest.mark.parametrize("post", ["", "layer", "rms"])
@pytest.mark.parametrize("pre", ["", "layer", "rms"])
@pytest.mark.parametrize("gate,per,gate_f32", [("", None, False), ("channel", None, True), ("sequence", 7, False), ("sequence", 1000, True), ("token", None, False)])
@pytest.mark.parametrize("dim", [200, 201])
def test_norm_forward_kinds_and_gates(ctx, g, post, pre, gate, per, gate_f32, dim):
    c = Case(g, 1500, dim, "f32", "bf16", post, pre, gate, per, 0.31, gate_f32)
    check_forward(ctx, c)
    if pre:
        check_forward(ctx, c, fp8=True)


@pytest.mark.parametrize("dim", [129, 256, 1000, 4096])
@pytest.mark.parametrize("pad,odd", [(0, 1), (3, 0), (5, 3), (8, 8)])
@pytest.mark.parametrize("rows", [3, 1200])
def test_norm_strides_and_addresses(ctx, g, rows, dim, pad, odd):
    """Rows at any address and distance; what lies before, between and behind them is NaN and stays."""
    c = Case(g, rows, dim, "bf16", "bf16", "layer", "layer", "sequence", 100, pad=pad, odd=odd)
    out, h = c.rows_of(c.xt), c.rows_of(c.yt)
    r = mq.residual_norm_forward(ctx, c.x, c.y, x_out=out, h=h, **c.args)
    check_forward(ctx, c, got=r)
    for t in (out, h):
        beside = torch.ones(t.untyped_storage().nbytes() // t.element_size(), dtype=torch.bool, device="cuda")
        torch.as_strided(beside, t.shape, t.stride(), t.storage_offset()).fill_(False)
        whole = torch.as_strided(t, beside.shape, (1,), 0)
        assert bool(torch.isnan(whole[beside]).all())
    check_backward(ctx, c, g)


@pytest.mark.parametrize("rows,dim", [(1, 4096), (3000, 768), (900, 771)])
def test_norm_in_place(ctx, g, rows, dim):
    c = Case(g, rows, dim, "bf16", "bf16")
    x, y = c.x.clone(), c.y.clone()
    r = mq.residual_norm_forward(ctx, c.x, c.y, x_out=c.x, h=c.y, **c.args)
    assert r.x is c.x and r.h is c.y
    check_forward(ctx, c, got=r, x=x, y=y)


def test_norm_without_a_sublayer(ctx, g):
    """Only the norm in front of the first sublayer: x is handed through; h of another type."""
    for dim, yt in ((96, "bf16"), (4096, "f32"), (333, "f16")):
        c = Case(g, 500, dim, "f32", yt, "", "layer", "")
        r = mq.residual_norm_forward(ctx, c.x, pre=c.pre, h_dtype=c.yt)
        assert r.x is c.x
        _, _, h, tol = norm_reference(c.x.double(), c.pre)
        within(r.h, h, tol + rounding(c.yt, h))
    assert mq.residual_norm_forward(ctx, torch.zeros(0, 64, device="cuda"), pre=mq.Norm("rms")).h.shape == (0, 64)


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_rows_without_spread_and_rows_that_are_no_numbers(ctx, g, kind):
    c = Case(g, 600, 640, "f32", "f32", kind, kind, "")
    c.y[3] = 0
    c.y[4] = 1e-30
    c.x[3] = 0
    c.y[5] = 123.0                                                  # a constant row: deviation 0
    c.y[6] = 1e4 + normal(g, 640)                                   # far from zero
    r = check_forward(ctx, c)
    c.y[7, 100], c.x[9, 5] = math.inf, math.nan
    s = mq.residual_norm_forward(ctx, c.x, c.y, **c.args)
    ill = torch.zeros(600, dtype=torch.bool, device="cuda")
    ill[7] = ill[9] = True
    assert torch.equal(s.x[~ill], r.x[~ill]) and torch.equal(s.h[~ill], r.h[~ill]) and bool(torch.isnan(s.h[ill]).all())


def backward_reference(c, x, dx_out, dh):
    """Gradients in 64 bits from the definition, by torch's automatic differentiation: written apart from the kernel's formulas."""
    def apply(v, norm, gamma, beta):
        if norm is None:
            return v
        d = v - v.mean(1, keepdim=True) if norm.kind == "layer" else v
        n = d / torch.sqrt((d * d).mean(1, keepdim=True) + norm.eps) * gamma
        return n if beta is None else n + beta
    def leaf(t):
        return None if t is None else t.detach().double().requires_grad_()
    x0, y = torch.zeros_like(x, dtype=torch.float64).requires_grad_(), leaf(c.y)
    gate = leaf(c.gate)
    pg, pb, ng, nb = (leaf(getattr(n, a)) if n is not None else None for n in (c.post, c.pre) for a in ("gamma", "beta"))
    step = apply(y, c.post, pg, pb) * c.scale
    if gate is not None:
        step = step * gate[c.which]
    # the gradient is taken at the given x', whatever x and the rounding made of it
    out = x0 + step + (x.double() - step).detach()
    loss = (out * dx_out.double()).sum() if dx_out is not None else 0
    if dh is not None:
        loss = loss + (apply(out, c.pre, ng, nb) * dh.double()).sum()
    loss.backward()
    grad = lambda t: None if t is None or t.grad is None else t.grad
    return dict(dx=x0.grad, dy=y.grad, dgate=grad(gate), dpost_gamma=grad(pg), dpost_beta=grad(pb), dpre_gamma=grad(ng), dpre_beta=grad(nb))


def backward_magnitudes(c, x, dx_out, dh):
    """For every gradient the magnitudes that its sums and products are made of, u counted: tolerances.
    Statistics and the two row sums of a gradient are chains of 40 additions; a normalised value is off by what norm_reference says."""
    def through(norm, v, d):
        if norm is None:
            return d.abs(), v.abs(), None, torch.zeros_like(v)
        n, rstd, _, _ = norm_reference(v, norm)
        noff = (25 * n.abs() + 2 * 40 * v.abs().mean(1, keepdim=True) * rstd * (1 + n.abs()) * (norm.kind == "layer")) * U
        e = d.abs() * norm.gamma.double().abs()
        # e - n mean(e n) - mean(e), times rstd: relative (25 + 40 + 8) u of all magnitudes, and n's error wherever n enters
        total = (e + n.abs() * (e * n.abs()).mean(1, keepdim=True) + e.mean(1, keepdim=True)) * rstd
        extra = (noff * (e * n.abs()).mean(1, keepdim=True) + n.abs() * (e * noff).mean(1, keepdim=True)) * rstd
        rel = 25 * U + 2 * 40 * U * v.abs().mean(1, keepdim=True) * rstd * (norm.kind == "layer")
        return total, n.abs(), noff, (75 * U + rel) * total + extra
    xd, tol = x.double(), {}
    dx, dxtol = torch.zeros_like(xd), torch.zeros_like(xd)
    ref = backward_reference(c, x, dx_out, dh)
    # the longest chain of a column sum: a worker's rows (at most rows, two of which are added at once), the workers of a CTA, the CTAs
    chain = c.rows + 40
    if dh is not None:
        total, n, noff, t = through(c.pre, xd, dh.double())
        dxtol = dxtol + t + U * total
        tol["dpre_gamma"] = (dh.double().abs() * (noff + 2 * U * n)).sum(0) + chain * U * (dh.double().abs() * n).sum(0)
        tol["dpre_beta"] = chain * U * dh.double().abs().sum(0)
    dxa = ref["dx"].abs()
    dxtol = dxtol + 2 * U * dxa
    tol["dx"] = dxtol + rounding(c.xt, dxa)
    factor = (c.gate64() * c.scale).abs() + torch.zeros_like(xd)
    w, wtol = dxa * factor, dxtol * factor + 3 * U * dxa * factor
    _, _, r, rtol = norm_reference(c.y.double(), c.post)
    if c.gate is not None:
        t = (dxtol * r.abs() + dxa * rtol) * abs(c.scale) + (chain + 4) * U * dxa * r.abs() * abs(c.scale)
        tol["dgate"] = torch.zeros_like(c.gate, dtype=torch.float64).index_add_(0, c.which, t)
    if c.post is None:
        tol["dy"] = wtol + rounding(c.yt, ref["dy"])
        return ref, tol
    total, n, noff, t = through(c.post, c.y.double(), w)
    carried, _, _, _ = through(c.post, c.y.double(), wtol)
    tol["dy"] = t + carried + rounding(c.yt, ref["dy"]) + U * total
    tol["dpost_gamma"] = (wtol * n + w * (noff + 2 * U * n)).sum(0) + chain * U * (w * n).sum(0)
    tol["dpost_beta"] = wtol.sum(0) + chain * U * w.sum(0)
    return ref, tol


def check_backward(ctx, c, g, with_dx=True, with_dh=True, x=None):
    x = x if x is not None else c.x
    dx_out = c.rows_of(c.xt) if with_dx else None
    if with_dx:
        dx_out.copy_(normal(g, c.rows, c.dim))
    dh = c.rows_of(c.yt) if with_dh and c.pre is not None else None
    if dh is not None:
        dh.copy_(normal(g, c.rows, c.dim) * 0.5)
    got = mq.residual_norm_backward(ctx, x, c.y, dx_out=dx_out, dh=dh, **c.args)
    ref, tol = backward_magnitudes(c, x, dx_out, dh)
    for name, want in ref.items():
        value = getattr(got, name)
        if want is None:
            assert value is None or float(value.abs().max()) == 0.0, name          # (a norm whose output no one used)
        else:
            within(value, want, tol[name], name)
    again = mq.residual_norm_backward(ctx, x, c.y, dx_out=dx_out, dh=dh, **c.args)
    for name in ref:
        assert getattr(got, name) is None or torch.equal(getattr(got, name), getattr(again, name)), name
    return got, dx_out, dh


@pytest.mark.parametrize("xt,yt", [("f32", "f32"), ("f32", "bf16"), ("f32", "f16"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("rows,dim", [(1, 1), (1, 4096), (3, 31), (49, 256), (700, 257), (20, 512), (3000, 64), (33, 1024), (9, 1001), (500, 2048), (301, 4095), (450, 4096), (4, 5000), (200, 8192), (3, 16384), (160, 16383)])
def test_norm_backward_types_and_widths(ctx, g, xt, yt, rows, dim):
    check_backward(ctx, Case(g, rows, dim, xt, yt, "rms", "layer"), g)


@pytest.mark.parametrize("xt,yt", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("rows,dim", [(1037, 4096), (901, 3001), (1037, 2056), (1037, 8192), (901, 8191), (1037, 6000)])
def test_norm_backward_refills_of_wide_rows(ctx, g, xt, yt, rows, dim):
    """Six or seven rows a worker: every stage of a ring is filled again, and the last one has an odd row over."""
    check_backward(ctx, Case(g, rows, dim, xt, yt, "layer", "layer", "sequence", 5, 0.5), g)


@pytest.mark.parametrize("post", ["", "layer", "rms"])
@pytest.mark.parametrize("pre", ["", "layer", "rms"])
@pytest.mark.parametrize("gate,per,gate_f32", [("", None, False), ("channel", None, True), ("sequence", 7, False), ("sequence", 1000, True), ("token", None, False)])
@pytest.mark.parametrize("dim", [200, 201, 3000])
def test_norm_backward_kinds_and_gates(ctx, g, post, pre, gate, per, gate_f32, dim):
    check_backward(ctx, Case(g, 1501, dim, "f32", "bf16", post, pre, gate, per, 0.31, gate_f32), g)


def test_norm_backward_parts(ctx, g):
    """Only one of the two incoming gradients; no sublayer; in place; no rows."""
    c = Case(g, 300, 320, "bf16", "bf16", "layer", "rms", "channel")
    check_backward(ctx, c, g, with_dx=False)
    check_backward(ctx, c, g, with_dh=False)
    dh, x = normal(g, 300, 320), normal(g, 300, 320)
    norm = mq.Norm("layer", normal(g, 320), normal(g, 320))
    got = mq.residual_norm_backward(ctx, x, dh=dh, pre=norm)
    assert got.dy is None and got.dgate is None and got.dpost_gamma is None
    v, gamma, beta = (t.double().requires_grad_() for t in (x, norm.gamma, norm.beta))
    (torch.nn.functional.layer_norm(v, (320,), gamma, beta, 1e-5) * dh.double()).sum().backward()
    within(got.dx, v.grad, 200 * U * v.grad.abs().amax(1, keepdim=True) + torch.zeros_like(v.grad))
    empty = mq.residual_norm_backward(ctx, x[:0], x[:0], post=norm, pre=norm, dx_out=x[:0], dh=x[:0])
    assert empty.dx.shape == (0, 320) and float(empty.dpre_gamma.abs().max()) == 0.0 and float(empty.dpost_beta.abs().max()) == 0.0


def test_norm_gradients_against_differences(ctx, g):
    """Central differences of the 64-bit definition along a random direction, for every input: d loss = sum of gradient times step."""
    c = Case(g, 37, 130, "f32", "f32", "layer", "rms", "sequence", 10, 0.6)
    fwd = mq.residual_norm_forward(ctx, c.x, c.y, **c.args)
    dx_out, dh = normal(g, 37, 130), normal(g, 37, 130)
    got = mq.residual_norm_backward(ctx, fwd.x, c.y, dx_out=dx_out, dh=dh, **c.args)

    def loss(x, y, gate, pg, pb, ng):
        def norm(v, kind, gamma, beta):
            d = v - v.mean(1, keepdim=True) if kind == "layer" else v
            n = d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5) * gamma
            return n if beta is None else n + beta
        out = x + c.scale * gate[c.which] * norm(y, "layer", pg, pb)
        return float((out * dx_out.double()).sum() + (norm(out, "rms", ng, None) * dh.double()).sum())
    leaves = [t.double() for t in (c.x, c.y, c.gate, c.post.gamma, c.post.beta, c.pre.gamma)]
    grads = [got.dx, got.dy, got.dgate, got.dpost_gamma, got.dpost_beta, got.dpre_gamma]
    for i, (leaf, grad) in enumerate(zip(leaves, grads)):
        step = normal(g, *leaf.shape).double()
        h = 1e-5
        hi, lo = list(leaves), list(leaves)
        hi[i], lo[i] = leaf + h * step, leaf - h * step
        want = (loss(*hi) - loss(*lo)) / (2 * h)
        have = float((grad.double() * step).sum())
        # third derivatives times h^2 / 6 (1e-10 of order one each), cancellation 1e-16 / h of the loss's terms, and binary32's 200 u
        scale = float((grad.double().abs() * step.abs()).sum())
        assert abs(have - want) <= 1e-6 * scale + 1e-6, (i, have, want)


def test_sequences_that_workers_share(ctx, g):
    """Lengths around the rows of a worker, so that sequences end in, at and beyond its last row."""
    for rows, per in ((148 * 4 + 1, 3), (148 * 8, 8), (5000, 33), (5000, 4999), (5000, 2), (1000, 999)):
        check_backward(ctx, Case(g, rows, 136, "f32", "f32", "rms", "rms", "sequence", per), g)


# ---- streams, graphs, the run of them together ----------------------------------------------------------------------------------
def sublayer(ctx, s, x, y):
    """One border and the next sublayer's product: norms, gate and residual, codes, product, the next border."""
    r = mq.residual_norm_forward(ctx, x, y, gate=s["gate"], scale=0.8, post=s["post"], pre=s["pre"], fp8=True)
    z = mq.fp8_matmul(ctx, r.h, s["w"], s["bias"])
    return r, z, mq.residual_norm_forward(ctx, r.x, z, gate=s["gate"], scale=0.8, post=s["post"], pre=s["pre"])


@pytest.mark.parametrize("rows", [1, 50, 3000])
def test_a_run_of_them_together(ctx, g, rows):
    dim = 768
    s = dict(gate=(normal(g, dim) * 0.1 + 0.5).bfloat16(), post=mq.Norm("rms", normal(g, dim) * 0.1 + 1), pre=mq.Norm("layer", normal(g, dim) * 0.1 + 1, normal(g, dim) * 0.1),
             w=mq.fp8_quantize(ctx, normal(g, dim, dim) * 0.02, block_rows=128), bias=normal(g, dim) * 0.1)
    x, y = normal(g, rows, dim), normal(g, rows, dim).bfloat16()
    r, z, last = sublayer(ctx, s, x, y)
    c = Case(g, rows, dim, "f32", "bf16", "", "", "")
    c.x, c.y, c.scale, c.gate, c.post, c.pre, c.which = x, y, 0.8, s["gate"][None], s["post"], s["pre"], torch.zeros(rows, dtype=torch.long, device="cuda")
    check_forward(ctx, c, fp8=True, got=r)
    want, mag = matmul_reference(r.h, s["w"], s["bias"])
    within(z, want, 150 * U * mag + rounding(torch.bfloat16, want))
    c.x, c.y = r.x, z
    check_forward(ctx, c, got=last)

    # the same on another stream, and captured and replayed on new data; two graphs at once, each with buffers of its own
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _, z2, last2 = sublayer(ctx, s, x, y)
    side.synchronize()
    assert torch.equal(z, z2) and torch.equal(last.x, last2.x) and torch.equal(last.h, last2.h)
    graphs = []
    for _ in range(2):
        xs, ys = x.clone(), y.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = sublayer(ctx, s, xs, ys)[2]
        graphs.append((graph, xs, ys, out))
    new_x, new_y = normal(g, rows, dim), normal(g, rows, dim).bfloat16()
    want = sublayer(ctx, s, new_x, new_y)[2]
    graphs[1][1].copy_(new_x)
    graphs[1][2].copy_(new_y)
    for graph, *_ in graphs:
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(graphs[0][3].h, last.h) and torch.equal(graphs[1][3].h, want.h) and torch.equal(graphs[1][3].x, want.x)


def test_gradients_captured_in_a_graph(ctx, g):
    """The gradients of a linear layer with codes on both sides: dx by the transposed weights, dw by the transposed rows."""
    rows, k, n = 700, 384, 200
    x, w, dy = normal(g, rows, k), normal(g, n, k) * 0.05, normal(g, rows, n)

    def gradients():
        dx = mq.fp8_matmul(ctx, mq.fp8_quantize(ctx, dy), mq.fp8_quantize(ctx, w, 128, transpose=True), out_dtype=torch.float32)
        qx, qdy = mq.fp8_quantize(ctx, x, transpose=True), mq.fp8_quantize(ctx, dy, transpose=True)
        return dx, mq.fp8_matmul(ctx, qdy, qx, out_dtype=torch.float32)
    dx, dw = gradients()
    # a code is off by 2^-4 of itself or 2^-10 of the scale, on either side
    def spread(t, block_rows):
        q = mq.fp8_quantize(ctx, t, block_rows)
        return 2.0 ** -4 * t.double().abs() + 2.0 ** -10 * q.scale.double().repeat_interleave(block_rows, 0)[:t.shape[0]].repeat_interleave(128, 1)[:, :t.shape[1]]
    a, b, ea, eb = dy.double(), w.double().t().contiguous(), spread(dy, 1), spread(w.t().contiguous(), 128)
    tol = ea @ b.t().abs().t().t() + a.abs() @ eb.t() + ea @ eb.t()
    within(dx, a @ b.t(), tol + 1e-4 * (a.abs() @ b.t().abs()))
    a, b, ea, eb = dy.double().t().contiguous(), x.double().t().contiguous(), spread(dy.t().contiguous(), 1), spread(x.t().contiguous(), 1)
    tol = ea @ b.abs().t() + a.abs() @ eb.t() + ea @ eb.t()
    within(dw, a @ b.t(), tol + 1e-4 * (a.abs() @ b.abs().t()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gx, gw = gradients()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(gx, dx) and torch.equal(gw, dw)


def test_norm_backward_captured(ctx, g):
    c = Case(g, 900, 512, "bf16", "bf16", "rms", "layer", "sequence", 100)
    dx_out, dh = normal(g, 900, 512).bfloat16(), normal(g, 900, 512).bfloat16()
    want = mq.residual_norm_backward(ctx, c.x, c.y, dx_out=dx_out, dh=dh, **c.args)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = mq.residual_norm_backward(ctx, c.x, c.y, dx_out=dx_out, dh=dh, **c.args)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for name, value in vars(want).items():
        assert value is None or torch.equal(value, getattr(got, name)), name


def test_profiling_names_the_row_operators(ctx, g):
    ctx.profile_begin()
    a = mq.fp8_quantize(ctx, normal(g, 64, 256))
    mq.fp8_matmul(ctx, a, a)
    mq.residual_norm_forward(ctx, normal(g, 64, 256), pre=mq.Norm("rms"))
    times = ctx.profile_end()
    for name in ("fp8_quantize", "fp8_matmul", "residual_norm"):
        assert times[name][1] == 1 and times[name][0] > 0.0


def test_offsets_beyond_32_bits(ctx, g):
    """Rows that lie more than 2^31 elements behind the first."""
    stride = (1 << 31) // 3 + 16 - ((1 << 31) // 3) % 16
    free, _ = torch.cuda.mem_get_info()
    if free < 24 << 30:
        pytest.skip("less than 24 GiB free")
    buf = torch.empty(3 * stride + 4096, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (4, 4096), (stride, 1))
    x.copy_(normal(g, 4, 4096))
    q = mq.fp8_quantize(ctx, x)
    codes, scale = quantize_reference(x, 1, False)
    assert torch.equal(q.codes.float(), codes) and torch.equal(q.scale, scale)
    pre = mq.Norm("rms", torch.ones(4096, device="cuda"))
    h = mq.residual_norm_forward(ctx, x, pre=pre).h
    _, _, want, tol = norm_reference(x.double(), pre)
    within(h, want, tol + rounding(torch.bfloat16, want))
    del buf, x
    far = torch.empty(3 * stride + 4096, dtype=torch.uint8, device="cuda")
    a = mq.Fp8Matrix(torch.as_strided(far.view(E4M3), (4, 4096), (stride, 1)), q.scale)
    a.codes.copy_(q.codes)
    y = torch.as_strided(torch.empty(3 * stride + 4, dtype=torch.bfloat16, device="cuda"), (4, 4), (stride, 1))
    mq.fp8_matmul(ctx, a, q, y=y)
    assert torch.equal(y, mq.fp8_matmul(ctx, q, q))
