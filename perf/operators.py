"""Performance cases of the row operators: block-scaled 8-bit floating-point quantizer and matrix product, and the norms at a
sublayer's border fused with its gate and residual scale (forward and backward).

With `own` false `run` computes the operators in plain torch operations, in binary32, rounded once at the end; with `own` true it
makes the calls that a user makes of `paper_2507_19131_b200.binding`.  `exact` restates them in binary64."""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
E4M3 = torch.float8_e4m3fn
BLOCK = 128                     # columns that share a scale
E4M3_MAX = 448.0
MIN_SCALE = 2.0 ** -126
EPS = 1e-5


def _quantize(name, rows, cols, dtype, block_rows=1, transpose=False, pow2=False):
    return dict(name=name, kind="quantize", rows=rows, cols=cols, dtype=dtype, block_rows=block_rows, transpose=transpose, pow2=pow2)


def _matmul(name, m, n, k, out, w_block_rows=128, bias=False):
    return dict(name=name, kind="matmul", m=m, n=n, k=k, out=out, w_block_rows=w_block_rows, bias=bias)


def _norm(name, rows, dim, x_dtype, y_dtype, post, pre, gate, rows_per_gate=1, fp8=False, backward=False, scale=1.0):
    return dict(name=name, kind="norm_backward" if backward else "norm", rows=rows, dim=dim, x_dtype=x_dtype, y_dtype=y_dtype, post=post,
                pre=pre, gate=gate, rows_per_gate=rows_per_gate, fp8=fp8, scale=scale)


def listed():
    return [
        # one window's tokens through a first-stage QKV projection: the smallest product, K below one block
        _matmul("matmul_49x288x96", 49, 288, 96, "f16", bias=True),
        # one token through a square projection: a pass over the weights
        _matmul("matmul_1x4096x4096", 1, 4096, 4096, "bf16"),
        # a few dozen tokens, ragged in every direction, weights with a scale per row, binary32 out
        _matmul("matmul_37x2000x4090_rowscale", 37, 2000, 4090, "f32", w_block_rows=1, bias=True),
        # a prompt through the second FFN matrix
        _matmul("matmul_2048x4096x16384", 2048, 4096, 16384, "bf16"),
        # a large batch of tokens through a square projection
        _matmul("matmul_8192x8192x8192", 8192, 8192, 8192, "bf16"),
        # weight gradient of a 384 -> 1536 layer: both operands carry a scale per row and 128 tokens, binary32 out
        _matmul("matmul_1536x384x66800_gradient", 1536, 384, 66800, "f32", w_block_rows=1),
        # the rows of a 200 x 334 token map before a product
        _quantize("quantize_66800x384", 66800, 384, "bf16"),
        # the same tokens' gradient, quantized along the tokens for the weight gradient
        _quantize("quantize_66801x1000_transposed", 66801, 1000, "bf16", transpose=True, pow2=True),
        # one token between two sublayers of a decoder: two norms, codes for the next product
        _norm("norm_1x4096_fp8", 1, 4096, "bf16", "bf16", "rms", "rms", "channel", fp8=True),
        # a binary32 residual stream of 16-bit sublayers, gate per sequence
        _norm("norm_32768x4096_fp8", 32768, 4096, "f32", "bf16", "layer", "rms", "sequence", rows_per_gate=2048, fp8=True, scale=0.5),
        # gradients at the border of two sublayers, gate per channel (learned residual scale)
        _norm("norm_backward_16384x4096", 16384, 4096, "bf16", "bf16", "rms", "layer", "channel", backward=True),
        # the same on short ragged sequences of an odd width with a gate per sequence
        _norm("norm_backward_9850x1001_sequence", 9850, 1001, "f32", "f16", "layer", "layer", "sequence", rows_per_gate=197, backward=True, scale=0.7),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: sizes uniform in their logarithm, odd ones as often as not."""
    kind = rng.choice(["matmul", "matmul", "matmul", "quantize", "quantize", "norm", "norm", "norm_backward", "norm_backward"])
    if kind == "matmul":
        m, n, k = _log_int(rng, 1, 16384), _log_int(rng, 16, 8192), _log_int(rng, 16, 16384)
        if rng.random() < 0.5:
            n, k = max(16, n // 64 * 64), max(16, k // 64 * 64)
        m = max(1, min(m, 8192 ** 3 // (n * k)))
        return _matmul("", m, n, k, rng.choice(["f32", "bf16", "bf16", "f16"]), rng.choice([128, 128, 1]), rng.random() < 0.5)
    if kind == "quantize":
        rows, cols = _log_int(rng, 1, 66801), _log_int(rng, 16, 16384)
        if rng.random() < 0.5:
            cols = max(16, cols // 64 * 64)
        rows = max(1, min(rows, 66801 * 1000 // cols))
        return _quantize("", rows, cols, rng.choice(["f32", "bf16", "f16"]), rng.choice([1, 1, 128]), rng.random() < 0.4, rng.random() < 0.5)
    backward = kind == "norm_backward"
    rows, dim = _log_int(rng, 1, 32768), _log_int(rng, 32, 8192)
    if rng.random() < 0.5:
        dim = dim // 32 * 32
    rows = max(1, min(rows, (16384 if backward else 32768) * 4096 // dim))
    x_dtype, y_dtype = rng.choice([("f32", "f32"), ("f32", "bf16"), ("f32", "f16"), ("bf16", "bf16"), ("f16", "f16")])
    gate = rng.choice(["", "channel", "sequence", "token"])
    post = rng.choice(["", "rms", "layer"])
    pre = rng.choice(["rms", "layer"] if rng.random() < 0.8 or gate == "" and post == "" else [""])
    return _norm("", rows, dim, x_dtype, y_dtype, post, pre, gate, _log_int(rng, 1, rows) if gate == "sequence" else 1,
                 fp8=pre != "" and not backward and rng.random() < 0.5, backward=backward, scale=rng.choice([1.0, 0.5, 0.31]))


# ---- what a user's program has in hand before the call ----------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _ceil(a, b):
    return -(-a // b)


def _codes(g, rows, cols, block_rows):
    """A quantized matrix: codes in rows of a multiple of 16 bytes, scales; the values are normal with a few larger rows."""
    ld = _ceil(cols, 16) * 16
    values = _normal(g, rows, ld) * 96.0
    codes = values.clamp_(-E4M3_MAX, E4M3_MAX).to(E4M3)[:, :cols]
    spread = torch.exp2(_normal(g, _ceil(cols, BLOCK), _ceil(rows, block_rows)) * 0.5) * (0.01 / 96.0)
    return codes, spread.t() if block_rows == 1 else spread.t().contiguous()


def _gate_rows(case):
    return {"": 0, "channel": 1, "sequence": _ceil(case["rows"], case["rows_per_gate"]), "token": case["rows"]}[case["gate"]]


def prepare(case, seed):
    g = _generator(seed)
    st = dict(case=case)
    if case["kind"] == "quantize":
        # activations: a channel in 64 is much larger than the others
        x = _normal(g, case["rows"], case["cols"])
        st["x"] = (x * torch.where(torch.rand(case["cols"], generator=g, device="cuda") < 1 / 64, 20.0, 1.0)).to(DTYPES[case["dtype"]])
    elif case["kind"] == "matmul":
        st["a"] = _codes(g, case["m"], case["k"], 1)
        st["w"] = _codes(g, case["n"], case["k"], case["w_block_rows"])
        st["bias"] = _normal(g, case["n"]) if case["bias"] else None
    else:
        rows, dim = case["rows"], case["dim"]
        xt, yt = DTYPES[case["x_dtype"]], DTYPES[case["y_dtype"]]
        st["x"] = (_normal(g, rows, dim) * (1.0 + 3.0 * torch.rand(rows, 1, generator=g, device="cuda")) + 0.1).to(xt)
        st["y"] = (_normal(g, rows, dim) * 2.0).to(yt)
        n = _gate_rows(case)
        st["gate"] = (0.5 + 0.2 * _normal(g, n, dim)).to(yt) if n else None
        for at in ("post", "pre"):
            st[at] = (1.0 + 0.1 * _normal(g, dim), 0.1 * _normal(g, dim) if case[at] == "layer" else None) if case[at] else None
        if case["kind"] == "norm_backward":
            st["dx_out"] = (_normal(g, rows, dim) * 0.01).to(xt)
            st["dh"] = (_normal(g, rows, dim) * 0.01).to(yt) if case["pre"] else None
    return st


# ---- the plain forms ----------------------------------------------------------------------------------------------------
def _plain_quantize(x, block_rows, pow2):
    rows, cols = x.shape
    rb, cb = _ceil(rows, block_rows), _ceil(cols, BLOCK)
    padded = torch.zeros((rb * block_rows, cb * BLOCK), device=x.device)
    padded[:rows, :cols] = x
    blocks = padded.view(rb, block_rows, cb, BLOCK)
    amax = blocks.abs().amax(dim=(1, 3))
    amax = torch.where(torch.isfinite(amax), amax, torch.nan)
    scale = amax / torch.full_like(amax, E4M3_MAX)          # (a quotient; division by a number multiplies with its reciprocal)
    if pow2:
        mantissa, exponent = torch.frexp(scale)
        scale = torch.where(scale > 0, torch.ldexp(torch.where(mantissa == 0.5, 0.5, 1.0) + 0.0 * amax, exponent), scale)
    scale = scale.clamp(min=MIN_SCALE)
    q = (blocks * (1.0 / scale)[:, None, :, None]).clamp(-E4M3_MAX, E4M3_MAX).to(E4M3)
    return q.view(rb * block_rows, cb * BLOCK)[:rows, :cols], scale


def _values(matrix, block_rows, dtype=torch.float32):
    codes, scale = matrix
    rows, cols = codes.shape
    scale = scale.to(dtype)
    if block_rows != 1:
        scale = scale.repeat_interleave(block_rows, dim=0)[:rows]
    return codes.to(dtype) * scale.repeat_interleave(BLOCK, dim=1)[:, :cols]


def _plain_matmul(st):
    y = _values(st["a"], 1) @ _values(st["w"], st["case"]["w_block_rows"]).t()
    if st["bias"] is not None:
        y = y + st["bias"]
    return y.to(DTYPES[st["case"]["out"]])


def _plain_norm(v, kind, parameters):
    """norm(v), and the two things its gradient needs: the normalised rows and the reciprocal deviation."""
    if not kind:
        return v, v, None
    if kind == "layer":
        v = v - v.mean(dim=-1, keepdim=True)
    rstd = torch.rsqrt((v * v).mean(dim=-1, keepdim=True) + EPS)
    n = v * rstd
    out = n * parameters[0]
    return out + parameters[1] if parameters[1] is not None else out, n, rstd


def _gate_of_rows(st):
    case, gate = st["case"], st["gate"]
    if gate is None:
        return None
    gate = gate.float()
    return gate.repeat_interleave(case["rows_per_gate"], dim=0)[:case["rows"]] if case["gate"] == "sequence" else gate


def _plain_norm_forward(st):
    case = st["case"]
    r = _plain_norm(st["y"].float(), case["post"], st["post"])[0]
    gate = _gate_of_rows(st)
    x = (st["x"].float() + case["scale"] * (r if gate is None else gate * r)).to(DTYPES[case["x_dtype"]])
    if not case["pre"]:
        return dict(x=x)
    h = _plain_norm(x.float(), case["pre"], st["pre"])[0]
    if not case["fp8"]:
        return dict(x=x, h=h.to(DTYPES[case["y_dtype"]]))
    codes, scale = _plain_quantize(h, 1, False)
    return dict(x=x, codes=codes, h_scale=scale)


def _plain_norm_gradient(dout, n, rstd, kind, gamma):
    d = dout * gamma
    g = d - n * (d * n).mean(dim=-1, keepdim=True)
    if kind == "layer":
        g = g - d.mean(dim=-1, keepdim=True)
    return g * rstd


def _plain_norm_backward(st):
    case = st["case"]
    rows, dim = case["rows"], case["dim"]
    out = {}
    dx = st["dx_out"].float()
    if case["pre"]:
        dh = st["dh"].float()
        _, n, rstd = _plain_norm(st["x"].float(), case["pre"], st["pre"])
        dx = dx + _plain_norm_gradient(dh, n, rstd, case["pre"], st["pre"][0])
        out["dpre_gamma"] = (dh * n).sum(dim=0)
        if case["pre"] == "layer":
            out["dpre_beta"] = dh.sum(dim=0)
    out["dx"] = dx.to(DTYPES[case["x_dtype"]])
    r, n, rstd = _plain_norm(st["y"].float(), case["post"], st["post"])
    u, gate = case["scale"] * dx, _gate_of_rows(st)
    if gate is not None:
        t = u * r
        if case["gate"] == "channel":
            t = t.sum(dim=0, keepdim=True)
        elif case["gate"] == "sequence":
            groups, per = _gate_rows(case), case["rows_per_gate"]
            full = torch.zeros((groups * per, dim), device=t.device)
            full[:rows] = t
            t = full.view(groups, per, dim).sum(dim=1)
        out["dgate"] = t
        u = u * gate
    if case["post"]:
        out["dpost_gamma"] = (u * n).sum(dim=0)
        if case["post"] == "layer":
            out["dpost_beta"] = u.sum(dim=0)
        u = _plain_norm_gradient(u, n, rstd, case["post"], st["post"][0])
    out["dy"] = u.to(DTYPES[case["y_dtype"]])
    return out


# ---- the framework's calls ----------------------------------------------------------------------------------------------
_ctx = None


def _own_norms(mq, st):
    case = st["case"]
    return [mq.Norm(case[at], *st[at], eps=EPS) if case[at] else None for at in ("post", "pre")]


def _own_run(st):
    global _ctx
    from paper_2507_19131_b200 import binding as mq
    if _ctx is None:
        _ctx = mq.Context(0)
    case = st["case"]
    if case["kind"] == "quantize":
        q = mq.fp8_quantize(_ctx, st["x"], block_rows=case["block_rows"], transpose=case["transpose"], pow2=case["pow2"])
        return dict(codes=q.codes, scale=q.scale)
    if case["kind"] == "matmul":
        a, w = mq.Fp8Matrix(*st["a"], block_rows=1), mq.Fp8Matrix(*st["w"], block_rows=case["w_block_rows"])
        return dict(y=mq.fp8_matmul(_ctx, a, w, bias=st["bias"], out_dtype=DTYPES[case["out"]]))
    post, pre = _own_norms(mq, st)
    per = case["rows_per_gate"] if case["gate"] == "sequence" else None
    if case["kind"] == "norm":
        r = mq.residual_norm_forward(_ctx, st["x"], st["y"], gate=st["gate"], rows_per_gate=per, scale=case["scale"], post=post, pre=pre, fp8=case["fp8"])
        if case["fp8"]:
            return dict(x=r.x, codes=r.h.codes, h_scale=r.h.scale)
        return dict(x=r.x, h=r.h) if pre is not None else dict(x=r.x)
    r = mq.residual_norm_backward(_ctx, st["x"], st["y"], gate=st["gate"], rows_per_gate=per, scale=case["scale"], post=post, pre=pre,
                                  dx_out=st["dx_out"], dh=st["dh"])
    return {k: v for k, v in vars(r).items() if v is not None}


def run(state):
    if own:
        return _own_run(state)
    case = state["case"]
    if case["kind"] == "quantize":
        codes, scale = _plain_quantize(state["x"].t() if case["transpose"] else state["x"], case["block_rows"], case["pow2"])
        return dict(codes=codes, scale=scale)
    if case["kind"] == "matmul":
        return dict(y=_plain_matmul(state))
    return _plain_norm_forward(state) if case["kind"] == "norm" else _plain_norm_backward(state)


# ---- what a pass cannot do without --------------------------------------------------------------------------------------
_SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def work(case):
    if case["kind"] == "quantize":
        rows, cols = (case["cols"], case["rows"]) if case["transpose"] else (case["rows"], case["cols"])
        n = rows * cols
        return {"bytes": n * (_SIZE[case["dtype"]] + 1) + 4 * _ceil(rows, case["block_rows"]) * _ceil(cols, BLOCK), "flops": 3 * n}
    if case["kind"] == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        scales = _ceil(k, BLOCK) * (m + _ceil(n, case["w_block_rows"]))
        return {"bytes": m * k + n * k + 4 * scales + m * n * _SIZE[case["out"]] + 4 * n * case["bias"], "flops": 2 * m * n * k}
    n, xs, ys = case["rows"] * case["dim"], _SIZE[case["x_dtype"]], _SIZE[case["y_dtype"]]
    vectors = sum({"": 0, "rms": 1, "layer": 2}[case[at]] for at in ("post", "pre"))
    gate = _gate_rows(case) * case["dim"]
    if case["kind"] == "norm":
        h = 0 if not case["pre"] else n + 4 * case["rows"] * _ceil(case["dim"], BLOCK) if case["fp8"] else n * ys
        return {"bytes": n * (2 * xs + ys) + h + gate * ys + 4 * case["dim"] * vectors, "flops": 16 * n}
    dh = n * ys if case["pre"] else 0
    return {"bytes": n * (3 * xs + 2 * ys) + dh + gate * (ys + 4) + 8 * case["dim"] * vectors, "flops": 32 * n}


# ---- the operators in binary64, from their definitions ------------------------------------------------------------------
def _exact_e4m3(v):
    """Nearest value of four significant bits (three below 2^-6), ties to the even one, at most 448."""
    _, e = torch.frexp(v)
    step = torch.ldexp(torch.ones_like(v), (e - 4).clamp(min=-9))
    return (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def _exact_quantize(x, block_rows, pow2):
    rows, cols = x.shape
    codes = torch.empty((rows, cols), dtype=torch.float64, device=x.device)
    scales = []
    for c in range(0, cols, BLOCK):
        part = x[:, c:c + BLOCK].double()
        amax = part.abs().amax(dim=1)
        if block_rows > 1:
            amax = torch.stack([a.amax() for a in amax.split(block_rows)])
        scale = amax / torch.full_like(amax, E4M3_MAX)
        scale = scale.clamp(min=MIN_SCALE)
        if pow2:
            power = torch.ldexp(torch.ones_like(scale), torch.floor(torch.log2(scale)).int() - 1)
            for _ in range(2):                     # up to the first power of two that is not below
                power = torch.where(power < scale, 2.0 * power, power)
            scale = power
        scales.append(scale)
        codes[:, c:c + BLOCK] = _exact_e4m3(part / scale.repeat_interleave(block_rows)[:rows, None])
    return codes, torch.stack(scales, dim=1)


def _exact_norm(v, kind, parameters):
    if kind == "":
        return v, v, None
    gamma = parameters[0].double()
    if kind == "layer":
        mean = v.sum(dim=1) / v.shape[1]
        v = v - mean[:, None]
    deviation = torch.sqrt(v.square().sum(dim=1) / v.shape[1] + EPS)[:, None]
    n = v / deviation
    return (n * gamma if parameters[1] is None else n * gamma + parameters[1].double()), n, deviation


def _exact_jacobian(d, n, deviation, kind):
    """d times the Jacobian of the normalisation."""
    along = torch.einsum("rc,rc->r", d, n) / d.shape[1]
    d = d - along[:, None] * n
    if kind == "layer":
        d = d - (d.sum(dim=1) / d.shape[1])[:, None]
    return d / deviation


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "quantize":
        codes, scale = _exact_quantize(st["x"].t() if case["transpose"] else st["x"], case["block_rows"], case["pow2"])
        return dict(codes=codes, scale=scale)
    if case["kind"] == "matmul":
        (a, sa), (w, sw) = st["a"], st["w"]
        y = torch.zeros((case["m"], case["n"]), dtype=torch.float64, device="cuda")
        if st["bias"] is not None:
            y += st["bias"].double()
        sw = sw.repeat_interleave(case["w_block_rows"], dim=0)[:case["n"]].double()
        span = 8 * BLOCK                       # blocks at a time
        for k in range(0, case["k"], span):
            b = slice(k // BLOCK, _ceil(min(k + span, case["k"]), BLOCK))
            left, right = a[:, k:k + span].double(), w[:, k:k + span].double()
            left = left * sa[:, b].double().repeat_interleave(BLOCK, dim=1)[:, :left.shape[1]]
            right = right * sw[:, b].repeat_interleave(BLOCK, dim=1)[:, :right.shape[1]]
            y.addmm_(left, right.t())
        return dict(y=y)
    rows = case["rows"]
    gate = st["gate"].double() if st["gate"] is not None else None
    which = torch.arange(rows, device="cuda") // {"sequence": case["rows_per_gate"], "token": 1}.get(case["gate"], rows)
    r, n, deviation = _exact_norm(st["y"].double(), case["post"], st["post"])
    if case["kind"] == "norm":
        x = st["x"].double() + (r if gate is None else r * gate[which]) * case["scale"]
        x = x.to(DTYPES[case["x_dtype"]]).double()           # the residual stream is rounded before it is normed
        if not case["pre"]:
            return dict(x=x)
        h = _exact_norm(x, case["pre"], st["pre"])[0]
        if not case["fp8"]:
            return dict(x=x, h=h)
        codes, scale = _exact_quantize(h, 1, False)
        return dict(x=x, codes=codes, h_scale=scale)
    out = {}
    dx = st["dx_out"].double()
    if case["pre"]:
        _, xn, xdev = _exact_norm(st["x"].double(), case["pre"], st["pre"])
        dh = st["dh"].double()
        out["dpre_gamma"] = torch.einsum("rc,rc->c", dh, xn)
        if case["pre"] == "layer":
            out["dpre_beta"] = dh.sum(dim=0)
        dx = dx + _exact_jacobian(dh * st["pre"][0].double(), xn, xdev, case["pre"])
    out["dx"] = dx
    dr = dx * case["scale"]
    if gate is not None:
        out["dgate"] = torch.zeros_like(gate).index_add_(0, which, dr * r)
        dr = dr * gate[which]
    if case["post"]:
        out["dpost_gamma"] = torch.einsum("rc,rc->c", dr, n)
        if case["post"] == "layer":
            out["dpost_beta"] = dr.sum(dim=0)
        dr = _exact_jacobian(dr * st["post"][0].double(), n, deviation, case["post"])
    out["dy"] = dr
    return out
