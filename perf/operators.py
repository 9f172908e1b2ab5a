"""Cases for the 8-bit operators around a linear layer: the root-mean-square norm that adds the residual and
writes 8 bits, its gradient, the quantiser, and the matrix product of 8-bit operands.

Weights are stored rows x cols = in x out, as in the shape sets of `workloads.py`: y = x @ W.  A quantised
matrix is a pair of an 8-bit matrix and one fp32 scale for each row (token) or column (channel); its rows
start 16 bytes apart or a multiple of that.

    norm        h = x + r in the stream's type; t = h * w; q = round(t * limit / max|t|) for each row,
                scale = max|t| / limit / sqrt(mean(h^2) + eps), so that q * scale is the norm's output
    norm_grad   its gradient, the rounding taken as the identity: g = grad_y * w, s = 1 / sqrt(mean(h^2) + eps),
                grad_x = s g - h s^3 mean(g h) + grad_h,  grad_w = sum over rows of grad_y h s
    quantize    the same rounding with a scale for each row of x * fold_cols and / or for each column of
                x * fold_rows
    product     out = (a @ b) * scale_a[:, None] * scale_b
    layer       norm, then the product with a weight: the forward pass of a layer
    layer_grad  its backward pass in 8 bits: the incoming gradient, times the scales that run along the
                sums, quantised by row and by column; then grad_x8 = g8 @ W8^T, grad_W = x8^T @ g8 and
                the norm's gradient
"""

import math

import torch

own = False

EPS = 1e-6
LIMIT = {"int8": 127.0, "e4m3": 448.0}
DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}
EIGHT = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def listed():
    return [
        # one token of a served model: launch and latency are all that counts
        {"name": "norm_one_token", "kind": "norm", "rows": 1, "cols": 2048, "io": "bf16", "weight": "bf16",
         "format": "e4m3", "residual": True},
        # fp32 stream whose rows are neither a multiple of a vector nor aligned to one; no residual yet (first block)
        {"name": "norm_ragged_fp32", "kind": "norm", "rows": 777, "cols": 1111, "io": "fp32", "weight": "fp32",
         "format": "e4m3", "residual": False},
        # a training batch of the widest stream that the benchmark times: memory bandwidth
        {"name": "norm_batch", "kind": "norm", "rows": 8192, "cols": 4096, "io": "bf16", "weight": "bf16",
         "format": "e4m3", "residual": True},
        # its backward pass, with the gradient that comes down the residual stream
        {"name": "norm_grad_batch", "kind": "norm_grad", "rows": 8192, "cols": 4096, "io": "bf16", "weight": "bf16",
         "grad_h": True},
        # few rows of an odd size, fp32 norm weight, nothing coming down the stream: the sum over rows is short
        {"name": "norm_grad_ragged", "kind": "norm_grad", "rows": 130, "cols": 1000, "io": "bf16", "weight": "fp32",
         "grad_h": False},
        # an MLP weight after the optimiser's step: one scale for each output channel (stored column)
        {"name": "quantize_weight", "kind": "quantize", "rows": 4096, "cols": 16384, "io": "bf16", "format": "e4m3",
         "by_rows": False, "by_cols": True, "fold": False},
        # a layer's incoming gradient for both of its backward products: by row and by column, scales folded in
        {"name": "quantize_grad", "kind": "quantize", "rows": 1500, "cols": 2048, "io": "bf16", "format": "e4m3",
         "by_rows": True, "by_cols": True, "fold": True},
        # one token through an MLP weight: the weight's bytes are the work
        {"name": "product_one_token", "kind": "product", "m": 1, "k": 4096, "n": 16384, "format": "int8", "out": "bf16",
         "a_t": False, "b_t": False},
        # odd sizes in every direction, 8-bit floats, fp32 result, weight stored out x in
        {"name": "product_ragged", "kind": "product", "m": 203, "k": 1000, "n": 515, "format": "e4m3", "out": "fp32",
         "a_t": False, "b_t": True},
        # a training batch through an MLP weight: matrix rate
        {"name": "product_batch", "kind": "product", "m": 8192, "k": 4096, "n": 16384, "format": "int8", "out": "bf16",
         "a_t": False, "b_t": False},
        # a prompt or small batch through norm and qkv
        {"name": "layer_prompt", "kind": "layer", "rows": 2048, "cols": 2048, "n": 6144, "format": "int8",
         "residual": True},
        # the backward pass of norm and MLP up-projection of a training step
        {"name": "layer_grad_batch", "kind": "layer_grad", "rows": 4096, "cols": 2048, "n": 8192, "format": "int8"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size of the range, spread over its logarithm: odd ones, multiples of 8 and of 128."""
    step = rng.choice((1, 8, 128))
    v = _log(rng, lo, hi)
    return v if step == 1 or v < step else max(lo, v // step * step)


def draw(rng):
    kind = rng.choice(("norm", "norm_grad", "quantize", "product", "layer", "layer_grad"))
    io, weight = rng.choice((("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32")))
    fmt = rng.choice(("int8", "e4m3"))
    if kind == "norm":
        return {"kind": kind, "rows": _log(rng, 1, 8192), "cols": _size(rng, 64, 8192), "io": io, "weight": weight,
                "format": "e4m3", "residual": rng.random() < 0.75}
    if kind == "norm_grad":
        return {"kind": kind, "rows": _log(rng, 1, 8192), "cols": _size(rng, 64, 8192), "io": io, "weight": weight,
                "grad_h": rng.random() < 0.75}
    if kind == "quantize":
        rows, cols = rng.choice(((True, False), (False, True), (True, True)))
        return {"kind": kind, "rows": _log(rng, 1, 8192), "cols": _size(rng, 64, 8192), "io": io, "format": "e4m3",
                "by_rows": rows, "by_cols": cols, "fold": rng.random() < 0.5}
    if kind == "product":
        return {"kind": kind, "m": _log(rng, 1, 8192), "k": _size(rng, 64, 8192), "n": _size(rng, 64, 8192),
                "format": fmt, "out": rng.choice(("bf16", "fp32")), "a_t": rng.random() < 0.3, "b_t": rng.random() < 0.5}
    if kind == "layer":
        return {"kind": kind, "rows": _log(rng, 1, 8192), "cols": _size(rng, 64, 4096), "n": _size(rng, 64, 8192),
                "format": fmt, "residual": rng.random() < 0.75}
    return {"kind": kind, "rows": _log(rng, 16, 8192), "cols": _size(rng, 64, 4096), "n": _size(rng, 64, 8192),
            "format": fmt}


# ------------------------------------------------------------------ inputs

class _Source:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g, device="cuda")

    def stream(self, rows, cols, dtype):
        """A residual stream: a few channels are ten times the others."""
        channel = 1 + 9 * (torch.rand(cols, generator=self.g, device="cuda") < 0.01)
        return (self.normal(rows, cols) * channel).to(dtype)

    def grad(self, rows, cols, dtype):
        """A gradient: small, and of another size for each token."""
        return (self.normal(rows, cols) * (1e-3 * torch.exp(self.normal(rows, 1)))).to(dtype)

    def norm_weight(self, cols, dtype):
        return (1 + 0.1 * self.normal(cols)).to(dtype)

    def eight(self, rows, cols, fmt, axis, std):
        """A Gaussian matrix in 8 bits with a scale for each row (axis 1) or column (axis 0), its rows padded to 16 bytes."""
        v = self.normal(rows, cols) * std
        top = v.abs().amax(axis, keepdim=True)
        v = v * (LIMIT[fmt] / top)
        q = torch.zeros(rows, -(-cols // 16) * 16, dtype=EIGHT[fmt], device="cuda")
        q[:, :cols] = (v.round() if fmt == "int8" else v).to(EIGHT[fmt])
        return q[:, :cols], (top / LIMIT[fmt]).reshape(-1)


def prepare(case, seed):
    s, c = _Source(seed), case
    kind = c["kind"]
    st = {"case": c}
    if kind in ("norm", "norm_grad"):
        io, rows, cols = DTYPE[c["io"]], c["rows"], c["cols"]
        st["w"] = s.norm_weight(cols, DTYPE[c["weight"]])
        if kind == "norm":
            st["x"] = s.stream(rows, cols, io)
            st["r"] = s.stream(rows, cols, io) if c["residual"] else None
        else:
            st["h"], st["grad_y"] = s.stream(rows, cols, io), s.grad(rows, cols, io)
            st["grad_h"] = s.grad(rows, cols, io) if c["grad_h"] else None
    elif kind == "quantize":
        st["x"] = s.grad(c["rows"], c["cols"], DTYPE[c["io"]])
        st["fold_rows"] = torch.exp(s.normal(c["rows"])) * 1e-2 if c["fold"] and c["by_cols"] else None
        st["fold_cols"] = torch.exp(s.normal(c["cols"])) * 1e-2 if c["fold"] and c["by_rows"] else None
    elif kind == "product":
        m, k, n, fmt = c["m"], c["k"], c["n"], c["format"]
        # a_t / b_t: the operand is stored the other way round and handed over as its transpose
        a, st["sa"] = s.eight(k, m, fmt, 0, 1.0) if c["a_t"] else s.eight(m, k, fmt, 1, 1.0)
        b, st["sb"] = s.eight(n, k, fmt, 1, 0.02) if c["b_t"] else s.eight(k, n, fmt, 0, 0.02)
        st["a"], st["b"] = a.t() if c["a_t"] else a, b.t() if c["b_t"] else b
    else:
        rows, cols, n, fmt = c["rows"], c["cols"], c["n"], c["format"]
        st["w"] = s.norm_weight(cols, torch.bfloat16)
        st["W"], st["sW"] = s.eight(cols, n, fmt, 0, 0.02)
        if kind == "layer":
            st["x"] = s.stream(rows, cols, torch.bfloat16)
            st["r"] = s.stream(rows, cols, torch.bfloat16) if c["residual"] else None
        else:
            st["h"] = s.stream(rows, cols, torch.bfloat16)
            st["grad_h"], st["grad_out"] = s.grad(rows, cols, torch.bfloat16), s.grad(rows, n, torch.bfloat16)
            # what the forward pass kept: its 8-bit input and the scale of each token
            st["x8"], st["sx"] = s.eight(rows, cols, fmt, 1, 1.0)
    return st


# ------------------------------------------------------------- plain forms

def _round8(t, top, fmt):
    """t in 8 bits where `top` (the largest magnitude that shares a scale) becomes the format's limit."""
    v = t * torch.where(top > 0, LIMIT[fmt] / top, torch.zeros_like(top))
    return (v.round() if fmt == "int8" else v).to(EIGHT[fmt]), (top / LIMIT[fmt]).reshape(-1)


def _plain_norm(x, r, w, fmt):
    h = None if r is None else (x.float() + r.float()).to(x.dtype)   # the stream is kept in its own type
    v = (x if r is None else h).float()
    t = v * w.float()
    q, scale = _round8(t, t.abs().amax(1, keepdim=True), fmt)
    return q, scale * torch.rsqrt(v.square().mean(1) + EPS), h


def _plain_norm_grad(grad_y, h, w, grad_h):
    v, gy = h.float(), grad_y.float()
    s = torch.rsqrt(v.square().mean(1, keepdim=True) + EPS)
    g = gy * w.float()
    grad_x = s * g - v * (s * s * s * (g * v).mean(1, keepdim=True))
    if grad_h is not None:
        grad_x = grad_x + grad_h.float()
    return grad_x.to(h.dtype), (gy * v * s).sum(0).to(w.dtype)


def _plain_quantize(x, by_rows, by_cols, fold_rows, fold_cols, fmt):
    out = []
    if by_rows:
        t = x.float() if fold_cols is None else x.float() * fold_cols
        out += _round8(t, t.abs().amax(1, keepdim=True), fmt)
    if by_cols:
        t = x.float() if fold_rows is None else x.float() * fold_rows[:, None]
        out += _round8(t, t.abs().amax(0, keepdim=True), fmt)
    return out


def _plain_product(a, sa, b, sb, dtype):
    out = a.float() @ b.float()
    if sa is not None:
        out = out * sa[:, None]
    if sb is not None:
        out = out * sb
    return out.to(dtype)


def _run_plain(st, c):
    kind = c["kind"]
    if kind == "norm":
        return _plain_norm(st["x"], st["r"], st["w"], c["format"])
    if kind == "norm_grad":
        return _plain_norm_grad(st["grad_y"], st["h"], st["w"], st["grad_h"])
    if kind == "quantize":
        return _plain_quantize(st["x"], c["by_rows"], c["by_cols"], st["fold_rows"], st["fold_cols"], c["format"])
    if kind == "product":
        return _plain_product(st["a"], st["sa"], st["b"], st["sb"], DTYPE[c["out"]])
    if kind == "layer":
        q, scale, h = _plain_norm(st["x"], st["r"], st["w"], c["format"])
        return _plain_product(q, scale, st["W"], st["sW"], torch.bfloat16), h
    gr, sr, gc, sc = _plain_quantize(st["grad_out"], True, True, st["sx"], st["sW"], c["format"])
    grad_y = _plain_product(gr, sr, st["W"].t(), None, torch.bfloat16)
    grad_W = _plain_product(st["x8"].t(), None, gc, sc, torch.bfloat16)
    return (grad_W,) + _plain_norm_grad(grad_y, st["h"], st["w"], st["grad_h"])


# ------------------------------------------------- the framework's operators

def _run_own(st, c):
    from paper_2608_20818_b200 import binding as B

    kind = c["kind"]
    if kind == "norm":
        return B.prm_rmsnorm_q8(st["x"], st["w"], EPS, residual=st["r"], format=c["format"])
    if kind == "norm_grad":
        return B.prm_rmsnorm_q8_backward(st["grad_y"], st["h"], st["w"], EPS, grad_h=st["grad_h"])
    if kind == "quantize":
        got = B.prm_quantize_q8(st["x"], by_rows=c["by_rows"], by_cols=c["by_cols"], fold_rows=st["fold_rows"],
                                fold_cols=st["fold_cols"], format=c["format"])
        return [v for v in got if v is not None]
    if kind == "product":
        return B.prm_matmul_q8(st["a"], st["sa"], st["b"], st["sb"], out_dtype=DTYPE[c["out"]])
    if kind == "layer":
        q, scale, h = B.prm_rmsnorm_q8(st["x"], st["w"], EPS, residual=st["r"], format=c["format"])
        return B.prm_matmul_q8(q, scale, st["W"], st["sW"]), h
    gr, sr, gc, sc = B.prm_quantize_q8(st["grad_out"], by_rows=True, by_cols=True, fold_rows=st["sx"],
                                       fold_cols=st["sW"], format=c["format"])
    grad_y = B.prm_matmul_q8(gr, sr, st["W"].t(), None)
    grad_W = B.prm_matmul_q8(st["x8"].t(), None, gc, sc)
    return (grad_W,) + tuple(B.prm_rmsnorm_q8_backward(grad_y, st["h"], st["w"], EPS, grad_h=st["grad_h"]))


def run(state):
    return _run_own(state, state["case"]) if own else _run_plain(state, state["case"])


# -------------------------------------------------------------------- work

def work(case):
    c, kind = case, case["kind"]
    es = lambda name: 2 if name == "bf16" else 4  # noqa: E731
    if kind == "norm":
        e = c["rows"] * c["cols"]
        per = (3 * es(c["io"]) if c["residual"] else es(c["io"])) + 1
        return {"bytes": e * per + c["cols"] * es(c["weight"]) + 4 * c["rows"], "flops": 6 * e}
    if kind == "norm_grad":
        e = c["rows"] * c["cols"]
        return {"bytes": e * es(c["io"]) * (4 if c["grad_h"] else 3) + 2 * c["cols"] * es(c["weight"]), "flops": 12 * e}
    if kind == "quantize":
        e, both = c["rows"] * c["cols"], int(c["by_rows"]) + int(c["by_cols"])
        scales = (c["rows"] + (c["cols"] if c["fold"] else 0)) * int(c["by_rows"]) + \
                 (c["cols"] + (c["rows"] if c["fold"] else 0)) * int(c["by_cols"])
        return {"bytes": e * (es(c["io"]) + both) + 4 * scales, "flops": 3 * e * both}
    if kind == "product":
        m, k, n = c["m"], c["k"], c["n"]
        return {"bytes": m * k + k * n + m * n * es(c["out"]) + 4 * (m + n), "flops": 2.0 * m * n * k}
    m, k, n = c["rows"], c["cols"], c["n"]
    if kind == "layer":
        stream = m * k * 2 * (3 if c["residual"] else 1)
        return {"bytes": stream + k * n + m * n * 2 + 2 * k + 4 * n, "flops": 2.0 * m * n * k + 6 * m * k}
    # gradient and weight in, the kept input, stream and its gradient in, three gradients out
    return {"bytes": 2 * m * n + k * n + m * k + 4 * m * k + 2 * k * n + 2 * m * k + 4 * (m + n + k),
            "flops": 4.0 * m * n * k + 6 * m * n + 12 * m * k}


# ----------------------------------------------------- the same in 64 bits

def _exact_codes(t, dim, fmt):
    """(codes, scale) of a 64-bit matrix along `dim`: the definition, read off without the plain form."""
    biggest = t.abs().max(dim, keepdim=True).values
    unit = biggest / LIMIT[fmt]
    ratio = t / unit.clamp_min(1e-300)
    if fmt == "int8":
        code = torch.round(ratio)
    else:
        # three bits after the leading one, in steps of 2^-9 below 2^-6
        exponent = torch.floor(torch.log2(ratio.abs().clamp_min(2.0 ** -6)))
        step = torch.exp2(exponent - 3)
        code = torch.round(ratio / step) * step
    return code, unit.squeeze(dim)


def _exact_norm(x, r, w, fmt):
    h = None if r is None else (x.double() + r.double()).to(x.dtype).double()
    v = x.double() if h is None else h
    code, unit = _exact_codes(v * w.double(), 1, fmt)
    return code, unit / torch.sqrt((v * v).mean(1) + EPS), h


def _exact_norm_grad(grad_y, h, w, grad_h):
    gy, v = grad_y.double(), h.double()
    n = v.shape[1]
    size = torch.sqrt((v * v).sum(1) / n + EPS)
    unit = v / size[:, None]
    down = gy * w.double()
    along = torch.einsum("ij,ij->i", down, unit) / n
    grad_x = (down - unit * along[:, None]) / size[:, None]
    if grad_h is not None:
        grad_x = grad_x + grad_h.double()
    return grad_x, torch.einsum("ij,ij->j", gy, unit)


def _exact_product(a, sa, b, sb):
    a = a.double() if sa is None else a.double() * sa.double()[:, None]
    b = b.double() if sb is None else b.double() * sb.double()[None, :]
    return torch.matmul(a, b)


def exact(case, seed):
    st, c = prepare(case, seed), case
    kind = c["kind"]
    if kind == "norm":
        return _exact_norm(st["x"], st["r"], st["w"], c["format"])
    if kind == "norm_grad":
        return _exact_norm_grad(st["grad_y"], st["h"], st["w"], st["grad_h"])
    if kind == "quantize":
        x, got = st["x"].double(), []
        if c["by_rows"]:
            got += _exact_codes(x if st["fold_cols"] is None else x * st["fold_cols"].double(), 1, c["format"])
        if c["by_cols"]:
            got += _exact_codes(x if st["fold_rows"] is None else x * st["fold_rows"].double()[:, None], 0, c["format"])
        return got
    if kind == "product":
        return _exact_product(st["a"], st["sa"], st["b"], st["sb"])
    if kind == "layer":
        code, scale, h = _exact_norm(st["x"], st["r"], st["w"], c["format"])
        return _exact_product(code, scale, st["W"], st["sW"]), h
    g = st["grad_out"].double()
    gr, sr = _exact_codes(g * st["sW"].double(), 1, c["format"])
    gc, sc = _exact_codes(g * st["sx"].double()[:, None], 0, c["format"])
    grad_y = _exact_product(gr, sr, st["W"].t(), None)
    grad_W = _exact_product(st["x8"].t(), None, gc, sc)
    return (grad_W,) + _exact_norm_grad(grad_y, st["h"], st["w"], st["grad_h"])
