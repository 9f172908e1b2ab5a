"""Cases for the operators of a training step around its matrix products: layer norm with the residual's addition,
dropout from a counter-based generator, and the softmax cross entropy of a linear head over a vocabulary.

    norm        d = x, or x dropped out (in 32 bits); h = d + r in the stream's type (kept where it is not x itself);
                y = (h - mean) rstd w + b, mean and rstd of each row.  w and b have one row, or one for each group of
                neighbouring rows (the samples of a batch); add_one: the weight is 1 + w
    norm_grad   its gradient from h, mean and rstd: with xhat = (h - mean) rstd and g = grad_y w,
                grad_r = rstd (g - mean(g) - xhat mean(g xhat)) + grad_h, grad_x = grad_r dropped out alike,
                grad_w = sum over a group's rows of grad_y xhat, grad_b = sum of grad_y
    dropout     out = x / (1 - p) where the element is kept, else 0, plus r
    loss        lse = log sum exp of x @ W, loss = lse - the label's logit; 0 for labels outside the vocabulary
    loss_grad   from the gradient of each row's loss and lse: grad_x and grad_W

The element in row i and column j is kept where word j % 4 of Philox4x32-10 at the counter (j // 4, i, low and high
half of the draw's number) under the seed is at least p 2^32; the draw's number is an offset plus a word on the device.
"""

import math

import numpy as np
import torch

own = False

EPS = 1e-6
DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # one token of a served model: launch and latency are all that counts
        {"name": "norm_one_token", "kind": "norm", "rows": 1, "cols": 2048, "io": "bf16", "weight": "bf16", "groups": 1,
         "add_one": False, "residual": True, "p": 0.0},
        # a training batch of the widest stream that the benchmark times, its branch dropped out on the way in
        {"name": "norm_batch", "kind": "norm", "rows": 8192, "cols": 4096, "io": "bf16", "weight": "bf16", "groups": 1,
         "add_one": False, "residual": True, "p": 0.1},
        # adaptive norm of a diffusion batch: scale and shift of each sample, cut from one wide product
        {"name": "norm_by_sample", "kind": "norm", "rows": 16384, "cols": 2048, "io": "bf16", "weight": "bf16", "groups": 64,
         "add_one": True, "residual": False, "p": 0.0},
        # the backward pass of a training batch, with the gradient that comes down the residual stream
        {"name": "norm_grad_batch", "kind": "norm_grad", "rows": 8192, "cols": 4096, "io": "bf16", "weight": "bf16",
         "groups": 1, "add_one": False, "grad_h": True, "p": 0.1},
        # that of the adaptive norm: sums over the rows of each sample
        {"name": "norm_grad_by_sample", "kind": "norm_grad", "rows": 16384, "cols": 2048, "io": "bf16", "weight": "bf16",
         "groups": 64, "add_one": True, "grad_h": True, "p": 0.0},
        # fp32 stream of an odd width: no row but the first starts on a vector's boundary
        {"name": "norm_grad_ragged_fp32", "kind": "norm_grad", "rows": 777, "cols": 1111, "io": "fp32", "weight": "fp32",
         "groups": 1, "add_one": False, "grad_h": False, "p": 0.0},
        # dropout of a large activation (gate of an MLP)
        {"name": "dropout_batch", "kind": "dropout", "rows": 8192, "cols": 8192, "io": "bf16", "residual": False, "p": 0.1},
        # odd width in fp32, joined to the residual stream
        {"name": "dropout_ragged_fp32", "kind": "dropout", "rows": 333, "cols": 1001, "io": "fp32", "residual": True, "p": 0.25},
        # one token's loss: the weight's bytes are the work
        {"name": "loss_one_token", "kind": "loss", "rows": 1, "d": 4096, "vocab": 32768, "stored": "in_out"},
        # a training batch over a large vocabulary
        {"name": "loss_batch", "kind": "loss", "rows": 8192, "d": 4096, "vocab": 131072, "stored": "in_out"},
        # odd sizes in every direction, the weight an embedding (vocabulary x d), some rows without a label
        {"name": "loss_grad_ragged", "kind": "loss_grad", "rows": 203, "d": 1000, "vocab": 10007, "stored": "out_in",
         "weighted": False},
        # the backward pass of a training batch
        {"name": "loss_grad_batch", "kind": "loss_grad", "rows": 8192, "d": 4096, "vocab": 65536, "stored": "in_out",
         "weighted": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size of the range, spread over its logarithm: odd ones, multiples of 8 and of 128."""
    step = rng.choice((1, 8, 128))
    v = _log(rng, lo, hi)
    return v if step == 1 or v < step else max(lo, v // step * step)


def draw(rng):
    kind = rng.choice(("norm", "norm_grad", "dropout", "loss", "loss_grad"))
    io, weight = rng.choice((("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32")))
    if kind in ("norm", "norm_grad"):
        groups = rng.choice((1, 1, _log(rng, 2, 128)))
        case = {"kind": kind, "rows": _log(rng, 1, 8192 // groups) * groups, "cols": _size(rng, 64, 8192), "io": io,
                "weight": weight, "groups": groups, "add_one": rng.random() < 0.5}
        case["residual" if kind == "norm" else "grad_h"] = rng.random() < 0.75
        return {**case, "p": rng.choice((0.0, 0.1, 0.5))}
    if kind == "dropout":
        return {"kind": kind, "rows": _log(rng, 1, 8192), "cols": _size(rng, 64, 8192), "io": io,
                "residual": rng.random() < 0.5, "p": rng.choice((0.1, 0.25, 0.5))}
    case = {"kind": kind, "rows": _log(rng, 1, 8192), "d": _size(rng, 64, 4096), "vocab": _size(rng, 256, 65536),
            "stored": rng.choice(("in_out", "out_in"))}
    return case if kind == "loss" else {**case, "weighted": rng.random() < 0.5}


# ------------------------------------------------------------------ inputs

class _Source:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g, device="cuda")

    def stream(self, rows, cols, dtype):
        """A residual stream: its mean is off zero and a few channels are ten times the others."""
        channel = 1 + 9 * (torch.rand(cols, generator=self.g, device="cuda") < 0.01)
        return (self.normal(rows, cols) * channel + 0.5).to(dtype)

    def grad(self, rows, cols, dtype):
        """A gradient: small, and of another size for each token."""
        return (self.normal(rows, cols) * (1e-3 * torch.exp(self.normal(rows, 1)))).to(dtype)

    def number(self, bits):
        return int(torch.randint(0, 1 << bits, (1,), generator=self.g, device="cuda"))


def prepare(case, seed):
    s, c = _Source(seed), case
    kind = c["kind"]
    st = {"case": c}
    if kind in ("norm", "norm_grad", "dropout"):
        io, rows, cols = DTYPE[c["io"]], c["rows"], c["cols"]
        st["seed"], st["offset"] = s.number(62), s.number(8)
        st["counter"] = torch.tensor([s.number(40)], dtype=torch.int64, device="cuda")
    if kind in ("norm", "norm_grad"):
        wt, groups = DTYPE[c["weight"]], c["groups"]
        # one product gives scale, shift and more for each sample; the norm takes two strips of it
        wide = (0.2 * s.normal(groups, 6 * cols) + (0.0 if c["add_one"] else 1.0)).to(wt)
        st["w"], st["b"] = wide[:, :cols], wide[:, 2 * cols:3 * cols]
        if groups == 1:
            st["w"], st["b"] = st["w"][0].clone(), st["b"][0].clone()
    if kind == "norm":
        st["x"] = s.stream(rows, cols, io)
        st["r"] = s.stream(rows, cols, io) if c["residual"] else None
    elif kind == "norm_grad":
        st["h"], st["grad_y"] = s.stream(rows, cols, io), s.grad(rows, cols, io)
        st["grad_h"] = s.grad(rows, cols, io) if c["grad_h"] else None
        # what the forward pass kept
        v = st["h"].double()
        st["mean"] = v.mean(1).float()
        st["rstd"] = (1 / torch.sqrt(v.var(1, unbiased=False) + EPS)).float()
    elif kind == "dropout":
        st["x"] = s.stream(rows, cols, io)
        st["r"] = s.stream(rows, cols, io) if c["residual"] else None
    else:
        rows, d, vocab = c["rows"], c["d"], c["vocab"]
        # normed rows, and a weight that gives logits of about the size 1 to 2
        st["x"] = s.normal(rows, d).to(torch.bfloat16)
        shape = (d, vocab) if c["stored"] == "in_out" else (vocab, d)
        st["W"] = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.5 * d ** -0.5, generator=s.g)
        # padded rows (one of 16) carry the label -100
        st["labels"] = torch.randint(0, vocab, (rows,), generator=s.g, device="cuda")
        st["labels"][torch.rand(rows, generator=s.g, device="cuda") < 1 / 16] = -100
        if rows == 1:
            st["labels"].clamp_(min=0)
        if kind == "loss_grad":
            live = st["labels"] >= 0
            gl = torch.exp(s.normal(rows)) if c["weighted"] else torch.ones(rows, device="cuda")
            st["grad_loss"] = gl / live.sum().clamp(min=1)
            logits = (st["x"].double() @ _in_out(st).double())
            st["lse"] = torch.logsumexp(logits, 1).float()
    return st


def _in_out(st):
    return st["W"] if st["case"]["stored"] == "in_out" else st["W"].t()


# ------------------------------------------------------------- plain forms

M0, M1, W0, W1, LOW = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85, 0xFFFFFFFF


def _plain_keep(rows, cols, p, seed, number):
    """Philox4x32-10 in 64-bit integers, whose products wrap; `number`: a device word."""
    quads = -(-cols // 4)
    c0 = torch.arange(quads, device="cuda").expand(rows, quads)
    c1 = torch.arange(rows, device="cuda")[:, None].expand(rows, quads)
    c2, c3 = (number & LOW).expand(rows, quads), ((number >> 32) & LOW).expand(rows, quads)
    k0, k1 = seed & LOW, seed >> 32
    for r in range(10):
        a, b = c0 * M0, c2 * M1
        c0, c1, c2, c3 = ((b >> 32) & LOW) ^ c1 ^ k0, b & LOW, ((a >> 32) & LOW) ^ c3 ^ k1, a & LOW
        k0, k1 = (k0 + W0) & LOW, (k1 + W1) & LOW
    return torch.stack((c0, c1, c2, c3), 2).reshape(rows, -1)[:, :cols] >= round(p * 2.0 ** 32)


def _plain_dropped(v, p, st):
    """v (32 bits) dropped out."""
    if p == 0:
        return v
    keep = _plain_keep(*v.shape, p, st["seed"], st["counter"] + st["offset"])
    return torch.where(keep, v * (1 / (1 - p)), torch.zeros((), device="cuda"))


def _plain_rows(t, rows):
    """A weight's row for each row of the stream, 32 bits."""
    t = t.float().reshape(-1, t.shape[-1])
    return t.repeat_interleave(rows // t.shape[0], 0) if t.shape[0] > 1 else t


def _plain_norm(st, c):
    x, r, p = st["x"], st["r"], c["p"]
    h = None
    if r is not None or p > 0:
        h = _plain_dropped(x.float(), p, st)
        h = (h if r is None else h + r.float()).to(x.dtype)
    v = (x if h is None else h).float()
    mean = v.mean(1, keepdim=True)
    rstd = torch.rsqrt((v - mean).square().mean(1, keepdim=True) + EPS)
    w = _plain_rows(st["w"], len(v))
    y = (v - mean) * rstd * (1 + w if c["add_one"] else w) + _plain_rows(st["b"], len(v))
    return [y.to(x.dtype), mean[:, 0], rstd[:, 0]] + ([] if h is None else [h])


def _plain_norm_grad(st, c):
    gy, v, rstd = st["grad_y"].float(), st["h"].float(), st["rstd"][:, None]
    xhat = (v - st["mean"][:, None]) * rstd
    w = _plain_rows(st["w"], len(v))
    g = gy * (1 + w if c["add_one"] else w)
    gr = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    if st["grad_h"] is not None:
        gr = gr + st["grad_h"].float()
    shape = (c["groups"], -1, v.shape[1])
    gw, gb = ((gy * xhat).reshape(shape).sum(1), gy.reshape(shape).sum(1))
    out = [gr.to(st["h"].dtype), gw.reshape(st["w"].shape).to(st["w"].dtype), gb.reshape(st["b"].shape).to(st["b"].dtype)]
    return out + ([_plain_dropped(gr, c["p"], st).to(st["h"].dtype)] if c["p"] > 0 else [])


def _plain_dropout(st, c):
    out = _plain_dropped(st["x"].float(), c["p"], st)
    return (out if st["r"] is None else out + st["r"].float()).to(st["x"].dtype)


def _plain_loss(st):
    logits, labels = st["x"].float() @ _in_out(st).float(), st["labels"]
    top = logits.amax(1, keepdim=True)
    lse = top[:, 0] + torch.log(torch.exp(logits - top).sum(1))
    live = labels >= 0
    at = logits.gather(1, labels.clamp(min=0)[:, None])[:, 0]
    return torch.where(live, lse - at, torch.zeros_like(lse)), lse


def _plain_loss_grad(st):
    x, W, labels = st["x"].float(), st["W"].float(), st["labels"]
    live = labels >= 0
    gl = torch.where(live, st["grad_loss"], torch.zeros_like(st["grad_loss"]))
    in_out = st["case"]["stored"] == "in_out"
    g = torch.exp(x @ (W if in_out else W.t()) - st["lse"][:, None])
    g[torch.arange(len(x), device="cuda"), labels.clamp(min=0)] -= 1
    g *= gl[:, None]
    return [(g @ (W.t() if in_out else W)).to(torch.bfloat16), (x.t() @ g if in_out else g.t() @ x).to(torch.bfloat16)]


def _run_plain(st, c):
    kind = c["kind"]
    if kind == "norm":
        return _plain_norm(st, c)
    if kind == "norm_grad":
        return _plain_norm_grad(st, c)
    if kind == "dropout":
        return _plain_dropout(st, c)
    return _plain_loss(st) if kind == "loss" else _plain_loss_grad(st)


# ------------------------------------------------- the framework's operators

def _run_own(st, c):
    from paper_2608_20818_b200 import binding as B

    kind = c["kind"]
    if kind == "norm":
        y, h, mean, rstd = B.prm_layernorm(st["x"], st["w"], st["b"], EPS, residual=st["r"], add_one=c["add_one"], p=c["p"],
                                           seed=st["seed"], offset=st["offset"], counter=st["counter"])
        return [y, mean, rstd] + ([] if h is None else [h])
    if kind == "norm_grad":
        gx, gr, gw, gb = B.prm_layernorm_backward(st["grad_y"], st["h"], st["mean"], st["rstd"], st["w"],
                                                  grad_h=st["grad_h"], add_one=c["add_one"], p=c["p"], seed=st["seed"],
                                                  offset=st["offset"], counter=st["counter"])
        return [gx, gw, gb] if gr is None else [gr, gw, gb, gx]
    if kind == "dropout":
        return B.prm_dropout(st["x"], c["p"], st["seed"], st["offset"], counter=st["counter"], residual=st["r"])
    if kind == "loss":
        return B.prm_head_loss(st["x"], _in_out(st), st["labels"])
    gx, gw = B.prm_head_loss_backward(st["grad_loss"], st["x"], _in_out(st), st["labels"], st["lse"])
    return [gx, gw if c["stored"] == "in_out" else gw.t()]


def run(state):
    return _run_own(state, state["case"]) if own else _run_plain(state, state["case"])


# -------------------------------------------------------------------- work

def work(case):
    c, kind = case, case["kind"]
    es = lambda name: 2 if name == "bf16" else 4  # noqa: E731
    if kind == "norm":
        e = c["rows"] * c["cols"]
        kept = c["residual"] or c["p"] > 0
        per = es(c["io"]) * (2 + int(c["residual"]) + int(kept))
        return {"bytes": e * per + 2 * c["groups"] * c["cols"] * es(c["weight"]) + 8 * c["rows"], "flops": 8 * e}
    if kind == "norm_grad":
        e = c["rows"] * c["cols"]
        per = es(c["io"]) * (3 + int(c["grad_h"]) + int(c["p"] > 0))
        return {"bytes": e * per + 3 * c["groups"] * c["cols"] * es(c["weight"]) + 8 * c["rows"], "flops": 14 * e}
    if kind == "dropout":
        e = c["rows"] * c["cols"]
        return {"bytes": e * es(c["io"]) * (2 + int(c["residual"])), "flops": 2 * e}
    n, d, v = c["rows"], c["d"], c["vocab"]
    if kind == "loss":
        return {"bytes": 2 * (n * d + d * v) + 16 * n, "flops": 2.0 * n * d * v}
    return {"bytes": 4 * (n * d + d * v) + 16 * n, "flops": 6.0 * n * d * v}


# ----------------------------------------------------- the same in 64 bits

def _exact_factor(rows, cols, p, st):
    """What each element is multiplied by: the generator on the host, in unsigned 64-bit integers, rows in parts."""
    if p == 0:
        return torch.ones((), dtype=torch.float64, device="cuda")
    number = (int(st["counter"]) + st["offset"]) % 2 ** 64
    out = torch.empty(rows, cols, dtype=torch.bool, device="cuda")
    part = max(1, (1 << 20) // -(-cols // 4))
    u = np.uint64
    half, low = u(32), u(LOW)
    for i in range(0, rows, part):
        n = min(part, rows - i)
        x = np.zeros((4, n, -(-cols // 4)), dtype=u)
        x[0] += np.arange(x.shape[2], dtype=u)
        x[1] += np.arange(i, i + n, dtype=u)[:, None]
        x[2] += u(number % 2 ** 32)
        x[3] += u(number >> 32)
        key = [st["seed"] % 2 ** 32, st["seed"] >> 32]
        for _ in range(10):
            even, odd = x[0] * u(M0), x[2] * u(M1)
            x = np.stack([(odd >> half) ^ x[1] ^ u(key[0]), odd & low, (even >> half) ^ x[3] ^ u(key[1]), even & low])
            key = [(key[0] + W0) % 2 ** 32, (key[1] + W1) % 2 ** 32]
        words = np.moveaxis(x, 0, 2).reshape(n, -1)[:, :cols]
        out[i:i + n] = torch.from_numpy(words >= u(round(p * 2 ** 32))).cuda()
    return out.double() / (1 - p)


def _exact_affine(st, c, rows):
    w, b = (torch.atleast_2d(st[k]).double() for k in ("w", "b"))
    group = torch.arange(rows, device="cuda") // (rows // c["groups"])
    return (w + 1 if c["add_one"] else w)[group], b[group]


def exact(case, seed):
    st, c = prepare(case, seed), case
    kind = c["kind"]
    if kind == "norm":
        x = st["x"]
        kept = st["r"] is not None or c["p"] > 0
        h = x
        if kept:
            # the norm is taken of the sum as it is stored: factor, sum and store round in 32 bits, 32 bits and the type
            h = (x.double() * _exact_factor(*x.shape, c["p"], st).float()).float()
            h = (h if st["r"] is None else (h.double() + st["r"].double()).float()).to(x.dtype)
        v = h.double()
        var, mean = torch.var_mean(v, 1, correction=0)
        w, b = _exact_affine(st, c, len(x))
        rstd = (var + EPS) ** -0.5
        y = torch.addcmul(b, (v - mean[:, None]) * rstd[:, None], w)
        return [y, mean, rstd] + ([v] if kept else [])
    if kind == "norm_grad":
        h, gy = st["h"].double(), st["grad_y"].double()
        n = h.shape[1]
        w, _ = _exact_affine({**st, "b": st["w"]}, c, len(h))
        rstd = st["rstd"].double()[:, None]
        xhat = (h - st["mean"].double()[:, None]) * rstd
        g = gy * w
        gr = rstd * (g - (g.sum(1, keepdim=True) + xhat * torch.einsum("ij,ij->i", g, xhat)[:, None]) / n)
        if st["grad_h"] is not None:
            gr = gr + st["grad_h"].double()
        by = lambda t: t.unflatten(0, (c["groups"], -1)).sum(1).reshape(st["w"].shape)  # noqa: E731
        out = [gr, by(gy * xhat), by(gy)]
        return out + ([gr * _exact_factor(*h.shape, c["p"], st)] if c["p"] > 0 else [])
    if kind == "dropout":
        out = st["x"].double() * _exact_factor(*st["x"].shape, c["p"], st)
        return out if st["r"] is None else out + st["r"].double()
    x, W, labels = st["x"].double(), st["W"].double(), st["labels"]
    spec = "ik,kv->iv" if c["stored"] == "in_out" else "ik,vk->iv"
    logits = torch.einsum(spec, x, W)
    live = (labels >= 0) & (labels < c["vocab"])
    if kind == "loss":
        lse = torch.logsumexp(logits, 1)
        loss = torch.zeros_like(lse)
        loss[live] = lse[live] - logits[live, labels[live]]
        return loss, lse
    g = torch.softmax(logits, 1)
    g[live, labels[live]] -= 1
    g = g * (st["grad_loss"].double() * live)[:, None]
    back = "iv,kv->ik" if c["stored"] == "in_out" else "iv,vk->ik"
    return [torch.einsum(back, g, W), torch.einsum("ik,iv->kv" if c["stored"] == "in_out" else "ik,iv->vk", x, g)]
