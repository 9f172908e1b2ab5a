"""Plain 64-bit forms of dropout, layer norm and the loss of a linear head, for the tests."""

import numpy as np
import torch

F32 = 2.0 ** -24          # half a unit in the last place of fp32, relative
BF16 = 2.0 ** -8          # of bf16


def store(dtype):
    return BF16 if dtype == torch.bfloat16 else F32


def philox(counter, key):
    """Philox4x32-10: counter, four arrays (or numbers) below 2^32; key, two numbers.  Four uint64 arrays."""
    c = [np.asarray(v, dtype=np.uint64) for v in counter]
    k = list(key)
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> half) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> half) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def keep(rows, cols, p, seed, number):
    """The elements that stay, on the CPU; `number`: offset + counter."""
    number, seed = number % 2 ** 64, seed % 2 ** 64
    quad, row = np.meshgrid(np.arange(-(-cols // 4)), np.arange(rows))
    ones = np.ones_like(quad)
    w = philox((quad, row, ones * (number % 2 ** 32), (ones * (number >> 32)).astype(np.uint64)), (seed % 2 ** 32, seed >> 32))
    w = np.stack(w, 2).reshape(rows, -1)[:, :cols]
    return torch.from_numpy(w >= np.uint64(round(p * 2 ** 32)))


def dropped(v, p, seed, number):
    """v (fp32) dropped out, each step rounded to fp32."""
    if p == 0:
        return v
    k = keep(*v.shape, p, seed, number).to(v.device)
    return torch.where(k, v * torch.tensor(1 / (1 - p), dtype=torch.float32, device=v.device), torch.zeros_like(v))


def by_row(t, rows, cols):
    """A scale or shift as rows x cols, 64 bits."""
    t = t.double().reshape(-1, cols)
    return t.repeat_interleave(rows // t.shape[0], 0) if len(t) > 1 else t.expand(rows, cols)


def norm(h, weight, bias, eps, add_one=False):
    """(y, mean, rstd) and the size of y's terms, of the stored h."""
    v = h.double()
    rows, cols = v.shape
    mean = v.mean(1)
    rstd = 1 / torch.sqrt((v - mean[:, None]).square().mean(1) + eps)
    w = torch.ones_like(v) if weight is None else by_row(weight, rows, cols) + (1 if add_one else 0)
    b = torch.zeros_like(v) if bias is None else by_row(bias, rows, cols)
    y = (v - mean[:, None]) * rstd[:, None] * w + b
    return y, mean, rstd, (v.abs() + v.abs().mean(1, keepdim=True)) * rstd[:, None] * w.abs() + b.abs()


def norm_backward(grad_y, h, mean, rstd, weight, grad_h=None, add_one=False):
    """(grad_residual, grad_weight, grad_bias) and the sums of their terms' magnitudes."""
    gy, v = grad_y.double(), h.double()
    rows, cols = v.shape
    mean, rstd = mean.double()[:, None], rstd.double()[:, None]
    xhat, xs = (v - mean) * rstd, (v.abs() + mean.abs()) * rstd
    w = torch.ones_like(v) if weight is None else by_row(weight, rows, cols) + (1 if add_one else 0)
    g = gy * w
    gr = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    size = rstd * (g.abs() + g.abs().mean(1, keepdim=True) + xs * (g.abs() * xs).mean(1, keepdim=True))
    if grad_h is not None:
        gr, size = gr + grad_h.double(), size + grad_h.double().abs()
    shape = (cols,) if weight is None else weight.shape
    by = lambda t: t.reshape(-1 if len(shape) == 1 else shape[0], rows // (1 if len(shape) == 1 else shape[0]), cols).sum(1).reshape(shape)  # noqa: E731
    return gr, by(gy * xhat), by(gy), size, by(gy.abs() * xs), by(gy.abs())


def head(x, weight, labels, grad_loss=None, part=4096):
    """loss, lse, how far a logit's sum may be off (fp32 sums of exact products, cut off at each of the steps of 16 at
    worst: 2^-23 of the magnitudes' sum each), and with grad_loss the gradients and the bounds of their errors."""
    n, d = x.shape
    vocab = weight.shape[1]
    W = weight.double()
    loss, lse = (torch.zeros(n, dtype=torch.float64, device=x.device) for _ in range(2))
    off = torch.zeros_like(loss)
    steps = (d / 16 + 4) * 2.0 ** -23
    gx = gw = bx = bw = None
    if grad_loss is not None:
        gx, bx = (torch.zeros(n, d, dtype=torch.float64, device=x.device) for _ in range(2))
        gw, bw = (torch.zeros(d, vocab, dtype=torch.float64, device=x.device) for _ in range(2))
    for i in range(0, n, part):
        xi, li = x[i:i + part].double(), labels[i:i + part]
        live = (li >= 0) & (li < vocab)
        logits = xi @ W
        each = torch.logsumexp(logits, 1)
        at = logits.gather(1, torch.where(live, li, torch.zeros_like(li))[:, None])[:, 0]
        lse[i:i + part] = each
        loss[i:i + part] = torch.where(live, each - at, torch.zeros_like(each))
        off[i:i + part] = steps * (xi.abs() @ W.abs()).amax(1)
        if grad_loss is None:
            continue
        gl = torch.where(live, grad_loss[i:i + part].double(), torch.zeros_like(each))[:, None]
        p = torch.exp(logits - each[:, None])
        hot = torch.zeros_like(p).scatter_(1, torch.where(live, li, torch.zeros_like(li))[:, None], 1.0)
        g = (p - hot) * gl
        # an entry's rounding to bf16, the exponential's error, the fp32 steps around them
        dg = BF16 * g.abs() + gl.abs() * (p * (2 * off[i:i + part, None] + 2.0 ** -19 + each.abs()[:, None] * 2.0 ** -22) + 2.0 ** -22 * hot)
        gx[i:i + part], bx[i:i + part] = g @ W.t(), dg @ W.t().abs()
        gw += xi.t() @ g
        bw += xi.abs().t() @ dg
    return loss, lse, off, gx, gw, bx, bw
