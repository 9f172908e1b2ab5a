"""Plain 64-bit forms of the 8-bit operators, for the tests."""

import torch

LIMIT = {"int8": 127.0, "e4m3": 448.0}
EIGHT = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
F32 = 2.0 ** -24          # half a unit in the last place of fp32, relative
BF16 = 2.0 ** -8          # of bf16 (8 significant bits)


def ratio(t, top, fmt):
    """What is rounded to a code: t * limit / top (0 where top is 0)."""
    return torch.where(top > 0, t * LIMIT[fmt] / torch.where(top > 0, top, torch.ones_like(top)), torch.zeros_like(t))


def half_step(v, fmt):
    """Half the distance of neighbouring codes at v."""
    if fmt == "int8":
        return torch.full_like(v, 0.5)
    e = torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6)))
    return torch.exp2(e - 4)


def check_codes(codes, t, top, fmt):
    """Every code is a nearest one.  The kernel rounds four times in fp32 (the product t, 1 / top, times limit,
    times t), so it may decide a tie's neighbourhood of 4 * 2^-24 of the value either way."""
    got, want = codes.double(), ratio(t, top, fmt)
    room = half_step(torch.maximum(got.abs(), want.abs()), fmt) + 4 * F32 * want.abs()
    assert torch.all((got - want).abs() <= room), float(((got - want).abs() - room).max())
    assert got.abs().max() <= LIMIT[fmt]


def norm(x, residual, weight, eps):
    """(h, t, top, s): the stored sum, h * w, its largest magnitude by row, 1 / sqrt(mean h^2 + eps)."""
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    v = h.double()
    t = v * weight.double()
    s = 1.0 / torch.sqrt(v.square().mean(1) + eps)
    return h, t, t.abs().amax(1, keepdim=True), s


def norm_output(h, weight, eps):
    return h * weight / torch.sqrt(h.square().mean(1, keepdim=True) + eps)


def norm_backward(grad_y, h, weight, eps, grad_h=None):
    """(grad_x, grad_weight) and, for tolerances, the sums of their terms' magnitudes."""
    gy, v, w = grad_y.double(), h.double(), weight.double()
    s = 1.0 / torch.sqrt(v.square().mean(1, keepdim=True) + eps)
    g = gy * w
    gx = s * g - v * s ** 3 * (g * v).mean(1, keepdim=True)
    gx_size = s * g.abs() + v.abs() * s ** 3 * (g * v).abs().mean(1, keepdim=True)
    if grad_h is not None:
        gx = gx + grad_h.double()
        gx_size = gx_size + grad_h.double().abs()
    each = gy * v * s
    return gx, each.sum(0), gx_size, each.abs().sum(0)


def matmul(a, scale_a, b, scale_b):
    out = a.double() @ b.double()
    if scale_a is not None:
        out = out * scale_a.double()[:, None]
    if scale_b is not None:
        out = out * scale_b.double()
    return out


def random_codes(rows, cols, fmt, gen, device, pad=0x55):
    """A rows x cols matrix of codes with rows padded to 16 bytes; the padding holds other codes."""
    ld = (cols + 15) // 16 * 16
    store = torch.full((rows, ld), pad, dtype=torch.uint8, device=device)
    if fmt == "int8":
        v = torch.randint(-127, 128, (rows, cols), generator=gen, device=device, dtype=torch.int32).to(torch.int8)
    else:
        v = (torch.randn(rows, cols, generator=gen, device=device) * 60).clamp(-448, 448).to(torch.float8_e4m3fn)
    store[:, :cols] = v.view(torch.uint8)
    return store.view(EIGHT[fmt])[:, :cols]
