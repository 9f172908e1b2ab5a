"""The 8-bit operators (norm with residual, its gradient, quantiser, product) against plain 64-bit forms."""

import pytest
import torch

import q8_reference as R
from paper_2608_20818_b200 import binding as B

IO = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-6
# one row, one column, less than a vector, odd, a warp's, a block's, past each limit of the row kernels
SHAPES = [(1, 1), (1, 8), (3, 5), (2, 256), (9, 257), (7, 512), (5, 1000), (3, 1024), (4, 1111), (1, 2048),
          (130, 2056), (3, 4096), (2, 4104), (2, 8192), (2, 8193), (1, 16384), (1, 16400), (1, 16401), (1, 32768),
          (2, 32776), (1, 40001), (1000, 64), (4099, 24), (0, 16),
          # rows that start on every offset from a vector, for each width of the kernels that walk them
          (17, 3), (40, 249), (33, 505), (310, 1001), (19, 2041), (310, 4089), (11, 8185), (9, 16377), (9, 20001),
          (9, 16378), (300, 4100), (12, 12), (3, 24576), (2, 32768),
          # large enough to be streamed: each group width, full and partly filled, rows that do not divide
          (8201, 512), (4700, 1000), (4099, 1024), (2050, 2056), (2100, 2048), (1030, 4096), (700, 6000), (519, 8192),
          # narrow rows, several to a warp: more than the grid takes in one turn; short rows by the block
          (40003, 64), (20011, 128), (10001, 256), (37, 120), (2051, 1000)]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def stored(ref, io):
    """Rounding of a value at its store."""
    return ref.abs() * (R.BF16 if io == torch.bfloat16 else R.F32) * 1.01


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("io,weight", [("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32")])
def test_norm(rows, cols, io, weight):
    g = gen(rows * 131 + cols)
    x, r = (randn(g, rows, cols).to(IO[io]) for _ in range(2))
    w = (1 + 0.2 * randn(g, cols)).to(IO[weight])
    for fmt in ("int8", "e4m3"):
        for res in (r, None):
            q, scale, h = B.prm_rmsnorm_q8(x, w, EPS, residual=res, format=fmt)
            assert q.dtype == R.EIGHT[fmt] and q.shape == (rows, cols) and q.stride(0) % 16 == 0
            ref_h, t, top, s = R.norm(x, res, w, EPS)
            if res is None:
                assert h is None
            else:
                assert torch.equal(h, ref_h)
            if rows == 0:
                continue
            R.check_codes(q, t, top, fmt)
            # the sum of squares: at most 64 additions after one another, then a handful of roundings
            ref = top[:, 0] / R.LIMIT[fmt] * s
            assert torch.all((scale.double() - ref).abs() <= 80 * R.F32 * ref)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("io,weight", [("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32")])
def test_norm_backward(rows, cols, io, weight):
    g = gen(rows * 17 + cols)
    h, gh = randn(g, rows, cols).to(IO[io]), randn(g, rows, cols).to(IO[io])
    gy = (1e-2 * randn(g, rows, cols)).to(IO[io])
    w = (1 + 0.2 * randn(g, cols)).to(IO[weight])
    for d in (gh, None):
        gx, gw = B.prm_rmsnorm_q8_backward(gy, h, w, EPS, grad_h=d)
        assert gx.dtype == h.dtype and gw.dtype == w.dtype
        rx, rw, sx, sw = R.norm_backward(gy, h, w, EPS, d)
        # every term goes through the two row sums and a handful of products: 100 roundings at most
        assert torch.all((gx.double() - rx).abs() <= 100 * R.F32 * sx + stored(rx, h.dtype))
        # added over the rows in turn at worst, on top of a term's own 100
        assert torch.all((gw.double() - rw).abs() <= (100 + rows) * R.F32 * sw + stored(rw, w.dtype))


def test_norm_gradient_formula_against_differences():
    g = torch.Generator().manual_seed(1)
    for rows, cols in ((1, 1), (3, 7), (5, 64)):
        h, w = (torch.randn(rows, cols, generator=g, dtype=torch.float64) for _ in range(2))
        w = w[0]
        gy, dh = (torch.randn(rows, cols, generator=g, dtype=torch.float64) for _ in range(2))
        dw = torch.randn(cols, generator=g, dtype=torch.float64)
        gx, gw, _, _ = R.norm_backward(gy, h, w, EPS)
        e = 1e-5
        f = lambda a, b: float((R.norm_output(a, b, EPS) * gy).sum())  # noqa: E731
        along_h = (f(h + e * dh, w) - f(h - e * dh, w)) / (2 * e)
        along_w = (f(h, w + e * dw) - f(h, w - e * dw)) / (2 * e)
        # the difference's own error: e^2 times a third derivative that reaches |h|^-3
        assert abs(along_h - float((gx * dh).sum())) < 1e-5 * (1 + abs(along_h)) / float(h.square().mean(1).min())
        assert abs(along_w - float((gw * dw).sum())) < 1e-7 * (1 + abs(along_w))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [s for s in SHAPES if s[0]] + [(300, 16384), (5, 24584), (2, 24584), (700, 40968)])
@pytest.mark.parametrize("io", ["bf16", "fp32"])
def test_quantize(rows, cols, io):
    g = gen(rows * 7 + cols)
    x = (randn(g, rows, cols) * torch.exp(randn(g, rows, 1))).to(IO[io])
    fr, fc = torch.exp(randn(g, rows)), torch.exp(randn(g, cols))
    for fmt in ("int8", "e4m3"):
        for by_rows, by_cols, fold in ((True, False, False), (False, True, False), (True, True, True), (False, True, True)):
            got = B.prm_quantize_q8(x, by_rows=by_rows, by_cols=by_cols, fold_rows=fr if fold else None,
                                    fold_cols=fc if fold else None, format=fmt)
            assert [v is not None for v in got] == [by_rows, by_rows, by_cols, by_cols]
            for dim, q, scale, f in ((1, got[0], got[1], fc[None, :]), (0, got[2], got[3], fr[:, None])):
                if q is None:
                    continue
                t = x.double() * f.double() if fold else x.double()
                top = t.abs().amax(dim, keepdim=True)
                R.check_codes(q, t, top, fmt)
                ref = top.reshape(-1) / R.LIMIT[fmt]
                assert torch.all((scale.double() - ref).abs() <= 3 * R.F32 * ref)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("cols", [40, 45, 2048])
def test_rows_without_a_scale(fmt, cols):
    """Zero rows, rows below 2^-100, infinities and NaN: each marks its own row (column) only."""
    x = randn(gen(3), 6, cols)
    x[1] = 0
    x[2] = 2.0 ** -110
    x[3, cols // 2] = float("inf")
    x[4, 7] = float("nan")
    w = torch.ones(cols, device="cuda")
    q, scale, h = B.prm_rmsnorm_q8(x, w, EPS, residual=torch.zeros_like(x), format=fmt)
    qr, sr, qc, sc = B.prm_quantize_q8(x, by_rows=True, by_cols=True, format=fmt)
    for codes, s in ((q, scale), (qr, sr)):
        assert torch.all(codes[1:5].float() == 0)
        assert s[1] == 0 and s[2] == 0 and torch.isnan(s[3]) and torch.isnan(s[4])
        assert torch.isfinite(s[[0, 5]]).all() and codes[0].float().abs().max() == R.LIMIT[fmt]
    bad = torch.zeros(cols, dtype=torch.bool, device="cuda")
    bad[[cols // 2, 7]] = True
    assert torch.equal(torch.isnan(sc), bad) and torch.all(qc[:, bad].float() == 0)
    assert torch.all(qc[:, ~bad].float().abs().amax(0) == R.LIMIT[fmt])
    y = B.prm_matmul_q8(q, scale, qr.t(), None, out_dtype=torch.float32)
    assert torch.isnan(y[3:5]).all() and torch.isfinite(y[[0, 1, 2, 5]]).all()
    x.zero_()
    qr, sr, qc, sc = B.prm_quantize_q8(x, by_rows=True, by_cols=True, format=fmt)
    assert not sr.any() and not sc.any() and not qr.float().any() and not qc.float().any()


# m, k, n: one of each, odd, tile edges (16, 128, 256), several tiles, a split sum, more tiles than SMs
PRODUCTS = [(1, 1, 1), (1, 16, 7), (2, 31, 64), (1, 4096, 512), (5, 1000, 130), (16, 128, 128), (17, 129, 127),
            (33, 2048, 515), (128, 640, 256), (130, 96, 300), (257, 1000, 129), (256, 4096, 640), (300, 33, 2100),
            (1000, 520, 3000), (2049, 384, 2500), (4096, 256, 4096)]


def codes_as(rows, cols, fmt, g, transposed):
    return R.random_codes(cols, rows, fmt, g, "cuda").t() if transposed else R.random_codes(rows, cols, fmt, g, "cuda")


def product_room(a, sa, b, sb, ref, fmt, dtype):
    if fmt == "int8":         # exact sum, its conversion, two scales
        room = 4 * R.F32 * ref.abs()
    else:                     # each of k products aligned to the largest and cut at 2^-23 of it, at worst
        size = a.double().abs() @ b.double().abs()
        size = size * (1.0 if sa is None else sa.double()[:, None]) * (1.0 if sb is None else sb.double())
        room = (a.shape[1] + 4) * 2 * R.F32 * size
    return room + stored(ref, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("m,k,n", PRODUCTS)
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_product(m, k, n, fmt):
    g = gen(m + k + n)
    sa, sb = torch.exp(randn(g, m)), torch.exp(randn(g, n))
    for a_t in (False, True):
        for b_t in (False, True):
            a, b = codes_as(m, k, fmt, g, a_t), codes_as(k, n, fmt, g, b_t)
            for ua, ub, dtype in ((sa, sb, torch.bfloat16), (None, sb, torch.float32), (sa, None, torch.bfloat16)):
                out = B.prm_matmul_q8(a, ua, b, ub, out_dtype=dtype)
                assert out.dtype == dtype and out.shape == (m, n)
                ref = R.matmul(a, ua, b, ub)
                room = product_room(a, ua, b, ub, ref, fmt, dtype)
                assert torch.all((out.double() - ref).abs() <= room), (a_t, b_t, dtype)
    assert B.prm_q8_status() == B.PRM_OK


@pytest.mark.gpu
def test_product_sizes_of_zero():
    g = gen(5)
    for m, k, n in ((0, 32, 16), (16, 32, 0), (3, 0, 5)):
        a, b = R.random_codes(m, k, "int8", g, "cuda"), R.random_codes(k, n, "int8", g, "cuda")
        out = B.prm_matmul_q8(a, None, b, None)
        assert out.shape == (m, n) and not out.any()


@pytest.mark.gpu
def test_product_lowest_code_and_long_sums():
    """-128 is no code of the quantiser but a legal int8; sums beyond 2^31 stay exact."""
    a = torch.full((3, 4096), -128, dtype=torch.int8, device="cuda")
    assert torch.all(B.prm_matmul_q8(a, None, a.t(), None, out_dtype=torch.float32) == 128.0 * 128 * 4096)
    k = 200000
    a = torch.full((3, k), 127, dtype=torch.int8, device="cuda")
    assert torch.all(B.prm_matmul_q8(a, None, a.t(), None, out_dtype=torch.float32).double()
                     == float(torch.tensor(127.0 * 127 * k)))
    x8 = torch.full((k, 32), 127, dtype=torch.int8, device="cuda")
    assert torch.all(B.prm_matmul_q8(x8.t(), None, x8, None, out_dtype=torch.float32).double()
                     == float(torch.tensor(127.0 * 127 * k)))
    with pytest.raises(B.PrmError) as e:
        a = torch.zeros((1, 1047553), dtype=torch.int8, device="cuda")
        B.prm_matmul_q8(a, None, a.t(), None)
    assert e.value.code == B.PRM_ERR_SHAPE


@pytest.mark.gpu
def test_product_special_floats():
    a = torch.ones((4, 64), device="cuda")
    a[2, 5] = float("nan")
    a8, b8 = a.to(torch.float8_e4m3fn), torch.ones((64, 40), device="cuda").to(torch.float8_e4m3fn)
    out = B.prm_matmul_q8(a8, None, b8, None, out_dtype=torch.float32)
    assert torch.isnan(out[2]).all() and torch.all(out[[0, 1, 3]] == 64)
    sa = torch.tensor([1.0, float("inf"), 0.0, float("nan")], device="cuda")
    out = B.prm_matmul_q8(b8[:, :4].t().contiguous(), sa, b8, None, out_dtype=torch.float32)
    assert torch.all(out[0] == 64) and torch.isinf(out[1]).all() and torch.all(out[2] == 0) and torch.isnan(out[3]).all()


@pytest.mark.gpu
def test_views_and_other_layouts():
    """Row slices, column slices off any alignment, repeated rows and transposed inputs, into given outputs."""
    g = gen(9)
    big = randn(g, 70, 700).to(torch.bfloat16)
    w = torch.ones(500, device="cuda", dtype=torch.bfloat16)
    for x in (big[3:60:2, 100:600], big[:50, 1:501], big[:1, 8:508].expand(9, 500), randn(g, 500, 20).to(torch.bfloat16).t()):
        q, scale, h = B.prm_rmsnorm_q8(x, w, EPS, residual=x)
        q2, scale2, h2 = B.prm_rmsnorm_q8(x.contiguous(), w, EPS, residual=x.contiguous())
        assert torch.equal(h, h2) and torch.equal(q, q2) and torch.all((scale - scale2).abs() <= 80 * R.F32 * scale2)
        gx, gw = B.prm_rmsnorm_q8_backward(x, h, w, EPS, grad_h=x)
        rx, rw, sx, sw = R.norm_backward(x, h, w, EPS, x)
        assert torch.all((gx.double() - rx).abs() <= 100 * R.F32 * sx + stored(rx, gx.dtype))
        assert torch.all((gw.double() - rw).abs() <= (100 + len(x)) * R.F32 * sw + stored(rw, gw.dtype))
        got, want = B.prm_quantize_q8(x, by_cols=True), B.prm_quantize_q8(x.contiguous(), by_cols=True)
        assert all(torch.equal(u, v) for u, v in zip(got, want))
    codes = R.random_codes(300, 400, "int8", g, "cuda")
    b = R.random_codes(100, 64, "int8", g, "cuda")
    for a in (codes[10:50, 16:116], codes[:, 3:103], codes[::3, ::4], codes.t()[16:60, 32:132], codes[7:8, :100]):
        ref = R.matmul(a, None, b, None)
        assert torch.equal(B.prm_matmul_q8(a, None, b, None, out_dtype=torch.float32).double(), ref)
        store = torch.full((a.shape[0] + 2, 90), 7.0, device="cuda")
        out = store[1:-1, 5:69]
        assert B.prm_matmul_q8(a, None, b, None, out=out) is out
        assert torch.equal(out.double(), ref)
        store[1:-1, 5:69] = 7.0
        assert torch.all(store == 7.0)          # nothing was written beside the given matrix


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_product_into_padded_output(dtype):
    g = gen(23)
    for m, k, n, ld in ((300, 256, 520, 528), (300, 256, 520, 523), (2049, 128, 2500, 2504), (2049, 128, 2500, 2501)):
        a, b = R.random_codes(m, k, "int8", g, "cuda"), R.random_codes(k, n, "int8", g, "cuda")
        store = torch.full((m + 1, ld), 7.0, device="cuda", dtype=dtype)
        out = store[:m, :n]
        B.prm_matmul_q8(a, None, b, None, out=out)
        assert torch.all((out.double() - R.matmul(a, None, b, None)).abs() <= stored(R.matmul(a, None, b, None), dtype))
        out.fill_(7.0)
        assert torch.all(store == 7.0)


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    step = (1 << 31) + 4096 + 64
    store = torch.zeros(2 * step + 8192, dtype=torch.bfloat16, device="cuda")      # 8.6 GB
    x = store.as_strided((3, 4096), (step, 1))
    x.copy_(randn(gen(1), 3, 4096))
    w = torch.ones(4096, device="cuda")
    q, scale, _ = B.prm_rmsnorm_q8(x, w, EPS)
    q2, scale2, _ = B.prm_rmsnorm_q8(x.contiguous(), w, EPS)
    assert torch.equal(q, q2) and torch.equal(scale, scale2)
    got, want = B.prm_quantize_q8(x, by_cols=True), B.prm_quantize_q8(x.contiguous(), by_cols=True)
    assert all(torch.equal(u, v) for u, v in zip(got, want))
    gx, gw = B.prm_rmsnorm_q8_backward(x, x, w, EPS, grad_h=x)
    gx2, gw2 = B.prm_rmsnorm_q8_backward(x.contiguous(), x.contiguous(), w, EPS, grad_h=x.contiguous())
    assert torch.equal(gx, gx2) and torch.equal(gw, gw2)
    b = R.random_codes(4096, 96, "int8", gen(2), "cuda")
    ref = R.matmul(q, scale, b, None)
    out = store.as_strided((3, 96), (step, 1))
    B.prm_matmul_q8(q, scale, b, None, out=out)
    assert torch.all((out.double() - ref).abs() <= 4 * R.F32 * ref.abs() + stored(ref, out.dtype))
    a = store.view(torch.int8).as_strided((3, 4096), (step, 1))
    a.copy_(q)
    assert torch.equal(B.prm_matmul_q8(a, scale, b, None), B.prm_matmul_q8(q, scale, b, None))
    del store, x, out, a
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_other_stream_and_graph():
    g = gen(4)
    x, r = (randn(g, 300, 640).to(torch.bfloat16) for _ in range(2))
    w = torch.ones(640, device="cuda", dtype=torch.bfloat16)
    W8, _, _, _ = B.prm_quantize_q8(randn(g, 640, 384).to(torch.bfloat16))
    sw = torch.ones(384, device="cuda")

    def layer(stream=None):
        q, s, h = B.prm_rmsnorm_q8(x, w, EPS, residual=r, stream=stream)
        y = B.prm_matmul_q8(q, s, W8, sw, stream=stream)
        gr, sr, gc, sc = B.prm_quantize_q8(y, by_cols=True, fold_cols=sw, fold_rows=s, stream=stream)
        gy = B.prm_matmul_q8(gr, sr, W8.t(), None, stream=stream)
        return (y, B.prm_matmul_q8(q.t(), None, gc, sc, stream=stream)) + tuple(
            B.prm_rmsnorm_q8_backward(gy, h, w, EPS, grad_h=h, stream=stream))

    want = layer()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = layer(side)
    side.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer()
    x.add_(1)
    graph.replay()
    torch.cuda.synchronize()
    want = layer()
    assert all(torch.equal(u, v) for u, v in zip(out, want))


@pytest.mark.gpu
def test_refusals():
    x = torch.zeros(4, 32, device="cuda", dtype=torch.bfloat16)
    w = torch.ones(32, device="cuda")
    q = torch.zeros(4, 32, device="cuda", dtype=torch.int8)
    with pytest.raises(ValueError):
        B.prm_rmsnorm_q8(x, w, EPS, format="int4")
    with pytest.raises(TypeError):
        B.prm_rmsnorm_q8(x.half(), w, EPS)
    with pytest.raises(ValueError):
        B.prm_rmsnorm_q8(x, w[:31], EPS)
    with pytest.raises(TypeError):
        B.prm_rmsnorm_q8(x, w.double(), EPS)
    with pytest.raises(TypeError):
        B.prm_rmsnorm_q8(x, w, EPS, residual=x.float())
    with pytest.raises(ValueError):
        B.prm_rmsnorm_q8(x, w, EPS, residual=x[:3])
    with pytest.raises(ValueError):
        B.prm_rmsnorm_q8(x[0], w, EPS)
    with pytest.raises(ValueError):
        B.prm_rmsnorm_q8(x.cpu(), w, EPS)
    with pytest.raises(B.PrmError):
        B.prm_rmsnorm_q8(x, w, -1.0)
    with pytest.raises(B.PrmError):
        B.prm_rmsnorm_q8(x[:, :0], w[:0], EPS)
    with pytest.raises(ValueError):
        B.prm_rmsnorm_q8_backward(x[:2], x, w, EPS)
    with pytest.raises(TypeError):
        B.prm_rmsnorm_q8_backward(x.float(), x, w, EPS)
    with pytest.raises(ValueError):
        B.prm_quantize_q8(x, by_rows=False)
    with pytest.raises(ValueError):
        B.prm_quantize_q8(x, fold_cols=w[:4])
    with pytest.raises(TypeError):
        B.prm_quantize_q8(x, fold_cols=w.to(torch.bfloat16))
    with pytest.raises(ValueError):
        B.prm_matmul_q8(q, None, q, None)
    with pytest.raises(TypeError):
        B.prm_matmul_q8(q, None, q.t().float(), None)
    with pytest.raises(TypeError):
        B.prm_matmul_q8(q, None, q.t().view(torch.float8_e4m3fn), None)
    with pytest.raises(TypeError):
        B.prm_matmul_q8(q, None, q.t(), None, out_dtype=torch.float16)
    with pytest.raises(ValueError):
        B.prm_matmul_q8(q, w, q.t(), None)
    with pytest.raises(ValueError):
        B.prm_matmul_q8(q, None, q.t(), None, out=torch.zeros(4, 5, device="cuda"))
    with pytest.raises(ValueError):
        B.prm_matmul_q8(q, None, q.t(), None, out=torch.zeros(4, 4, device="cuda").t())


def test_codes_of_refusals_without_a_device():
    """Arguments are checked before anything touches the device."""
    L = B.lib()
    P = 1 << 20                     # an address that is never read
    norm = dict(x=P, ldx=64, r=P, ldr=64, w=P, rows=4, cols=64, io=0, wf=0, eps=1e-6, fmt=0, h=P, ldh=64, q=P, ldq=64,
                s=P, stream=None)
    back = dict(gy=P, ldgy=64, h=P, ldh=64, w=P, gh=P, ldgh=64, rows=4, cols=64, io=0, wf=0, eps=1e-6, gx=P, ldgx=64,
                gw=P, scratch=P, nbytes=4 * 64 * 4, stream=None)
    quant = dict(x=P, ldx=64, rows=4, cols=64, io=0, fmt=0, fr=P, fc=P, qr=P, ldqr=64, sr=P, qc=P, ldqc=64, sc=P,
                 scratch=P, nbytes=256, stream=None)
    mul = dict(a=P, lda=64, at=0, sa=P, b=P, ldb=64, bt=0, sb=P, m=4, k=64, n=64, fmt=0, out=P, ldo=64, f32=0, stream=None)
    for fn, args, wrong in (
        (L.prm_rmsnorm_q8, norm, [(B.PRM_ERR_ARG, dict(fmt=2)), (B.PRM_ERR_ARG, dict(eps=-1.0)), (B.PRM_ERR_ARG, dict(eps=float("nan"))),
                                  (B.PRM_ERR_ARG, dict(x=None)), (B.PRM_ERR_ARG, dict(h=None)), (B.PRM_ERR_ARG, dict(rows=-1)),
                                  (B.PRM_ERR_SHAPE, dict(cols=0)), (B.PRM_ERR_SHAPE, dict(ldq=63)), (B.PRM_ERR_SHAPE, dict(ldh=63)),
                                  (B.PRM_ERR_SHAPE, dict(ldx=-1)), (B.PRM_ERR_SHAPE, dict(rows=1 << 31)), (B.PRM_ERR_ALIGN, dict(x=P + 1)),
                                  (B.PRM_ERR_ALIGN, dict(s=P + 2)), (B.PRM_OK, dict(rows=0, x=None))]),
        (L.prm_rmsnorm_q8_backward, back, [(B.PRM_ERR_ARG, dict(gw=None)), (B.PRM_ERR_ARG, dict(gy=None)), (B.PRM_ERR_ARG, dict(scratch=None)),
                                           (B.PRM_ERR_SHAPE, dict(cols=0)), (B.PRM_ERR_SHAPE, dict(ldgx=63)),
                                           (B.PRM_ERR_ALIGN, dict(gw=P + 1)), (B.PRM_ERR_ALIGN, dict(scratch=P + 8)),
                                           (B.PRM_ERR_WORKSPACE, dict(nbytes=16))]),
        (L.prm_quantize_q8, quant, [(B.PRM_ERR_ARG, dict(fmt=-1)), (B.PRM_ERR_ARG, dict(qr=None, qc=None)), (B.PRM_ERR_ARG, dict(sr=None)),
                                    (B.PRM_ERR_ARG, dict(x=None)), (B.PRM_ERR_SHAPE, dict(cols=0)), (B.PRM_ERR_SHAPE, dict(ldqc=8)),
                                    (B.PRM_ERR_ALIGN, dict(fc=P + 1)), (B.PRM_ERR_WORKSPACE, dict(nbytes=255)),
                                    (B.PRM_ERR_WORKSPACE, dict(scratch=None))]),
        (L.prm_matmul_q8, mul, [(B.PRM_ERR_ARG, dict(fmt=7)), (B.PRM_ERR_ARG, dict(out=None)), (B.PRM_ERR_ARG, dict(a=None)),
                                (B.PRM_ERR_SHAPE, dict(m=-1)), (B.PRM_ERR_SHAPE, dict(ldo=63)), (B.PRM_ERR_SHAPE, dict(lda=48)),
                                (B.PRM_ERR_SHAPE, dict(k=1047553, lda=1047568)), (B.PRM_ERR_ALIGN, dict(a=P + 8)),
                                (B.PRM_ERR_ALIGN, dict(ldb=72)), (B.PRM_ERR_ALIGN, dict(out=P + 1)), (B.PRM_OK, dict(m=0, a=None))]),
    ):
        for code, change in wrong:
            assert fn(*{**args, **change}.values()) == code, (fn.__name__, change)
    assert L.prm_rmsnorm_q8_scratch_bytes(0, 5) == 0 and L.prm_rmsnorm_q8_scratch_bytes(4, 64) == 1024
