"""The operators of the 8-bit layer against their definitions in 64 bits: sizes from one row and one column on, rows that no vector
divides, views into wider matrices, both float types and every block size, rows of zeros and rows that are not finite.

Tolerances follow from the arithmetic: u = 2^-24 is the unit roundoff of fp32 (24 significant bits), b = 2^-8 that of bf16 (8); a code may be off by its rounding
(0.5) and by the roundings in front of it; a sum of n products is off by at most (roundings of a term + n) u of the sum of their
magnitudes."""
import math

import pytest
import torch

import paper_2604_06836_amd as stq

pytestmark = pytest.mark.gpu

U, B = 2.0 ** -24, 2.0 ** -8
LEAST = 2.0 ** -100
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
KIND = {torch.float32: stq.STQ_F32, torch.bfloat16: stq.STQ_BF16, torch.int8: stq.STQ_Q8}


@pytest.fixture(scope="module")
def ctx():
    c = stq.Context(0, 4)
    yield c
    torch.cuda.synchronize()
    c.close()


def stream():
    return torch.cuda.current_stream().cuda_stream


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


class Buffer:
    """A rows x cols view at an odd place of a wider matrix, whose other elements must stay as they are."""

    def __init__(self, rows, cols, dtype, pad=0, value=None):
        self.whole = torch.full((rows, cols + pad), 77, dtype=dtype, device="cuda")
        self.at = 1 if pad else 0
        self.t = self.whole[:, self.at:self.at + cols]
        if value is not None:
            self.t.copy_(value)
        self.pad = pad

    def mat(self, scales=None, block=0):
        return matrix(self.t, scales, block)

    def untouched(self):
        rest = torch.cat([self.whole[:, :self.at], self.whole[:, self.at + self.t.shape[1]:]], 1)
        return bool((rest == 77).all())


def matrix(t, scales=None, block=0):
    return stq.make_matrix(t.data_ptr(), t.shape[0], t.shape[1], KIND[t.dtype], stride=max(t.stride(0), t.shape[1]),
                           scales=None if scales is None else scales.data_ptr(), block=block)


class Codes:
    def __init__(self, rows, cols, block=0, pad=0):
        self.block = block
        self.q = Buffer(rows, cols, torch.int8, pad)
        self.s = torch.full((rows, -(-cols // block) if block else 1), 55.0, device="cuda")
        self.mat = self.q.mat(self.s, block)

    def each_scale(self):
        width = self.block or self.q.t.shape[1]
        at = torch.arange(self.q.t.shape[1], device="cuda") // width
        return self.s.double()[:, at]

    def value(self):
        return self.q.t.double() * self.each_scale()


def filled(g, rows, cols, block=0, pad=0, size=1.0):
    """Codes of random values (in the state that the library's own conversion would leave them)."""
    c = Codes(rows, cols, block, pad)
    c.q.t.copy_(torch.randint(-127, 128, (rows, cols), device="cuda", generator=g).to(torch.int8))
    c.s.copy_(size * torch.exp(0.5 * torch.randn(c.s.shape, device="cuda", generator=g)) / 127)
    return c


def group_max(v, block):
    width = block or v.shape[1]
    return torch.stack([p.abs().amax(1) for p in v.split(width, 1)], 1)


def check_codes(codes, v, roundings, scale_of_rows=None):
    """codes hold v (64 bits): scales within their roundings, every code the nearest but for the roundings in front of it."""
    a = group_max(v, codes.block).clamp_min(LEAST)
    rows = 1.0 if scale_of_rows is None else scale_of_rows[:, None]
    scale = a / 127 * rows
    assert ((codes.s.double() - scale).abs() <= (roundings + 4) * U * scale).all()
    width = codes.block or v.shape[1]
    at = torch.arange(v.shape[1], device="cuda") // width
    exact = v * 127 / a[:, at]
    off = (codes.q.t.double() - exact).abs().max().item()
    assert off <= 0.5 + 127 * (2 * roundings + 4) * U, off
    assert codes.q.untouched()


def values(g, rows, cols, dtype, zero_row=True):
    v = torch.randn(rows, cols, device="cuda", generator=g) * torch.exp(torch.randn(rows, 1, device="cuda", generator=g))
    if zero_row and rows > 2:
        v[1] = 0
    return v.to(dtype)


SIZES = [(1, 1), (1, 4096), (2, 7), (5, 8), (3, 63), (300, 64), (257, 100), (4, 1023), (9, 1024), (7, 1025), (3, 1600), (33, 4096), (2, 4099),
         (3, 8191), (2, 11008), (2, 16384), (2, 16385), (3, 40001)]


# ------------------------------------------------------------------------------------------------ conversion
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("block,pad", [(0, 0), (64, 0), (128, 3), (256, 5)])
@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_conversion_and_back(ctx, rows, cols, block, pad, kind):
    x = Buffer(rows, cols, TYPES[kind], pad, values(gen(rows + cols), rows, cols, TYPES[kind]))
    c = Codes(rows, cols, block, pad)
    ctx.quantize_rows(x.mat(), c.mat, stream())
    check_codes(c, x.t.double(), 1)
    for to in TYPES.values():
        back = Buffer(rows, cols, to, pad)
        ctx.dequantize_rows(c.mat, back.mat(), stream())
        width = block or cols
        at = torch.arange(cols, device="cuda") // width
        assert torch.equal(back.t, (c.q.t.float() * c.s[:, at]).to(to)) and back.untouched()


def test_extremes_of_the_conversion(ctx):
    big, tiny = 3.4028234663852886e38, 1.0e-45
    x = torch.zeros(6, 130, device="cuda")
    x[0, 5], x[1, 7], x[1, 3], x[2, 129], x[3, 0], x[4, 1] = big, big, -big, tiny, 1e-20, -1e-35
    c = Codes(6, 130, 64)
    ctx.quantize_rows(matrix(x), c.mat, stream())
    check_codes(c, x.double(), 1)
    assert (c.q.t[5] == 0).all() and torch.isfinite(c.s).all() and (c.s > 0).all()


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_what_is_not_finite_makes_its_group_nan(ctx, bad, kind):
    x = values(gen(3), 5, 300, TYPES[kind])
    x[2, 130] = bad
    for block in (0, 64, 128, 256):
        c = Codes(5, 300, block)
        ctx.quantize_rows(matrix(x), c.mat, stream())
        width = block or 300
        hit = torch.zeros_like(c.s, dtype=torch.bool)
        hit[2, 130 // width] = True
        assert torch.equal(torch.isnan(c.s), hit)
        assert (c.q.t[2, 130 // width * width:(130 // width + 1) * width] == 0).all()
        assert torch.isfinite(c.s[~hit]).all()
    # through the norm, the activation and the products: the row, and no other
    w = torch.ones(300, device="cuda")
    y, s, rstd = Codes(5, 300), Codes(5, 300, 128), torch.empty(5, device="cuda")
    ctx.rms_norm(matrix(x), None, w.data_ptr(), 1e-6, None, y.mat, s.mat, rstd.data_ptr(), stream())
    row = torch.arange(5, device="cuda") == 2
    assert torch.equal(torch.isnan(y.s[:, 0]), row) and torch.equal(torch.isnan(rstd), row)
    assert torch.equal(torch.isnan(s.s).any(1), row) and (y.q.t[2] == 0).all()
    out, codes = torch.empty(5, 40, device="cuda"), filled(gen(4), 40, 300)
    ctx.matmul(y.mat, codes.mat, matrix(out), stream())
    assert torch.equal(torch.isnan(out), row[:, None].expand(5, 40))
    other = values(gen(5), 5, 300, TYPES[kind])
    for gate, up in ((x, other), (other, x)):
        y = Codes(5, 300)
        ctx.gated_silu(matrix(gate), matrix(up), y.mat, None, None, stream())
        assert torch.equal(torch.isnan(y.s[:, 0]), row) or (bad == -math.inf and gate is x)


# ------------------------------------------------------------------------------------------------ norm
def depth(cols):
    """Additions one behind the other in the sum over a row."""
    threads = 64 if cols <= 1024 else 256 if cols <= 4096 else 512 if cols <= 8192 else 1024
    return 8 * (-(-cols // (8 * threads))) + 6 + threads // 64


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("kind,residual,block,pad", [("bf16", True, 128, 0), ("bf16", False, 0, 1), ("fp32", True, 64, 3), ("fp32", False, 256, 0),
                                                     ("bf16", True, None, 5)])
def test_norm(ctx, rows, cols, kind, residual, block, pad):
    g, dtype, eps = gen(rows * 7 + cols), TYPES[kind], 1e-5
    x = Buffer(rows, cols, dtype, pad, values(g, rows, cols, dtype))
    r = Buffer(rows, cols, dtype, pad, values(g, rows, cols, dtype)) if residual else None
    w = 1 + 0.3 * torch.randn(cols, device="cuda", generator=g)
    total, y = Buffer(rows, cols, dtype, pad), Codes(rows, cols, 0, pad)
    saved = None if block is None else Codes(rows, cols, block, pad)
    rstd = torch.empty(rows, device="cuda")
    before = (x.whole.clone(), r.whole.clone() if r else None)
    ctx.rms_norm(x.mat(), r.mat() if r else None, w.data_ptr(), eps, total.mat(), y.mat, saved.mat if saved else None, rstd.data_ptr(), stream())
    h = (x.t.float() + r.t.float()).to(dtype) if r else x.t
    assert torch.equal(total.t, h) and total.untouched()
    assert torch.equal(x.whole, before[0]) and (r is None or torch.equal(r.whole, before[1]))
    h = h.double()
    want = 1 / torch.sqrt((h * h).mean(1) + eps)
    assert ((rstd.double() - want).abs() <= (depth(cols) + 6) * U * want).all()
    check_codes(y, h * w.double(), 2 + depth(cols), rstd.double())
    if saved:
        check_codes(saved, h, 1)
    # the sum in place of either input, and outputs that are not asked for
    y2 = Codes(rows, cols, 0, pad)
    into = r if r else x
    ctx.rms_norm(x.mat(), r.mat() if r else None, w.data_ptr(), eps, into.mat(), y2.mat, None, None, stream())
    assert torch.equal(into.t.double(), h) and torch.equal(y2.q.t, y.q.t) and torch.equal(y2.s, y.s)
    if not r:
        ctx.rms_norm(x.mat(), None, w.data_ptr(), eps, None, y2.mat, None, None, stream())
        assert torch.equal(y2.q.t, y.q.t) and torch.equal(y2.s, y.s)


def test_norm_of_squares_beyond_fp32(ctx):
    x = torch.ones(3, 64, device="cuda")
    x[1] = 1e30
    y, rstd = Codes(3, 64), torch.empty(3, device="cuda")
    ctx.rms_norm(matrix(x), None, torch.ones(64, device="cuda").data_ptr(), 1e-6, None, y.mat, None, rstd.data_ptr(), stream())
    assert torch.isnan(rstd).tolist() == [False, True, False] and torch.isnan(y.s[:, 0]).tolist() == [False, True, False]


def run_norm_grad(ctx, x, w, rstd, dy, dres, dx, rows, cols):
    dw = torch.full((cols,), 9.0, device="cuda")
    n = stq.rms_norm_grad_bytes(rows, cols)
    work = torch.full((max(n // 4, 1) + 4,), 88.0, device="cuda")
    ctx.rms_norm_grad(x, w.data_ptr(), rstd.data_ptr(), dy, dres, dx, dw.data_ptr(), work.data_ptr(), n, stream())
    assert (work[max(n // 4, 1):] == 88.0).all()
    return dw


@pytest.mark.parametrize("rows,cols", SIZES + [(2200, 96), (1500, 1100)])
@pytest.mark.parametrize("kept,kind,dres,block,pad", [("q8", "bf16", True, 64, 0), ("q8", "fp32", False, 128, 3), ("bf16", "bf16", True, 0, 1),
                                                      ("fp32", "fp32", True, 0, 0), ("q8", "bf16", False, 0, 5), ("q8", "fp32", True, 256, 0)])
def test_norm_gradients(ctx, rows, cols, kept, kind, dres, block, pad):
    g, dtype = gen(rows * 3 + cols), TYPES[kind]
    if kept == "q8":
        c = filled(g, rows, cols, block, pad)
        x, xmat = c.value(), c.mat
    else:
        b = Buffer(rows, cols, TYPES[kept], pad, values(g, rows, cols, TYPES[kept]))
        x, xmat = b.t.double(), b.mat()
    w = 1 + 0.3 * torch.randn(cols, device="cuda", generator=g)
    rstd = (1 / torch.sqrt((x * x).mean(1) + 1e-5)).float()
    dy = Buffer(rows, cols, dtype, pad, values(g, rows, cols, dtype))
    dr = Buffer(rows, cols, dtype, pad, values(g, rows, cols, dtype)) if dres else None
    dx = Buffer(rows, cols, dtype, pad)
    dw = run_norm_grad(ctx, xmat, w, rstd, dy.mat(), dr.mat() if dr else None, dx.mat(), rows, cols)
    d, n = dy.t.double(), x * rstd.double()[:, None]
    u = d * w.double()
    mean, mag = (u * n).mean(1, keepdim=True), (u * n).abs().mean(1, keepdim=True)
    r = rstd.double()[:, None]
    want = r * (u - n * mean) + (dr.t.double() if dr else 0)
    size = r * (u.abs() + n.abs() * mag) + (dr.t.double().abs() if dr else 0)
    tol = (depth(cols) + 12) * U * size + (B * want.abs() if kind == "bf16" else 0)
    assert ((dx.t.double() - want).abs() <= tol).all() and dx.untouched()
    wanted = (d * n).sum(0)
    assert ((dw.double() - wanted).abs() <= (rows + 8) * U * (d * n).abs().sum(0) + 1e-37).all()
    # in place of dy, and the same bits again
    dw2 = run_norm_grad(ctx, xmat, w, rstd, dy.mat(), dr.mat() if dr else None, dy.mat(), rows, cols)
    assert torch.equal(dy.t, dx.t) and torch.equal(dw2, dw)


def test_norm_gradients_against_differences(ctx):
    rows, cols, eps, step = 3, 37, 1e-3, 1e-4
    g = gen(1)
    x, w, dy = torch.randn(rows, cols, device="cuda", generator=g), torch.rand(cols, device="cuda", generator=g) + 0.5, torch.randn(rows, cols, device="cuda", generator=g)

    def loss(x, w):
        return (x / torch.sqrt((x * x).mean(1, keepdim=True) + eps) * w * dy.double()).sum()

    x64, w64 = x.double(), w.double()
    rstd = (1 / torch.sqrt((x64 * x64).mean(1) + eps)).float()
    dx = torch.empty_like(x)
    dw = run_norm_grad(ctx, matrix(x), w, rstd, matrix(dy), None, matrix(dx), rows, cols)
    for i in range(rows):
        for j in range(0, cols, 5):
            e = torch.zeros_like(x64)
            e[i, j] = step
            assert abs((loss(x64 + e, w64) - loss(x64 - e, w64)).item() / (2 * step) - dx[i, j].item()) < 1e-4
    for j in range(0, cols, 3):
        e = torch.zeros_like(w64)
        e[j] = step
        assert abs((loss(x64, w64 + e) - loss(x64, w64 - e)).item() / (2 * step) - dw[j].item()) < 1e-4


# ------------------------------------------------------------------------------------------------ gated activation
def silu(g):
    return g * torch.sigmoid(g)


def sigma_error(g):
    """Relative error of sigmoid and silu in fp32: the exponential's argument carries its rounding into the result."""
    return (2 * g.abs() + 10) * U


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("kind,block,pad", [("bf16", 128, 0), ("bf16", 0, 1), ("fp32", 64, 3), ("fp32", 256, 0), ("bf16", None, 5)])
def test_gated(ctx, rows, cols, kind, block, pad):
    g, dtype = gen(rows * 11 + cols), TYPES[kind]
    both = Buffer(rows, 2 * cols, dtype, pad, values(g, rows, 2 * cols, dtype))
    gate, up = both.t[:, :cols], both.t[:, cols:]
    y = Codes(rows, cols, 0, pad)
    kept = [None, None] if block is None else [Codes(rows, cols, block, pad), Codes(rows, cols, block, pad)]
    ctx.gated_silu(matrix(gate), matrix(up), y.mat, *(k.mat if k else None for k in kept), stream())
    v = silu(gate.double()) * up.double()
    check_codes(y, v, 4 + (sigma_error(gate.double()) / U).max().item())
    for k, t in zip(kept, (gate, up)):
        if k:
            check_codes(k, t.double(), 1)


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("kept,kind,block,pad", [("q8", "bf16", 64, 0), ("q8", "fp32", 128, 3), ("bf16", "bf16", 0, 1), ("fp32", "fp32", 0, 0),
                                                 ("q8", "bf16", 0, 5), ("q8", "fp32", 256, 0)])
def test_gated_gradients(ctx, rows, cols, kept, kind, block, pad):
    g, dtype = gen(rows * 13 + cols), TYPES[kind]
    if kept == "q8":
        cg, cu = filled(g, rows, cols, block, pad, size=3.0), filled(g, rows, cols, block, pad)
        gate, up, mg, mu = cg.value(), cu.value(), cg.mat, cu.mat
    else:
        bg, bu = (Buffer(rows, cols, TYPES[kept], pad, values(g, rows, cols, TYPES[kept])) for _ in range(2))
        gate, up, mg, mu = bg.t.double(), bu.t.double(), bg.mat(), bu.mat()
    dy = Buffer(rows, cols, dtype, pad, values(g, rows, cols, dtype))
    both = Buffer(rows, 2 * cols, dtype, pad)
    ctx.gated_silu_grad(mg, mu, dy.mat(), matrix(both.t[:, :cols]), matrix(both.t[:, cols:]), stream())
    d, s = dy.t.double(), torch.sigmoid(gate)
    slope = s + gate * s * (1 - s)
    want = torch.cat([d * up * slope, d * gate * s], 1)
    err = sigma_error(gate) + 6 * U
    # 1 + gate (1 - s): each of the terms is off by its own size
    size = torch.cat([(d * up).abs() * s * (1 + 2 * gate.abs()) * err, (d * gate).abs() * s * err], 1)
    tol = size + (B * want.abs() if kind == "bf16" else 0) + 1e-37
    assert ((both.t.double() - want).abs() <= tol).all() and both.untouched()
    ctx.gated_silu_grad(mg, mu, dy.mat(), dy.mat(), matrix(both.t[:, cols:]), stream())
    assert torch.equal(dy.t, both.t[:, :cols])


def test_gated_at_the_ends(ctx):
    """Gates so large that the exponential overflows or vanishes."""
    gate = torch.tensor([[-1e30, -200.0, -100.0, -88.0, 88.0, 100.0, 200.0, 1e30]], device="cuda")
    up, dy = torch.ones_like(gate), torch.ones_like(gate)
    y, dg, du = Codes(1, 8), torch.empty_like(gate), torch.empty_like(gate)
    ctx.gated_silu(matrix(gate), matrix(up), y.mat, None, None, stream())
    assert y.q.t[0].tolist() == [0, 0, 0, 0, 0, 0, 0, 127]
    ctx.gated_silu_grad(matrix(gate), matrix(up), matrix(dy), matrix(dg), matrix(du), stream())
    assert dg[0].abs().max() <= 1 and torch.isfinite(du).all()
    assert torch.allclose(dg[0, 4:], torch.ones(4, device="cuda")) and dg[0, :4].abs().max() < 1e-30


def test_gated_gradients_against_differences(ctx):
    g, step = gen(2), 1e-4
    gate, up, dy = (torch.randn(4, 33, device="cuda", generator=g) for _ in range(3))
    dg, du = torch.empty_like(gate), torch.empty_like(gate)
    ctx.gated_silu_grad(matrix(gate), matrix(up), matrix(dy), matrix(dg), matrix(du), stream())

    def f(a, b):
        return silu(a) * b * dy.double()

    a, b = gate.double(), up.double()
    assert ((f(a + step, b) - f(a - step, b)) / (2 * step) - dg.double()).abs().max() < 1e-4
    assert ((f(a, b + step) - f(a, b - step)) / (2 * step) - du.double()).abs().max() < 1e-4


# ------------------------------------------------------------------------------------------------ products
PRODUCTS = [(1, 1, 1), (1, 64, 64), (1, 1000, 4096), (1, 4096, 11008), (2, 129, 100), (3, 33, 4097), (7, 768, 768), (8, 257, 15), (15, 65, 129),
            (16, 128, 1024), (17, 300, 200), (33, 1000, 768), (64, 96, 4096), (65, 70, 80), (128, 128, 128), (129, 257, 191), (300, 1000, 784),
            (512, 512, 2048), (1000, 520, 1111), (2048, 1536, 512), (5001, 320, 64)]


@pytest.mark.parametrize("m,n,k", PRODUCTS)
@pytest.mark.parametrize("kind,pad", [("bf16", 0), ("fp32", 0), ("bf16", 16), ("fp32", 3)])
def test_product(ctx, m, n, k, kind, pad):
    g = gen(m + n + k)
    x, w, out = filled(g, m, k, 0, pad), filled(g, n, k, 0, pad), Buffer(m, n, TYPES[kind], pad)
    x.q.t[0] = 127
    w.q.t[0] = -127
    ctx.matmul(x.mat, w.mat, out.mat(), stream())
    want = (x.q.t.double() @ w.q.t.double().t()) * x.s.double() * w.s.double().t()
    tol = (4 * U + (B if kind == "bf16" else 0)) * want.abs()
    assert ((out.t.double() - want).abs() <= tol).all() and out.untouched()


def test_product_at_the_largest_inner_size(ctx):
    k = stq.STQ_MAX_INNER
    x, w = filled(gen(1), 3, k), filled(gen(2), 5, k)
    x.q.t[0], w.q.t[0], w.q.t[1] = -128, -128, 127
    out = torch.empty(3, 5, device="cuda")
    ctx.matmul(x.mat, w.mat, matrix(out), stream())
    want = (x.q.t.double() @ w.q.t.double().t()) * x.s.double() * w.s.double().t()
    assert ((out.double() - want).abs() <= 4 * U * want.abs()).all()


GRADS = [(1, 1, 1), (1, 64, 64), (2, 129, 100), (16, 40, 1024), (33, 1000, 768), (65, 70, 80), (128, 128, 128), (129, 257, 191), (300, 1000, 784),
         (1000, 520, 1111), (512, 1024, 2048), (5001, 320, 64), (20000, 64, 72)]


def of_terms(out, terms):
    """What a term dy * s * q and the output may be off by: dy * s in fp32 and then bf16, or two of them."""
    return (U + B, B) if terms == 1 else (U + B * B, U)


def gradient(g, rows, cols, dtype, pad):
    v = 1e-3 * torch.randn(rows, cols, device="cuda", generator=g) * torch.exp(torch.randn(rows, 1, device="cuda", generator=g))
    if rows > 4:
        v[3] = 0
    return Buffer(rows, cols, dtype, pad, v.to(dtype))


@pytest.mark.parametrize("m,n,k", GRADS)
@pytest.mark.parametrize("of,kind,pad", [("bf16", "bf16", 0), ("bf16", "fp32", 0), ("fp32", "bf16", 1), ("fp32", "fp32", 0), ("bf16", "bf16", 8),
                                         ("bf16", "bf16", 3)])
def test_gradient_of_input(ctx, m, n, k, of, kind, pad):
    g = gen(m + n + k)
    dy, w, dx = gradient(g, m, n, TYPES[of], pad), filled(g, n, k, 0, pad), Buffer(m, k, TYPES[kind], pad)
    ctx.matmul_grad_input(dy.mat(), w.mat, dx.mat(), stream())
    d, v = dy.t.double(), w.value()
    want, size = d @ v, d.abs() @ v.abs()
    term, last = of_terms(kind, 2 if kind == "fp32" else 1)
    assert ((dx.t.double() - want).abs() <= (term + n * U) * size + last * want.abs() + 1e-37).all() and dx.untouched()


@pytest.mark.parametrize("m,n,k", GRADS)
@pytest.mark.parametrize("of,kind,pad", [("bf16", "bf16", 0), ("bf16", "fp32", 0), ("fp32", "bf16", 1), ("fp32", "fp32", 0), ("bf16", "bf16", 8),
                                         ("bf16", "bf16", 3)])
def test_gradient_of_weight(ctx, m, n, k, of, kind, pad):
    g = gen(m + n + k)
    dy, x, dw = gradient(g, m, n, TYPES[of], pad), filled(g, m, k, 0, pad), Buffer(n, k, TYPES[kind], pad)
    need = stq.matmul_grad_weight_bytes(m, n, k)
    work = torch.full((need // 4 + 4,), 88.0, device="cuda")

    def run(out):
        ctx.matmul_grad_weight(dy.mat(), x.mat, out.mat(), work.data_ptr(), need, stream())
    run(dw)
    assert (work[need // 4:] == 88.0).all()
    d, v = dy.t.double(), x.value()
    want, size = d.t() @ v, d.abs().t() @ v.abs()
    term, last = of_terms(kind, 2 if kind == "fp32" else 1)
    assert ((dw.t.double() - want).abs() <= (term + m * U) * size + last * want.abs() + 1e-37).all() and dw.untouched()
    again = Buffer(n, k, TYPES[kind], pad)
    run(again)
    assert torch.equal(again.t, dw.t)


def test_gradients_against_differences(ctx):
    """<dy, x w> by differences in the values of x and w."""
    g = gen(9)
    x, w, dy = filled(g, 9, 40), filled(g, 11, 40), gradient(g, 9, 11, torch.float32, 0)
    dx, dw = torch.empty(9, 40, device="cuda"), torch.empty(11, 40, device="cuda")
    ctx.matmul_grad_input(dy.mat(), w.mat, matrix(dx), stream())
    need = stq.matmul_grad_weight_bytes(9, 11, 40)
    work = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    ctx.matmul_grad_weight(dy.mat(), x.mat, matrix(dw), work.data_ptr(), need, stream())
    a, b, d = x.value(), w.value(), dy.t.double()

    def loss(a, b):
        return ((a @ b.t()) * d).sum()
    scale = (d.abs().sum() * b.abs().max() * a.abs().max()).item()
    for i, j in [(0, 0), (4, 17), (8, 39), (2, 5)]:
        e = torch.zeros_like(a)
        e[i, j] = 0.5
        assert abs((loss(a + e, b) - loss(a - e, b)).item() - dx[i, j].item()) < 1e-5 * scale
        e = torch.zeros_like(b)
        e[i, j] = 0.5
        assert abs((loss(a, b + e) - loss(a, b - e)).item() - dw[i, j].item()) < 1e-5 * scale


# ------------------------------------------------------------------------------------------------ no rows, streams, graphs, far offsets
def test_no_rows(ctx):
    x, c = torch.empty(0, 40, device="cuda"), Codes(0, 40)
    w = torch.ones(40, device="cuda")
    ctx.quantize_rows(matrix(x), c.mat, stream())
    ctx.dequantize_rows(c.mat, matrix(x), stream())
    ctx.rms_norm(matrix(x), None, w.data_ptr(), 1e-6, None, c.mat, None, None, stream())
    dw = run_norm_grad(ctx, matrix(x), w, torch.empty(0, device="cuda"), matrix(x), None, matrix(x), 0, 40)
    assert (dw == 0).all()
    ctx.gated_silu(matrix(x), matrix(x), c.mat, None, None, stream())
    ctx.gated_silu_grad(matrix(x), matrix(x), matrix(x), matrix(x), matrix(x), stream())
    weights, dy = filled(gen(1), 24, 40), torch.empty(0, 24, device="cuda")
    ctx.matmul(c.mat, weights.mat, matrix(dy), stream())
    ctx.matmul_grad_input(matrix(dy), weights.mat, matrix(x), stream())
    dw = torch.full((24, 40), 3.0, device="cuda")
    assert stq.matmul_grad_weight_bytes(0, 24, 40) == 0
    ctx.matmul_grad_weight(matrix(dy), c.mat, matrix(dw), None, 0, stream())
    assert (dw == 0).all()


def test_calls_on_two_streams_at_once(ctx):
    """One context, no buffer of its own: the calls of two streams do not meet."""
    inputs = [(filled(gen(s), 700, 512), filled(gen(s + 1), 900, 512)) for s in (1, 5)]
    outs = [torch.empty(700, 900, device="cuda") for _ in inputs]
    streams = [torch.cuda.Stream() for _ in inputs]
    torch.cuda.synchronize()
    for _ in range(10):
        for (x, w), out, s in zip(inputs, outs, streams):
            ctx.matmul(x.mat, w.mat, matrix(out), s.cuda_stream)
    torch.cuda.synchronize()
    for (x, w), out in zip(inputs, outs):
        want = (x.q.t.double() @ w.q.t.double().t()) * x.s.double() * w.s.double().t()
        assert ((out.double() - want).abs() <= 4 * U * want.abs()).all()


def test_recorded_layer(ctx):
    """Forward and backward of a layer in a graph, replayed on other inputs, against the calls themselves."""
    rows, d, f = 192, 256, 320
    g = gen(7)
    x, w = torch.empty(rows, d, dtype=torch.bfloat16, device="cuda"), torch.ones(d, device="cuda")
    dy = torch.empty(rows, f, dtype=torch.bfloat16, device="cuda")
    weights = filled(g, f, d)

    def make():
        return dict(y=Codes(rows, d), saved=Codes(rows, d, 128), rstd=torch.empty(rows, device="cuda"), out=torch.empty(rows, f, dtype=torch.bfloat16, device="cuda"),
                    dn=torch.empty(rows, d, dtype=torch.bfloat16, device="cuda"), dw=torch.empty(f, d, device="cuda"), dx=torch.empty(rows, d, dtype=torch.bfloat16, device="cuda"),
                    dweight=torch.empty(d, device="cuda"), work=torch.empty(max(stq.rms_norm_grad_bytes(rows, d), stq.matmul_grad_weight_bytes(rows, f, d)), dtype=torch.uint8, device="cuda"))

    def layer(b):
        s, size = stream(), b["work"].numel()
        ctx.rms_norm(matrix(x), None, w.data_ptr(), 1e-6, None, b["y"].mat, b["saved"].mat, b["rstd"].data_ptr(), s)
        ctx.matmul(b["y"].mat, weights.mat, matrix(b["out"]), s)
        ctx.matmul_grad_input(matrix(dy), weights.mat, matrix(b["dn"]), s)
        ctx.matmul_grad_weight(matrix(dy), b["y"].mat, matrix(b["dw"]), b["work"].data_ptr(), size, s)
        ctx.rms_norm_grad(b["saved"].mat, w.data_ptr(), b["rstd"].data_ptr(), matrix(b["dn"]), None, matrix(b["dx"]), b["dweight"].data_ptr(),
                          b["work"].data_ptr(), size, s)
    recorded, eager = make(), make()
    x.copy_(torch.randn(rows, d, device="cuda", generator=g))
    dy.copy_(1e-3 * torch.randn(rows, f, device="cuda", generator=g))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(recorded)
    for _ in range(4):
        x.copy_(torch.randn(rows, d, device="cuda", generator=g))
        dy.copy_(1e-3 * torch.randn(rows, f, device="cuda", generator=g))
        graph.replay()
        layer(eager)
        torch.cuda.synchronize()
        for name in ("out", "dn", "dw", "dx", "dweight", "rstd"):
            assert torch.equal(recorded[name], eager[name]), name
        assert torch.equal(recorded["y"].q.t, eager["y"].q.t)


def test_rows_far_apart(ctx):
    """Offsets beyond 32 bits: a few rows of a view whose stride is 2^30 elements and more."""
    stride, rows, cols = (1 << 30) + 24, 6, 200
    big = torch.empty(rows * stride, dtype=torch.int8, device="cuda")
    q = big.as_strided((rows, cols), (stride, 1))
    src = filled(gen(3), rows, cols)
    q.copy_(src.q.t)
    far = stq.make_matrix(big.data_ptr(), rows, cols, stq.STQ_Q8, stride=stride, scales=src.s.data_ptr())
    w, dy = filled(gen(4), 33, cols), gradient(gen(5), rows, 33, torch.bfloat16, 0)
    out, want = torch.empty(rows, 33, device="cuda"), torch.empty(rows, 33, device="cuda")
    ctx.matmul(far, w.mat, matrix(out), stream())
    ctx.matmul(src.mat, w.mat, matrix(want), stream())
    assert torch.equal(out, want)
    ctx.matmul(w.mat, far, matrix(a := torch.empty(33, rows, device="cuda")), stream())
    assert torch.allclose(a, want.t(), rtol=1e-6, atol=0)
    dw, dw2 = torch.empty(33, cols, device="cuda"), torch.empty(33, cols, device="cuda")
    need = stq.matmul_grad_weight_bytes(rows, 33, cols)
    work = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    ctx.matmul_grad_weight(dy.mat(), far, matrix(dw), work.data_ptr(), need, stream())
    ctx.matmul_grad_weight(dy.mat(), src.mat, matrix(dw2), work.data_ptr(), need, stream())
    assert torch.equal(dw, dw2)
    back, back2 = torch.empty(rows, cols, device="cuda"), torch.empty(rows, cols, device="cuda")
    ctx.dequantize_rows(far, matrix(back), stream())
    ctx.dequantize_rows(src.mat, matrix(back2), stream())
    assert torch.equal(back, back2)
    back.mul_(3)
    ctx.quantize_rows(matrix(back), far, stream())
    c = Codes(rows, cols)
    ctx.quantize_rows(matrix(back), c.mat, stream())
    assert torch.equal(q, c.q.t)
    del big, q


# ------------------------------------------------------------------------------------------------ refusals
def code_of(call):
    with pytest.raises(stq.StqError) as e:
        call()
    return e.value.code


def test_refusals(ctx):
    f, h = torch.empty(8, 64, device="cuda"), torch.empty(8, 64, dtype=torch.bfloat16, device="cuda")
    c, blocked, w = Codes(8, 64), Codes(8, 64, 64), torch.ones(64, device="cuda")
    null, s = stq.make_matrix(None, 8, 64, stq.STQ_F32), stream()

    def odd(m, **change):
        r = stq.make_matrix(m.data, m.rows, m.cols, m.dtype, stride=m.stride, scales=m.scales, block=m.block)
        for k, v in change.items():
            setattr(r, k, v)
        return r
    F, H, Q = matrix(f), matrix(h), c.mat
    EINVAL, EALIGN, EBLOCK, ESHAPE, EDTYPE = -1, -2, -4, -9, -10
    assert code_of(lambda: ctx.quantize_rows(None, Q, s)) == EINVAL
    assert code_of(lambda: ctx.quantize_rows(F, None, s)) == EINVAL
    assert code_of(lambda: ctx.quantize_rows(null, Q, s)) == EINVAL
    assert code_of(lambda: ctx.quantize_rows(F, odd(Q, scales=None), s)) == EINVAL
    assert code_of(lambda: ctx.quantize_rows(Q, Q, s)) == EDTYPE
    assert code_of(lambda: ctx.quantize_rows(F, H, s)) == EDTYPE
    assert code_of(lambda: ctx.quantize_rows(odd(F, dtype=7), Q, s)) == EDTYPE
    assert code_of(lambda: ctx.quantize_rows(F, odd(Q, block=32), s)) == EBLOCK
    assert code_of(lambda: ctx.quantize_rows(F, odd(Q, rows=7), s)) == ESHAPE
    assert code_of(lambda: ctx.quantize_rows(odd(F, stride=63), Q, s)) == ESHAPE
    assert code_of(lambda: ctx.quantize_rows(odd(F, cols=0), Q, s)) == ESHAPE
    assert code_of(lambda: ctx.quantize_rows(odd(F, rows=1 << 31), Q, s)) == ESHAPE
    assert code_of(lambda: ctx.quantize_rows(odd(F, stride=1 << 62), Q, s)) == ESHAPE
    assert code_of(lambda: ctx.quantize_rows(odd(F, data=f.data_ptr() + 2), Q, s)) == EALIGN
    assert code_of(lambda: ctx.quantize_rows(odd(H, data=h.data_ptr() + 1), Q, s)) == EALIGN
    assert code_of(lambda: ctx.quantize_rows(F, odd(Q, scales=c.s.data_ptr() + 2), s)) == EALIGN
    assert code_of(lambda: ctx.dequantize_rows(F, F, s)) == EDTYPE
    norm = lambda x=F, r=None, w=w.data_ptr(), eps=1e-6, t=None, y=Q, k=None, rstd=None: code_of(lambda: ctx.rms_norm(x, r, w, eps, t, y, k, rstd, s))  # noqa: E731
    assert norm(r=H) == EDTYPE and norm(t=H) == EDTYPE and norm(y=F) == EDTYPE and norm(k=F) == EDTYPE
    assert norm(y=blocked.mat) == EBLOCK and norm(w=None) == EINVAL and norm(w=w.data_ptr() + 1) == EALIGN
    assert norm(eps=0.0) == EINVAL and norm(eps=math.nan) == EINVAL and norm(eps=math.inf) == EINVAL and norm(rstd=f.data_ptr() + 2) == EALIGN
    need = stq.rms_norm_grad_bytes(8, 64)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    grad = lambda x=Q, dy=F, dr=None, dx=F, dw=w.data_ptr(), wk=work.data_ptr(), n=need: code_of(  # noqa: E731
        lambda: ctx.rms_norm_grad(x, w.data_ptr(), w.data_ptr(), dy, dr, dx, dw, wk, n, s))
    assert grad(n=need - 1) == EINVAL and grad(wk=None) == EINVAL and grad(wk=work.data_ptr() + 4) == EALIGN and grad(dw=None) == EINVAL
    assert grad(dx=H) == EDTYPE and grad(dr=H) == EDTYPE and grad(dy=Q) == EDTYPE and grad(x=odd(Q, cols=63)) == ESHAPE
    assert code_of(lambda: ctx.gated_silu(F, H, Q, None, None, s)) == EDTYPE
    assert code_of(lambda: ctx.gated_silu(F, F, Q, blocked.mat, None, s)) == EINVAL
    assert code_of(lambda: ctx.gated_silu(F, F, Q, blocked.mat, c.mat, s)) == EBLOCK
    assert code_of(lambda: ctx.gated_silu(F, F, blocked.mat, None, None, s)) == EBLOCK
    assert code_of(lambda: ctx.gated_silu_grad(Q, blocked.mat, F, F, F, s)) == EBLOCK
    assert code_of(lambda: ctx.gated_silu_grad(Q, F, F, F, F, s)) == EDTYPE
    assert code_of(lambda: ctx.gated_silu_grad(F, F, F, H, F, s)) == EDTYPE
    out = torch.empty(8, 8, device="cuda")
    assert code_of(lambda: ctx.matmul(blocked.mat, Q, matrix(out), s)) == EBLOCK
    assert code_of(lambda: ctx.matmul(Q, F, matrix(out), s)) == EDTYPE
    assert code_of(lambda: ctx.matmul(Q, odd(Q, cols=60), matrix(out), s)) == ESHAPE
    assert code_of(lambda: ctx.matmul(Q, Q, F, s)) == ESHAPE
    assert code_of(lambda: ctx.matmul(odd(Q, cols=1 << 17, stride=1 << 17), Q, matrix(out), s)) == ESHAPE
    assert code_of(lambda: ctx.matmul_grad_input(matrix(out), Q, H if False else matrix(out), s)) == ESHAPE
    assert code_of(lambda: ctx.matmul_grad_input(Q, Q, F, s)) == EDTYPE
    assert code_of(lambda: ctx.matmul_grad_weight(matrix(out), F, F, None, 0, s)) == EDTYPE
    assert code_of(lambda: ctx.matmul_grad_weight(F, odd(Q, rows=7), F, None, 0, s)) == ESHAPE
    torch.cuda.synchronize()
