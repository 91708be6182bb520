"""The 8-bit layer's operators at the ends of their ranges, against 64 bits."""
import math

import pytest
import torch

import paper_2604_06836_amd as stq
from test_gpu_operators import B, LEAST, TYPES, U, Codes, check_codes, matrix, silu, stream

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = stq.Context(0, 4)
    yield c
    torch.cuda.synchronize()
    c.close()


@pytest.fixture(autouse=True)
def memory_back():
    yield
    torch.cuda.empty_cache()


# ------------------------------------------------------------------------------------------------ gated activation
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [8, 100, 600, 4096, 20000])
@pytest.mark.parametrize("keep", [False, True])
def test_rows_of_large_negative_gates(ctx, dtype, cols, keep):
    """A gate whose exponential passes fp32's range gives 0, also where no other element sets the row's scale: a mask of the type's
    lowest value above all.  Next to that range the quotient is as precise as elsewhere."""
    ends = [-1e30, -1e38, torch.finfo(dtype).min, -89.0, -200.0, -1e4]
    near = [-88.5, -87.5, -87.0, -86.0, -60.0]
    gate = torch.tensor(ends + near, device="cuda")[:, None].expand(-1, cols).contiguous().to(dtype)
    beside = torch.randn(len(ends), cols, device="cuda", generator=torch.Generator("cuda").manual_seed(cols)).to(dtype)
    beside[:, ::2] = gate[:len(ends), ::2]
    gate = torch.cat([gate, beside])
    up = (1 + torch.rand(gate.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(1))).to(dtype)
    up[len(ends):len(ends) + len(near)] *= 1e37  # gates near the end: values of an ordinary size
    y, kept = Codes(len(gate), cols), [Codes(len(gate), cols, 128) if keep else None for _ in range(2)]
    ctx.gated_silu(matrix(gate), matrix(up), y.mat, *(k.mat if k else None for k in kept), stream())
    g = gate.double()
    # roundings: two of the exponential (one unit in the last place), the sum's, the quotient's, the product's
    check_codes(y, torch.where(g < -88.7229, 0.0, silu(g)) * up.double(), 5)
    assert (y.q.t[:len(ends)] == 0).all() and (y.q.t[len(ends)].abs().max() == 127)
    dg, du = torch.empty_like(up), torch.empty_like(up)
    ctx.gated_silu_grad(matrix(gate), matrix(up), matrix(up), matrix(dg), matrix(du), stream())
    assert (dg[:len(ends)] == 0).all() and (du[:len(ends)] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [500, 1000, 4096, 10000, 20000])
def test_codes_of_the_gated_activation(ctx, dtype, cols):
    """Rows of gates of one size each, -80 to 80, so that codes follow the least bits of their exponentials.  In units of 2^-24: y is off by
    the exponential's last place (2), the sum, the quotient and the product, 5; its largest by as much; 1 / a, 127 and the product, 3."""
    g = torch.Generator("cuda").manual_seed(cols)
    gate = torch.linspace(-80, 80, 161, device="cuda")[:, None] + torch.rand(161, cols, device="cuda", generator=g)
    gate, up = gate.to(dtype), torch.randn(161, cols, device="cuda", generator=g).to(dtype)
    y = Codes(161, cols)
    ctx.gated_silu(matrix(gate), matrix(up), y.mat, None, None, stream())
    v = silu(gate.double()) * up.double()
    a = v.abs().amax(1, keepdim=True).clamp_min(LEAST)
    assert ((y.s.double() - a / 127).abs() <= 8 * U * a / 127).all()
    assert ((y.q.t.double() - v * 127 / a).abs() <= 0.5 + 127 * 14 * U).all()


def test_gates_that_are_not_finite(ctx):
    """x / (1 + exp(-x)) of infinities and NaN: none of them has a code."""
    for bad in (math.inf, -math.inf, math.nan):
        gate = torch.ones(3, 64, device="cuda")
        gate[1, 7] = bad
        y = Codes(3, 64)
        ctx.gated_silu(matrix(gate), matrix(torch.ones_like(gate)), y.mat, None, None, stream())
        assert torch.isnan(y.s[:, 0]).tolist() == [False, True, False] and (y.q.t[1] == 0).all()


# ------------------------------------------------------------------------------------------------ conversion
@pytest.mark.parametrize("block", [0, 64])
@pytest.mark.parametrize("size", [2.0 ** -90, 2.0 ** 63, 2.0 ** 64, 2.0 ** 120, 2.0 ** 125, 2.0 ** 126, 2.0 ** 127])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_codes_of_large_numbers(ctx, block, size, dtype):
    """Bit for bit up to fp32's largest numbers, of which 1 / a has 24 bits although it is below fp32's normal ones."""
    x = (torch.rand(300, 128, device="cuda", generator=torch.Generator("cuda").manual_seed(3)) * 3.9 - 1.95).to(dtype)
    x[:, 5], x[:, 100] = 1.95 * torch.rand(300, device="cuda", generator=torch.Generator("cuda").manual_seed(4)), 1.95
    codes, v = Codes(300, 128, block), x.float() * size
    ctx.quantize_rows(matrix(v.to(dtype)), codes.mat, stream())
    assert torch.isfinite(v).all() and torch.equal(v.to(dtype).float(), v)
    width = block or 128
    a = v.view(300, -1, width).abs().amax(2, keepdim=True)
    small = a * 2.0 ** -64 if size > 1 else a
    inv = 127.0 * (1.0 / small)
    q = torch.round(v.view(300, -1, width) * (inv * 2.0 ** -64 if size > 1 else inv))
    assert torch.equal(codes.s, (a * torch.tensor(1 / 127, dtype=torch.float32, device="cuda")).squeeze(2)) and torch.equal(codes.q.t, q.view(300, 128).to(torch.int8))


@pytest.mark.parametrize("cols", [7, 512, 1600, 4096, 20000])
@pytest.mark.parametrize("eps", [1e-5, 0.25, 4.0, 1e10])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_of_nothing_and_little(ctx, cols, eps, dtype):
    """Codes and scales of rows of zeros, of less than 2^-100 and of little more, bit for bit: a = max(max|y|, rstd 2^-100, 2^-100)."""
    x = torch.randn(6, cols, device="cuda", generator=torch.Generator("cuda").manual_seed(cols)).to(dtype)
    x *= torch.tensor([0, 1e-36, 1e-32, 1e-29, 1e-27, 1], device="cuda").to(dtype)[:, None]
    w = torch.linspace(0.5, 1.5, cols, device="cuda")
    y, rstd = Codes(6, cols), torch.empty(6, device="cuda")
    ctx.rms_norm(matrix(x), None, w.data_ptr(), eps, None, y.mat, None, rstd.data_ptr(), stream())
    v = x.float() * rstd[:, None] * w
    a = torch.maximum(v.abs().amax(1), rstd * LEAST).clamp_min(LEAST)
    assert torch.equal(y.s[:, 0], a * torch.tensor(1 / 127, dtype=torch.float32, device="cuda"))
    assert torch.equal(y.q.t, torch.round(v * (127.0 * (1.0 / a))[:, None]).to(torch.int8))
    assert (y.q.t[0] == 0).all() and torch.equal(rstd[0], (1 / torch.sqrt(torch.tensor(eps, device="cuda"))))


# ------------------------------------------------------------------------------------------------ gradients
SHAPES = [(4099, 4111, 100), (4096, 4096, 64), (2049, 2050, 601), (2056, 2040, 640), (333, 999, 777), (1000, 1000, 24), (31, 641, 13), (32, 640, 8),
          (64, 64, 2048), (100, 99, 3001), (3, 5, 200)]  # results i x j over a sum of c, for each tile, whole and ragged


def sums(ctx, which, dy, q, s, kind):
    """The gradient whose rows are dy's [i][c] (transposed for a weight's) over codes [c][j]."""
    i, j = len(dy), q.shape[1]
    out = torch.empty(i, j, dtype=TYPES[kind], device="cuda")
    if which == "input":
        ctx.matmul_grad_input(matrix(dy), matrix(q, s), matrix(out), stream())
        return out
    n = stq.matmul_grad_weight_bytes(len(q), i, j)
    work = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    across = dy.t().contiguous()
    ctx.matmul_grad_weight(matrix(across), matrix(q, s), matrix(out), work.data_ptr(), n, stream())
    return out


def operands(i, j, c):
    """Small gradients, codes of -1, 0 and 1, scales of powers of two: sums that large elements do not leave fp32's range with."""
    g = torch.Generator("cuda").manual_seed(i + 2 * j + 3 * c)
    dy = torch.randn(i, c, device="cuda", generator=g)
    q = torch.randint(-1, 2, (c, j), device="cuda", generator=g, dtype=torch.int8)
    return dy, q, torch.exp2(torch.randint(-2, 1, (c, 1), device="cuda", generator=g).float())


@pytest.mark.parametrize("which", ["input", "weight"])
@pytest.mark.parametrize("i,j,c", SHAPES)
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("of", ["bf16", "fp32"])
def test_infinities_of_gradients(ctx, which, i, j, c, kind, of):
    """An infinity of dy, or of a scale, is one in the results: NaN only where it meets a code of zero, or another sign."""
    dy, q, s = operands(i, j, c)
    dy = dy.to(TYPES[of])
    at, at2 = (i - 1, c // 2), (i // 2, c - 1)
    dy[at], dy[at2], dy[0, 0] = math.inf, -math.inf, math.nan
    got = sums(ctx, which, dy, q, s, kind).double()
    for row, col in (at, at2):
        want = dy[row, col].double() * q[col].double()  # the other elements are finite
        assert torch.equal(torch.isnan(got[row]), torch.isnan(want)) and torch.equal(got[row][q[col] != 0], want[q[col] != 0])
    assert torch.isnan(got[0]).all()
    rest = torch.ones(i, dtype=torch.bool, device="cuda")
    rest[[0, at[0], at2[0]]] = False
    assert torch.isfinite(got[rest]).all()
    dy[0, 0] = dy[at] = dy[at2] = 1.0
    s[c // 3] = math.inf
    got = sums(ctx, which, dy, q, s, kind).double()
    want = (dy[:, c // 3].double() * math.inf)[:, None] * q[c // 3].double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[~torch.isnan(want)], want[~torch.isnan(want)])


@pytest.mark.parametrize("which", ["input", "weight"])
@pytest.mark.parametrize("i,j,c", SHAPES)
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_terms_of_gradients(ctx, which, i, j, c, kind):
    """dy * s with all of its 24 bits in fp32 results, and with 16 in bf16 ones.  Two elements of dy in a row and no others, so that there is
    little of the sum's own rounding: of six terms or four, and one of dy * s.  They cancel to a part of 2^-5 and less, which leaves little
    of a bf16 result's rounding."""
    dy, q, s = operands(i, j, c)
    g = torch.Generator("cuda").manual_seed(1)
    q = torch.randint(-127, 128, (c, j), device="cuda", generator=g, dtype=torch.int8)
    a, b = c // 3, c - 1
    q[b] = q[a]
    s[a], s[b] = 0.7, 0.9
    first = torch.randn(i, device="cuda", generator=g)
    dy.zero_()
    dy[:, a], dy[:, b] = first / s[a], -first * (1 + torch.rand(i, device="cuda", generator=g) / 32) / s[b]
    got = sums(ctx, which, dy, q, s, kind).double()
    d = dy.double() * s.double().t()
    want, size = d @ q.double(), d.abs() @ q.double().abs()
    # a last place, two units, for each addition of the matrix cores; three terms hold all of dy * s (two are off by up to 2^-16)
    bound = ((1 + 2 * 6) * U + (0 if kind == "fp32" else 2.0 ** -16)) * size + (U if kind == "fp32" else B) * want.abs()
    assert ((got - want).abs() <= bound).all()


@pytest.mark.parametrize("which", ["input", "weight"])
@pytest.mark.parametrize("i,j,c", SHAPES)
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_gradients_beyond_the_largest_bf16(ctx, which, i, j, c, kind):
    """dy * s between bf16's largest number and fp32's: a finite factor as any other."""
    dy, q, s = operands(i, j, c)
    big, a, b = 3.4025e38, c // 4, c // 2
    s[a] = s[b] = 1.0
    q[b] = q[a]
    dy[i - 1, a], dy[i - 1, b], dy[0, a], dy[0, b] = big, -big, -big, 0.0
    got = sums(ctx, which, dy, q, s, kind).double()
    d = dy.double() * s.double().t()
    want, size = d @ q.double(), d.abs() @ q.double().abs()
    if kind == "bf16":
        assert torch.isfinite(got[i - 1]).all()
        hit = q[a] != 0
        assert torch.equal(torch.isinf(got[0]), hit) and torch.equal(got[0][hit].sign(), want[0][hit].sign())  # rounded to bf16
        got, want, size = got[1:], want[1:], size[1:]
    # a factor's own rounding, its terms' (24 bits, or 16), a sum's, the result's
    bound = (U + (2.0 ** -16 if kind == "bf16" else 2.0 ** -24) + (c + 2) * U) * size + (B if kind == "bf16" else U) * want.abs()
    assert ((got - want).abs() <= bound).all()


# ------------------------------------------------------------------------------------------------ places
@pytest.mark.parametrize("m,n", [(4096, 4096), (4000, 4091), (2048, 2048), (2000, 2045), (200, 300), (131, 77), (30, 70)])
def test_every_element_in_its_place(ctx, m, n):
    """Results that name their row and column, exact in fp32, through the LDS of each tile's waves."""
    x, w = (torch.ones(r, 1, dtype=torch.int8, device="cuda") for r in (m, n))
    row, col = 1.0 + torch.arange(m, device="cuda"), (1.0 + torch.arange(n, device="cuda")) / 4096
    got = product(ctx, (x, row[:, None].contiguous()), (w, col[:, None].contiguous()), torch.float32)
    assert torch.equal(got, row[:, None] * col)
    at = torch.arange(n, device="cuda")
    q = torch.zeros(8, n, dtype=torch.int8, device="cuda")
    q[1], q[6] = (at % 127).to(torch.int8), (at // 127).to(torch.int8)
    dy = torch.zeros(m, 8, device="cuda")
    dy[:, 1], dy[:, 6] = row, 127 * row
    for which in ("input", "weight"):
        assert torch.equal(sums(ctx, which, dy, q, torch.ones(8, 1, device="cuda"), "fp32"), row[:, None] * at)


# ------------------------------------------------------------------------------------------------ sizes whose launches pass 2^32 threads
PERIOD = 1021  # rows repeat, so that results can be known without a product of the whole size


def repeated(base, rows):
    t = torch.empty(rows, *base.shape[1:], dtype=base.dtype, device="cuda")
    whole = rows // PERIOD
    t[:whole * PERIOD].view(whole, *base.shape).copy_(base)
    t[whole * PERIOD:].copy_(base[:rows - whole * PERIOD])
    return t


def repeats(t, base):
    whole = len(t) // PERIOD
    return all(bool((p == base).all()) for p in t[:whole * PERIOD].view(whole, *base.shape).split(1 << 16)) and torch.equal(
        t[whole * PERIOD:], base[:len(t) - whole * PERIOD])


def codes_and_scales(seed, rows, cols):
    g = torch.Generator("cuda").manual_seed(seed)
    return (torch.randint(-127, 128, (rows, cols), device="cuda", generator=g, dtype=torch.int8), torch.rand(rows, 1, device="cuda", generator=g) + 0.5)


def product(ctx, x, w, dtype=torch.bfloat16):
    out = torch.empty(len(x[0]), len(w[0]), dtype=dtype, device="cuda")
    ctx.matmul(matrix(*x), matrix(*w), matrix(out), stream())
    return out


@pytest.mark.parametrize("tokens,outputs", [(1, (1 << 27) + 5), (17, (1 << 28) + 37), (40, (1 << 27) + 3)])
def test_few_tokens_by_many_outputs(ctx, tokens, outputs):
    """40 tokens: by rows too far apart for tiles, of which this kernel then takes up to 64."""
    x, w = codes_and_scales(1, tokens, 16), codes_and_scales(2, PERIOD, 16)
    if tokens > 32:
        apart = torch.zeros(tokens, 1 << 22, dtype=torch.int8, device="cuda")
        apart[:, :16] = x[0]
        x = (apart[:, :16], x[1])
    want = product(ctx, x, w).t().contiguous()
    exact = (w[0].double() @ x[0].double().t()) * w[1].double() * x[1].double().t()
    assert ((want.double() - exact).abs() <= 2.0 ** -8 * exact.abs()).all()
    out = product(ctx, x, (repeated(w[0], outputs), repeated(w[1], outputs)))
    for t in range(tokens):
        assert repeats(out[t], want[:, t])


def test_many_tokens_by_one_output(ctx):
    """Tiles of 256 x 256 at the largest number of rows."""
    tokens = (1 << 31) - 1
    x, w = codes_and_scales(3, PERIOD, 16), codes_and_scales(4, 1, 16)
    want = product(ctx, x, w)
    exact = (x[0].double() @ w[0].double().t()) * w[1].double() * x[1].double()
    assert ((want.double() - exact).abs() <= 2.0 ** -8 * exact.abs()).all()
    assert repeats(product(ctx, (repeated(x[0], tokens), repeated(x[1], tokens)), w), want)


def test_gradient_of_many_tokens(ctx):
    """Tiles of the gradients at the largest number of rows."""
    tokens = (1 << 31) - 1
    dy = torch.randn(PERIOD, 8, device="cuda", generator=torch.Generator("cuda").manual_seed(5)).bfloat16()
    w = codes_and_scales(6, 8, 8)

    def grad(dy):
        dx = torch.empty(len(dy), 8, dtype=torch.bfloat16, device="cuda")
        ctx.matmul_grad_input(matrix(dy), matrix(*w), matrix(dx), stream())
        return dx
    want = grad(dy)
    values = w[0].double() * w[1].double()
    exact, size = dy.double() @ values, dy.double().abs() @ values.abs()
    assert ((want.double() - exact).abs() <= 2.0 ** -8 * exact.abs() + 2.0 ** -16 * (1 + 2.0 ** -7) * size).all()
    assert repeats(grad(repeated(dy, tokens)), want)


def test_gradient_of_many_inputs(ctx):
    """Narrow gradients, one token of one output: dx = dy * scale * code."""
    inputs = (1 << 29) + 77
    q, s = codes_and_scales(7, PERIOD, 1)[0].view(-1), torch.full((1, 1), 0.75, device="cuda")
    dy, dx = torch.full((1, 1), 3.0, device="cuda"), torch.empty(1, inputs, device="cuda")
    ctx.matmul_grad_input(matrix(dy), matrix(repeated(q, inputs).view(1, inputs), s), matrix(dx), stream())
    assert repeats(dx[0], q.float() * 2.25)


def test_norm_gradients_of_many_columns(ctx):
    cols = (1 << 26) + 19
    g = torch.Generator("cuda").manual_seed(8)
    x, dy = (torch.randn(1, cols, device="cuda", generator=g).bfloat16() for _ in range(2))
    w, rstd = torch.ones(cols, device="cuda"), torch.ones(1, device="cuda")
    dx, dw = torch.empty_like(dy), torch.full((cols,), 9.0, device="cuda")
    n = stq.rms_norm_grad_bytes(1, cols)
    work = torch.empty(n, dtype=torch.uint8, device="cuda")
    ctx.rms_norm_grad(matrix(x), w.data_ptr(), rstd.data_ptr(), matrix(dy), None, matrix(dx), dw.data_ptr(), work.data_ptr(), n, stream())
    assert torch.equal(dw, (dy.float() * x.float())[0])  # one row: a product of 16 significant bits
    mean = (dy.double() * x.double()).mean()
    want = dy.double() - x.double() * mean
    # the sum of 8192 products and ten levels more in each lane, in fp32, and the result's own rounding
    assert ((dx.double() - want).abs() <= 2.0 ** -8 * want.abs() + 8300 * 8 * U * (dy.double() * x.double()).abs().mean() * x.double().abs() + 8 * U * want.abs()).all()
