"""The products of the 8-bit layer at sizes that lead to each of their tiles: whole and ragged ones, rows in 16-byte pieces and not,
sums in one and in several parts, short sums, and matrices whose last vectors end with them.  Elementwise against 64 bits, with the
bounds of test_gpu_operators.py."""
import math

import pytest
import torch

import paper_2604_06836_amd as stq
from test_gpu_operators import B, TYPES, U, Buffer, filled, gen, gradient, matrix, of_terms, stream

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = stq.Context(0, 4)
    yield c
    torch.cuda.synchronize()
    c.close()


def worst(got, want, tol):
    """The largest error in units of its tolerance (64-bit matrices, a block of rows at a time)."""
    return max(((g.double() - w).abs() / t).max().item() for g, w, t in zip(got.split(512), want.split(512), tol.split(512)))


# ------------------------------------------------------------------------------------------------ codes by codes
@pytest.mark.parametrize("m,n,k", [
    (4096, 4096, 256), (4100, 4111, 208), (4097, 4160, 1), (4352, 4096, 640),   # 256 x 256
    (2048, 2048, 384), (2050, 2001, 129), (2111, 1999, 31), (1921, 2177, 513),  # 128 x 128
    (100, 100, 128), (65, 1, 16), (70, 33, 17), (129, 640, 1000), (200, 3, 5), (64, 1, 15), (1000, 1, 15)])
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_product_of_each_tile(ctx, m, n, k, kind):
    g = gen(m + 3 * n + k)
    x, w, out = filled(g, m, k), filled(g, n, k), Buffer(m, n, TYPES[kind], 0)
    x.q.t[m - 1], w.q.t[n - 1] = 127, -127
    ctx.matmul(x.mat, w.mat, out.mat(), stream())
    want = (x.q.t.double() @ w.q.t.double().t()) * x.s.double() * w.s.double().t()
    assert worst(out.t, want, (4 * U + (B if kind == "bf16" else 0)) * want.abs() + 1e-300) <= 1


@pytest.mark.parametrize("tokens", [1, 15, 16, 17, 32, 33, 64])
@pytest.mark.parametrize("n,k", [(1, 1024), (17, 127), (31, 128), (50, 2049), (9000, 1025), (8208, 64)])
def test_product_of_few_tokens(ctx, tokens, n, k):
    g = gen(tokens + n + k)
    x, w, out = filled(g, tokens, k), filled(g, n, k), torch.empty(tokens, n, device="cuda")
    ctx.matmul(x.mat, w.mat, matrix(out), stream())
    want = (x.q.t.double() @ w.q.t.double().t()) * x.s.double() * w.s.double().t()
    assert worst(out, want, 4 * U * want.abs() + 1e-300) <= 1


def test_product_of_fewer_codes_than_a_load(ctx):
    for m, n, k in ((1, 3, 5), (3, 1, 5), (1, 1, 15), (70, 1, 4), (2, 2, 7)):
        x, w, out = filled(gen(m), m, k), filled(gen(n + 9), n, k), torch.empty(m, n, device="cuda")
        ctx.matmul(x.mat, w.mat, matrix(out), stream())
        want = (x.q.t.double() @ w.q.t.double().t()) * x.s.double() * w.s.double().t()
        assert worst(out, want, 4 * U * want.abs() + 1e-300) <= 1


# ------------------------------------------------------------------------------------------------ gradients
# (results i x j over a sum of c; for the input i = tokens, j = in, c = out; for the weight i = out, j = in, c = tokens)
SUMS = [
    (4096, 4096, 64), (4112, 4104, 520), (4099, 4111, 100), (4103, 4097, 515),              # 256 x 256, short and long
    (2048, 2048, 96), (2056, 2040, 640), (2051, 2047, 33), (2049, 2050, 601),               # 128 x 128
    (1000, 1000, 24), (500, 700, 512), (501, 703, 41), (333, 999, 777),                     # 64 x 64 in two parts
    (32, 640, 8), (16, 1000, 96), (31, 641, 13), (9, 64, 1025), (8, 8, 8), (20, 72, 4096),  # 32 x 64 in four
    (64, 64, 2048), (100, 99, 3001), (768, 300, 1600), (8, 9, 1111), (640, 640, 5000),      # parts for workgroups of their own (weights)
    (7, 100, 50), (100, 7, 50), (100, 100, 7), (1, 1, 1), (3, 5, 2000)]                     # too narrow for tiles


def operands(which, i, j, c, of, kind):
    g = gen(i + 2 * j + 3 * c)
    dy = gradient(g, *((i, c) if which == "input" else (c, i)), TYPES[of], 0)
    return dy, filled(g, c, j), Buffer(i, j, TYPES[kind], 0)


def run(ctx, which, dy, codes, out):
    if which == "input":
        ctx.matmul_grad_input(dy.mat(), codes.mat, out.mat(), stream())
    else:
        need = stq.matmul_grad_weight_bytes(dy.t.shape[0], dy.t.shape[1], codes.q.t.shape[1])
        work = torch.full((need // 4 + 4,), 88.0, device="cuda")
        ctx.matmul_grad_weight(dy.mat(), codes.mat, out.mat(), work.data_ptr(), need, stream())
        assert (work[need // 4:] == 88.0).all()


@pytest.mark.parametrize("which", ["input", "weight"])
@pytest.mark.parametrize("i,j,c", SUMS)
@pytest.mark.parametrize("of,kind", [("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32"), ("fp32", "bf16")])
def test_gradient_of_each_tile(ctx, which, i, j, c, of, kind):
    dy, codes, out = operands(which, i, j, c, of, kind)
    run(ctx, which, dy, codes, out)
    d, v = dy.t.double() if which == "input" else dy.t.double().t(), codes.value()
    want, size = d @ v, d.abs() @ v.abs()
    term, last = of_terms(kind, 2 if kind == "fp32" else 1)
    assert worst(out.t, want, (term + c * U) * size + last * want.abs() + 1e-37) <= 1


@pytest.mark.parametrize("which", ["input", "weight"])
@pytest.mark.parametrize("i,j,c", [(4099, 4111, 100), (2049, 2050, 601), (333, 999, 777), (31, 641, 13), (100, 99, 3001), (3, 5, 200), (40, 64, 96)])
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_what_is_not_finite_stays_in_its_row(ctx, which, i, j, c, kind, bad):
    """Also at the last element of the gradient, which vectors and rows that are not there repeat."""
    for at in ((0, 0), (i // 2, c // 3), (i - 1, c - 1)):
        dy, codes, out = operands(which, i, j, c, "bf16", kind)
        dy.t[at if which == "input" else at[::-1]] = bad
        run(ctx, which, dy, codes, out)
        finite = torch.isfinite(out.t.float())
        hit = torch.zeros(i, dtype=torch.bool, device="cuda")
        hit[at[0]] = True
        assert not finite[hit].any() and finite[~hit].all(), at


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_scale_that_is_not_finite(ctx, kind):
    """A row of codes whose scale is NaN is part of every sum."""
    for which, i, j, c in (("input", 100, 90, 70), ("weight", 90, 100, 70)):
        dy, codes, out = operands(which, i, j, c, "bf16", kind)
        codes.s[c - 1] = math.nan
        run(ctx, which, dy, codes, out)
        assert torch.isnan(out.t.float()).all()


def test_views_of_any_alignment(ctx):
    """The same operands at every offset of 16 bytes, in rows of odd strides: the same results, bit for bit."""
    m, n, k = 150, 140, 200
    x, w, dy = filled(gen(1), m, k), filled(gen(2), n, k), gradient(gen(3), m, n, torch.bfloat16, 0)
    out, dx, dw = torch.empty(m, n, device="cuda"), torch.empty(m, k, device="cuda"), torch.empty(n, k, device="cuda")
    ctx.matmul(x.mat, w.mat, matrix(out), stream())
    ctx.matmul_grad_input(dy.mat(), w.mat, matrix(dx), stream())
    ctx.matmul_grad_weight(dy.mat(), x.mat, matrix(dw), None, 0, stream())
    assert stq.matmul_grad_weight_bytes(m, n, k) == 0
    for at in range(1, 17, 3):
        def moved(t, extra):
            big = torch.zeros(t.shape[0] * (t.shape[1] + extra) + at + 32, dtype=t.dtype, device="cuda")
            v = big[at:].as_strided(t.shape, (t.shape[1] + extra, 1), at)
            v.copy_(t)
            return v
        xq, wq, d = moved(x.q.t, at), moved(w.q.t, 2 * at + 1), moved(dy.t, at)
        xm, wm = matrix(xq, x.s), matrix(wq, w.s)
        for which, want, call in (("out", out, lambda o: ctx.matmul(xm, wm, matrix(o), stream())),
                                  ("dx", dx, lambda o: ctx.matmul_grad_input(matrix(d), wm, matrix(o), stream())),
                                  ("dw", dw, lambda o: ctx.matmul_grad_weight(matrix(d), xm, matrix(o), None, 0, stream()))):
            o = moved(torch.zeros_like(want), at)
            call(o)
            assert torch.equal(o, want), (which, at)
