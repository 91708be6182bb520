"""Roundings of the 8-bit layer's operators: codes and scales as their formulas say, step by step in fp32, and gradients whose
small elements stand beside large ones."""
import pytest
import torch

import paper_2604_06836_amd as stq

pytestmark = pytest.mark.gpu

LEAST = 2.0 ** -100
KIND = {torch.float32: stq.STQ_F32, torch.bfloat16: stq.STQ_BF16, torch.int8: stq.STQ_Q8}


@pytest.fixture(scope="module")
def ctx():
    c = stq.Context(0, 4)
    yield c
    torch.cuda.synchronize()
    c.close()


def mat(t, scales=None, block=0):
    return stq.make_matrix(t.data_ptr(), t.shape[0], t.shape[1], KIND[t.dtype], scales=None if scales is None else scales.data_ptr(), block=block)


def stream():
    return torch.cuda.current_stream().cuda_stream


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def written(x, block):
    """q = rint(x * (127 * (1 / a))), s = a * (1 / 127), every step in fp32."""
    rows, cols = x.shape
    width = block or cols
    pad = -cols % width
    v = torch.nn.functional.pad(x, (0, pad)).view(rows, -1, width)
    a = v.abs().amax(2, keepdim=True).clamp_min(LEAST)
    one = torch.ones_like(a)
    q = torch.round(v * (one / a * 127.0)).view(rows, cols + pad)[:, :cols]
    return q.to(torch.int8), (a * torch.tensor(1.0 / 127.0, dtype=torch.float32, device="cuda")).squeeze(2)


def codes_like(rows, cols, block):
    return torch.zeros(rows, cols, dtype=torch.int8, device="cuda"), torch.zeros(rows, (cols - 1) // (block or cols) + 1, device="cuda")


@pytest.mark.parametrize("rows,cols", [(1, 1), (300, 64), (257, 100), (40, 1600), (64, 4096), (3, 40001)])
@pytest.mark.parametrize("block", [0, 64, 128])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", [1.0, 2.0 ** -90, 2.0 ** 100])
def test_codes_bit_for_bit(ctx, rows, cols, block, dtype, size):
    x = (torch.randn(rows, cols, device="cuda", generator=gen(rows + cols)) * size).to(dtype)
    q, s = codes_like(rows, cols, block)
    ctx.quantize_rows(mat(x), mat(q, s, block), stream())
    want_q, want_s = written(x.float(), block)
    assert torch.equal(s, want_s) and torch.equal(q, want_q)


@pytest.mark.parametrize("rows,cols", [(300, 64), (40, 1600), (200, 4096), (9, 16384), (3, 40001)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_codes_of_norm_bit_for_bit(ctx, rows, cols, dtype):
    """From the norm's own sum and reciprocal root."""
    g = gen(rows * 3 + cols)
    x, r = [torch.randn(rows, cols, device="cuda", generator=g).to(dtype) for _ in range(2)]
    x[:, cols // 3] *= 30
    w = 1 + 0.3 * torch.randn(cols, device="cuda", generator=g)
    total, rstd = torch.empty_like(x), torch.empty(rows, device="cuda")
    (q, s), (kq, ks) = codes_like(rows, cols, 0), codes_like(rows, cols, 128)
    ctx.rms_norm(mat(x), mat(r), w.data_ptr(), 1e-5, mat(total), mat(q, s), mat(kq, ks, 128), rstd.data_ptr(), stream())
    h = (x.float() + r.float()).to(dtype)
    assert torch.equal(total, h)
    for got, want in (((q, s), written(h.float() * rstd[:, None] * w, 0)), ((kq, ks), written(h.float(), 128))):
        assert torch.equal(got[1], want[1]) and torch.equal(got[0], want[0])


@pytest.mark.parametrize("which", ["input", "weight"])
@pytest.mark.parametrize("i,j,c", [(20, 72, 200), (300, 200, 320), (1100, 1200, 300), (4096, 4096, 520), (65, 1001, 2049), (7, 300, 90)])
@pytest.mark.parametrize("of", [torch.float32, torch.bfloat16])
def test_small_elements_beside_large(ctx, which, i, j, c, of):
    """Rows of the result a thousandfold of others.  Each element is off by its own rounding to bf16 (2^-8 of it), by what two terms of
    dy * s leave (2^-16 of each product, with the product's own 2^-24) and by a sum in fp32 (2^-24 of the magnitudes' sum for each of
    its c additions)."""
    g = gen(i + 2 * j + 3 * c)
    large = torch.exp2(10 * torch.rand(i, 1, device="cuda", generator=g))
    dy = (torch.randn(i, c, device="cuda", generator=g) * large).to(of)
    q = torch.randint(-127, 128, (c, j), device="cuda", generator=g, dtype=torch.int8)
    s = torch.rand(c, device="cuda", generator=g) + 0.01
    out = torch.empty(i, j, device="cuda", dtype=torch.bfloat16)
    if which == "input":  # i tokens, c outputs, j inputs
        ctx.matmul_grad_input(mat(dy), mat(q, s), mat(out), stream())
    else:  # i outputs, c tokens, j inputs
        n = stq.matmul_grad_weight_bytes(c, i, j)
        work = torch.empty(max(n, 16), device="cuda", dtype=torch.uint8)
        across = dy.t().contiguous()
        ctx.matmul_grad_weight(mat(across), mat(q, s), mat(out), work.data_ptr(), n, stream())
    a, b = dy.double() * s.double(), q.double()
    want, most = a @ b, a.abs() @ b.abs()
    bound = 2.0 ** -8 * want.abs() + (2.0 ** -16 + (c + 2) * 2.0 ** -24) * (1 + 2.0 ** -7) * most
    assert ((out.double() - want).abs() <= bound).all()
