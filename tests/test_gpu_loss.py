"""The cross entropy over 8-bit codes and its gradients against 64 bits: sizes from one token and one class on, several pieces of the classes,
strides, tokens without a target, tokens predicted with certainty, rows that are not finite.

Tolerances follow from the arithmetic (u = 2^-24, b = 2^-8): a logit is off by 3 roundings; an exponential's argument by those of the logit, of its
reference and of a difference and a product, its value by two units in the last place more; sums of n terms are taken in parts of which none
is longer than n / 64 + 64.  Factors of the gradients' products enter with 11 significant bits (half a step: 2^-11) for results in
bf16 and with 22 (2^-22) for results in fp32.  They are fp16 numbers, whose steps are 2^-24 at least (half of one: 2^-25), after a power of two
that brings the largest of the result's row to 2^14 or above: 2^-39 of that largest is what any of them may be off absolutely.  The largest
of a row of dx is what a token's own loss bounds it by, max(|dloss + dlse| (1 - p), |g at the target|) with 1 - p as 2^-20 (1 + |lse|) at least,
times the largest of the classes' scales."""
import math

import pytest
import torch

import paper_2604_06836_amd as stq
from test_gpu_operators import B, TYPES, U, Buffer, Codes, matrix, stream

pytestmark = pytest.mark.gpu

IGNORE = -100


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


class Problem:
    """Codes of logits of a size of about 3; every third token predicted with certainty (or nearly), some without a target."""

    def __init__(self, t, v, n, seed=0, pad=0, ignore=True):
        g = torch.Generator("cuda").manual_seed(seed + 7 * t + v + n)
        self.t, self.v, self.n = t, v, n
        self.x, self.w = Codes(t, n, pad=pad), Codes(v, n, pad=pad)
        self.w.q.t.copy_(torch.randint(-127, 128, (v, n), device="cuda", generator=g).to(torch.int8))
        self.x.q.t.copy_(torch.randint(-127, 128, (t, n), device="cuda", generator=g).to(torch.int8))
        self.w.s.copy_(torch.exp(0.1 * torch.randn(v, 1, device="cuda", generator=g)) / 127)
        self.x.s.copy_(3 * torch.exp(0.3 * torch.randn(t, 1, device="cuda", generator=g)) / 127 / (n / 3) ** 0.5)
        self.target = torch.randint(0, v, (t,), device="cuda", generator=g)
        self.target[0] = v - 1
        sure = torch.arange(t, device="cuda") % 3 == 1
        self.x.q.t[sure] = self.w.q.t[self.target[sure]]
        if t > 3:
            self.target[3] = 0
            if ignore:
                self.target[2] = IGNORE
                self.target[t - 1] = -1
        self.loss, self.lse = torch.full((t,), 5.0, device="cuda"), torch.full((t,), 5.0, device="cuda")
        self.dloss = torch.randn(t, device="cuda", generator=g)

    def work(self, n):
        return torch.full((max(n, 16),), 255, dtype=torch.uint8, device="cuda")  # NaN in every type

    def forward(self, ctx):
        n = stq.cross_entropy_bytes(self.t, self.v, self.n)
        w = self.work(n)
        ctx.cross_entropy(self.x.mat, self.w.mat, self.target.data_ptr(), self.loss.data_ptr(), self.lse.data_ptr(), w.data_ptr(), n, stream())

    def backward(self, ctx, dx, dw, dlse=None):
        n = stq.cross_entropy_grad_bytes(self.t, self.v, self.n)
        w = self.work(n)
        ctx.cross_entropy_grad(self.x.mat, self.w.mat, self.target.data_ptr(), self.loss.data_ptr(), self.lse.data_ptr(), self.dloss.data_ptr(),
                               None if dlse is None else dlse.data_ptr(), dx, dw, w.data_ptr(), n, stream())

    def exact(self):
        """Logits, log-sums, losses in 64 bits, and how far the computed ones may be off, by token."""
        z = self.x.value() @ self.w.value().t()
        there = self.target >= 0
        at = self.target.clamp_min(0)[:, None]
        zt = z.gather(1, at)[:, 0]
        others = torch.where(there[:, None], z.scatter(1, at, -math.inf), z)
        o = torch.logsumexp(others, 1)
        d = torch.where(there, o - zt, torch.full_like(o, -math.inf))
        loss = torch.nn.functional.softplus(d, beta=1, threshold=800)
        loss = torch.where(d < -30, torch.exp(d), loss)
        lse = torch.logsumexp(z, 1)
        top = z.abs().amax(1)
        off = U * (12 * top + self.v / 64 + 64 + 16)  # of a difference of log-sum and logit
        # (below 2^-126 fp32 numbers are 2^-149 apart, whatever their size: the exponential, the logarithm and the sum are off by up to one each)
        return z, lse, loss, off, torch.sigmoid(d) * off + 8 * U * loss + 2.0 ** -147


def check_forward(p):
    z, lse, loss, off, off_loss = p.exact()
    assert ((p.lse.double() - lse).abs() <= off).all()
    assert ((p.loss.double() - loss).abs() <= off_loss).all()
    assert (p.loss[p.target < 0] == 0).all()


def check_backward(p, dx, dw, dlse=None):
    z, lse, loss, off, off_loss = p.exact()
    there = p.target >= 0
    rows = torch.arange(p.t, device="cuda")[there]
    dloss = torch.where(there, p.dloss.double(), 0.0)
    dl = torch.zeros_like(dloss) if dlse is None else dlse.double()
    soft = torch.exp(z - lse[:, None])
    g = soft * (dloss + dl)[:, None]
    # logits and log-sums as above, and the roundings of a difference, two products and the exponential
    g_off = g.abs() * (2 * off[:, None] + U * (2 * (z - lse[:, None]).abs() + 8)) + soft * U * (dloss.abs() + dl.abs())[:, None]
    # (the hardware's exponential gives 0 where the result lies below fp32's normal numbers)
    g_off += 2.0 ** -126 * (dloss.abs() + dl.abs())[:, None]
    sure = torch.exp(-loss)[there]
    g[rows, p.target[there]] = (dl * torch.exp(-loss) + dloss * torch.expm1(-loss))[there]
    g_off[rows, p.target[there]] = ((dl.abs() + dloss.abs()) * torch.exp(-loss) * off_loss)[there] \
        + 8 * U * (dl.abs()[there] * sure + dloss.abs()[there] * (1 - sure))
    g_off += 2.0 ** -148
    w, x = p.w.value(), p.x.value()
    largest = (dloss + dl).abs() * torch.where(there, torch.maximum(-torch.expm1(-loss), 2.0 ** -20 * (1 + lse.abs())), torch.maximum(torch.ones_like(lse), 2.0 ** -20 * (1 + lse.abs())))
    largest[rows] = torch.maximum(largest[rows], g[rows, p.target[there]].abs())
    largest = largest[:, None] * p.w.s.double().max()
    largest_of_class = (g.t().abs() * p.x.s.double().view(1, -1)).amax(1, keepdim=True)
    for out, f, f_off, m, scale, n, most in ((dx, g, g_off, w, p.w.s, p.v, largest), (dw, g.t(), g_off.t(), x, p.x.s, p.t, largest_of_class)):
        if out is None:
            continue
        bf16 = out.t.dtype == torch.bfloat16
        term = 2.0 ** -11 if bf16 else 2.0 ** -22
        size = f.abs() @ m.abs()
        least = most * 2.0 ** -39 * (1 + B) * m.div(scale.double()).abs().sum(0, keepdim=True)
        # (a factor g * scale is rounded to fp32, whose numbers below 2^-126 are 2^-149 apart)
        least = least + 2.0 ** -149 * m.div(scale.double()).abs().sum(0, keepdim=True)
        want = f @ m
        bound = f_off @ m.abs() + (term + (n + 8) * U) * size + least + (B * want.abs() * (1 + B) if bf16 else 0.0) + 2.0 ** -133
        off_by = (out.t.double() - want).abs()
        assert (off_by <= bound).all(), (off_by / bound).max().item()
        assert out.untouched()


SIZES = [(1, 1, 1), (1, 7, 5), (2, 2, 300), (1, 1000, 64), (1, 5003, 768), (5, 257, 33), (16, 999, 128), (17, 4096, 64), (33, 5003, 130), (64, 300, 768),
         (65, 2049, 96), (300, 1001, 100), (257, 4096, 256), (1000, 777, 64), (513, 9001, 304), (2049, 3001, 129), (3, 70001, 16), (700, 16, 8), (40, 9, 2000)]


@pytest.mark.parametrize("t,v,n", SIZES)
@pytest.mark.parametrize("pad", [0, 3])
def test_loss(ctx, t, v, n, pad):
    p = Problem(t, v, n, pad=pad)
    p.forward(ctx)
    check_forward(p)


@pytest.mark.parametrize("t,v,n", SIZES)
@pytest.mark.parametrize("kinds,pad,with_dlse", [(("fp32", "fp32"), 0, False), (("bf16", "bf16"), 0, False), (("bf16", "fp32"), 3, True),
                                                 (("fp32", "bf16"), 5, False)])
def test_gradients(ctx, t, v, n, kinds, pad, with_dlse):
    p = Problem(t, v, n, seed=1, pad=pad)
    dx, dw = Buffer(t, n, TYPES[kinds[0]], pad), Buffer(v, n, TYPES[kinds[1]], pad)
    dlse = torch.randn(t, device="cuda", generator=torch.Generator("cuda").manual_seed(t)) if with_dlse else None
    p.forward(ctx)
    p.backward(ctx, dx.mat(), dw.mat(), dlse)
    check_backward(p, dx, dw, dlse)
    if not with_dlse and t > 3:
        assert (dx.t[2] == 0).all()


# Results of large, ordinary and small tiles behind logits of each tile, sums in parts and not, and sizes that no tile divides.
@pytest.mark.parametrize("t,v,n", [(192, 27392, 645), (1024, 8192, 1024), (2048, 8192, 512), (2500, 9000, 500), (640, 5003, 768), (128, 20000, 128), (3000, 600, 1000),
                                   (1500, 2500, 130), (257, 40000, 40)])
@pytest.mark.parametrize("kinds", [("fp32", "fp32"), ("bf16", "bf16"), ("fp32", "bf16"), ("bf16", "fp32")])
def test_every_tile(ctx, t, v, n, kinds):
    p = Problem(t, v, n, seed=17)
    p.dloss *= torch.exp(4 * torch.randn(t, device="cuda", generator=torch.Generator("cuda").manual_seed(3)))  # units that change from tile to tile
    p.forward(ctx)
    dx, dw = Buffer(t, n, TYPES[kinds[0]]), Buffer(v, n, TYPES[kinds[1]])
    p.backward(ctx, dx.mat(), dw.mat())
    check_backward(p, dx, dw)


@pytest.mark.parametrize("t,v,n", [(4099, 20001, 64), (70001, 1500, 16)])
@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_several_pieces(ctx, t, v, n, kind):
    p = Problem(t, v, n, seed=2)
    p.forward(ctx)
    check_forward(p)
    dx, dw = Buffer(t, n, TYPES[kind]), Buffer(v, n, TYPES[kind])
    p.backward(ctx, dx.mat(), dw.mat())
    check_backward(p, dx, dw)


@pytest.mark.parametrize("t,v,n", [(70001, 5003, 16), (16411, 20001, 64), (16411, 20001, 301), (1, 3 * 2 ** 20 + 5, 16), (17, 2200007, 24)])
@pytest.mark.parametrize("kinds", [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32")])
def test_classes_that_do_not_fit_one_piece(ctx, t, v, n, kinds):
    # Factors of all classes at once, two of at least two bytes each, would not fit the workspace: so there are several pieces, for either type.
    assert stq.cross_entropy_grad_bytes(t, v, n) < 4 * ((t + 127) // 128 * 128) * v
    p = Problem(t, v, n, seed=12)
    p.forward(ctx)
    check_forward(p)
    dx, dw = Buffer(t, n, TYPES[kinds[0]]), Buffer(v, n, TYPES[kinds[1]])
    p.backward(ctx, dx.mat(), dw.mat())
    check_backward(p, dx, dw)
    one = Buffer(t, n, TYPES[kinds[0]])
    if kinds[0] == kinds[1]:  # (with dw in fp32 the pieces would be others than without it)
        p.backward(ctx, one.mat(), None)
        assert torch.equal(one.t, dx.t)


# Rows so far apart that the last of the classes' lie beyond 2^32 bytes and (of dw) 2^31 elements; at 2^22 codes and more the kernels are others.
@pytest.mark.parametrize("t,v,stride", [(3, 2200, 1 << 21), (300, 2200, 1 << 21), (300, 2200, (1 << 21) + 5), (5, 1100, 1 << 22), (70, 1100, 1 << 22)])
@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_rows_far_apart(ctx, t, v, stride, kind):
    n = 64
    p = Problem(t, v, n, seed=13)
    x, w = p.x, p.w
    p.x, p.w = Codes(t, n, pad=stride - n), Codes(v, n, pad=stride - n)
    for to, of in ((p.x, x), (p.w, w)):
        if stride % 16 == 0:  # rows that begin at 16 bytes
            to.q.at, to.q.t = 0, to.q.whole[:, :n]
            to.mat = to.q.mat(to.s)
        to.q.t.copy_(of.q.t)
        to.s.copy_(of.s)
    p.forward(ctx)
    check_forward(p)
    dx, dw = Buffer(t, n, TYPES[kind], pad=(1 << 20) - n), Buffer(v, n, TYPES[kind], pad=(1 << 20) - n)
    p.backward(ctx, dx.mat(), dw.mat())
    check_backward(p, dx, dw)


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_one_gradient_alone(ctx, kind):
    p = Problem(300, 1001, 100, seed=3)
    p.forward(ctx)
    both = Buffer(300, 100, TYPES[kind]), Buffer(1001, 100, TYPES[kind])
    one = Buffer(300, 100, TYPES[kind]), Buffer(1001, 100, TYPES[kind])
    p.backward(ctx, both[0].mat(), both[1].mat())
    p.backward(ctx, one[0].mat(), None)
    p.backward(ctx, None, one[1].mat())
    assert torch.equal(both[0].t, one[0].t) and torch.equal(both[1].t, one[1].t)  # the same bits, call after call


def test_no_tokens(ctx):
    w = Codes(50, 64)
    w.q.t.zero_()
    w.s.fill_(1.0)
    empty = stq.make_matrix(None, 0, 64, stq.STQ_Q8)
    ctx.cross_entropy(empty, w.mat, None, None, None, None, 0, stream())
    dw = torch.full((50, 64), 7.0, device="cuda")
    ctx.cross_entropy_grad(empty, w.mat, None, None, None, None, None, stq.make_matrix(None, 0, 64, stq.STQ_F32), matrix(dw), None, 0, stream())
    assert (dw == 0).all()


def test_no_targets_at_all(ctx):
    p = Problem(40, 300, 64, seed=4)
    p.target.fill_(IGNORE)
    p.forward(ctx)
    check_forward(p)
    dx, dw = Buffer(40, 64, torch.float32), Buffer(300, 64, torch.bfloat16)
    p.backward(ctx, dx.mat(), dw.mat())
    assert (dx.t == 0).all() and (dw.t == 0).all()


@pytest.mark.parametrize("t", [3, 40, 500])
def test_padding_that_is_not_finite(ctx, t):
    """A token without a target, whose codes' scale is NaN (as a row with a NaN is written): its own log-sum is, and nothing else."""
    p = Problem(t, 500, 64, seed=5, ignore=False)
    p.forward(ctx)
    clean = Buffer(t, 64, torch.float32), Buffer(500, 64, torch.float32)
    p.target[1] = IGNORE
    loss = p.loss.clone()
    p.forward(ctx)
    p.backward(ctx, clean[0].mat(), clean[1].mat())
    p.x.s[1] = math.nan
    p.x.q.t[1] = 0
    p.forward(ctx)
    dx, dw = Buffer(t, 64, torch.float32), Buffer(500, 64, torch.float32)
    p.backward(ctx, dx.mat(), dw.mat())
    assert p.lse[1].isnan() and p.loss[1] == 0 and p.lse.isnan().sum() == 1
    assert torch.equal(p.loss[2:], loss[2:])
    assert torch.equal(dx.t, clean[0].t) and torch.equal(dw.t, clean[1].t)


@pytest.mark.parametrize("t", [3, 40, 500])
@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_tokens_that_are_not_finite(ctx, t, kind):
    p = Problem(t, 500, 64, seed=6)
    p.x.s[0] = math.nan
    p.forward(ctx)
    assert p.lse[0].isnan() and p.loss[0].isnan() and p.lse[1:].isfinite().all()
    dx, dw = Buffer(t, 64, TYPES[kind]), Buffer(500, 64, TYPES[kind])
    p.backward(ctx, dx.mat(), dw.mat())
    assert dx.t[0].isnan().all() and dx.t[1:].isfinite().all() and dw.t.isnan().all()


@pytest.mark.parametrize("t", [2, 40, 500])
def test_a_class_that_is_not_finite(ctx, t):
    p = Problem(t, 500, 64, seed=7)
    p.w.s[17] = math.nan
    p.forward(ctx)
    assert p.lse.isnan().all() and (p.loss.isnan() | (p.target < 0)).all()


@pytest.mark.parametrize("t", [2, 40, 500])
@pytest.mark.parametrize("beyond", [500, 1 << 31, (1 << 32) + 3, (1 << 63) - 1])
def test_targets_beyond_the_classes(ctx, t, beyond):
    p = Problem(t, 500, 64, seed=8)
    want = Problem(t, 500, 64, seed=8)
    want.forward(ctx)
    p.target[1] = beyond
    p.forward(ctx)
    assert p.loss[1].isnan() and p.loss.isnan().sum() == 1
    assert ((p.lse - want.lse).abs() <= 1e-4).all() and torch.equal(p.loss[2:], want.loss[2:])
    dx, dw = Buffer(t, 64, torch.float32), Buffer(500, 64, torch.float32)
    p.backward(ctx, dx.mat(), dw.mat())
    assert dx.t[1].isnan().all() and dx.t[0].isfinite().all() and dx.t[2:].isfinite().all() and dw.t.isnan().all()


def test_large_and_equal_logits(ctx):
    """Logits of thousands, all of one row equal, and a class that has everything."""
    t, v, n = 40, 1000, 64
    p = Problem(t, v, n, seed=9)
    p.x.s.mul_(1000.0)
    p.x.q.t[5] = 0
    p.forward(ctx)
    check_forward(p)
    dx, dw = Buffer(t, n, torch.float32), Buffer(v, n, torch.float32)
    p.backward(ctx, dx.mat(), dw.mat())
    check_backward(p, dx, dw)
    assert p.loss.isfinite().all() and abs(p.lse[5].item() - math.log(v)) <= U * (v / 64 + 100)


def test_rows_of_very_different_size(ctx):
    """Classes that no token comes near have gradients far below the others', and losses weigh from 1e-12 to 1e12."""
    t, v, n = 300, 1000, 64
    p = Problem(t, v, n, seed=10)
    p.w.s[::7] *= 4.0
    p.dloss = torch.logspace(-12, 12, t, device="cuda")
    p.forward(ctx)
    for kind in ("fp32", "bf16"):
        dx, dw = Buffer(t, n, TYPES[kind]), Buffer(v, n, TYPES[kind])
        p.backward(ctx, dx.mat(), dw.mat())
        check_backward(p, dx, dw)


@pytest.mark.parametrize("t,v,n", [(40, 300, 64), (300, 1001, 256), (513, 3001, 768)])
@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_losses_that_are_differences(ctx, t, v, n, kind):
    """Losses from elsewhere: fp32 log-sums less fp32 logits, 0 or slightly wrong for tokens predicted with certainty.  Nothing overflows, and the
    gradients are off by no more than the losses are: two roundings of numbers of lse's size, and the logit's own three."""
    p = Problem(t, v, n, seed=16)
    z, lse, loss, off, off_loss = p.exact()
    there = p.target >= 0
    at = p.target.clamp_min(0)[:, None]
    p.lse = lse.float()
    p.loss = torch.where(there, p.lse - z.float().gather(1, at)[:, 0], 0.0)
    assert (p.loss[there] == 0).any()
    dx, dw = Buffer(t, n, TYPES[kind]), Buffer(v, n, TYPES[kind])
    p.backward(ctx, dx.mat(), dw.mat())
    g = torch.exp(z - lse[:, None]) * torch.where(there, p.dloss.double(), 0.0)[:, None]
    g_off = g.abs() * (2 * off[:, None] + U * (2 * (z - lse[:, None]).abs() + 9)) + 2.0 ** -126 * p.dloss.abs().double()[:, None]
    rows = torch.arange(t, device="cuda")[there]
    g[rows, p.target[there]] = (p.dloss.double() * torch.expm1(-loss))[there]
    g_off[rows, p.target[there]] = (p.dloss.double().abs() * (off + U * 4 * lse.abs()))[there]
    w, x = p.w.value(), p.x.value()
    largest = p.dloss.abs().double() * torch.where(there, torch.maximum(-torch.expm1(-loss) + U * 4 * lse.abs(), 2.0 ** -20 * (1 + lse.abs())), 0.0)
    for out, f, f_off, m, scale, k, most in ((dx, g, g_off, w, p.w.s, v, largest[:, None] * p.w.s.double().max()),
                                             (dw, g.t(), g_off.t(), x, p.x.s, t, ((g.t().abs() + g_off.t()) * p.x.s.double().view(1, -1)).amax(1, keepdim=True))):
        bf16 = out.t.dtype == torch.bfloat16
        want = f @ m
        bound = f_off @ m.abs() + ((2.0 ** -11 if bf16 else 2.0 ** -22) + (k + 8) * U) * (f.abs() @ m.abs()) + (B * want.abs() * (1 + B) if bf16 else 0.0) \
            + most * 2.0 ** -39 * (1 + B) * m.div(scale.double()).abs().sum(0, keepdim=True) + 2.0 ** -126
        assert ((out.t.double() - want).abs() <= bound).all()


def test_gradients_against_differences(ctx):
    """The loss in 64 bits, moved along random directions of the values behind the codes, against the kernels' gradients."""
    p = Problem(40, 300, 64, seed=11)
    p.forward(ctx)
    dx, dw = Buffer(40, 64, torch.float32), Buffer(300, 64, torch.float32)
    dlse = torch.randn(40, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    p.backward(ctx, dx.mat(), dw.mat(), dlse)
    g = torch.Generator("cuda").manual_seed(2)
    x, w, there = p.x.value(), p.w.value(), p.target >= 0

    def total(x, w):
        z = x @ w.t()
        lse = torch.logsumexp(z, 1)
        loss = torch.where(there, lse - z.gather(1, p.target.clamp_min(0)[:, None])[:, 0], 0.0)
        return (p.dloss.double() * loss + dlse.double() * lse).sum()
    for _ in range(5):
        ux, uw = torch.randn(x.shape, device="cuda", generator=g).double(), torch.randn(w.shape, device="cuda", generator=g).double()
        h = 1e-5
        slope = (total(x + h * ux, w + h * uw) - total(x - h * ux, w - h * uw)) / (2 * h)
        got = (dx.t.double() * ux).sum() + (dw.t.double() * uw).sum()
        # differences: h^2 of a third derivative, and 64 bits' roundings of the totals over 2h
        assert abs(got - slope).item() <= 1e-4 * ((dx.t.double() * ux).abs().sum() + (dw.t.double() * uw).abs().sum()).item()


def test_calls_on_two_streams_at_once(ctx):
    problems = [Problem(300, 1001, 100, seed=12), Problem(257, 4096, 256, seed=13)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = [(Buffer(p.t, p.n, torch.float32), Buffer(p.v, p.n, torch.bfloat16)) for p in problems]
    works = [p.work(max(stq.cross_entropy_bytes(p.t, p.v, p.n), stq.cross_entropy_grad_bytes(p.t, p.v, p.n))) for p in problems]
    torch.cuda.synchronize()
    for _ in range(3):
        for p, s, (dx, dw), w in zip(problems, streams, outs, works):
            ctx.cross_entropy(p.x.mat, p.w.mat, p.target.data_ptr(), p.loss.data_ptr(), p.lse.data_ptr(), w.data_ptr(), w.numel(), s.cuda_stream)
            ctx.cross_entropy_grad(p.x.mat, p.w.mat, p.target.data_ptr(), p.loss.data_ptr(), p.lse.data_ptr(), p.dloss.data_ptr(), None, dx.mat(), dw.mat(),
                                   w.data_ptr(), w.numel(), s.cuda_stream)
    torch.cuda.synchronize()
    for p, (dx, dw) in zip(problems, outs):
        check_forward(p)
        check_backward(p, dx, dw)


def test_recorded(ctx):
    """Loss, gradients, their norm and clipping as one graph, replayed on new inputs in place with eager calls between the replays."""
    p = Problem(300, 1001, 100, seed=14)
    dx, dw = torch.empty(300, 100, device="cuda"), torch.empty(1001, 100, dtype=torch.bfloat16, device="cuda")
    w = p.work(max(stq.cross_entropy_bytes(300, 1001, 100), stq.cross_entropy_grad_bytes(300, 1001, 100)))
    norm = torch.zeros(2, dtype=torch.float64, device="cuda")
    r = stq.make_grads([dict(grad=dx.data_ptr(), numel=dx.numel(), dtype=stq.STQ_F32), dict(grad=dw.data_ptr(), numel=dw.numel(), dtype=stq.STQ_BF16)])

    def all_of(s):
        ctx.cross_entropy(p.x.mat, p.w.mat, p.target.data_ptr(), p.loss.data_ptr(), p.lse.data_ptr(), w.data_ptr(), w.numel(), s)
        ctx.cross_entropy_grad(p.x.mat, p.w.mat, p.target.data_ptr(), p.loss.data_ptr(), p.lse.data_ptr(), p.dloss.data_ptr(), None, matrix(dx), matrix(dw),
                               w.data_ptr(), w.numel(), s)
        ctx.grad_norm(r, norm.data_ptr(), s)
        ctx.clip_grads(r, norm.data_ptr(), 1.0, s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            all_of(torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for turn in range(4):
        new = Problem(300, 1001, 100, seed=20 + turn)
        for a, b in ((p.x.q.t, new.x.q.t), (p.x.s, new.x.s), (p.w.q.t, new.w.q.t), (p.w.s, new.w.s), (p.target, new.target), (p.dloss, new.dloss)):
            a.copy_(b)
        all_of(stream())
        torch.cuda.synchronize()
        want = [t.clone() for t in (p.loss, p.lse, dx, dw, norm)]
        for t in (p.loss, p.lse, dx, dw, norm):
            t.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (p.loss, p.lse, dx, dw, norm)))
        check_forward(p)


def test_workspace_is_all_that_is_written(ctx):
    """Nothing is written behind the workspace's stated end."""
    for t, v, n in ((1, 1000, 64), (33, 5003, 130), (300, 1001, 100), (65, 2049, 96)):
        p = Problem(t, v, n, seed=15)
        dx, dw = Buffer(t, n, torch.float32), Buffer(v, n, torch.float32)
        f, b = stq.cross_entropy_bytes(t, v, n), stq.cross_entropy_grad_bytes(t, v, n)
        work = torch.full((max(f, b) + 4096,), 200, dtype=torch.uint8, device="cuda")
        ctx.cross_entropy(p.x.mat, p.w.mat, p.target.data_ptr(), p.loss.data_ptr(), p.lse.data_ptr(), work.data_ptr(), f, stream())
        assert (work[f:] == 200).all()
        ctx.cross_entropy_grad(p.x.mat, p.w.mat, p.target.data_ptr(), p.loss.data_ptr(), p.lse.data_ptr(), p.dloss.data_ptr(), None, dx.mat(), dw.mat(),
                               work.data_ptr(), b, stream())
        assert (work[max(f, b):] == 200).all()


def test_refusals(ctx):
    def code_of(call):
        with pytest.raises(stq.StqError) as e:
            call()
        return e.value.code

    def odd(m, **change):
        r = stq.make_matrix(m.data, m.rows, m.cols, m.dtype, stride=m.stride, scales=m.scales, block=m.block)
        for k, v in change.items():
            setattr(r, k, v)
        return r
    EINVAL, EALIGN, EBLOCK, ESHAPE, EDTYPE = -1, -2, -4, -9, -10
    x, w, blocked, s = Codes(8, 64), Codes(30, 64), Codes(8, 64, 64), stream()
    target, f = torch.zeros(8, dtype=torch.int64, device="cuda"), torch.zeros(8, device="cuda")
    n = max(stq.cross_entropy_bytes(8, 30, 64), stq.cross_entropy_grad_bytes(8, 30, 64))
    work = torch.zeros(n, dtype=torch.uint8, device="cuda")
    T, F, W = target.data_ptr(), f.data_ptr(), work.data_ptr()
    call = lambda x=x.mat, w=w.mat, t=T, lo=F, ls=F, wk=W, b=n: code_of(lambda: ctx.cross_entropy(x, w, t, lo, ls, wk, b, s))  # noqa: E731
    need = stq.cross_entropy_bytes(8, 30, 64)
    assert call(x=None) == EINVAL and call(w=None) == EINVAL and call(t=None) == EINVAL and call(lo=None) == EINVAL and call(ls=None) == EINVAL
    assert call(wk=None) == EINVAL and call(b=need - 1) == EINVAL and call(wk=W + 4) == EALIGN and call(t=T + 4) == EALIGN and call(lo=F + 2) == EALIGN
    assert call(x=blocked.mat) == EBLOCK and call(x=odd(x.mat, cols=63)) == ESHAPE and call(w=odd(w.mat, rows=0)) == ESHAPE
    assert call(x=odd(x.mat, cols=1 << 17, stride=1 << 17), w=odd(w.mat, cols=1 << 17, stride=1 << 17)) == ESHAPE
    assert call(x=odd(x.mat, dtype=0)) == EDTYPE and call(x=odd(x.mat, scales=None)) == EINVAL
    dx, dw = torch.zeros(8, 64, device="cuda"), torch.zeros(30, 64, device="cuda")
    X, D = matrix(dx), matrix(dw)
    call = lambda x=x.mat, w=w.mat, t=T, lo=F, ls=F, dl=F, de=None, dx=X, dw=D, wk=W, b=n: code_of(  # noqa: E731
        lambda: ctx.cross_entropy_grad(x, w, t, lo, ls, dl, de, dx, dw, wk, b, s))
    need = stq.cross_entropy_grad_bytes(8, 30, 64)
    assert call(x=None) == EINVAL and call(t=None) == EINVAL and call(lo=None) == EINVAL and call(ls=None) == EINVAL and call(dl=None) == EINVAL
    assert call(dx=None, dw=None) == EINVAL and call(b=need - 1) == EINVAL and call(wk=None) == EINVAL and call(wk=W + 8) == EALIGN
    assert call(de=F + 1) == EALIGN and call(dx=D) == ESHAPE and call(dw=X) == ESHAPE and call(dx=x.mat) == EDTYPE and call(dw=odd(D, dtype=2)) == EDTYPE
    assert call(w=odd(w.mat, cols=60)) == ESHAPE and call(x=blocked.mat) == EBLOCK
    torch.cuda.synchronize()
    assert (dx == 0).all() and (dw == 0).all() and (f == 0).all()
