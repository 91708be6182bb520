"""The global gradient norm and clipping against 64 bits: tensors of both types in one call, sizes that no vector divides, any alignment,
numbers whose squares fp32 cannot hold, infinities and NaN, in place and not.

Tolerances follow from the arithmetic: squares of fp32 numbers are exact in fp64 and n of them add up within n 2^-53; a clipped element has
the factor's rounding to fp32, the product's (2^-24 each), and for bf16 one more (2^-8)."""
import math

import pytest
import torch

import paper_2604_06836_amd as stq

pytestmark = pytest.mark.gpu

U, B = 2.0 ** -24, 2.0 ** -8
KIND = {torch.float32: stq.STQ_F32, torch.bfloat16: stq.STQ_BF16}
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = stq.Context(0, 700)
    yield c
    torch.cuda.synchronize()
    c.close()


def stream():
    return torch.cuda.current_stream().cuda_stream


def tensors(sizes, dtypes, seed=0, shift=0, scale=1e-2):
    """Slices of one guarded buffer for each type, `shift` elements behind a multiple of 16 bytes; what lies between them is 77."""
    g = torch.Generator("cuda").manual_seed(seed)
    out = []
    for n, t in zip(sizes, dtypes):
        whole = torch.full((n + shift + 64,), 77.0, device="cuda", dtype=t)
        v = whole[shift:shift + n]
        v.copy_(scale * torch.exp(torch.randn((), device="cuda", generator=g)) * torch.randn(n, device="cuda", generator=g))
        out.append((whole, v))
    return out


def records(grads, outs=None):
    return stq.make_grads(dict(grad=g.data_ptr() if g.numel() else None, out=None if outs is None else o.data_ptr(), numel=g.numel(), dtype=KIND[g.dtype])
                          for g, o in zip(grads, outs or grads))


def squares(grads):
    return sum((g.double() ** 2).sum() for g in grads)


def factor_of(total, most):
    return min(1.0, most / (math.sqrt(float(total)) + 1e-6)) if math.isfinite(float(total)) else (0.0 if float(total) > 0 else math.nan)


def check_norm(norm, grads):
    want, n = float(squares(grads)), sum(g.numel() for g in grads)
    assert abs(norm[0].item() - want) <= n * 2.0 ** -53 * want
    assert abs(norm[1].item() - math.sqrt(want)) <= (n + 4) * 2.0 ** -53 * math.sqrt(want)


def check_clipped(out, g, c):
    want = g.double() * c
    bound = (2 * U + (B if g.dtype == BF16 else 0.0)) * want.abs() * (1 + B) + 2.0 ** -149
    assert ((out.double() - want).abs() <= bound).all()


SETS = [([1], "f"), ([7], "b"), ([2048], "f"), ([2049, 1, 2047], "bfb"), ([5, 0, 40001, 8, 0], "bffbb"), ([0, 0], "fb"), ([1 << 20, (1 << 20) + 3], "bf"),
        ([768] * 300 + [3 * 2048 + 11] * 30, "fb"), ([5_000_001, 3, 9_999_999], "bfb")]


@pytest.mark.parametrize("sizes,kinds", SETS, ids=[str(i) for i in range(len(SETS))])
@pytest.mark.parametrize("shift", [0, 1, 3])
@pytest.mark.parametrize("most", [1e-3, 1e6])
def test_norm_and_clip(ctx, sizes, kinds, shift, most):
    dtypes = [dict(f=F32, b=BF16)[kinds[i % len(kinds)]] for i in range(len(sizes))]
    ts = tensors(sizes, dtypes, len(sizes), shift)
    grads, before = [v for _, v in ts], [v.clone() for _, v in ts]
    outs = tensors(sizes, dtypes, 1, (shift * 5) % 7)
    norm = torch.full((3,), 5.0, dtype=torch.float64, device="cuda")
    into, place = records(grads, [v for _, v in outs]), records(grads)
    ctx.grad_norm(into, norm.data_ptr(), stream())
    ctx.clip_grads(into, norm.data_ptr(), most, stream())
    check_norm(norm, before)
    assert norm[2].item() == 5.0
    c = factor_of(norm[0], most)
    assert (c < 1) == (most < 1) or sum(sizes) == 0
    for (whole, o), g, b in zip(outs, grads, before):
        check_clipped(o, b, c)
        assert torch.equal(g, b)  # not in place
        assert (whole[:o.storage_offset()] == 77).all() and (whole[o.storage_offset() + o.numel():] == 77).all()
    again = torch.empty(2, dtype=torch.float64, device="cuda")
    ctx.grad_norm(place, again.data_ptr(), stream())
    assert torch.equal(again, norm[:2])  # the same bits
    ctx.clip_grads(place, again.data_ptr(), most, stream())
    for (whole, g), (_, o) in zip(ts, outs):
        assert torch.equal(g, o)
        assert (whole[:shift] == 77).all() and (whole[shift + g.numel():] == 77).all()


def test_no_tensors(ctx):
    norm = torch.full((2,), 5.0, dtype=torch.float64, device="cuda")
    none = stq.make_grads([])
    ctx.grad_norm(none, norm.data_ptr(), stream())
    ctx.clip_grads(none, norm.data_ptr(), 1.0, stream())
    assert norm.tolist() == [0.0, 0.0]


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_squares_that_fp32_cannot_hold(ctx, dtype):
    for value in (torch.finfo(dtype).max, 1e30, 1e-30, 2.0 ** -126, 2.0 ** -149 if dtype == F32 else 2.0 ** -133):
        g = torch.full((5000,), value, device="cuda", dtype=dtype)
        norm, r = torch.empty(2, dtype=torch.float64, device="cuda"), records([g])
        ctx.grad_norm(r, norm.data_ptr(), stream())
        check_norm(norm, [g])
        assert norm[0].item() > 0
        before = g.clone()
        ctx.clip_grads(r, norm.data_ptr(), 0.25, stream())
        check_clipped(g, before, factor_of(norm[0], 0.25))


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_what_is_not_finite(ctx, bad, dtype):
    g, h = torch.ones(4000, device="cuda", dtype=dtype), torch.ones(100, device="cuda")
    g[3999] = bad
    norm, r = torch.empty(2, dtype=torch.float64, device="cuda"), records([h, g])
    ctx.grad_norm(r, norm.data_ptr(), stream())
    ctx.clip_grads(r, norm.data_ptr(), 1.0, stream())
    if math.isnan(bad):
        assert norm.isnan().all() and g.isnan().all() and h.isnan().all()
    else:
        assert norm.tolist() == [math.inf, math.inf]
        assert (g[:3999] == 0).all() and g[3999].isnan() and (h == 0).all()


def test_the_factor_at_one(ctx):
    """A norm of just max_norm is clipped by 1e-6 of itself, one a little below not at all, and the norm's root is not what clipping reads."""
    g = torch.full((4,), 0.5, device="cuda")
    for most, c in ((1.0, 1.0 / (1.0 + 1e-6)), (1.0 + 1e-6, 1.0), (1.1, 1.0)):
        a, norm = g.clone(), torch.tensor([1.0, math.nan], dtype=torch.float64, device="cuda")
        ctx.clip_grads(records([a]), norm.data_ptr(), most, stream())
        assert torch.equal(a, (g * torch.tensor(c, dtype=torch.float64).float().cuda()))


def test_sums_of_two_processes(ctx):
    """Two processes' shares: their sums of squares added up, each clips its own part as one would clip all."""
    ts = [v for _, v in tensors([3000, 5001], [F32, F32], 5)]
    whole, norm = [v.clone() for v in ts], torch.empty(3, 2, dtype=torch.float64, device="cuda")
    ctx.grad_norm(records(whole), norm[2].data_ptr(), stream())
    for k in range(2):
        ctx.grad_norm(records([ts[k]]), norm[k].data_ptr(), stream())
    total = norm[0] + norm[1]
    for k in range(2):
        ctx.clip_grads(records([ts[k]]), total.data_ptr(), 0.1, stream())
    ctx.clip_grads(records(whole), norm[2].data_ptr(), 0.1, stream())
    for a, b in zip(ts, whole):
        assert ((a - b).abs() <= 2 * U * b.abs()).all()


def test_many_argument_sets_and_streams(ctx):
    """More sets than tables are kept, on two streams in turn."""
    sets = [tensors([100 * k + 1, 3000], [F32, BF16], k) for k in range(12)]
    norms = torch.empty(12, 2, dtype=torch.float64, device="cuda")
    other = torch.cuda.Stream()
    for turn in range(2):
        for k, ts in enumerate(sets):
            r = records([v for _, v in ts])
            s = other if k % 2 else torch.cuda.current_stream()
            torch.cuda.synchronize()
            ctx.grad_norm(r, norms[k].data_ptr(), s.cuda_stream)
        torch.cuda.synchronize()
        for k, ts in enumerate(sets):
            check_norm(norms[k], [v for _, v in ts])


def test_recorded(ctx):
    """Replays, with the program's own calls of other arguments between them, against the eager result."""
    ts = tensors([70_001, 5, 3000], [BF16, F32, F32], 3)
    grads, start = [v for _, v in ts], [v.clone() for _, v in ts]
    norm, r = torch.zeros(2, dtype=torch.float64, device="cuda"), records([v for _, v in ts])
    others = [records([v for _, v in tensors([50 + k], [F32], k)]) for k in range(10)]
    keep = [tensors([50 + k], [F32], k) for k in range(10)]
    others = [records([v for _, v in t]) for t in keep]
    spare = torch.zeros(2, dtype=torch.float64, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            ctx.grad_norm(r, norm.data_ptr(), torch.cuda.current_stream().cuda_stream)
            ctx.clip_grads(r, norm.data_ptr(), 0.01, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for turn in range(4):
        for g, b in zip(grads, start):
            g.copy_(b * (turn + 1))
        eager = [g.clone() for g in grads]
        e_norm = torch.zeros(2, dtype=torch.float64, device="cuda")
        ctx.grad_norm(records(eager), e_norm.data_ptr(), stream())
        ctx.clip_grads(records(eager), e_norm.data_ptr(), 0.01, stream())
        for o in others:
            ctx.grad_norm(o, spare.data_ptr(), stream())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, e_norm)
        assert all(torch.equal(a, b) for a, b in zip(grads, eager))


def test_before_the_step(ctx):
    """Norm, clipping and the quantized step in a row, on gradients of one type, against the step on gradients clipped in torch."""
    from paper_2604_06836_amd import binding
    sizes, g = [5000, 2048, 333], torch.Generator("cuda").manual_seed(1)
    runs = []
    grads0 = [torch.randn(n, device="cuda", generator=g) for n in sizes]
    params0 = [torch.randn(n, device="cuda", generator=g) for n in sizes]
    for own in (True, False):
        params, grads = [p.clone() for p in params0], [x.clone() for x in grads0]
        keep, items = [], []
        for p, x in zip(params, grads):
            state = [torch.empty(b, dtype=torch.uint8, device="cuda") for _ in range(2) for b in stq.state_bytes(p.numel(), 64, 8)]
            keep.append(state)
            items.append(dict(param=p.data_ptr(), grad=x.data_ptr(), numel=p.numel(), m_codes=state[0].data_ptr(), m_scales=state[1].data_ptr(),
                              v_codes=state[2].data_ptr(), v_scales=state[3].data_ptr()))
        ts, plan = binding.make_tensors(items), binding.make_plan([(8, 8)] * 3)
        ctx.zero_state(ts, plan, 64, stream())
        for t in range(1, 4):
            for x, b in zip(grads, grads0):
                x.copy_(b * t)
            norm = torch.empty(2, dtype=torch.float64, device="cuda")
            r = records(grads)
            ctx.grad_norm(r, norm.data_ptr(), stream())
            if own:
                ctx.clip_grads(r, norm.data_ptr(), 0.5, stream())
            else:
                c = (0.5 / (norm[0].sqrt() + 1e-6)).clamp_max(1.0).float()
                for x in grads:
                    x.mul_(c)
            ctx.step(ts, plan, binding.HParams(1e-2, 0.9, 0.99, 1e-8, 0.0, t, 64, 0, 0), stream())
        torch.cuda.synchronize()
        runs.append(params)
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_refusals(ctx):
    g, norm, s = torch.ones(100, device="cuda"), torch.zeros(2, dtype=torch.float64, device="cuda"), stream()

    def code_of(call):
        with pytest.raises(stq.StqError) as e:
            call()
        return e.value.code

    def one(**change):
        r = records([g])
        for k, v in change.items():
            setattr(r[0], k, v)
        return r
    EINVAL, EALIGN, EDTYPE = -1, -2, -10
    for call in (lambda r, n=norm.data_ptr(): ctx.grad_norm(r, n, s), lambda r, n=norm.data_ptr(): ctx.clip_grads(r, n, 1.0, s)):
        assert code_of(lambda: call(one(grad=None))) == EINVAL
        assert code_of(lambda: call(one(dtype=2))) == EDTYPE
        assert code_of(lambda: call(one(grad=g.data_ptr() + 2))) == EALIGN
        assert code_of(lambda: call(one(out=g.data_ptr() + 1, dtype=1))) == EALIGN
        assert code_of(lambda: call(one(numel=1 << 60))) == EINVAL
        assert code_of(lambda: call(one(), None)) == EINVAL
        assert code_of(lambda: call(one(), norm.data_ptr() + 4)) == EALIGN
        assert code_of(lambda: call(records([g] * 701))) == EINVAL
    for most in (0.0, -1.0, math.nan, math.inf):
        assert code_of(lambda: ctx.clip_grads(one(), norm.data_ptr(), most, s)) == EINVAL
    torch.cuda.synchronize()
    assert (g == 1).all() and (norm == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_tensor_of_more_than_32_bits_of_elements(ctx, dtype):
    n = 2 ** 32 + 2051
    t = torch.zeros(n, dtype=dtype, device="cuda")
    at = torch.tensor([0, 2 ** 31 - 1, 2 ** 31, 2 ** 32 - 1, 2 ** 32, 2 ** 32 + 2047, n - 1], device="cuda")
    t[at] = torch.tensor([1.0, 2.0, 3.0, 4.0, 5.0, 6.0, 8.0], device="cuda").to(t.dtype)
    norm = torch.zeros(2, dtype=torch.float64, device="cuda")
    grads = stq.make_grads([dict(grad=t.data_ptr(), numel=n, dtype=KIND[dtype])])
    s = torch.cuda.current_stream().cuda_stream
    ctx.grad_norm(grads, norm.data_ptr(), s)
    assert norm[0].item() == 155.0  # exact in fp64
    before = t[at].double()
    ctx.clip_grads(grads, norm.data_ptr(), 1.0, s)
    c = 1.0 / (math.sqrt(155.0) + 1e-6)
    # the factor and the product each rounded to fp32, and to bf16
    off = 2.0 ** -24 * 2.01 + (2.0 ** -8 * 1.01 if dtype == BF16 else 0.0)
    assert ((t[at].double() - before * c).abs() <= off * before * c).all()
    t[at] = 0
    assert not any(part.any().item() for part in t.split(2 ** 28))
    del t
    torch.cuda.empty_cache()
