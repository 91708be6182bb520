"""A classifier's training step out of this library's calls: norm, codes, loss, its gradients, the norm's gradient, the global norm, clipping and
the quantized step, eagerly and as one graph.  The gradients are held to the formulas in 64 bits over the codes that the step has written, the
clipping to the norm of what it reads, the parameters to the step on gradients that are clipped in torch."""
import math

import pytest
import torch

import paper_2604_06836_amd as stq
from paper_2604_06836_amd import binding
from test_gpu_operators import U, Codes, matrix, stream

pytestmark = pytest.mark.gpu

T, D, V, EPS, MOST = 300, 128, 1003, 1e-6, 0.05


class Step:
    def __init__(self, ctx, seed, clip=True):
        g = torch.Generator("cuda").manual_seed(seed)
        self.ctx, self.clip = ctx, clip
        self.w, self.gain = torch.randn(V, D, device="cuda", generator=g) / D ** 0.5, 1 + 0.1 * torch.randn(D, device="cuda", generator=g)
        self.x, self.target = torch.randn(T, D, device="cuda", generator=g), torch.randint(0, V, (T,), device="cuda", generator=g)
        self.target[::7] = -1
        self.dloss = torch.full((T,), 1.0 / T, device="cuda")
        self.wq, self.y = Codes(V, D), Codes(T, D)
        self.total, self.rstd = torch.empty(T, D, device="cuda"), torch.empty(T, device="cuda")
        self.loss, self.lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
        self.dy, self.dx, self.dw, self.dgain = (torch.empty(*s, device="cuda") for s in ((T, D), (T, D), (V, D), (D,)))
        self.norm = torch.zeros(2, dtype=torch.float64, device="cuda")
        self.work = torch.empty(max(stq.cross_entropy_bytes(T, V, D), stq.cross_entropy_grad_bytes(T, V, D), stq.rms_norm_grad_bytes(T, D)), dtype=torch.uint8, device="cuda")
        self.grads = stq.make_grads([dict(grad=self.dw.data_ptr(), numel=V * D, dtype=stq.STQ_F32), dict(grad=self.dgain.data_ptr(), numel=D, dtype=stq.STQ_F32)])
        self.state, items = [], []
        for p, d in ((self.w, self.dw), (self.gain, self.dgain)):
            state = [torch.empty(b, dtype=torch.uint8, device="cuda") for _ in range(2) for b in stq.state_bytes(p.numel(), 64, 8)]
            self.state.append(state)
            items.append(dict(param=p.data_ptr(), grad=d.data_ptr(), numel=p.numel(), m_codes=state[0].data_ptr(), m_scales=state[1].data_ptr(),
                              v_codes=state[2].data_ptr(), v_scales=state[3].data_ptr()))
        self.tensors, self.plan = binding.make_tensors(items), binding.make_plan([(8, 8)] * 2)
        ctx.zero_state(self.tensors, self.plan, 64, stream())

    def gradients(self):
        c, s, size = self.ctx, stream(), self.work.numel()
        c.quantize_rows(matrix(self.w), self.wq.mat, s)
        c.rms_norm(matrix(self.x), None, self.gain.data_ptr(), EPS, matrix(self.total), self.y.mat, None, self.rstd.data_ptr(), s)
        c.cross_entropy(self.y.mat, self.wq.mat, self.target.data_ptr(), self.loss.data_ptr(), self.lse.data_ptr(), self.work.data_ptr(), size, s)
        c.cross_entropy_grad(self.y.mat, self.wq.mat, self.target.data_ptr(), self.loss.data_ptr(), self.lse.data_ptr(), self.dloss.data_ptr(), None,
                             matrix(self.dy), matrix(self.dw), self.work.data_ptr(), size, s)
        c.rms_norm_grad(matrix(self.total), self.gain.data_ptr(), self.rstd.data_ptr(), matrix(self.dy), None, matrix(self.dx), self.dgain.data_ptr(),
                        self.work.data_ptr(), size, s)

    def update(self, t):
        self.ctx.grad_norm(self.grads, self.norm.data_ptr(), stream())
        if self.clip:
            self.ctx.clip_grads(self.grads, self.norm.data_ptr(), MOST, stream())
        else:
            factor = (MOST / (self.norm[0].sqrt() + 1e-6)).clamp_max(1.0).float()
            self.dw.mul_(factor)
            self.dgain.mul_(factor)
        self.ctx.step(self.tensors, self.plan, binding.HParams(1e-2, 0.9, 0.99, 1e-8, 0.0, t, 64, 0, 0), stream())


@pytest.fixture(scope="module")
def ctx():
    c = stq.Context(0, 8)
    yield c
    torch.cuda.synchronize()
    c.close()


def test_steps(ctx):
    a, b = Step(ctx, 1), Step(ctx, 1, clip=False)
    for t in range(1, 5):
        for s in (a, b):
            s.gradients()
        y, w, there = a.y.value(), a.wq.value(), a.target >= 0
        z = y @ w.t()
        g = torch.softmax(z, 1)
        g[torch.arange(T, device="cuda")[there], a.target[there]] -= 1
        g *= (a.dloss.double() * there)[:, None]
        # a logit's roundings and the log-sum's, in the gradients' terms; sums of V and T products
        off = U * (40 * z.abs().max() + V / 16 + 200)
        for got, f, m, n in ((a.dy, g, w, V), (a.dw, g.t(), y, T)):
            assert ((got.double() - f @ m).abs() <= (off + 2.0 ** -22 + n * U) * (f.abs() @ m.abs()) + off * a.dloss[0].item() * 2.0 ** -20 * m.abs().sum(0)).all()
        before = [a.dw.clone(), a.dgain.clone()]
        want = sum((d.double() ** 2).sum() for d in before)
        for s in (a, b):
            s.update(t)
        assert abs(a.norm[0] - want).item() <= 1e-10 * want.item() and MOST < a.norm[1].item()
        c = MOST / (math.sqrt(want.item()) + 1e-6)
        for d, r in zip((a.dw, a.dgain), before):
            assert ((d.double() - c * r.double()).abs() <= 3 * U * c * r.double().abs() + 2.0 ** -149).all()
        assert torch.equal(a.w, b.w) and torch.equal(a.gain, b.gain)


def test_recorded_steps(ctx):
    """The gradients and their clipping as a graph, with the step behind it eager: the same parameters as without the graph."""
    a, b = Step(ctx, 2), Step(ctx, 2)
    b.gradients()  # (tables of the arguments are on the device)
    ctx.grad_norm(b.grads, b.norm.data_ptr(), stream())
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            b.gradients()
            ctx.grad_norm(b.grads, b.norm.data_ptr(), stream())
            ctx.clip_grads(b.grads, b.norm.data_ptr(), MOST, stream())
    torch.cuda.synchronize()
    for t in range(1, 5):
        a.gradients()
        a.update(t)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        ctx.step(b.tensors, b.plan, binding.HParams(1e-2, 0.9, 0.99, 1e-8, 0.0, t, 64, 0, 0), stream())
        torch.cuda.synchronize()
        assert torch.equal(a.loss, b.loss) and torch.equal(a.norm, b.norm) and torch.equal(a.w, b.w) and torch.equal(a.gain, b.gain)
