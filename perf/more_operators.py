"""The two ends of a backward pass as a training program calls them: the loss of a classifier over 8-bit codes with its gradients,
without its logits in memory, and the norm of all gradients together with their clipping.

The classifier's logits are z[t][v] = xs[t] ws[v] sum over i of xq[t][i] wq[v][i], x and w in int8 codes with a scale for each row.  A
token whose target is negative has no loss.  Gradients of many tensors of both float types lie in one buffer for each type, as a program's
gradient buckets do.  `prepare` makes what a program has in hand; `run` is one pass.
"""
from __future__ import annotations

import random

import torch

own = False  # whether run() calls the library's operators, or computes them by elementary torch operations
TYPES = dict(bf16=torch.bfloat16, fp32=torch.float32)
GAP = 64     # tensors begin at multiples of so many elements of their buffer


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # scoring the next token of a single sequence: the classifier's bytes are all that counts
        dict(name="loss one token", op="loss", tokens=1, classes=32000, inn=4096),
        # evaluation of a short ragged batch, of a width that no vector divides
        dict(name="loss ragged", op="loss", tokens=333, classes=5003, inn=1001),
        # one training step's tokens through the classifier of a 4096-wide model: the largest forward pass
        dict(name="loss training", op="loss", tokens=16384, classes=32000, inn=4096),
        # fine-tuning a small model on an odd number of tokens, gradients in fp32
        dict(name="loss grad small", op="loss_grad", tokens=601, classes=5003, inn=768, type="fp32"),
        # a 768-wide model with a vocabulary of 50257, whose rows no vector divides
        dict(name="loss grad odd classes", op="loss_grad", tokens=4096, classes=50257, inn=768, type="bf16"),
        # the classifier of a 4096-wide model at a training step's tokens: the largest call
        dict(name="loss grad training", op="loss_grad", tokens=8192, classes=32000, inn=4096, type="bf16"),
        # a small network's odd-sized tensors: the call is little more than its launches
        dict(name="norm ragged small", op="norm", shapes="ragged", count=24, largest=40001, vectors="fp32"),
        # a small language model whose matrices have gradients in bf16 and whose vectors in fp32
        dict(name="norm 124 M", op="norm", shapes="model", d=768, layers=12, vocab=50257, vectors="fp32"),
        # one GPU's share of a 7 B model
        dict(name="norm 3.5 G", op="norm", shapes="slice", total=3_500_000_000, vectors="bf16"),
        # norm and clipping of a small network's tensors
        dict(name="clip ragged small", op="clip", shapes="ragged", count=24, largest=40001, vectors="fp32", most=0.1),
        # of a small language model
        dict(name="clip 124 M", op="clip", shapes="model", d=768, layers=12, vocab=50257, vectors="fp32", most=1.0),
        # of a 1600-wide model with 48 layers
        dict(name="clip 1.56 G", op="clip", shapes="model", d=1600, layers=48, vocab=50257, vectors="bf16", most=1.0),
    ]


def _size(rng, low, high):
    """Spread over the logarithm; half of them multiples of 64, the rest as they come."""
    n = int(low * (high / low) ** rng.random())
    return max(low, n // 64 * 64) if rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(["loss", "loss_grad", "loss_grad", "norm", "clip", "clip"])
    if op in ("loss", "loss_grad"):
        most = 16384 * 32000 * 4096 if op == "loss" else 8192 * 32000 * 4096
        while True:
            tokens, classes, inn = _size(rng, 1 if op == "loss" else 32, 16384), _size(rng, 500, 65000), _size(rng, 64, 8192)
            if tokens * classes * inn <= most and tokens * classes <= 16384 * 32000:
                break
        c = dict(op=op, tokens=tokens, classes=classes, inn=inn)
        return c if op == "loss" else dict(c, type=rng.choice(["bf16", "bf16", "fp32"]))
    c = dict(op=op, vectors=rng.choice(["bf16", "fp32"]), shapes=rng.choice(["ragged", "model", "slice"]))
    if c["shapes"] == "ragged":
        c.update(count=int(10 ** rng.uniform(0, 2.8)), largest=int(10 ** rng.uniform(2.5, 6.3)))
    elif c["shapes"] == "model":
        c.update(d=64 * int(2 ** rng.uniform(1, 4.4)), layers=rng.randrange(2, 37), vocab=rng.choice([5003, 32000, 50257]))
    else:
        c.update(total=int(10 ** rng.uniform(7, 9.15)))
    return c if op == "norm" else dict(c, most=10 ** rng.uniform(-2, 1))


# ----------------------------------------------------------------------------------------------- inputs
def _normal(g, rows, cols, of_rows=0.3, of_cols=0.5):
    """Normal values with a size of their own for each row and column, a few columns far larger than the rest."""
    x = torch.randn(rows, cols, device="cuda", generator=g)
    sizes = torch.exp(of_cols * torch.randn(cols, device="cuda", generator=g))
    sizes[torch.rand(cols, device="cuda", generator=g) < 0.002] *= 20.0
    return x.mul_(sizes).mul_(torch.exp(of_rows * torch.randn(rows, 1, device="cuda", generator=g)))


def _codes(x):
    largest = x.abs().amax(1, keepdim=True).clamp_min(2.0 ** -100)
    return torch.round(x * (127.0 / largest)).to(torch.int8), (largest / 127.0).view(-1)


def _loss_inputs(case, g):
    """Hidden states that point to their target's weights, more or less: tokens predicted with certainty, well, badly and not at all."""
    t, v, n = case["tokens"], case["classes"], case["inn"]
    w = _normal(g, v, n, of_cols=0.1)
    x = _normal(g, t, n)
    target = (v * torch.rand(t, device="cuda", generator=g).pow(3)).long().clamp_max(v - 1)  # some classes far more often than others
    near = w[target]
    x = x / x.square().mean(1, keepdim=True).sqrt() + near * (0.25 * torch.rand(t, 1, device="cuda", generator=g))
    w *= 2.0 / n ** 0.5
    if t > 8:  # padding and prompts
        target[torch.rand(t, device="cuda", generator=g) < 0.1] = -100
    s = dict(case=case, target=target)
    s["xq"], s["xs"] = _codes(x)
    s["wq"], s["ws"] = _codes(w)
    return s


def _sizes(case):
    kind = case["shapes"]
    if kind == "ragged":
        r = random.Random(case["count"])
        return [max(1, int(case["largest"] ** r.random())) for _ in range(case["count"])] + [case["largest"]]
    if kind == "model":
        d = case["d"]
        return [case["vocab"] * d, 1024 * d] + [d, d, 3 * d * d, d * d, d, d, 4 * d * d, 4 * d * d] * case["layers"] + [d, d]
    d, f, out, left = 4096, 11008, [], case["total"]  # a contiguous slice of a 7 B model, cut at `total` elements
    for n in [32000 * d] + [d, d * d, d * d, d * d, d * d, d, d * f, d * f, f * d] * 32:
        if left:
            out.append(min(n, left))
            left -= out[-1]
    return out


def _layout(case):
    """(type, first element, elements) of each tensor, and the elements of each type's buffer."""
    ends, places = dict(bf16=0, fp32=0), []
    for n in _sizes(case):
        kind = case["vectors"] if n < 65536 else "bf16"
        places.append((kind, ends[kind], n))
        ends[kind] += -(-n // GAP) * GAP
    return places, ends


def _gradient_inputs(case, g):
    places, ends = _layout(case)
    s = dict(case=case, places=places)
    s["grads"] = {k: torch.zeros(n, dtype=TYPES[k], device="cuda") for k, n in ends.items() if n}
    sizes = torch.exp(torch.randn(len(places), generator=g, device="cuda")).tolist()
    for (kind, at, n), size in zip(places, sizes):
        s["grads"][kind][at:at + n].normal_(0.0, 1e-3 * size, generator=g)
    if case["op"] == "clip":
        s["outs"] = {k: torch.zeros_like(t) for k, t in s["grads"].items()}
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if case["op"] in ("norm", "clip"):
        return _gradient_inputs(case, g)
    s = _loss_inputs(case, g)
    if case["op"] == "loss_grad":  # what the forward pass left, and the gradient of a mean over tokens of different weight
        s["loss"], s["lse"] = _forward(s)
        weight = torch.exp(0.3 * torch.randn(case["tokens"], device="cuda", generator=g))
        s["dloss"] = weight / weight.sum()
    return s


# ------------------------------------------------------------------------------------------- plain form
def _logits(s):
    return (s["xq"].float() @ s["wq"].float().t()) * s["xs"][:, None] * s["ws"]


def _forward(s):
    z, target = _logits(s), s["target"]
    most = z.amax(1)
    lse = most + torch.exp(z - most[:, None]).sum(1).log()
    at = z.gather(1, target.clamp_min(0)[:, None])[:, 0]
    return torch.where(target < 0, torch.zeros_like(lse), lse - at), lse


def _plain(s):
    case = s["case"]
    if case["op"] == "loss":
        loss, lse = _forward(s)
        return dict(loss=loss, lse=lse)
    if case["op"] == "loss_grad":
        d = torch.where(s["target"] < 0, torch.zeros_like(s["dloss"]), s["dloss"])
        dz = _logits(s).sub_(s["lse"][:, None]).exp_().mul_(d[:, None])
        dz.scatter_add_(1, s["target"].clamp_min(0)[:, None], -d[:, None])
        dx = dz @ (s["wq"].float() * s["ws"][:, None])
        dw = dz.t() @ (s["xq"].float() * s["xs"][:, None])
        return dict(dx=dx.to(TYPES[case["type"]]), dw=dw.to(TYPES[case["type"]]))
    total = sum(t.double().square().sum() for t in s["grads"].values())
    norm = total.sqrt()
    if case["op"] == "norm":
        return dict(norm=torch.stack([total, norm]))
    factor = (case["most"] / (norm + 1e-6)).clamp_max(1.0).float()
    return dict(norm=torch.stack([total, norm]), grads={k: (t.float() * factor).to(t.dtype) for k, t in s["grads"].items()})


# ------------------------------------------------------------------------------------ the library's calls
_library = {}


def _context():
    """The context that a program opens once."""
    if not _library:
        import paper_2604_06836_amd as stq
        _library["stq"], _library["ctx"] = stq, stq.Context(0, 1024)
    return _library["stq"], _library["ctx"]


def _matrix(stq, t, scales=None):
    kind = {torch.float32: stq.STQ_F32, torch.bfloat16: stq.STQ_BF16, torch.int8: stq.STQ_Q8}[t.dtype]
    return stq.make_matrix(t.data_ptr(), t.shape[0], t.shape[1], kind, stride=t.stride(0),
                           scales=scales.data_ptr() if scales is not None else None)


def _arrange(s):
    """The buffers that a program keeps for its outputs, and the records that describe all of them to the library."""
    stq, ctx = _context()
    case = s["case"]
    a = dict(ctx=ctx)
    if case["op"] in ("loss", "loss_grad"):
        t, v, n = case["tokens"], case["classes"], case["inn"]
        a["x"], a["w"] = _matrix(stq, s["xq"], s["xs"]), _matrix(stq, s["wq"], s["ws"])
        if case["op"] == "loss":
            a["bytes"] = stq.cross_entropy_bytes(t, v, n)
            a["out"] = dict(loss=torch.empty(t, device="cuda"), lse=torch.empty(t, device="cuda"))
        else:
            a["bytes"] = stq.cross_entropy_grad_bytes(t, v, n)
            a["out"] = {k: torch.empty(r, n, dtype=TYPES[case["type"]], device="cuda") for k, r in (("dx", t), ("dw", v))}
            a["dx"], a["dw"] = _matrix(stq, a["out"]["dx"]), _matrix(stq, a["out"]["dw"])
        a["work"] = torch.empty(max(a["bytes"], 1), dtype=torch.uint8, device="cuda")
        return a
    norm, outs = torch.empty(2, dtype=torch.float64, device="cuda"), s.get("outs")
    at = lambda bufs, kind, first: bufs[kind].data_ptr() + first * bufs[kind].element_size()  # noqa: E731
    a["grads"] = stq.make_grads(dict(grad=at(s["grads"], kind, first), out=at(outs, kind, first) if outs else None, numel=n,
                                     dtype=dict(fp32=stq.STQ_F32, bf16=stq.STQ_BF16)[kind]) for kind, first, n in s["places"])
    a["norm"] = norm.data_ptr()
    a["out"] = dict(norm=norm, grads=outs) if outs else dict(norm=norm)
    return a


def _calls(s):
    a = s.get("args")
    if a is None:
        a = s["args"] = _arrange(s)
    ctx, op = a["ctx"], s["case"]["op"]
    stream = torch.cuda.current_stream().cuda_stream
    if op == "loss":
        ctx.cross_entropy(a["x"], a["w"], s["target"].data_ptr(), a["out"]["loss"].data_ptr(), a["out"]["lse"].data_ptr(),
                          a["work"].data_ptr(), a["bytes"], stream)
    elif op == "loss_grad":
        ctx.cross_entropy_grad(a["x"], a["w"], s["target"].data_ptr(), s["loss"].data_ptr(), s["lse"].data_ptr(), s["dloss"].data_ptr(), None,
                               a["dx"], a["dw"], a["work"].data_ptr(), a["bytes"], stream)
    else:
        ctx.grad_norm(a["grads"], a["norm"], stream)
        if op == "clip":
            ctx.clip_grads(a["grads"], a["norm"], s["case"]["most"], stream)
    return a["out"]


def run(state):
    return _calls(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------- work, exact
def work(case):
    """Inputs once, outputs once; of a clipping pass the gradients once, since the norm comes before it on another reading."""
    size = dict(bf16=2, fp32=4)
    if case["op"] in ("loss", "loss_grad"):
        t, v, n = case["tokens"], case["classes"], case["inn"]
        read = t * n + v * n + 4 * (t + v) + 8 * t
        if case["op"] == "loss":
            return dict(bytes=read + 8 * t, flops=2 * t * v * n)
        return dict(bytes=read + 12 * t + (t + v) * n * size[case["type"]], flops=6 * t * v * n)
    places, _ = _layout(case)
    every, bytes_ = sum(n for _, _, n in places), sum(n * size[kind] for kind, _, n in places)
    if case["op"] == "norm":
        return dict(bytes=bytes_ + 16, flops=2 * every)
    return dict(bytes=2 * bytes_ + 16, flops=3 * every)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("loss", "loss_grad"):
        x, w = s["xq"].double() * s["xs"].double()[:, None], s["wq"].double() * s["ws"].double()[:, None]
        z, there = x @ w.t(), s["target"] >= 0
        rows = torch.arange(case["tokens"], device="cuda")[there]
        if case["op"] == "loss":
            lse = torch.logsumexp(z, 1)
            loss = torch.zeros_like(lse)
            loss[there] = lse[there] - z[rows, s["target"][there]]
            return dict(loss=loss, lse=lse)
        p = torch.softmax(z, 1)
        p[rows, s["target"][there]] -= 1.0
        p *= (s["dloss"].double() * there)[:, None]
        return dict(dx=p @ w, dw=p.t() @ x)
    total = 0.0
    for t in s["grads"].values():
        for part in t.split(1 << 28):
            total = total + (part.double() ** 2).sum()
    norm = torch.sqrt(total)
    if case["op"] == "norm":
        return dict(norm=torch.stack([total, norm]))
    factor = torch.minimum(case["most"] / (norm + 1e-6), torch.ones_like(norm))
    return dict(norm=torch.stack([total, norm]), grads={k: t.double() * factor for k, t in s["grads"].items()})
