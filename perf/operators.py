"""The operators of an 8-bit training layer as a user calls them: the norm that writes codes, the products over codes and
their gradients, the gated activation whose inputs are kept in 8 bits, and the conversion of matrices to codes and back.

A matrix in 8 bits is int8 codes, -127 to 127, with a scale in fp32 for each row, or for each `block` columns of a row:
x = scale * code, scale = max|x| / 127.  `prepare` makes what a training or serving program has in hand; `run` is one
pass.  Codes that a pass writes are returned as the values they stand for, read back by the library's own call.
"""
from __future__ import annotations

import torch

own = False      # whether run() calls the library's operators, or computes them by elementary torch operations
EPS = 1e-5       # of the norm
LEAST = 2.0 ** -100  # a row's largest magnitude counts as at least this much, so that a row of zeros has codes
TYPES = dict(bf16=torch.bfloat16, fp32=torch.float32)


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # serving a single token: the gate projection of a 4096-wide layer, where the weights' bytes are all that counts
        dict(name="product one token", op="matmul", tokens=1, out=11008, inn=4096, type="bf16"),
        # the classifier of a 768-wide model over a ragged batch of tokens, with logits in fp32
        dict(name="product ragged", op="matmul", tokens=333, out=1000, inn=768, type="fp32"),
        # one training step's tokens through the gate projection of a 4096-wide layer: the largest product
        dict(name="product training", op="matmul", tokens=16384, out=11008, inn=4096, type="bf16"),
        # the gradient with respect to the input of the down projection (11008 to 4096)
        dict(name="grad input", op="grad_input", tokens=8192, out=4096, inn=11008, grad="bf16", type="bf16"),
        # the gradient of a 768 by 768 projection over an odd number of tokens, accumulated as fp32 gradients are
        dict(name="grad weight small", op="grad_weight", tokens=5001, out=768, inn=768, grad="bf16", type="fp32"),
        # the gradient of the gate projection, in the bf16 that the optimizer's step reads
        dict(name="grad weight training", op="grad_weight", tokens=8192, out=11008, inn=4096, grad="bf16", type="bf16"),
        # serving a single token: the residual's addition and the norm, with the codes for the projections
        dict(name="norm one token", op="norm", rows=1, cols=4096, type="bf16", block=0, keep=False),
        # training: the same over a step's tokens, with the sum kept in 8 bits for the backward pass
        dict(name="norm training", op="norm", rows=16384, cols=4096, type="bf16", block=128, keep=True),
        # the backward pass of a 1600-wide model's norm from the sum kept in 8 bits, with the residual's own gradient
        dict(name="norm grad", op="norm_grad", rows=8192, cols=1600, saved="q8", block=64, grad="bf16"),
        # the weights of a gate projection to codes, once per optimizer step
        dict(name="weights to codes", op="codes", rows=11008, cols=4096, type="fp32", block=0),
        # training: the activation between the projections, both inputs out of one product, kept in 8 bits
        dict(name="gated training", op="gated", rows=8192, cols=11008, type="bf16", block=128, keep=True),
        # its backward pass from the codes, at an odd width of rows that no vector divides
        dict(name="gated grad ragged", op="gated_grad", rows=2049, cols=2731, saved="q8", block=64, grad="bf16"),
    ]


def _size(rng, low, high):
    """Spread over the logarithm; half of them multiples of 64, the rest as they come."""
    n = int(low * (high / low) ** rng.random())
    if rng.random() < 0.5:
        n = max(low, n // 64 * 64)
    return n + 64 if n == 3072 else n


def draw(rng):
    op = rng.choice(["matmul", "matmul", "grad_input", "grad_weight", "norm", "norm_grad", "gated", "gated_grad", "codes"])
    any_type = rng.choice(["bf16", "bf16", "fp32"])
    if op in ("matmul", "grad_input", "grad_weight"):
        most = 16384 * 11008 * 4096 if op == "matmul" else 8192 * 11008 * 4096
        while True:
            tokens, out, inn = _size(rng, 1 if op == "matmul" else 16, 16384), _size(rng, 64, 16384), _size(rng, 64, 16384)
            if tokens * out * inn <= most:
                break
        c = dict(op=op, tokens=tokens, out=out, inn=inn, type=any_type)
        return c if op == "matmul" else dict(c, grad=rng.choice(["bf16", "bf16", "fp32"]))
    while True:
        rows, cols = _size(rng, 1, 16384), _size(rng, 64, 16384)
        if rows * cols <= 8192 * 11008:
            break
    block = rng.choice([0, 64, 128, 256])
    if op in ("norm", "gated"):
        return dict(op=op, rows=rows, cols=cols, type=any_type, block=block, keep=rng.random() < 0.7)
    if op == "codes":
        return dict(op=op, rows=rows, cols=cols, type=any_type, block=block)
    return dict(op=op, rows=rows, cols=cols, saved=rng.choice(["q8", "q8", "bf16", "fp32"]), block=block, grad=any_type)


# ----------------------------------------------------------------------------------------------- inputs
def _normal(g, rows, cols, of_rows=0.3, of_cols=0.5):
    """Normal values with a size of their own for each row and column, a few columns far larger than the rest."""
    x = torch.randn(rows, cols, device="cuda", generator=g)
    sizes = torch.exp(of_cols * torch.randn(cols, device="cuda", generator=g))
    sizes[torch.rand(cols, device="cuda", generator=g) < 0.002] *= 20.0
    return x.mul_(sizes).mul_(torch.exp(of_rows * torch.randn(rows, 1, device="cuda", generator=g)))


def _gradient(g, rows, cols, kind):
    """A gradient of activations: small, of different size from token to token, and nothing where the loss is masked."""
    d = 1e-3 * _normal(g, rows, cols, of_rows=1.0)
    if rows > 8:
        d[torch.rand(rows, device="cuda", generator=g) < 0.05] = 0.0
    return d.to(TYPES[kind])


def _codes(x, block):
    """Codes (as fp32) and scales of a matrix: one scale a row where `block` is 0, else one for each `block` columns."""
    rows, cols = x.shape
    width = block or cols
    pad = -cols % width
    groups = torch.nn.functional.pad(x, (0, pad)).view(rows, -1, width)
    largest = groups.abs().amax(2, keepdim=True).clamp_min(LEAST)
    q = torch.round(groups * (127.0 / largest)).view(rows, cols + pad)[:, :cols]
    return q, (largest / 127.0).squeeze(2)


def _values(q, scales, block):
    cols = q.shape[1]
    width = block or cols
    return q * scales.to(q.dtype).repeat_interleave(width, 1)[:, :cols]


def _kept(g, x, saved, block):
    """An activation as the forward pass left it: in 8 bits, or as it is."""
    if saved != "q8":
        return dict(x=x.to(TYPES[saved]))
    q, scales = _codes(x, block)
    return dict(q=q.to(torch.int8), scales=scales)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(case=case)
    op = case["op"]
    if op in ("matmul", "grad_input", "grad_weight"):
        m, n, k = case["tokens"], case["out"], case["inn"]
        if op != "grad_input":
            q, scales = _codes(_normal(g, m, k), 0)
            s.update(xq=q.to(torch.int8), xs=scales.view(-1))
        if op != "grad_weight":
            q, scales = _codes(0.02 * _normal(g, n, k, of_cols=0.1), 0)
            s.update(wq=q.to(torch.int8), ws=scales.view(-1))
        if op != "matmul":
            s["dy"] = _gradient(g, m, n, case["grad"])
        return s
    rows, cols = case["rows"], case["cols"]
    if op == "norm":
        s["x"] = _normal(g, rows, cols).to(TYPES[case["type"]])
        s["residual"] = (2.0 * _normal(g, rows, cols)).to(TYPES[case["type"]])
        if rows > 8:  # padding tokens
            s["x"][rows // 2] = 0.0
            s["residual"][rows // 2] = 0.0
        s["weight"] = 1.0 + 0.2 * torch.randn(cols, device="cuda", generator=g)
    elif op == "norm_grad":
        x = _normal(g, rows, cols)
        s["rstd"] = (x.square().mean(1) + EPS).rsqrt()
        s["kept"] = _kept(g, x, case["saved"], case["block"])
        s["weight"] = 1.0 + 0.2 * torch.randn(cols, device="cuda", generator=g)
        s["dy"] = _gradient(g, rows, cols, case["grad"])
        s["dresidual"] = _gradient(g, rows, cols, case["grad"])
    elif op == "codes":
        s["x"] = (0.02 * _normal(g, rows, cols, of_cols=0.1)).to(TYPES[case["type"]])
    elif op == "gated":  # gate and up beside each other, as one product leaves them
        s["both"] = _normal(g, rows, 2 * cols).to(TYPES[case["type"]])
    else:
        s["gate"] = _kept(g, _normal(g, rows, cols), case["saved"], case["block"])
        s["up"] = _kept(g, _normal(g, rows, cols), case["saved"], case["block"])
        s["dy"] = _gradient(g, rows, cols, case["grad"])
    return s


# ------------------------------------------------------------------------------------------- plain form
def _read(kept, block):
    return kept["x"].float() if "x" in kept else _values(kept["q"].float(), kept["scales"], block)


def _written(x, block):
    """What a matrix is read back as after its conversion, in bf16, and the scales."""
    q, scales = _codes(x, block)
    return _values(q, scales, block).to(torch.bfloat16), scales


def _plain(s):
    case = s["case"]
    op, block = case["op"], case.get("block", 0)
    if op == "matmul":
        y = s["xq"].float() @ s["wq"].float().t()
        return dict(y=(y * s["xs"][:, None] * s["ws"]).to(TYPES[case["type"]]))
    if op == "grad_input":
        return dict(dx=(s["dy"].float() @ (s["wq"].float() * s["ws"][:, None])).to(TYPES[case["type"]]))
    if op == "grad_weight":
        return dict(dw=(s["dy"].float().t() @ (s["xq"].float() * s["xs"][:, None])).to(TYPES[case["type"]]))
    if op == "norm":
        total = (s["x"].float() + s["residual"].float()).to(s["x"].dtype)
        h = total.float()
        rstd = (h.square().mean(1) + EPS).rsqrt()
        y, scales = _written(h * rstd[:, None] * s["weight"], 0)
        r = dict(total=total, rstd=rstd, y=y, scales=scales)
        if case["keep"]:
            r["kept"], r["kept_scales"] = _written(h, block)
        return r
    if op == "norm_grad":
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        xhat = _read(s["kept"], block) * rstd
        dxhat = dy * s["weight"]
        dx = rstd * (dxhat - xhat * (dxhat * xhat).mean(1, keepdim=True)) + s["dresidual"].float()
        return dict(dx=dx.to(s["dy"].dtype), dweight=(dy * xhat).sum(0))
    if op == "codes":
        value, scales = _written(s["x"].float(), block)
        return dict(value=value, scales=scales)
    if op == "gated":
        gate, up = (t.float() for t in s["both"].chunk(2, 1))
        y, scales = _written(gate / (1.0 + torch.exp(-gate)) * up, 0)
        r = dict(y=y, scales=scales)
        if case["keep"]:
            r["gate"], r["gate_scales"] = _written(gate, block)
            r["up"], r["up_scales"] = _written(up, block)
        return r
    gate, up, dy = _read(s["gate"], block), _read(s["up"], block), s["dy"].float()
    sigma = 1.0 / (1.0 + torch.exp(-gate))
    dgate = dy * up * (sigma * (1.0 + gate * (1.0 - sigma)))
    return dict(both=torch.cat([dgate, dy * (gate * sigma)], 1).to(s["dy"].dtype))


# ------------------------------------------------------------------------------------ the library's calls
_library = {}


def _context():
    """The context that a program opens once."""
    if not _library:
        import paper_2604_06836_amd as stq
        _library["stq"], _library["ctx"] = stq, stq.Context(0, 8)
    return _library["stq"], _library["ctx"]


def _matrix(stq, t, scales=None, block=0):
    kind = {torch.float32: stq.STQ_F32, torch.bfloat16: stq.STQ_BF16, torch.int8: stq.STQ_Q8}[t.dtype]
    return stq.make_matrix(t.data_ptr(), t.shape[0], t.shape[1], kind, stride=t.stride(0),
                           scales=scales.data_ptr() if scales is not None else None, block=block)


def _arrange(s):
    """The buffers that a program keeps for a layer's outputs, and the records that describe them to the library."""
    stq, ctx = _context()
    case = s["case"]
    op, block = case["op"], case.get("block", 0)
    a = dict(ctx=ctx)

    def new(rows, cols, dtype):
        return torch.empty(rows, cols, dtype=dtype, device="cuda")

    def codes(rows, cols, block):
        q, scales = new(rows, cols, torch.int8), new(rows, -(-cols // block) if block else 1, torch.float32)
        back = new(rows, cols, torch.bfloat16)
        return _matrix(stq, q, scales, block), _matrix(stq, back), back, scales, q

    def kept(k):
        return _matrix(stq, k["x"]) if "x" in k else _matrix(stq, k["q"], k["scales"], block)

    if op in ("matmul", "grad_input", "grad_weight"):
        m, n, k = case["tokens"], case["out"], case["inn"]
        if "xq" in s:
            a["x"] = _matrix(stq, s["xq"], s["xs"])
        if "wq" in s:
            a["w"] = _matrix(stq, s["wq"], s["ws"])
        if "dy" in s:
            a["dy"] = _matrix(stq, s["dy"])
        rows, cols, name = dict(matmul=(m, n, "y"), grad_input=(m, k, "dx"), grad_weight=(n, k, "dw"))[op]
        out = new(rows, cols, TYPES[case["type"]])
        a["to"], a["out"] = _matrix(stq, out), {name: out}
        if op == "grad_weight":
            a["bytes"] = stq.matmul_grad_weight_bytes(m, n, k)
            a["work"] = torch.empty(max(a["bytes"], 1), dtype=torch.uint8, device="cuda")
        return a
    rows, cols = case["rows"], case["cols"]
    if op == "norm":
        total, rstd = torch.empty_like(s["x"]), torch.empty(rows, device="cuda")
        a["x"], a["residual"], a["total"] = (_matrix(stq, t) for t in (s["x"], s["residual"], total))
        a["y"], a["y_back"], y, scales, a["q"] = codes(rows, cols, 0)
        a["out"] = dict(total=total, rstd=rstd, y=y, scales=scales)
        a["kept"] = None
        if case["keep"]:
            a["kept"], a["kept_back"], a["out"]["kept"], a["out"]["kept_scales"], a["kq"] = codes(rows, cols, block)
    elif op == "norm_grad":
        dx, dweight = torch.empty_like(s["dy"]), torch.empty(cols, device="cuda")
        a["kept"] = kept(s["kept"])
        a["dy"], a["dresidual"], a["dx"] = (_matrix(stq, t) for t in (s["dy"], s["dresidual"], dx))
        a["bytes"] = stq.rms_norm_grad_bytes(rows, cols)
        a["work"] = torch.empty(max(a["bytes"], 1), dtype=torch.uint8, device="cuda")
        a["out"] = dict(dx=dx, dweight=dweight)
    elif op == "codes":
        a["x"] = _matrix(stq, s["x"])
        a["y"], a["y_back"], y, scales, a["q"] = codes(rows, cols, block)
        a["out"] = dict(value=y, scales=scales)
    elif op == "gated":
        a["gate"], a["up"] = (_matrix(stq, t) for t in s["both"].chunk(2, 1))
        a["y"], a["y_back"], y, scales, a["q"] = codes(rows, cols, 0)
        a["out"] = dict(y=y, scales=scales)
        a["kgate"] = a["kup"] = None
        if case["keep"]:
            a["kgate"], a["gate_back"], a["out"]["gate"], a["out"]["gate_scales"], a["gq"] = codes(rows, cols, block)
            a["kup"], a["up_back"], a["out"]["up"], a["out"]["up_scales"], a["uq"] = codes(rows, cols, block)
    else:
        both = new(rows, 2 * cols, s["dy"].dtype)
        a["gate"], a["up"], a["dy"] = kept(s["gate"]), kept(s["up"]), _matrix(stq, s["dy"])
        a["dgate"], a["dup"] = (_matrix(stq, t) for t in both.chunk(2, 1))
        a["out"] = dict(both=both)
    return a


def _calls(s):
    a = s.get("args")
    if a is None:
        a = s["args"] = _arrange(s)
    ctx, op = a["ctx"], s["case"]["op"]
    stream = torch.cuda.current_stream().cuda_stream
    if op == "matmul":
        ctx.matmul(a["x"], a["w"], a["to"], stream)
    elif op == "grad_input":
        ctx.matmul_grad_input(a["dy"], a["w"], a["to"], stream)
    elif op == "grad_weight":
        ctx.matmul_grad_weight(a["dy"], a["x"], a["to"], a["work"].data_ptr(), a["bytes"], stream)
    elif op == "norm":
        ctx.rms_norm(a["x"], a["residual"], s["weight"].data_ptr(), EPS, a["total"], a["y"], a["kept"],
                     a["out"]["rstd"].data_ptr(), stream)
        ctx.dequantize_rows(a["y"], a["y_back"], stream)
        if a["kept"] is not None:
            ctx.dequantize_rows(a["kept"], a["kept_back"], stream)
    elif op == "norm_grad":
        ctx.rms_norm_grad(a["kept"], s["weight"].data_ptr(), s["rstd"].data_ptr(), a["dy"], a["dresidual"], a["dx"],
                          a["out"]["dweight"].data_ptr(), a["work"].data_ptr(), a["bytes"], stream)
    elif op == "codes":
        ctx.quantize_rows(a["x"], a["y"], stream)
        ctx.dequantize_rows(a["y"], a["y_back"], stream)
    elif op == "gated":
        ctx.gated_silu(a["gate"], a["up"], a["y"], a["kgate"], a["kup"], stream)
        ctx.dequantize_rows(a["y"], a["y_back"], stream)
        if a["kgate"] is not None:
            ctx.dequantize_rows(a["kgate"], a["gate_back"], stream)
            ctx.dequantize_rows(a["kup"], a["up_back"], stream)
    else:
        ctx.gated_silu_grad(a["gate"], a["up"], a["dy"], a["dgate"], a["dup"], stream)
    return a["out"]


def run(state):
    return _calls(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------- work, exact
def work(case):
    """Inputs once, outputs once: the codes that a pass writes, and the values that it reads them back as."""
    op, block = case["op"], case.get("block", 0)
    size = dict(bf16=2, fp32=4, q8=1)
    if op in ("matmul", "grad_input", "grad_weight"):
        m, n, k = case["tokens"], case["out"], case["inn"]
        bytes_ = dict(matmul=m * k + n * k + 4 * (m + n) + m * n * size[case["type"]],
                      grad_input=m * n * size[case.get("grad", "bf16")] + n * k + 4 * n + m * k * size[case["type"]],
                      grad_weight=m * n * size[case.get("grad", "bf16")] + m * k + 4 * m + n * k * size[case["type"]])[op]
        return dict(bytes=bytes_, flops=2 * m * n * k)
    rows, cols = case["rows"], case["cols"]
    every = rows * cols
    scales = 4 * rows * (-(-cols // block) if block else 1)
    if op == "norm":
        bytes_ = every * (3 * size[case["type"]] + 3) + 8 * rows + 4 * cols + (every * 3 + scales if case["keep"] else 0)
        return dict(bytes=bytes_, flops=8 * every)
    if op == "norm_grad":
        kept = every * size[case["saved"]] + (scales if case["saved"] == "q8" else 0)
        return dict(bytes=kept + 3 * every * size[case["grad"]] + 4 * rows + 8 * cols, flops=10 * every)
    if op == "codes":
        return dict(bytes=every * (size[case["type"]] + 3) + scales, flops=4 * every)
    if op == "gated":
        return dict(bytes=every * (2 * size[case["type"]] + 3) + 4 * rows + (2 * (every * 3 + scales) if case["keep"] else 0),
                    flops=12 * every)
    kept = 2 * (every * size[case["saved"]] + (scales if case["saved"] == "q8" else 0))
    return dict(bytes=kept + 3 * every * size[case["grad"]], flops=12 * every)


def exact(case, seed):
    s = prepare(case, seed)
    op, block = case["op"], case.get("block", 0)

    def through(v, width):
        """v after its conversion to codes and back, and the scales."""
        width = width or v.shape[1]
        scales = torch.stack([p.abs().amax(1) for p in v.split(width, 1)], 1).clamp_min(LEAST) / 127.0
        each = scales.repeat_interleave(width, 1)[:, :v.shape[1]]
        return torch.round(v / each) * each, scales

    def of_kept(k):
        if "x" in k:
            return k["x"].double()
        width = block or k["q"].shape[1]
        at = torch.arange(k["q"].shape[1], device="cuda") // width
        return k["q"].double() * k["scales"].double()[:, at]

    if op == "matmul":
        return dict(y=(s["xq"].double() * s["xs"].double()[:, None]) @ (s["wq"].double() * s["ws"].double()[:, None]).t())
    if op == "grad_input":
        return dict(dx=(s["dy"].double() * s["ws"].double()) @ s["wq"].double())
    if op == "grad_weight":
        return dict(dw=(s["dy"].double() * s["xs"].double()[:, None]).t() @ s["xq"].double())
    if op == "norm":
        total = (s["x"].double() + s["residual"].double()).to(s["x"].dtype)
        h = total.double()
        rstd = 1.0 / torch.sqrt((h * h).sum(1) / h.shape[1] + EPS)
        y = h * s["weight"].double()  # the codes do not depend on rstd: it multiplies a whole row
        y, scales = through(y, 0)
        r = dict(total=total.double(), rstd=rstd, y=y * rstd[:, None], scales=scales * rstd[:, None])
        if case["keep"]:
            r["kept"], r["kept_scales"] = through(h, block)
        return r
    if op == "norm_grad":
        # y_c = w_c x_c r, r = (sum x^2 / n + eps)^(-1/2), so dx_c = w_c dy_c r - x_c r^3 / n * sum_j(w_j dy_j x_j), with r as kept
        x, r, dy = of_kept(s["kept"]), s["rstd"].double()[:, None], s["dy"].double()
        u = dy * s["weight"].double()
        dx = u * r - x * r.pow(3) / x.shape[1] * (u * x).sum(1, keepdim=True) + s["dresidual"].double()
        return dict(dx=dx, dweight=(dy * x * r).sum(0))
    if op == "codes":
        value, scales = through(s["x"].double(), block)
        return dict(value=value, scales=scales)
    if op == "gated":
        n = case["cols"]
        gate, up = s["both"][:, :n].double(), s["both"][:, n:].double()
        y, scales = through(gate * torch.sigmoid(gate) * up, 0)
        r = dict(y=y, scales=scales)
        if case["keep"]:
            r["gate"], r["gate_scales"] = through(gate, block)
            r["up"], r["up_scales"] = through(up, block)
        return r
    gate, up, dy = of_kept(s["gate"]), of_kept(s["up"]), s["dy"].double()
    sigma = torch.sigmoid(gate)
    slope = sigma + gate * sigma * torch.sigmoid(-gate)
    return dict(both=torch.cat([dy * up * slope, dy * gate * sigma], 1))
