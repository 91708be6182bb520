"""The 8-bit layer's operators at the ends of their ranges, against 64 bits."""
import math

import pytest
import torch

import paper_2604_06836_amd as stq
from test_gpu_operators import U, Codes, check_codes, matrix, silu, stream

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = stq.Context(0, 4)
    yield c
    torch.cuda.synchronize()
    c.close()


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


def test_gates_that_are_not_finite(ctx):
    """x / (1 + exp(-x)) of infinities and NaN: none of them has a code."""
    for bad in (math.inf, -math.inf, math.nan):
        gate = torch.ones(3, 64, device="cuda")
        gate[1, 7] = bad
        y = Codes(3, 64)
        ctx.gated_silu(matrix(gate), matrix(torch.ones_like(gate)), y.mat, None, None, stream())
        assert torch.isnan(y.s[:, 0]).tolist() == [False, True, False] and (y.q.t[1] == 0).all()
