"""How many bits of its factors a weight gradient keeps: 22 of a float32 gradient's, whatever the result's type, so that sums which all but cancel are theirs."""
import pytest
import torch

from paper_1603_05279_amd import xnor
from tests.lowbit_helpers import EPS32, HALF_ULP, SMALLEST, TYPES, filled, generator, normal
from tests.test_weight_gradient_gpu import make, values

pytestmark = pytest.mark.gpu

ACTIVE = 16


@pytest.mark.parametrize("wname", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("group", [0, 32, 128])
@pytest.mark.parametrize("rows,cin,out", [(1200, 130, 60), (300, 2100, 2300), (400, 4100, 4100), (70, 50, 40)])
def test_sums_that_all_but_cancel(rows, cin, out, group, wname):
    """Sixteen rows have gradients, in pairs of nearly opposite ones on the same inputs: the sum is a thousandth of its terms.  Zeros add nothing, so that an error is the
    factors' representation and sixteen additions'."""
    gen = generator(rows + group)
    q, scale, _ = make(gen, rows, cin, out, group, "f32")
    at = torch.randperm(rows, generator=gen)[:ACTIVE]
    q[at[1::2]], scale[at[1::2]] = q[at[::2]], scale[at[::2]]
    g = torch.zeros((rows, out))
    half = normal(gen, ACTIVE // 2, out)
    g[at[::2]], g[at[1::2]] = half, -half * (1 + 2.0 ** -10 * normal(gen, ACTIVE // 2, out))
    x, d = values(q, scale, group).cuda(), g.double().cuda()
    total, want = d.abs().t().contiguous() @ x.abs(), d.t().contiguous() @ x
    work = filled((xnor.q8_weight_gradient_workspace_bytes(rows, cin, out, group, torch.float32, TYPES[wname]),), torch.uint8)
    g_w = filled((out, cin), TYPES[wname])
    xnor.xnor_q8_weight_gradient(q.cuda(), scale.cuda(), g.cuda(), g_w, None, work, rows, cin, out, group)
    # both factors to 2^-22 and the product of both remainders left out, the scale's product with the code; an instruction's sixteen rows in an order of its own
    err = total * (3.01 * 2.0 ** -22 + EPS32 + 2 * EPS32 * (ACTIVE + 2)) + 2.0 ** -39 * ACTIVE * d.abs().amax(0)[:, None] * 127 * scale.abs().max().double().cuda()
    bound = err + (HALF_ULP[wname] * (want.abs() + err) + SMALLEST[wname] if wname != "f32" else 0)
    assert int((~((g_w.double() - want).abs() <= bound)).sum()) == 0
