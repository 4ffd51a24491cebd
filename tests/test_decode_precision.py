"""Decode attention where 16-bit parts could lose what counts: weights that are small beside the largest, scales and
queries of very different sizes.  Outputs are 32 bits wide; u = 2^-24.

A weight (over an 8-bit cache: a weight times its row's value scale) enters the product with the values as two f16 parts after
the largest has been brought to 2^14.  A part is off by half a unit of its 11 bits, at least by half the smallest step,
2^-25: so the weight is off by 2^-22 of itself or 2^-39 of the largest, and 2^x by another 2^-22.
"""

import math

import pytest
import torch

from paper_2004_09362_gb300 import gar

U32 = 2.0 ** -24


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


@pytest.mark.gpu
@pytest.mark.parametrize("dim,heads,page", [(64, 1, 16), (128, 12, 16), (256, 4, 16), (192, 3, 5)])
@pytest.mark.parametrize("n,t", [(1400, 14.2), (700, 18.0), (16384, 22.3), (16384, 25.5), (60000, 30.0), (40, 20.0)])
def test_small_weights_of_f16_values(dim, heads, page, n, t):
    """One row has nearly all of the weight and values of zero (a sink): the output is what the small weights give."""
    pages = -(-n // page)
    k = torch.zeros(pages, 1, page, dim, dtype=torch.float16, device="cuda")
    scale = 0.125
    k.view(-1, dim)[:, 0] = -t * math.log(2) / scale
    v = (torch.rand(k.shape, generator=_gen(n), device="cuda") + 0.5).half()
    sink = n // 3
    k.view(-1, dim)[sink], v.view(-1, dim)[sink] = 0, 0
    q = torch.zeros(1, heads, dim, dtype=torch.float16, device="cuda")
    q[..., 0] = 1
    out = torch.empty(1, heads, dim, device="cuda")
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    plan = gar.gar_attn_plan_create(heads, 1, dim)
    gar.gar_decode_attention(plan, q, gar.KVCache(k, v), table, lens, scale=scale, out=out)
    y = k.view(-1, dim)[:n, 0].double() * scale
    p = torch.softmax(y, 0)
    rows = v.view(-1, dim)[:n].double()
    want = p @ rows
    # a score is one product, exact, times a rounded constant; its difference to the maximum rounds again
    e = 4 * U32 * float(y.abs().max())
    tol = (2 * e + 2.0 ** -21 + 2 * n * U32) * want + n * 2.0 ** -39 * float(p.max()) * rows.amax(0)
    assert bool(((out[0].double() - want).abs() <= tol).all())
