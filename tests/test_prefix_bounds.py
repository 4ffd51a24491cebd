"""Attention over shared prefixes beside the usual calls: scales next to zero.

Tolerances come from the arithmetic, not from observed errors.  u = 2^-24 is the relative rounding error of 32 bits.
"""

import pytest
import torch

from paper_2004_09362_gb300 import gar
from test_decode_operators import U32
from test_serving_operators import _prefix_case


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [0.0, 1e-40, -1e-40, 3e-38, -3e-38])
@pytest.mark.parametrize("wide", [False, True])
def test_scales_next_to_nothing(scale, wide):
    """Scores of up to 2^122 and scales that leave nothing of them, or a little.  The scale's product with log2 e may be a subnormal number, off by
    2^-150: 2^-17 of 1e-40.  A score is off by (dim + 8) u of scale sum|q||k| beside that, weights, sums and the join by less than 2^-15."""
    dim = 64
    cache, pt, pn, t, n, q, both = _prefix_case([300], [b % 9 for b in range(40)], 40, 4, 2, dim, 16, "bf16", "bf16", wide=wide)
    big = 2.0 ** 59
    cache.k.mul_(big)
    q.mul_(big)
    plan = gar.gar_attn_plan_create(4, 2, dim)
    out, lse = gar.gar_prefix_attention(plan, q, cache, pt, pn, t, n, scale=scale, lse=True)
    scale = float(torch.tensor(scale, dtype=torch.float32))           # as the call has it
    for b in range(q.shape[0]):
        k, v = (x.repeat_interleave(2, 1) for x in (both[b][0] * big, both[b][1]))
        y = torch.einsum("hd,nhd->hn", q[b].double(), k) * scale
        size = abs(scale) * torch.einsum("hd,nhd->hn", q[b].double().abs(), k.abs())
        e = (2.0 ** -17 * y.abs() + (dim + 8) * U32 * size).amax(-1) + 2.0 ** -15
        p = torch.softmax(y, -1)
        want = torch.einsum("hn,nhd->hd", p, v)
        off = (out[b].double() - want).abs()
        assert bool((off <= 2 * e[:, None] * torch.einsum("hn,nhd->hd", p, v.abs()) + 2.0 ** -8 * want.abs() * (1 + 2 ** -7)).all()), b
        assert bool(((lse[b].double() - torch.logsumexp(y, -1)).abs() <= e).all()), b
    gar.gar_kv_status(cache)
