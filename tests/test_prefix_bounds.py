"""Attention over shared prefixes beside the usual calls: scales next to zero, the workspace.

Tolerances come from the arithmetic, not from observed errors.  u = 2^-24 is the relative rounding error of 32 bits.
"""

import ctypes

import pytest
import torch

from paper_2004_09362_gb300 import gar
from test_decode_binding import _fake_cache
from test_decode_operators import U32, _cache_raw
from test_serving_operators import _check_prefix, _prefix_case


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


# ---------------------------------------------------------------------------- the workspace

def test_workspace_sizes():
    plan, cache = gar.gar_attn_plan_create(32, 2, 64), _fake_cache(0)
    need = lambda c, *a: gar.gar_prefix_attention_call_bytes(plan, c, *a)  # noqa: E731
    sums = 2 * 64 * 32 * (64 + 1) * 4                       # two parts' outputs and sums
    assert need(cache, 64, 1, 10, 2) == 0 and need(cache, 0, 0, 1 << 20, 0) == 0
    assert need(cache, 64, 1, 1 << 20, 2) == gar.gar_prefix_attention_bytes(plan, 64, 1) > 10 * sums
    for kind in (gar.GAR_F32, gar.GAR_I8, gar.GAR_E4M3):
        other = _fake_cache(0)
        other._c.dtype = kind
        if kind != gar.GAR_F32:
            other._c.k_scale = other._c.v_scale = 4096
        assert need(other, 64, 1, 1 << 20, 2) == sums
    assert need(cache, 64, 64, 1 << 20, 2) == sums          # 16 queries of a head and a prefix
    for bad in ((5, 2, 1, 1), (-1, 1, 1, 1), (3, 0, 1, 1), (1, 1, -1, 1), (1, 1, 1, -1)):
        with pytest.raises(gar.GarError):
            need(cache, *bad)
    with pytest.raises(gar.GarError):
        need(_fake_cache(0, heads=3), 64, 1, 1, 1)
    with pytest.raises(ValueError):
        need(cache, 1, 1, 1 << 32, 1)
    n = ctypes.c_size_t()
    assert gar._lib.gar_prefix_attention_call_bytes(None, _cache_raw(), 1, 1, 1, 1, n) == -1
    assert gar._lib.gar_prefix_attention_call_bytes(plan.handle, None, 1, 1, 1, 1, n) == -1
    assert gar._lib.gar_prefix_attention_call_bytes(plan.handle, _cache_raw(), 1, 1, 1, 1, None) == -1


@pytest.mark.gpu
@pytest.mark.parametrize("kind,dtype,share,wide", [("bf16", "bf16", 40, True), ("f16", "f16", 150, True), ("i8", "bf16", 40, True),
                                                   ("f32", "f32", 40, True), ("bf16", "bf16", 3, True), ("bf16", "bf16", 40, False)])
def test_a_call_needs_what_it_says(kind, dtype, share, wide):
    """A workspace of just that size, or none: the result is right, nothing is written behind it, one byte less is refused."""
    cache, pt, pn, t, n, q, both = _prefix_case([500], [b % 21 for b in range(share)], share, 8, 2, 64, 16, kind, dtype, wide=wide)
    plan = gar.gar_attn_plan_create(8, 2, 64)
    want = gar.gar_prefix_attention(plan, q, cache, pt, pn, t, n, lse=True)
    need = gar.gar_prefix_attention_call_bytes(plan, cache, share, 1, pt.shape[1], t.shape[1])
    assert (need == 0) == (not wide) and need <= gar.gar_prefix_attention_bytes(plan, share, 1)
    room = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((share, 8), device="cuda")
    code = {"f32": gar.GAR_F32, "bf16": gar.GAR_BF16, "f16": gar.GAR_F16}[dtype]

    def call(at, size):
        return gar._lib.gar_prefix_attention(plan.handle, cache._c, q.data_ptr(), 512, 64, code, out.data_ptr(), 512, 64, code, lse.data_ptr(),
                                             pt.data_ptr(), pt.stride(0), pt.shape[1], pn.data_ptr(), 1, t.data_ptr(), t.stride(0), t.shape[1],
                                             n.data_ptr(), share, 0.125, at, size, torch.cuda.current_stream().cuda_stream)
    assert call(room.data_ptr() if need else None, need) == 0
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and bool((room[need:] == 0x5a).all())
    _check_prefix(out, lse, q, both, 0.125, dtype)
    if need:
        assert call(room.data_ptr(), need - 1) == -6 and call(None, need) == -6
    # what a call through the binding takes from the allocator
    del room, want
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    gar.gar_prefix_attention(plan, q, cache, pt, pn, t, n, out=out, lse=lse)
    assert torch.cuda.max_memory_allocated() - before <= need + (1 << 20) + 512   # (a block may be so much larger)
