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


def _cached(kind, k_codes, k_scale, v_codes, v_scale, page):
    """A cache of one head that holds rows of given codes and scales, and those rows in 64 bits."""
    n, dim = k_codes.shape
    pages = -(-n // page)
    rows = []
    tensors = []
    for codes, scale in ((k_codes, k_scale), (v_codes, v_scale)):
        t = torch.zeros(pages * page, dim, dtype=torch.int8, device="cuda").view(kind)
        t.view(torch.uint8)[:n] = codes.to(kind).view(torch.uint8)
        s = torch.zeros(pages * page, device="cuda")
        s[:n] = scale
        tensors += [t.view(pages, 1, page, dim), s.view(pages, 1, page)]
        rows.append(codes.to(kind).double() * s[:n].double()[:, None])
    cache = gar.KVCache(tensors[0], tensors[2], tensors[1], tensors[3])
    return cache, torch.arange(pages, dtype=torch.int32, device="cuda")[None], rows[0], rows[1]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("dim,heads,dtype", [(64, 1, torch.float32), (128, 12, torch.bfloat16), (256, 4, torch.float16), (192, 8, torch.float32)])
@pytest.mark.parametrize("n", [20, 300, 5000])
@pytest.mark.parametrize("small", [1e-6, 1e-9, 1e-11, 1e-20])
def test_value_scales_of_rows_without_weight(kind, dim, heads, dtype, n, small):
    """The rows that have the weight have value scales a million times smaller, and less, than those that have none.  (All
    the others' weights together, 2^-126 of a row's, times the quotient of the scales is below 2^-50.)"""
    g = _gen(n)
    heavy = torch.zeros(n, dtype=torch.bool, device="cuda")
    heavy[n // 2], heavy[n - 1] = True, True
    codes = [torch.randint(-120, 121, (n, dim), generator=g, device="cuda").float() for _ in range(2)]
    codes[0][:, 0] = torch.where(heavy, 100.0, -100.0)
    codes[0][:, 1:] = 0
    k_scale = torch.full((n,), 0.01, device="cuda")
    v_scale = torch.where(heavy, small, 1.0) * (torch.rand(n, generator=g, device="cuda") + 0.5)
    cache, table, k, v = _cached(kind, codes[0], k_scale, codes[1], v_scale, 16)
    q = torch.zeros(1, heads, dim, dtype=dtype, device="cuda")
    q[..., 0] = 1
    out, lse = torch.empty(1, heads, dim, device="cuda"), torch.empty(1, heads, device="cuda")
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    plan = gar.gar_attn_plan_create(heads, 1, dim)
    scale = 64.0                            # scores of about +-64: the light rows weigh e^-128
    gar.gar_decode_attention(plan, q, cache, table, lens, scale=scale, out=out, lse=lse)
    y = k[:, 0] * scale
    p = torch.softmax(y, 0)
    want, size = p @ v, p @ v.abs()
    # a score: two scales and the constant rounded, their products, the difference to the reference (|log2 scale| <= 67 of it)
    e = 6 * U32 * float(y.abs().max() + 67)
    tol = (2 * e + 2.0 ** -21 + 2 * n * U32) * size + n * 2.0 ** -39 * float((p * v_scale).max()) * 128
    assert bool(((out[0].double() - want).abs() <= tol).all())
    assert bool(((lse[0].double() - torch.logsumexp(y, 0)).abs() <= e + 2.0 ** -21 + n * U32 + 2.0 ** -22 * float(y.abs().max())).all())


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.int8, torch.float8_e4m3fn])
def test_value_scales_at_the_ends_of_their_range(kind):
    """Scales of zero, subnormal, next to the largest; an infinite or NaN scale gives no number rather than a finite one."""
    dim, n = 64, 48
    g = _gen(5)
    codes = [torch.randint(-120, 121, (n, dim), generator=g, device="cuda").float() for _ in range(2)]
    q = torch.full((1, 1, dim), 0.01, device="cuda")
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    plan = gar.gar_attn_plan_create(1, 1, dim)
    for low, high in ((0.0, 0.0), (0.0, 1.0), (1e-42, 1e-42), (1e-28, 1e-28), (1e-30, 1e30), (1e36, 1e36), (1e-3, float("inf")), (1e-3, float("nan"))):
        v_scale = torch.full((n,), low, device="cuda")
        v_scale[n // 2] = high
        cache, table, k, v = _cached(kind, codes[0], torch.full((n,), 0.01, device="cuda"), codes[1], v_scale, 16)
        out, lse = gar.gar_decode_attention(plan, q, cache, table, lens, lse=True)
        y = (k @ q[0, 0].double()) / 8
        p = torch.softmax(y, 0)
        assert bool((lse[0].double() - torch.logsumexp(y, 0)).abs() <= 1e-4), (low, high)     # unharmed by the values
        if not math.isfinite(high):
            assert not bool(out.isfinite().any())
            continue
        size = p @ v.abs()
        # the largest product of weight and scale counts as 2^-96 at least
        tol = 2.0 ** -16 * size + n * 2.0 ** -39 * max(float((p * v_scale).max()), 2.0 ** -96) * 128
        assert bool(((out[0, 0].double() - p @ v).abs() <= tol).all()), (low, high)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32, torch.float16])
@pytest.mark.parametrize("dim,heads", [(64, 1), (128, 12), (192, 4), (256, 8)])
@pytest.mark.parametrize("large", [2.0 ** 10, 2.0 ** 18, 2.0 ** 24, 2.0 ** 100])
def test_queries_with_one_large_channel_over_8_bits(kind, dtype, dim, heads, large):
    """One channel of the query is much larger than the others, and the keys have it as zero: the scores are those of
    the others.  (Over bf16 and 32-bit queries alike; f16 ones hold 65504 at most.)"""
    if dtype == torch.float16:
        large = min(large, 2.0 ** 15)
    n = 200
    g = _gen(dim)
    codes = [torch.randint(-120, 121, (n, dim), generator=g, device="cuda").float() for _ in range(2)]
    codes[0][:, 5] = 0
    ones = torch.ones(n, device="cuda")
    cache, table, k, v = _cached(kind, codes[0], 0.01 * ones, codes[1], 0.01 * ones, 16)
    q = torch.randn(1, heads, dim, generator=g, device="cuda").to(dtype)
    q[..., 5] = large
    for tiny in (1.0, 2.0 ** -120) if dtype != torch.float16 else (1.0,):    # queries whose channels are next to subnormal too
        x = q if tiny == 1.0 else (q.double() * tiny).to(dtype)
        scale = 0.125 if tiny == 1.0 else 0.125 * 2.0 ** 100
        plan = gar.gar_attn_plan_create(heads, 1, dim)
        out, lse = torch.empty(1, heads, dim, device="cuda"), torch.empty(1, heads, device="cuda")
        gar.gar_decode_attention(plan, x, cache, table, torch.tensor([n], dtype=torch.int32, device="cuda"), scale=scale, out=out, lse=lse)
        x = x[0].double()
        y, size = x @ k.T * scale, x.abs() @ k.abs().T * scale
        # a sum of dim products, two scales and a constant, the difference to the reference; the query's own parts
        # (channels under 2^-126 of 32 bits are taken as zero where they are subnormal: none is here for 1, and for tiny
        # ones they are within the same 2^-39 of the largest)
        parts = scale * x.abs().amax(-1, keepdim=True) * 2.0 ** -39 * k.abs().sum(-1)
        e = ((dim + 6) * U32 * size + 2.0 ** -22 * size + parts).amax(-1) + 8 * U32
        assert bool(((lse[0].double() - torch.logsumexp(y, -1)).abs() <= e + 2.0 ** -21 + n * U32 + 2.0 ** -22 * y.abs().amax(-1)).all()), tiny
        p = torch.softmax(y, -1)
        tol = (2 * e[:, None] + 2.0 ** -21 + 2 * n * U32) * (p @ v.abs()) + n * 2.0 ** -39 * 128 * 0.01
        assert bool(((out[0].double() - p @ v).abs() <= tol).all()), tiny


@pytest.mark.gpu
@pytest.mark.parametrize("dim,heads", [(4, 1), (8, 9), (16, 2), (64, 8), (80, 12), (128, 1), (192, 5), (256, 8)])
@pytest.mark.parametrize("n", [1, 40, 300, 5000])
def test_products_of_32_bit_caches(dim, heads, n):
    """What is promised of a 32-bit cache: products off by 2^-21.  Numbers as a high part of 11 bits and a low one (12 at most, of
    which the product takes 11: 2^-23), the product of the low parts (2^-22) left out: 2 * 2^-23 + 2^-22."""
    g = _gen(dim + n)
    page = 16
    pages = -(-n // page)
    k, v = (torch.randn(pages, 1, page, dim, generator=g, device="cuda") for _ in range(2))
    q = torch.randn(1, heads, dim, generator=g, device="cuda") / 4
    plan = gar.gar_attn_plan_create(heads, 1, dim)
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    out, lse = gar.gar_decode_attention(plan, q, gar.KVCache(k, v), table, torch.tensor([n], dtype=torch.int32, device="cuda"), lse=True)
    scale = dim ** -0.5
    x, rows, values = q[0].double(), k.view(-1, dim)[:n].double(), v.view(-1, dim)[:n].double()
    y, size = x @ rows.T * scale, x.abs() @ rows.abs().T * scale
    e = (((dim + 4) * U32 + 2.0 ** -21) * size).amax(-1)
    p = torch.softmax(y, -1)
    tol = (2 * e[:, None] + 2.0 ** -21 + 2.0 ** -21 + 2 * n * U32) * (p @ values.abs()) + U32 * (p @ values).abs()
    assert bool(((out[0].double() - p @ values).abs() <= tol).all())
    want = torch.logsumexp(y, -1)
    assert bool(((lse[0].double() - want).abs() <= e + 2.0 ** -22 + n * U32 + 2.0 ** -22 * want.abs()).all())


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("low,high", [(0.0, 1.0), (0.0, 1e12), (1e-35, 1e10), (0.0, 1e30), (1e-30, 1e30)])
@pytest.mark.parametrize("n", [40, 100, 700, 20000])
@pytest.mark.parametrize("large_last", [True, False])
def test_value_scales_far_apart_with_equal_weights(kind, low, high, n, large_last):
    """Rows of values of zero, or next to it, weigh as much as rows of large ones, whichever come first: across tiles, warps and
    CTAs."""
    dim, heads = 64, 3
    codes = torch.full((n, dim), 100.0, device="cuda")
    large = torch.arange(n, device="cuda") * 4 >= 3 * n
    if not large_last:
        large = large.flip(0)
    v_scale = torch.where(large, high, low).float()
    cache, table, k, v = _cached(kind, torch.zeros(n, dim, device="cuda"), torch.ones(n, device="cuda"), codes, v_scale, 16)
    q = torch.ones(1, heads, dim, device="cuda")
    plan = gar.gar_attn_plan_create(heads, 1, dim)
    out, lse = gar.gar_decode_attention(plan, q, cache, table, torch.tensor([n], dtype=torch.int32, device="cuda"), lse=True)
    # weights are all alike: each 2^x by 2^-22, its difference to the reference (of up to 220) rounded, two parts by 2^-22; sums by n u
    tol = 2.0 ** -22 + 220 * U32 + 2.0 ** -22 + 2 * n * U32
    assert bool(((lse.double() - math.log(n)).abs() <= tol + 2.0 ** -21 * math.log(n)).all())
    want = v.mean(0)
    assert bool(((out[0].double() - want).abs() <= 2 * tol * want).all())
