"""Attention over shared prefixes held to what is stated: the mass of every tile, each cache type's precision, and the calls beside the
usual ones (strides, orders, lengths past the tables, many prefixes, scales next to zero, the workspace).

Tolerances come from the arithmetic, not from observed errors.  u = 2^-24 is the relative rounding error of 32 bits.
"""

import ctypes
import math

import pytest
import torch

from paper_2004_09362_gb300 import gar
from test_decode_binding import _fake_cache
from test_decode_operators import QMAX, ROUND, TINY, TORCH, U32, _attn_case, _cache_raw, _randn
from test_serving_operators import _check_prefix, _prefix_case

I32 = torch.int32


def _bounds(out, lse, q, both, scale, kind, out_type):
    """Bounds.  A score, `dim` products in 32 bits (over 32-bit caches of two parts each, 2^-21; 8-bit ones of codes and queries, 2^-22, and a scale)
    and three roundings more, is off by e = (dim + 8) u + 2^-21 of scale sum|q||k|; the same counts for its difference to the maximum.  The weight has 2^-22 more;
    its parts keep 2^-21 (f32), 2^-22 of it and 2^-39 of the largest product of a weight and a scale (8 bits, f16), 2^-17 (bf16); on the tensor memory's
    way 2^-17 (bf16) or 2^-22 and 2^-34 of the largest (f16), and sums of up to 16 tiles 2^-15 (here: one tile of 16 products of a truncation each,
    2^-19).  32-bit sums over n rows: chains of n / 64 at most, rounded, and joins of lanes, warps and parts, n / 64 + 32 roundings.  The two
    parts' weights come from logarithms off by 2^-22 of themselves and 2^-22, and from exponentials, a sum and a quotient, 2^-21 together."""
    group = q.shape[1] // both[0][0].shape[1]
    weight = {"f32": 2.0 ** -21, "bf16": 2.0 ** -17 + 2.0 ** -19, "f16": 2.0 ** -22 + 2.0 ** -19, "i8": 2.0 ** -22, "e4m3": 2.0 ** -22}[kind]
    least = {"f16": 2.0 ** -34}.get(kind, 2.0 ** -39)
    for b in range(q.shape[0]):
        k, v = (x.repeat_interleave(group, 1) for x in both[b])
        n = k.shape[0]
        if n == 0:
            assert bool((out[b] == 0).all()) and bool((lse[b] == -math.inf).all())
            continue
        y = torch.einsum("hd,nhd->hn", q[b].double(), k) * scale
        e = ((q.shape[2] + 8) * U32 + 2.0 ** -21) * abs(scale) * torch.einsum("hd,nhd->hn", q[b].double().abs(), k.abs()).amax(-1)
        p = torch.softmax(y, -1)
        want, size = torch.einsum("hn,nhd->hd", p, v), torch.einsum("hn,nhd->hd", p, v.abs())
        want_lse = torch.logsumexp(y, -1)
        sums = (n / 64 + 32) * U32
        lse_off = 2 * e + 2.0 ** -21 + sums + 2.0 ** -22 * torch.maximum(want_lse.abs(), y.abs().amax(-1))
        rel = 2 * e + 2.0 ** -21 + weight + 2 * sums + 2 * lse_off + 2.0 ** -21
        small = n * least * p.amax(-1)[:, None] * v.abs().amax(0)
        tol = rel[:, None] * size + small + ROUND[out_type] * want.abs() * (1 + 2 ** -7) + TINY[out_type]
        off = (out[b].double() - want).abs()
        assert bool((off <= tol).all()), (b, n, float((off / tol.clamp(min=1e-300)).max()))
        assert bool(((lse[b].double() - want_lse).abs() <= 2 * lse_off + 2.0 ** -21).all()), (b, n)


# ---------------------------------------------------------------------------- every tile counts once

TILES = pytest.mark.parametrize("kind,dim,page_size,order,share,q_heads,kv_heads,prefixes", [
    ("bf16", 128, 64, "head", 32, 32, 8, [60000]),            # one block: two streams, boxes of pages
    ("f16", 128, 24, "head", 32, 32, 8, [40001]),             # rows one by one
    ("bf16", 128, 256, "token", 64, 32, 8, [33000]),          # pairs of blocks, boxes, another order
    ("f16", 64, 32, "token", 100, 16, 4, [50129]),
    ("bf16", 96, 16, "head", 24, 8, 2, [40000]),
    ("f16", 128, 8, "head", 70, 8, 2, [20007]),
    ("bf16", 128, 128, "head", 76, 64, 16, [50100]),          # parts of over 16 tiles of each stream
    ("f16", 64, 16, "head", 20, 32, 32, [30011]),
    ("bf16", 128, 16, "head", 9, 16, 2, [3000, 0, 129, 1, 9000]),
    ("f16", 128, 128, "token", 40, 16, 2, [700, 12800, 128]),
    ("i8", 128, 64, "head", 32, 8, 2, [30000]), ("f32", 64, 16, "head", 12, 8, 4, [20001])])


@pytest.mark.gpu
@TILES
def test_every_tile_has_its_mass(kind, dim, page_size, order, share, q_heads, kv_heads, prefixes):
    """Queries of zero: all weights are equal, and values that mark the rows of a tile in a channel of its own, some tiles at a time, come out
    as each tile's share of the rows.  Weights are one exactly, sums of them whole numbers, so only the join rounds: its factors 2^-22, their
    logarithms 2^-22 of at most 12, sums, a quotient and a product."""
    own = [(b * 13) % 40 for b in range(share * len(prefixes))]
    cache, pt, pn, t, n, q, _ = _prefix_case(prefixes, own, share, q_heads, kv_heads, dim, page_size, kind, "bf16" if kind in QMAX else kind, order=order)
    q.zero_()
    if kind in QMAX:
        cache.v_scale.fill_(1.0)
    plan = gar.gar_attn_plan_create(q_heads, kv_heads, dim)
    out = torch.empty(q.shape, device="cuda")
    lens = torch.tensor(prefixes, device="cuda").repeat_interleave(share)
    counts = lens + torch.tensor(own, device="cuda")
    tiles = -(-max(prefixes) // 128)
    v = cache.v.view(torch.uint8) if kind in QMAX else cache.v
    for first in range(0, tiles, dim):
        v.zero_()
        for g, rows in enumerate(prefixes):
            at = torch.arange(min(rows, first * 128), min(rows, (first + dim) * 128), device="cuda")
            page, row, tile = pt[g, at // page_size].long(), at % page_size, at // 128 - first
            v[page, :, row, tile] = 1
        _, lse = gar.gar_prefix_attention(plan, q, cache, pt, pn, t, n, lse=True, out=out)
        tile = torch.arange(first, first + dim, device="cuda")
        here = (lens[:, None] - tile * 128).clamp(0, 128)
        want = torch.where(counts[:, None] > 0, here / counts[:, None].clamp(min=1).double(), 0.0)[:, None].expand(out.shape)
        assert bool(((out.double() - want).abs() <= 2.0 ** -18 * want).all()), float(((out.double() - want).abs() / want.clamp(min=1e-9)).max())
        want = counts.double().log()[:, None].expand(lse.shape)
        assert bool(((lse.double() - want).abs()[counts > 0] <= 2.0 ** -20 + 2.0 ** -21 * want[counts > 0]).all())
        assert bool((lse[counts == 0] == -math.inf).all())
    gar.gar_kv_status(cache)


@pytest.mark.gpu
@TILES
def test_every_half_tile_has_its_weight(kind, dim, page_size, order, share, q_heads, kv_heads, prefixes):
    """Keys whose first channel is a number of their 64 rows, queries that are a number each: weights e^(c s), of which values that mark those rows
    in a channel of their own bring each half tile's share.  Scores are one product, exact, of 3 at most, times a rounded factor; weights are off by 2^-22, their parts
    by 2^-16 and 2^-34 of the largest, 2^9 times theirs, sums in tensor memory by 2^-15, in 32 bits by 2^-17, joins by less than 2^-18: 2^-14 together."""
    cache, pt, pn, t, n, q, _ = _prefix_case(prefixes, [0] * share * len(prefixes), share, q_heads, kv_heads, dim, page_size, kind,
                                             "bf16" if kind in QMAX else kind, order=order)
    k, v = (x.view(torch.uint8) if kind in QMAX else x for x in (cache.k, cache.v))
    if kind in QMAX:
        cache.k_scale.fill_(1 / 32)
        cache.v_scale.fill_(1.0)
    k.zero_()
    q.zero_()
    factor = torch.tensor([1.0, -1.0, 0.5, 0.25, -0.5], device="cuda")[(torch.arange(q[..., 0].numel(), device="cuda") * 7) % 5].view(q.shape[:2])
    q[..., 0] = factor.to(q.dtype)
    halves = -(-max(prefixes) // 64)
    mark = (torch.arange(halves, device="cuda") * 37) % 192 - 96            # of 64 rows, in 1/32
    lens = torch.tensor(prefixes, device="cuda")
    rows = (lens[:, None] - torch.arange(halves, device="cuda") * 64).clamp(0, 64).repeat_interleave(share, 0)[:, None]
    weight = rows * torch.exp(factor.double()[..., None] * mark / 32)
    share_of = weight / weight.sum(-1, keepdim=True).clamp(min=1e-300)
    for g, count in enumerate(prefixes):
        at = torch.arange(count, device="cuda")
        to = mark[at // 64][:, None]
        k[pt[g, at // page_size].long(), :, at % page_size, 0] = (to.to(torch.int8).view(torch.uint8) if kind in QMAX else (to / 32).to(k.dtype))
    plan = gar.gar_attn_plan_create(q_heads, kv_heads, dim)
    out = torch.empty(q.shape, device="cuda")
    for first in range(0, halves, dim):
        v.zero_()
        for g, count in enumerate(prefixes):
            at = torch.arange(min(count, first * 64), min(count, (first + dim) * 64), device="cuda")
            v[pt[g, at // page_size].long(), :, at % page_size, at // 64 - first] = 1
        _, lse = gar.gar_prefix_attention(plan, q, cache, pt, pn, t, n, scale=1.0, lse=True, out=out)
        want = torch.zeros_like(out, dtype=torch.float64)
        here = share_of[..., first:first + dim]
        want[..., :here.shape[-1]] = here
        assert bool(((out.double() - want).abs() <= 2.0 ** -14 * want).all()), float(((out.double() - want).abs() / want.clamp(min=1e-9)).max())
        want = weight.sum(-1).log()
        assert bool(((lse.double() - want).abs()[want > -math.inf] <= 2.0 ** -16).all()) and bool((lse[want == -math.inf] == -math.inf).all())
    gar.gar_kv_status(cache)


@pytest.mark.gpu
@pytest.mark.parametrize("groups,share,q_heads,heads,dim,page_size,kind", [
    (64, 8, 32, 8, 128, 16, "bf16"), (128, 5, 32, 8, 128, 16, "bf16"), (60, 20, 8, 8, 64, 64, "f16"), (40, 40, 32, 8, 128, 24, "f16"), (150, 17, 4, 4, 64, 128, "bf16")])
def test_many_parts_to_a_cta(groups, share, q_heads, heads, dim, page_size, kind):
    """Many prefixes of one to some dozen tiles: each CTA takes many parts, one after the other, and no wait runs out."""
    prefixes = [max(0, int(2000 * ((g * 0.6180339887498949) % 1.0))) for g in range(groups)]
    own = [1 + b % share for b in range(groups * share)]
    cache, pt, pn, t, n, q, both = _prefix_case(prefixes, own, share, q_heads, heads, dim, page_size, kind, kind, every=53)
    plan = gar.gar_attn_plan_create(q_heads, heads, dim)
    out, lse = gar.gar_prefix_attention(plan, q, cache, pt, pn, t, n, lse=True)
    gar.gar_kv_status(cache)
    _check_prefix(out[::53], lse[::53], q[::53], both, dim ** -0.5, kind)
    for _ in range(30):
        again = gar.gar_prefix_attention(plan, q, cache, pt, pn, t, n, lse=True)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    gar.gar_kv_status(cache)


# ---------------------------------------------------------------------------- precision

@pytest.mark.gpu
@pytest.mark.parametrize("kind,dtype", [("f32", "f32"), ("i8", "bf16"), ("i8", "f16"), ("i8", "f32"), ("e4m3", "bf16"), ("e4m3", "f16"),
                                        ("e4m3", "f32"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("q_heads,kv_heads,dim,share,prefix", [(8, 2, 64, 3, 300), (16, 2, 128, 12, 129), (32, 4, 64, 20, 128), (4, 4, 96, 40, 250)])
@pytest.mark.parametrize("wide", [False, True])
def test_each_types_precision(kind, dtype, q_heads, kv_heads, dim, share, prefix, wide):
    own = [(5 * b) % 37 for b in range(share)]
    cache, pt, pn, t, n, q, both = _prefix_case([prefix], own, share, q_heads, kv_heads, dim, 16, kind, dtype, sharp=0.1, wide=wide)
    plan = gar.gar_attn_plan_create(q_heads, kv_heads, dim)
    out = torch.empty(q.shape, device="cuda")
    _, lse = gar.gar_prefix_attention(plan, q, cache, pt, pn, t, n, lse=True, out=out)
    _bounds(out, lse, q, both, dim ** -0.5, kind, "f32")
    gar.gar_kv_status(cache)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,wide", [("bf16", True), ("bf16", False), ("f16", True), ("f16", False)])
def test_weights_come_out_as_their_parts_hold_them(kind, wide):
    """Each row's value marks a channel of its own, so its weight comes out alone.  Scores are one product, exact, of 3 at most, times a rounded factor: 2^-20;
    weights 2^-22, their parts 2^-17 (bf16) or 2^-22 (f16, and 2^-34 of the largest, 2^9 times the smallest), sums of weights and joins 2^-20."""
    n, dim, share = 128, 128, 40
    cache, pt, pn, t, lens, q, _ = _prefix_case([n], [0] * share, share, 8, 2, dim, 16, kind, kind, wide=wide)
    at = torch.arange(n, device="cuda")
    page = pt[0, at // 16].long()
    mark = ((at * 37) % 192 - 96) / 32
    cache.k.zero_()
    cache.v.zero_()
    cache.k[page, :, at % 16, 0] = mark.to(cache.k.dtype)[:, None]
    cache.v[page, :, at % 16, at] = 1
    q.zero_()
    q[..., 0] = (1 - torch.arange(share, device="cuda") / 64).to(q.dtype)[:, None]
    out = torch.empty(q.shape, device="cuda")
    gar.gar_prefix_attention(gar.gar_attn_plan_create(8, 2, dim), q, cache, pt, pn, t, lens, scale=1.0, out=out)
    want = torch.softmax(q[..., :1].double() * mark.double(), -1)
    off = float(((out.double() - want).abs() / want).max())
    assert off <= (2.0 ** -17 if kind == "bf16" else 2.0 ** -22 + 2.0 ** -25) + 2.0 ** -20 + 2.0 ** -22 + 2.0 ** -20, off
    gar.gar_kv_status(cache)


# ---------------------------------------------------------------------------- strides and orders

@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("dim,page_size,share", [(128, 64, 24), (128, 256, 64), (64, 32, 70), (96, 16, 20), (64, 128, 17), (72, 128, 40)])
@pytest.mark.parametrize("out_type", ["own", "f32"])
@pytest.mark.parametrize("pad", [1, 4, 8])
def test_strides_on_the_tensor_memorys_way(kind, dim, page_size, share, out_type, pad):
    """Caches in the order of tokens, queries that are strided but aligned, outputs that four at once can and cannot be stored to."""
    own = [(7 * b) % 20 for b in range(share)]
    cache, pt, pn, t, n, q, both = _prefix_case([777], own, share, 8, 4, dim, page_size, kind, kind, order="token")
    many = torch.full((share, 10, dim + 8), math.nan, device="cuda").to(q.dtype)
    many[:, 1:9, 8:] = q
    out_type = kind if out_type == "own" else out_type
    room = torch.full((share, 9, dim + pad), 7.0, device="cuda").to(TORCH[out_type])
    plan = gar.gar_attn_plan_create(8, 4, dim)
    out, lse = gar.gar_prefix_attention(plan, many[:, 1:9, 8:], cache, pt, pn, t, n, lse=True, out=room[:, 1:, :dim])
    _check_prefix(out, lse, q, both, dim ** -0.5, out_type)
    assert bool((room[:, 0] == 7).all()) and bool((room[:, :, dim:] == 7).all())
    gar.gar_kv_status(cache)


# ---------------------------------------------------------------------------- lengths past the tables

@pytest.mark.gpu
@pytest.mark.parametrize("kind,dtype,q_heads,kv_heads,share", [("bf16", "bf16", 4, 2, 64), ("f16", "f16", 8, 2, 33), ("i8", "f16", 4, 2, 128),
                                                               ("f32", "f32", 4, 2, 32), ("bf16", "bf16", 2, 2, 12), ("bf16", "bf16", 4, 2, 2)])
@pytest.mark.parametrize("bad", [10 ** 6, 2 ** 31 - 1, -7, -2 ** 31])
def test_lengths_that_the_tables_cannot_hold(kind, dtype, q_heads, kv_heads, share, bad):
    """Too long counts as all that the table holds, negative as nothing, for the prefix and for own rows alike."""
    dim, ps = 64, 16
    size = 2 if kind in ("bf16", "f16") else 4 if kind == "f32" else 1
    # a table just past what is read for each sequence, or (two sequences) far below it
    times = (1 << 27) // (share * kv_heads * dim * size * 2) // 160 + 1 if share > 2 else 1
    cache, table, lens, _, kvs = _attn_case([160] + [40] * share, q_heads, kv_heads, dim, ps, kind, dtype)
    prefix = table[:1, :10].repeat(1, times)
    plan = gar.gar_attn_plan_create(q_heads, kv_heads, dim)
    q = _randn((share, q_heads, dim), dtype, 3)
    own = table[1:, :2].contiguous()                        # 32 of the 40 rows
    n = lens[1:].clone()
    n[:] = 5
    n[1] = bad
    pn = torch.tensor([bad], dtype=I32, device="cuda")
    out, lse = gar.gar_prefix_attention(plan, q, cache, prefix, pn, own, n, lse=True)
    with pytest.raises(gar.GarError) as e:
        gar.gar_kv_status(cache)
    assert "length" in str(e.value)
    both = []
    for b in range(share):
        mine = 5 if b != 1 else 32 if bad > 0 else 0
        both.append(tuple(torch.cat([kvs[0][i]] * (times if bad > 0 else 0) + [kvs[1 + b][i][:mine]]) for i in (0, 1)))
    _check_prefix(out, lse, q, both, dim ** -0.5, dtype)


# ---------------------------------------------------------------------------- more prefixes than the tensor memory's way takes

@pytest.mark.gpu
@pytest.mark.parametrize("groups,share,q_heads,heads,prefix", [(129, 5, 32, 8, 200), (128, 5, 32, 8, 200), (1025, 1, 17, 1, 100)])
def test_many_prefixes(groups, share, q_heads, heads, prefix):
    """Blocks of queries up to their limit and past it."""
    prefixes = [(prefix * (g % 7 + 1)) // 7 for g in range(groups)]
    own = [b % 3 for b in range(groups * share)]
    cache, pt, pn, t, n, q, both = _prefix_case(prefixes, own, share, q_heads, heads, 64, 16, "bf16", "bf16", every=37)
    plan = gar.gar_attn_plan_create(q_heads, heads, 64)
    out, lse = gar.gar_prefix_attention(plan, q, cache, pt, pn, t, n, lse=True)
    _check_prefix(out[::37], lse[::37], q[::37], both, 0.125, "bf16")
    gar.gar_kv_status(cache)


# ---------------------------------------------------------------------------- scales

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
