"""Attention over shared prefixes, the weights that cached rows gather, eviction by them and the verification of drafted
tokens, against plain 64-bit versions.

Tolerances come from the arithmetic, not from observed errors.  u = 2^-24 is the relative rounding error of 32 bits.
"""

import math

import pytest
import torch

from paper_2004_09362_gb300 import gar
from test_decode_operators import QMAX, ROUND, TINY, TORCH, U32, _attn_case, _cache_raw, _empty_cache, _gen, _randn

KINDS = [("bf16", "bf16"), ("f16", "f16"), ("f32", "f32"), ("i8", "bf16"), ("i8", "f16"), ("i8", "f32"), ("e4m3", "bf16"),
         ("e4m3", "f16"), ("e4m3", "f32")]


# ---------------------------------------------------------------------------- refusals (no GPU work)

def _prefix_raw(plan, c, **kw):
    a = dict(q=4096, qb=256, qh=64, qt=gar.GAR_BF16, out=4096, ob=256, oh=64, ot=gar.GAR_BF16, lse=None, pt=4096, ps=2, pw=2, pl=4096,
             groups=2, t=4096, ts=2, tw=2, n=4096, batch=4, scale=0.1, ws=4096, wb=1 << 30)
    a.update(kw)
    return gar._lib.gar_prefix_attention(plan, c, a["q"], a["qb"], a["qh"], a["qt"], a["out"], a["ob"], a["oh"], a["ot"], a["lse"],
                                         a["pt"], a["ps"], a["pw"], a["pl"], a["groups"], a["t"], a["ts"], a["tw"], a["n"],
                                         a["batch"], a["scale"], a["ws"], a["wb"], None)


@pytest.mark.parametrize("bad,code", [
    (dict(q=None), -1), (dict(out=None), -1), (dict(n=None), -1), (dict(pl=None), -1), (dict(t=None), -1), (dict(pt=None), -1),
    (dict(qt=gar.GAR_F16), -1), (dict(qt=gar.GAR_I8), -1), (dict(ot=gar.GAR_F16), -1), (dict(groups=0), -1), (dict(groups=3), -1),
    (dict(groups=-1), -1), (dict(batch=-4), -1), (dict(tw=-1), -1), (dict(pw=-1), -1), (dict(scale=float("nan")), -1),
    (dict(q=4097), -3), (dict(out=4097), -3), (dict(lse=4097), -3), (dict(pl=4097), -3), (dict(n=4098), -3), (dict(ws=4104), -3),
    (dict(ws=None), -6), (dict(wb=16), -6)])
def test_prefix_refusals(bad, code):
    plan = gar.gar_attn_plan_create(4, 2, 64)
    assert _prefix_raw(plan.handle, _cache_raw(), **bad) == code
    assert gar.gar_last_error()


def test_prefix_refusals_of_plans_and_sizes():
    plan = gar.gar_attn_plan_create(4, 2, 64)
    assert _prefix_raw(None, _cache_raw()) == -1
    assert _prefix_raw(plan.handle, _cache_raw(heads=3)) == -1
    assert _prefix_raw(plan.handle, _cache_raw()) == -6             # no workspace of the plan's
    assert _prefix_raw(plan.handle, _cache_raw(), batch=0, groups=0) == 0
    assert gar.gar_prefix_attention_bytes(plan, 0, 0) >= 0
    assert gar.gar_prefix_attention_bytes(plan, 6, 2) >= 2 * 6 * 4 * 65 * 4
    for batch, groups in ((5, 2), (-1, 1), (3, 0), (1 << 30, 1)):
        with pytest.raises(gar.GarError):
            gar.gar_prefix_attention_bytes(plan, batch, groups)
    with pytest.raises(ValueError):
        gar.gar_prefix_attention_bytes(plan, 1 << 32, 1)


@pytest.mark.parametrize("bad,code", [
    (dict(q=None), -1), (dict(lse=None), -1), (dict(w=None), -1), (dict(out=None), -1), (dict(n=None), -1), (dict(t=None), -1),
    (dict(qt=gar.GAR_F32), -1), (dict(qt=gar.GAR_E4M3), -1), (dict(heads=3), -1), (dict(heads=0), -1), (dict(batch=-1), -1),
    (dict(tw=-1), -1), (dict(window=-1), -1), (dict(rows=-1), -1), (dict(scale=float("inf")), -1), (dict(out=4096, ob=64), -1),
    (dict(q=4097), -3), (dict(lse=4098), -3), (dict(w=4098), -3), (dict(out=8194), -3), (dict(t=4097), -3)])
def test_weigh_refusals(bad, code):
    a = dict(q=4096, qt=gar.GAR_BF16, heads=4, lse=4096, w=4096, out=8192, ob=96, rows=48, t=4096, tw=3, n=4096, batch=2, scale=0.1,
             window=0)
    a.update(bad)
    assert gar._lib.gar_kv_weigh(_cache_raw(), a["q"], 256, 64, a["qt"], a["heads"], a["lse"], a["w"], 96, 48, a["out"], a["ob"], 48,
                                 a["rows"], a["t"], 3, a["tw"], a["n"], a["batch"], a["scale"], a["window"], None) == code
    assert gar._lib.gar_kv_weigh(None, 4096, 256, 64, 1, 4, 4096, 4096, 96, 48, 8192, 96, 48, 48, 4096, 3, 3, 4096, 2, 0.1, 0, None) == -1


@pytest.mark.parametrize("bad,code", [
    (dict(w=None), -1), (dict(p=None), -1), (dict(t=None), -1), (dict(n=None), -1), (dict(ow=None), -1), (dict(op=None), -1),
    (dict(on=None), -1), (dict(rows=-1), -1), (dict(rows=(1 << 24) + 1), -1), (dict(tw=-1), -1), (dict(batch=-1), -1), (dict(keep=0), -1),
    (dict(first=-1), -1), (dict(recent=-1), -1), (dict(first=5, recent=4), -1), (dict(first=2 ** 31 - 1, recent=2 ** 31 - 1), -1),
    (dict(ow=4096), -1), (dict(op=4352), -1), (dict(on=4864), -1), (dict(w=4097), -3), (dict(p=4097), -3), (dict(on=8194), -3)])
def test_evict_refusals(bad, code):
    a = dict(w=4096, p=4352, rows=32, t=4608, tw=2, n=4864, batch=2, keep=8, first=0, recent=0, ow=8192, op=8448, on=8704)
    a.update(bad)
    assert gar._lib.gar_kv_evict(_cache_raw(), a["w"], a["p"], a["rows"], a["t"], 2, a["tw"], a["n"], a["batch"], a["keep"], a["first"],
                                 a["recent"], a["ow"], a["op"], a["on"], None) == code
    assert gar._lib.gar_kv_evict(_cache_raw(dim=0), 4096, 4352, 32, 4608, 2, 2, 4864, 2, 8, 0, 0, 8192, 8448, 8704, None) == -1


@pytest.mark.parametrize("bad,code", [
    (dict(p=None), -1), (dict(q=None), -1), (dict(t=None), -1), (dict(u=None), -1), (dict(out=None), -1), (dict(acc=None), -1),
    (dict(type=gar.GAR_I32), -1), (dict(type=gar.GAR_I8), -1), (dict(vocab=0), -1), (dict(vocab=1 << 31), -1), (dict(width=2), -1),
    (dict(batch=-1), -1), (dict(batch=2 ** 31 - 1), -1), (dict(drafts=-1), -1), (dict(p=4098), -3), (dict(q=4098), -3), (dict(t=4100), -3),
    (dict(u=4098), -3), (dict(out=4100), -3), (dict(acc=4098), -3)])
def test_verify_refusals(bad, code):
    a = dict(p=4096, q=4096, type=gar.GAR_F32, vocab=10, t=4096, width=8, u=4096, batch=2, drafts=3, out=8192, acc=4096)
    a.update(bad)
    assert gar._lib.gar_verify_drafts(a["p"], 40, 10, a["q"], 30, 10, a["type"], a["vocab"], a["t"], a["width"], a["u"], a["batch"],
                                      a["drafts"], a["out"], a["acc"], None) == code
    assert gar.gar_last_error()


# ---------------------------------------------------------------------------- attention over shared prefixes

def _prefix_case(prefixes, own, share, q_heads, kv_heads, dim, page_size, kind, dtype, seed=0, order="head", sharp=1.0, every=1, wide=True):
    """(cache, prefix table and lengths, table and lengths, q, each sequence's keys and values in 64 bits)."""
    cache, table, lens, _, kvs = _attn_case(prefixes + own, q_heads, kv_heads, dim, page_size, kind, dtype, seed, order)
    groups = len(prefixes)
    q = _randn((len(own), q_heads, dim), dtype, seed + 7) * sharp
    # (a table wide enough for so many rows that they are not read for each sequence)
    pad = torch.full((groups, (1 << 22) // page_size if wide else 0), -1, dtype=torch.int32, device="cuda")
    table = torch.cat([table[:groups], pad], 1), table[groups:]
    both = [tuple(torch.cat([kvs[b // share][i], kvs[groups + b][i]]) for i in (0, 1)) for b in range(0, len(own), every)]
    return cache, table[0], lens[:groups], table[1], lens[groups:], q, both


def _check_prefix(out, lse, q, both, scale, out_type):
    """Bounds.  A score is off by at most e = (dim + 4) u scale sum|q||k|, a weight by 2^-22 more, as two 16-bit parts by 2^-16,
    sums over n rows by n u.  The two parts' weights come from logarithms that are each off by e + 2^-22 + n u + 2^-22 |lse|, and
    from two exponentials, a sum and a quotient, 2^-21 together."""
    group = q.shape[1] // both[0][0].shape[1]
    for b in range(q.shape[0]):
        k, v = (x.repeat_interleave(group, 1) for x in both[b])
        n = k.shape[0]
        if n == 0:
            assert bool((out[b] == 0).all()) and bool((lse[b] == -math.inf).all())
            continue
        y = torch.einsum("hd,nhd->hn", q[b].double(), k) * scale
        e = ((q.shape[2] + 4) * U32 * abs(scale) * torch.einsum("hd,nhd->hn", q[b].double().abs(), k.abs())).amax(-1)
        p = torch.softmax(y, -1)
        want, size = torch.einsum("hn,nhd->hd", p, v), torch.einsum("hn,nhd->hd", p, v.abs())
        want_lse = torch.logsumexp(y, -1)
        lse_off = e + 2.0 ** -22 + n * U32 + 2.0 ** -22 * torch.maximum(want_lse.abs(), y.abs().amax(-1))
        rel = 2 * e + 2.0 ** -21 + 2.0 ** -16 + 2 * n * U32 + 2 * lse_off + 2.0 ** -21
        tol = rel[:, None] * size + ROUND[out_type] * want.abs() * (1 + 2 ** -7) + TINY[out_type]
        off = (out[b].double() - want).abs()
        assert bool((off <= tol).all()), (b, n, float((off / tol.clamp(min=1e-300)).max()))
        assert bool(((lse[b].double() - want_lse).abs() <= 2 * lse_off + 2.0 ** -21).all()), (b, n)


OWN = [0, 1, 5, 16, 17, 33, 3, 0, 64, 65, 2, 130]


@pytest.mark.gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("q_heads,kv_heads,dim,page_size", [
    (8, 2, 128, 16), (1, 1, 64, 1), (6, 6, 80, 5), (10, 2, 96, 24), (16, 1, 256, 32), (9, 1, 64, 48), (40, 2, 72, 7), (3, 3, 33, 4),
    (2, 1, 1, 3), (24, 8, 200, 48), (32, 4, 128, 64)])
@pytest.mark.parametrize("share", [1, 3, 12])
@pytest.mark.parametrize("wide", [False, True])
def test_prefix_attention(kind, dtype, q_heads, kv_heads, dim, page_size, share, wide):
    prefixes = [129, 0, 1, 300, 64, 127, 128, 2, 31, 33, 500, 16][:12 // share]
    if share == 12:
        prefixes = [777]
    order = "token" if page_size % 2 else "head"
    cache, pt, pn, t, n, q, both = _prefix_case(prefixes, OWN, share, q_heads, kv_heads, dim, page_size, kind, dtype, order=order, wide=wide)
    plan = gar.gar_attn_plan_create(q_heads, kv_heads, dim)
    out, lse = gar.gar_prefix_attention(plan, q, cache, pt, pn, t, n, lse=True)
    assert out.dtype == q.dtype
    _check_prefix(out, lse, q, both, dim ** -0.5, dtype)
    # 32-bit outputs, strided query and output, another scale, workspaces that are used again
    wide_q = torch.zeros(len(OWN), q_heads, dim + 5, dtype=q.dtype, device="cuda")
    wide_q[..., 3:3 + dim] = q
    wide = torch.full((len(OWN), q_heads + 1, dim), 7.0, device="cuda")
    got, lse = gar.gar_prefix_attention(plan, wide_q[..., 3:3 + dim], cache, pt, pn, t, n, scale=0.3, lse=True, out=wide[:, 1:])
    _check_prefix(got, lse, q, both, 0.3, "f32")
    assert bool((wide[:, 0] == 7).all())
    gar.gar_kv_status(cache)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,dtype,dim", [("bf16", "bf16", 128), ("f16", "f16", 64), ("bf16", "bf16", 96), ("i8", "bf16", 128),
                                            ("e4m3", "f16", 128), ("f32", "f32", 64), ("f16", "f16", 80), ("i8", "f16", 64)])
@pytest.mark.parametrize("share,q_heads,kv_heads,prefix", [(40, 8, 2, 5000), (150, 4, 1, 1025), (33, 16, 2, 255), (300, 2, 2, 640),
                                                           (16, 8, 1, 20000), (129, 1, 1, 3)])
def test_prefix_attention_of_many_queries(kind, dtype, dim, share, q_heads, kv_heads, prefix):
    own = [(7 * b) % 40 for b in range(share)]
    cache, pt, pn, t, n, q, both = _prefix_case([prefix], own, share, q_heads, kv_heads, dim, 16, kind, dtype, sharp=3.0)
    plan = gar.gar_attn_plan_create(q_heads, kv_heads, dim)
    out, lse = gar.gar_prefix_attention(plan, q, cache, pt, pn, t, n, lse=True)
    _check_prefix(out, lse, q, both, dim ** -0.5, dtype)
    again = gar.gar_prefix_attention(plan, q, cache, pt, pn, t, n, lse=True)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    gar.gar_kv_status(cache)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,dim,page_size,share,prefix", [
    ("bf16", 128, 64, 32, 60000), ("f16", 64, 128, 32, 50001), ("bf16", 128, 256, 64, 33000), ("f16", 128, 24, 32, 40000),
    ("bf16", 64, 32, 100, 40129), ("bf16", 96, 16, 24, 40000), ("f16", 128, 8, 64, 20000)])
def test_prefix_attention_many_tiles_each(kind, dim, page_size, share, prefix):
    """Parts of dozens of tiles: every stage of the ring is used many times; results do not depend on timing."""
    own = [(7 * b) % 40 for b in range(share)]
    cache, pt, pn, t, n, q, both = _prefix_case([prefix], own, share, 32, 8, dim, page_size, kind, kind, sharp=2.0, every=9)
    plan = gar.gar_attn_plan_create(32, 8, dim)
    out, lse = gar.gar_prefix_attention(plan, q, cache, pt, pn, t, n, lse=True)
    for _ in range(20):
        again = gar.gar_prefix_attention(plan, q, cache, pt, pn, t, n, lse=True)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    _check_prefix(out[::9], lse[::9], q[::9], both, dim ** -0.5, kind)
    gar.gar_kv_status(cache)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_prefix_attention_holds_its_sums(kind):
    """131072 rows of values that are all the same, a whole item to a CTA.  The tensor cores cut off less than 2^-23 of a sum for each
    product; the sums of 16 tiles, of 16 products each, are held by them: 2^-15.  The weights' two parts 2^-16, and sums in 32 bits of
    them, 64 to an addition chain, 32 chains of a tile's 4 and 2048 of a part: under 2^-16 if they are rounded."""
    n, share, q_heads, heads, dim, ps = 131072, 76, 256, 8, 64, 128
    pages = n // ps
    k = _randn((pages, heads, ps, dim), kind, 1)
    v = torch.full((pages, heads, ps, dim), 1.0 / 3, device="cuda").to(TORCH[kind])
    cache, plan = gar.KVCache(k, v), gar.gar_attn_plan_create(q_heads, heads, dim)
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    none, zero = torch.zeros((share, 0), dtype=torch.int32, device="cuda"), torch.zeros(share, dtype=torch.int32, device="cuda")
    q = _randn((share, q_heads, dim), kind, 2) * 0.2
    out = torch.empty((share, q_heads, dim), device="cuda")
    gar.gar_prefix_attention(plan, q, cache, table, lens, none, zero, out=out)
    off = (out.double() / float(v[0, 0, 0, 0]) - 1).abs().max()
    assert float(off) <= 2.0 ** -15 + 2.0 ** -16 + 2.0 ** -16, float(off)


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [0.0, -0.1])
@pytest.mark.parametrize("wide", [False, True])
def test_prefix_attention_scales(scale, wide):
    cache, pt, pn, t, n, q, both = _prefix_case([300], [b % 9 for b in range(40)], 40, 4, 2, 64, 16, "bf16", "bf16", wide=wide)
    plan = gar.gar_attn_plan_create(4, 2, 64)
    out, lse = gar.gar_prefix_attention(plan, q, cache, pt, pn, t, n, scale=scale, lse=True)
    _check_prefix(out, lse, q, both, scale, "bf16")


@pytest.mark.gpu
@pytest.mark.parametrize("kind,dtype", [("bf16", "bf16"), ("i8", "f16"), ("f32", "f32")])
def test_prefix_attention_several_prefixes_of_many_queries(kind, dtype):
    prefixes = [700, 0, 1, 2500, 129]
    share, q_heads, kv_heads, dim = 21, 16, 2, 128
    own = [(5 * b) % 23 for b in range(share * len(prefixes))]
    cache, pt, pn, t, n, q, both = _prefix_case(prefixes, own, share, q_heads, kv_heads, dim, 24, kind, dtype)
    plan = gar.gar_attn_plan_create(q_heads, kv_heads, dim)
    out, lse = gar.gar_prefix_attention(plan, q, cache, pt, pn, t, n, lse=True)
    _check_prefix(out, lse, q, both, dim ** -0.5, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,dtype,dim,share", [("bf16", "bf16", 128, 2), ("bf16", "bf16", 128, 64), ("f16", "f16", 64, 64), ("f32", "f32", 64, 64)])
@pytest.mark.parametrize("wide", [False, True])
def test_prefix_attention_drafts_are_one_long_sequence(kind, dtype, dim, share, wide):
    """Drafts over a context, their rows in pages of one table: each sees those before it."""
    cache, table, lens, _, kvs = _attn_case([1000, share], 8, 2, dim, 16, kind, dtype)
    q = _randn((share, 8, dim), dtype, 3)
    n = torch.arange(1, share + 1, dtype=torch.int32, device="cuda")
    plan = gar.gar_attn_plan_create(8, 2, dim)
    prefix = torch.cat([table[:1], torch.full((1, 1 << 18 if wide else 1), -1, dtype=torch.int32, device="cuda")], 1)
    out, lse = gar.gar_prefix_attention(plan, q, cache, prefix, lens[:1], table[1:].expand(share, -1), n, lse=True)
    both = [tuple(torch.cat([kvs[0][i], kvs[1][i][:b + 1]]) for i in (0, 1)) for b in range(share)]
    _check_prefix(out, lse, q, both, dim ** -0.5, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("share,wide", [(2, False), (2, True), (64, False), (64, True)])
def test_prefix_attention_bad_pages_and_lengths(share, wide):
    """A page that is none counts as rows of zeros, a length past the table as the longest."""
    dim, ps = 64, 16
    cache, table, lens, _, kvs = _attn_case([40] + [3] * share, 4, 2, dim, ps, "bf16", "bf16")
    q = _randn((share, 4, dim), "bf16", 3)
    plan = gar.gar_attn_plan_create(4, 2, dim)
    for bad in (-1, cache.pages, 2 ** 31 - 1):
        broken = torch.cat([table[:1], torch.full((1, 1 << 18 if wide else 1), -1, dtype=torch.int32, device="cuda")], 1)
        broken[0, 1] = bad
        out, lse = gar.gar_prefix_attention(plan, q, cache, broken[:1], lens[:1], table[1:], lens[1:], lse=True)
        both = []
        for b in range(share):
            kv = [torch.cat([kvs[0][i], kvs[1 + b][i]]) for i in (0, 1)]
            kv = [x.clone() for x in kv]
            for x in kv:
                x[16:32] = 0
            both.append(tuple(kv))
        _check_prefix(out, lse, q, both, dim ** -0.5, "bf16")
        with pytest.raises(gar.GarError) as e:
            gar.gar_kv_status(cache)
        assert "page" in str(e.value)
    for bad in (-5, 10 ** 6):
        n = lens[:1].clone()
        n[0] = bad
        narrow = table[:1, :3].clone()
        narrow[0, 2] = narrow[0, 1]
        if wide and bad < 0:
            narrow = torch.cat([narrow, torch.full((1, 1 << 18), -1, dtype=torch.int32, device="cuda")], 1)
        out, lse = gar.gar_prefix_attention(plan, q, cache, narrow, n, table[1:], lens[1:], lse=True)
        with pytest.raises(gar.GarError) as e:
            gar.gar_kv_status(cache)
        assert "length" in str(e.value)
        if bad < 0:
            _check_prefix(out, lse, q, [kvs[1 + b] for b in range(share)], dim ** -0.5, "bf16")


@pytest.mark.gpu
def test_prefix_attention_without_a_table():
    """Widths of zero: nothing but the prefix, or nothing but the sequences' own rows, or nothing."""
    cache, table, lens, _, kvs = _attn_case([100, 20, 30], 4, 2, 64, 16, "bf16", "bf16")
    q = _randn((2, 4, 64), "bf16", 5)
    plan = gar.gar_attn_plan_create(4, 2, 64)
    zero = torch.zeros(2, dtype=torch.int32, device="cuda")
    none = torch.zeros((2, 0), dtype=torch.int32, device="cuda")
    out, lse = gar.gar_prefix_attention(plan, q, cache, table[:1], lens[:1], none, zero, lse=True)
    _check_prefix(out, lse, q, [kvs[0]] * 2, 0.125, "bf16")
    out, lse = gar.gar_prefix_attention(plan, q, cache, none[:1], zero[:1], table[1:], lens[1:], lse=True)
    _check_prefix(out, lse, q, kvs[1:], 0.125, "bf16")
    out, lse = gar.gar_prefix_attention(plan, q, cache, none[:1], zero[:1], none, zero, lse=True)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    out = gar.gar_prefix_attention(plan, q[:0], cache, none[:0], zero[:0], none[:0], zero[:0])
    assert out.shape == (0, 4, 64)


# ---------------------------------------------------------------------------- weights that rows gather

def _check_weigh(got, weights, q, kvs, lengths, lse, window, scale):
    """Bounds.  e, a score's, as above; its logarithm's factor, a difference and an exponential 2^-22 |lse| + 2^-21;
    sums over the queries and the last addition of u each."""
    group = q.shape[1] // weights.shape[1]
    want = weights.double()
    tol = torch.zeros_like(want)
    for b, n in enumerate(lengths):
        lo = max(0, n - window) if window else 0
        if n == lo:
            continue
        k = kvs[b][0][lo:].repeat_interleave(group, 1)
        y = torch.einsum("hd,nhd->hn", q[b].double(), k) * scale
        e = (q.shape[2] + 8) * U32 * scale * torch.einsum("hd,nhd->hn", q[b].double().abs(), k.abs())
        p = torch.where(lse[b].double()[:, None] == -math.inf, 0.0, torch.exp(y - lse[b].double()[:, None]))
        rel = e + 2.0 ** -22 * lse[b].double().abs()[:, None].nan_to_num(posinf=0) + 2.0 ** -21 + (group + 1) * U32
        want[b, :, lo:n] += p.view(-1, group, n - lo).sum(1)
        tol[b, :, lo:n] = (rel * p).view(-1, group, n - lo).sum(1) * (1 + 2 ** -7) + U32 * want[b, :, lo:n].abs() * 2 + 1e-37
    off = (got.double() - want).abs()
    assert bool((off <= tol).all()), float((off / tol.clamp(min=1e-300)).max())


@pytest.mark.gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("q_heads,kv_heads,dim,page_size,window", [
    (8, 2, 128, 16, 0), (1, 1, 64, 1, 0), (6, 6, 80, 5, 7), (10, 2, 96, 24, 0), (16, 1, 256, 32, 0), (32, 2, 128, 64, 100),
    (9, 1, 64, 16, 1), (40, 2, 72, 7, 33), (3, 3, 33, 4, 0), (2, 1, 1, 3, 0), (24, 8, 200, 48, 0), (130, 2, 192, 16, 0)])
def test_weigh(kind, dtype, q_heads, kv_heads, dim, page_size, window):
    lengths = [0, 1, 2, 15, 16, 17, 31, 33, 64, 65, 127, 128, 130, 300]
    order = "token" if page_size % 2 else "head"
    cache, table, lens, q, kvs = _attn_case(lengths, q_heads, kv_heads, dim, page_size, kind, dtype, order=order)
    plan = gar.gar_attn_plan_create(q_heads, kv_heads, dim)
    _, lse = gar.gar_decode_attention(plan, q, cache, table, lens, window=window, lse=True)
    rows = table.shape[1] * page_size
    weights = torch.rand((len(lengths), kv_heads, rows), generator=_gen(1), device="cuda")
    kept = weights.clone()
    got = gar.gar_kv_weigh(q, cache, table, lens, lse, weights, window=window)
    assert torch.equal(weights, kept) and got.shape == weights.shape
    _check_weigh(got, weights, q, kvs, lengths, lse, window, dim ** -0.5)
    # what was added is the queries' number
    for b, n in enumerate(lengths):
        if n:
            assert abs(float((got[b].double() - weights[b].double()).sum()) - q_heads) < 1e-3 * q_heads
    # in place, strided, another scale
    wide_q = torch.zeros(len(lengths), q_heads, dim + 5, dtype=q.dtype, device="cuda")
    wide_q[..., 3:3 + dim] = q
    wide = torch.full((len(lengths), kv_heads + 1, rows + 3), 7.0, device="cuda")
    part = wide[:, 1:, 2:2 + rows]
    part.copy_(weights)
    back = gar.gar_kv_weigh(wide_q[..., 3:3 + dim], cache, table, lens, lse, part, scale=0.2 * dim ** -0.5, window=window, out=part)
    assert back is part
    _check_weigh(part, weights, q, kvs, lengths, lse, window, 0.2 * dim ** -0.5)
    assert bool((wide[:, 0] == 7).all()) and bool((wide[:, :, :2] == 7).all()) and bool((wide[:, :, -1] == 7).all())
    gar.gar_kv_status(cache)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,dtype,q_heads,kv_heads,dim,lengths", [
    ("bf16", "bf16", 8, 2, 128, [20000]), ("i8", "f16", 4, 4, 64, [9000, 3, 0, 5000, 1]), ("f32", "f32", 6, 2, 80, [7000, 200]),
    ("f16", "f16", 2, 1, 64, [(37 * b) % 90 for b in range(500)]), ("e4m3", "bf16", 8, 8, 128, [4000] * 9)])
def test_weigh_long_and_many(kind, dtype, q_heads, kv_heads, dim, lengths):
    cache, table, lens, q, kvs = _attn_case(lengths, q_heads, kv_heads, dim, 16, kind, dtype, sharp=2.0)
    plan = gar.gar_attn_plan_create(q_heads, kv_heads, dim)
    _, lse = gar.gar_decode_attention(plan, q, cache, table, lens, lse=True)
    weights = torch.rand((len(lengths), kv_heads, table.shape[1] * 16 + 5), generator=_gen(1), device="cuda")
    got = gar.gar_kv_weigh(q, cache, table, lens, lse, weights)
    _check_weigh(got, weights, q, kvs, lengths, lse, 0, dim ** -0.5)
    assert torch.equal(got, gar.gar_kv_weigh(q, cache, table, lens, lse, weights))


@pytest.mark.gpu
@pytest.mark.parametrize("kind,dtype,dim", [("bf16", "bf16", 64), ("f32", "f32", 64), ("f16", "f16", 33)])
def test_weigh_edges(kind, dtype, dim):
    """Heads whose sum is nothing; infinite keys; bad pages and lengths; fewer rows than the table holds."""
    cache, table, lens, q, kvs = _attn_case([40, 20], 4, 2, dim, 16, kind, dtype)
    weights = torch.rand((2, 2, 50), generator=_gen(1), device="cuda")
    plan = gar.gar_attn_plan_create(4, 2, dim)
    _, lse = gar.gar_decode_attention(plan, q, cache, table, lens, lse=True)
    lse[0, 1] = -math.inf
    lse[1, 2] = math.inf                     # all of its weights vanish
    got = gar.gar_kv_weigh(q, cache, table, lens, lse, weights)
    _check_weigh(got, weights, q, kvs, [40, 20], lse.where(lse < math.inf, 1e5), 0, dim ** -0.5)
    # a key of -infinity against a positive query has no weight, the others keep theirs
    _, lse = gar.gar_decode_attention(plan, q, cache, table, lens, lse=True)
    q2 = q.clone()
    q2[..., 0] = 1.0
    kvs2 = [tuple(x.clone() for x in kv) for kv in kvs]
    page, row = int(table[0, 1]), 3
    cache.k[page, :, row, 0] = -math.inf
    kvs2[0][0][19, :, 0] = -1e9
    got = gar.gar_kv_weigh(q2, cache, table, lens, lse, weights)
    assert torch.equal(got[0, :, 19], weights[0, :, 19])
    got[0, :, 19] = weights[0, :, 19]
    kvs2[0][0][19] = 0
    kvs2[0][0][19, :, 0] = -1e5
    _check_weigh(got, weights, q2, kvs2, [40, 20], lse, 0, dim ** -0.5)
    gar.gar_kv_status(cache)
    broken = table.clone()
    broken[1, 0] = cache.pages
    got = gar.gar_kv_weigh(q, cache, broken, lens, lse, weights)
    kvs2 = [kvs[0], tuple(torch.cat([torch.zeros_like(x[:16]), x[16:]]) for x in kvs[1])]
    _check_weigh(got[1:], weights[1:], q[1:], kvs2[1:], [20], lse[1:], 0, dim ** -0.5)
    with pytest.raises(gar.GarError) as e:
        gar.gar_kv_status(cache)
    assert "page" in str(e.value)
    short = weights[:, :, :10].contiguous()
    got = gar.gar_kv_weigh(q, cache, table, lens, lse, short)
    _check_weigh(got[1:], short[1:], q[1:], [tuple(x[:10] for x in kvs[1])], [10], lse[1:], 0, dim ** -0.5)
    with pytest.raises(gar.GarError) as e:
        gar.gar_kv_status(cache)
    assert "length" in str(e.value)
    empty = gar.gar_kv_weigh(q[:0], cache, table[:0], lens[:0], lse[:0], weights[:0])
    assert empty.shape == (0, 2, 50)


# ---------------------------------------------------------------------------- eviction

def _evict_reference(weights, positions, n, keep, first, recent):
    """(targets, sources) of one sequence's head, by sorting on the CPU."""
    if n <= keep:
        return [], []
    newest = max(positions[:n])
    key = []
    for r in range(n):
        w = weights[r]
        if r < first or positions[r] > newest - recent:
            key.append((-2, 0.0, r))
        else:
            key.append((0, 0.0, r) if math.isnan(w) else (-1, -w, r))
    kept = set(r for _, _, r in sorted(key)[:keep])
    return [r for r in range(keep) if r not in kept], sorted(r for r in kept if r >= keep)


def _check_evict(cache, table, lens, weights, positions, keep, first, recent, order_check=True):
    ps = cache.page_size
    before = [t.clone() for t in cache.tensors]
    got_w, got_p, got_n = gar.gar_kv_evict(cache, weights, positions, table, lens, keep, first=first, recent=recent)
    want = [t.view(torch.uint8) if t.element_size() == 1 else t for t in [x.clone() for x in before]]
    old = [t.view(torch.uint8) if t.element_size() == 1 else t for t in before]
    w, p, tab = weights.cpu(), positions.cpu(), table.cpu()
    want_w, want_p = torch.zeros_like(w), torch.full_like(p, -1)
    for b, n in enumerate(lens.tolist()):
        m = min(n, keep)
        for h in range(cache.heads):
            to, frm = _evict_reference(w[b, h].tolist(), p[b, h].tolist(), n, keep, first, recent)
            assert len(to) == len(frm)
            want_w[b, h, :m], want_p[b, h, :m] = w[b, h, :m], p[b, h, :m]
            if to:
                to, frm = torch.tensor(to), torch.tensor(frm)
                want_w[b, h, to], want_p[b, h, to] = w[b, h, frm], p[b, h, frm]
                tp, fp = tab[b, to // ps].long().cuda(), tab[b, frm // ps].long().cuda()
                tr, fr = (to % ps).cuda(), (frm % ps).cuda()
                for x, y in zip(want, old):
                    x[tp, h, tr] = y[fp, h, fr]
    assert torch.equal(got_n.cpu(), lens.cpu().clamp(max=keep))
    assert torch.equal(got_p.cpu(), want_p)
    assert torch.equal(got_w.cpu().view(torch.int32), want_w.view(torch.int32))
    for got, x in zip(cache.tensors, want):
        y = got.view(torch.uint8) if got.element_size() == 1 else got
        assert torch.equal(y.view(torch.uint8) if y.dtype == torch.uint8 else y.view(torch.int16 if y.element_size() == 2 else torch.int32),
                           x.view(torch.uint8) if x.dtype == torch.uint8 else x.view(torch.int16 if x.element_size() == 2 else torch.int32))
    return got_w, got_p, got_n


def _evict_case(lengths, heads, dim, page_size, kind, seed=0, order="head", extra=0, shape="mixed"):
    need = [-(-n // page_size) for n in lengths]
    g = _gen(seed)
    pages = sum(need) + 2
    cache = _empty_cache(pages, heads, page_size, dim, kind, order)
    for t in cache.tensors:
        if t.element_size() == 1:
            t.view(torch.uint8).copy_(torch.randint(0, 256, t.shape, generator=g, device="cuda", dtype=torch.uint8))
        else:
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
    ids = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    width = max(need + [1])
    table = torch.full((len(lengths), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, k in enumerate(need):
        table[b, :k] = ids[at:at + k]
        at += k
    size = (len(lengths), heads, width * page_size + extra)
    w = torch.randn(size, generator=g, device="cuda")
    u = torch.rand(size, generator=g, device="cuda")
    if shape == "mixed":
        w = torch.where(u < 0.1, 0.0, torch.where(u < 0.2, -0.0, torch.where(u < 0.4, 1.5, w.exp())))
    elif shape == "same":
        w = torch.ones_like(w)
    elif shape == "odd":
        for i, x in enumerate((math.nan, math.inf, -math.inf, 1e-42, -1e-42, -math.nan, 0.0, -0.0)):
            w = torch.where((u > i * 0.1) & (u < i * 0.1 + 0.1), x, w)
    pos = torch.rand(size, generator=g, device="cuda").argsort(-1).to(torch.int32) * 3 + 5
    return cache, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), w, pos


LENGTHS = [0, 1, 7, 8, 9, 33, 64, 100, 257, 300]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32", "i8", "e4m3"])
@pytest.mark.parametrize("heads,dim,page_size,order", [(2, 128, 16, "head"), (3, 33, 5, "token"), (1, 1, 1, "head"), (2, 96, 24, "token"),
                                                       (1, 256, 64, "head"), (5, 2, 3, "head")])
def test_evict(kind, heads, dim, page_size, order):
    cache, table, lens, w, p = _evict_case(LENGTHS, heads, dim, page_size, kind, order=order, extra=3)
    for keep, first, recent in ((8, 0, 0), (8, 4, 4), (64, 3, 20), (257, 0, 1), (1, 0, 0), (1, 1, 0), (1, 0, 1), (500, 2, 2), (33, 33, 0), (33, 0, 33)):
        _check_evict(cache, table, lens, w, p, keep, first, recent)
    gar.gar_kv_status(cache)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", ["same", "odd", "mixed"])
@pytest.mark.parametrize("keep,first,recent", [(1, 0, 0), (100, 0, 0), (256, 5, 31), (299, 0, 0), (150, 0, 150)])
def test_evict_equal_and_odd_weights(shape, keep, first, recent):
    cache, table, lens, w, p = _evict_case([300, 299, 257, 512], 2, 16, 16, "bf16", shape=shape)
    _check_evict(cache, table, lens, w, p, keep, first, recent)


@pytest.mark.gpu
@pytest.mark.parametrize("lengths,keep,heads", [([5000, 16384, 100, 8191], 2048, 2), ([70000], 30000, 1), ([140001, 3], 70000, 2), ([20000] * 3, 19999, 1),
                                                ([2049] * 170, 2048, 2)])
def test_evict_long_sequences(lengths, keep, heads):
    cache, table, lens, w, p = _evict_case(lengths, heads, 8, 64, "bf16")
    _check_evict(cache, table, lens, w, p, keep, 4, keep // 10)


@pytest.mark.gpu
def test_evict_positions_at_the_ends_of_the_type():
    cache, table, lens, w, p = _evict_case([100, 100], 1, 16, 16, "bf16")
    p[0] = torch.arange(112, device="cuda") - 2 ** 31
    p[1] = 2 ** 31 - 1 - torch.arange(112, device="cuda")
    for recent in (0, 1, 50):
        _check_evict(cache, table, lens, w, p, 50, 0, recent)
    p.fill_(7)                               # all the newest: the lowest rows stay
    _check_evict(cache, table, lens, w, p, 50, 0, 1)


@pytest.mark.gpu
def test_evict_bad_pages_and_lengths():
    cache, table, lens, w, p = _evict_case([100, 60], 2, 16, 16, "bf16")
    lens = torch.tensor([500, -3], dtype=torch.int32, device="cuda")
    _, _, n = gar.gar_kv_evict(cache, w, p, table, lens, 50)
    assert n.tolist() == [50, 0]
    with pytest.raises(gar.GarError) as e:
        gar.gar_kv_status(cache)
    assert "length" in str(e.value)
    # rows on a page that is none are not copied; their weights and positions go on
    cache, table, lens, w, p = _evict_case([100, 60], 2, 16, 16, "bf16", seed=5)
    w[0, :, 80:96] = 100.0
    table[0, 5] = cache.pages
    before = [t.clone() for t in cache.tensors]
    got_w, _, _ = gar.gar_kv_evict(cache, w, p, table, lens, 50)
    assert int((got_w[0, 0] == 100).sum()) == 16
    with pytest.raises(gar.GarError) as e:
        gar.gar_kv_status(cache)
    assert "page" in str(e.value)
    used = table[:, :4].flatten()[table[:, :4].flatten() >= 0].long()
    other = [i for i in range(cache.pages) if i not in used.tolist()]
    for x, y in zip(cache.tensors, before):
        assert torch.equal(x[other], y[other])
    empty = gar.gar_kv_evict(cache, w[:0], p[:0], table[:0], lens[:0], 5)
    assert empty[2].shape == (0,)


# ---------------------------------------------------------------------------- verification of drafts

def _verify_reference(target, draft, tokens, uniform):
    clamp = lambda x: torch.where(x > 0, x, 0.0).clamp(max=1.0).double()
    p, q = clamp(target.cpu()), clamp(draft.cpu())
    u = torch.where(uniform.cpu() > 0, uniform.cpu(), 0.0).double()
    batch, drafts = tokens.shape
    vocab = p.shape[2]
    out = torch.full((batch, drafts + 1), -1, dtype=torch.int64)
    accepted = torch.zeros(batch, dtype=torch.int32)
    for b in range(batch):
        a, r = 0, None
        while a < drafts and int(tokens[b, a]) >= 0:
            t = int(tokens[b, a])
            if t >= vocab or not float(u[b, a] * q[b, a, t]) < float(p[b, a, t]):
                r = (p[b, a] - q[b, a]).clamp(min=0)
                break
            out[b, a] = t
            a += 1
        if r is None or not bool((r > 0).any()):
            r = p[b, a]
        total = r.cumsum(0)
        past = (total > u[b, drafts] * total[-1]).nonzero()
        some = (r > 0).nonzero()
        out[b, a] = int(past[0]) if len(past) else int(some[-1]) if len(some) else -1
        accepted[b] = a
    return out, accepted


def _verify_case(batch, drafts, vocab, dtype, seed=0, wide=True, spread=2.0):
    g = _gen(seed)
    x = torch.randn((batch, drafts + 1, vocab), generator=g, device="cuda") * spread
    target = torch.softmax(x, -1).to(TORCH[dtype])
    draft = torch.softmax(x[:, :-1] + torch.randn((batch, drafts, vocab), generator=g, device="cuda") * 0.5, -1).to(TORCH[dtype])
    tokens = torch.zeros((batch, drafts), dtype=torch.int64, device="cuda")
    if drafts:
        tokens = torch.multinomial(draft.float().flatten(0, 1), 1, generator=g).view(batch, drafts)
    return target, draft, tokens if wide else tokens.int(), torch.rand((batch, drafts + 1), generator=g, device="cuda")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("batch,drafts,vocab,wide", [(1, 4, 32768, True), (33, 3, 5003, False), (7, 0, 1000, True), (300, 1, 33, True), (5, 40, 100, False),
                                                     (3, 2, 1, True), (4, 33, 2, True), (2, 5, 200001, True), (700, 2, 4097, False), (3, 1, 31, True)])
def test_verify(dtype, batch, drafts, vocab, wide):
    target, draft, tokens, uniform = _verify_case(batch, drafts, vocab, dtype, wide=wide)
    got, accepted = gar.gar_verify_drafts(target, draft, tokens, uniform)
    want, want_accepted = _verify_reference(target, draft, tokens, uniform)
    assert got.dtype == tokens.dtype and torch.equal(accepted.cpu(), want_accepted) and torch.equal(got.cpu().long(), want)
    # strides, given outputs
    many = torch.full((batch, drafts + 2, vocab + 3), float("nan"), dtype=target.dtype, device="cuda")
    many[:, 1:, 1:1 + vocab] = target
    more = torch.full((drafts + 1, batch, vocab + 1), float("nan"), dtype=target.dtype, device="cuda")
    more[:drafts, :, :vocab] = draft.transpose(0, 1)
    out = torch.full((batch, drafts + 1), 5, dtype=tokens.dtype, device="cuda"), torch.zeros(batch, dtype=torch.int32, device="cuda")
    back = gar.gar_verify_drafts(many[:, 1:, 1:1 + vocab], more[:drafts, :, :vocab].transpose(0, 1), tokens, uniform, out=out)
    assert back is out and torch.equal(out[0].cpu().long(), want) and torch.equal(out[1].cpu(), want_accepted)


@pytest.mark.gpu
def test_verify_edges():
    vocab, n = 600, 12
    target, draft, tokens, uniform = _verify_case(n, 3, vocab, "f32", seed=4)
    tokens[0, 0] = -1                         # no drafts at all
    tokens[1, 1] = -7                         # one
    tokens[2, 0], tokens[3, 2] = vocab, 2 ** 40   # past the vocabulary
    uniform[4], uniform[5] = 0.0, 1.0 - 2.0 ** -24
    uniform[6] = 5.0                          # past every border: the last token that can be drawn
    uniform[7], uniform[8] = math.nan, -1.0
    target[9] = 0.0                           # nothing to draw
    target[10, :, ::2] = math.nan
    target[10, :, 1::4] = -3.0
    draft[11] = target[11, :3] * 2            # nothing is left of the target
    uniform[11, 0] = 0.9
    got, accepted = gar.gar_verify_drafts(target, draft, tokens, uniform)
    want, want_accepted = _verify_reference(target, draft, tokens, uniform)
    assert torch.equal(accepted.cpu(), want_accepted) and torch.equal(got.cpu(), want)
    assert got[9].tolist() == [-1] * 4
    empty = gar.gar_verify_drafts(target[:0], draft[:0], tokens[:0], uniform[:0])
    assert empty[0].shape == (0, 4) and empty[1].shape == (0,)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_verify_borders_are_exact(dtype):
    """Probabilities of 1/4096 each: sums are exact, and u = v/4096 is the border of tokens v - 1 and v."""
    vocab = 4096
    target = torch.full((vocab, 1, vocab), 2.0 ** -12, device="cuda", dtype=TORCH[dtype])
    uniform = torch.arange(vocab, device="cuda").float()[:, None] / vocab
    none = torch.zeros((vocab, 0, vocab), device="cuda", dtype=TORCH[dtype])
    got, _ = gar.gar_verify_drafts(target, none, torch.zeros((vocab, 0), dtype=torch.int64, device="cuda"), uniform)
    assert torch.equal(got[:, 0], torch.arange(vocab, device="cuda"))
    below = torch.nextafter(uniform, torch.zeros_like(uniform))
    got, _ = gar.gar_verify_drafts(target, none, torch.zeros((vocab, 0), dtype=torch.int64, device="cuda"), below)
    assert torch.equal(got[:, 0], (torch.arange(vocab, device="cuda") - 1).clamp(min=0))


@pytest.mark.gpu
def test_verify_gives_the_targets_distribution():
    """Over a fine grid of both random numbers: the mass of each token is the target's, to the grid's step."""
    p, q = torch.tensor([0.125, 0.5, 0.0, 0.25, 0.125]), torch.tensor([0.5, 0.125, 0.125, 0.25, 0.0])
    steps, mass = 64, torch.zeros(5, dtype=torch.float64)
    grid = (torch.arange(steps, device="cuda") + 0.5) / steps
    uniform = torch.stack(torch.meshgrid(grid, grid, indexing="ij"), -1).flatten(0, 1)
    for token in range(5):
        if q[token] == 0:
            continue
        n = uniform.shape[0]
        target, draft = p.cuda().expand(n, 2, 5), q.cuda().expand(n, 1, 5)
        got, accepted = gar.gar_verify_drafts(target, draft, torch.full((n, 1), token, dtype=torch.int64, device="cuda"), uniform)
        first = got[:, 0].cpu()
        for v in range(5):
            mass[v] += float(q[token]) * float((first == v).double().mean())
        assert float(accepted.double().mean()) == min(1.0, float(p[token] / q[token]))     # (multiples of 1/64)
    # what may be left of the target, (0, 0.375, 0, 0, 0.125), has its border at 48 of 64 steps
    assert bool((mass == p.double()).all()), mass
