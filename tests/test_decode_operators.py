"""Rotary positions, the paged cache and decode attention against plain 64-bit versions.

Tolerances come from the arithmetic, not from observed errors.  u = 2^-24 is the relative
rounding error of 32 bits, U that of the output type (2^-24, 2^-8 bf16, 2^-11 f16 -- half a
unit in the last place -- plus the type's smallest step for f16).
"""

import math

import pytest
import torch

from paper_2004_09362_gb300 import gar

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "i8": torch.int8,
         "e4m3": torch.float8_e4m3fn}
U32 = 2.0 ** -24
ROUND = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}
QMAX = {"i8": 127.0, "e4m3": 448.0}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(shape, dtype, seed):
    return torch.randn(shape, generator=_gen(seed), device="cuda").to(TORCH[dtype])


# ---------------------------------------------------------------------------- frequencies (CPU)

def test_frequencies():
    f, m = gar.gar_rope_frequencies(64, 10000.0)
    assert m == 1.0 and len(f) == 32
    assert all(abs(f[i] - 10000.0 ** (-2 * i / 64)) < 1e-15 for i in range(32))
    g, m = gar.gar_rope_frequencies(64, 10000.0, "linear", 4.0)
    assert m == 1.0 and all(abs(a / 4 - b) < 1e-15 for a, b in zip(f, g))
    g, m = gar.gar_rope_frequencies(64, 10000.0, "base", 4.0)
    assert m == 1.0 and g[0] == 1.0 and abs(g[-1] * 4 / f[-1] - 1) < 1e-12   # fastest kept, slowest divided
    g, m = gar.gar_rope_frequencies(64, 10000.0, "parts", 4.0, 4096.0)
    assert abs(m - (0.1 * math.log(4.0) + 1)) < 1e-15
    for a, b in zip(f, g):
        turns = 4096 * a / (2 * math.pi)
        want = a if turns >= 32 else a / 4 if turns <= 1 else None
        if want is not None:
            assert abs(b / want - 1) < 1e-12
        else:
            assert a / 4 < b < a


@pytest.mark.parametrize("args", [(0,), (3,), (258,), (64, 1.0), (64, float("nan")), (64, 1e4, 9), (64, 1e4, "linear", 0.5),
                                  (64, 1e4, "parts", 2.0, 0.0), (2, 1e4, "base", 2.0)])
def test_frequency_refusals(args):
    with pytest.raises((gar.GarError, ValueError)):
        gar.gar_rope_frequencies(*args)


# ---------------------------------------------------------------------------- refusals (no GPU work)

def _rope_raw(x=4096, out=8192, dtype=gar.GAR_BF16, tokens=4, heads=2, dim=64, rot=64, positions=4096, width=8,
              table=4096, rows=16, layout=0, xs=(128, 64), os_=(128, 64)):
    return gar._lib.gar_rope(x, xs[0], xs[1], out, os_[0], os_[1], dtype, tokens, heads, dim, rot, positions, width,
                             table, rows, layout, 0, None)


@pytest.mark.parametrize("bad,code", [
    (dict(x=None), -1), (dict(out=None), -1), (dict(positions=None), -1), (dict(table=None), -1), (dict(dtype=gar.GAR_I32), -1),
    (dict(dtype=gar.GAR_I8), -1), (dict(dim=257, rot=64), -1), (dict(rot=3), -1), (dict(rot=66), -1), (dict(rot=0), -1),
    (dict(tokens=-1), -1), (dict(heads=-1), -1), (dict(heads=(1 << 20) + 1), -1), (dict(layout=2), -1), (dict(width=2), -1), (dict(rows=-1), -1),
    (dict(x=4097), -3), (dict(table=4100), -3), (dict(positions=4100), -3), (dict(out=4096, os_=(64, 64)), -1)])
def test_rope_refusals(bad, code):
    assert _rope_raw(**bad) == code
    assert gar.gar_last_error()


def _cache_raw(**kw):
    f = dict(k=4096, v=8192, k_scale=None, v_scale=None, status=None, pages=4, page_stride=16 * 2 * 64,
             head_stride=16 * 64, token_stride=64, dtype=gar.GAR_BF16, heads=2, dim=64, page_size=16)
    f.update(kw)
    return gar.gar_kv_cache(**f)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=gar.GAR_I32), -1), (dict(dtype=9), -1), (dict(heads=0), -1), (dict(dim=0), -1), (dict(dim=300), -1),
    (dict(page_size=0), -1), (dict(pages=-1), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(dtype=gar.GAR_I8), -1),
    (dict(k=4097), -3), (dict(dtype=gar.GAR_E4M3, k_scale=4098, v_scale=4096), -3)])
def test_cache_refusals(bad, code):
    c = _cache_raw(**bad)
    args = (4096, 128, 64, 4096, 128, 64, gar.GAR_BF16, 4, 4096, None, 8, None, 0, 0, 0, None)
    assert gar._lib.gar_kv_write(c, *args) == code
    assert gar._lib.gar_kv_read(c, 4096, 4, 4096, 8192, gar.GAR_BF16, None) == code
    assert gar._lib.gar_kv_status(c, None, None) == code


def test_write_and_read_refusals():
    c = _cache_raw()
    ok = dict(k=4096, ks=(128, 64), v=4096, vs=(128, 64), dtype=gar.GAR_BF16, tokens=4, slots=4096, positions=None,
              width=8, table=None, rows=0, rot=0, layout=0)

    def write(**kw):
        a = dict(ok, **kw)
        return gar._lib.gar_kv_write(c, a["k"], *a["ks"], a["v"], *a["vs"], a["dtype"], a["tokens"], a["slots"],
                                     a["positions"], a["width"], a["table"], a["rows"], a["rot"], a["layout"], None)

    rotated = dict(positions=4096, table=4096, rows=8, rot=64)
    for kw, code in [(dict(dtype=gar.GAR_F32), -1), (dict(dtype=gar.GAR_I8), -1), (dict(tokens=-1), -1), (dict(k=None), -1),
                     (dict(v=None), -1), (dict(slots=None), -1), (dict(slots=4100), -3), (dict(k=4097), -3),
                     (dict(rotated, rot=66), -1), (dict(rotated, rot=7), -1), (dict(rotated, layout=5), -1),
                     (dict(rotated, width=3), -1), (dict(rotated, table=None), -1), (dict(rotated, table=4100), -3)]:
        assert write(**kw) == code, kw
    assert write(tokens=0, k=None, v=None, slots=None) == 0
    for args, code in [((None, 4, 4096, 8192, gar.GAR_BF16), -1), ((4096, 4, None, 8192, gar.GAR_BF16), -1),
                       ((4096, -1, 4096, 8192, gar.GAR_BF16), -1), ((4096, 4, 4096, 8192, gar.GAR_F32), -1),
                       ((4096, 4, 4097, 8192, gar.GAR_BF16), -3)]:
        assert gar._lib.gar_kv_read(c, *args, None) == code, args
    assert gar._lib.gar_kv_read(None, 4096, 4, 4096, 8192, gar.GAR_BF16, None) == -1


@pytest.mark.parametrize("args", [(0, 1, 64), (4, 0, 64), (5, 2, 64), (4, 2, 0), (4, 2, 257)])
def test_plan_refusals(args):
    with pytest.raises(gar.GarError) as e:
        gar.gar_attn_plan_create(*args)
    assert e.value.code == -1


def test_plan_shape():
    plan = gar.gar_attn_plan_create(6, 2, 80)
    assert gar.gar_attn_plan_shape(plan) == (6, 2, 80)
    assert gar._lib.gar_attn_plan_shape(None, None, None, None) == -1


def test_attention_refusals_without_a_gpu():
    plan = gar.gar_attn_plan_create(4, 2, 64)
    assert gar.gar_attn_plan_bytes(plan) > 0
    with pytest.raises(gar.GarError) as e:
        gar.gar_attn_plan_set_workspace(plan, 4100, 1 << 30)
    assert e.value.code == -3
    with pytest.raises(gar.GarError) as e:
        gar.gar_attn_plan_set_workspace(plan, 4096, 16)
    assert e.value.code == -6

    def call(cache=None, q=4096, q_dtype=gar.GAR_BF16, out=8192, out_dtype=gar.GAR_BF16, lse=None, table=4096, width=4,
             lengths=4096, batch=2, scale=0.125, window=0, p=plan.handle):
        return gar._lib.gar_decode_attention(p, cache or _cache_raw(), q, 256, 64, q_dtype, out, 256, 64, out_dtype, lse,
                                             table, width, width, lengths, batch, scale, window, None)

    for kw, code in [(dict(p=None), -1), (dict(cache=_cache_raw(heads=3)), -1), (dict(cache=_cache_raw(dim=32)), -1),
                     (dict(q_dtype=gar.GAR_I8), -1), (dict(q_dtype=gar.GAR_F16), -1), (dict(out_dtype=gar.GAR_F16), -1),
                     (dict(batch=-1), -1), (dict(width=-1), -1), (dict(window=-1), -1), (dict(scale=float("inf")), -1),
                     (dict(q=None), -1), (dict(out=None), -1), (dict(lengths=None), -1), (dict(table=None), -1),
                     (dict(q=4097), -3), (dict(lse=4098), -3), (dict(lengths=4098), -3), (dict(), -6)]:
        assert call(**kw) == code, kw
    assert call(batch=0) == 0
    gar.gar_attn_plan_destroy(plan)
    with pytest.raises(ValueError):
        plan.handle


def test_allreduce_plans_refuse_the_decoding_types():
    for t in (gar.GAR_F16, gar.GAR_I8, gar.GAR_E4M3):
        with pytest.raises(gar.GarError):
            gar.gar_plan_create(4, 16, dtype=t)


# ---------------------------------------------------------------------------- rotary positions

def _rope64(x, pos, f, m, layout, inverse):
    rot = 2 * len(f)
    a = pos.double()[:, None, None] * torch.tensor(f, dtype=torch.float64, device="cuda")
    c, s = a.cos() * m, a.sin() * m * (-1 if inverse else 1)
    y = x.double().clone()
    i = slice(0, rot // 2) if layout == "half" else slice(0, rot, 2)
    j = slice(rot // 2, rot) if layout == "half" else slice(1, rot, 2)
    u, v = x[..., i].double(), x[..., j].double()
    y[..., i], y[..., j] = u * c - v * s, v * c + u * s
    # each pair's larger magnitude bounds the errors of both its channels
    size = torch.zeros_like(y)
    size[..., i] = size[..., j] = (u.abs() + v.abs()) * m
    return y, size


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("tokens,heads,dim,rot", [(1, 1, 2, 2), (1, 8, 128, 128), (7, 3, 80, 32), (33, 5, 96, 96), (5, 2, 50, 26),
                                                  (257, 40, 128, 64), (3, 1, 256, 256), (2000, 70, 64, 64)])
def test_rope(dtype, layout, tokens, heads, dim, rot):
    f, m = gar.gar_rope_frequencies(rot, 10000.0, "parts" if rot > 32 else "plain", 4.0, 512.0)
    table = gar.gar_rope_table(1000, f, m)
    # a strided view: heads of a wider buffer, tokens in reverse
    x = _randn((tokens, heads + 1, dim), dtype, tokens + dim)[:, 1:]
    pos = torch.randint(0, 1000, (tokens,), generator=_gen(3), device="cuda", dtype=torch.int32 if heads % 2 else torch.int64)
    for inverse in (False, True):
        want, size = _rope64(x, pos, f, m, layout, inverse)
        got = gar.gar_rope(x, pos, table, layout, inverse)
        # table entry, product and sum: three roundings of 32 bits, then the output's
        tol = 4 * U32 * size + ROUND[dtype] * want.abs() * (1 + 2 ** -8) + TINY[dtype] + 1e-45
        tol[..., rot:] = 0
        assert bool(((got.double() - want).abs() <= tol).all())
        again = x.clone()
        held = gar.gar_rope(again, pos, table, layout, inverse, out=again)
        assert held is again and torch.equal(again, got)
        wide = torch.full((tokens, heads, dim + 8), 7.0, dtype=x.dtype, device="cuda")
        gar.gar_rope(x, pos, table, layout, inverse, out=wide[..., :dim])
        assert torch.equal(wide[..., :dim], got) and bool((wide[..., dim:] == 7).all())


@pytest.mark.gpu
def test_rope_gradient_by_differences():
    """The rotation is linear, so its gradient is a difference quotient with any step: d<g, rope(x)>/dx."""
    f, m = gar.gar_rope_frequencies(12, 100.0, "parts", 2.0, 32.0)
    table = gar.gar_rope_table(64, f, m)
    x, g = _randn((3, 2, 16), "f32", 1), _randn((3, 2, 16), "f32", 2)
    pos = torch.tensor([0, 5, 63], device="cuda")
    for layout in ("half", "interleaved"):
        grad = gar.gar_rope(g, pos, table, layout, inverse=True)
        base = gar.gar_rope(x, pos, table, layout).double()
        for i in range(0, x.numel(), 5):
            y = x.clone()
            y.view(-1)[i] += 1.0
            step = (y.view(-1)[i] - x.view(-1)[i]).double()
            d = ((gar.gar_rope(y, pos, table, layout).double() - base) * g.double()).sum() / step
            # two channels differ, each off by at most 4u(|u| + |v|)m in both evaluations
            assert abs(float(d) - float(grad.view(-1)[i])) <= 64 * U32 * float((x.abs().max() + 1) * g.abs().max()) * m


@pytest.mark.gpu
def test_rope_table_far_positions_and_bad_positions():
    f, m = gar.gar_rope_frequencies(8, 1e6)
    first = 10 ** 9
    table = gar.gar_rope_table(5, f, m, first=first)
    a = (first + torch.arange(5, dtype=torch.float64))[:, None] * torch.tensor(f, dtype=torch.float64)
    want = torch.stack([a.cos(), a.sin()], -1)
    # the angle's own rounding in 64 bits: 2^-53 * 10^9 radians; then one rounding to 32 bits
    assert float((table.cpu().double() - want).abs().max()) <= U32 + 4e-7 * 2 ** -1
    x = _randn((4, 2, 10), "bf16", 0)
    for t in (torch.int32, torch.int64):
        y = gar.gar_rope(x, torch.tensor([0, 5, -1, 4], device="cuda", dtype=t), table)
        bad = torch.tensor([False, True, True, False])
        assert torch.equal(y[..., :8].isnan().all(-1).all(-1).cpu(), bad)
        assert not bool(y[~bad.cuda()].isnan().any()) and torch.equal(y[..., 8:], x[..., 8:])
    assert gar.gar_rope(x[:0], torch.empty(0, dtype=torch.int64, device="cuda"), table).shape == (0, 2, 10)
    assert gar.gar_rope_table(0, f).shape == (0, 4, 2)


@pytest.mark.gpu
def test_python_checks():
    x = _randn((4, 2, 16), "bf16", 0)
    table = gar.gar_rope_table(8, gar.gar_rope_frequencies(16)[0])
    pos = torch.arange(4, device="cuda")
    for bad in (lambda: gar.gar_rope(x[0], pos, table), lambda: gar.gar_rope(x, pos[:3], table),
                lambda: gar.gar_rope(x, pos.float(), table), lambda: gar.gar_rope(x, pos, table[:, :, :1]),
                lambda: gar.gar_rope(x.int(), pos, table), lambda: gar.gar_rope(x, pos, table, "third"),
                lambda: gar.gar_rope(x, pos, table, out=x.float()), lambda: gar.gar_rope(x.cpu(), pos, table),
                lambda: gar.gar_rope(x.transpose(1, 2), pos, table), lambda: gar.gar_rope(x[..., :8], pos, table),
                lambda: gar.KVCache(x, x), lambda: gar.KVCache(x[None].to(torch.int8), x[None].to(torch.int8)),
                lambda: gar.KVCache(x[None], x[None], x, x), lambda: gar.KVCache(x[None], x[None].float())):
        with pytest.raises(ValueError):
            bad()
    cache = gar.KVCache(torch.zeros(2, 2, 4, 16, device="cuda"), torch.zeros(2, 2, 4, 16, device="cuda"))
    plan = gar.gar_attn_plan_create(4, 2, 16)
    k, q = _randn((4, 2, 16), "f32", 0), _randn((4, 4, 16), "f32", 0)
    pt, n = torch.zeros(4, 1, dtype=torch.int32, device="cuda"), torch.ones(4, dtype=torch.int32, device="cuda")
    for bad in (lambda: gar.gar_kv_write(cache, k, k, pos.int()), lambda: gar.gar_kv_write(cache, k, k[:, :1], pos),
                lambda: gar.gar_kv_write(cache, k, k, pos, pos), lambda: gar.gar_kv_read(cache, pos, "i8"),
                lambda: gar.gar_kv_read(cache, pos, out=(k, k[:3])), lambda: gar.gar_decode_attention(plan, k, cache, pt, n),
                lambda: gar.gar_decode_attention(plan, q, cache, pt.long(), n), lambda: gar.gar_decode_attention(plan, q, cache, pt, n.long()),
                lambda: gar.gar_decode_attention(plan, q, cache, pt[:2], n), lambda: gar.gar_decode_attention(plan, q, cache, pt, n[:2]),
                lambda: gar.gar_decode_attention(plan, q, cache, pt, n, out=q[:2]), lambda: gar.gar_decode_attention(plan, q, cache, pt, n, lse=q)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(gar.GarError):       # a float cache takes its own type
        gar.gar_kv_write(cache, k.half(), k.half(), pos)
    with pytest.raises(gar.GarError):
        gar.gar_decode_attention(plan, q.half(), cache, pt, n)


# ---------------------------------------------------------------------------- the cache

def _empty_cache(pages, heads, page_size, dim, kind, order="head", fill=0):
    """A cache whose storage is head-major or token-major; 8-bit storage filled with one byte."""
    shape = (pages, heads, page_size, dim) if order == "head" else (pages, page_size, heads, dim)
    t = [torch.full(shape, fill, device="cuda", dtype=torch.uint8).view(TORCH[kind]) if kind in QMAX
         else torch.full(shape, float(fill), device="cuda", dtype=TORCH[kind]) for _ in range(2)]
    t = [x if order == "head" else x.transpose(1, 2) for x in t]
    if kind not in QMAX:
        return gar.KVCache(*t)
    s = [torch.full(shape[:3], 5.0, device="cuda") for _ in range(2)]
    s = [x if order == "head" else x.transpose(1, 2) for x in s]
    return gar.KVCache(*t, *s)


def _quantise(x, kind):
    """(codes as 32-bit floats, scale) of rows, by 32-bit IEEE operations on the CPU."""
    x = x.cpu().float()
    scale = x.abs().amax(-1) * (torch.ones(()) / QMAX[kind])
    y = x / torch.where(scale > 0, scale, torch.ones(()))[..., None]
    y = y.clamp(-QMAX[kind], QMAX[kind])
    return (y.round() if kind == "i8" else y.to(TORCH[kind]).float()), scale


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["i8", "e4m3", "own"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("tokens,heads,dim,page_size,order", [(1, 1, 128, 16, "head"), (37, 3, 80, 5, "token"), (50, 2, 33, 1, "head"),
                                                              (129, 8, 256, 64, "token"), (9, 1, 1, 3, "head"), (300, 5, 64, 24, "head")])
def test_cache_write_and_read(kind, dtype, tokens, heads, dim, page_size, order):
    kind = dtype if kind == "own" else kind
    pages = -(-tokens // page_size) + 3
    cache = _empty_cache(pages, heads, page_size, dim, kind, order, fill=3)
    both = _randn((tokens, 2, heads, dim), dtype, tokens + dim)      # keys and values of one buffer: strided
    k, v = both[:, 0], both[:, 1]
    v[0] = 0                                                         # a row of zeros
    slots = torch.randperm(pages * page_size, generator=_gen(1), device="cuda")[:tokens]
    slots[tokens // 2] = -1 if tokens > 1 else slots[0]
    before = [t.clone() for t in (cache.k, cache.v)]
    gar.gar_kv_write(cache, k, v, slots)
    kept = (slots >= 0).cpu()
    page, row = (slots // page_size).cpu()[kept], (slots % page_size).cpu()[kept]
    for x, t, s, old in ((k, cache.k, cache.k_scale, before[0]), (v, cache.v, cache.v_scale, before[1])):
        rows = t.cpu()[page, :, row] if kind not in QMAX else t.cpu().view(torch.uint8)[page, :, row].view(TORCH[kind]).float()
        if kind in QMAX:
            code, scale = _quantise(x[kept.cuda()], kind)
            assert torch.equal(s.cpu()[page, :, row], scale)
            assert torch.equal(rows, code)
            # and within half a step of what they stand for: a code's own size for the floats
            err = (code.double() * scale.double()[..., None] - x.cpu()[kept].double()).abs()
            step = scale.double()[..., None] * (0.5 if kind == "i8" else (code.abs().double() / 16).clamp(min=2.0 ** -10))
            assert bool((err <= step * (1 + 2.0 ** -3)).all())
        else:
            assert torch.equal(rows, x.cpu()[kept])
        # nothing else was written
        touched = torch.zeros(pages, page_size, dtype=torch.bool)
        touched[page, row] = True
        same = (t.cpu().view(torch.uint8) == old.cpu().view(torch.uint8)).transpose(1, 2)
        assert bool(same[~touched].all())
    for out in ("f32", "bf16", "f16") if kind in QMAX else (kind,):
        got = gar.gar_kv_read(cache, slots, out)
        for x, y in ((k, got[0]), (v, got[1])):
            assert y.dtype == TORCH[out] and bool((y[~kept.cuda()] == 0).all())
            if kind in QMAX:
                code, scale = _quantise(x[kept.cuda()], kind)
                want = (code * scale[..., None]).to(TORCH[out])
            else:
                want = x.cpu()[kept]
            assert torch.equal(y[kept.cuda()].cpu(), want)
    gar.gar_kv_status(cache)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("kind,dtype,dim,rot", [("i8", "bf16", 128, 128), ("e4m3", "f16", 80, 48), ("f32", "f32", 33, 10),
                                                ("bf16", "bf16", 64, 32), ("i8", "f32", 256, 256), ("f16", "f16", 96, 96)])
def test_cache_write_rotates_keys(layout, kind, dtype, dim, rot):
    tokens, heads = 29, 3
    f, m = gar.gar_rope_frequencies(rot)
    table = gar.gar_rope_table(50, f, m)
    cache = _empty_cache(4, heads, 8, dim, kind)
    k, v = _randn((tokens, heads, dim), dtype, 1), _randn((tokens, heads, dim), dtype, 2)
    slots, pos = torch.arange(tokens, device="cuda"), torch.arange(tokens, device="cuda", dtype=torch.int32) + 20
    gar.gar_kv_write(cache, k, v, slots, pos, table, layout)
    # in 32 bits by gar_rope (bit for bit the same rotation), then quantised or rounded
    turned = gar.gar_rope(k.float(), pos, table, layout)
    other = _empty_cache(4, heads, 8, dim, kind)
    if kind in QMAX:
        gar.gar_kv_write(other, turned, v.float(), slots)
    else:
        gar.gar_kv_write(other, turned.to(k.dtype), v, slots)
    for a, b in ((cache.k, other.k), (cache.v, other.v)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    if kind in QMAX:
        assert torch.equal(cache.k_scale, other.k_scale) and torch.equal(cache.v_scale, other.v_scale)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["i8", "e4m3"])
def test_cache_rows_that_are_not_finite_and_tiny(kind):
    x = torch.ones(5, 1, 64, device="cuda")
    x[0, 0, 3], x[1, 0, 63], x[2, 0, 0] = float("nan"), float("inf"), -float("inf")
    x[3] *= 1e-40                          # subnormal scale
    cache = _empty_cache(1, 1, 8, 64, kind)
    slots = torch.arange(5, device="cuda")
    gar.gar_kv_write(cache, x, x, slots)
    k, v = gar.gar_kv_read(cache, slots, "f32")
    assert bool(k[:3].isnan().all()) and bool(v[:3].isnan().all()) and bool((k[4] == 1).all() or (k[4] - 1).abs().max() <= 2 ** -22)
    code, scale = _quantise(x[3:4], kind)
    assert torch.equal(k[3:4].cpu(), code * scale[..., None])


@pytest.mark.gpu
def test_cache_bad_indices_are_reported():
    cache = _empty_cache(2, 1, 4, 16, "bf16")
    x = _randn((3, 1, 16), "bf16", 0)
    slots = torch.tensor([1, 8, 1 << 40], device="cuda")
    gar.gar_kv_write(cache, x, x, slots)
    with pytest.raises(gar.GarError) as e:
        gar.gar_kv_status(cache)
    assert e.value.code == -1 and "slot" in str(e.value)
    gar.gar_kv_status(cache)               # cleared
    k, _ = gar.gar_kv_read(cache, slots)
    assert torch.equal(k[0], x[0]) and bool((k[1:] == 0).all())
    with pytest.raises(gar.GarError):
        gar.gar_kv_status(cache)
    table = gar.gar_rope_table(4, gar.gar_rope_frequencies(16)[0])
    gar.gar_kv_write(cache, x[:1], x[:1], slots[:1], torch.tensor([4], device="cuda"), table)
    with pytest.raises(gar.GarError) as e:
        gar.gar_kv_status(cache)
    assert "position" in str(e.value)
    gar.gar_kv_write(cache, x[:0], x[:0], slots[:0])
    assert gar.gar_kv_read(cache, slots[:0])[0].shape == (0, 1, 16)


# ---------------------------------------------------------------------------- attention

def _attn_case(lengths, q_heads, kv_heads, dim, page_size, kind, dtype, seed=0, order="head", spare=2, sharp=1.0):
    """A cache in scattered pages.  Float caches hold NaN and infinities, 8-bit ones NaN scales,
    wherever no sequence's row is; unused table entries are -1."""
    need = [-(-n // page_size) for n in lengths]
    pages = sum(need) + spare
    width = max(need + [1]) + 1
    g = _gen(seed)
    order_ids = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lengths), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order_ids[at:at + n]
        at += n
    cache = _empty_cache(pages, kv_heads, page_size, dim, kind, order)
    rows = []
    for b, n in enumerate(lengths):
        i = torch.arange(n, device="cuda")
        page, row = table[b, i // page_size].long(), i % page_size
        kv = []
        for w, (t, s) in enumerate(((cache.k, cache.k_scale), (cache.v, cache.v_scale))):
            if kind == "i8":
                x = torch.randint(-127, 128, (n, kv_heads, dim), generator=g, device="cuda", dtype=torch.int8)
            else:
                x = torch.randn((n, kv_heads, dim), generator=g, device="cuda")
                x = (x * 100).clamp(-448, 448).to(TORCH[kind]) if kind == "e4m3" else x.to(TORCH[kind])
            sc = torch.rand((n, kv_heads), generator=g, device="cuda") * 0.01 + 0.005 if kind in QMAX else None
            kv.append(x.double() * (sc.double()[..., None] if sc is not None else 1.0))
            rows.append((t, page, row, x, s, sc))
        rows[-1] = rows[-1] + (kv,)
    # poison, then the rows
    for t, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        if kind in QMAX:
            s.fill_(float("nan"))
            t.view(torch.uint8).fill_(0x7f)
        else:
            t.fill_(float("nan"))
            t[..., ::3] = float("inf")
    kvs = []
    for r in rows:
        t, page, row, x, s, sc = r[:6]
        (t.view(torch.uint8) if kind in QMAX else t)[page, :, row] = x.view(torch.uint8) if kind in QMAX else x
        if kind in QMAX:
            s[page, :, row] = sc
        if len(r) > 6:
            kvs.append(r[6])
    q = _randn((len(lengths), q_heads, dim), dtype, seed + 1) * sharp
    return cache, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), q, kvs


def _check_attn(out, lse, q, kvs, lengths, window, scale, out_type):
    """out and lse against 64 bits.  Bounds: a score is a sum of `dim` products in 32 bits and two
    roundings more, off by at most e = (dim + 4) u scale sum|q||k|; a weight 2^x by 2^-22; the
    weights as two 16-bit parts by 2^-16; sums over n rows by n u.  So out is off by
    (2 e + 2^-21 + 2^-16 + 2 n u) sum p|v| and its own rounding, lse by e + 2^-22 + n u + 2^-22 |lse|."""
    group = q.shape[1] // (kvs[0][0].shape[1] if kvs else 1)
    for b, n in enumerate(lengths):
        lo = max(0, n - window) if window else 0
        if n == 0:
            assert bool((out[b] == 0).all()) and bool((lse[b] == -math.inf).all())
            continue
        k, v = (x[lo:].repeat_interleave(group, 1) for x in kvs[b])
        qb = q[b].double()
        y = torch.einsum("hd,nhd->hn", qb, k) * scale
        e = ((q.shape[2] + 4) * U32 * scale * torch.einsum("hd,nhd->hn", qb.abs(), k.abs())).amax(-1)
        p = torch.softmax(y, -1)
        want = torch.einsum("hn,nhd->hd", p, v)
        size = torch.einsum("hn,nhd->hd", p, v.abs())
        rel = 2 * e[:, None] + 2.0 ** -21 + 2.0 ** -16 + 2 * n * U32
        tol = rel * size + ROUND[out_type] * want.abs() * (1 + 2 ** -7) + TINY[out_type]
        off = (out[b].double() - want).abs()
        assert bool((off <= tol).all()), (b, n, float((off / tol.clamp(min=1e-300)).max()))
        want_lse = torch.logsumexp(y, -1)
        assert bool(((lse[b].double() - want_lse).abs() <= e + 2.0 ** -22 + n * U32 + 2.0 ** -22 * want_lse.abs()).all()), (b, n)


SHORT = [0, 1, 2, 15, 16, 17, 31, 33, 64, 65, 127, 128, 130, 300]


@pytest.mark.gpu
@pytest.mark.parametrize("kind,dtype", [("bf16", "bf16"), ("f16", "f16"), ("f32", "f32"), ("i8", "bf16"), ("i8", "f16"), ("i8", "f32"),
                                        ("e4m3", "bf16"), ("e4m3", "f16"), ("e4m3", "f32")])
@pytest.mark.parametrize("q_heads,kv_heads,dim,page_size,window", [
    (8, 2, 128, 16, 0), (1, 1, 64, 1, 0), (6, 6, 80, 5, 7), (10, 2, 96, 24, 0), (16, 1, 256, 32, 0), (32, 2, 128, 64, 100),
    (9, 1, 64, 16, 1), (40, 2, 72, 7, 33), (3, 3, 33, 4, 0), (2, 1, 1, 3, 0), (24, 8, 200, 48, 0)])
def test_attention(kind, dtype, q_heads, kv_heads, dim, page_size, window):
    order = "token" if page_size % 2 else "head"
    cache, table, lens, q, kvs = _attn_case(SHORT, q_heads, kv_heads, dim, page_size, kind, dtype, order=order)
    plan = gar.gar_attn_plan_create(q_heads, kv_heads, dim)
    out, lse = gar.gar_decode_attention(plan, q, cache, table, lens, window=window, lse=True)
    assert out.dtype == q.dtype
    _check_attn(out, lse, q, kvs, SHORT, window, dim ** -0.5, dtype)
    # 32-bit outputs, strided query and output, another scale; the workspace is used again
    wide_q = torch.zeros(len(SHORT), q_heads, dim + 5, dtype=q.dtype, device="cuda")
    wide_q[..., 3:3 + dim] = q
    wide = torch.full((len(SHORT), q_heads + 1, dim), 7.0, device="cuda")
    got, lse = gar.gar_decode_attention(plan, wide_q[..., 3:3 + dim], cache, table, lens, scale=0.3, window=window, lse=True,
                                        out=wide[:, 1:])
    _check_attn(got, lse, q, kvs, SHORT, window, 0.3, "f32")
    assert bool((wide[:, 0] == 7).all())
    gar.gar_kv_status(cache)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,dtype,q_heads,kv_heads,dim,lengths", [
    ("bf16", "bf16", 8, 1, 128, [70001]), ("f16", "f16", 12, 1, 64, [30000, 5, 0, 12345]), ("i8", "bf16", 4, 4, 128, [20000, 20011]),
    ("e4m3", "f16", 16, 2, 128, [40000, 1]), ("f32", "f32", 3, 1, 80, [9999, 10001]), ("bf16", "bf16", 32, 4, 256, [5000]),
    ("bf16", "bf16", 4, 2, 64, [(37 * b) % 400 for b in range(300)])])
def test_attention_split_over_long_and_many_sequences(kind, dtype, q_heads, kv_heads, dim, lengths):
    cache, table, lens, q, kvs = _attn_case(lengths, q_heads, kv_heads, dim, 16, kind, dtype, sharp=2.0)
    plan = gar.gar_attn_plan_create(q_heads, kv_heads, dim)
    first = gar.gar_decode_attention(plan, q, cache, table, lens, lse=True)
    _check_attn(*first, q, kvs, lengths, 0, dim ** -0.5, dtype)
    for _ in range(3):                     # whatever CTA arrives last, the bits stay
        again = gar.gar_decode_attention(plan, q, cache, table, lens, lse=True)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.gpu
@pytest.mark.parametrize("kind,dtype", [("bf16", "bf16"), ("f32", "f32"), ("i8", "f16")])
def test_attention_values_past_finite(kind, dtype):
    """Scores at minus infinity weigh nothing; a row of them has no weights at all; a NaN that is
    attended reaches its head's output and no other."""
    cache, table, lens, q, kvs = _attn_case([40, 40, 40], 2, 2, 64, 16, kind, dtype)
    plan = gar.gar_attn_plan_create(2, 2, 64)
    base, base_lse = gar.gar_decode_attention(plan, q, cache, table, lens, lse=True)
    if kind != "i8":
        q[:] = 1
        base, base_lse = gar.gar_decode_attention(plan, q, cache, table, lens, lse=True)
        cache.k[table[0, 1].long(), 0, 3, 0] = -math.inf                       # one row of sequence 0, head 0
        cache.k[table[1, :3].long(), 0, :, 5] = -math.inf                      # all of sequence 1, head 0
        cache.k[table[2, 0].long(), 1, 7, 5] = float("nan")
    else:
        cache.v_scale[table[2, 0].long(), 1, 7] = float("nan")
    out, lse = gar.gar_decode_attention(plan, q, cache, table, lens, lse=True)
    nan = torch.zeros(3, 2, dtype=torch.bool, device="cuda")
    nan[2, 1] = True
    assert torch.equal(out.isnan().any(-1), nan) and torch.equal(out.isnan().all(-1), nan)
    assert torch.equal(out[2, 0], base[2, 0])
    if kind != "i8":
        assert bool((out[1, 0] == 0).all()) and float(lse[1, 0]) == -math.inf
        kept = [i for i in range(40) if i != 19]
        _check_attn(out[:1, :1], lse[:1, :1], q[:1, :1], [[x[kept][:, :1] for x in kvs[0]]], [39], 0, 0.125, dtype)


@pytest.mark.gpu
def test_attention_bad_pages_and_lengths():
    cache, table, lens, q, kvs = _attn_case([20, 20, 20], 4, 2, 64, 16, "bf16", "bf16")
    plan = gar.gar_attn_plan_create(4, 2, 64)
    base = gar.gar_decode_attention(plan, q, cache, table, lens)
    gar.gar_kv_status(cache)
    table2 = table.clone()
    table2[1, 1] = cache.pages
    got = gar.gar_decode_attention(plan, q, cache, table2, lens)
    with pytest.raises(gar.GarError) as e:
        gar.gar_kv_status(cache)
    assert "page" in str(e.value) and torch.equal(got[0], base[0]) and torch.equal(got[2], base[2])
    k, v = (x.clone() for x in kvs[1])
    k[16:], v[16:] = 0, 0
    out, lse = gar.gar_decode_attention(plan, q, cache, table2, lens, lse=True)
    _check_attn(out[1:2], lse[1:2], q[1:2], [[k, v]], [20], 0, 0.125, "bf16")
    with pytest.raises(gar.GarError):
        gar.gar_kv_status(cache)
    got = gar.gar_decode_attention(plan, q, cache, table, torch.tensor([20, -3, 20], dtype=torch.int32, device="cuda"))
    with pytest.raises(gar.GarError) as e:
        gar.gar_kv_status(cache)
    assert "length" in str(e.value) and bool((got[1] == 0).all()) and torch.equal(got[2], base[2])
    lens2 = torch.tensor([20, 2 ** 31 - 1, 20], dtype=torch.int32, device="cuda")
    got = gar.gar_decode_attention(plan, q, cache, table[:, :2].contiguous(), lens2, window=4)
    with pytest.raises(gar.GarError) as e:
        gar.gar_kv_status(cache)
    assert "length" in str(e.value)
    none = gar.gar_decode_attention(plan, q, cache, table[:, :0].contiguous(), torch.zeros_like(lens))
    assert bool((none == 0).all())
    assert gar.gar_decode_attention(plan, q[:0], cache, table[:0], lens[:0]).shape == (0, 4, 64)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "i8"])
def test_attention_offsets_past_32_bits(kind):
    """A cache of more than 2^32 elements: the rows lie in its first and last pages."""
    kv_heads, dim, page_size = 2, 128, 64
    pages = (1 << 32) // (kv_heads * dim * page_size) + 10
    t = [torch.empty((pages, kv_heads, page_size, dim), dtype=TORCH[kind], device="cuda") for _ in range(2)]
    s = [torch.empty((pages, kv_heads, page_size), device="cuda") for _ in range(2)] if kind in QMAX else []
    cache = gar.KVCache(*t, *s)
    n = 150
    k, v = _randn((n, kv_heads, dim), "bf16", 1), _randn((n, kv_heads, dim), "bf16", 2)
    table = torch.tensor([[pages - 1, 0, pages - 2]], dtype=torch.int32, device="cuda")
    at = torch.arange(n, device="cuda")
    slots = table[0].long()[at // page_size] * page_size + at % page_size
    gar.gar_kv_write(cache, k, v, slots)
    back = gar.gar_kv_read(cache, slots, "f32" if kind in QMAX else None)
    if kind not in QMAX:
        assert torch.equal(back[0], k) and torch.equal(back[1], v)
    q = _randn((1, 8, dim), "bf16", 3)
    plan = gar.gar_attn_plan_create(8, kv_heads, dim)
    out, lse = gar.gar_decode_attention(plan, q, cache, table, torch.tensor([n], dtype=torch.int32, device="cuda"), lse=True)
    # reading back rounds code * scale once more: a relative 2^-24 of each value, within the bounds' slack
    _check_attn(out, lse, q, [[x.double() for x in back]], [n], 0, dim ** -0.5, "bf16")
    gar.gar_kv_status(cache)
    del cache, t, s
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_streams_and_graphs():
    """Calls on a side stream, and a captured decoding step replayed after tokens, slots and lengths changed."""
    f, _ = gar.gar_rope_frequencies(64)
    table = gar.gar_rope_table(100, f)
    cache = _empty_cache(8, 2, 16, 64, "i8")
    plan = gar.gar_attn_plan_create(4, 2, 64)
    k, v, q = (_randn((1, h, 64), "bf16", h) for h in (2, 2, 4))
    slots = torch.zeros(1, dtype=torch.int64, device="cuda")
    pages = torch.arange(8, dtype=torch.int32, device="cuda")[None]
    lens = torch.ones(1, dtype=torch.int32, device="cuda")

    def step():
        qr = gar.gar_rope(q, slots, table)
        gar.gar_kv_write(cache, k, v, slots, slots, table)
        return gar.gar_decode_attention(plan, qr, cache, pages, lens)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    graph = torch.cuda.CUDAGraph()
    side.synchronize()
    with torch.cuda.graph(graph):
        held = step()
    got, want = [], []
    keys = []
    for i in range(40):
        for t, s in ((k, 1), (v, 2), (q, 3)):
            t.copy_(_randn(t.shape, "bf16", 100 * i + s))
        slots.fill_(i)
        lens.fill_(i + 1)
        graph.replay()
        got.append(held.clone())
        keys.append((k.clone(), v.clone(), q.clone()))
    for t in (cache.k, cache.v):
        t.zero_()
    main = torch.cuda.current_stream()
    for i in range(40):
        for t, x in zip((k, v, q), keys[i]):
            t.copy_(x)
        slots.fill_(i)
        lens.fill_(i + 1)
        side.wait_stream(main)
        qr = gar.gar_rope(q, slots, table, stream=side)
        gar.gar_kv_write(cache, k, v, slots, slots, table, stream=side.cuda_stream)
        want.append(gar.gar_decode_attention(plan, qr, cache, pages, lens, stream=side.cuda_stream))
        main.wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


# ---------------------------------------------------------------------------- the kernels' other paths

@pytest.mark.gpu
@pytest.mark.parametrize("kind,dtype", [("bf16", "bf16"), ("i8", "bf16"), ("f32", "f32")])
def test_attention_of_thousands_of_short_sequences(kind, dtype):
    """More segments to a CTA than it notes at a time, many of them empty."""
    lengths = [(i * 7) % 90 if i % 3 else (i % 5 == 0) * 150 for i in range(2500)]
    cache, table, lens, q, kvs = _attn_case(lengths, 8, 4, 64, 16, kind, dtype)
    plan = gar.gar_attn_plan_create(8, 4, 64)
    out, lse = gar.gar_decode_attention(plan, q, cache, table, lens, lse=True)
    some = [i for i in range(len(lengths)) if i % 37 == 0 or lengths[i] == 150]
    _check_attn(out[some], lse[some], q[some], [kvs[i] for i in some], [lengths[i] for i in some], 0, 0.125, dtype)
    empty = lens == 0
    assert bool((out[empty] == 0).all()) and bool((lse[empty] == -math.inf).all()) and bool(lse[~empty].isfinite().all())
    assert torch.equal(out, gar.gar_decode_attention(plan, q, cache, table, lens))


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [1, 31, 32, 33, 200])
@pytest.mark.parametrize("window", [0, 300])
def test_attention_both_ways_of_sharing(batch, window):
    """Batches on both sides of where the rows are shared out another way."""
    lengths = [1 + (b * 1013) % 1777 for b in range(batch)]
    cache, table, lens, q, kvs = _attn_case(lengths, 6, 3, 128, 8, "bf16", "bf16")
    plan = gar.gar_attn_plan_create(6, 3, 128)
    out, lse = gar.gar_decode_attention(plan, q, cache, table, lens, window=window, lse=True)
    _check_attn(out, lse, q, kvs, lengths, window, 128 ** -0.5, "bf16")


@pytest.mark.gpu
@pytest.mark.parametrize("kind,dtype", [("bf16", "bf16"), ("f16", "f16"), ("f32", "f32"), ("i8", "f32"), ("e4m3", "bf16")])
@pytest.mark.parametrize("dim,q_heads", [(48, 2), (72, 5), (96, 12), (112, 3), (144, 4), (176, 11), (192, 1), (208, 9)])
def test_attention_head_sizes(kind, dtype, dim, q_heads):
    """On both sides of the sizes that the tiles are made for, groups of one row of heads and of two."""
    lengths = [300, 0, 33, 1, 5000]
    cache, table, lens, q, kvs = _attn_case(lengths, q_heads, 1, dim, 16, kind, dtype)
    plan = gar.gar_attn_plan_create(q_heads, 1, dim)
    out, lse = gar.gar_decode_attention(plan, q, cache, table, lens, lse=True)
    _check_attn(out, lse, q, kvs, lengths, 0, dim ** -0.5, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,dtype,dim", [("bf16", "bf16", 64), ("e4m3", "f16", 128), ("f32", "f32", 48), ("f16", "f16", 33)])
def test_attention_of_few_heads_over_ragged_sequences(kind, dtype, dim):
    """Shares of the rows that are smaller than what an item counts beside them, so that some hold no row of theirs."""
    lengths = [0 if b % 4 == 3 else 3000 if b % 4 == 2 else 1 + b * 61 for b in range(40)]
    cache, table, lens, q, kvs = _attn_case(lengths, 4, 1, dim, 16, kind, dtype)
    plan = gar.gar_attn_plan_create(4, 1, dim)
    out, lse = gar.gar_decode_attention(plan, q, cache, table, lens, lse=True)
    _check_attn(out, lse, q, kvs, lengths, 0, dim ** -0.5, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,dtype", [("i8", "f16"), ("e4m3", "bf16"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "f32")])
def test_attention_strides_and_alignments(kind, dtype):
    """Caches cut out of larger tensors, scales with strides of their own, queries that are not aligned."""
    lengths, heads, dim, page = [70, 33, 1], 2, 64, 16
    base, table, lens, q, kvs = _attn_case(lengths, 6, heads, dim, page, kind, dtype)
    plan = gar.gar_attn_plan_create(6, heads, dim)
    want = gar.gar_decode_attention(plan, q, base, table, lens)
    n = base.k.shape[0]

    def copy_into(width, offset):
        wide = [torch.zeros((n, heads, page, width), dtype=torch.float32, device="cuda").to(base.k.dtype) for _ in range(2)]
        cut = [t[..., offset:offset + dim] for t in wide]
        for c, x in zip(cut, (base.k, base.v)):
            (c.view(torch.uint8) if kind in QMAX else c).copy_(x.view(torch.uint8) if kind in QMAX else x)
        return cut

    step = 16 // base.k.element_size()
    for width, offset in ((dim + step, 0), (dim + step, step), (dim + 1, 1), (dim + 3, 0)):
        scales = [] if kind not in QMAX else [base.k_scale, base.v_scale]
        got = gar.gar_decode_attention(plan, q, gar.KVCache(*copy_into(width, offset), *scales), table, lens)
        close = 2 * ROUND[dtype] * want.float().abs() + 2.0 ** -14 * want.float().abs().max()
        assert bool(((got.float() - want.float()).abs() <= close).all())
    if kind in QMAX:
        for make in (lambda s: torch.stack([s, s], -1)[..., 0], lambda s: s.transpose(1, 2).contiguous().transpose(1, 2),
                     lambda s: torch.nn.functional.pad(s, (1, 2))[..., 1:-2]):
            got = gar.gar_decode_attention(plan, q, gar.KVCache(base.k, base.v, make(base.k_scale), make(base.v_scale)), table, lens)
            assert torch.equal(got, want)
    shifted = torch.zeros(len(lengths) * 6 * dim + 1, dtype=q.dtype, device="cuda")[1:].view(len(lengths), 6, dim)
    shifted.copy_(q)
    got = gar.gar_decode_attention(plan, shifted, base, table, lens)
    assert bool(((got.float() - want.float()).abs() <= 2 * ROUND[dtype] * want.float().abs() + 2.0 ** -14 * want.float().abs().max()).all())
    into = torch.zeros(len(lengths), 6, dim + 1, dtype=q.dtype, device="cuda")
    gar.gar_decode_attention(plan, q, base, table, lens, out=into[..., 1:])
    assert torch.equal(into[..., 1:], want) and bool((into[..., 0] == 0).all())


@pytest.mark.gpu
def test_attention_holds_its_sums_in_32_bits():
    """All-positive values over 200000 rows: a sum that is cut off at each step would be off by 1e-4."""
    n, dim = 200000, 128
    for dtype in ("bf16", "f32"):
        k = torch.zeros(n // 64, 1, 64, dim, device="cuda", dtype=TORCH[dtype])
        v = (_randn((n // 64, 1, 64, dim), dtype, 1).float().abs() + 1).to(TORCH[dtype])
        table = torch.arange(n // 64, dtype=torch.int32, device="cuda")[None].repeat(152, 1)   # one CTA for each sequence
        lens = torch.full((152,), n, dtype=torch.int32, device="cuda")
        plan = gar.gar_attn_plan_create(1, 1, dim)
        out = torch.empty(152, 1, dim, device="cuda")
        gar.gar_decode_attention(plan, _randn((152, 1, dim), dtype, 2), gar.KVCache(k, v), table, lens, out=out)
        want = v.double().mean((0, 1, 2))
        # weights are all 1; 12 warps' sums of n / 12 rows, 16 at a time, then their join: random roundings of
        # u each, at most n / 192 of them in a row
        assert float(((out[:, 0].double() - want) / want).abs().max()) <= 2 * (n / 192) ** 0.5 * U32 + 2.0 ** -21


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["i8", "e4m3"])
def test_attention_rows_of_very_different_scales(kind):
    """Values a million times smaller than others of the sequence, with nearly all of the weight."""
    cache, table, lens, q, kvs = _attn_case([100], 2, 1, 64, 16, kind, "f32")
    row = 37
    page, at = table[0, row // 16].long(), row % 16
    cache.k.view(torch.uint8)[page, 0, at] = torch.tensor([100] * 64, dtype=torch.int8, device="cuda").to(cache.k.dtype).view(torch.uint8)
    cache.k_scale[page, 0, at], cache.v_scale[page, 0, at] = 0.1, 1e-8
    q[:] = 0.5
    k, v = gar.gar_kv_read(cache, page * 16 + torch.arange(16, device="cuda"), "f32")
    kvs = [[x.clone() for x in kvs[0]]]
    kvs[0][0][row], kvs[0][1][row] = k[at].double(), v[at].double()
    plan = gar.gar_attn_plan_create(2, 1, 64)
    out, lse = gar.gar_decode_attention(plan, q, cache, table, lens, lse=True)
    y = torch.einsum("hd,nhd->hn", q[0].double(), kvs[0][0].repeat_interleave(2, 1)) / 8
    want = torch.einsum("hn,nhd->hd", torch.softmax(y, -1), kvs[0][1].repeat_interleave(2, 1))
    assert float(torch.softmax(y, -1)[:, row].min()) > 1 - 1e-9
    # the weight is 2^14 * 1e-6 in f16, in two parts: off by 2^-25 of f16's unit, 2^-11 of it in the worst case
    assert float((out[0].double() - want).norm() / want.norm()) <= 2.0 ** -10
