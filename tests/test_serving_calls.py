"""The serving operators' calls: streams, graphs, memory, devices, refusals, and a run of them together."""

import math
import os
import re
import threading

import pytest
import torch

from paper_2004_09362_gb300 import gar
from test_decode_binding import _fake, _fake_cache
from test_decode_operators import _attn_case, _gen, _randn
from test_serving_operators import _check_evict, _check_prefix, _check_weigh, _prefix_case, _verify_case, _verify_reference

CSRC = os.path.join(os.path.dirname(gar.__file__), "csrc")
I64, I32, F32 = torch.int64, torch.int32, torch.float32


@pytest.mark.parametrize("name", ["prefix.cu", "prefix.cuh", "prefix_mma.cu", "tcgen05.cuh", "cluster.cuh", "weigh.cu", "evict.cu", "verify.cu"])
def test_no_loads_that_take_memory_for_constant(name):
    """The kernels may be resident while the one that writes their inputs runs."""
    with open(os.path.join(CSRC, name)) as f:
        assert not re.search(r"__ldg\b|ld\.global(\.\w+)*\.nc|__restrict__", f.read())


# ---------------------------------------------------------------------------- refusals (no GPU)

def _calls(devices, grad=None):
    """(name, number of tensors, call): the call with tensor i on GPU devices[i]; a gradient asked of tensor `grad`."""
    d = list(devices) + [0] * 8

    def t(i, shape, dtype=torch.bfloat16):
        x = _fake(shape, dtype, d[i])
        return x.requires_grad_() if i == grad else x

    def prefix():
        gar.gar_prefix_attention(gar.gar_attn_plan_create(4, 2, 64), t(0, (6, 4, 64)), _fake_cache(d[1]), t(2, (2, 3), I32), t(3, (2,), I32),
                                 t(4, (6, 2), I32), t(5, (6,), I32), out=t(6, (6, 4, 64)), lse=t(7, (6, 4), F32))

    def weigh():
        gar.gar_kv_weigh(t(0, (3, 4, 64)), _fake_cache(d[1]), t(2, (3, 2), I32), t(3, (3,), I32), t(4, (3, 4), F32), t(5, (3, 2, 32), F32),
                         out=t(6, (3, 2, 32), F32))

    def evict():
        gar.gar_kv_evict(_fake_cache(d[1]), t(0, (3, 2, 32), F32), t(2, (3, 2, 32), I32), t(3, (3, 2), I32), t(4, (3,), I32), 8,
                         out=(t(5, (3, 2, 32), F32), t(6, (3, 2, 32), I32), t(7, (3,), I32)))

    def verify():
        gar.gar_verify_drafts(t(0, (3, 5, 100), F32), t(1, (3, 4, 100), F32), t(2, (3, 4), I64), t(3, (3, 5), F32),
                              out=(t(4, (3, 5), I64), t(5, (3,), I32)))
    return {"prefix": (8, prefix, (0, 6, 7)), "weigh": (7, weigh, (0, 4, 5, 6)), "evict": (8, evict, (0, 5)), "verify": (6, verify, (0, 1, 3))}


@pytest.mark.parametrize("name", ["prefix", "weigh", "evict", "verify"])
def test_tensors_of_two_gpus_are_refused(name):
    for i in range(_calls([])[name][0]):
        with pytest.raises(ValueError, match="on GPU 1, |on GPU 0, "):
            _calls([int(j == i) for j in range(8)])[name][1]()


@pytest.mark.parametrize("name", ["prefix", "weigh", "evict", "verify"])
def test_tensors_that_ask_for_a_gradient_are_refused(name):
    for i in _calls([])[name][2]:
        with pytest.raises(ValueError, match="gradient"):
            _calls([], grad=i)[name][1]()


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["prefix", "weigh", "evict", "verify"])
def test_tensors_of_a_gpu_that_is_not_current_are_refused(name):
    torch.zeros(1, device="cuda")
    with pytest.raises(ValueError, match="the current device is GPU 0"):
        _calls([1] * 8)[name][1]()


def test_shapes_and_types_are_checked():
    plan, cache = gar.gar_attn_plan_create(4, 2, 64), _fake_cache(0)
    q, lens, table = _fake((6, 4, 64)), _fake(6, I32), _fake((6, 2), I32)
    pt, pn = _fake((2, 3), I32), _fake(2, I32)
    w, lse, p = _fake((6, 2, 32), F32), _fake((6, 4), F32), _fake((6, 2, 32), I32)
    target, draft, tokens, u = _fake((3, 5, 100), F32), _fake((3, 4, 100), F32), _fake((3, 4), I64), _fake((3, 5), F32)
    for call in (
            lambda: gar.gar_prefix_attention(plan, _fake((6, 3, 64)), cache, pt, pn, table, lens),
            lambda: gar.gar_prefix_attention(plan, _fake((6, 4, 60)), cache, pt, pn, table, lens),
            lambda: gar.gar_prefix_attention(plan, q, cache, _fake((4, 3), I32), _fake(4, I32), table, lens),     # 6 is no multiple of 4
            lambda: gar.gar_prefix_attention(plan, q, cache, _fake((0, 3), I32), _fake(0, I32), table, lens),
            lambda: gar.gar_prefix_attention(plan, q, cache, pt, _fake(3, I32), table, lens),
            lambda: gar.gar_prefix_attention(plan, q, cache, _fake((2, 3), I64), pn, table, lens),
            lambda: gar.gar_prefix_attention(plan, q, cache, pt, pn, _fake((5, 2), I32), lens),
            lambda: gar.gar_prefix_attention(plan, q, cache, pt, pn, table, _fake(6, I64)),
            lambda: gar.gar_prefix_attention(plan, q, cache, pt, pn, table, lens, out=_fake((1, 4, 64)).expand(6, 4, 64)),
            lambda: gar.gar_prefix_attention(plan, q, cache, pt, pn, table, lens, lse=_fake((6, 3), F32)),
            lambda: gar.gar_kv_weigh(_fake((6, 4, 60)), cache, table, lens, lse, w),
            lambda: gar.gar_kv_weigh(q, cache, table, lens, _fake((6, 3), F32), w),
            lambda: gar.gar_kv_weigh(q, cache, table, lens, lse, _fake((6, 3, 32), F32)),
            lambda: gar.gar_kv_weigh(q, cache, table, lens, lse, _fake((6, 2, 32))),
            lambda: gar.gar_kv_weigh(q, cache, table, lens, lse, w, out=_fake((6, 2, 31), F32)),
            lambda: gar.gar_kv_weigh(q, cache, table, lens, lse, w, out=_fake((1, 2, 32), F32).expand(6, 2, 32)),
            lambda: gar.gar_kv_evict(cache, _fake((6, 3, 32), F32), p, table, lens, 4),
            lambda: gar.gar_kv_evict(cache, w.transpose(0, 1), p, table, lens, 4),
            lambda: gar.gar_kv_evict(cache, w, _fake((6, 2, 32), I64), table, lens, 4),
            lambda: gar.gar_kv_evict(cache, w, p, table, lens, 1 << 32), lambda: gar.gar_kv_evict(cache, w, p, table, lens, 4, first=1 << 40),
            lambda: gar.gar_kv_evict(cache, w, p, table, lens, 4, out=(w, p)),
            lambda: gar.gar_verify_drafts(target, _fake((3, 5, 100), F32), tokens, u),
            lambda: gar.gar_verify_drafts(target, _fake((3, 4, 100)), tokens, u),
            lambda: gar.gar_verify_drafts(target, draft, _fake((3, 4), F32), u), lambda: gar.gar_verify_drafts(target, draft, _fake((3, 5), I64), u),
            lambda: gar.gar_verify_drafts(target, draft, tokens, _fake((3, 4), F32)),
            lambda: gar.gar_verify_drafts(target.transpose(1, 2), draft, tokens, u),
            lambda: gar.gar_verify_drafts(target, draft, tokens, u, out=(tokens, u))):
        with pytest.raises((ValueError, gar.GarError)):
            call()
    for call in (lambda: gar.gar_prefix_attention(cache, q, cache, pt, pn, table, lens), lambda: gar.gar_prefix_attention(plan, q, plan, pt, pn, table, lens),
                 lambda: gar.gar_kv_weigh(q, plan, table, lens, lse, w), lambda: gar.gar_kv_evict(plan, w, p, table, lens, 4),
                 lambda: gar.gar_kv_evict(cache, w, p, table, lens), lambda: gar.gar_verify_drafts(target, draft, tokens, None)):
        with pytest.raises(TypeError):
            call()


# ---------------------------------------------------------------------------- streams, graphs, threads

@pytest.mark.gpu
@pytest.mark.parametrize("share,wide", [(3, False), (3, True), (40, True)])
def test_streams_and_graphs(share, wide):
    """All of them, captured and replayed after their inputs changed, and on a side stream, give what eager calls give."""
    own = [b % 17 + 1 for b in range(share)]
    cache, pt, pn, t, n, q, _ = _prefix_case([400], own, share, 8, 2, 64, 16, "bf16", "bf16", wide=wide)
    plan = gar.gar_attn_plan_create(8, 2, 64)
    rows = t.shape[1] * 16
    weights = torch.rand((share, 2, rows), generator=_gen(3), device="cuda")
    pos = torch.arange(rows, dtype=torch.int32, device="cuda").expand(share, 2, rows).contiguous()
    target, draft, tokens, uniform = _verify_case(share, 3, 501, "f32")
    kept = [x.clone() for x in cache.tensors]

    def step(stream=None):
        out, lse = gar.gar_prefix_attention(plan, q, cache, pt, pn, t, n, lse=True, stream=stream)
        w = gar.gar_kv_weigh(q, cache, t, n, lse, weights, stream=stream)
        left = gar.gar_kv_evict(cache, w, pos, t, n, 5, first=1, recent=2, stream=stream)
        after = gar.gar_prefix_attention(plan, q, cache, pt, pn, t, left[2], stream=stream)
        return (out, lse, w, *left, after, *gar.gar_verify_drafts(target, draft, tokens, uniform, stream=stream))

    def change(i):
        for x, y in zip(cache.tensors, kept):
            x.copy_(y)
        q.copy_(_randn(q.shape, "bf16", 50 + i))
        uniform.copy_(torch.rand(uniform.shape, generator=_gen(70 + i), device="cuda"))
        weights.copy_(torch.rand(weights.shape, generator=_gen(90 + i), device="cuda"))

    want = []
    for i in range(8):
        change(i)
        want.append(step())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    with torch.cuda.graph(other):              # a second graph of the same plan, replayed in turn
        held2 = step()
    for i in range(8):
        change(i)
        (graph if i % 2 else other).replay()
        for a, b in zip(held if i % 2 else held2, want[i]):
            assert torch.equal(a, b)
        change(i)
        side.wait_stream(torch.cuda.current_stream())
        got = step(side if i % 2 else side.cuda_stream)
        torch.cuda.current_stream().wait_stream(side)
        for a, b in zip(got, want[i]):
            assert torch.equal(a, b)
    gar.gar_kv_status(cache)


@pytest.mark.gpu
def test_two_threads_with_a_stream_and_a_plan_each():
    cache, pt, pn, t, n, q, _ = _prefix_case([3000], [b % 30 for b in range(48)], 48, 8, 2, 128, 16, "bf16", "bf16")
    want = gar.gar_prefix_attention(gar.gar_attn_plan_create(8, 2, 128), q, cache, pt, pn, t, n)
    target, draft, tokens, uniform = _verify_case(20, 3, 5001, "f32")
    want_tokens = gar.gar_verify_drafts(target, draft, tokens, uniform)[0]
    torch.cuda.synchronize()
    bad = []

    def work():
        stream, plan = torch.cuda.Stream(), gar.gar_attn_plan_create(8, 2, 128)
        with torch.cuda.stream(stream):
            for _ in range(30):
                a = gar.gar_prefix_attention(plan, q, cache, pt, pn, t, n)
                b = gar.gar_verify_drafts(target, draft, tokens, uniform)[0]
                if not (torch.equal(a, want) and torch.equal(b, want_tokens)):
                    bad.append(1)
        stream.synchronize()

    threads = [threading.Thread(target=work) for _ in range(2)]
    for x in threads:
        x.start()
    for x in threads:
        x.join()
    assert not bad


@pytest.mark.gpu
@pytest.mark.parametrize("page_size,share,tile", [(16, 40, 0), (64, 40, 1), (24, 40, 0), (16, 5, 0), (16, 24, 3)])
def test_waits_that_run_out(page_size, share, tile):
    """With copies and products on their way: the call ends, says so, and the next one is right."""
    cache, pt, pn, t, n, q, _ = _prefix_case([30000], [3] * share, share, 32, 4, 128, page_size, "bf16", "bf16")
    plan = gar.gar_attn_plan_create(32, 4, 128)
    want = gar.gar_prefix_attention(plan, q, cache, pt, pn, t, n, lse=True)
    gar.gar_kv_status(cache)
    for _ in range(2):
        gar.gar_attn_plan_debug_wait(plan, tile)
        gar.gar_prefix_attention(plan, q, cache, pt, pn, t, n)
        with pytest.raises(gar.GarError) as e:
            gar.gar_kv_status(cache)
        assert e.value.code == -8
        gar.gar_attn_plan_debug_wait(plan)
        got = gar.gar_prefix_attention(plan, q, cache, pt, pn, t, n, lse=True)
        gar.gar_kv_status(cache)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.gpu
def test_memory_that_calls_write_counts_as_changed():
    cache, table, lens, q, _ = _attn_case([40, 20], 4, 2, 64, 16, "bf16", "bf16")
    w = torch.zeros((2, 2, 64), device="cuda")
    pos = torch.arange(64, dtype=I32, device="cuda").expand(2, 2, 64).contiguous()
    lse = torch.zeros((2, 4), device="cuda")
    before = [x._version for x in (w, cache.k, cache.v)]
    gar.gar_kv_weigh(q, cache, table, lens, lse, w, out=w)
    gar.gar_kv_evict(cache, w, pos, table, lens, 10)
    assert all(x._version > v for x, v in zip((w, cache.k, cache.v), before))
    for off in (torch.no_grad(), torch.inference_mode()):
        with off:
            gar.gar_kv_weigh(q.clone().requires_grad_(), cache, table, lens, lse, w.clone())


# ---------------------------------------------------------------------------- sizes past 32 bits

@pytest.mark.gpu
def test_offsets_past_32_bits():
    """A cache of more than 2^32 elements whose rows lie in its first and last pages."""
    heads, dim, ps = 2, 128, 64
    pages = (1 << 32) // (heads * dim * ps) + 10
    k, v = (torch.empty((pages, heads, ps, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache = gar.KVCache(k, v)
    n = 300
    x = [_randn((n, heads, dim), "bf16", i) for i in (1, 2)]
    table = torch.tensor([[pages - 1, 0, pages - 2, 5, pages - 3, -1]], dtype=I32, device="cuda")
    at = torch.arange(n, device="cuda")
    slots = table[0].long()[at // ps] * ps + at % ps
    gar.gar_kv_write(cache, *x, slots)
    lens = torch.tensor([n], dtype=I32, device="cuda")
    zero, none = torch.zeros(40, dtype=I32, device="cuda"), torch.zeros((40, 0), dtype=I32, device="cuda")
    plan = gar.gar_attn_plan_create(8, heads, dim)
    q = _randn((40, 8, dim), "bf16", 3)
    kv = tuple(y.double() for y in x)
    for width in (6, 1 << 16):
        pt = torch.cat([table, torch.full((1, width - 6), -1, dtype=I32, device="cuda")], 1)
        out, lse = gar.gar_prefix_attention(plan, q, cache, pt, lens, none, zero, lse=True)
        _check_prefix(out, lse, q, [kv] * 40, dim ** -0.5, "bf16")
    w = torch.rand((1, heads, 6 * ps), generator=_gen(1), device="cuda")
    got = gar.gar_kv_weigh(q[:1], cache, table, lens, lse[:1], w)
    _check_weigh(got, w, q[:1], [kv], [n], lse[:1], 0, dim ** -0.5)
    pos = torch.arange(6 * ps, dtype=I32, device="cuda").expand(1, heads, 6 * ps).contiguous()
    ids = table[0, :5].long()
    small = gar.KVCache(k[ids].clone(), v[ids].clone())
    got = gar.gar_kv_evict(cache, w, pos, table, lens, 70, 3, 10)
    want = _check_evict(small, torch.arange(6, dtype=I32, device="cuda")[None], lens, w, pos, 70, 3, 10)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(k[ids], small.k) and torch.equal(v[ids], small.v)
    gar.gar_kv_status(cache)
    del cache, small, k, v
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_a_vocabulary_past_32_bits_of_offsets():
    vocab, batch = 700_000_001, 4
    target = torch.zeros((batch, 1, vocab), dtype=torch.bfloat16, device="cuda")
    want = [0, 123_456_789, vocab - 1, 699_999_999]
    for b, t in enumerate(want):
        target[b, 0, t] = 0.5
        target[b, 0, (t + vocab // 2) % vocab] = 2.0 ** -30
    u = torch.full((batch, 1), 0.25, device="cuda")
    got, _ = gar.gar_verify_drafts(target, target[:, :0], torch.zeros((batch, 0), dtype=I64, device="cuda"), u)
    assert got[:, 0].tolist() == want
    del target
    torch.cuda.empty_cache()


# ---------------------------------------------------------------------------- together

@pytest.mark.gpu
@pytest.mark.parametrize("kind,dtype", [("bf16", "bf16"), ("i8", "f16"), ("f32", "f32")])
def test_serving_a_batch(kind, dtype):
    """Twelve steps of a batch behind one prompt: tokens written, attention over prompt and own rows, the weights gathered, and the
    caches cut back to their size; every step against 64 bits, on what the cache then holds."""
    batch, q_heads, heads, dim, ps, keep, prompt = 5, 6, 2, 64, 8, 24, 100
    cache, table, lens, _, kvs = _attn_case([prompt] + [20 + b for b in range(batch)], q_heads, heads, dim, ps, kind, dtype, spare=20)
    pt, pn, n = table[:1], lens[:1], lens[1:].clone()
    used = set(table.flatten().tolist())
    free = [p for p in range(cache.pages) if p not in used]
    width = -(-(keep + 4) // ps)
    own = torch.full((batch, width), -1, dtype=I32, device="cuda")
    for b in range(batch):
        for p in range(width):
            own[b, p] = table[1 + b, p] if p < table.shape[1] and int(table[1 + b, p]) >= 0 else free.pop()
    rows = width * ps
    weights = torch.zeros((batch, heads, rows), device="cuda")
    pos = torch.full((batch, heads, rows), -1, dtype=I32, device="cuda")
    for b in range(batch):
        pos[b, :, :int(n[b])] = torch.arange(int(n[b]), dtype=I32, device="cuda")
    plan = gar.gar_attn_plan_create(q_heads, heads, dim)
    told = n.clone()
    for i in range(12):
        k, v = (_randn((batch, heads, dim), dtype, 10 * i + s) for s in (1, 2))
        q = _randn((batch, q_heads, dim), dtype, 10 * i + 3)
        at = n.long()
        slots = own.gather(1, (at // ps)[:, None]).squeeze(1).long() * ps + at % ps
        gar.gar_kv_write(cache, k, v, slots)
        for b in range(batch):
            pos[b, :, int(at[b])] = told[b]
        n, told = n + 1, told + 1
        held = []
        for b in range(batch):
            j = torch.arange(int(n[b]), device="cuda")
            x = gar.gar_kv_read(cache, own[b].long()[j // ps] * ps + j % ps, "f32")if kind == "i8" else \
                gar.gar_kv_read(cache, own[b].long()[j // ps] * ps + j % ps)
            held.append(tuple(y.double() for y in x))
        out, lse = gar.gar_prefix_attention(plan, q, cache, pt, pn, own, n, lse=True)
        both = [tuple(torch.cat([kvs[0][w], held[b][w]]) for w in (0, 1)) for b in range(batch)]
        _check_prefix(out, lse, q, both, dim ** -0.5, dtype)
        before = weights
        weights = gar.gar_kv_weigh(q, cache, own, n, lse, weights)
        _check_weigh(weights, before, q, held, n.tolist(), lse, 0, dim ** -0.5)
        weights, pos, n = _check_evict(cache, own, n, weights, pos, keep, 2, 4)
        assert bool((n <= keep).all())
    # the newest tokens are there, and the first two rows never moved
    for b in range(batch):
        for h in range(heads):
            there = set(pos[b, h, :int(n[b])].tolist())
            assert {0, 1} <= there and set(range(int(told[b]) - 4, int(told[b]))) <= there and len(there) == int(n[b])
    gar.gar_kv_status(cache)


@pytest.mark.gpu
def test_drafts_are_verified_against_the_models_probabilities():
    """Attention of a context's drafts in one call, a projection to tokens, the verification: what stands is what step-by-step decoding
    would accept with the same numbers."""
    q_heads, heads, dim, ps, vocab, drafts = 8, 2, 64, 16, 300, 4
    cache, table, lens, _, kvs = _attn_case([500, drafts + 1], q_heads, heads, dim, ps, "bf16", "bf16")
    plan = gar.gar_attn_plan_create(q_heads, heads, dim)
    q = _randn((drafts + 1, q_heads, dim), "bf16", 5)
    n = torch.arange(1, drafts + 2, dtype=I32, device="cuda")
    out = gar.gar_prefix_attention(plan, q, cache, table[:1], lens[:1], table[1:].expand(drafts + 1, -1), n)
    head = torch.randn((q_heads * dim, vocab), generator=_gen(8), device="cuda") * 0.3
    target = torch.softmax(out.float().flatten(1) @ head, -1)[None]
    draft = torch.softmax(out.float().flatten(1)[:drafts] @ head + torch.randn((drafts, vocab), generator=_gen(9), device="cuda"), -1)[None]
    tokens = torch.multinomial(draft[0], 1, generator=_gen(10)).view(1, drafts)
    for i in range(20):
        u = torch.rand((1, drafts + 1), generator=_gen(100 + i), device="cuda")
        got, accepted = gar.gar_verify_drafts(target, draft, tokens, u)
        want, want_accepted = _verify_reference(target, draft, tokens, u)
        assert torch.equal(got.cpu(), want) and torch.equal(accepted.cpu(), want_accepted)
    one = []
    for b in range(drafts + 1):                # one by one, over a single table
        whole = torch.cat([kvs[0][0], kvs[1][0][:b + 1]]), torch.cat([kvs[0][1], kvs[1][1][:b + 1]])
        one.append(whole)
    lse = gar.gar_prefix_attention(plan, q, cache, table[:1], lens[:1], table[1:].expand(drafts + 1, -1), n, lse=True)[1]
    _check_prefix(out, lse, q, one, dim ** -0.5, "bf16")
    assert math.isfinite(float(lse.sum()))
