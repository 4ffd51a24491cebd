"""The decoding operators' Python calls: memory, streams, devices, types and gradients."""

import ctypes
import gc
import os
import re
import subprocess
import threading
import time
import types
from unittest import mock

import pytest
import torch
from torch._subclasses import fake_tensor
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2004_09362_gb300 import gar


class _Recorded:
    """Stands for a workspace tensor."""

    def __init__(self):
        self.streams = []

    def data_ptr(self):
        return 4096

    def record_stream(self, stream):
        self.streams.append(stream)


def test_workspace_is_kept_for_every_stream_that_uses_it(monkeypatch):
    """A plan's workspace is allocated under the first call's stream, and later calls' streams are recorded."""
    under, attached = [], []
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda raw, device=None: raw)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda *a: None)
    made = _Recorded()
    monkeypatch.setattr(gar, "_empty", lambda shape, dtype, device, stream: under.append(stream) or made)
    monkeypatch.setattr(gar, "gar_attn_plan_set_workspace", lambda plan, ptr, n: attached.append((ptr, n)))
    plan = gar.gar_attn_plan_create(4, 2, 64)
    like = types.SimpleNamespace(device=torch.device("cpu"))
    gar._use_workspace(plan, like, 7000)
    assert under == [7000] and attached == [(4096, gar.gar_attn_plan_bytes(plan))] and plan.stream == 7000
    gar._use_workspace(plan, like, 8000)
    assert made.streams == [8000] and plan.stream == 8000 and len(under) == 1
    gar._use_workspace(plan, like, 7000)
    assert made.streams == [8000, 7000] and len(under) == 1


def _problem(batch=3, q_heads=8, kv_heads=2, dim=64, length=2000, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    pages = -(-length // 16) * batch
    k, v = (torch.randn(pages, kv_heads, 16, dim, generator=g, device="cuda").bfloat16() for _ in range(2))
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(batch, -1)
    q = torch.randn(batch, q_heads, dim, generator=g, device="cuda").bfloat16()
    return gar.KVCache(k, v), table, torch.full((batch,), length, dtype=torch.int32, device="cuda"), q


@pytest.mark.gpu
@pytest.mark.parametrize("first_on_side", [True, False])
def test_plan_dropped_while_its_call_is_pending(first_on_side):
    """The call waits on a side stream; its plan is dropped, and memory of the workspace's size is taken and written on the main one."""
    cache, table, lens, q = _problem()
    plan = gar.gar_attn_plan_create(8, 2, 64)
    want = gar.gar_decode_attention(plan, q, cache, table, lens)
    side = torch.cuda.Stream()
    if first_on_side:
        plan = gar.gar_attn_plan_create(8, 2, 64)
        with torch.cuda.stream(side):           # allocates; nothing is pending yet
            gar.gar_decode_attention(plan, q, cache, table, lens)
    torch.cuda.synchronize()
    n, at = plan.workspace.numel(), plan.workspace.data_ptr()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)          # some 0.1 s
    got = gar.gar_decode_attention(plan, q, cache, table, lens, stream=side)
    del plan
    gc.collect()
    taken = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for _ in range(3)]
    assert all(t.data_ptr() != at for t in taken)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and all(bool((t == 255).all()) for t in taken)


def test_a_workspace_of_the_callers_own_is_used(monkeypatch):
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda raw, device=None: raw)
    calls = []
    monkeypatch.setattr(gar._lib, "gar_attn_plan_set_workspace", lambda plan, ptr, n: calls.append(ptr.value) or 0)

    def never(*a):
        raise AssertionError("allocates")

    monkeypatch.setattr(gar, "_empty", never)
    plan = gar.gar_attn_plan_create(4, 2, 64)
    gar.gar_attn_plan_set_workspace(plan, 4096, gar.gar_attn_plan_bytes(plan))
    like = types.SimpleNamespace(device=torch.device("cpu"))
    gar._use_workspace(plan, like, 7000)
    gar._use_workspace(plan, like, 8000)
    assert calls == [4096] and plan.stream == 8000
    gar.gar_attn_plan_set_workspace(plan, 0, 0)
    assert calls == [4096, None] and plan.workspace is None and plan.stream is None


@pytest.mark.gpu
def test_attention_with_the_callers_workspace():
    cache, table, lens, q = _problem()
    want = gar.gar_decode_attention(gar.gar_attn_plan_create(8, 2, 64), q, cache, table, lens)
    plan = gar.gar_attn_plan_create(8, 2, 64)
    n = gar.gar_attn_plan_bytes(plan)
    mine = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    gar.gar_attn_plan_set_workspace(plan, mine.data_ptr(), n)
    assert torch.equal(gar.gar_decode_attention(plan, q, cache, table, lens), want)
    assert bool((mine != 255).any()) and plan.workspace == (mine.data_ptr(), n)


def test_what_belongs_to_a_device_is_done_for_each(tmp_path):
    """The kernels' shared memory is allowed for each device that they are launched on, and again after a refusal."""
    csrc = os.path.join(os.path.dirname(gar.__file__), "csrc")
    (tmp_path / "t.cpp").write_text("""
        #include "device_once.hpp"
        #include <cstdio>
        #include <initializer_list>
        int main() {
          static gar::DeviceSet set;
          for (int device : {0, 0, 1, 63, 0, 1, 63, 64, 64, 2, 2, 2}) {
            int called = 0;
            static int left = 1;   // device 2 is refused once
            const int e = gar::once_for_device(set, device, [&] { called = 1; return device == 2 && left-- > 0 ? 7 : 0; });
            std::printf("%d%d ", called, e);
          }
        }""")
    exe = str(tmp_path / "t")
    subprocess.run(["g++", "-std=c++17", "-I", csrc, str(tmp_path / "t.cpp"), "-o", exe], check=True)
    got = subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()
    assert got == ["10", "00", "10", "10", "00", "00", "00", "10", "10", "17", "10", "00"]
    for name in os.listdir(csrc):           # and nothing keeps such a result for the process
        with open(os.path.join(csrc, name)) as f:
            assert not re.search(r"static\s+(const\s+)?(cudaError_t|CUresult)\s+\w+\s*=", f.read()), name


def _fake(shape, dtype=torch.bfloat16, device=0):
    """A tensor that says it is on a GPU, there or not; it has no memory."""
    with mock.patch.object(fake_tensor, "init_gpu_context", lambda device: None, create=True), FakeTensorMode():
        return torch.empty(shape, dtype=dtype, device=f"cuda:{int(device)}")


def _fake_cache(device, heads=2, dim=64, page_size=16):
    """A KVCache over addresses that nothing reads."""
    cache = gar.KVCache.__new__(gar.KVCache)
    cache._c = gar.gar_kv_cache(4096, 8192, None, None, None, 4, heads * page_size * dim, page_size * dim, dim, 0, 0, 0, gar.GAR_BF16,
                                heads, dim, page_size)
    cache.address, cache.device_index = ctypes.addressof(cache._c), device
    return cache


def _calls(devices):
    """(name, number of tensors, call): the call with tensor i on GPU devices[i]."""
    d = list(devices) + [0] * 8
    i64, i32, f32 = torch.int64, torch.int32, torch.float32

    def rope():
        gar.gar_rope(_fake((4, 2, 64), device=d[0]), _fake(4, i64, d[1]), _fake((8, 32, 2), f32, d[2]), out=_fake((4, 2, 64), device=d[3]))

    def write():
        gar.gar_kv_write(_fake_cache(d[0]), _fake((4, 2, 64), device=d[1]), _fake((4, 2, 64), device=d[2]), _fake(4, i64, d[3]),
                         _fake(4, i64, d[4]), _fake((8, 32, 2), f32, d[5]))

    def read():
        gar.gar_kv_read(_fake_cache(d[0]), _fake(4, i64, d[1]), out=(_fake((4, 2, 64), device=d[2]), _fake((4, 2, 64), device=d[3])))

    def attention():
        gar.gar_decode_attention(gar.gar_attn_plan_create(4, 2, 64), _fake((3, 4, 64), device=d[0]), _fake_cache(d[1]), _fake((3, 2), i32, d[2]),
                                 _fake(3, i32, d[3]), out=_fake((3, 4, 64), device=d[4]), lse=_fake((3, 4), f32, d[5]))
    return {"rope": (4, rope), "write": (6, write), "read": (4, read), "attention": (6, attention)}


@pytest.mark.parametrize("name", ["rope", "write", "read", "attention"])
def test_tensors_of_two_gpus_are_refused(name):
    for i in range(_calls([])[name][0]):
        with pytest.raises(ValueError, match="on GPU 1, |on GPU 0, "):
            _calls([int(j == i) for j in range(6)])[name][1]()


def test_a_cache_on_two_gpus_is_refused():
    shape = (4, 2, 16, 64)
    for i in range(4):
        t = [_fake(shape, torch.int8, i == 0), _fake(shape, torch.int8, i == 1), _fake(shape[:3], torch.float32, i == 2),
             _fake(shape[:3], torch.float32, i == 3)]
        with pytest.raises(ValueError, match="one GPU"):
            gar.KVCache(*t)
    with pytest.raises(ValueError, match="one GPU"):
        gar.KVCache(_fake(shape), _fake(shape, device=1))


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["rope", "write", "read", "attention"])
def test_tensors_of_a_gpu_that_is_not_current_are_refused(name):
    torch.zeros(1, device="cuda")
    with pytest.raises(ValueError, match="the current device is GPU 0"):
        _calls([1] * 6)[name][1]()


class _Words:
    """Stands for a tensor of status words on a GPU."""
    made = []

    def __init__(self, n, dtype=None, device=None):
        self.shape, self.device = (n,), device
        _Words.made.append(self)

    def __getitem__(self, i):
        return id(self), i


@pytest.fixture
def status_words(monkeypatch):
    waited = []
    _Words.made = []
    monkeypatch.setattr(gar, "_status_words", {})
    monkeypatch.setattr(torch, "zeros", _Words)
    monkeypatch.setattr(torch.cuda, "synchronize", waited.append)
    return waited


def test_status_words_of_two_gpus(status_words):
    """Each GPU has words of its own, made once and waited for on that GPU."""
    a, b = torch.device("cuda:0"), torch.device("cuda:1")
    got = [gar._status_word(d) for d in (a, b, a, b, a)]
    assert len(set(got)) == 5 and [w.device for w in _Words.made] == [a, b] and status_words == [a, b]


def test_threads_take_different_status_words(status_words, monkeypatch):
    """A thread that is stopped between looking and taking (here while the words are made) leaves none for two."""
    def slow(device):
        status_words.append(device)
        time.sleep(0.05)

    monkeypatch.setattr(torch.cuda, "synchronize", slow)
    got = []
    threads = [threading.Thread(target=lambda: got.append(gar._status_word(torch.device("cuda:0")))) for _ in range(8)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(set(got)) == 8 and len(_Words.made) == 1


def test_rotation_into_memory_has_no_gradient():
    table, pos = _fake((8, 32, 2), torch.float32), _fake(4, torch.int64)
    for x, out in ((_fake((4, 2, 64)).requires_grad_(), _fake((4, 2, 64))), (_fake((4, 2, 64)), _fake((4, 2, 64)).requires_grad_())):
        with pytest.raises(ValueError, match="gradient"):
            gar.gar_rope(x, pos, table, out=out)
    with pytest.raises(ValueError, match="gradient"):
        gar.gar_rope(_fake((4, 2, 64)), pos, table.requires_grad_())


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype,dim,rot", [(torch.float32, 20, 12), (torch.bfloat16, 128, 128)])
def test_gradients_through_the_rotation(layout, dtype, dim, rot):
    f, m = gar.gar_rope_frequencies(rot, 10000.0, "parts", 2.0, 32.0)
    table = gar.gar_rope_table(50, f, m)
    pos = torch.arange(7, device="cuda") * 5
    x = torch.randn(7, 3, dim, device="cuda").to(dtype).requires_grad_()
    g = torch.randn(7, 3, dim, device="cuda").to(dtype)
    plain = gar.gar_rope(x.detach(), pos, table, layout)
    assert not plain.requires_grad
    y = gar.gar_rope(x, pos, table, layout)
    assert y.requires_grad and torch.equal(y, plain)
    grad, = torch.autograd.grad(y, x, g)
    assert torch.equal(grad, gar.gar_rope(g, pos, table, layout, inverse=True))
    # a gradient that is one number everywhere (strides of zero), and one of another order
    grad, = torch.autograd.grad(gar.gar_rope(x, pos, table, layout).sum(), x)
    assert torch.equal(grad, gar.gar_rope(torch.ones_like(g), pos, table, layout, inverse=True))
    turned = g.permute(2, 1, 0).contiguous().permute(2, 1, 0)
    grad, = torch.autograd.grad(gar.gar_rope(x, pos, table, layout, inverse=True), x, turned)
    assert torch.equal(grad, gar.gar_rope(g, pos, table, layout))
    # the gradient's own gradient is the rotation again
    h = torch.randn_like(g).requires_grad_()
    grad, = torch.autograd.grad(gar.gar_rope(x, pos, table, layout), x, h, create_graph=True)
    again, = torch.autograd.grad(grad, h, g)
    assert torch.equal(again, gar.gar_rope(g, pos, table, layout))
    # under a stream of the call's own
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = gar.gar_rope(x, pos, table, layout, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    grad, = torch.autograd.grad(y, x, g)
    assert torch.equal(y, plain) and torch.equal(grad, gar.gar_rope(g, pos, table, layout, inverse=True))
    with torch.no_grad():
        assert not gar.gar_rope(x, pos, table, layout).requires_grad
        assert torch.equal(gar.gar_rope(x, pos, table, layout, out=torch.empty_like(g)), plain)
    if dtype == torch.float32:              # 32-bit differences of a linear map, whatever the step
        loss = lambda t: (gar.gar_rope(t, pos, table, layout).double() * g.double()).sum()
        grad, = torch.autograd.grad(loss(x), x)
        with torch.no_grad():
            for i in range(0, x.numel(), 37):
                t = x.detach().clone()
                t.view(-1)[i] += 1
                step = float(t.view(-1)[i] - x.view(-1)[i])
                d = float(loss(t) - loss(x)) / step
                # two channels differ, each off by at most 4u(|u| + |v|)m in both evaluations
                assert abs(d - float(grad.view(-1)[i])) <= 64 * 2.0 ** -24 * float((x.abs().max() + 1) * g.abs().max()) * m
    many = torch.ones(1, 1, dim, device="cuda", dtype=dtype).expand(1, (1 << 20) + 1, dim)
    for t in (many, many.clone().requires_grad_()):
        with pytest.raises(gar.GarError, match="heads"):
            gar.gar_rope(t, pos[:1], table, layout)
    table2 = table.clone()
    y = gar.gar_rope(x, pos, table2, layout)
    table2 += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(y, x, g)


def test_calls_without_a_gradient_refuse_tensors_that_ask_for_one():
    i64, i32, f32 = torch.int64, torch.int32, torch.float32
    k, g = _fake((4, 2, 64)), _fake((4, 2, 64)).requires_grad_()
    cache, slots, table = _fake_cache(0), _fake(4, i64), _fake((8, 32, 2), f32)
    plan, pages, lens = gar.gar_attn_plan_create(2, 2, 64), _fake((4, 2), i32), _fake(4, i32)
    lse = _fake((4, 2), f32).requires_grad_()
    for call in (lambda: gar.gar_kv_write(cache, g, k, slots), lambda: gar.gar_kv_write(cache, k, g, slots),
                 lambda: gar.gar_kv_write(cache, k, k, slots, slots, _fake((8, 32, 2), f32).requires_grad_()),
                 lambda: gar.gar_kv_read(cache, slots, out=(k, g)), lambda: gar.gar_decode_attention(plan, g, cache, pages, lens),
                 lambda: gar.gar_decode_attention(plan, k, cache, pages, lens, out=g),
                 lambda: gar.gar_decode_attention(plan, k, cache, pages, lens, lse=lse)):
        with pytest.raises(ValueError, match="gradient"):
            call()
    x = _fake((4, 2, 16, 64))
    with pytest.raises(ValueError, match="gradient"):
        gar.KVCache(x, _fake((4, 2, 16, 64)).requires_grad_())


@pytest.mark.gpu
def test_without_gradients_the_same_tensors_are_taken():
    cache, table, lens, q = _problem()
    plan = gar.gar_attn_plan_create(8, 2, 64)
    want = gar.gar_decode_attention(plan, q, cache, table, lens)
    q.requires_grad_()
    for off in (torch.no_grad(), torch.inference_mode()):
        with off:
            assert torch.equal(gar.gar_decode_attention(plan, q, cache, table, lens), want)
            k = q[:, :2].contiguous()
            gar.gar_kv_write(cache, k, k, torch.arange(3, device="cuda"))
            assert torch.equal(gar.gar_kv_read(cache, torch.arange(3, device="cuda"))[0], k)
            cache, table, lens, _ = _problem()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.int8])
def test_autograd_sees_what_calls_write(kind):
    """Memory that a call has written counts as changed: a tensor that autograd has kept is not used with other contents."""
    shape = (2, 2, 16, 64)
    k, v = (torch.zeros(shape, device="cuda").to(kind) for _ in range(2))
    scales = [torch.zeros(shape[:3], device="cuda") for _ in range(2 if kind == torch.int8 else 0)]
    cache = gar.KVCache(k, v, *scales)
    x = torch.randn(4, 2, 64, device="cuda").bfloat16()
    slots, table = torch.arange(4, device="cuda"), gar.gar_rope_table(8, gar.gar_rope_frequencies(64)[0])
    plan, pages = gar.gar_attn_plan_create(2, 2, 64), torch.zeros(4, 1, dtype=torch.int32, device="cuda")
    lens = torch.full((4,), 4, dtype=torch.int32, device="cuda")
    a, b, lse = torch.empty_like(x), torch.empty_like(x), torch.empty(4, 2, device="cuda")
    for call, written in ((lambda: gar.gar_kv_write(cache, x, x, slots), [k, v, *scales]),
                          (lambda: gar.gar_rope(x, slots, table, out=a), [a]),
                          (lambda: gar.gar_kv_read(cache, slots, out=(a, b)), [a, b]),
                          (lambda: gar.gar_decode_attention(plan, x, cache, pages, lens, out=a, lse=lse), [a, lse])):
        others = [t for t in (k, v, *scales, x, a, b, lse) if all(t is not w for w in written)]
        before = [t._version for t in written + others]
        call()
        assert [t._version - n for t, n in zip(written + others, before)] == [1] * len(written) + [0] * len(others)
    y = a.detach().requires_grad_()         # shares a's memory and count
    z = (y * y).sum()
    gar.gar_rope(x, slots, table, out=a)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.backward()
    with torch.inference_mode():
        t = torch.empty_like(x)
    gar.gar_rope(x, slots, table, out=t)    # not counted, and taken
    assert torch.equal(t, a)


def test_more_items_than_the_line_has_room_for_are_refused():
    """Counts of sequences times heads up to the largest that an int holds: refused, or taken as far as to the missing
    workspace (-6), never a number that the line cannot hold."""
    cache = gar.gar_kv_cache(4096, 8192, None, None, None, 4, 1024, 1024, 64, 0, 0, 0, gar.GAR_BF16, 1, 64, 16)

    def call(batch, width, heads=1):
        plan = gar.gar_attn_plan_create(heads, 1, 64)
        return gar._lib.gar_decode_attention(plan.handle, cache, 4096, 64 * heads, 64, gar.GAR_BF16, 8192, 64 * heads, 64, gar.GAR_BF16, None,
                                             4096, width, width, 4096, batch, 0.125, 0, None)

    assert call(178956970, 0) == -6 and call(178956971, 0) == -1
    for batch in (178956971, 200000000, (1 << 28) - 1, 1 << 28, 2 ** 31 - 1):
        for width in (0, 1, 100, 2 ** 31 - 1):
            assert call(batch, width) == -1, (batch, width)
    assert call(8000, 2 ** 31 - 1) == -6 and call(9000, 2 ** 31 - 1) == -1      # 2^31 / 2^15 units of each sequence
    assert call(22369621, 0, 64) == -6 and call(22369622, 0, 64) == -1          # 8 groups of query heads


def test_numbers_past_an_int_are_refused():
    """They were cut to 32 bits: a window of 2^32 + 5 rows was one of 5."""
    i64, i32, f32 = torch.int64, torch.int32, torch.float32
    x, pos, table, cache = _fake((4, 2, 64)), _fake(4, i64), _fake((8, 32, 2), f32), _fake_cache(0)
    plan, pages, lens = gar.gar_attn_plan_create(2, 2, 64), _fake((4, 2), i32), _fake(4, i32)
    many = (1 << 32) + 2
    for call in (lambda: gar.gar_rope(x, pos, table, 1 << 32), lambda: gar.gar_rope(x, pos, table, -(1 << 32) + 1),
                 lambda: gar.gar_kv_write(cache, x, x, pos, pos, table, 1 << 32),
                 lambda: gar.gar_rope(_fake((4, many, 64)), pos, table), lambda: gar.gar_kv_write(cache, *[_fake((4, many, 64))] * 2, pos),
                 lambda: gar.gar_kv_write(cache, *[_fake((4, 2, many + 62))] * 2, pos),
                 lambda: gar.gar_decode_attention(plan, x, cache, pages, lens, window=(1 << 32) + 5),
                 lambda: gar.gar_decode_attention(plan, x, cache, pages, lens, window=-(1 << 32) + 5),
                 lambda: gar.gar_decode_attention(plan, x, cache, _fake((4, many), i32), lens),
                 lambda: gar.gar_decode_attention(plan, _fake((many, 2, 64)), cache, _fake((many, 2), i32), _fake(many, i32)),
                 lambda: gar.gar_attn_plan_create(many, 1, 64), lambda: gar.gar_attn_plan_create(2, many, 64),
                 lambda: gar.gar_attn_plan_create(2, 2, many), lambda: gar.gar_rope_frequencies(many + 62),
                 lambda: gar.gar_rope_frequencies(64, scaling=1 << 32), lambda: gar.KVCache(*[_fake((1, many, 1, 4))] * 2),
                 lambda: gar.KVCache(*[_fake((1, 1, many, 4))] * 2), lambda: gar.KVCache(*[_fake((1, 1, 1, many))] * 2)):
        with pytest.raises(ValueError, match="out of range"):
            call()


def test_objects_of_another_class_are_refused():
    """A plan where the cache belongs, and the other way round, has an address too: of something else."""
    i64, i32 = torch.int64, torch.int32
    x, slots, pages, lens = _fake((4, 2, 64)), _fake(4, i64), _fake((4, 2), i32), _fake(4, i32)
    cache, plan = _fake_cache(0), gar.gar_attn_plan_create(2, 2, 64)

    class Own(gar.KVCache):
        pass

    other = types.SimpleNamespace(address=cache.address, device_index=0, stream=None)
    for wrong in (plan, other, 5, "cache"):
        for call in (lambda: gar.gar_kv_write(wrong, x, x, slots), lambda: gar.gar_kv_read(wrong, slots),
                     lambda: gar.gar_decode_attention(plan, x, wrong, pages, lens)):
            with pytest.raises(TypeError, match="KVCache"):
                call()
    for wrong in (cache, other, 5):
        with pytest.raises(TypeError, match="AttnPlan"):
            gar.gar_decode_attention(wrong, x, cache, pages, lens)
    cache.__class__ = Own                   # a class of the caller's own made from it is one
    with pytest.raises(ValueError, match="alike"):
        gar.gar_kv_write(cache, x, x[:1], slots)


def test_names_of_layouts_are_the_headers():
    """The compiled calls know them alone; their codes are the header's."""
    x, pos, table = _fake((4, 2, 64)), _fake(4, torch.int64), _fake((8, 32, 2), torch.float32, 1)
    for layout in ("half", "interleaved", gar.GAR_ROPE_HALF, gar.GAR_ROPE_INTERLEAVED):
        with pytest.raises(ValueError, match="GPU 1"):
            gar.gar_rope(x, pos, table, layout)
    with pytest.raises(ValueError, match="layout"):
        gar.gar_rope(x, pos, _fake((8, 32, 2), torch.float32), "third")
    assert not hasattr(gar, "ROPE_LAYOUTS")
