"""Decoding kernels become resident before the kernel ahead of them on the stream has finished, so what that one writes
has to be read as memory that changes."""

import os
import re

import pytest
import torch

from paper_2004_09362_gb300 import gar

CSRC = os.path.join(os.path.dirname(gar.__file__), "csrc")


@pytest.mark.parametrize("name", ["gar_device.cuh", "rope.cu", "cache.cu", "decode.cuh", "decode_general.cu", "decode_mma.cuh"])
def test_no_loads_that_take_memory_for_constant(name):
    with open(os.path.join(CSRC, name)) as f:
        assert not re.search(r"__ldg\b|ld\.global(\.\w+)*\.nc|__restrict__", f.read())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,heads,dim,layout", [(torch.bfloat16, 8, 128, "half"), (torch.float32, 3, 10, "half"),
                                                    (torch.float16, 40, 64, "interleaved")])
def test_a_table_rewritten_between_calls(dtype, heads, dim, layout):
    """Table, rotation, table, write, all in one place and back to back: each call sees the table before it."""
    f, _ = gar.gar_rope_frequencies(dim)
    tokens, rows = 37, 64
    x = torch.randn(tokens, heads, dim, device="cuda").to(dtype)
    pos = torch.arange(tokens, device="cuda")
    tables = [gar.gar_rope_table(rows, f, first=1000 * i) for i in range(6)]
    want = [gar.gar_rope(x, pos, t, layout) for t in tables]
    caches = []
    for i in range(6):
        k, v = (torch.zeros(3, heads, 16, dim, device="cuda", dtype=dtype) for _ in range(2))
        caches.append(gar.KVCache(k, v))
    table, got = torch.empty_like(tables[0]), [torch.empty_like(x) for _ in range(6)]
    fc, stream = (gar.ctypes.c_double * len(f))(*f), gar._stream_handle(None)
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(6):
            assert gar._lib.gar_rope_table(table.data_ptr(), 1000 * i, rows, dim, fc, 1.0, stream) == 0
            gar.gar_rope(x, pos, table, layout, out=got[i])
            gar.gar_kv_write(caches[i], x, x, pos, pos, table, layout)
        for i in range(6):
            assert torch.equal(got[i], want[i])
            assert torch.equal(gar.gar_kv_read(caches[i], pos, {torch.float32: "f32", torch.float16: "f16"}.get(dtype, "bf16"))[0], want[i])
