"""A wait for a copy that runs out: the kernel ends, says so, and the next call is right."""

import pytest
import torch

from paper_2004_09362_gb300 import gar

TIMEOUT = -8


def test_debug_wait_refusals():
    assert gar._lib.gar_attn_plan_debug_wait(None, 0) == -1
    plan = gar.gar_attn_plan_create(4, 2, 64)
    gar.gar_attn_plan_debug_wait(plan, 3)
    gar.gar_attn_plan_debug_wait(plan)
    with pytest.raises(ValueError, match="out of range"):
        gar.gar_attn_plan_debug_wait(plan, 1 << 40)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,heads,lengths", [
    (torch.bfloat16, 8, [5000]), (torch.float16, 16, [3000, 0, 40, 1, 20000]), (torch.float32, 4, [2000, 17, 333]),
    (torch.bfloat16, 4, [(b * 37) % 700 for b in range(600)])])
@pytest.mark.parametrize("tile", [0, 1, 5])
def test_waits_that_run_out(dtype, heads, lengths, tile):
    """Real copies are on their way when the waits report that they ran out: by tile, in segments of one warp and of
    many, with and without a join between CTAs, and with more segments than a CTA notes at a time."""
    dim, page = 256, 16
    need = [-(-n // page) for n in lengths]
    table = torch.full((len(lengths), max(need)), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = torch.arange(at, at + n, dtype=torch.int32)
        at += n
    table = table.cuda()
    k, v = (torch.randn(at, 1, page, dim, device="cuda").to(dtype) for _ in range(2))
    cache, lens = gar.KVCache(k, v), torch.tensor(lengths, dtype=torch.int32, device="cuda")
    q = torch.randn(len(lengths), heads, dim, device="cuda").to(dtype)
    # where the batch's pieces of 64 rows, four tiles, are no more than the CTAs, each is a segment: there is no tile 4
    many = sum(max(1, -(-n // 64)) for n in lengths) > min(152, torch.cuda.get_device_properties(0).multi_processor_count)
    plan = gar.gar_attn_plan_create(heads, 1, dim)
    want = gar.gar_decode_attention(plan, q, cache, table, lens, lse=True)
    gar.gar_kv_status(cache)
    for _ in range(2):
        gar.gar_attn_plan_debug_wait(plan, tile)
        gar.gar_decode_attention(plan, q, cache, table, lens)
        if tile < 4 or many:
            with pytest.raises(gar.GarError) as e:
                gar.gar_kv_status(cache)
            assert e.value.code == TIMEOUT and "did not end" in str(e.value)
        else:
            gar.gar_kv_status(cache)
        gar.gar_attn_plan_debug_wait(plan)
        got = gar.gar_decode_attention(plan, q, cache, table, lens, lse=True)
        gar.gar_kv_status(cache)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
