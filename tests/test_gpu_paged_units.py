"""Attention over pages on the GPU where a worker of the line has several units of its own."""
import math

import pytest
import torch

import paged_reference as ref
from paper_2311_08263_b200 import engine, lib
from test_gpu_paged import _close, _dealt, _on_tcgen05, _queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd,ps,B,lens", [
    (64, 5, 48, [65, 75, 66, 130]), (64, 100, 64, [65, 70, 75]), (64, 1, 64, [70]), (64, 20, 48, [3, 64, 127, 1, 200]), (128, 5, 48, [65, 75, 66, 130]),
    (128, 100, 64, [60, 70, 5]), (64, 16, 48, [65, 75, 66, 130])])
def test_several_units_of_a_few_tiles_per_worker(hd, ps, B, lens):
    """Queries of one unit after the other go into two places: seven and more units of one to four tiles to a CTA, beginning at odd and even tiles, by copies
    (pages that are not whole groups of eight slots) and by TMA."""
    hq, hkv, c = 32, 4, 64
    lens = (lens * B)[:B]
    gen = torch.Generator().manual_seed(hd + ps)
    table, n_pages = _dealt(lens, c, ps, gen)
    k, v = (torch.randn(n_pages, hkv, ps, hd, generator=gen).to(torch.bfloat16).cuda() for _ in range(2))
    table, kv_len = table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    q = _queries(B * c, hq * hd, torch.bfloat16, 1)
    assert _on_tcgen05(k, table, c, hq)
    want, tol = ref.attention(q, k, v, table, kv_len, c, hq)
    first = engine.fc_op_paged_attention(q, k, v, table, kv_len, c, hq)
    _close(first, want, tol)
    for _ in range(20):
        assert torch.equal(engine.fc_op_paged_attention(q, k, v, table, kv_len, c, hq), first)


@pytest.mark.parametrize("dtype,hkv,n,ps,warps,floats", [("bf16", 48, 2047, 64, 12, 8 * 66), ("bf16", 32, 143, 16, 8, 8 * 66), ("f32", 32, 2047, 64, 8, 68)])
def test_what_follows_whole_units_reads_their_results(dtype, hkv, n, ps, warps, floats):
    """As many units of one length as the plan has workers, told by its scratch: none is joined, and the next kernel of the stream finds all of them done."""
    dt, B, hd = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype], 37, 64
    workers = 148 * warps
    assert B * hkv == workers                                                # one query per kv head: a unit each
    width = n // ps + 1
    size = lib.load().fc_op_paged_attention_scratch_bytes(B, 1, hkv, hkv, hd, lib.FC_F32 if dtype == "f32" else lib.FC_BF16, width, ps, 0, 0)
    assert size == 256 + -(-workers * 2 * floats * 4 // 256) * 256
    k, v = (torch.randn(width, hkv, ps, hd, generator=torch.Generator().manual_seed(3)).to(dt).cuda() for _ in range(2))
    table = torch.arange(width, dtype=torch.int32).cuda().repeat(B, 1)                          # one prompt, read by all
    kv_len = torch.full((B,), n, dtype=torch.int32).cuda()
    q = _queries(B, hkv * hd, dt, 1)
    want, tol = ref.attention(q[:2], k, v, table[:2], kv_len[:2], 1, hkv)
    for _ in range(20):
        torch.full((B, hkv * hd), math.nan, device="cuda")                                       # the memory that the result gets
        out = engine.fc_op_paged_attention(q, k, v, table, kv_len, 1, hkv)
        copy = out + 0
        torch.cuda.synchronize()
        assert torch.equal(copy, out) and out.isfinite().all()
    _close(copy[:2], want, tol)
