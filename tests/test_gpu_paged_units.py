"""Attention over pages on the GPU where a worker of the line has several units of its own."""
import pytest
import torch

import paged_reference as ref
from paper_2311_08263_b200 import engine
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
