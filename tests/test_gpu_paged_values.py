"""Attention over pages on the GPU: values that are not finite, and how much of a probability there is in a result."""
import math

import pytest
import torch

import paged_reference as ref
from paper_2311_08263_b200 import engine
from test_gpu_paged import _cache, _close, _queries, _widened

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,hkv,hd,c,n,ps,width", [
    (8, 2, 64, 1, 300, 16, 20), (8, 2, 64, 1, 300, 16, 3000), (4, 2, 128, 1, 700, 16, 3000), (16, 4, 32, 4, 300, 5, 3000),       # one row per sequence: seen by all
    (16, 2, 128, 16, 300, 16, 20), (32, 4, 64, 16, 700, 16, 3000), (32, 4, 128, 16, 700, 16, 3000), (32, 4, 64, 16, 700, 20, 3000)])
def test_values_that_are_not_finite_in_tiles_seen_whole(dtype, hq, hkv, hd, c, n, ps, width):
    """Infinities and NaN in an early key that every row sees: no finite result in those elements of its kv head, whichever kernel it is; the others as ever."""
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    k, v, table, kv_len = _cache([n, 7], c, hkv, hd, ps, dt, "hnd", 3)
    table = _widened(table, ps, width * ps)
    q = _queries(2 * c, hq * hd, dt, 4)
    want, tol = ref.attention(q, k, v, table, kv_len, c, hq)
    for bad in (math.inf, -math.inf, math.nan):
        v2 = v.clone()
        v2[int(table[0, 37 // ps]), 1, 37 % ps, 2::5] = bad
        out = engine.fc_op_paged_attention(q, k, v2, table, kv_len, c, hq).view(2, c, hkv, hq // hkv, hd)
        hit = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
        hit[0, :, 1, :, 2::5] = True
        assert torch.equal(out.isfinite(), ~hit)
        _close(torch.where(hit, 0.0, out), torch.where(hit.cpu().view_as(want), 0.0, want), tol)
