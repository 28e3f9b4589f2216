"""Attention over pages on the GPU: values that are not finite, and how much of a probability there is in a result."""
import math

import pytest
import torch

import paged_reference as ref
from paper_2311_08263_b200 import engine
from test_gpu_paged import _cache, _close, _on_tcgen05, _queries, _widened

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


@pytest.mark.parametrize("hq,hkv,hd,c,B,ps,width", [
    (16, 2, 64, 1, 60, 16, 1), (16, 2, 64, 1, 300, 16, 1000), (64, 4, 128, 1, 2, 16, 1), (64, 4, 128, 1, 30, 16, 1000), (32, 4, 32, 1, 60, 16, 1000),
    (256, 2, 64, 1, 20, 16, 4000), (256, 2, 128, 1, 20, 16, 4000), (256, 2, 64, 1, 20, 20, 4000)])
def test_probabilities_enter_the_products_whole(hq, hkv, hd, c, B, ps, width):
    """Two keys whose values are all 1: the result is (p0 + p1) / (p0 + p1).

    Numerator: three bf16 parts hold a probability's 24 bits, so that only sums can be off.  The product of the high parts adds three terms of at most 1, each cut
    off at 2^-23; those of the middle and low parts are at most 2^-8 and 2^-16 of that.  Denominator: one sum rounded (2^-24, sums with zero are exact).
    The reciprocal and its product: 2^-24 each.  Together less than 5 x 2^-23, for numerator and denominator are at least 1 - 2^-22.  Two parts would leave up to
    2^-18 of p1 out."""
    k, v, table, kv_len = _cache([1] * B, c, hkv, hd, ps, torch.bfloat16, "hnd", 11)
    q = _queries(B, hq * hd, torch.bfloat16, 12) * 0.4
    v = torch.where(v.isnan(), v, 1.0)
    table = _widened(table, ps, width * ps)
    if hq // hkv > 32:
        assert _on_tcgen05(k, table, c, hq)
    bound = 5 * 2.0 ** -23
    out = engine.fc_op_paged_attention(q, k, v, table, kv_len, c, hq)
    assert (out.double() - 1).abs().max() <= bound
    # and that these probabilities would tell
    at = table[:, 0].long()
    s = torch.einsum("bhgd,bhnd->bhgn", q.double().view(B, hkv, -1, hd), k[at, :, :2].double()) / math.sqrt(hd)
    p = (s - s.amax(-1, keepdim=True)).exp().float()
    high = p.bfloat16().float()
    two = high.double() + (p - high).bfloat16().double()
    assert ((two.sum(-1) - p.double().sum(-1)) / p.double().sum(-1)).abs().max() > 2 * bound
