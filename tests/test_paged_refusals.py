"""Paged K/V cache without a GPU: sizes of scratch and calls refuse the same, and the binding passes no number on that C would read as another."""
import pytest
import torch

from paper_2311_08263_b200 import build, engine, lib

P = 1 << 20                                  # stands for device pointers: a refused call touches none


@pytest.fixture(scope="module")
def l():
    build.build()
    return lib.load()


GOOD = dict(batch=3, c=2, hq=8, hkv=4, hd=64, dtype=lib.FC_BF16, width=5000, page=16, window=0, n_sink=0)


@pytest.mark.parametrize("change", [
    dict(batch=1 << 27, c=64, hq=4),                                          # rows times heads beyond 2^30
    dict(page=1 << 24, hkv=4, width=100), dict(page=1 << 23, hkv=8, hd=64, width=1),      # pages of more than 2^31 elements
    dict(hq=516), dict(hq=1024, hkv=1), dict(c=65), dict(hd=96), dict(width=1 << 28), dict(dtype=2)])
def test_no_scratch_for_an_attention_that_is_refused(l, change):
    a = dict(GOOD, **change)
    rows = a["page"] * a["hd"]
    pool = lib.fc_pages(P, 2 * P, a["dtype"], 1, 1, a["hkv"], a["page"], a["hd"], 0, a["hkv"] * rows, rows, a["hd"])
    assert l.fc_op_paged_attention(pool, 0, P, a["width"], P, P, a["hq"] * a["hd"], P, a["batch"], a["c"], a["hq"], a["window"], a["n_sink"], P, 1 << 50, None) < 0
    assert l.fc_op_paged_attention_scratch_bytes(*a.values()) == 0


def test_the_largest_pages_and_calls_have_scratch(l):
    assert l.fc_op_paged_attention_scratch_bytes(*dict(GOOD, page=1 << 23, hkv=4, width=1).values()) > 256                # 2^31 elements
    assert l.fc_op_paged_attention_scratch_bytes(*dict(GOOD, batch=(1 << 30) // 16 - 1, width=5).values()) > 256


BIG = 1 << 32                                # C would see 0, and BIG + 1 as 1


@pytest.mark.parametrize("big", [BIG, BIG + 1, 1 << 31, -BIG, -BIG + 1])
def test_binding_passes_no_number_that_c_would_read_as_another(big):
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    table, lens, refs = torch.zeros(3, 3, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    q = torch.zeros(3, 2 * 64, dtype=torch.bfloat16)
    for call in (lambda: engine.fc_op_paged_attention(q, k, k.clone(), table, lens, 1, 2, window=big),
                 lambda: engine.fc_op_paged_attention(q, k, k.clone(), table, lens, 1, 2, window=4, n_sink=big),
                 lambda: engine.fc_op_pages_reserve(k[None], k[None].clone(), table, lens, refs, big),
                 lambda: engine.fc_op_pages_fork(table, lens, refs, big, [0], [1]),
                 lambda: engine.fc_op_pages_free(table, lens, refs, big, [0]),
                 lambda: engine.fc_op_pages_free(table, lens, refs, 16, [0], window=big),
                 lambda: engine.fc_op_pages_free(table, lens, refs, 16, [0], window=4, n_sink=big),
                 lambda: engine._list([0, big])):
        with pytest.raises(ValueError, match="beyond 32 bits"):
            call()
    assert list(engine._list([])) == [] and list(engine._list([0, -1, 2 ** 31 - 1])) == [0, -1, 2 ** 31 - 1]
