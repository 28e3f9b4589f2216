"""Paged K/V cache without a GPU: calls that are refused before anything is launched, scratch sizes, the index arithmetic of the kernels."""
import ctypes as C
import os
import random
import subprocess

import pytest
import torch

import paged_reference as ref
from paper_2311_08263_b200 import build, engine, lib

P = 1 << 20                                  # stands for device pointers: a refused call touches none


def _pool(**kw):
    p = lib.fc_pages(P, 2 * P, lib.FC_BF16, 2, 10, 4, 16, 64, 10 * 4 * 16 * 64, 4 * 16 * 64, 16 * 64, 64)
    for name, value in kw.items():
        setattr(p, name, value)
    return p


@pytest.fixture(scope="module")
def l():
    build.build()
    return lib.load()


def _store(l, pool=None, layer=0, table=P, width=5, kv_len=P, qkv=P, stride=16 * 64, q=P, batch=3, c=2, hq=8, theta=1e4):
    return l.fc_op_paged_store(_pool() if pool is None else pool, layer, table, width, kv_len, qkv, stride, q, batch, c, hq, theta, None)


def _attention(l, pool=None, layer=0, table=P, width=5, kv_len=P, q=P, stride=8 * 64, out=P, batch=3, c=2, hq=8, window=0, n_sink=0,
               scratch=P, nbytes=1 << 40):                      # long enough for the line: scratch is used
    return l.fc_op_paged_attention(_pool() if pool is None else pool, layer, table, width, kv_len, q, stride, out, batch, c, hq, window, n_sink, scratch,
                                   nbytes, None)


def _reserve(l, pool=None, table=P, width=5, n=3, kv_len=P, refs=P, rows=2, scratch=P, nbytes=1 << 40):
    return l.fc_op_pages_reserve(_pool() if pool is None else pool, table, width, n, kv_len, refs, rows, None, scratch, nbytes, None)


def _compact(l, pool=None, table=P, width=5, n=3, refs=P, scratch=P, nbytes=1 << 40):
    return l.fc_op_pages_compact(_pool() if pool is None else pool, table, width, n, refs, None, scratch, nbytes, None)


def _list(*ids):
    return (C.c_int32 * max(1, len(ids)))(*ids)


def _free(l, seqs=(0, 2), n=None, table=P, width=5, rows=3, kv_len=P, refs=P, pages=10, ps=16, window=0, n_sink=0):
    a = _list(*seqs) if seqs is not None else None
    return l.fc_op_pages_free(table, width, rows, kv_len, refs, pages, ps, a, len(seqs) if n is None else n, window, n_sink, None)


def _fork(l, src=(0,), dst=(1,), n=None, table=P, width=5, rows=3, kv_len=P, refs=P, pages=10, ps=16):
    return l.fc_op_pages_fork(table, width, rows, kv_len, refs, pages, ps, _list(*src), _list(*dst), len(dst) if n is None else n, None)


BAD_POOLS = [
    (dict(k=None), lib.FC_ERR_ARG), (dict(v=None), lib.FC_ERR_ARG), (dict(v=P), lib.FC_ERR_ARG), (dict(k=P + 8), lib.FC_ERR_ARG),
    (dict(dtype=7), lib.FC_ERR_ARG), (dict(n_layers=0), lib.FC_ERR_ARG), (dict(n_pages=0), lib.FC_ERR_ARG), (dict(n_kv_heads=0), lib.FC_ERR_ARG),
    (dict(page_size=0), lib.FC_ERR_ARG), (dict(head_dim=96), lib.FC_ERR_SHAPE), (dict(slot_stride=60), lib.FC_ERR_ARG),
    (dict(slot_stride=32), lib.FC_ERR_ARG),                                                  # rows overlap
    (dict(head_stride=8 * 64), lib.FC_ERR_ARG),                                              # heads overlap
    (dict(page_stride=0), lib.FC_ERR_ARG), (dict(layer_stride=4 * 16 * 64), lib.FC_ERR_ARG), (dict(page_stride=-4096), lib.FC_ERR_ARG),
    (dict(head_stride=1 << 46), lib.FC_ERR_ARG), (dict(page_size=1 << 24, n_kv_heads=1), lib.FC_ERR_ARG),
    (dict(page_size=1 << 26, n_kv_heads=1, head_stride=1 << 32, page_stride=1 << 32, layer_stride=1 << 36), lib.FC_ERR_CAPACITY),
]


@pytest.mark.parametrize("change,code", BAD_POOLS)
def test_pools_that_are_refused(l, change, code):
    for call in (_store, _attention, _reserve, _compact):
        assert call(l, pool=_pool(**change)) == code


def test_null_pool(l):
    none = C.POINTER(lib.fc_pages)()
    for call in (_store, _attention, _reserve, _compact):
        assert call(l, pool=none) == lib.FC_ERR_ARG


@pytest.mark.parametrize("kw,code", [
    (dict(layer=-1), -1), (dict(layer=2), -1), (dict(table=None), -1), (dict(width=0), -1), (dict(kv_len=None), -1), (dict(qkv=None), -1),
    (dict(qkv=P + 4), -1), (dict(stride=16 * 64 - 4), -1), (dict(stride=16 * 64 + 2), -1), (dict(q=None), -1), (dict(q=P + 8), -1),
    (dict(batch=0), -1), (dict(c=0), -1), (dict(c=65), -1), (dict(hq=6), -1), (dict(hq=0), -1), (dict(theta=0.0), -1), (dict(theta=float("nan")), -1),
    (dict(theta=float("inf")), -1), (dict(width=1 << 28), lib.FC_ERR_CAPACITY), (dict(batch=1 << 30, c=4), lib.FC_ERR_CAPACITY)])
def test_store_refusals(l, kw, code):
    assert _store(l, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(layer=-1), -1), (dict(layer=2), -1), (dict(table=None), -1), (dict(width=0), -1), (dict(kv_len=None), -1), (dict(q=None), -1), (dict(q=P + 8), -1),
    (dict(stride=8 * 64 - 8), -1), (dict(stride=8 * 64 + 4), -1), (dict(out=None), -1), (dict(out=P + 4), -1), (dict(batch=0), -1), (dict(c=0), -1),
    (dict(c=65), -1), (dict(hq=6), -1), (dict(window=-1), -1), (dict(n_sink=-1), -1), (dict(width=5000, scratch=None), -1), (dict(scratch=P + 16), -1),
    (dict(width=5000, nbytes=1000), lib.FC_ERR_CAPACITY), (dict(width=1 << 28), lib.FC_ERR_CAPACITY),
    (dict(width=2 ** 31 // 16 - 100, c=64, hq=512, stride=512 * 64), lib.FC_ERR_CAPACITY), (dict(hq=516, stride=516 * 64), lib.FC_ERR_CAPACITY)])
def test_attention_refusals(l, kw, code):
    assert _attention(l, **kw) == code


def test_attention_scratch_bytes(l):
    size = l.fc_op_paged_attention_scratch_bytes
    args = dict(batch=3, c=2, hq=8, hkv=4, hd=64, dtype=lib.FC_BF16, width=5000, page=16, window=0, n_sink=0)
    good = size(*args.values())
    assert good > 256 and good % 256 == 0
    assert size(*dict(args, width=5).values()) == 256                      # clusters: none is used
    assert size(*dict(args, window=64).values()) == 256
    for bad in (dict(batch=0), dict(c=0), dict(c=65), dict(hq=7), dict(hq=516), dict(hkv=0), dict(hd=80), dict(dtype=2), dict(width=0), dict(page=0),
                dict(width=1 << 28), dict(window=-1), dict(n_sink=-1)):
        assert size(*dict(args, **bad).values()) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(table=None), -1), (dict(width=0), -1), (dict(n=0), -1), (dict(kv_len=None), -1), (dict(refs=None), -1), (dict(rows=0), -1), (dict(rows=65), -1),
    (dict(scratch=None), -1), (dict(scratch=P + 128), -1), (dict(nbytes=64), lib.FC_ERR_CAPACITY), (dict(width=1 << 28), lib.FC_ERR_CAPACITY)])
def test_reserve_refusals(l, kw, code):
    assert _reserve(l, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(table=None), -1), (dict(width=0), -1), (dict(n=0), -1), (dict(refs=None), -1), (dict(scratch=None), -1), (dict(scratch=P + 128), -1),
    (dict(nbytes=64), lib.FC_ERR_CAPACITY)])
def test_compact_refusals(l, kw, code):
    assert _compact(l, **kw) == code


@pytest.mark.parametrize("kw", [
    dict(seqs=(0, 0)), dict(seqs=(3,)), dict(seqs=(-1,)), dict(n=-1), dict(seqs=None, n=1), dict(table=None), dict(width=0), dict(rows=0), dict(kv_len=None),
    dict(refs=None), dict(pages=0), dict(ps=0), dict(window=-1), dict(n_sink=-1)])
def test_free_refusals(l, kw):
    assert _free(l, **kw) == lib.FC_ERR_ARG


@pytest.mark.parametrize("kw", [
    dict(src=(0, 0), dst=(1, 1)), dict(src=(0,), dst=(0,)), dict(src=(0, 1), dst=(1, 2)), dict(src=(3,)), dict(src=(-1,)), dict(dst=(3,)), dict(dst=(-1,)),
    dict(n=-1), dict(table=None), dict(width=0), dict(rows=0), dict(kv_len=None), dict(refs=None), dict(pages=0), dict(ps=0)])
def test_fork_refusals(l, kw):
    assert _fork(l, **kw) == lib.FC_ERR_ARG


def test_nothing_to_free_or_fork(l):
    assert _free(l, seqs=()) == lib.FC_OK and _fork(l, src=(), dst=()) == lib.FC_OK


def test_binding_refuses_tensors_that_do_not_fit():
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    table, lens, refs = torch.zeros(1, 3, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    q = torch.zeros(1, 2 * 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="one CUDA device"):
        engine.fc_op_paged_attention(q, k, k.clone(), table, lens, 1, 2)
    with pytest.raises(ValueError, match="same shape and strides"):
        engine.fc_op_paged_attention(q, k, k.float(), table, lens, 1, 2)
    with pytest.raises(ValueError, match="same shape and strides"):
        engine.fc_op_paged_attention(q, k.half(), k.half(), table, lens, 1, 2)
    with pytest.raises(ValueError, match="same shape and strides"):
        engine.fc_op_paged_attention(q, k, k.transpose(1, 2).contiguous().transpose(1, 2), table, lens, 1, 2)
    with pytest.raises(ValueError, match="CUDA device"):
        engine.fc_op_pages_free(table, lens, refs, 16, [0])


# ---- index arithmetic, compiled with the host compiler
WRAP = """
#include "fc_paged.h"
extern "C" {
int page_of(const int *row, int width, int t, int ps, int n) { return fc::page_of(row, width, t, ps, n); }
int sees(int p, int t, int w, int s) { return fc::sees(p, t, w, s); }
int window_first(int p, int w) { return fc::window_first(p, w); }
int page_unseen(int i, int ps, int len, int w, int s) { return fc::page_unseen(i, ps, len, w, s); }
int clamp_len(int len, int cap) { return fc::clamp_len(len, cap); }
}
"""


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    d = tmp_path_factory.mktemp("paged")
    src, so = d / "wrap.cpp", d / "wrap.so"
    src.write_text(WRAP)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", build.CSRC, "-I", build.INCLUDE, str(src), "-o", str(so)])
    return C.CDLL(str(so))


def test_pages_that_are_not_in_the_pool_have_no_address(host):
    row = (C.c_int32 * 6)(3, -1, 4, 5, 2 ** 31 - 1, -2 ** 31)
    got = [host.page_of(row, 6, t, 4, 5) for t in range(0, 32)]
    assert got == [3] * 4 + [-1] * 4 + [4] * 4 + [-1] * 20
    assert host.page_of(row, 6, -1, 4, 5) == -1 and host.page_of(row, 6, 2 ** 31 - 1, 1, 5) == -1


@pytest.mark.parametrize("window,n_sink", [(0, 0), (1, 0), (1, 3), (4, 0), (4, 2), (7, 100), (2 ** 31 - 1, 5)])
def test_what_a_row_sees(host, window, n_sink):
    for p in range(20):
        want = ref.visible(p, window, n_sink)
        assert [t for t in range(30) if host.sees(p, t, window, n_sink)] == want
        assert host.window_first(p, window) == (want[-1] - len([t for t in want if t > p - window]) + 1 if window else 0)


def test_pages_released_under_a_window_are_those_that_no_later_row_sees(host):
    for ps in (1, 3, 4):
        for window in (1, 2, 5, 9):
            for n_sink in (0, 1, 4, 7):
                for n in range(0, 25):
                    for i in range(9):
                        seen = any(host.sees(p, t, window, n_sink) for p in range(n, n + 12) for t in range(i * ps, i * ps + ps))
                        beyond = (i + 1) * ps > n                             # nothing there yet: written later, then seen
                        assert bool(host.page_unseen(i, ps, n, window, n_sink)) == (not seen and not beyond)
    assert host.page_unseen(0, 16, 2 ** 31 - 1, 1, 0) and not host.page_unseen(0, 16, -1, 1, 0)


def test_lengths_stay_within_the_table(host):
    assert [host.clamp_len(n, 100) for n in (-2 ** 31, -1, 0, 99, 100, 101, 2 ** 31 - 1)] == [-1, -1, 0, 99, 100, 100, 100]


@pytest.fixture(scope="module")
def parts(tmp_path_factory):
    d = tmp_path_factory.mktemp("parts")
    src, so = d / "wrap.cpp", d / "wrap.so"
    src.write_text("""
#include "fc_paged.h"
extern "C" {
int part_floats(int q, int hd) { return fc::part_floats(q, hd); }
void key_tiles(int len, int rows, int cap, int w, int s, int keys, int *out) {
  const fc::KeyTiles t = fc::key_tiles(len, rows, cap, w, s, keys);
  out[0] = t.n;
  for (int i = 0; i < t.n && i < 4000; ++i) out[1 + i] = fc::tile_key(t, i, keys);
}
int chunk_of(int total, int n) { return fc::chunk_of(total, n); }
int quotient16(int x, int n) { return fc::quotient16(x, fc::reciprocal16(n)); }
int line_batch(int u, int cap, int k) { return fc::line_batch(u, cap, k); }
void plan(int b, int c, int hq, int hkv, int hd, int f32, int cap, int w, int s, long long *out) {
  const fc::PagedPlan p = fc::paged_plan(b, c, hq, hkv, hd, f32 != 0, cap, w, s);
  out[0] = p.kind; out[1] = p.queries; out[2] = p.keys; out[3] = p.units; out[4] = p.ctas; out[5] = p.workers; out[6] = (long long)p.scratch; out[7] = p.fits;
}
void unit_parts(int begin, int n, int chunk, int *out) { const fc::UnitParts p = fc::unit_parts(begin, n, chunk); out[0] = p.first; out[1] = p.last; }
int part_place(int begin, int worker, int chunk) { return fc::part_place(begin, worker, chunk); }

}
""")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", build.CSRC, "-I", build.INCLUDE, str(src), "-o", str(so)])
    lib_ = C.CDLL(str(so))
    return lib_


def test_parts_are_whole_16_byte_pieces(parts):
    """Parts follow one another in scratch and are read and written 16 bytes at a time, for any number of queries."""
    for hd in (32, 64, 128):
        for q in range(1, 129):
            n = parts.part_floats(q, hd)
            assert n % 4 == 0 and n >= q * (hd + 2)


@pytest.mark.parametrize("keys", [8, 16, 32, 64])
def test_tiles_hold_every_key_that_is_seen_once(parts, keys):
    r = random.Random(keys)
    out = (C.c_int * 4001)()
    for _ in range(3000):
        cap = r.choice([1, 5, 100, 1000])
        n, rows = r.choice([-1, 0, 1, r.randint(0, cap), cap, cap + 3]), r.choice([1, 2, 17, 64])
        window = r.choice([0, 1, 3, r.randint(1, 200), 10 ** 9])
        sinks = r.choice([0, 1, 5, r.randint(0, 100), 10 ** 9]) if window else 0
        parts.key_tiles(min(n, cap), rows, cap, window, sinks, keys, out)
        tiles = [out[1 + i] for i in range(out[0])]
        if n < 0:
            assert not tiles
            continue
        assert tiles == sorted(set(tiles)) and all(t % keys == 0 for t in tiles)
        held = {t + i for t in tiles for i in range(keys)}
        for p in range(min(n, cap), min(n, cap) + rows):
            if p < cap:
                assert held.issuperset(ref.visible(p, window, sinks))
        if n < cap:                                                          # and no tile without a key that some row sees
            seen = {t for p in range(n, min(n + rows, cap)) for t in ref.visible(p, window, sinks)}
            whole = {t // keys for t in seen}
            assert {t // keys for t in tiles} >= whole and len(tiles) <= len(whole) + rows // keys + 1


def test_pieces_of_the_line_and_the_parts_of_units(parts):
    """Every worker's piece cut at units: a unit that one worker has whole is written by it, others by the joining kernel from exactly the places
    that the workers left their parts in."""
    r = random.Random(5)
    out = (C.c_int * 2)()
    for _ in range(500):
        units = [r.choice([1, 2, 7, 100, 1000]) for _ in range(r.randint(1, 60))]
        workers, total = r.choice([1, 3, 148]), sum(units)
        chunk = parts.chunk_of(total, workers)
        begin, starts = 0, []
        for n in units:
            starts.append(begin)
            begin += n
        left = {}
        for w in range(workers):
            at, end = w * chunk, min(total, (w + 1) * chunk)
            first = True
            while at < end:
                u = max(i for i, s in enumerate(starts) if s <= at)
                n = min(end, starts[u] + units[u]) - at
                if n < units[u]:
                    left[(u, w)] = 0 if first else 1
                at, first = at + n, False
        for u, (s, n) in enumerate(zip(starts, units)):
            parts.unit_parts(s, n, chunk, out)
            have = {w: place for (v, w), place in left.items() if v == u}
            if out[0] == out[1]:
                assert not have
            else:
                assert have == {w: parts.part_place(s, w, chunk) for w in range(out[0], out[1] + 1)}


def test_numbers_of_the_line_stay_within_31_bits(parts):
    for total in (0, 1, 147, 148, 149, 2 ** 31 - 1):
        chunk = parts.chunk_of(total, 148)
        assert chunk * 148 >= total and (total == 0 or chunk * 148 - total < 148)
    for units, cap, keys in ((1, 16, 16), (4096, 2 ** 20, 16), (7, 2 ** 31 - 1024, 8), (2 ** 20, 2 ** 31 - 1024, 8)):
        n = parts.line_batch(units, cap, keys)
        most = units * -(-cap // keys)
        assert n * most < 2 ** 31 and (n == 0) == (units * (cap // keys + 1) >= 2 ** 31)


def test_queries_are_divided_exactly(parts):
    for n in list(range(1, 70)) + [128, 255, 512]:
        assert all(parts.quotient16(x, n) == x // n for x in range(0, 65536, 7 if n > 16 else 1))


def _plan(parts, *args):
    out = (C.c_longlong * 8)()
    parts.plan(*args, out)
    return dict(zip(("kind", "queries", "keys", "units", "ctas", "workers", "scratch", "fits"), out))


def test_plans(parts):
    """Kernels and forms: clusters only where they all run at once and no warp has more than four tiles; scratch for the parts of every worker."""
    for batch in (1, 2, 16, 200):
        for hkv in (1, 4, 32, 40):
            for group in (1, 8):
                for c in (1, 5, 16, 64):
                    for hd in (32, 64, 128):
                        for f32 in (0, 1):
                            for cap in (16, 500, 832, 4096, 100000):
                                for window in (0, 64):
                                    p = _plan(parts, batch, c, hkv * group, hkv, hd, f32, cap, window, 4)
                                    nq = group * c
                                    assert p["fits"] and p["units"] == hkv * -(-nq // p["queries"])
                                    assert (p["kind"] == 0) == bool(f32) and (p["kind"] != 2 or (nq > 32 and hd >= 64))
                                    assert p["queries"] in ({0: (1, 8), 1: (8, 16), 2: (128,)}[p["kind"]])
                                    if p["ctas"]:
                                        assert p["kind"] != 2 and batch * p["units"] * p["ctas"] <= 148 and p["scratch"] == 0
                                        assert (min(cap, window + c + 4 + 32) if window else cap) <= p["ctas"] * 8 * 4 * p["keys"]
                                    else:
                                        assert p["scratch"] >= p["workers"] * 2 * 4 * p["queries"] * (hd + 2)
    assert not _plan(parts, 1, 64, 512, 64, 128, 1, 2 ** 30, 0, 0)["fits"]
    # where each of the two bf16 kernels was measured to be the faster one
    for args, kind in (((4, 64, 32, 32, 128, 0, 1064, 0, 0), 2), ((8, 16, 32, 8, 128, 0, 2016, 0, 0), 2), ((16, 16, 32, 4, 64, 0, 4112, 0, 0), 2),
                       ((1, 16, 32, 8, 128, 0, 4016, 0, 0), 1), ((8, 32, 40, 40, 128, 0, 1056, 0, 0), 1), ((1, 16, 32, 4, 64, 0, 657, 0, 0), 1),
                       ((4, 51, 32, 32, 128, 0, 64, 0, 0), 1)):
        assert _plan(parts, *args)["kind"] == kind


def test_workers_of_a_line(parts):
    """Twelve warps per SM where the table may hold ten tiles and more for each of eight, on bf16 only; one CTA per SM with tcgen05."""
    for args, workers in (((1, 1, 32, 4, 64, 0, 32064, 0, 0), 8), ((8, 16, 40, 40, 128, 0, 1056, 0, 0), 12), ((4, 16, 32, 32, 128, 0, 832, 0, 0), 8),
                          ((8, 4, 40, 40, 128, 0, 16032, 2048, 4), 12), ((16, 1, 32, 32, 128, 1, 2064, 0, 0), 8), ((16, 16, 32, 4, 64, 0, 4112, 0, 0), 1)):
        p = _plan(parts, *args)
        assert p["ctas"] == 0 and p["workers"] == 148 * workers
