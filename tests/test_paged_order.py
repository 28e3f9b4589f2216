"""Attention over pages on tcgen05 where tiles are loaded by copies: who waits for what, without a GPU.  The roles of the kernel as coroutines on barriers that know
no more than theirs do, in many orders."""
import ctypes as C
import random
import subprocess

import pytest

from paper_2311_08263_b200 import build


@pytest.fixture(scope="module")
def query_copier(tmp_path_factory):
    d = tmp_path_factory.mktemp("copier")
    src, so = d / "wrap.cpp", d / "wrap.so"
    src.write_text('#include "fc_paged.h"\nextern "C" int query_copier(int tile) { return fc::query_copier(tile); }\n')
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", build.CSRC, "-I", build.INCLUDE, str(src), "-o", str(so)])
    return C.CDLL(str(so)).query_copier


class _Barrier:
    """A barrier of as many arrivals as `count`; a wait names only the parity of the phase that it waits for."""

    def __init__(self, count=1):
        self.count, self.left, self.phase = count, count, 0

    def arrive(self):
        self.left -= 1
        if self.left == 0:
            self.phase, self.left = self.phase + 1, self.count

    def over(self, parity):
        return self.phase & 1 != parity


def _copy_form(segments, stages, apart, query_copier, r, lazy):
    """Tiles and queries of `segments` (tiles of each) through the rings of k_paged_umma.cu's copy form, its roles taking turns at random, those of `lazy` only where
    nobody else can go on.  Asserts that every product finds its own tile and queries and that all of them are made."""
    owner = [s for s, n in enumerate(segments) for _ in range(n)]
    n, first = len(owner), {sum(segments[:s]): s for s in range(len(segments))}
    last = {i for i in range(n) if i + 1 == n or owner[i + 1] != owner[i]}
    bars = lambda k: [_Barrier() for _ in range(k)]
    k_full, v_full, k_empty, v_empty = bars(stages), bars(stages), bars(stages), bars(stages)
    q_full, q_free, s_ready, s_free, p_ready, o_ready = (bars(2) for _ in range(6))
    tile, queries, products, scores, sums, keys_done = [None] * stages, [None, None], [], [], [], [0] * len(segments)

    def load_queries(so):
        if so >= 2:
            yield q_free[so & 1], (so >> 1) - 1 & 1
            assert keys_done[so - 2] == segments[so - 2], "queries overwritten in front of their products"
        assert q_full[so & 1].phase == so >> 1, "queries out of order"
        queries[so & 1] = so
        yield
        q_full[so & 1].arrive()

    def copies(lw):
        pending = None

        def landed():
            nonlocal pending
            if pending is not None:
                k_full[pending].arrive()
                v_full[pending].arrive()
            pending = None

        def step(i):
            if i in first and lw == query_copier(i):
                landed()
                yield from load_queries(first[i])

        if lw == query_copier(0):
            yield from load_queries(0)
        for i in range(1, min(lw + 1, n)):
            yield from step(i)
        for i in range(lw, n, 2):
            st = i % stages
            if i >= stages:
                for bar in (k_empty[st], v_empty[st]):
                    if not bar.over(i // stages - 1 & 1):
                        landed()
                        yield bar, i // stages - 1 & 1
            tile[st] = i
            yield
            landed()
            pending = st
            for t in range(i + 1, min(i + 3, n)):
                yield from step(t)
        landed()

    def issue_scores():
        for i in range(n):
            if i in first:
                yield q_full[owner[i] & 1], owner[i] >> 1 & 1
            yield k_full[i % stages], i // stages & 1
            if i >= 2:
                yield (s_free if apart else o_ready)[i & 1], (i - 2 >> 1) & 1
            products.append(("scores", i))

    def issue_sums():
        for i in range(n):
            yield v_full[i % stages], i // stages & 1
            yield p_ready[i & 1], i >> 1 & 1
            products.append(("sums", i))

    def tensor_core():
        while len(sums) < n:
            if not products:
                yield
                continue
            kind, i = products.pop(0)
            assert tile[i % stages] == i
            if kind == "scores":
                assert queries[owner[i] & 1] == owner[i], "another segment's queries"
                scores.append(i)
                keys_done[owner[i]] += 1
                s_ready[i & 1].arrive()
                k_empty[i % stages].arrive()
                if i in last:
                    q_free[owner[i] & 1].arrive()
            else:
                sums.append(i)
                o_ready[i & 1].arrive()
                v_empty[i % stages].arrive()
            yield

    def softmax(w):
        for i in range(w, n, 2):
            yield s_ready[w], i >> 1 & 1
            yield v_full[i % stages], i // stages & 1
            if i >= 2:
                yield o_ready[w], (i - 2 >> 1) & 1
            s_free[w].arrive()
            yield
            p_ready[w].arrive()

    roles = {"copies 0": copies(0), "copies 1": copies(1), "scores": issue_scores(), "sums": issue_sums(), "tensor": tensor_core(), "softmax 0": softmax(0),
             "softmax 1": softmax(1)}
    wait, idle = dict.fromkeys(roles), 0
    while roles:
        ready = [x for x in roles if wait[x] is None or wait[x][0].over(wait[x][1])]
        eager = [x for x in ready if x not in lazy]
        before = (len(roles), len(products), len(scores), len(sums), [b.phase for b in k_full + v_full + q_full + p_ready])
        x = r.choice(eager if eager and idle < 40 else ready)
        try:
            wait[x] = next(roles[x])
        except StopIteration:
            del roles[x]
        idle = 0 if before != (len(roles), len(products), len(scores), len(sums), [b.phase for b in k_full + v_full + q_full + p_ready]) else idle + 1
        assert idle < 2000, "nobody can go on"
    assert scores == sums == list(range(n))


@pytest.mark.parametrize("stages,apart", [(8, True), (4, False)])             # hd 64, hd 128
def test_queries_of_short_segments_wait_for_the_products_in_front(stages, apart, query_copier):
    """Segments of a few tiles, whose first tiles fall to either copying warp: no queries are overwritten in front of their products, in any order of the roles."""
    _copy_form([1, 2, 2, 1], stages, apart, query_copier, random.Random(0), ("scores", "tensor"))
    r = random.Random(stages)
    for k in range(400):
        segments = [r.choice([1, 1, 2, 2, 3, 4, 9]) for _ in range(r.randint(1, 14))]
        lazy = r.choice([(), ("scores", "tensor"), ("tensor",), ("copies 0",), ("copies 1",), ("softmax 0", "softmax 1"), ("scores", "tensor", "copies 1")])
        _copy_form(segments, stages, apart, query_copier, random.Random(k), lazy)
