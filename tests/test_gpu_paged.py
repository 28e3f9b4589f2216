"""The paged K/V cache on the GPU against plain Python in 64 bits: rotation and write, attention with and without a sliding window, and
what manages the pages.  Slots that nobody should read hold NaN."""
import math
import random

import pytest
import torch

import paged_reference as ref
from paper_2311_08263_b200 import engine, lib

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _pools(n_pages, hkv, ps, hd, dtype, order="hnd", fill=math.nan):
    """K and V [pages, kv heads, slots, hd] in one of the layouts: hnd, nhd, K and V taking turns page by page, padded rows."""
    if order == "hnd":
        return [torch.full((n_pages, hkv, ps, hd), fill, dtype=dtype, device="cuda") for _ in range(2)]
    if order == "nhd":
        return [torch.full((n_pages, ps, hkv, hd), fill, dtype=dtype, device="cuda").transpose(1, 2) for _ in range(2)]
    if order == "turns":
        both = torch.full((n_pages, 2, hkv, ps, hd), fill, dtype=dtype, device="cuda")
        return [both[:, 0], both[:, 1]]
    assert order == "padded"
    return [torch.full((n_pages + 1, hkv, ps + 1, hd + 8), fill, dtype=dtype, device="cuda")[1:, :, 1:, 8:] for _ in range(2)]


def _dealt(lens, c, ps, gen, extra=2):
    """A table with slots for lens[b] + c positions, pages in random order, -1 elsewhere; pages of the pool."""
    need = [-(-(n + c) // ps) if n >= 0 else 0 for n in lens]
    ids = torch.randperm(sum(need) + extra, generator=gen).tolist()
    table = torch.full((len(lens), max(max(need), 1) + 1), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = torch.tensor(ids[at:at + n], dtype=torch.int32)
        at += n
    return table, len(ids)


def _cache(lens, c, hkv, hd, ps, dtype, order, seed, window=0, n_sink=0):
    """Pools in which only the slots that some row sees hold numbers; table, lengths."""
    gen = torch.Generator().manual_seed(seed)
    table, n_pages = _dealt(lens, c, ps, gen)
    k, v = _pools(n_pages, hkv, ps, hd, dtype, order)
    for b, n in enumerate(lens):
        if n < 0:
            continue
        t = sorted({i for j in range(c) for i in ref.visible(n + j, window, n_sink)})
        page, slot = table[b, [i // ps for i in t]].long().cuda(), torch.tensor([i % ps for i in t]).cuda()
        for x in (k, v):
            x[page, :, slot] = torch.randn(len(t), hkv, hd, generator=gen).to(dtype).cuda()
    return k, v, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()


def _queries(n, width, dtype, seed):
    return (1.5 * torch.randn(n, width, generator=torch.Generator().manual_seed(seed))).to(dtype).cuda()


def _close(got, want, tol):
    got = got.double().cpu().view_as(want)
    assert torch.equal(got.isnan(), want.isnan())
    fine = ~want.isnan()
    off = ((got - want).abs() - tol)[fine]
    assert off.numel() == 0 or off.max() <= 1e-30, (off.max(), (got - want).abs()[fine].max())


# ---------------------------------------------------------------------------------------------------------------- store
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,hkv,hd,ps,order,c", [
    (4, 4, 32, 16, "hnd", 8), (8, 2, 64, 5, "nhd", 1), (8, 8, 128, 1, "turns", 3), (6, 2, 128, 16, "padded", 64), (32, 4, 64, 64, "hnd", 2)])
def test_store(dtype, hq, hkv, hd, ps, order, c):
    lens = [0, 7, -1, 130, 63, 64]
    gen = torch.Generator().manual_seed(hd + ps)
    table, n_pages = _dealt(lens, c, ps, gen)
    table[4, lens[4] // ps] = -1                                             # a page that is missing
    table[5, lens[5] // ps] = n_pages                                        # and one beyond the pool
    k, v = _pools(n_pages, hkv, ps, hd, DT[dtype], order, 7.0)
    wide = torch.randn(len(lens) * c, (hq + 2 * hkv) * hd + 4, generator=gen).cuda()
    qkv = wide[:, 4:]
    theta = 10000.0
    q = engine.fc_op_paged_store(qkv, k, v, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), c, hq, theta)
    x = qkv.double().cpu().view(len(lens), c, -1, hd)
    want_k, want_v = torch.full((n_pages, hkv, ps, hd), 7.0, dtype=torch.float64), torch.full((n_pages, hkv, ps, hd), 7.0, dtype=torch.float64)
    # a rotated element is two products and a sum of rounded factors: the angle's fraction rounded once (half a step of up to a half turn, times
    # pi), sine and cosine off by 2 steps; then the type's own rounding
    for b, n in enumerate(lens):
        if n < 0:
            continue
        rot = ref.rotated(x[b], range(n, n + c), theta)
        size = x[b].abs()[..., :hd // 2] + x[b].abs()[..., hd // 2:]
        size = torch.cat([size, size], -1)
        half = torch.finfo(DT[dtype]).eps / 2
        tol = size * (math.pi * 2 ** -24 + 6 * 2.0 ** -24) + (rot.abs() + size * 1e-6) * half
        got = q.view(len(lens), c, hq, hd)[b].double().cpu()
        assert ((got - rot[:, :hq]).abs() <= tol[:, :hq]).all()
        for j in range(c):
            page = int(table[b, (n + j) // ps])
            if 0 <= page < n_pages:
                want_k[page, :, (n + j) % ps], want_v[page, :, (n + j) % ps] = rot[j, hq:hq + hkv], x[b, j, hq + hkv:]
                at = (page, slice(None), (n + j) % ps)
                assert ((k[at].double().cpu() - rot[j, hq:hq + hkv]).abs() <= tol[j, hq:hq + hkv]).all()
                assert torch.equal(v[at].cpu(), qkv.view(len(lens), c, -1, hd)[b, j, hq + hkv:].cpu().to(DT[dtype]))
    untouched = want_k == 7.0
    assert (k.double().cpu()[untouched] == 7.0).all() and (v.double().cpu()[want_v == 7.0] == 7.0).all()


def test_store_far_positions():
    """Positions whose angle a 32-bit product would miss by whole radians."""
    hd, n = 128, 2 ** 30 + 12345
    k, v = _pools(2, 1, 1 << 16, hd, torch.float32, fill=0.0)
    width = n // (1 << 16) + 2
    table = torch.full((1, width), -1, dtype=torch.int32)
    table[0, n // (1 << 16)] = 1
    x = torch.randn(2, 3 * hd, generator=torch.Generator().manual_seed(1))
    q = engine.fc_op_paged_store(x.cuda(), k, v, table.cuda(), torch.tensor([n], dtype=torch.int32).cuda(), 2, 1, 1e6)
    want = ref.rotated(x.double().view(2, 3, hd)[:, :1], [n, n + 1], 1e6)
    # a 64-bit product of 2^30 turns is off by 2^-53 x 2^28, and so is the reference's angle
    assert (q.double().cpu().view(2, 1, hd) - want).abs().max() < 4 * (2 ** -24 * 8 + 2 ** -22)
    slot = n % (1 << 16)
    assert torch.equal(v[1, 0, slot].cpu(), x[0, 2 * hd:]) and torch.equal(v[1, 0, slot + 1].cpu(), x[1, 2 * hd:])


# ---------------------------------------------------------------------------------------------------------------- attention
EDGES = [0, 1, 7, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, -1, 260]
ATTENTION = [
    # hq, hkv, hd, c, page, layout, lens, window, sinks
    (4, 4, 32, 8, 16, "hnd", [70], 0, 0),
    (4, 4, 32, 1, 16, "hnd", EDGES, 0, 0),
    (8, 2, 64, 1, 16, "nhd", EDGES, 0, 0),
    (8, 8, 128, 1, 32, "turns", EDGES, 0, 0),
    (8, 1, 64, 5, 24, "padded", EDGES, 0, 0),
    (8, 8, 128, 16, 16, "hnd", [803], 0, 0),
    (32, 4, 64, 16, 64, "hnd", [300, 0, 129], 0, 0),                         # 128 queries per kv head
    (4, 2, 128, 64, 48, "nhd", [200, 1, -1, 77], 0, 0),
    (5, 5, 64, 3, 1, "hnd", [40, 2, 0], 0, 0),                               # a slot per page
    (6, 2, 128, 2, 1000, "hnd", [999, 998, 1000], 0, 0),                     # a sequence per page
    (16, 1, 128, 7, 5, "hnd", [333, 5, 64], 0, 0),                           # 112 queries on one kv head, pages that end inside tiles
    (4, 4, 32, 3, 16, "hnd", EDGES, 1, 0),
    (8, 2, 64, 4, 16, "nhd", EDGES, 20, 4),
    (8, 8, 128, 1, 16, "hnd", [500, 90, 3], 64, 1),
    (4, 1, 128, 16, 8, "hnd", [700, 250], 100, 200),                         # sinks that reach past the window's start in one of them
    (8, 2, 64, 64, 32, "hnd", [400, 10], 33, 5),
    (2, 2, 64, 1, 64, "hnd", [9000], 0, 0),                                  # two heads: split over the length
    (2, 1, 128, 2, 16, "hnd", [5000, 0, 3], 4096, 16),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", range(len(ATTENTION)))
def test_attention(dtype, case):
    hq, hkv, hd, c, ps, order, lens, window, n_sink = ATTENTION[case]
    k, v, table, kv_len = _cache(lens, c, hkv, hd, ps, DT[dtype], order, 100 + case, window, n_sink)
    wide = _queries(len(lens) * c, hq * hd + 8, DT[dtype], case)
    for q in (wide[:, 8:], wide[:, 8:].contiguous()):
        out = engine.fc_op_paged_attention(q, k, v, table, kv_len, c, hq, window=window, n_sink=n_sink)
        _close(out, *ref.attention(q, k, v, table, kv_len, c, hq, window, n_sink))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("seed", range(24))
def test_attention_random_shapes(dtype, seed):
    r = random.Random(seed)
    hkv, group, hd = r.choice([1, 2, 3]), r.choice([1, 2, 3, 8, 13]), r.choice([32, 64, 128])
    c, ps, B = r.choice([1, 1, 2, 5, 16, 33, 64]), r.choice([1, 3, 8, 16, 20, 64, 128]), r.randint(1, 5)
    lens = [r.choice([-1, 0, 1, r.randint(2, 60), r.randint(60, 500)]) for _ in range(B)]
    window = r.choice([0, 0, 1, r.randint(2, 40), r.randint(40, 300)])
    n_sink = r.choice([0, 1, 5, 40])
    k, v, table, kv_len = _cache(lens, c, hkv, hd, ps, DT[dtype], r.choice(["hnd", "nhd", "turns", "padded"]), seed, window, n_sink)
    q = _queries(B * c, hkv * group * hd, DT[dtype], seed)
    out = engine.fc_op_paged_attention(q, k, v, table, kv_len, c, hkv * group, window=window, n_sink=n_sink)
    _close(out, *ref.attention(q, k, v, table, kv_len, c, hkv * group, window, n_sink))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (6, 2)])
def test_later_rows_do_not_reach_earlier_ones(dtype, window, n_sink):
    """Infinities and NaN in the window's later keys and values: rows that do not see them stay as they are, bit for bit."""
    hq, hkv, hd, c, ps, lens = 8, 2, 64, 12, 16, [50, 3, 0]
    k, v, table, kv_len = _cache(lens, c, hkv, hd, ps, DT[dtype], "hnd", 5, window, n_sink)
    q = _queries(len(lens) * c, hq * hd, DT[dtype], 6)
    good = engine.fc_op_paged_attention(q, k, v, table, kv_len, c, hq, window=window, n_sink=n_sink).view(len(lens), c, hq, hd)
    for bad in (math.nan, math.inf, -math.inf):
        for at in (4, 11):
            k2, v2 = k.clone(), v.clone()
            for b, n in enumerate(lens):
                page, slot = int(table[b, (n + at) // ps]), (n + at) % ps
                v2[page, :, slot, ::3] = bad
                if bad != bad:
                    k2[page, :, slot, 5] = bad
            out = engine.fc_op_paged_attention(q, k2, v2, table, kv_len, c, hq, window=window, n_sink=n_sink).view(len(lens), c, hq, hd)
            for j in range(c):
                sees = [at + n in ref.visible(n + j, window, n_sink) for n in lens]
                for b in range(len(lens)):
                    if not sees[b]:
                        assert torch.equal(out[b, j], good[b, j]), (b, j)
                    elif bad != bad:
                        assert out[b, j].isnan().all()
                    else:
                        assert (out[b, j, :, ::3] == bad).all() and out[b, j, :, 1::3].isfinite().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_bad_pages_reach_only_the_rows_that_see_them(dtype):
    hq, hkv, hd, c, ps, lens = 4, 2, 128, 4, 16, [100, 100, 100, 40]
    k, v, table, kv_len = _cache(lens, c, hkv, hd, ps, DT[dtype], "hnd", 8, 40, 2)
    table[0, 2:3] = -1                                                       # positions 32..47: no row sees them
    table[1, 5] = k.shape[0]                                                 # beyond the pool, seen by all rows
    table[2, 6] = 2 ** 31 - 1                                                # the window's own page: positions 96..111
    table[3, 2] = -5                                                         # positions 32..47
    q = _queries(len(lens) * c, hq * hd, DT[dtype], 6)
    out = engine.fc_op_paged_attention(q, k, v, table, kv_len, c, hq, window=40, n_sink=2)
    _close(out, *ref.attention(q, k, v, table, kv_len, c, hq, 40, 2))
    assert out.view(4, -1)[0].isfinite().all() and all(out.view(4, -1)[b].isnan().all() for b in (1, 2, 3))
    # a table that is too short: the rows at positions beyond it
    short = table[3:4, :2].contiguous()
    short[0, 1] = table[3, 1]
    for n in (28, 29, 31, 32, 2 ** 31 - 1):
        lens1 = torch.tensor([n], dtype=torch.int32).cuda()
        k[:], v[:] = 0.5, 0.25
        out = engine.fc_op_paged_attention(q[:c], k, v, short, lens1, c, hq)
        for j in range(c):
            assert out[j].isnan().all() if n + j >= 32 else torch.equal(out[j], torch.full_like(out[j], 0.25))


def test_table_without_sequences():
    k, v = _pools(3, 2, 16, 64, torch.bfloat16)
    table = torch.full((5, 4), -1, dtype=torch.int32).cuda()
    q = _queries(10, 4 * 64, torch.bfloat16, 0)
    out = engine.fc_op_paged_attention(q, k, v, table, torch.full((5,), -1, dtype=torch.int32).cuda(), 2, 4)
    assert torch.equal(out, torch.zeros_like(out))


def test_one_visible_key_is_its_value():
    k, v, table, kv_len = _cache([0, 0], 1, 3, 64, 16, torch.bfloat16, "hnd", 3)
    out = engine.fc_op_paged_attention(_queries(2, 6 * 64, torch.bfloat16, 0), k, v, table, kv_len, 1, 6)
    want = v[table[:, 0].long(), :, 0].float().repeat_interleave(2, 1).view(2, -1)
    assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_scores(dtype):
    """Scores of some thousands: the running maximum keeps the exponentials in range; what is far below it counts as nothing."""
    hq, hkv, hd, c, ps = 2, 2, 128, 2, 16
    k, v, table, kv_len = _cache([300], c, hkv, hd, ps, DT[dtype], "hnd", 3)
    q = _queries(c, hq * hd, DT[dtype], 1) * 300
    out = engine.fc_op_paged_attention(q, k, v, table, kv_len, c, hq)
    _close(out, *ref.attention(q, k, v, table, kv_len, c, hq))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_offsets_beyond_32_bits(dtype):
    """Pages that lie more than 2^32 bytes and 2^31 elements into the pool."""
    hkv, hd, ps, hq = 8, 128, 64, 8
    n_pages = 2 ** 31 // (hkv * hd * ps) + 40
    k, v = (torch.empty(n_pages, hkv, ps, hd, dtype=DT[dtype], device="cuda") for _ in range(2))
    table = torch.tensor([[n_pages - 1, 0, n_pages - 3, n_pages - 2]], dtype=torch.int32).cuda()
    for x in (k, v):
        for p in table[0].tolist():
            x[p] = torch.randn(hkv, ps, hd, generator=torch.Generator().manual_seed(p)).to(DT[dtype]).cuda()
    n = 200
    qkv = torch.randn(1, 3 * hq * hd, generator=torch.Generator().manual_seed(2)).cuda()
    kv_len = torch.tensor([n], dtype=torch.int32).cuda()
    q = engine.fc_op_paged_store(qkv, k, v, table, kv_len, 1, hq, 1e4)
    assert torch.equal(v[n_pages - 2, :, n - 192].cpu(), qkv[0, 2 * hq * hd:].view(hkv, hd).cpu().to(DT[dtype]))
    out = engine.fc_op_paged_attention(q, k, v, table, kv_len, 1, hq)
    few = table[0].long()
    _close(out, *ref.attention(q, k[few], v[few], torch.tensor([[0, 1, 2, 3]]), kv_len, 1, hq))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_slab_of_a_context_is_a_pool(dtype):
    """One page of max_seq slots per sequence: the same as fc_op_window_attention over the slab."""
    B, hkv, max_seq, hd, hq, c = 3, 2, 200, 64, 8, 4
    gen = torch.Generator().manual_seed(4)
    k, v = (torch.randn(B, hkv, max_seq, hd, generator=gen).to(DT[dtype]).cuda() for _ in range(2))
    kv_len = torch.tensor([150, 0, 196], dtype=torch.int32).cuda()
    q = _queries(B * c, hq * hd, DT[dtype], 4)
    table = torch.arange(B, dtype=torch.int32).cuda().view(B, 1)
    out = engine.fc_op_paged_attention(q, k, v, table, kv_len, c, hq)
    want, tol = ref.attention(q, k, v, table, kv_len, c, hq)
    _close(out, want, tol)
    slab = engine.fc_op_window_attention(q, k, v, kv_len, c, hq, 196)
    # that kernel's own error is of the same kind; its probabilities are one bf16 pair as well
    _close(slab, want, 2 * tol + 1e-6)


def test_repeated_and_concurrent_calls_give_the_same_bits():
    cases = []
    for i, (hq, hkv, hd, c, lens, window) in enumerate([(32, 4, 64, 1, [5000], 0), (8, 8, 128, 16, [803, 20], 0), (16, 2, 64, 16, [900, 31, 2], 300)]):
        k, v, table, kv_len = _cache(lens, c, hkv, hd, 16, torch.bfloat16, "hnd", i, window, 3)
        cases.append((_queries(len(lens) * c, hq * hd, torch.bfloat16, i), k, v, table, kv_len, c, hq, window, 3))
    first = [engine.fc_op_paged_attention(*a) for a in cases]
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for s, a in zip(streams, cases):
            with torch.cuda.stream(s):
                got.append(engine.fc_op_paged_attention(*a))
    torch.cuda.synchronize()
    for i, x in enumerate(got):
        assert torch.equal(x, first[i % 3])


# ---------------------------------------------------------------------------------------------------------------- pages
class _Both:
    """The device's pool and its model in Python, compared after every operation."""

    def __init__(self, n_pages, n_seqs, width, ps, order="hnd", dtype=torch.bfloat16, layers=3, hkv=2, hd=64):
        self.model = ref.Pool(n_pages, n_seqs, width, ps)
        # every page of every layer is filled with one number of its own
        self.k, self.v = (torch.stack([x for _ in range(layers)]) for x in _pools(n_pages, hkv, ps, hd, dtype, order))
        if order == "nhd":
            self.k, self.v = (torch.empty(layers, n_pages, ps, hkv, hd, dtype=dtype, device="cuda").transpose(2, 3) for _ in range(2))
        if order == "padded":
            self.k, self.v = (torch.full((layers, n_pages, hkv, ps + 3, hd + 8), 9.0, dtype=dtype, device="cuda")[:, :, :, 1:-2, 8:] for _ in range(2))
        if order == "turns":
            both = torch.empty(n_pages, layers, 2, hkv, ps, hd, dtype=dtype, device="cuda")
            self.k, self.v = both[:, :, 0].transpose(0, 1), both[:, :, 1].transpose(0, 1)
        mark = torch.arange(n_pages, dtype=torch.float32).view(1, -1, 1, 1, 1)
        lay = torch.arange(layers, dtype=torch.float32).view(-1, 1, 1, 1, 1)
        slot = torch.arange(ps, dtype=torch.float32).view(1, 1, 1, -1, 1) % 2
        self.want = lambda m, sign: (sign * (torch.tensor(m, dtype=torch.float32).view(1, -1, 1, 1, 1) + 64 * lay + 0.5 * slot)).expand(
            layers, len(m), hkv, ps, hd).to(dtype)
        for x, sign in ((self.k, 1), (self.v, -1)):
            x.copy_(self.want(list(range(n_pages)), sign).cuda())
        self.table = torch.full((n_seqs, width), -1, dtype=torch.int32).cuda()
        self.kv_len = torch.full((n_seqs,), -1, dtype=torch.int32).cuda()
        self.refs = torch.zeros(n_pages, dtype=torch.int32).cuda()

    def check(self):
        m = self.model
        assert self.table.tolist() == m.table and self.kv_len.tolist() == m.kv_len and self.refs.tolist() == m.refs
        held = [p for p, r in enumerate(m.refs) if r > 0]                     # what free pages hold means nothing
        for x, sign in ((self.k, 1), (self.v, -1)):
            assert torch.equal(x[:, held].cpu(), self.want([m.content[p] for p in held], sign))
        counts = [0] * len(m.refs)
        for row in m.table:
            for p in row:
                if p >= 0:
                    counts[p] += 1
        assert counts == m.refs

    def start(self, s, n):
        self.kv_len[s] = self.model.kv_len[s] = n

    grow = start

    def free(self, seqs, window=0, n_sink=0):
        self.model.free(seqs, window, n_sink)
        engine.fc_op_pages_free(self.table, self.kv_len, self.refs, self.model.ps, seqs, window, n_sink)

    def fork(self, src, dst):
        self.model.fork(src, dst)
        engine.fc_op_pages_fork(self.table, self.kv_len, self.refs, self.model.ps, src, dst)

    def reserve(self, rows):
        want = self.model.reserve(rows)
        got = engine.fc_op_pages_reserve(self.k, self.v, self.table, self.kv_len, self.refs, rows).tolist()
        assert got == want
        return want

    def compact(self):
        want = self.model.compact()
        assert engine.fc_op_pages_compact(self.k, self.v, self.table, self.refs).tolist() == [want]
        self.model.content = list(self.model.content)


@pytest.mark.parametrize("order", ["hnd", "nhd", "padded", "turns"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_fork_and_copy_on_write(order, dtype):
    p = _Both(40, 6, 8, 5, order, DT[dtype])
    p.start(0, 0)
    p.reserve(13)                                                            # pages 0..2
    p.grow(0, 13)
    p.fork([0, 0, 0], [1, 2, 4])
    p.check()
    assert p.model.refs[:3] == [4, 4, 4]
    assert p.reserve(4) == [1, 1, 1, 0, 1, 0]                                # three copies of page 2, the last sequence keeps it
    p.check()
    assert p.model.table[4][2] == 2 and p.model.refs[:3] == [4, 4, 1]
    p.free([0, 1])
    p.check()
    p.fork([2], [4])                                                         # 4 gives up what it held
    p.check()
    p.free([2, 4])
    p.check()
    assert sum(p.model.refs) == 0


@pytest.mark.parametrize("seed", range(6))
def test_random_lives_of_sequences(seed):
    r = random.Random(seed)
    n_seqs, width, ps = r.choice([3, 9, 40]), r.choice([4, 9]), r.choice([1, 3, 8])
    p = _Both(r.choice([12, 30, 64]), n_seqs, width, ps, r.choice(["hnd", "nhd", "padded", "turns"]), layers=2, hkv=1, hd=32)
    for _ in range(40):
        what = r.choice(["start", "fork", "reserve", "reserve", "reserve", "free", "window", "compact"])
        used = [s for s in range(n_seqs) if p.model.kv_len[s] >= 0]
        if what == "start" and len(used) < n_seqs:
            p.start(r.choice([s for s in range(n_seqs) if s not in used]), 0)
        elif what == "fork" and used and n_seqs > 1:
            dst = r.sample(range(n_seqs), r.randint(1, min(3, n_seqs - 1)))
            src = [s for s in range(n_seqs) if s not in dst]
            p.fork([r.choice(src) for _ in dst], dst)
        elif what == "reserve":
            rows = r.choice([1, 2, 7, 20])
            for b, ok in enumerate(p.reserve(rows)):
                if ok:
                    p.grow(b, p.model.kv_len[b] + r.randint(0, rows))
        elif what == "free" and used:
            p.free(r.sample(used, r.randint(1, len(used))))
        elif what == "window" and used:
            p.free(r.sample(used, r.randint(1, len(used))), r.choice([1, 4, 9]), r.choice([0, 1, 4]))
        elif what == "compact":
            p.compact()
        p.check()


def test_reserve_serves_in_order_while_pages_last():
    p = _Both(6, 5, 4, 4)
    for s, n in ((0, 0), (1, 0), (2, -1), (3, 0), (4, 0)):
        p.start(s, n)
    assert p.reserve(8) == [1, 1, 0, 1, 0]                                   # two pages each, six in the pool
    p.check()
    assert p.reserve(8) == [1, 1, 0, 1, 0]
    p.check()
    p.grow(1, 12)
    assert p.reserve(8)[1] == 0                                              # beyond the table
    p.check()


def test_many_pages_and_sequences():
    """More pages, sequences and listed rows than one block has threads."""
    n = 1500
    p = _Both(5000, n, 3, 2, layers=1, hkv=1, hd=32)
    p.start(0, 0)
    p.reserve(3)
    p.grow(0, 3)
    p.fork([0] * (n - 1), list(range(1, n)))
    p.check()
    assert sum(p.reserve(2)) == n
    p.check()
    p.free(list(range(0, n, 2)))
    p.check()
    p.compact()
    p.check()


def test_compact_of_a_compact_pool_and_of_an_empty_one():
    p = _Both(20, 3, 6, 4)
    p.compact()
    p.check()
    p.start(1, 0)
    p.reserve(17)
    p.compact()
    p.check()


# ---------------------------------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_questions_behind_one_prompt(dtype):
    """A prompt cached once and forked, windows of rows stored, some accepted, a sliding window whose old pages are freed, compaction in
    between, the step captured once and replayed as the caches grow: every step as if each sequence had a cache of its own."""
    hq, hkv, hd, ps, c, layers, window, n_sink, theta = 8, 2, 64, 8, 4, 2, 24, 3, 1e4
    n_pages, n_seqs, width = 60, 4, 16
    gen = torch.Generator().manual_seed(9)
    k, v = (torch.full((layers, n_pages, hkv, ps, hd), math.nan, dtype=DT[dtype], device="cuda") for _ in range(2))
    table = torch.full((n_seqs, width), -1, dtype=torch.int32).cuda()
    kv_len = torch.full((n_seqs,), -1, dtype=torch.int32).cuda()
    refs = torch.zeros(n_pages, dtype=torch.int32).cuda()
    qkv = torch.zeros(layers, n_seqs * c, (hq + 2 * hkv) * hd).cuda()
    own = {b: [] for b in range(n_seqs)}                                     # committed rows of each sequence, [layers, width]

    def step():
        served = engine.fc_op_pages_reserve(k, v, table, kv_len, refs, c)
        outs = []
        for i in range(layers):
            q = engine.fc_op_paged_store(qkv[i], k[i], v[i], table, kv_len, c, hq, theta)
            outs.append((q, engine.fc_op_paged_attention(q, k[i], v[i], table, kv_len, c, hq, window=window, n_sink=n_sink)))
        return served, outs

    def check(served, outs):
        for b in range(n_seqs):
            n = int(kv_len[b])
            if n < 0:
                assert all((o.view(n_seqs, -1)[b] == 0).all() for _, o in outs)
                continue
            assert int(served[b]) == 1
            half = torch.finfo(DT[dtype]).eps / 2
            seen = sorted({t for j in range(c) for t in ref.visible(n + j, window, n_sink)})
            page = table[b, [t // ps for t in seen]].long()
            slot = torch.tensor([t % ps for t in seen]).cuda()
            for i in range(layers):
                # what the sequence sees is its own, wherever it lies
                rows = torch.stack([x[i] for x in own[b]] + list(qkv[i].view(n_seqs, c, -1)[b].cpu())).view(n + c, -1, hd)[seen]
                rot = ref.rotated(rows[:, hq:hq + hkv].double(), seen, theta)
                assert ((k[i][page, :, slot].double().cpu() - rot).abs() <= rot.abs() * half + 16 * 2.0 ** -24 * (1 + half)).all()
                assert torch.equal(v[i][page, :, slot].cpu(), rows[:, hq + hkv:].to(DT[dtype]))
                want, tol = ref.attention(outs[i][0].view(n_seqs, c, -1)[b], k[i], v[i], table[b:b + 1], kv_len[b:b + 1], c, hq, window, n_sink)
                _close(outs[i][1].view(n_seqs, c, hq, hd)[b], want, tol)

    kv_len[0] = 0
    r = random.Random(3)

    def advance(served, outs, most):
        check(served, outs)
        lens = kv_len.tolist()
        for b in range(n_seqs):
            if lens[b] >= 0:
                take = r.randint(1, most)
                own[b] += [qkv[:, b * c + j].cpu() for j in range(take)]
                kv_len[b] = lens[b] + take

    for _ in range(8):                                                       # the prompt, up to c rows at a time
        qkv.copy_(torch.randn(qkv.shape, generator=gen))
        advance(*step(), c)
    engine.fc_op_pages_fork(table, kv_len, refs, ps, [0, 0], [1, 3])
    own[1], own[3] = list(own[0]), list(own[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        kept = step()
    for i in range(14):
        qkv.copy_(torch.randn(qkv.shape, generator=gen))
        graph.replay()
        advance(*kept, c)
        if i % 4 == 1:
            engine.fc_op_pages_free(table, kv_len, refs, ps, [b for b in range(n_seqs) if int(kv_len[b]) >= 0], window, n_sink)
        if i % 5 == 2:
            engine.fc_op_pages_compact(k, v, table, refs)
        if i == 6:
            engine.fc_op_pages_free(table, kv_len, refs, ps, [1])
            engine.fc_op_pages_fork(table, kv_len, refs, ps, [3], [2])
            own[2], own[1] = list(own[3]), []
    held = table[table >= 0].tolist()
    assert [held.count(p) for p in range(n_pages)] == refs.tolist()


# ---------------------------------------------------------------------------------------------------------------- many queries per kv head
def _widened(table, ps, cap):
    """The table with columns of -1 for `cap` keys: which kernel a call takes follows from what its table may hold."""
    more = -(-cap // ps) - table.shape[1]
    return torch.cat([table, torch.full((table.shape[0], more), -1, dtype=torch.int32, device="cuda")], 1).contiguous() if more > 0 else table


def _on_tcgen05(k, table, c, hq, window=0, n_sink=0):
    """Whether the call asks for the scratch of the kernel with units of 128 queries: a status word for each of 148 CTAs, two parts of each."""
    hkv, ps, hd = k.shape[1:]
    want = 1024 + 148 * 2 * 128 * (hd + 2) * 4
    return lib.load().fc_op_paged_attention_scratch_bytes(table.shape[0], c, hq, hkv, hd, lib.FC_BF16, table.shape[1], ps, window, n_sink) == want


MANY = [
    # hq, hkv, hd, c, page, layout, lens, window, sinks
    (32, 4, 64, 16, 16, "hnd", EDGES, 0, 0),                                 # units of 128: queries, keys and values by TMA
    (32, 4, 64, 16, 64, "nhd", EDGES, 0, 0),
    (32, 4, 128, 16, 24, "turns", EDGES, 0, 0),
    (32, 4, 128, 16, 8, "padded", EDGES, 0, 0),                              # eight boxes a tile
    (16, 2, 128, 33, 128, "hnd", EDGES, 0, 0),                               # 264 queries, the last unit has eight
    (16, 16, 64, 64, 40, "hnd", [300, 0, -1, 77], 0, 0),                     # one query per row: a box of 128 rows takes the next sequence's too
    (12, 4, 64, 64, 16, "nhd", [300, 0, -1, 77, 1], 0, 0),                   # three: units begin inside rows
    (26, 2, 128, 51, 1000, "hnd", [999, 998, 1000, 0], 0, 0),
    (32, 4, 64, 16, 5, "hnd", EDGES, 0, 0),                                  # keys and values by copies
    (32, 4, 128, 16, 1, "padded", EDGES, 0, 0),
    (20, 4, 128, 64, 20, "turns", [200, 1, -1, 77], 0, 0),
    (32, 4, 64, 16, 16, "hnd", [900] + EDGES, 130, 5),
    (32, 4, 128, 16, 48, "nhd", [900] + EDGES, 1, 0),
    (16, 2, 128, 64, 20, "hnd", [700, 3, 65], 100, 200),
    (8, 4, 64, 64, 8, "hnd", [700, 250, 5], 33, 0),
]


@pytest.mark.parametrize("case", range(len(MANY)))
def test_many_queries(case):
    hq, hkv, hd, c, ps, order, lens, window, n_sink = MANY[case]
    k, v, table, kv_len = _cache(lens, c, hkv, hd, ps, torch.bfloat16, order, 200 + case, window, n_sink)
    rep = -(-320 // (len(lens) * hkv)) if window else 1                      # under a window the table's bound says little: the same sequences again
    table = _widened(table, ps, 40000)
    B = len(lens)
    assert _on_tcgen05(k, table.repeat(rep, 1), c, hq, window, n_sink)
    wide = _queries(B * c, hq * hd + 8, torch.bfloat16, case)
    for q in (wide[:, 8:], wide[:, 8:].contiguous()):
        want = ref.attention(q, k, v, table, kv_len, c, hq, window, n_sink)
        q = wide.repeat(rep, 1)[:, 8:] if q.stride(0) > q.shape[1] else q.repeat(rep, 1)
        out = engine.fc_op_paged_attention(q, k, v, table.repeat(rep, 1), kv_len.repeat(rep), c, hq, window=window, n_sink=n_sink)
        _close(out, *(x.repeat(rep, 1, 1) for x in want))


@pytest.mark.parametrize("hd,ps", [(64, 16), (64, 20), (128, 64), (128, 9)])
def test_many_queries_and_long_lines(hd, ps):
    """Some forty tiles per CTA and several units of each: every stage of the rings is used many times, units end and begin inside a piece."""
    hq, hkv, c, lens = 64, 8, 16, [3000, 2999, 64, 0, 1500, 1, 700, 2048, 127, 63, 2400, 5, -1, 1900, 1000, 2500]
    gen = torch.Generator().manual_seed(hd)
    table, n_pages = _dealt(lens, c, ps, gen)
    k, v = (torch.randn(n_pages, hkv, ps, hd, generator=gen).to(torch.bfloat16).cuda() for _ in range(2))
    table, kv_len = table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    q = _queries(len(lens) * c, hq * hd, torch.bfloat16, 1)
    assert _on_tcgen05(k, table, c, hq)
    out = engine.fc_op_paged_attention(q, k, v, table, kv_len, c, hq)
    _close(out, *ref.attention(q, k, v, table, kv_len, c, hq))


@pytest.mark.parametrize("hd,ps", [(64, 16), (64, 5), (128, 24), (128, 7)])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (6, 2)])
def test_many_queries_later_rows_do_not_reach_earlier_ones(hd, ps, window, n_sink):
    hq, hkv, c, lens = 64, 4, 12, [150, 3, 0, 63, 64, 500] * 14              # 192 queries per kv head
    k, v, table, kv_len = _cache(lens, c, hkv, hd, ps, torch.bfloat16, "hnd", 5, window, n_sink)
    table = _widened(table, ps, 5000)
    q = _queries(len(lens) * c, hq * hd, torch.bfloat16, 6)
    good = engine.fc_op_paged_attention(q, k, v, table, kv_len, c, hq, window=window, n_sink=n_sink).view(len(lens), c, hq, hd)
    assert _on_tcgen05(k, table, c, hq, window, n_sink)
    tab = table.tolist()
    for bad in (math.nan, math.inf, -math.inf):
        for at in (4, 11):
            k2, v2 = k.clone(), v.clone()
            for b, n in enumerate(lens):
                page, slot = tab[b][(n + at) // ps], (n + at) % ps
                v2[page, :, slot, ::3] = bad
                if bad != bad:
                    k2[page, :, slot, 5] = bad
            out = engine.fc_op_paged_attention(q, k2, v2, table, kv_len, c, hq, window=window, n_sink=n_sink).view(len(lens), c, hq, hd)
            for j in range(c):
                for b, n in enumerate(lens):
                    if at + n not in ref.visible(n + j, window, n_sink):
                        assert torch.equal(out[b, j], good[b, j]), (b, j)
                    elif bad != bad:
                        assert out[b, j].isnan().all()
                    else:
                        assert (out[b, j, :, ::3] == bad).all() and out[b, j, :, 1::3].isfinite().all()


@pytest.mark.parametrize("hd,ps", [(64, 16), (128, 16), (64, 20), (128, 64)])
def test_many_queries_and_bad_pages(hd, ps):
    hq, hkv, c, lens = 32, 4, 16, [390, 400, 400, 140, 0, 60]
    k, v, table, kv_len = _cache(lens, c, hkv, hd, ps, torch.bfloat16, "hnd", 8)
    table[0, 400 // ps] = -1                                                 # in the window: the rows from there on, where a page begins there
    table[1, 5] = k.shape[0]
    table[2, 0] = 2 ** 31 - 1
    table[3, 160 // ps + 1] = -5                                             # no row sees it
    table[5, (60 + 8) // ps] = -1
    table = _widened(table, ps, 40000)
    q = _queries(len(lens) * c, hq * hd, torch.bfloat16, 6)
    assert _on_tcgen05(k, table, c, hq)
    out = engine.fc_op_paged_attention(q, k, v, table, kv_len, c, hq)
    want, tol = ref.attention(q, k, v, table, kv_len, c, hq)
    rows = want.view(len(lens), c, -1).isnan().all(2).sum(1).tolist()
    assert rows[:3] == [c if ps == 64 else 6, c, c] and rows[3:] == [0, 0, c if ps == 20 else 12]
    assert not want.view(len(lens), -1)[3:5].isnan().any()
    _close(out, want, tol)


def test_many_queries_and_offsets_beyond_32_bits():
    hkv, hd, ps, hq, c, n = 8, 128, 64, 64, 16, 230
    n_pages = 2 ** 31 // (hkv * hd * ps) + 40
    k, v = (torch.empty(n_pages, hkv, ps, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.tensor([[n_pages - 1, 0, n_pages - 3, n_pages - 2]], dtype=torch.int32).cuda()
    for x in (k, v):
        for p in table[0].tolist():
            x[p] = torch.randn(hkv, ps, hd, generator=torch.Generator().manual_seed(p)).to(torch.bfloat16).cuda()
    kv_len = torch.tensor([n], dtype=torch.int32).cuda()
    wide = _widened(table, ps, 40000)
    q = _queries(c, hq * hd, torch.bfloat16, 3)
    assert _on_tcgen05(k, wide, c, hq)
    out = engine.fc_op_paged_attention(q, k, v, wide, kv_len, c, hq)
    few = table[0].long()
    _close(out, *ref.attention(q, k[few], v[few], torch.tensor([[0, 1, 2, 3]]), kv_len, c, hq))


def test_many_queries_captured_and_on_two_streams():
    """The same bits from calls on two streams at once and from a graph that is replayed with other lengths, as from calls one by one."""
    cases = []
    for i, (hq, hkv, hd, ps) in enumerate([(32, 4, 64, 16), (64, 8, 128, 20)]):
        lens = [1200, 40, 900, 0, 641, 64, 300, 2]
        k, v, table, kv_len = _cache(lens, 16, hkv, hd, ps, torch.bfloat16, "hnd", i)
        k, v = (torch.nan_to_num(x) for x in (k, v))
        cases.append((_queries(len(lens) * 16, hq * hd, torch.bfloat16, i), k, v, _widened(table, ps, 40000), kv_len, 16, hq))
        assert _on_tcgen05(k, cases[-1][3], 16, hq)
    first = [engine.fc_op_paged_attention(*a) for a in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for s, a in zip(streams, cases):
            with torch.cuda.stream(s):
                got.append(engine.fc_op_paged_attention(*a))
    torch.cuda.synchronize()
    assert all(torch.equal(x, first[i % 2]) for i, x in enumerate(got))
    graphs, outs = [], []
    for a in cases:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(engine.fc_op_paged_attention(*a))
    shorter = [a[4] // 3 for a in cases]
    want = [engine.fc_op_paged_attention(*a[:4], n, *a[5:]) for a, n in zip(cases, shorter)]
    for a, n in zip(cases, shorter):
        a[4].copy_(n)
    torch.cuda.synchronize()
    for _ in range(3):                                                       # both graphs at once
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(outs, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,c", [(2, 1), (8, 2), (16, 8)])
def test_tables_of_more_tiles_than_one_launch_counts(dtype, hq, c):
    """Pages of 2^20 slots, 2^10 of them to a sequence: tiles are counted in 31 bits, so that the sequences are dealt out to several launches."""
    hkv, hd, ps, B = 1, 64, 1 << 20, 400
    k, v = _pools(2, hkv, ps, hd, DT[dtype])
    for x in (k, v):
        x[:, :, :260] = torch.randn(2, hkv, 260, hd, generator=torch.Generator().manual_seed(2)).to(DT[dtype]).cuda()
    table = torch.full((B, 1 << 10), -1, dtype=torch.int32).cuda()
    table[:, 0] = torch.arange(B, dtype=torch.int32).cuda() % 2
    kv_len = torch.tensor([(7 * b) % 250 - 1 for b in range(B)], dtype=torch.int32).cuda()
    q = _queries(B * c, hq * hd, DT[dtype], 1)
    if dtype == "bf16" and hq * c > 32:
        assert _on_tcgen05(k, table, c, hq)
    out = engine.fc_op_paged_attention(q, k, v, table, kv_len, c, hq)
    _close(out, *ref.attention(q, k, v, table, kv_len, c, hq))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd,ps,c", [(64, 16, 8), (128, 24, 16), (32, 5, 3), (128, 16, 2)])
def test_rows_of_long_lines_keep_their_bits(dtype, hd, ps, c):
    """A value that is not finite in the last key of the window: earlier rows have the same bits where it meets sums of earlier tiles too."""
    hq, hkv, lens = 4, 4, [701, 640, 655, 3, 320] * 8
    k, v, table, kv_len = _cache(lens, c, hkv, hd, ps, DT[dtype], "hnd", 7)
    q = _queries(len(lens) * c, hq * hd, DT[dtype], 6)
    good = engine.fc_op_paged_attention(q, k, v, table, kv_len, c, hq).view(len(lens), c, hq, hd)
    tab = table.tolist()
    for b, n in enumerate(lens):
        v[tab[b][(n + c - 1) // ps], :, (n + c - 1) % ps, ::3] = math.inf
    out = engine.fc_op_paged_attention(q, k, v, table, kv_len, c, hq).view(len(lens), c, hq, hd)
    assert torch.equal(out[:, :-1], good[:, :-1]) and (out[:, -1, :, ::3] == math.inf).all()
    fine = torch.arange(hd).cuda() % 3 != 0
    assert torch.allclose(out[:, -1][..., fine], good[:, -1][..., fine], rtol=0, atol=1e-5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,c,n,width", [(2, 1, 40, 3), (2, 1, 9000, 600), (16, 2, 300, 30), (8, 16, 300, 2500)])
def test_infinite_scores(dtype, hq, c, n, width):
    """Scores of minus infinity weigh nothing; a row that sees no other is NaN, and so is one that sees plus infinity."""
    hkv, hd, ps = 2, 64, 16
    k, v, table, kv_len = _cache([n] * 3, c, hkv, hd, ps, DT[dtype], "hnd", 3)
    table = _widened(table, ps, width * ps)
    q = _queries(3 * c, hq * hd, DT[dtype], 1).abs() + 0.1
    live = (n + c - 1) // ps + 1
    fine = k.clone()
    for page in table[0, :live].tolist():                                    # every key of the first sequence
        k[page, :, :, 3] = -math.inf
    k[table[1, 0].item(), :, 5, 3] = -math.inf                                # one key of the second
    k[table[2, 0].item(), 1, 5, 3] = math.inf                                # one key of one head of the third
    out = engine.fc_op_paged_attention(q, k, v, table, kv_len, c, hq).view(3, c, hkv, -1)
    want, tol = ref.attention(q, k, v, table, kv_len, c, hq)
    want, tol = want.view(3, c, hkv, -1), tol.view(3, c, hkv, -1)
    assert want[0].isnan().all() and want[2, :, 1].isnan().all() and not want[1].isnan().any() and not want[2, :, 0].isnan().any()
    assert torch.equal(out.isnan().cpu(), want.isnan())
    # the bound from finite scores, twice, because the other keys weigh more without that one
    _, tol = ref.attention(q, fine, v, table, kv_len, c, hq)
    assert ((out[1].double().cpu() - want[1]).abs() <= 2 * tol.view(3, c, hkv, -1)[1]).all()


def test_a_single_row_may_have_any_stride():
    k, v, table, kv_len = _cache([20], 1, 2, 64, 16, torch.float32, "hnd", 3)
    q = _queries(1, 4 * 64, torch.float32, 0)
    odd = q.as_strided((1, 256), (1, 1))
    a, b = (engine.fc_op_paged_attention(x, k, v, table, kv_len, 1, 4) for x in (q, odd))
    assert torch.equal(a, b)
    qkv = torch.randn(1, 8 * 64, generator=torch.Generator().manual_seed(1)).cuda()
    a, b = (engine.fc_op_paged_store(x, k, v, table, kv_len, 1, 4, 1e4) for x in (qkv, qkv.as_strided((1, 512), (3, 1))))
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_follows_a_line_of_whole_units_reads_its_results(dtype):
    """As many units of one length as there are workers: each is whole, nothing is joined, and the next kernel of the stream finds them done."""
    B, hkv, hd, ps, n = 37, 32, 64, 64, 2047
    k, v = (torch.randn(n // ps + 1, hkv, ps, hd, generator=torch.Generator().manual_seed(3)).to(DT[dtype]).cuda() for _ in range(2))
    table = torch.arange(n // ps + 1, dtype=torch.int32).cuda().repeat(B, 1)                    # one prompt, read by all
    kv_len = torch.full((B,), n, dtype=torch.int32).cuda()
    q = _queries(B, hkv * hd, DT[dtype], 1)
    for _ in range(5):
        torch.full((B, hkv * hd), math.nan, device="cuda")                                       # the memory that the result gets
        out = engine.fc_op_paged_attention(q, k, v, table, kv_len, 1, hkv)
        copy = out + 0
        torch.cuda.synchronize()
        assert torch.equal(copy, out) and out.isfinite().all()


def test_copies_beyond_32_bits():
    """Copy on write between pages, and compaction of pages, that lie more than 2^32 bytes and 2^31 elements into a layer."""
    hkv, hd, ps, layers = 8, 128, 64, 2
    n = 2 ** 31 // (hkv * hd * ps) + 40
    k, v = (torch.empty(layers, n, hkv, ps, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    fill = {p: torch.randn(2, layers, hkv, ps, hd, generator=torch.Generator().manual_seed(p)).to(torch.bfloat16).cuda() for p in (0, n - 3, n - 2)}
    for p, x in fill.items():
        k[:, p], v[:, p] = x[0], x[1]
    table = torch.tensor([[n - 2, -1], [n - 2, -1], [0, n - 3]], dtype=torch.int32).cuda()
    kv_len = torch.tensor([10, 10, 70], dtype=torch.int32).cuda()
    refs = torch.ones(n, dtype=torch.int32).cuda()
    refs[n - 2], refs[n - 1] = 2, 0                                          # the only free page is the last
    assert engine.fc_op_pages_reserve(k, v, table, kv_len, refs, 1).tolist() == [1, 1, 1]
    assert table.tolist() == [[n - 1, -1], [n - 2, -1], [0, n - 3]] and refs[n - 3:].tolist() == [1, 1, 1]
    for x, y in ((k, fill[n - 2][0]), (v, fill[n - 2][1])):
        assert torch.equal(x[:, n - 1], y)
    refs.zero_()
    refs[0], refs[n - 3:] = 1, 1
    assert engine.fc_op_pages_compact(k, v, table, refs).tolist() == [4]
    assert table.tolist() == [[3, -1], [2, -1], [0, 1]] and refs[:4].tolist() == [1] * 4 and refs[4:].sum() == 0
    for p, at in ((0, 0), (n - 3, 1), (n - 2, 2), (n - 2, 3)):
        assert torch.equal(k[:, at], fill[p][0]) and torch.equal(v[:, at], fill[p][1])


MORE = [
    # hq, hkv, hd, c, page, layout, lens, window, sinks: up to 32 queries per kv head over tables that may hold much
    (4, 4, 32, 8, 16, "hnd", EDGES, 0, 0),
    (8, 2, 32, 7, 5, "padded", EDGES, 0, 0),
    (8, 2, 64, 1, 16, "nhd", EDGES, 0, 0),
    (8, 2, 64, 5, 24, "turns", EDGES, 0, 0),
    (8, 8, 128, 1, 32, "turns", EDGES, 0, 0),
    (8, 8, 128, 16, 16, "hnd", EDGES, 0, 0),
    (6, 2, 128, 9, 1000, "nhd", [999, 998, 1000, 0, -1], 0, 0),
    (8, 2, 64, 4, 16, "nhd", EDGES, 20, 4),
    (8, 8, 128, 2, 7, "hnd", [500, 90, 3], 64, 1),
    (4, 4, 32, 3, 16, "hnd", EDGES, 1, 0),
]


@pytest.mark.parametrize("case", range(len(MORE)))
def test_lines_of_more_warps(case):
    hq, hkv, hd, c, ps, order, lens, window, n_sink = MORE[case]
    k, v, table, kv_len = _cache(lens, c, hkv, hd, ps, torch.bfloat16, order, 300 + case, window, n_sink)
    rep = -(-8000 // (len(lens) * hkv)) if window else 1                     # under a window: the same sequences again
    table = table if window else _widened(table, ps, 1 << 17)
    queries = 8 if hq // hkv * c <= 8 else 16
    want = 256 + 148 * 12 * 2 * queries * (hd + 2) * 4                       # the scratch of twelve warps per SM
    assert lib.load().fc_op_paged_attention_scratch_bytes(len(lens) * rep, c, hq, hkv, hd, lib.FC_BF16, table.shape[1], ps, window, n_sink) == want
    q = _queries(len(lens) * c, hq * hd, torch.bfloat16, case)
    res = ref.attention(q, k, v, table, kv_len, c, hq, window, n_sink)
    out = engine.fc_op_paged_attention(q.repeat(rep, 1), k, v, table.repeat(rep, 1), kv_len.repeat(rep), c, hq, window=window, n_sink=n_sink)
    _close(out, *(x.repeat(rep, 1, 1) for x in res))


@pytest.mark.parametrize("hd,ps,c", [(64, 16, 8), (128, 24, 16), (32, 5, 3)])
def test_lines_of_more_warps_and_long_pieces(hd, ps, c):
    """Rings used many times, units that end inside pieces; and a value that is not finite in the window's last row."""
    hq, hkv, lens = 4, 4, [1500, 1400, 655, 3, 0, 900, 1111, 64] * 10
    gen = torch.Generator().manual_seed(hd)
    table, n_pages = _dealt(lens, c, ps, gen)
    k, v = (torch.randn(n_pages, hkv, ps, hd, generator=gen).to(torch.bfloat16).cuda() for _ in range(2))
    table, kv_len = table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    q = _queries(len(lens) * c, hq * hd, torch.bfloat16, 1)
    good = engine.fc_op_paged_attention(q, k, v, table, kv_len, c, hq)
    _close(good, *ref.attention(q, k, v, table, kv_len, c, hq))
    tab = table.tolist()
    for b, n in enumerate(lens):
        v[tab[b][(n + c - 1) // ps], :, (n + c - 1) % ps, ::3] = math.nan
    out = engine.fc_op_paged_attention(q, k, v, table, kv_len, c, hq).view(len(lens), c, -1, hd)
    assert torch.equal(out[:, :-1], good.view(out.shape)[:, :-1]) and out[:, -1, :, ::3].isnan().all() and out[:, -1, :, 1::3].isfinite().all()
