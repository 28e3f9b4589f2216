"""The paged key/value cache as cases that can be timed: window attention over pages (with and without a sliding window), the
rotation and K/V write into pages, copy on write behind a fork, and compaction.

With `own` false every operator runs in its plain form, elementary torch operations in 32 bits; with `own` true as the calls of
`paper_2311_08263_b200.engine` that a user makes.

A case is a dict: `op`, `model` (a key of MODELS: query heads, kv heads, head size and layers of the shapes that the decoder runs),
`dtype`, `page` (slots per page) and, by op, what follows.

  attention  `batch` sequences of up to `length` cached tokens, `c` window rows each; `window` / `sinks`: sliding window (0: all keys);
             `order`: how a page is laid out, "hnd" (kv head, slot) or "nhd" (slot, kv head)
  store      the QKV rows of `batch` windows of `c` rows on their way into pages, at positions up to `length`
  fork       `parents` prompts of up to `length` tokens, `children` questions behind each: the children's pages are freed, the prompt is
             forked to them, and `c` window rows are reserved for every sequence (copy on write of the last prompt page), all layers
  compact    a pool with `live` pages in use, `moves` of them beyond the first `live`, all layers

Sequences of a batch have different lengths; the pages of a pool are dealt in random order.
"""
import math

import torch

own = False

# query heads, kv heads, head size, layers
MODELS = {"tiny": (4, 4, 32, 2), "1b": (32, 4, 64, 22), "7b": (32, 32, 128, 32), "13b": (40, 40, 128, 40)}
THETA = 10000.0


def listed():
    return [
        # the fp32 shape in the middle of a generation: the smallest call, latency
        dict(name="attn-tiny-c8", op="attention", model="tiny", dtype="f32", batch=1, c=8, length=70, page=16, window=0, sinks=0, order="hnd"),
        # one user, plain decoding behind a very long context: four kv heads, so the work is split over the cache's length
        dict(name="attn-1b-c1-long", op="attention", model="1b", dtype="bf16", batch=1, c=1, length=31999, page=64, window=0, sinks=0, order="hnd"),
        # one user, the window of the paper's experiments behind a few-shot prompt
        dict(name="attn-7b-c16", op="attention", model="7b", dtype="bf16", batch=1, c=16, length=803, page=16, window=0, sinks=0, order="hnd"),
        # a batch decoded autoregressively, small pages with the slots outermost
        dict(name="attn-7b-b16-c1", op="attention", model="7b", dtype="bf16", batch=16, c=1, length=2048, page=16, window=0, sinks=0, order="nhd"),
        # a batch of windows on grouped heads: 128 queries for every key
        dict(name="attn-1b-b16-c16", op="attention", model="1b", dtype="bf16", batch=16, c=16, length=4096, page=32, window=0, sinks=0, order="hnd"),
        # a few users, long rationales under a sliding window with sinks; pages that nothing sees any more are gone
        dict(name="attn-13b-b8-sliding", op="attention", model="13b", dtype="bf16", batch=8, c=4, length=15999, page=24, window=2048, sinks=4, order="hnd"),
        # the K/V of one row per sequence
        dict(name="store-1b-b8-c1", op="store", model="1b", dtype="bf16", batch=8, c=1, length=2048, page=16),
        # the rows of the largest shape's serving batch
        dict(name="store-13b-b8-c32", op="store", model="13b", dtype="bf16", batch=8, c=32, length=31000, page=64),
        # one prompt, three questions
        dict(name="fork-1b-3", op="fork", model="1b", dtype="bf16", parents=1, children=3, length=513, c=1, page=16),
        # two prompts, eight questions behind each
        dict(name="fork-7b-16", op="fork", model="7b", dtype="bf16", parents=2, children=8, length=803, c=16, page=32),
        # a small pool tidied up
        dict(name="compact-1b", op="compact", model="1b", dtype="bf16", live=90, moves=11, page=16),
        # a server's pool after many requests have ended
        dict(name="compact-7b", op="compact", model="7b", dtype="bf16", live=300, moves=130, page=16),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    dearest = {}
    for c in listed():
        for k, v in work(c).items():
            dearest[c["op"], k] = max(dearest.get((c["op"], k), 0), v)
    while True:
        op = rng.choice(["attention", "attention", "attention", "store", "fork", "compact"])
        case = dict(op=op, model=rng.choice(["tiny", "1b", "1b", "7b", "7b", "13b"]), page=rng.choice([1, 5, 8, 16, 16, 24, 32, 64, 100, 128, 256]))
        case["dtype"] = "f32" if case["model"] == "tiny" or rng.random() < 0.15 else "bf16"
        if op == "attention":
            case.update(batch=_log_int(rng, 1, 64), c=_log_int(rng, 1, 64), length=_log_int(rng, 1, 32000), order=rng.choice(["hnd", "nhd"]))
            sliding = rng.random() < 0.4
            case.update(window=_log_int(rng, 1, 4096) if sliding else 0, sinks=rng.choice([0, 1, 4, 16]) if sliding else 0)
            hq, hkv, hd, _ = MODELS[case["model"]]
            keys = case["batch"] * (case["length"] + case["c"] + case["page"])
            # what the plain form holds: keys and values in 32 bits, scores
            if keys * hkv * hd * 8 + 3 * keys * hq * case["c"] * 4 > 16e9:
                continue
        elif op == "store":
            case.update(batch=_log_int(rng, 1, 32), c=_log_int(rng, 1, 64), length=_log_int(rng, 1, 32000))
        elif op == "fork":
            case.update(parents=_log_int(rng, 1, 8), children=_log_int(rng, 1, 16), length=_log_int(rng, 1, 1500), c=_log_int(rng, 1, 64))
            case["page"] = max(8, case["page"])
        else:
            case["live"] = _log_int(rng, 8, 600)
            case["moves"] = rng.randint(1, case["live"] // 2)
            case["page"] = max(8, case["page"])
        if op in ("fork", "compact") and _pool_bytes(case) > 8e9:
            continue
        if all(v <= dearest[op, k] for k, v in work(case).items()):
            return case


def _es(case):
    return 4 if case["dtype"] == "f32" else 2


def _lengths(case, n):
    """Different lengths for n sequences, the first the longest."""
    m = case["length"]
    return [m - (i * 61) % (m // 4 + 1) for i in range(n)]


def _visible(case):
    """(visible (row, key) pairs, keys that some row sees) over all sequences."""
    pairs = keys = 0
    w, sinks, c = case["window"], case["sinks"], case["c"]
    for m in _lengths(case, case["batch"]):
        for j in range(c):
            p = m + j
            first = max(0, p - w + 1) if w else 0
            pairs += p + 1 - first + min(sinks if w else 0, first)
        first = max(0, m - w + 1) if w else 0
        keys += m + c - first + min(sinks if w else 0, first)
    return pairs, keys


def _page_bytes(case):
    """Bytes of one page over all layers, keys and values."""
    _, hkv, hd, layers = MODELS[case["model"]]
    return 2 * layers * hkv * case["page"] * hd * _es(case)


def _fork_shape(case):
    """(sequences, table width, pages of a pool)"""
    n = case["parents"] * (1 + case["children"])
    width = -(-(case["length"] + case["c"]) // case["page"]) + 1
    return n, width, case["parents"] * width + n * ((case["c"] - 1) // case["page"] + 2) + 5


def _pool_bytes(case):
    pages = _fork_shape(case)[2] if case["op"] == "fork" else case["live"] + 2 * case["moves"] + 7
    return pages * _page_bytes(case)


def work(case):
    """Attention: the visible keys and values, the queries and the result once, four operations per element of a visible (query, key)
    pair.  Store: the QKV rows read, q, k and v written.  Fork, compact: the copied pages read and written."""
    hq, hkv, hd, _ = MODELS[case["model"]]
    es = _es(case)
    if case["op"] == "attention":
        pairs, keys = _visible(case)
        rows = case["batch"] * case["c"]
        return {"bytes": float(2 * keys * hkv * hd * es + rows * hq * hd * (es + 4)), "flops": float(4 * hd * hq * pairs)}
    if case["op"] == "store":
        rows = case["batch"] * case["c"]
        return {"bytes": float(rows * (hq + 2 * hkv) * hd * (4 + es)), "flops": float(6 * rows * (hq + hkv) * hd)}
    n, width = _fork_shape(case)[:2] if case["op"] == "fork" else (0, 0)
    if case["op"] == "fork":
        copies = sum(case["children"] for m in _lengths(case, case["parents"]) if m % case["page"])
        return {"bytes": float(2 * copies * _page_bytes(case) + 8 * n * width), "flops": 0.0}
    return {"bytes": float(2 * case["moves"] * _page_bytes(case)), "flops": 0.0}


# ---------------------------------------------------------------------------------------------------------------- inputs
def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _pool(case, gen, layers, pages, order="hnd"):
    """Keys and values of a pool, [layers, pages, kv heads, slots, head size] however a page is laid out."""
    _, hkv, hd, _ = MODELS[case["model"]]
    shape = (layers, pages, hkv, case["page"], hd) if order == "hnd" else (layers, pages, case["page"], hkv, hd)
    pair = [torch.empty(shape, dtype=_type(case), device="cuda") for _ in range(2)]
    for t in pair:
        for part in t.view(-1).split(1 << 30):
            part.normal_(generator=gen)
    return pair if order == "hnd" else [t.transpose(2, 3) for t in pair]


def _dealt(case, gen, lens, rows, extra=3):
    """A table that holds lens[b] + rows slots of every sequence, its pages in random order; (table, pages of the pool)."""
    ps = case["page"]
    need = [-(-(m + rows) // ps) for m in lens]
    width, pages = max(need) + 1, sum(need) + extra
    ids = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    at, of = [], []
    for i, k in enumerate(need):
        at += [i * width + j for j in range(k)]
        of += range(len(of), len(of) + k)
    table = torch.full((len(lens) * width,), -1, dtype=torch.int32, device="cuda")
    table[torch.tensor(at, device="cuda")] = ids[torch.tensor(of, device="cuda")]
    return table.view(len(lens), width), pages


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    hq, hkv, hd, layers = MODELS[case["model"]]
    s = {"case": case, "op": case["op"], "n_heads": hq}
    if case["op"] in ("attention", "store"):
        b, c, ps = case["batch"], case["c"], case["page"]
        lens = _lengths(case, b)
        s["table"], pages = _dealt(case, gen, lens, c)
        s["kv_len"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        k, v = _pool(case, gen, 1, pages, case.get("order", "hnd"))
        s["k"], s["v"], s["c"] = k[0], v[0], c
        if case["op"] == "store":
            s["qkv"] = torch.randn(b * c, (hq + 2 * hkv) * hd, generator=gen, device="cuda")
            return s
        s["q"] = (1.5 * torch.randn(b * c, hq * hd, generator=gen, device="cuda")).to(_type(case))
        s["window"], s["sinks"] = case["window"], case["sinks"]
        if case["window"]:                       # pages that no row sees any more have been freed
            first = torch.arange(s["table"].shape[1], device="cuda") * ps
            gone = (first + ps <= (s["kv_len"] - case["window"] + 1)[:, None]) & (first >= case["sinks"])
            s["table"][gone] = -1
        return s
    if case["op"] == "fork":
        n, width, pages = _fork_shape(case)
        heads = _lengths(case, case["parents"])
        held, _ = _dealt(case, gen, heads, 0)
        s["table"] = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
        s["table"][:case["parents"], :held.shape[1] - 1] = held[:, :-1]
        s["kv_len"] = torch.full((n,), -1, dtype=torch.int32, device="cuda")
        s["kv_len"][:case["parents"]] = torch.tensor(heads, dtype=torch.int32, device="cuda")
        s["refs"] = torch.zeros(pages, dtype=torch.int32, device="cuda")
        s["refs"][held[held >= 0].long()] = 1
        s["dst"] = list(range(case["parents"], n))
        s["src"] = [i % case["parents"] for i in range(len(s["dst"]))]
        s["src_d"], s["dst_d"] = torch.tensor(s["src"], device="cuda"), torch.tensor(s["dst"], device="cuda")
        s["c"] = case["c"]
    else:
        live, moves = case["live"], case["moves"]
        pages = live + 2 * moves + 7
        used = torch.zeros(pages, dtype=torch.bool, device="cuda")
        used[:live] = True
        used[torch.randperm(live, generator=gen, device="cuda")[:moves]] = False
        used[live + torch.randperm(pages - live, generator=gen, device="cuda")[:moves]] = True
        ids = used.nonzero()[:, 0]
        ids = ids[torch.randperm(live, generator=gen, device="cuda")].to(torch.int32)
        n, width = 8, live // 6 + 1
        table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
        table.view(-1)[:min(live, 6 * width)] = ids[:6 * width]
        table[6] = table[0]                      # a sequence that shares another one's pages
        s["refs0"] = torch.bincount(table[table >= 0].long(), minlength=pages).to(torch.int32)
        s["refs0"][ids.long()] += (s["refs0"][ids.long()] == 0).to(torch.int32)
        s["table0"] = table
        s["table"], s["refs"] = s["table0"].clone(), s["refs0"].clone()
    s["k"], s["v"] = _pool(case, gen, layers, pages)
    return s


# ---------------------------------------------------------------------------------------------------------------- plain forms
def _attention(s):
    q, k, v, table, c = s["q"], s["k"], s["v"], s["table"].long(), s["c"]
    hkv, ps, hd = k.shape[1:]
    b, width = table.shape
    at = table.clamp(min=0)
    keys = k[at].float().transpose(1, 2).reshape(b, hkv, width * ps, hd)
    values = v[at].float().transpose(1, 2).reshape(b, hkv, width * ps, hd)
    query = q.float().view(b, c, hkv, -1, hd).permute(0, 2, 3, 1, 4)                     # [b, hkv, group, c, hd]
    score = (query.reshape(b, hkv, -1, hd) @ keys.transpose(2, 3) / math.sqrt(hd)).view(b, hkv, -1, c, width * ps)
    t = torch.arange(width * ps, device=q.device)
    pos = (s["kv_len"].long()[:, None] + torch.arange(c, device=q.device))[:, :, None]
    seen = t <= pos
    if s["window"]:
        seen = seen & ((t > pos - s["window"]) | (t < s["sinks"]))
    seen = (seen & (s["kv_len"] >= 0)[:, None, None])[:, None, None]
    score = score.masked_fill(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.where(seen, (score - torch.where(top == -math.inf, 0.0, top)).exp(), 0.0)
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    out = (p.view(b, hkv, -1, width * ps) @ values).view(b, hkv, -1, c, hd)
    return out.permute(0, 3, 1, 2, 4).reshape(b * c, -1)


def _store(s):
    qkv, k, v, c, hq = s["qkv"], s["k"], s["v"], s["c"], s["n_heads"]
    hkv, ps, hd = k.shape[1:]
    rows = qkv.shape[0]
    pos = (s["kv_len"].long()[:, None] + torch.arange(c, device=qkv.device)).view(-1)
    freq = THETA ** (-torch.arange(0, hd, 2, dtype=torch.float64, device=qkv.device) / hd)
    angle = pos[:, None].double() * freq                                                # far positions: 32 bits lose the angle
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    x = qkv.view(rows, -1, hd)
    a, b = x[:, :hq + hkv, :hd // 2], x[:, :hq + hkv, hd // 2:]
    turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    page = s["table"].long()[torch.arange(rows, device=qkv.device) // c, pos // ps]
    k[page, :, pos % ps] = turned[:, hq:].to(k.dtype)
    v[page, :, pos % ps] = x[:, hq + hkv:].to(v.dtype)
    return turned[:, :hq].reshape(rows, -1).to(k.dtype)


def _fork(s):
    table, kv_len, refs, k, v = s["table"], s["kv_len"], s["refs"], s["k"], s["v"]
    src, dst, rows, ps = s["src_d"], s["dst_d"], s["c"], k.shape[3]
    width, pages = table.shape[1], refs.shape[0]
    # the children's pages are freed
    old = table[dst]
    refs.index_add_(0, old.clamp(min=0).view(-1).long(), -(old >= 0).view(-1).to(torch.int32))
    # and the prompts shared
    held = torch.arange(width, device=table.device) < -(-kv_len[src] // ps)[:, None]
    got = torch.where(held, table[src], -1)
    refs.index_add_(0, got.clamp(min=0).view(-1).long(), (got >= 0).view(-1).to(torch.int32))
    table[dst], kv_len[dst] = got, kv_len[src]
    # pages for the window rows: those not there yet, and one's own instead of a shared one
    first = kv_len.long() // ps
    col = first[:, None] + torch.arange((rows - 1) // ps + 2, device=table.device)
    write = (col <= (kv_len.long()[:, None] + rows - 1) // ps) & (kv_len >= 0)[:, None]
    col = col.clamp(max=width - 1)
    now = table.gather(1, col)
    page = now.clamp(min=0).long()
    there = write & (now >= 0)
    seq = torch.arange(table.shape[0], device=table.device)[:, None].expand_as(col)
    writers = torch.zeros(pages, dtype=torch.int32, device=table.device).index_add_(0, page.view(-1), there.view(-1).to(torch.int32))
    last = torch.full((pages,), -1, dtype=torch.int64, device=table.device)
    last = last.scatter_reduce(0, page.view(-1), torch.where(there, seq, -1).view(-1), "amax")
    keeps = there & (writers[page] == refs[page]) & (last[page] == seq)
    need = write & ~keeps
    count = need.sum(1)
    served = (count.cumsum(0) <= (refs == 0).sum()) & (kv_len >= 0)
    need = need & served[:, None]
    free = torch.sort((refs != 0).to(torch.int32), stable=True).indices.to(torch.int32)
    fresh = free[(need.view(-1).long().cumsum(0) - 1).clamp(min=0, max=pages - 1)].view_as(now)
    copy = need & there & (col == first[:, None]) & (kv_len % ps > 0)[:, None]
    to, of = fresh[copy].long(), now[copy].long()
    k[:, to], v[:, to] = k[:, of], v[:, of]
    refs.index_add_(0, page.view(-1), -(need & there).view(-1).to(torch.int32))
    refs[fresh[need].long()] = 1
    table.scatter_(1, col, torch.where(need, fresh, now))
    return served.to(torch.int32)


def _compact(s):
    table, refs, k, v = s["table"], s["refs"], s["k"], s["v"]
    live, at = refs > 0, torch.arange(refs.shape[0], device=refs.device)
    n_live = live.sum()
    to, of = (~live & (at < n_live)).nonzero()[:, 0], (live & (at >= n_live)).nonzero()[:, 0]
    k[:, to], v[:, to] = k[:, of], v[:, of]
    place = at.to(torch.int32)
    place[of] = to.to(torch.int32)
    table.copy_(torch.where(table >= 0, place[table.clamp(min=0).long()], table))
    refs[to], refs[of] = refs[of], 0
    return n_live.to(torch.int32).view(1)


def run(s):
    op = s["op"]
    if own:
        from paper_2311_08263_b200 import engine
    if op == "attention":
        if own:
            return engine.fc_op_paged_attention(s["q"], s["k"], s["v"], s["table"], s["kv_len"], s["c"], s["n_heads"], window=s["window"],
                                                n_sink=s["sinks"])
        return _attention(s)
    if op == "store":
        if own:
            q = engine.fc_op_paged_store(s["qkv"], s["k"], s["v"], s["table"], s["kv_len"], s["c"], s["n_heads"], THETA)
        else:
            q = _store(s)
        return {"q": q, "k": s["k"], "v": s["v"]}
    if op == "fork":
        if own:
            ps = s["k"].shape[3]
            engine.fc_op_pages_free(s["table"], s["kv_len"], s["refs"], ps, s["dst"])
            engine.fc_op_pages_fork(s["table"], s["kv_len"], s["refs"], ps, s["src"], s["dst"])
            served = engine.fc_op_pages_reserve(s["k"], s["v"], s["table"], s["kv_len"], s["refs"], s["c"])
        else:
            served = _fork(s)
        return {"k": s["k"], "v": s["v"], "table": s["table"], "kv_len": s["kv_len"], "refs": s["refs"], "served": served}
    # the pool as it was before: the moved pages are still where they came from
    s["table"].copy_(s["table0"])
    s["refs"].copy_(s["refs0"])
    n_live = engine.fc_op_pages_compact(s["k"], s["v"], s["table"], s["refs"]) if own else _compact(s)
    return {"k": s["k"], "v": s["v"], "table": s["table"], "refs": s["refs"], "n_live": n_live}


# ---------------------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    """Attention and store in 64 bits, sequence by sequence; what fork and compact give is copied, not computed."""
    if case["op"] not in ("attention", "store"):
        return None
    s = prepare(case, seed)
    hq, hkv, hd, _ = MODELS[case["model"]]
    c, ps, table = case["c"], case["page"], s["table"].cpu().tolist()
    if case["op"] == "attention":
        out = torch.zeros(case["batch"] * c, hq, hd, dtype=torch.float64, device="cuda")
        for b, m in enumerate(_lengths(case, case["batch"])):
            for j in range(c):
                p = m + j
                keys = list(range(p + 1))
                if case["window"] and p >= case["window"]:
                    low = p - case["window"] + 1
                    keys = list(range(min(case["sinks"], low))) + list(range(low, p + 1))
                if j == 0:
                    first = keys
            # the keys of the first row and the rows' own: what the later rows see is among them
            union = torch.tensor(sorted(set(first) | set(range(m, m + c))), device="cuda")
            page = torch.tensor([table[b][t // ps] for t in union.tolist()], device="cuda")
            kk, vv = (s[n][page, :, union % ps].double() for n in ("k", "v"))             # [keys, hkv, hd]
            pos = torch.arange(m, m + c, device="cuda")[:, None]
            hidden = union > pos
            if case["window"]:
                hidden = hidden | ((union <= pos - case["window"]) & (union >= case["sinks"]))
            for h in range(hkv):
                g = hq // hkv
                qq = s["q"].view(-1, hq, hd)[b * c:(b + 1) * c, h * g:(h + 1) * g].double()
                sc = torch.einsum("rgd,td->grt", qq, kk[:, h]) * hd ** -0.5
                w = torch.softmax(sc.masked_fill(hidden, -math.inf), -1)
                out[b * c:(b + 1) * c, h * g:(h + 1) * g] = torch.einsum("grt,td->rgd", w, vv[:, h])
        return out.view(-1, hq * hd)
    k, v = s["k"].double(), s["v"].double()
    x = s["qkv"].double().view(-1, hq + 2 * hkv, hd)
    pair = torch.complex(x[..., :hd // 2], x[..., hd // 2:])
    turn = torch.tensor([THETA ** (-2 * i / hd) for i in range(hd // 2)], dtype=torch.float64, device="cuda")
    pos = torch.tensor([m + j for m in _lengths(case, case["batch"]) for j in range(c)], device="cuda")
    pair = pair * torch.polar(torch.ones_like(turn), pos[:, None].double() * turn)[:, None]
    rot = torch.cat([pair.real, pair.imag], -1)
    page = torch.tensor([table[r // c][p // ps] for r, p in enumerate(pos.tolist())], device="cuda")
    k[page, :, pos % ps] = rot[:, hq:hq + hkv]
    v[page, :, pos % ps] = x[:, hq + hkv:]
    return {"q": rot[:, :hq].reshape(len(pos), -1), "k": k, "v": v}
