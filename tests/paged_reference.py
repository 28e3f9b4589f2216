"""The paged K/V cache in plain Python and 64 bits: what the tests of its operations compare with."""
import math

import torch


def visible(p, window, n_sink):
    """Positions that the row at position p sees."""
    low = max(0, p - window + 1) if window else 0
    return list(range(min(n_sink, low) if window else 0)) + list(range(low, p + 1))


def attention(q, k, v, table, kv_len, c, n_heads, window=0, n_sink=0):
    """(result, bound on the error of an fp32 evaluation), both [B*c, n_heads, hd] in 64 bits.  Rows that see a missing page are NaN.

    The bound, with u = 2^-23 (sums of the tensor cores are cut off, not rounded): a score is a sum of hd products, off by at most hd u sum |q_i k_i| /
    sqrt(hd), and its exponential by that, by |score| u for the scaling and by 4 u for itself; numerator and denominator both have these errors.
    Probabilities in two bf16 parts lose 2^-17.  Sums over n keys lose n u of the sum of the absolute terms."""
    B, hkv, hd = table.shape[0], k.shape[1], k.shape[3]
    g, ps, n_pages = n_heads // hkv, k.shape[2], k.shape[0]
    out = torch.zeros(B * c, n_heads, hd, dtype=torch.float64)
    tol = torch.zeros_like(out)
    qd, kd, vd = q.double().cpu().view(B * c, n_heads, hd), k.cpu(), v.cpu()
    tab, lens = table.cpu().tolist(), kv_len.cpu().tolist()
    for b in range(B):
        if lens[b] < 0:
            continue
        for j in range(c):
            t = visible(lens[b] + j, window, n_sink)
            pages = [tab[b][i // ps] if i // ps < len(tab[b]) else -1 for i in t]
            if any(p < 0 or p >= n_pages for p in pages):
                out[b * c + j] = math.nan
                continue
            at, slot = torch.tensor(pages), torch.tensor([i % ps for i in t])
            kk, vv = kd[at, :, slot].double(), vd[at, :, slot].double()                          # [n, hkv, hd]
            qq = qd[b * c + j].view(hkv, g, hd)
            s = torch.einsum("hgd,nhd->hgn", qq, kk) / math.sqrt(hd)
            w = torch.softmax(s, -1)
            u = 2.0 ** -23
            off = hd * u * torch.einsum("hgd,nhd->hgn", qq.abs(), kk.abs()) / math.sqrt(hd) + (s.abs() + 4) * u
            rel = 2 * off.amax(-1, keepdim=True) + 2.0 ** -17 + 2 * (len(t) + 32) * u
            out[b * c + j] = torch.einsum("hgn,nhd->hgd", w, vv).reshape(n_heads, hd)
            tol[b * c + j] = (torch.einsum("hgn,nhd->hgd", w, vv.abs()) * rel).reshape(n_heads, hd)
    return out, tol


def rotated(x, pos, theta):
    """x [rows, heads, hd] in 64 bits, rows at positions pos."""
    hd = x.shape[-1]
    f = theta ** (-torch.arange(0, hd, 2, dtype=torch.float64) / hd)
    a = torch.tensor(pos, dtype=torch.float64)[:, None] * f
    cos, sin = a.cos()[:, None], a.sin()[:, None]
    x0, x1 = x[..., :hd // 2], x[..., hd // 2:]
    return torch.cat([x0 * cos - x1 * sin, x0 * sin + x1 * cos], -1)


class Pool:
    """Tables, lengths, counts and the content of pages (any list of values per page) as Python lists."""

    def __init__(self, n_pages, n_seqs, width, page_size):
        self.ps, self.width = page_size, width
        self.refs, self.table = [0] * n_pages, [[-1] * width for _ in range(n_seqs)]
        self.kv_len = [-1] * n_seqs
        self.content = list(range(n_pages))                                   # page p holds the mark content[p]

    def free(self, seqs, window=0, n_sink=0):
        for s in seqs:
            for i in range(self.width):
                if window and not ((i + 1) * self.ps <= self.kv_len[s] - window + 1 and i * self.ps >= n_sink):
                    continue
                if self.table[s][i] >= 0:
                    self.refs[self.table[s][i]] -= 1
                self.table[s][i] = -1
            if not window:
                self.kv_len[s] = -1

    def fork(self, src, dst):
        for a, b in zip(src, dst):
            self.free([b])
            self.kv_len[b] = self.kv_len[a]
            for i in range(-(-max(0, self.kv_len[a]) // self.ps)):
                self.table[b][i] = self.table[a][i]
                if self.table[a][i] >= 0:
                    self.refs[self.table[a][i]] += 1

    def reserve(self, rows):
        ranges, writers = {}, {}
        for b, n in enumerate(self.kv_len):
            if n >= 0 and (n + rows - 1) // self.ps < self.width:
                ranges[b] = range(n // self.ps, (n + rows - 1) // self.ps + 1)
                for i in ranges[b]:
                    writers.setdefault(self.table[b][i], []).append(b)
        keeps = {p: w[-1] for p, w in writers.items() if p >= 0 and len(w) == self.refs[p]}
        free = [p for p, r in enumerate(self.refs) if r == 0]
        served, over = [0] * len(self.kv_len), False
        for b, r in ranges.items():
            need = [i for i in r if self.table[b][i] < 0 or keeps.get(self.table[b][i]) != b]
            if over or len(need) > len(free):
                over = True
                continue
            served[b] = 1
            for i in need:
                p, old = free.pop(0), self.table[b][i]
                self.refs[p] = 1
                if old >= 0:
                    self.refs[old] -= 1
                    if i == r[0] and self.kv_len[b] % self.ps:
                        self.content[p] = self.content[old]
                self.table[b][i] = p
        return served

    def compact(self):
        n = sum(r > 0 for r in self.refs)
        holes = [p for p in range(n) if self.refs[p] == 0]
        high = [p for p in range(n, len(self.refs)) if self.refs[p] > 0]
        place = dict(zip(high, holes))
        for a, b in place.items():
            self.content[b] = self.content[a]
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.table = [[place.get(p, p) for p in row] for row in self.table]
        return n
