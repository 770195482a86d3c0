"""Plain models of a paged cache for the tests: the pool as Python lists, attention in 64 bits."""
import numpy as np
import torch

from paper_2601_15013_amd import binding

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# half a step of the type, relative to the value
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def status_word():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


class Pool:
    """What the page calls do, one entry after the other (pages by their contents' origin are compared through the tensor)."""

    def __init__(self, n_pages, page, max_seqs, max_pages):
        self.page, self.refs = page, [0] * n_pages
        self.table = [[-1] * max_pages for _ in range(max_seqs)]
        self.lens = [0] * max_seqs

    def take(self):
        p = self.refs.index(0)
        self.refs[p] = 1
        return p

    def held(self, s):
        return -(-self.lens[s] // self.page)

    def extend(self, slots, news, pages=None):
        own = [n > 0 and self.lens[s] % self.page != 0 and self.refs[self.table[s][self.lens[s] // self.page]] > 1
               for s, n in zip(slots, news)]
        past = [self.lens[s] for s in slots]
        freed = []
        for s, n, o in zip(slots, news, own):
            if o:
                j = self.lens[s] // self.page
                old, new = self.table[s][j], self.take()
                freed.append(old)
                self.table[s][j] = new
                if pages is not None:
                    rest = self.lens[s] % self.page
                    pages[:, new, :, :, :rest] = pages[:, old, :, :, :rest]
            for j in range(self.held(s), -(-(self.lens[s] + n) // self.page)):
                self.table[s][j] = self.take()
            self.lens[s] += n
        for p in freed:                     # a page that all its holders left in this call is free after it
            self.refs[p] -= 1
        return past

    def fork(self, parents, children, pages=None):
        for p, c in zip(parents, children):
            for j in range(self.lens[p] // self.page):
                self.table[c][j] = self.table[p][j]
                self.refs[self.table[p][j]] += 1
        for p, c in zip(parents, children):
            rest = self.lens[p] % self.page
            if rest:
                j = self.lens[p] // self.page
                new = self.take()
                self.table[c][j] = new
                if pages is not None:
                    pages[:, new, :, :, :rest] = pages[:, self.table[p][j], :, :, :rest]
            self.lens[c] = self.lens[p]

    def free(self, slots, keep=None):
        for i, s in enumerate(slots):
            k = max(0, keep[i]) if keep is not None else 0
            for j in range(-(-k // self.page), len(self.table[s])):
                if self.table[s][j] >= 0:
                    self.refs[self.table[s][j]] -= 1
                    self.table[s][j] = -1
            self.lens[s] = min(self.lens[s], k)

    def compact(self, pages=None):
        used = sum(r != 0 for r in self.refs)
        src = [p for p in range(used, len(self.refs)) if self.refs[p]]
        dst = [p for p in range(used) if not self.refs[p]]
        to = dict(zip(src, dst))
        for s, d in to.items():
            self.refs[d], self.refs[s] = self.refs[s], 0
            if pages is not None:
                pages[:, d] = pages[:, s]
        self.table = [[to.get(e, e) for e in row] for row in self.table]
        return used

    def agrees(self, cache):
        assert cache.page_refs.tolist() == self.refs
        assert cache.page_table.tolist() == self.table
        assert cache.seq_lens.tolist() == self.lens


def random_cache(seed, lens, kv, hd, page, dtype, layers=1, spare=3, extra_pages=2, scale=1.0, poison=False):
    """A cache of len(lens) slots with random contents on scattered pages.  poison: NaN in every row that belongs to no sequence."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for n in lens]
    n_pages, max_pages = sum(need) + spare, max(need + [1]) + extra_pages
    order = torch.randperm(n_pages, generator=g).tolist()
    table = [[-1] * max_pages for _ in lens]
    at = 0
    pages = (torch.randn((layers, n_pages, 2, kv, page, hd), generator=g) * scale).to(DT[dtype])
    mine = torch.zeros((n_pages, page), dtype=torch.bool)
    for b, n in enumerate(need):
        table[b][:n] = order[at:at + n]
        at += n
        for p in range(lens[b]):
            mine[table[b][p // page], p % page] = True
    if poison:
        pages.masked_fill_(~mine[None, :, None, None, :, None], float("nan"))
    refs = [0] * n_pages
    for p in order[:at]:
        refs[p] = 1
    return binding.Cache(pages.cuda(), i32(refs), i32(table), i32(list(lens)))


def rows_of(cache, layer, slot, n, kind, pages=None, table=None):
    """Keys (0) or values (1) of positions 0 .. n - 1 of a slot in 64 bits: [n, kv, hd] on the CPU."""
    pages = cache.pages[layer].cpu() if pages is None else pages
    table = cache.page_table.cpu().long() if table is None else table
    at, page = torch.arange(n), pages.shape[3]
    return pages[table[slot, at // page], kind, :, at % page].double()


def attention_ref(cache, layer, q, cu, past, slots=None):
    """(o, a): the outputs in 64 bits and the softmax-weighted mean of |v|, which bounds what a rounded probability can do."""
    q = q.cpu().double()
    N, hq, hd = q.shape
    o, a = torch.zeros_like(q), torch.zeros_like(q)
    pages, table = cache.pages[layer].cpu(), cache.page_table.cpu().long()
    for b in range(len(cu) - 1):
        n = cu[b + 1] - cu[b]
        if n <= 0 or past[b] < 0:
            continue
        k, v = (rows_of(cache, layer, slots[b] if slots else b, past[b] + n, kind, pages, table) for kind in (0, 1))
        g = hq // k.shape[1]
        for h in range(hq):
            s = q[cu[b]:cu[b + 1], h] @ k[:, h // g].T / hd ** 0.5
            pos = torch.arange(past[b] + n)
            s = s.masked_fill(pos[None, :] > past[b] + torch.arange(n)[:, None], float("-inf"))
            p = torch.softmax(s, -1)
            o[cu[b]:cu[b + 1], h] = p @ v[:, h // g]
            a[cu[b]:cu[b + 1], h] = p @ v[:, h // g].abs()
    return o, a


def attention_tolerance(dtype, o, a, hd, longest):
    """Largest error by arithmetic.  Scores: a sum of hd products in fp32, |q||k| of up to 25 each way here, scaled by 1/sqrt(hd):
    (hd + 4) 2^-24 times sum |q k| / sqrt(hd) <= 4e-4 for standard normal entries, and as much relative to every p.  Sums of p and of
    p v over `longest` keys: at most log-many roundings matter in blocked sums, bounded by (longest / 4 + 64) 2^-24.  Then for
    16-bit types half a step on every p (16-bit floats below 2^-14 lose at most 2^-25 absolutely) and half a step on the result."""
    u = HALF_STEP[dtype]
    rel = 4e-4 + 2 * (longest / 4 + 64) * 2.0 ** -24
    tol = rel * a + u * o.abs()
    if dtype != "f32":
        tol = tol + u * a * (1 + rel)
    if dtype == "f16":
        tol = tol + 2.0 ** -25 * longest * 6.0 + 2.0 ** -25      # |v| <= 6, row sum >= 1
    return tol + 1e-30


def ragged(news):
    return np.concatenate([[0], np.cumsum(news)]).astype(int).tolist()
