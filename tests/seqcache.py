"""Plain 64-bit statements of the calls on a cache of several sequences, and caches to run them on."""
import math

import torch

PAGE = 16


def pages(n):
    return (n + PAGE - 1) // PAGE


class Model:
    """The pages of a cache on the host: lists of ids, counts, lengths; `data` holds what a page holds, per layer."""

    def __init__(self, num_pages, max_seqs, max_pages):
        self.num, self.max_pages = num_pages, max_pages
        self.table = [[-1] * max_pages for _ in range(max_seqs)]
        self.lens = [0] * max_seqs
        self.refs = [0] * num_pages
        self.data = list(range(num_pages))  # which original contents a page shows

    def reserve(self, seqs, add):
        n = len(self.lens)
        if any(not 0 <= s < n for s in seqs) or len(set(seqs)) < len(seqs):
            return 3
        if any(a < 0 or self.lens[s] + a > PAGE * self.max_pages for s, a in zip(seqs, add)):
            return 2
        takes = []
        for s, a in zip(seqs, add):
            ln = self.lens[s]
            copy = a > 0 and ln % PAGE and self.refs[self.table[s][ln // PAGE]] > 1
            takes += [(s, j, copy and j == ln // PAGE) for j in range(ln // PAGE if copy else pages(ln), pages(ln + a))]
        free = [p for p, r in enumerate(self.refs) if r == 0]
        if len(free) < len(takes):
            return 1
        for (s, j, copy), p in zip(takes, free):
            if copy:
                self.data[p] = self.data[self.table[s][j]]
                self.refs[self.table[s][j]] -= 1
            self.table[s][j] = p
            self.refs[p] = 1
        for s, a in zip(seqs, add):
            self.lens[s] += a
        return 0

    def fork(self, src, dst, keep):
        n = len(self.lens)
        if any(not 0 <= s < n for s in src + dst) or len(set(dst)) < len(dst) or any(self.lens[d] for d in dst):
            return 3
        if any(k < 0 or k > self.lens[s] for s, k in zip(src, keep)):
            return 2
        for s, d, k in zip(src, dst, keep):
            for j in range(pages(k)):
                self.table[d][j] = self.table[s][j]
                self.refs[self.table[s][j]] += 1
        for d, k in zip(dst, keep):
            self.lens[d] = k
        return 0

    def truncate(self, seqs, keep):
        if any(not 0 <= s < len(self.lens) for s in seqs) or len(set(seqs)) < len(seqs):
            return 3
        if any(k < 0 for k in keep):
            return 2
        for s, k in zip(seqs, keep):
            for j in range(pages(min(k, self.lens[s])), pages(self.lens[s])):
                self.refs[self.table[s][j]] -= 1
                self.table[s][j] = -1
            self.lens[s] = min(k, self.lens[s])
        return 0

    def compact(self):
        n = sum(r > 0 for r in self.refs)
        to = dict(zip([p for p in range(n, self.num) if self.refs[p]], [p for p in range(n) if not self.refs[p]]))
        for a, b in to.items():
            self.data[b] = self.data[a]
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.table = [[to.get(p, p) for p in row] for row in self.table]
        return n


def i32(v, device="cuda"):
    return torch.tensor(v, dtype=torch.int32, device=device)


def filled(lens, hkv, dh, dtype, seed, layers=1, spare=3, extra_pages=0, stale=float("nan")):
    """A PagedCache whose sequences hold lens keys, in shuffled pages; slots past a sequence's keys hold `stale`.
    Also the keys and values per sequence, [layers][2][KV heads][len][dh]."""
    from paper_2605_30852_amd.cache import PagedCache
    g = torch.Generator().manual_seed(seed)
    counts = [pages(n) for n in lens]
    num = sum(counts) + spare
    ids = torch.randperm(num, generator=g).int()
    kv = torch.full((layers, num, 2, hkv, PAGE, dh), stale, dtype=dtype)
    table = torch.full((len(lens), max(1, max(counts)) + extra_pages), -1, dtype=torch.int32)
    refs = torch.zeros(num, dtype=torch.int32)
    rows, at = [], 0
    for s, n in enumerate(lens):
        x = torch.randn(layers, 2, hkv, n, dh, generator=g).to(dtype)
        mine = ids[at:at + counts[s]]
        at += counts[s]
        table[s, :counts[s]] = mine
        refs[mine.long()] = 1
        for j in range(counts[s]):
            part = x[:, :, :, j * PAGE:(j + 1) * PAGE]
            kv[:, int(mine[j]), :, :, :part.shape[3]] = part
        rows.append(x)
    return PagedCache(kv.cuda(), table.cuda(), i32(list(lens)), refs.cuda()), rows


def agree(cache, first, other, n):
    """The first n keys and values of sequence `other` become those of `first`."""
    j = torch.arange(n, device="cuda")
    a, b = cache.page_table[first, j // PAGE].long(), cache.page_table[other, j // PAGE].long()
    cache.kv[:, b, :, :, j % PAGE] = cache.kv[:, a, :, :, j % PAGE]


def attend(q, k, v, limits):
    """q [n][heads][dh] over k, v [KV heads][len][dh], row i the first limits[i] keys: outputs in 64 bits, and
    sum p |v|, which scales the error of rounded probabilities."""
    n, hq, dh = q.shape
    G = hq // k.shape[0]
    out, mag = torch.zeros(n, hq, dh, dtype=torch.float64), torch.zeros(n, hq, dh, dtype=torch.float64)
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    for i in range(n):
        m = limits[i]
        if m <= 0:
            continue
        for h in range(hq):
            p = torch.softmax(k[h // G, :m] @ q[i, h] / math.sqrt(dh), 0)
            out[i, h], mag[i, h] = p @ v[h // G, :m], p @ v[h // G, :m].abs()
    return out, mag


def check(got, want, mag, what):
    """fp32: a score of dh = 128 products of fp32 sums is off by some sqrt(128) 2^-24 sum |q k| / sqrt(dh), with queries
    of deviation 1.5 about 8e-6, which moves a probability by as much of itself: 2e-5 of sum p |v| holds it twice.
    bf16: at most half a step, 2^-8, of each rounded probability and 2^-8 of the output, beside that."""
    got = got.double().cpu()
    assert torch.isfinite(got).all(), what
    bound = 2e-5 * mag + 1e-30
    if what[0] == "bf16":
        bound = bound + 2 ** -8 * (want.abs() + 1.01 * mag)
    worst = ((got - want).abs() / bound).max().item() if got.numel() else 0.0
    assert worst <= 1.0, (what, worst)
