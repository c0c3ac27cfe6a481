"""Performance cases of the operators that serve several sequences from one paged cache.

  append   rotary embedding of new queries and keys, keys and values into the sequences' pages (PagedCache.append);
  prompt   causal attention of packed prompts over the pages (PagedCache.prompt_attention);
  prefix   one decode row per sequence, groups of rows sharing a prefix (PagedCache.prefix_attention);
  fork     children of running sequences and their first token: truncate, fork, reserve with copy on write;
  compact  the live pages of a fragmented pool to its lowest ids (PagedCache.compact).

A pool is [layers][pages][K, V][KV heads][16 keys][head_dim], a sequence's logical page i is page_table[seq][i] (-1: none),
refs counts the sequences that hold a page. With `own` false the operators run in plain torch operations."""
import math
import random

import torch

own = False

PAGE = 16


# ------------------------------------------------------------------------------------------------ the cases
def _append(name, rows, cached, hq, hkv, dh, dtype, cache, fused):
    """rows: new rows of each sequence; cached: keys it has already; fused: q, k, v are slices of one projection."""
    return {"name": name, "kind": "append", "rows": _text(rows), "cached": _text(cached), "hq": hq, "hkv": hkv,
            "dh": dh, "dtype": dtype, "cache": cache, "fused": fused}


def _prompt(name, rows, cached, hq, hkv, dh, dtype, cache):
    return {"name": name, "kind": "prompt", "rows": _text(rows), "cached": _text(cached), "hq": hq, "hkv": hkv,
            "dh": dh, "dtype": dtype, "cache": cache}


def _prefix(name, groups, prefix, suffix, hq, hkv, dh, dtype, cache):
    """groups: rows of each group; prefix: its shared keys; suffix: every row's own keys, 0 .. suffix, from the seed."""
    return {"name": name, "kind": "prefix", "groups": _text(groups), "prefix": _text(prefix), "suffix": suffix,
            "hq": hq, "hkv": hkv, "dh": dh, "dtype": dtype, "cache": cache}


def _fork(name, layers, parents, children, longest, hkv, dh, cache):
    """children of each of `parents` sequences of up to `longest` keys."""
    return {"name": name, "kind": "fork", "layers": layers, "parents": parents, "children": children,
            "longest": longest, "hkv": hkv, "dh": dh, "cache": cache}


def _compact(name, layers, pages, seqs, live, hkv, dh, cache):
    """A pool of `pages` of which about `live` percent are held by `seqs` sequences, anywhere in it."""
    return {"name": name, "kind": "compact", "layers": layers, "pages": pages, "seqs": seqs, "live": live, "hkv": hkv,
            "dh": dh, "cache": cache}


def _text(v):
    return " ".join(str(int(x)) for x in v)


def _ints(s):
    return [int(x) for x in s.split()]


def listed():
    return [
        # a decode step of a batch: one new token a sequence, bf16 activations
        _append("append_step_64", [1] * 64, [1900 + 7 * i for i in range(64)], 32, 8, 128, "bf16", "bf16", True),
        # five requests' prompts at once, fp32 activations out of one fused projection
        _append("append_prompts_f32", [2048, 1501, 384, 45, 2021], [0, 0, 130, 0, 7], 32, 8, 128, "f32", "bf16", True),
        # short requests to a small fp32 model: the smallest call
        _prompt("prompt_tiny_f32", [1, 17, 45], [0, 0, 20], 4, 2, 64, "f32", "f32"),
        # an ordinary batch of ragged prompts, some behind cached keys
        _prompt("prompt_packed_bf16", [2048, 1501, 384, 45, 1, 999, 1200, 77, 640, 1296], [0] * 8 + [500, 33],
                32, 8, 128, "bf16", "bf16"),
        # one prompt with the framework's fp32 activations
        _prompt("prompt_2048_f32", [2048], [0], 32, 8, 128, "f32", "bf16"),
        # a long document: the largest
        _prompt("prompt_16381_bf16", [16381], [0], 32, 8, 128, "bf16", "bf16"),
        # a few new rows behind long caches: the turn of a conversation, a block of drafted tokens
        _prompt("prompt_turn_bf16", [96, 8], [12000, 9001], 32, 8, 128, "bf16", "bf16"),
        # four samples of a short prompt, small model: latency
        _prefix("prefix_4x300", [4], [300], 40, 8, 2, 64, "f32", "bf16"),
        # 64 samples of one long prompt
        _prefix("prefix_64x8192", [64], [8192], 512, 32, 8, 128, "bf16", "bf16"),
        # requests behind several system prompts, some alone, fp32 activations
        _prefix("prefix_groups_f32", [9, 24, 1, 3, 16, 1, 5, 12], [6000, 2048, 0, 777, 4100, 3000, 500, 1501], 900,
                32, 8, 128, "f32", "bf16"),
        # 64 samples begin from four prompts: shared pages, their last ones copied for the first token
        _fork("fork_4x16", 8, 4, 16, 2051, 8, 128, "bf16"),
        # a pool of which two fifths are live, gathered
        _compact("compact_8192", 10, 8192, 64, 40, 2, 128, "bf16"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))

    def heads():
        hkv = rng.choice([1, 2, 4, 8])
        return hkv * rng.choice([1, 2, 3, 4, 8]), hkv, rng.choice([64, 128])

    def types():
        return rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])

    kind = rng.choice(["append", "prompt", "prompt", "prefix", "prefix", "fork", "compact"])
    if kind in ("append", "prompt"):
        hq, hkv, dh = heads()
        dtype, cache = types()
        n = log_int(1, 48)
        most = 8000 if dtype == "bf16" or kind == "append" else 4000
        total = max(n, log_int(1, most))
        cut = sorted(rng.sample(range(1, total), n - 1)) if total > n else list(range(1, n))
        rows = [b - a for a, b in zip([0] + cut, cut + [total])]
        far = rng.random() < 0.4
        cached = [rng.choice([0, log_int(1, 12000 if total < 1000 else 2000)]) if far else 0 for _ in rows]
        if kind == "append":
            c = _append("", rows, cached, hq, hkv, dh, dtype, cache, rng.random() < 0.5)
        else:
            c = _prompt("", rows, cached, hq, hkv, dh, dtype, cache)
    elif kind == "prefix":
        hq, hkv, dh = heads()
        dtype, cache = types()
        groups = [log_int(1, 64) for _ in range(log_int(1, 6))]
        longest = log_int(16, 16000)
        prefix = [rng.choice([longest, log_int(1, longest), log_int(1, longest), 0]) for _ in groups]
        c = _prefix("", groups, prefix, log_int(1, 1000), hq, hkv, dh, dtype, cache)
    else:
        hkv, dh, cache = rng.choice([1, 2, 4, 8]), rng.choice([64, 128]), rng.choice(["bf16", "bf16", "f32"])
        if kind == "fork":
            c = _fork("", log_int(1, 8), log_int(1, 8), log_int(1, 24), log_int(1, 2100), hkv, dh, cache)
        else:
            c = _compact("", log_int(1, 6), log_int(64, 5000), log_int(2, 64), rng.randint(5, 90), hkv, dh, cache)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------ inputs
def _dt(s):
    return torch.bfloat16 if s == "bf16" else torch.float32


def _normal(g, shape, dtype, scale=1.0):
    """N(0, scale), a piece at a time: a large pool takes no copy in 32 bits."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for i in range(0, flat.numel(), 1 << 26):
        flat[i:i + (1 << 26)].normal_(0.0, scale, generator=g)
    return out


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _starts(rows):
    out = [0]
    for r in rows:
        out.append(out[-1] + r)
    return out


def _pool(g, py, layers, page_lists, hkv, dh, cache, seqs, num=None, width=None):
    """A pool of num pages that holds the sequences' pages in a shuffled order, and a table of `width` pages a sequence.

    page_lists: for every sequence, its pages as labels (a label that several hold is a shared page)."""
    labels = sorted({x for p in page_lists for x in p})
    num = num or len(labels) + 3
    ids = list(range(num))
    py.shuffle(ids)
    where = dict(zip(labels, ids))
    width = width or max(1, max(len(p) for p in page_lists))
    table = torch.full((seqs, width), -1, dtype=torch.int32)
    refs = torch.zeros(num, dtype=torch.int32)
    for s, p in enumerate(page_lists):
        if p:
            row = torch.tensor([where[x] for x in p], dtype=torch.int32)
            table[s, :len(p)] = row
            refs[row.long()] += 1
    return {"kv": _normal(g, (layers, num, 2, hkv, PAGE, dh), _dt(cache)), "table": table.cuda(), "refs": refs.cuda()}


def _pages(n):
    return (n + PAGE - 1) // PAGE


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    py = random.Random(seed)
    kind, hkv, dh = case["kind"], case["hkv"], case["dh"]
    st = {"case": case}
    if kind in ("append", "prompt"):
        rows, cached, hq = _ints(case["rows"]), _ints(case["cached"]), case["hq"]
        n, total, cu = len(rows), sum(rows), _starts(rows)
        lens = [r + c for r, c in zip(rows, cached)]
        slots = list(range(n))
        py.shuffle(slots)  # sequence i of the batch is in slot slots[i] of the cache
        lists = [[] for _ in range(n)]
        for i, s in enumerate(slots):
            lists[s] = [(s, j) for j in range(_pages(lens[i]))]
        st.update(_pool(g, py, 1, lists, hkv, dh, case["cache"], n))
        by_slot = [0] * n
        for i, s in enumerate(slots):
            by_slot[s] = lens[i]
        st.update(lens=_i32(by_slot), seqs=_i32(slots), cu=_i32(cu), h_cu=cu, h_lens=lens, h_slots=slots,
                  max_len=max(lens))
        if kind == "prompt":
            st["q"] = _normal(g, (total, hq, dh), _dt(case["dtype"]), 1.5)
        else:
            if case["fused"]:
                x = _normal(g, (total, hq + 2 * hkv, dh), _dt(case["dtype"]))
                st["q"], st["k"], st["v"] = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
            else:
                st["q"] = _normal(g, (total, hq, dh), _dt(case["dtype"]))
                st["k"] = _normal(g, (total, hkv, dh), _dt(case["dtype"]))
                st["v"] = _normal(g, (total, hkv, dh), _dt(case["dtype"]))
            places = st["table"].shape[1] * PAGE
            ang = torch.arange(places, dtype=torch.float64, device="cuda")[:, None] * torch.pow(
                torch.tensor(10000.0, dtype=torch.float64, device="cuda"),
                -2.0 * torch.arange(dh // 2, dtype=torch.float64, device="cuda") / dh)[None, :]
            st["cos"], st["sin"] = ang.cos().float(), ang.sin().float()
    elif kind == "prefix":
        groups, prefix, hq = _ints(case["groups"]), _ints(case["prefix"]), case["hq"]
        n = sum(groups)
        lists, lens = [], []
        for gi, (r, p) in enumerate(zip(groups, prefix)):
            full = p // PAGE
            for i in range(r):
                ln = p + py.randint(0 if p else 1, max(1, case["suffix"]))
                # the pages that the prefix fills are shared, one that it ends inside is the row's own copy
                lists.append([(gi, -1, j) for j in range(full)] + [(gi, i, j) for j in range(full, _pages(ln))])
                lens.append(ln)
        st.update(_pool(g, py, 1, lists, hkv, dh, case["cache"], n))
        at = 0
        for r, p in zip(groups, prefix):
            if p % PAGE:
                ids = st["table"][at:at + r, p // PAGE].long()
                st["kv"][0, ids[1:], :, :, :p % PAGE] = st["kv"][0, ids[0], :, :, :p % PAGE]
            at += r
        st.update(lens=_i32(lens), seqs=_i32(list(range(n))), cu=_i32(_starts(groups)), prefix=_i32(prefix),
                  h_lens=lens, max_len=max(lens))
        st["q"] = _normal(g, (n, hq, dh), _dt(case["dtype"]), 1.5)
    elif kind == "fork":
        p, c = case["parents"], case["children"]
        lens = [py.randint(max(1, case["longest"] // 2), case["longest"]) for _ in range(p)]
        lists = [[(s, j) for j in range(_pages(ln))] for s, ln in enumerate(lens)] + [[] for _ in range(p * c)]
        room = _pages(case["longest"] + 1)
        st.update(_pool(g, py, case["layers"], lists, hkv, dh, case["cache"], p * (c + 1), p * (room + c) + 5, room))
        kids = list(range(p, p * (c + 1)))
        src = [i % p for i in range(p * c)]
        st.update(lens=_i32(lens + [0] * (p * c)), src=_i32(src), dst=_i32(kids), keep=_i32([lens[s] for s in src]),
                  none=_i32([0] * (p * c)), one=_i32([1] * (p * c)))
    else:
        s, held = case["seqs"], max(1, case["pages"] * case["live"] // 100)
        sizes = [held // s + (i < held % s) for i in range(s)]
        for i in range(0, s - 1, 2):  # ragged: one sequence's pages go to the next
            d = py.randint(0, sizes[i])
            sizes[i], sizes[i + 1] = sizes[i] - d, sizes[i + 1] + d
        lists = [[(i, j) for j in range(n)] for i, n in enumerate(sizes)]
        st.update(_pool(g, py, case["layers"], lists, hkv, dh, case["cache"], s, case["pages"], 2 * (held // s + 1)))
        st["lens"] = _i32([max(0, n * PAGE - py.randint(0, PAGE - 1)) for n in sizes])
        st["table0"], st["refs0"] = st["table"].clone(), st["refs"].clone()
    if own:
        from paper_2605_30852_amd.cache import PagedCache
        st["cache"] = PagedCache(st["kv"], st["table"], st["lens"], st["refs"])
    return st


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    kind = st["case"]["kind"]
    if own:
        return _own(st, kind)
    return {"append": _plain_append, "prompt": _plain_prompt, "prefix": _plain_prefix, "fork": _plain_fork,
            "compact": _plain_compact}[kind](st)


def _own(st, kind):
    c = st["cache"]
    if kind == "append":
        q = c.append(0, st["k"], st["v"], st["seqs"], st["cu"], q=st["q"], rope=(st["cos"], st["sin"]))
        return {"q": q, "kv": st["kv"]}
    if kind == "prompt":
        return c.prompt_attention(0, st["q"], st["seqs"], st["cu"], max_len=st["max_len"])
    if kind == "prefix":
        return c.prefix_attention(0, st["q"], st["seqs"], st["cu"], st["prefix"], max_len=st["max_len"])
    if kind == "fork":  # the samples of the last pass end, new ones begin
        a = c.truncate(st["dst"], st["none"])
        b = c.fork(st["src"], st["dst"], st["keep"])
        d = c.reserve(st["dst"], st["one"])
        return {"status": [a, b, d], "table": st["table"], "lens": st["lens"], "refs": st["refs"], "kv": st["kv"]}
    # the state as a scheduler hands it over, then the compaction
    st["table"].copy_(st["table0"])
    st["refs"].copy_(st["refs0"])
    live = c.compact()
    return {"live": live, "table": st["table"], "refs": st["refs"], "kv": st["kv"]}


def _plain_append(st):
    c = st["case"]
    hkv, half = c["hkv"], c["dh"] // 2
    rows = st["q"].shape[0]
    r = torch.arange(rows, device="cuda")
    i = torch.searchsorted(st["cu"][1:].contiguous(), r, right=True)
    seq = st["seqs"][i].long()
    pos = (st["lens"][seq] - (st["cu"][i + 1] - st["cu"][i]) + (r - st["cu"][i])).long()
    cos, sin = st["cos"][pos][:, None], st["sin"][pos][:, None]

    def turn(x):
        a, b = x[..., :half].float(), x[..., half:].float()
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    page = st["table"][seq, pos // PAGE].long()
    kv = st["kv"][0]
    kv[page, 0, :, pos % PAGE] = turn(st["k"]).to(kv.dtype)
    kv[page, 1, :, pos % PAGE] = st["v"].to(kv.dtype)
    return {"q": turn(st["q"]).to(st["q"].dtype), "kv": st["kv"]}


def _rows(kv, table, n):
    """The first n keys and values of a sequence, [KV heads][n][head_dim] each, in 32 bits."""
    ids = table[:_pages(n)].long()
    x = kv[ids].permute(1, 2, 0, 3, 4).flatten(2, 3)[:, :, :n].float()
    return x[0], x[1]


def _attend(q, k, v, first, hkv):
    """Rows q [n][Hq][dh] at positions first, first + 1, .. over keys k, v [KV heads][len][dh]."""
    n, hq, dh = q.shape
    G, ln = hq // hkv, k.shape[1]
    out = torch.empty((n, hq, dh), dtype=torch.float32, device="cuda")
    step = max(1, (1 << 28) // max(1, G * ln))
    key = torch.arange(ln, device="cuda")
    for a in range(0, n, step):
        b = min(n, a + step)
        end = min(ln, first + b)
        late = key[:end][None, :] > torch.arange(first + a, first + b, device="cuda")[:, None]
        for h in range(hkv):
            x = q[a:b, h * G:(h + 1) * G].float().reshape(-1, dh)
            s = (x @ k[h, :end].t()) * (1.0 / math.sqrt(dh))
            s = s.view(b - a, G, end).masked_fill_(late[:, None], float("-inf")).view(-1, end)
            s = torch.exp_(s - s.amax(-1, keepdim=True))
            o = (s @ v[h, :end]) / s.sum(-1, keepdim=True)
            out[a:b, h * G:(h + 1) * G] = o.view(b - a, G, dh)
    return out


def _plain_prompt(st):
    q, hkv, out = st["q"], st["case"]["hkv"], []
    for i, (ln, slot) in enumerate(zip(st["h_lens"], st["h_slots"])):
        a, b = st["h_cu"][i], st["h_cu"][i + 1]
        k, v = _rows(st["kv"][0], st["table"][slot], ln)
        out.append(_attend(q[a:b], k, v, ln - (b - a), hkv))
    return torch.cat(out).to(q.dtype)


def _plain_prefix(st):
    q, hkv, out = st["q"], st["case"]["hkv"], []
    for i, ln in enumerate(st["h_lens"]):
        k, v = _rows(st["kv"][0], st["table"][i], ln)
        out.append(_attend(q[i:i + 1], k, v, ln - 1, hkv))
    return torch.cat(out).to(q.dtype)


def _plain_truncate(st, seqs, keep):
    table, lens, refs = st["table"], st["lens"], st["refs"]
    seq = seqs.long()
    keep = torch.minimum(keep, lens[seq])
    j = torch.arange(table.shape[1], device="cuda")[None, :]
    drop = (j >= ((keep + PAGE - 1) // PAGE)[:, None]) & (j < ((lens[seq] + PAGE - 1) // PAGE)[:, None])
    rows = table[seq]
    refs.index_add_(0, rows[drop].long(), torch.full_like(rows[drop], -1))
    table[seq] = torch.where(drop, -1, rows)
    lens[seq] = keep


def _plain_fork_into(st, src, dst, keep):
    table, refs = st["table"], st["refs"]
    j = torch.arange(table.shape[1], device="cuda")[None, :]
    share = j < ((keep + PAGE - 1) // PAGE)[:, None]
    rows = torch.where(share, table[src.long()], -1)
    refs.index_add_(0, rows[share].long(), torch.ones_like(rows[share]))
    table[dst.long()] = rows
    st["lens"][dst.long()] = keep


def _plain_reserve(st, seqs, add):
    table, refs, kv = st["table"], st["refs"], st["kv"]
    seq = seqs.long()
    ln = st["lens"][seq]
    have, want = (ln + PAGE - 1) // PAGE, (ln + add + PAGE - 1) // PAGE
    last = table[seq, (have - 1).clamp(min=0).long()].clamp(min=0).long()
    copy = (add > 0) & (ln % PAGE != 0) & (refs[last] > 1)
    begin = torch.where(copy, have - 1, have)  # a copied page is the first that is taken
    need = want - begin
    at = torch.cumsum(need, 0) - need
    free = (refs == 0).nonzero()[:, 0].int()
    j = torch.arange(table.shape[1], device="cuda")[None, :]
    new = (j >= begin[:, None]) & (j < want[:, None])
    ids = free[(at[:, None] + j - begin[:, None]).clamp(0, free.numel() - 1).long()]
    table[seq] = torch.where(new, ids, table[seq])
    refs[ids[new].long()] = 1
    refs.index_add_(0, last[copy], torch.full_like(last[copy], -1, dtype=torch.int32))
    kv[:, table[seq, (have - 1).clamp(min=0).long()][copy].long()] = kv[:, last[copy]]
    st["lens"][seq] = ln + add


def _plain_fork(st):
    _plain_truncate(st, st["dst"], st["none"])
    _plain_fork_into(st, st["src"], st["dst"], st["keep"])
    _plain_reserve(st, st["dst"], st["one"])
    done = torch.zeros(1, dtype=torch.int32, device="cuda")
    return {"status": [done, done, done], "table": st["table"], "lens": st["lens"], "refs": st["refs"], "kv": st["kv"]}


def _plain_compact(st):
    st["table"].copy_(st["table0"])
    st["refs"].copy_(st["refs0"])
    table, refs, kv = st["table"], st["refs"], st["kv"]
    live = refs > 0
    n = live.sum()
    ids = torch.arange(refs.numel(), device="cuda")
    src, dst = ids[live & (ids >= n)], ids[~live & (ids < n)]
    kv[:, dst] = kv[:, src]
    refs[dst] = refs[src]
    refs[src] = 0
    ids[src] = dst
    table.copy_(torch.where(table >= 0, ids[table.clamp(min=0).long()].int(), table))
    return {"live": n.to(torch.int32).view(1), "table": table, "refs": refs, "kv": kv}


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    global own
    keep, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = keep
    return {"append": _exact_append, "prompt": _exact_prompt, "prefix": _exact_prefix, "fork": _exact_fork,
            "compact": _exact_compact}[case["kind"]](st)


def _exact_append(st):
    c = st["case"]
    dh, kv = c["dh"], st["kv"].double()
    q = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    for i, (ln, slot) in enumerate(zip(st["h_lens"], st["h_slots"])):
        a, b = st["h_cu"][i], st["h_cu"][i + 1]
        pos = torch.arange(ln - (b - a), ln, device="cuda")
        z = torch.complex(st["cos"][pos].double(), st["sin"][pos].double())[:, None]  # e^(i angle) of each dim pair

        def turned(x):
            y = torch.complex(x[a:b, :, :dh // 2].double(), x[a:b, :, dh // 2:].double()) * z
            return torch.cat([y.real, y.imag], -1)

        q[a:b] = turned(st["q"])
        page = st["table"][slot].long()[torch.div(pos, PAGE, rounding_mode="floor")]
        kv[0, page, 0, :, pos - PAGE * torch.div(pos, PAGE, rounding_mode="floor")] = turned(st["k"])
        kv[0, page, 1, :, pos - PAGE * torch.div(pos, PAGE, rounding_mode="floor")] = st["v"][a:b].double()
    return {"q": q, "kv": kv}


def _exact_rows(st, slot, ln, q, first):
    """Head by head: weights exp(s - log sum exp s) of the visible keys."""
    n, hq, dh = q.shape
    hkv = st["case"]["hkv"]
    slots = torch.arange(ln, device="cuda")
    ids = st["table"][slot].long()[slots // PAGE]
    out = torch.empty((n, hq, dh), dtype=torch.float64, device="cuda")
    step = max(1, (1 << 27) // max(1, ln))
    for h in range(hq):
        k = st["kv"][0, ids, 0, h * hkv // hq, slots % PAGE].double()
        v = st["kv"][0, ids, 1, h * hkv // hq, slots % PAGE].double()
        for a in range(0, n, step):
            b = min(n, a + step)
            s = torch.matmul(q[a:b, h].double() / dh ** 0.5, k.t().contiguous())
            hidden = slots[None, :] > first + torch.arange(a, b, device="cuda")[:, None]
            s[hidden] = -float("inf")
            out[a:b, h] = torch.matmul(torch.exp(s - torch.logsumexp(s, 1)[:, None]), v)
    return out


def _exact_prompt(st):
    cu = st["h_cu"]
    return torch.cat([_exact_rows(st, slot, ln, st["q"][cu[i]:cu[i + 1]], ln - (cu[i + 1] - cu[i]))
                      for i, (ln, slot) in enumerate(zip(st["h_lens"], st["h_slots"]))])


def _exact_prefix(st):
    return torch.cat([_exact_rows(st, i, ln, st["q"][i:i + 1], ln - 1) for i, ln in enumerate(st["h_lens"])])


def _exact_fork(st):
    """One child after the other, page by page, on the host."""
    table, lens, refs = st["table"].tolist(), st["lens"].tolist(), st["refs"].tolist()
    kv = st["kv"]
    src, dst, keep = st["src"].tolist(), st["dst"].tolist(), st["keep"].tolist()
    for s, d, k in zip(src, dst, keep):
        for j in range(_pages(k)):
            table[d][j] = table[s][j]
            refs[table[s][j]] += 1
        lens[d] = k
    held = list(refs)
    spare = iter([p for p, r in enumerate(refs) if r == 0])
    old, new = [], []
    for d in dst:
        if lens[d] % PAGE == 0:
            table[d][lens[d] // PAGE] = p = next(spare)
            refs[p] = 1
        elif held[table[d][lens[d] // PAGE]] > 1:
            p = next(spare)
            old.append(table[d][lens[d] // PAGE])
            new.append(p)
            refs[old[-1]] -= 1
            refs[p] = 1
            table[d][lens[d] // PAGE] = p
        lens[d] += 1
    for a, b in zip(old, new):
        kv[:, b] = kv[:, a]
    zero = _i32([0])
    return {"status": [zero, zero, zero], "table": _i32(table), "lens": _i32(lens), "refs": _i32(refs), "kv": kv}


def _exact_compact(st):
    table, refs, kv = st["table"].tolist(), st["refs"].tolist(), st["kv"]
    n = sum(1 for r in refs if r)
    holes = [p for p in range(n) if not refs[p]]
    late = [p for p in range(n, len(refs)) if refs[p]]
    to = dict(zip(late, holes))
    for a, b in to.items():
        kv[:, b] = kv[:, a]
        refs[b], refs[a] = refs[a], 0
    table = [[to.get(p, p) for p in row] for row in table]
    return {"live": _i32([n]), "table": _i32(table), "refs": _i32(refs), "kv": kv}


# ------------------------------------------------------------------------------------------------ what it takes
def work(case):
    kind, hkv, dh = case["kind"], case["hkv"], case["dh"]
    e = 2 if case["cache"] == "bf16" else 4
    key = 2 * hkv * dh * e  # K and V of one key in one layer
    if kind in ("append", "prompt"):
        rows, cached, hq = _ints(case["rows"]), _ints(case["cached"]), case["hq"]
        a, n = 2 if case["dtype"] == "bf16" else 4, sum(rows)
        if kind == "append":
            return {"bytes": n * (2 * hq * dh * a + 2 * hkv * dh * a + key + 4 * dh), "flops": 6 * n * (hq + hkv) * dh // 2}
        seen = sum(r * c + r * (r + 1) // 2 for r, c in zip(rows, cached))
        return {"bytes": 2 * n * hq * dh * a + key * (n + sum(cached)), "flops": 4 * seen * hq * dh}
    if kind == "prefix":
        groups, prefix, hq = _ints(case["groups"]), _ints(case["prefix"]), case["hq"]
        a, n, own_keys = 2 if case["dtype"] == "bf16" else 4, sum(groups), (case["suffix"] + 1) // 2
        return {"bytes": 2 * n * hq * dh * a + key * (sum(prefix) + n * own_keys),
                "flops": 4 * hq * dh * sum(r * (p + own_keys) for r, p in zip(groups, prefix))}
    page = PAGE * key * case["layers"]
    if kind == "fork":
        n, held = case["parents"] * case["children"], _pages(case["longest"] * 3 // 4)
        # the copied pages, and the table's entries and counts read and written
        return {"bytes": n * (2 * page * (PAGE - 1) // PAGE + 4 * 4 * held), "flops": 0}
    held = max(1, case["pages"] * case["live"] // 100)
    moved = held * (case["pages"] - held) // case["pages"]
    return {"bytes": 2 * moved * page + 8 * case["pages"] + 2 * 4 * held, "flops": 0}
