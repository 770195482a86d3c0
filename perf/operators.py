"""The operators of a paged key/value cache and of scored tokens: cases, inputs, plain forms and the framework's calls.

A cache is pages[layer, page, K/V, kv head, slot, element] with page_refs[page] (how many table entries hold the page, 0 = free),
page_table[sequence slot, i] (the page with tokens i * page_size ..., -1 = none) and seq_lens[sequence slot].

  attend   o[i, h] = softmax(q[i, h] K^T / sqrt(hd)) V over the cached positions up to the token's own
  append   keys and values of new tokens stored at their positions
  fork     free(children), fork(parents -> children), extend(children): shared full pages, a copied tail, room for new tokens
  compact  used pages moved to the front of the pool, tables following them
  copy     pages copied in all layers
  logprobs log-probabilities of given tokens, entropy and the k likeliest tokens of every row of logits

`own` decides between the plain forms (torch, 32 bits) and the framework's own calls."""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # one short sequence, next token: a single user at a small model, nothing but latency
        dict(name="attend_one_short", kind="attend", dtype="bf16", B=1, ones=1, new_lo=1, new_hi=1, past_lo=200, past_hi=200, heads=16,
             kv_heads=8, hd=128, page=16, layout=1),
        # a full decoding batch of ragged lengths: the ordinary step of a server
        dict(name="attend_decode", kind="attend", dtype="bf16", B=64, ones=64, new_lo=1, new_hi=1, past_lo=500, past_hi=4000, heads=32,
             kv_heads=8, hd=128, page=64, layout=2),
        # the next token of one very long sequence: few rows, all the work along the keys
        dict(name="attend_long_one", kind="attend", dtype="f16", B=1, ones=1, new_lo=1, new_hi=1, past_lo=131071, past_hi=131071, heads=32,
             kv_heads=8, hd=128, page=128, layout=3),
        # chunks of long prompts after what is cached already: the products bound it
        dict(name="attend_chunks", kind="attend", dtype="f16", B=4, ones=0, new_lo=900, new_hi=1100, past_lo=2000, past_hi=8000, heads=32,
             kv_heads=8, hd=128, page=64, layout=4),
        # a mixed step: most sequences decode, a few bring candidates' passages behind a cached query
        dict(name="attend_mixed", kind="attend", dtype="bf16", B=64, ones=56, new_lo=60, new_hi=700, past_lo=300, past_hi=2500, heads=16,
             kv_heads=8, hd=128, page=32, layout=5),
        # the fp32 model: short suffixes over a cached prefix
        dict(name="attend_f32", kind="attend", dtype="f32", B=8, ones=2, new_lo=10, new_hi=60, past_lo=100, past_hi=450, heads=4, kv_heads=2,
             hd=64, page=16, layout=6),
        # keys and values of one decoding step
        dict(name="append_step", kind="append", dtype="bf16", B=64, ones=64, new_lo=1, new_hi=1, past_lo=100, past_hi=1000, heads=16,
             kv_heads=8, hd=128, page=16, layout=7),
        # keys and values of a prefill's tokens
        dict(name="append_prefill", kind="append", dtype="f16", B=32, ones=0, new_lo=100, new_hi=1200, past_lo=0, past_hi=300, heads=32,
             kv_heads=8, hd=128, page=64, layout=8),
        # four continuations of each of eight sequences, every step anew: a small model's whole cache
        dict(name="fork_beams", kind="fork", dtype="bf16", parents=8, fan=4, len_lo=150, len_hi=600, new=1, layers=28, kv_heads=8, hd=128,
             page=32, layout=9),
        # a pool of which half has been freed in places
        dict(name="compact_half", kind="compact", dtype="f16", seqs=40, len_lo=20, len_hi=900, layers=28, kv_heads=8, hd=128, page=64,
             layout=10),
        # a reranker's answer: two tokens' probabilities at the last position of a few candidates
        dict(name="logprobs_rerank", kind="logprobs", dtype="f32", rows=8, vocab=151936, given=2, top=5, pad=0, layout=11),
        # every token of some documents scored
        dict(name="logprobs_score", kind="logprobs", dtype="f32", rows=2048, vocab=151936, given=1, top=1, pad=0, layout=12),
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], even over its logarithm where the range is wide."""
    if hi > 10 * max(lo, 1):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(max(lo, 0.5)), math.log(hi)))))))
    return rng.randint(lo, hi)


def draw(rng):
    limit = {}
    for c in listed():
        w = work(c)
        for k in w:
            limit[k] = max(limit.get(k, 0), w[k])
    while True:
        kind = rng.choice(["attend", "attend", "attend", "append", "fork", "compact", "copy", "logprobs", "logprobs"])
        dtype = rng.choice(["bf16", "f16", "bf16", "f16", "f32"])
        kv = rng.choice([1, 2, 4, 8])
        hd = rng.choice([32, 64, 80, 128]) if dtype == "f32" else 128
        page = rng.choice([16, 32, 64, 128, 256])
        c = dict(kind=kind, dtype=dtype, kv_heads=kv, hd=hd, page=page, layout=rng.randrange(1 << 30))
        if kind in ("attend", "append"):
            c["heads"] = kv * rng.choice([1, 2, 3, 4, 5, 8])
            c["B"] = _spread(rng, 1, 128 if dtype != "f32" else 16)
            c["ones"] = rng.choice([0, c["B"] // 2, c["B"], c["B"]])
            a, b = _spread(rng, 1, 1500 if dtype != "f32" else 200), _spread(rng, 1, 1500 if dtype != "f32" else 200)
            c["new_lo"], c["new_hi"] = min(a, b), max(a, b)
            a, b = _spread(rng, 0, 8000 if dtype != "f32" else 1000), _spread(rng, 1, 8000 if dtype != "f32" else 1000)
            c["past_lo"], c["past_hi"] = min(a, b), max(a, b)
            if kind == "append":
                c["past_hi"] = min(c["past_hi"], 600)
                c["past_lo"] = min(c["past_lo"], 600)
        elif kind == "fork":
            c.update(parents=_spread(rng, 1, 16), fan=_spread(rng, 1, 6), layers=rng.choice([2, 28, 36]), new=_spread(rng, 1, 20))
            a, b = _spread(rng, 1, 800), _spread(rng, 1, 800)
            c["len_lo"], c["len_hi"] = min(a, b), max(a, b)
        elif kind == "compact":
            c.update(seqs=_spread(rng, 2, 60), layers=rng.choice([2, 28, 36]))
            a, b = _spread(rng, 1, 1000), _spread(rng, 1, 1000)
            c["len_lo"], c["len_hi"] = min(a, b), max(a, b)
        elif kind == "copy":
            c.update(pairs=_spread(rng, 1, 150), layers=rng.choice([2, 28, 36]))
        else:
            del c["kv_heads"], c["hd"], c["page"]
            c.update(rows=_spread(rng, 1, 2000), vocab=rng.choice([1024, 32000, 50257, 128256, 151936]), given=rng.choice([0, 1, 2, 4]),
                     top=rng.choice([0, 1, 5, 20]), pad=rng.choice([0, 0, 64]))
            if c["given"] == 0 and c["top"] == 0:
                c["top"] = 1
        w = work(c)
        if all(w[k] <= limit[k] for k in w) and _pool_bytes(c) <= 2 << 30:
            return c


# ---- what a case is made of (from the case alone)

def _es(case):
    return 4 if case["dtype"] == "f32" else 2


def _lengths(case):
    """(tokens cached before, new tokens) of every sequence."""
    r = random.Random(case["layout"])
    past = [r.randint(case["past_lo"], case["past_hi"]) for _ in range(case["B"])]
    new = [1] * case["ones"] + [r.randint(case["new_lo"], case["new_hi"]) for _ in range(case["B"] - case["ones"])]
    r.shuffle(new)
    return past, new


def _cdiv(a, b):
    return -(-a // b)


def _parent_lengths(case):
    r = random.Random(case["layout"])
    return [r.randint(case["len_lo"], case["len_hi"]) for _ in range(case["parents"])]


def _compact_lengths(case):
    """Lengths of the sequences of a pool and which of them are still there."""
    r = random.Random(case["layout"])
    lens = [r.randint(case["len_lo"], case["len_hi"]) for _ in range(case["seqs"])]
    alive = [r.random() < 0.5 for _ in lens]
    alive[-1] = True
    return lens, alive


def _pool_pages(case):
    P = case.get("page")
    if case["kind"] in ("attend", "append"):
        past, new = _lengths(case)
        n = sum(_cdiv(a + b, P) for a, b in zip(past, new))
        return n + _cdiv(n, 16) + 1
    if case["kind"] == "fork":
        lens = _parent_lengths(case)
        return sum(_cdiv(n, P) for n in lens) + case["fan"] * sum(_cdiv(n + case["new"], P) - n // P for n in lens) + 3
    if case["kind"] == "compact":
        lens, _ = _compact_lengths(case)
        return sum(_cdiv(n, P) for n in lens) + 2
    if case["kind"] == "copy":
        return 2 * case["pairs"] + 5
    return 0


def _pool_bytes(case):
    if case["kind"] == "logprobs":
        return 0
    return _pool_pages(case) * case.get("layers", 1) * 2 * case["kv_heads"] * case["page"] * case["hd"] * _es(case)


def work(case):
    es = _es(case)
    if case["kind"] == "attend":
        past, new = _lengths(case)
        hq, kv, hd = case["heads"], case["kv_heads"], case["hd"]
        seen = sum(n * p + n * (n + 1) // 2 for p, n in zip(past, new))
        keys = sum(p + n for p, n in zip(past, new))
        return {"bytes": keys * 2 * kv * hd * es + 2 * sum(new) * hq * hd * es, "flops": 4 * hq * hd * seen}
    if case["kind"] == "append":
        _, new = _lengths(case)
        return {"bytes": 4 * sum(new) * case["kv_heads"] * case["hd"] * es, "flops": 0}
    if case["kind"] == "fork":
        rows = case["fan"] * sum(n % case["page"] for n in _parent_lengths(case))
        table = case["fan"] * sum(_cdiv(n + case["new"], case["page"]) for n in _parent_lengths(case)) * 8
        return {"bytes": rows * 4 * case["layers"] * case["kv_heads"] * case["hd"] * es + table, "flops": 0}
    if case["kind"] == "compact":
        lens, alive = _compact_lengths(case)
        # the used pages behind the first `used` ones; with random places about the freed share of them
        pages = [_cdiv(n, case["page"]) for n in lens]
        used = sum(p for p, a in zip(pages, alive) if a)
        r = random.Random(case["layout"] + 1)
        moves = sum(1 for i in _used_pages(case, r) if i >= used)
        return {"bytes": moves * 4 * case["layers"] * case["kv_heads"] * case["page"] * case["hd"] * es + 8 * _pool_pages(case), "flops": 0}
    if case["kind"] == "copy":
        return {"bytes": case["pairs"] * 4 * case["layers"] * case["kv_heads"] * case["page"] * case["hd"] * es, "flops": 0}
    n = case["rows"] * case["vocab"]
    return {"bytes": n * es + case["rows"] * (8 * case["given"] + 8 * case["top"] + 4), "flops": 8 * n}


def _used_pages(case, r):
    """Pages of the living sequences of a compact case, in the order of their table entries."""
    lens, alive = _compact_lengths(case)
    order = list(range(_pool_pages(case)))
    r.shuffle(order)
    out, at = [], 0
    for n, a in zip(lens, alive):
        p = _cdiv(n, case["page"])
        if a:
            out.extend(order[at:at + p])
        at += p
    return out


# ---- inputs

def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _randn(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(shape, generator=g, dtype=torch.float32 if dtype == torch.float32 else dtype, device="cuda")
    return x.mul_(scale) if scale != 1.0 else x


def _pool(case, seed, max_seqs, max_pages):
    shape = (case.get("layers", 1), _pool_pages(case), 2, case["kv_heads"], case["page"], case["hd"])
    st = {"pages": _randn(shape, DTYPES[case["dtype"]], seed),
          "page_refs": torch.zeros(shape[1], dtype=torch.int32, device="cuda"),
          "page_table": torch.full((max_seqs, max_pages), -1, dtype=torch.int32, device="cuda"),
          "seq_lens": torch.zeros(max_seqs, dtype=torch.int32, device="cuda")}
    return st


def _own_cache(st):
    """The framework's handle on the pool that the tensors make, and a workspace: kept by the program as the pool is."""
    if not own:
        return
    from paper_2601_15013_amd import binding
    st["cache"] = binding.Cache(st["pages"], st["page_refs"], st["page_table"], st["seq_lens"])


def _own_page_ws(st, n):
    if not own:
        return
    from paper_2601_15013_amd import binding
    st["ws"] = binding.alloc_workspace(binding.radix_cache_workspace_bytes(st["cache"], n))


def prepare(case, seed):
    kind = case["kind"]
    P = case.get("page")
    st = {"case": case, "kind": kind}
    if kind in ("attend", "append"):
        past, new = _lengths(case)
        B, N = case["B"], sum(new)
        counts = [_cdiv(a + b, P) for a, b in zip(past, new)]
        st.update(_pool(case, seed, B, max(counts)))
        order = list(range(_pool_pages(case)))
        random.Random(seed).shuffle(order)
        table = [[-1] * max(counts) for _ in range(B)]
        at = 0
        for b, n in enumerate(counts):
            table[b][:n] = order[at:at + n]
            at += n
        st["page_table"].copy_(_i32(table))
        st["page_refs"][torch.tensor(order[:at], device="cuda")] = 1
        st["seq_lens"].copy_(_i32([a + b for a, b in zip(past, new)]))
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        st.update(past=_i32(past), cu=_i32(cu), max_new=max(new), lens_host=list(zip(past, new)), cu_host=cu)
        hq, kv, hd = case["heads"], case["kv_heads"], case["hd"]
        # the projections' fused row: q | k | v, as a forward has it
        rows = _randn((N, (hq + 2 * kv) * hd), DTYPES[case["dtype"]], seed + 1, 1.5)
        st["q"] = rows[:, :hq * hd].view(N, hq, hd)
        st["k"] = rows[:, hq * hd:(hq + kv) * hd].view(N, kv, hd)
        st["v"] = rows[:, (hq + kv) * hd:].view(N, kv, hd)
        _own_cache(st)
        if own and kind == "attend":
            from paper_2601_15013_amd import binding
            st["ws"] = binding.alloc_workspace(binding.radix_paged_attention_workspace_bytes(st["cache"], hq, N, B, st["max_new"]))
    elif kind == "fork":
        lens = _parent_lengths(case)
        n_par, fan = case["parents"], case["fan"]
        width = max(_cdiv(n + case["new"], P) for n in lens) + 1
        st.update(_pool(case, seed, n_par * (1 + fan), width))
        order = list(range(_pool_pages(case)))
        random.Random(seed).shuffle(order)
        table = [[-1] * width for _ in range(n_par * (1 + fan))]
        at = 0
        for b, n in enumerate(lens):
            table[b][:_cdiv(n, P)] = order[at:at + _cdiv(n, P)]
            at += _cdiv(n, P)
        st["page_table"].copy_(_i32(table))
        st["page_refs"][torch.tensor(order[:at], device="cuda")] = 1
        st["seq_lens"][:n_par] = _i32(lens)
        n = n_par * fan
        st["parents"] = _i32([i // fan for i in range(n)])
        children = list(range(n_par, n_par + n))
        random.Random(seed + 1).shuffle(children)
        st["children"] = _i32(children)
        st["cu"] = _i32([i * case["new"] for i in range(n + 1)])
        _own_cache(st)
        _own_page_ws(st, n)
    elif kind == "compact":
        lens, alive = _compact_lengths(case)
        width = max(_cdiv(n, P) for n in lens)
        st.update(_pool(case, seed, len(lens), width))
        used = _used_pages(case, random.Random(case["layout"] + 1))
        table = [[-1] * width for _ in lens]
        at = 0
        for b, (n, a) in enumerate(zip(lens, alive)):
            if a:
                table[b][:_cdiv(n, P)] = used[at:at + _cdiv(n, P)]
                at += _cdiv(n, P)
        st["page_table"].copy_(_i32(table))
        st["page_refs"][torch.tensor(used, device="cuda")] = 1
        st["seq_lens"].copy_(_i32([n if a else 0 for n, a in zip(lens, alive)]))
        st["table_before"], st["refs_before"] = st["page_table"].clone(), st["page_refs"].clone()
        _own_cache(st)
        _own_page_ws(st, 0)
    elif kind == "copy":
        st.update(_pool(case, seed, 1, 1))
        order = list(range(_pool_pages(case)))
        random.Random(seed).shuffle(order)
        st["src"], st["dst"] = _i32(order[:case["pairs"]]), _i32(order[case["pairs"]:2 * case["pairs"]])
        _own_cache(st)
        _own_page_ws(st, case["pairs"])
    else:
        R, V = case["rows"], case["vocab"]
        x = _randn((R, V + case["pad"]), DTYPES[case["dtype"]], seed, 2.5)[:, :V]
        g = torch.Generator(device="cuda").manual_seed(seed + 1)
        given = torch.randint(0, V, (R, case["given"]), generator=g, dtype=torch.int32, device="cuda")
        if case["given"]:
            rows = torch.arange(0, R, 2, device="cuda")
            x[rows, given[rows, 0].long()] += 12.0                     # half of the texts say what the model expects
            given[R // 3, -1] = -1                                     # a position without a token
        banned = torch.randperm(V, generator=g, device="cuda")[:V // 200]
        x[1::2, banned] = -math.inf                                    # and every other answer is held to a grammar
        st.update(logits=x, given=given)
        if own:
            from paper_2601_15013_amd import binding
            st["ws"] = binding.alloc_workspace(binding.radix_token_logprobs_workspace_bytes(R, V, case["given"], case["top"]))
    return st


# ---- one pass

def run(st):
    if own:
        return _run_own(st)
    return {"attend": _plain_attend, "append": _plain_append, "fork": _plain_fork, "compact": _plain_compact, "copy": _plain_copy,
            "logprobs": _plain_logprobs}[st["kind"]](st)


def _run_own(st):
    from paper_2601_15013_amd import binding as rb
    kind = st["kind"]
    if kind == "attend":
        return rb.radix_paged_attention(st["cache"], 0, st["q"], st["cu"], st["past"], st["max_new"], st["ws"])
    if kind == "append":
        rb.radix_cache_append(st["cache"], 0, st["k"], st["v"], st["cu"], st["past"])
        return st["pages"]
    if kind == "fork":
        rb.radix_cache_free(st["cache"], st["children"])
        rb.radix_cache_fork(st["cache"], st["parents"], st["children"], st["ws"])
        past = rb.radix_cache_extend(st["cache"], st["cu"], st["ws"], slots=st["children"])
        return {"table": st["page_table"], "refs": st["page_refs"], "lens": st["seq_lens"], "past": past, "pages": st["pages"]}
    if kind == "compact":
        st["page_table"].copy_(st["table_before"])
        st["page_refs"].copy_(st["refs_before"])
        used = rb.radix_cache_compact(st["cache"], st["ws"])
        return {"table": st["page_table"], "refs": st["page_refs"], "used": used, "pages": st["pages"]}
    if kind == "copy":
        rb.radix_cache_copy_pages(st["cache"], st["src"], st["dst"], st["ws"])
        return st["pages"]
    out = rb.radix_token_logprobs(st["logits"], st["given"], st["ws"], top_k=st["case"]["top"])
    return {"logprobs": out[0], "entropy": out[1], "top_ids": out[2], "top_logprobs": out[3]}


def _plain_attend(st):
    case = st["case"]
    hq, kv, hd, P = case["heads"], case["kv_heads"], case["hd"], case["page"]
    g = hq // kv
    out = torch.empty_like(st["q"], memory_format=torch.contiguous_format)
    for b, (past, new) in enumerate(st["lens_host"]):
        L = past + new
        ids = st["page_table"][b, :_cdiv(L, P)].long()
        kvp = st["pages"][0, ids].float()                              # [pages, 2, kv, P, hd]
        k = kvp[:, 0].transpose(0, 1).reshape(kv, -1, hd)[:, :L]
        v = kvp[:, 1].transpose(0, 1).reshape(kv, -1, hd)[:, :L]
        rows = slice(st["cu_host"][b], st["cu_host"][b + 1])
        q = st["q"][rows].float().view(new, kv, g, hd).permute(1, 2, 0, 3).reshape(kv, g * new, hd)
        s = torch.matmul(q, k.transpose(1, 2)) * (1.0 / math.sqrt(hd))
        if new > 1:
            ahead = torch.arange(L, device="cuda")[None, :] > past + torch.arange(new, device="cuda")[:, None]
            s = s.view(kv, g, new, L).masked_fill_(ahead, -math.inf).view(kv, g * new, L)
        e = torch.exp(s - s.amax(-1, keepdim=True))
        o = torch.matmul(e, v) / e.sum(-1, keepdim=True)
        out[rows] = o.view(kv, g, new, hd).permute(2, 0, 1, 3).reshape(new, hq, hd).to(out.dtype)
    return out


def _token_places(st):
    """(page, slot in it) of every new token."""
    cu, P = st["cu"].long(), st["case"]["page"]
    i = torch.arange(st["k"].shape[0], device="cuda")
    b = torch.bucketize(i, cu[1:], right=True)
    p = st["past"].long()[b] + i - cu[b]
    return st["page_table"][b, p // P].long(), p % P


def _plain_append(st):
    page, slot = _token_places(st)
    st["pages"][0][page, 0, :, slot] = st["k"]
    st["pages"][0][page, 1, :, slot] = st["v"]
    return st["pages"]


def _plain_fork(st):
    case, P = st["case"], st["case"]["page"]
    table, refs, lens, pages = st["page_table"], st["page_refs"], st["seq_lens"], st["pages"]
    par, ch = st["parents"].long(), st["children"].long()
    one = torch.ones((), dtype=torch.int32, device="cuda")
    # free
    e = table[ch]
    e = e[e >= 0].long()
    refs.index_add_(0, e, -one.expand(e.numel()))
    table[ch] = -1
    lens[ch] = 0
    # fork
    n = lens[par]
    full, rest = n // P, n % P
    cols = torch.arange(table.shape[1], device="cuda")
    rows = torch.where(cols < full[:, None], table[par], -1)
    e = rows[rows >= 0].long()
    refs.index_add_(0, e, one.expand(e.numel()))
    table[ch] = rows
    tail = (rest > 0).nonzero()[:, 0]
    dst = (refs == 0).nonzero()[:tail.numel(), 0]
    src = table[par[tail], full[tail].long()].long()
    table[ch[tail], full[tail].long()] = dst.int()
    refs[dst] = 1
    keep = torch.arange(P, device="cuda") < rest[tail, None]                         # [tails, P]
    pages[:, dst] = torch.where(keep[None, :, None, None, :, None], pages[:, src], pages[:, dst])
    lens[ch] = n
    # extend
    new = (st["cu"][1:] - st["cu"][:-1])
    past = lens[ch]
    have, want = (past + P - 1) // P, (past + new + P - 1) // P
    ask = (cols >= have[:, None]) & (cols < want[:, None])
    at = ask.nonzero()
    got = (refs == 0).nonzero()[:at.shape[0], 0]
    table[ch[at[:, 0]], at[:, 1]] = got.int()
    refs[got] = 1
    lens[ch] = past + new
    return {"table": table, "refs": refs, "lens": lens, "past": past, "pages": pages}


def _plain_compact(st):
    table, refs, pages = st["page_table"], st["page_refs"], st["pages"]
    table.copy_(st["table_before"])
    refs.copy_(st["refs_before"])
    used = (refs > 0).sum().int().view(1)
    ids = torch.arange(refs.numel(), device="cuda")
    src = ((refs > 0) & (ids >= used)).nonzero()[:, 0]
    dst = ((refs == 0) & (ids < used)).nonzero()[:, 0]
    to = ids.clone()
    to[src] = dst
    pages[:, dst] = pages[:, src]
    refs[dst] = refs[src]
    refs[src] = 0
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()].int(), table))
    return {"table": table, "refs": refs, "used": used, "pages": pages}


def _plain_copy(st):
    st["pages"][:, st["dst"].long()] = st["pages"][:, st["src"].long()]
    return st["pages"]


def _plain_logprobs(st):
    R, V = st["logits"].shape
    k = st["case"]["top"]
    given = st["given"]
    out = {"logprobs": torch.empty(given.shape, device="cuda"), "entropy": torch.empty(R, device="cuda"),
           "top_ids": torch.empty((R, k), dtype=torch.int32, device="cuda"), "top_logprobs": torch.empty((R, k), device="cuda")}
    ids = torch.arange(V, device="cuda", dtype=torch.int32)
    for r0 in range(0, R, 512):
        rows = slice(r0, min(R, r0 + 512))
        x = st["logits"][rows].float()
        d = x - x.amax(1, keepdim=True)
        e = torch.exp(d)
        s = e.sum(1, keepdim=True)
        lse = x.amax(1, keepdim=True) + torch.log(s)
        out["entropy"][rows] = (torch.log(s) - (torch.where(e > 0, d, 0.0) * e).sum(1, keepdim=True) / s)[:, 0]
        if given.shape[1]:
            t = given[rows].long()
            out["logprobs"][rows] = torch.where(t >= 0, x.gather(1, t.clamp(min=0)) - lse, 0.0)
        x = x.clone()
        for i in range(k):                                             # the largest, of equal ones the lowest id, then without it
            best = x.amax(1, keepdim=True)
            at = torch.where(x == best, ids, V).amin(1)
            out["top_ids"][rows, i] = at
            out["top_logprobs"][rows, i] = (best - lse)[:, 0]
            x[torch.arange(x.shape[0], device="cuda"), at.long()] = -math.inf
    return out


# ---- the definition in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "attend":
        return _exact_attend(st)
    if kind == "logprobs":
        return _exact_logprobs(st)
    if kind == "append":
        pages, P = st["pages"], case["page"]
        table = st["page_table"].tolist()
        for b, (past, new) in enumerate(st["lens_host"]):              # page by page: a run of tokens each
            i, end = st["cu_host"][b], st["cu_host"][b + 1]
            p = past
            while i < end:
                n = min(P - p % P, end - i)
                page = pages[0, table[b][p // P]]
                page[0, :, p % P:p % P + n] = st["k"][i:i + n].transpose(0, 1)
                page[1, :, p % P:p % P + n] = st["v"][i:i + n].transpose(0, 1)
                i, p = i + n, p + n
        return pages
    if kind == "copy":
        for s, d in zip(st["src"].tolist(), st["dst"].tolist()):
            st["pages"][:, d] = st["pages"][:, s]
        return st["pages"]
    table, refs, lens, pages = st["page_table"].tolist(), st["page_refs"].tolist(), st["seq_lens"].tolist(), st["pages"]
    P = case["page"]
    if kind == "fork":
        for c, p in zip(st["children"].tolist(), st["parents"].tolist()):
            full, rest = divmod(lens[p], P)
            for j in range(full):
                table[c][j] = table[p][j]
                refs[table[p][j]] += 1
            lens[c] = lens[p]
        for c, p in zip(st["children"].tolist(), st["parents"].tolist()):
            full, rest = divmod(lens[p], P)
            if rest:
                d = refs.index(0)
                refs[d] = 1
                table[c][full] = d
                pages[:, d, :, :, :rest] = pages[:, table[p][full], :, :, :rest]
        past = []
        for c in st["children"].tolist():
            past.append(lens[c])
            for j in range(_cdiv(lens[c], P), _cdiv(lens[c] + case["new"], P)):
                d = refs.index(0)
                refs[d] = 1
                table[c][j] = d
            lens[c] += case["new"]
        return {"table": _i32(table), "refs": _i32(refs), "lens": _i32(lens), "past": _i32(past), "pages": pages}
    used = sum(1 for r in refs if r)                                   # compact
    for s in range(used, len(refs)):
        if refs[s]:
            d = refs.index(0)
            pages[:, d] = pages[:, s]
            refs[d], refs[s] = refs[s], 0
            table = [[d if e == s else e for e in row] for row in table]
    return {"table": _i32(table), "refs": _i32(refs), "used": _i32([used]), "pages": pages}


def _exact_attend(st):
    case = st["case"]
    hq, kv, hd, P = case["heads"], case["kv_heads"], case["hd"], case["page"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    for b, (past, new) in enumerate(st["lens_host"]):
        at = torch.arange(past + new, device="cuda")
        page, slot = st["page_table"][b, at // P].long(), at % P
        first = st["cu_host"][b]
        hidden = at[None, :] > (past + torch.arange(new, device="cuda"))[:, None]
        for h in range(hq):
            j = h // (hq // kv)
            k = st["pages"][0][page, 0, j, slot].double()
            v = st["pages"][0][page, 1, j, slot].double()
            s = st["q"][first:first + new, h].double() @ k.t().contiguous() / hd ** 0.5
            s[hidden] = -math.inf
            out[first:first + new, h] = torch.exp(s - torch.logsumexp(s, 1, keepdim=True)) @ v
    return out


def _exact_logprobs(st):
    R, V = st["logits"].shape
    k = st["case"]["top"]
    res = {"logprobs": [], "entropy": [], "top_ids": [], "top_logprobs": []}
    for r0 in range(0, R, 64):
        x = st["logits"][r0:r0 + 64].double()
        lp = x - torch.logsumexp(x, 1, keepdim=True)
        p = torch.exp(lp)
        res["entropy"].append(-torch.where(p > 0, p * lp, 0.0).sum(1))
        order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]
        res["top_ids"].append(order.int())
        res["top_logprobs"].append(lp.gather(1, order))
        t = st["given"][r0:r0 + 64].long()
        res["logprobs"].append(torch.where(t >= 0, lp.gather(1, t.clamp(min=0)), 0.0))
    return {n: torch.cat(v) for n, v in res.items()}
