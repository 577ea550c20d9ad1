"""Several new tokens per request over the paged cache, and pages that several requests hold, as measurable cases.

Keys of a case
    call     "chunk" (pact_chunk_attention: the attention of prompts, further turns or drafted tokens over the cached rows), "fork" (pact_cache_fork: requests
             that go on with the rows of others, or are cut, or end), "copy" (pact_page_copy: one layer's rows of the pages that a fork or a compaction
             copies), "compact" (pact_cache_compact: the used pages to the lowest ids)
    B, rows  requests, and cached rows of the longest one; `ragged`: the requests differ in length, and from eight on one holds none
    page     rows of a page
    n_qh, n_kvh, d_h   query heads, key heads, head width
    dtype, out         element types of the cache and the queries, and of the attention's result ("bf16" or "fp32")
    new      "chunk": new tokens of the longest request, the last of its cached rows (0: all of them, a whole prompt)
    stride   "chunk": 0 for packed new rows, else the rows that each request has room for
    causal   "chunk": a token attends to the rows up to its own; otherwise to all
    sizes    the cached rows carry the log of a cluster size, which the attention adds to the logits
    bounds   "copy": the cache keeps bounds of its pages' keys
    heads_first   order of a page's axes: key heads before rows, or rows before key heads
    kind     "fork": "beams" (each request goes on with one of its group), "samples" (the first of a group is forked to all), "cut" (drafted rows
             that were not accepted are dropped, a few requests end); "copy": "tails" (the part-filled pages of a fork), "whole" (whole pages)
    group    "fork", "compact": requests that share the pages of a prompt
    pages    "copy": pages to copy; "compact": pages of the cache
"""
import functools
import math
import random

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}

_BASE = {"call": "chunk", "B": 1, "rows": 2500, "ragged": False, "page": 64, "n_qh": 28, "n_kvh": 4, "d_h": 128, "dtype": "bf16", "out": "bf16", "new": 0,
         "stride": 0, "causal": True, "sizes": True, "bounds": True, "heads_first": True, "kind": "", "group": 1, "pages": 0}


def _case(name=None, **kw):
    c = dict(_BASE, **kw)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # a short prompt on a small fp32 model: the smallest call
        _case("chunk_tiny_fp32", rows=212, new=40, n_qh=2, n_kvh=2, d_h=64, page=16, dtype="fp32", out="fp32"),
        # one chat about one large image: the next question
        _case("chunk_turn_2500", rows=2500, new=40),
        # drafted tokens of 32 chats are looked at together
        _case("chunk_drafts_32", B=32, rows=8192, ragged=True, new=5, n_qh=32, n_kvh=8),
        # whole reduced prompts of 12 requests, as they lie in the padded output of the reduction
        _case("chunk_prompts_12", B=12, rows=2948, ragged=True, new=0, stride=2948),
        # a piece of the prompt about hours of video, far into it
        _case("chunk_long_65536", rows=65536, new=1024, n_qh=32, n_kvh=8),
        # text that looks at all states of an encoder, small pages with rows before heads, the result in fp32
        _case("chunk_cross_8", B=8, rows=2916, ragged=True, new=256, causal=False, page=16, out="fp32", sizes=False, heads_first=False),
        # a step of beam search: 32 prompts with 4 beams each
        _case("fork_beams_128", call="fork", B=128, rows=3000, ragged=True, page=16, kind="beams", group=4),
        # eight answers to one long video
        _case("fork_samples_8", call="fork", B=8, rows=131072, kind="samples", group=8),
        # the part-filled pages of those beams, one layer
        _case("copy_tails_96", call="copy", kind="tails", pages=96, page=16),
        # one layer of a cache that is being compacted
        _case("copy_whole_4000", call="copy", kind="whole", pages=4000, n_qh=32, n_kvh=8),
        # a small cache after some requests have ended
        _case("compact_2048", call="compact", B=24, rows=4000, ragged=True, pages=2048),
        # a large one of small pages, prompts shared
        _case("compact_65536", call="compact", B=128, rows=8192, ragged=True, page=16, group=4, pages=65536),
    ]


# (n_qh, n_kvh, d_h) of the models a caller may bring
_MODELS = [(2, 2, 64), (14, 2, 64), (16, 4, 128), (4, 4, 128), (28, 4, 128), (32, 8, 128), (32, 8, 80)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """One more case of the same ranges."""
    call = rng.choices(["chunk", "fork", "copy", "compact"], [52, 18, 15, 15])[0]
    n_qh, n_kvh, d_h = rng.choices(_MODELS, [1, 1, 1, 1, 3, 3, 1])[0]
    B = rng.choices([1, _log_int(rng, 2, 64)], [1, 2])[0]
    kw = {"call": call, "n_qh": n_qh, "n_kvh": n_kvh, "d_h": d_h, "B": B, "ragged": B > 1 and rng.random() < 0.8,
          "page": rng.choice([16, 32, 64, 128]), "sizes": rng.random() < 0.8, "heads_first": rng.random() < 0.7}
    if call == "chunk":
        f32 = rng.random() < 0.15
        if f32:
            kw.update(dtype="fp32", out="fp32")
        elif rng.random() < 0.25:
            kw["out"] = "fp32"
        pairs = 12 * 28 * 2948 * 2948 // (16 if f32 else 2)                        # of a query head with a row, at most
        new = _log_int(rng, 1, min(2948, int((pairs / (B * n_qh)) ** 0.5)))
        rows = _log_int(rng, new, max(new, min(65536, pairs // (B * n_qh * new), 1 << 30)))
        kw.update(rows=rows, new=0 if rng.random() < 0.25 and rows * rows * B * n_qh <= pairs else new, causal=rng.random() < 0.8)
        n = kw["new"] or rows
        kw["stride"] = 0 if rng.random() < 0.6 else n + rng.randint(0, 40)
    elif call == "fork":
        kw["kind"] = rng.choice(["beams", "samples", "cut"])
        kw["group"] = rng.randint(2, 8) if kw["kind"] != "cut" else 1
        kw["B"] = max(1, B // kw["group"]) * kw["group"]
        kw["rows"] = _log_int(rng, 20, min(131072, 600000 // kw["B"]))
    elif call == "copy":
        kw["kind"] = rng.choice(["tails", "whole"])
        if rng.random() < 0.2:
            kw.update(dtype="fp32", out="fp32")
        kw["bounds"] = rng.random() < 0.7
        most = 4000 * 64 * 8 * 128 * 2 // (kw["page"] * n_kvh * d_h * (4 if kw.get("dtype") == "fp32" else 2))
        kw["pages"] = _log_int(rng, 1, min(4000, most))
    else:
        kw["group"] = rng.choice([1, rng.randint(2, 8)])
        kw["B"] = max(1, B // kw["group"]) * kw["group"]
        kw["rows"] = _log_int(rng, 20, min(65536, 400000 // kw["B"]))
        kw["pages"] = int(sum(-(-n // kw["page"]) for n in _lengths(_case(**kw))) * rng.uniform(1.05, 3)) + 3
    return _case(**kw)


# ---- inputs ------------------------------------------------------------------------------------------------------

def _lengths(case):
    """Cached rows of each request."""
    B, rows = case["B"], case["rows"]
    if not case["ragged"]:
        return [rows] * B
    n = [max(1, rows - (rows * 3 * b) // (4 * B) - b % 7) for b in range(B)]
    if B >= 8:
        n[-1] = 0
    random.Random(B).shuffle(n)
    return n


def _new(case):
    """New tokens of each request, the last of its rows."""
    return [n if not case["new"] else min(n, case["new"] - (b % 3 if case["ragged"] else 0)) if case["new"] > 3 else min(n, case["new"])
            for b, n in enumerate(_lengths(case))]


def _holders(case):
    """Requests that share prompts: lengths, block tables of names 0, 1, .. of pages (-1: none), holders of each page beside the first."""
    page, B, G = case["page"], case["B"], case["group"]
    lengths = _lengths(case)
    width = max(1, -(-max(lengths) // page)) + 2
    table, extra, name = np.full((B, width), -1, np.int32), [], 0
    for g in range(0, B, G):
        if case["kind"] == "samples":                  # one prompt, the others of the group are empty
            lengths[g + 1:g + G] = [0] * (len(lengths[g:g + G]) - 1)
        common = 0 if G == 1 or case["kind"] == "samples" else min(lengths[g:g + G]) * 4 // 5 // page
        held_outside = case["kind"] == "beams" and g % (3 * G) == 0               # prompts that the program keeps for requests to come
        for b in range(g, min(B, g + G)):
            n = -(-lengths[b] // page)
            own_from = common if b > g else 0
            table[b, :common] = table[g, :common]
            table[b, own_from:n] = np.arange(name, name + n - own_from)
            name += n - own_from
            extra += [len(range(g, min(B, g + G))) - 1 + held_outside] * (common if b == g else 0)
            extra += [0] * (n - common)
    return lengths, table, np.asarray(extra, np.int32)


def _sources(case, lengths):
    """"fork": the request that each goes on with, and how many of its rows."""
    B, G = case["B"], case["group"]
    rng = random.Random(B * 17 + case["rows"])
    if case["kind"] == "cut":
        source = [-1 if B > 4 and b % 9 == 5 else b for b in range(B)]
        return source, [0 if s < 0 else max(0, lengths[b] - rng.randint(0, 5)) for b, s in enumerate(source)]
    source = []
    for b in range(B):
        g = b // G * G
        if case["kind"] == "samples":
            source.append(g)
        else:
            source.append(-1 if g // G % 8 == 7 else g + min(rng.randrange(G), rng.randrange(G)))
    return source, [0 if s < 0 else lengths[s] for s in source]


def _scale(case):
    return float(np.float32(1.0 / math.sqrt(case["d_h"])))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dev = {"device": "cuda", "generator": g}
    B, page, H, D, dt = case["B"], case["page"], case["n_kvh"], case["d_h"], _TYPES[case["dtype"]]
    i32 = lambda v: torch.tensor(np.asarray(v, np.int32), device="cuda")   # noqa: E731
    st = {"case": case, "page": page, "status": i32([0])}
    if case["call"] in ("fork", "compact"):
        lengths, names, extra = _holders(case)
        n_used = len(extra)
        n_pages = case["pages"] or n_used + B + 40
        perm = torch.randperm(n_pages, **dev).cpu().numpy().astype(np.int32)
        table = np.where(names >= 0, perm[np.maximum(names, 0)], -1).astype(np.int32)
        shared, free = np.zeros(n_pages, np.int32), np.full(n_pages, -1, np.int32)
        shared[perm[:n_used]] = extra
        free[:n_pages - n_used] = perm[n_used:]
        st.update(table=i32(table), length=i32(lengths), shared=i32(shared), free=i32(free), n_free=i32([n_pages - n_used]),
                  table_out=i32(np.full_like(table, -1)), shared_out=i32([0] * n_pages), free_out=i32([-1] * n_pages), n_copies=i32([0]))
        if case["call"] == "fork":
            source, rows = _sources(case, lengths)
            st.update(source=i32(source), rows=i32(rows), length_out=i32([0] * B), n_free_out=i32([0]),
                      copies=i32(np.zeros((B, 3))))
        else:
            st.update(moved_to=i32([0] * n_pages), copies=i32(np.zeros((n_pages // 2 + 1, 3))))
        return st
    lengths, new = (_lengths(case), _new(case)) if case["call"] == "chunk" else ([], [])
    pages_of = [-(-n // page) for n in lengths]
    n_pages = sum(pages_of) + 24 if case["call"] == "chunk" else 2 * case["pages"] + 7
    perm = torch.randperm(n_pages, **dev).cpu().numpy().astype(np.int32)
    shape = (n_pages, H, page, D) if case["heads_first"] else (n_pages, page, H, D)
    st["K"], st["V"] = torch.randn(shape, dtype=dt, **dev), torch.randn(shape, dtype=dt, **dev)
    # neighbouring rows of a sequence have keys alike
    st["K"].mul_(0.6).add_(torch.randn((n_pages,) + ((H, 1, D) if case["heads_first"] else (1, H, D)), dtype=dt, **dev).mul_(0.8))
    if not case["heads_first"]:
        st["K"], st["V"] = st["K"].transpose(1, 2), st["V"].transpose(1, 2)
    # most rows stand for one token, merged ones for some, as the reduction leaves them
    st["logw"] = torch.log(torch.floor(1 + 0.5 * torch.rand(n_pages, page, **dev).pow(-0.7))) if case["sizes"] else None
    st["bounds"] = st["w_max"] = None
    if case["call"] == "copy":
        if case["bounds"]:
            st["bounds"] = torch.stack([st["K"].amin(2), st["K"].amax(2)], 2)
            st["w_max"] = st["logw"].amax(1) if case["sizes"] else torch.zeros(n_pages, device="cuda")
        n = case["pages"]
        copies = np.full((n + 5, 3), -1, np.int32)     # the list has room for a few more
        copies[:n, 0], copies[:n, 1], copies[:n, 2] = perm[:n], perm[n:2 * n], _copied_rows(case)
        st.update(copies=i32(copies), n_copies=i32([n]))
        return st
    width = max(1, max(pages_of)) + 1
    table, at = np.full((B, width), -1, np.int32), 0
    for b, n in enumerate(pages_of):
        table[b, :n] = perm[at:at + n]
        at += n
    starts = [b * case["stride"] for b in range(B)] if case["stride"] else np.concatenate([[0], np.cumsum(new)])
    n_rows = B * case["stride"] if case["stride"] else sum(new) + 5               # a captured step has room for a few rows more
    st.update(table=i32(table), length=i32(lengths), new=i32(new), start=i32(starts), scale=_scale(case))
    st["q"] = torch.randn(n_rows, case["n_qh"], D, dtype=dt, **dev)
    st["out"] = torch.zeros(n_rows, case["n_qh"], D, dtype=_TYPES[case["out"]], device="cuda")
    st["lse"] = torch.zeros(n_rows, case["n_qh"], device="cuda")
    st["most"] = (max(max(new), 1), max(max(lengths), 1))                         # what the plain form pads to
    return st


def _copied_rows(case):
    rng = random.Random(case["pages"])
    return [case["page"] if case["kind"] == "whole" else rng.randint(1, case["page"] - 1) for _ in range(case["pages"])]


# ---- the framework's calls ------------------------------------------------------------------------------------------

@functools.lru_cache(maxsize=None)
def _context(n_qh, n_kvh, d_h, dtype, out):
    """The context that a serving program keeps for its model."""
    from paper_2504_08966_b200 import binding as pb
    return pb.Context(n_qh * d_h, n_qh, n_kvh, d_h, _TYPES[dtype], _TYPES[out])


def _call(st):
    case = st["case"]
    ctx = _context(case["n_qh"], case["n_kvh"], case["d_h"], case["dtype"], case["out"])
    if case["call"] == "fork":
        ctx.pact_cache_fork(st["page"], st["table"], st["length"], st["source"], st["shared"], st["free"], st["n_free"], st["table_out"], st["length_out"],
                            st["shared_out"], st["free_out"], st["n_free_out"], st["copies"], st["n_copies"], rows=st["rows"], status=st["status"])
        return {k: st[k] for k in ("table_out", "length_out", "shared_out", "free_out", "n_free_out", "copies", "n_copies", "status")}
    if case["call"] == "compact":
        ctx.pact_cache_compact(st["page"], st["table"], st["length"], st["shared"], st["free"], st["n_free"], st["table_out"], st["shared_out"], st["free_out"],
                               st["moved_to"], st["copies"], st["n_copies"], status=st["status"])
        return {k: st[k] for k in ("table_out", "shared_out", "free_out", "moved_to", "copies", "n_copies", "status")}
    cache = st.get("cache")
    if cache is None:                                  # the handle that a program keeps beside a layer's cache
        from paper_2504_08966_b200 import binding as pb
        cache = st["cache"] = pb.PagedCache(st["K"], st["V"], st["logw"], st["bounds"], st["w_max"])
    if case["call"] == "copy":
        ctx.pact_page_copy(cache, st["copies"], st["n_copies"], status=st["status"])
        return {k: st[k] for k in ("K", "V", "logw", "bounds", "w_max", "status")}
    ctx.pact_chunk_attention(cache, st["q"], st["table"], st["length"], st["new"], st["out"], row_start=None if case["stride"] else st["start"],
                             row_stride=case["stride"], lse=st["lse"], causal=case["causal"], scale=st["scale"], status=st["status"])
    return {"out": st["out"], "lse": st["lse"], "status": st["status"]}


# ---- the plain forms ---------------------------------------------------------------------------------------------------

def _chunk(st):
    """softmax(scale q.k + logw) v of every new token over the rows up to its own, or over all."""
    q, K, V, page, table, length, new = st["q"], st["K"], st["V"], st["page"], st["table"].long(), st["length"].long(), st["new"].long()
    n_rows, n_qh, D = q.shape
    B, H = table.shape[0], K.shape[1]
    n, L = st["most"]
    i, p = torch.arange(n, device=q.device), torch.arange(L, device=q.device)
    row = st["start"][:B, None].long() + i
    there = i < new[:, None]
    x = q[torch.where(there, row, 0)].float().view(B, n, H, -1, D).permute(0, 2, 3, 1, 4).reshape(B, H, -1, D)      # [B, H, heads x tokens, D]
    at, place = table[:, p // page].clamp(min=0), p % page
    k, v = (X[at, :, place].transpose(1, 2).float() for X in (K, V))
    seen = (p < length[:, None])[:, None, :]
    if st["case"]["causal"]:
        seen = seen & (p <= (length - new)[:, None, None] + i[:, None])
    s = (x * st["scale"]) @ k.transpose(2, 3)
    s = s.view(B, H, -1, n, L)
    if st["logw"] is not None:
        s += st["logw"][at, place][:, None, None, None]
    s.masked_fill_(~seen[:, None, None], -math.inf)
    m = s.amax(4, keepdim=True).clamp(min=-3e38)
    s.sub_(m).exp_()
    total = s.sum(4, keepdim=True)
    v = torch.where((p < length[:, None])[:, None, :, None], v, 0.0)
    out = (s.view(B, H, -1, L) @ v).view(B, H, -1, n, D) / torch.where(total > 0, total, 1.0)
    lse = (m + torch.log(total)).squeeze(4)
    # rows of no token stay as they are
    to = torch.where(there, row, n_rows).reshape(-1)
    o, l = (torch.cat([t, t[:1]]) for t in (st["out"], st["lse"]))
    o[to] = out.permute(0, 3, 1, 2, 4).reshape(B * n, n_qh, D).to(o.dtype)
    l[to] = lse.permute(0, 3, 1, 2).reshape(B * n, n_qh)
    return {"out": o[:n_rows], "lse": l[:n_rows], "status": st["status"]}


def _fork(st):
    """Every request becomes the first `rows` rows of what its source was.  A page that ends up part-filled is kept by the first request of those that want it if
    nobody else holds it; the others copy it to pages of their own."""
    page, table, length, source, shared, free, n_free = st["page"], st["table"].long(), st["length"].long(), st["source"].long(), st["shared"], st["free"], st["n_free"].long()
    rows = torch.where(source >= 0, st["rows"].long(), 0)
    B, width = table.shape
    P = shared.numel()
    j, b = torch.arange(width, device=table.device), torch.arange(B, device=table.device)
    old = j < ((length + page - 1) // page)[:, None]
    mine = table[source.clamp(min=0)]
    full = j < (rows // page)[:, None]
    tail = rows % page > 0
    tail_page = torch.where(tail, mine.gather(1, (rows // page)[:, None]).squeeze(1), P)
    count = lambda mask, ids: torch.zeros(P + 1, dtype=torch.long, device=ids.device).scatter_add(0, torch.where(mask, ids, P).reshape(-1), mask.long().reshape(-1))   # noqa: E731
    held, fulls = count(old, table), count(full, mine)
    outside = torch.where(held[:P] > 0, shared + 1 - held[:P], 0)
    first_tail = torch.full((P + 1,), B, device=table.device).scatter_reduce(0, tail_page, b, "amin")
    keeps = tail & (first_tail[tail_page] == b) & (fulls[tail_page] == 0) & (torch.nn.functional.pad(outside, (0, 1))[tail_page] == 0)
    now = outside + fulls[:P] + count(keeps, tail_page)[:P]
    # pages that nobody holds any more, in the order of their first places in the old tables
    line = (b[:, None] * width + j).reshape(-1)
    first = torch.full((P + 1,), B * width, device=table.device).scatter_reduce(0, torch.where(old, table, P).reshape(-1), torch.where(old.reshape(-1), line, B * width), "amin")
    gone = (old & (first[torch.where(old, table, P)] == line.view(B, width)) & (now[table.clamp(min=0)] == 0)).reshape(-1)
    F = gone.sum()
    stack = torch.cat([free, torch.zeros(B * width + 1, dtype=torch.int32, device=free.device)])
    stack = stack.scatter(0, torch.where(gone, n_free + gone.cumsum(0) - 1, stack.numel() - 1), table.reshape(-1).int())
    copies = tail & ~keeps
    k = copies.cumsum(0) - 1
    C = copies.sum()
    fresh = stack[torch.where(copies, n_free + F - 1 - k, 0)].long()
    last = torch.where(keeps, tail_page, fresh)
    out = torch.where(full, mine, torch.where(tail[:, None] & (j == (rows // page)[:, None]), last[:, None], -1))
    left = n_free + F - C
    i = torch.arange(P, device=free.device)
    to = torch.where(copies, k, B)
    listed_ = torch.tensor([-1, -1, 0], device=table.device).repeat(B + 1, 1)
    listed_[to] = torch.stack([tail_page, fresh, rows % page], 1)
    return {"table_out": out.int(), "length_out": rows.int(), "shared_out": torch.where(held[:P] > 0, (now - 1).clamp(min=0).int(), shared),
            "free_out": torch.where(i < left, stack[:P], -1), "n_free_out": left.int(), "copies": listed_[:B].int(), "n_copies": C.int().reshape(1), "status": st["status"]}


def _copy(st):
    """Rows of pages onto others, with the biases and the bounds."""
    K, V = st["K"], st["V"]
    c = st["copies"].long()
    c = c[torch.arange(c.shape[0], device=c.device) < st["n_copies"]]
    src, dst, n = c.unbind(1)
    row = torch.arange(st["page"], device=c.device)
    take = row < n[:, None]
    for X in (K, V):
        X[dst] = torch.where(take[:, None, :, None], X[src], X[dst])
    if st["logw"] is not None:
        st["logw"][dst] = torch.where(take, st["logw"][src], st["logw"][dst])
    if st["bounds"] is not None:
        st["bounds"][dst], st["w_max"][dst] = st["bounds"][src], st["w_max"][src]
    return {k: st[k] for k in ("K", "V", "logw", "bounds", "w_max", "status")}


def _compact(st):
    """The k-th used page beyond the first n_used ids goes to the k-th free one among them."""
    table, shared, free, n_free, page = st["table"].long(), st["shared"], st["free"].long(), st["n_free"].long(), st["page"]
    P, room = shared.numel(), st["copies"].shape[0]
    i = torch.arange(P, device=free.device)
    used = torch.ones(P + 1, dtype=torch.bool, device=free.device)
    used[torch.where(i < n_free, free, P)] = False
    used = used[:P]
    n_used = P - n_free
    stray, hole = used & (i >= n_used), ~used & (i < n_used)
    rank = torch.where(stray, stray.cumsum(0) - 1, room)
    place = torch.where(hole, hole.cumsum(0) - 1, room)
    from_, to = (torch.full((room + 1,), -1, device=free.device).scatter(0, x, torch.where(m, i, -1)) for x, m in ((rank, stray), (place, hole)))
    from_[room] = to[room] = -1
    moved = torch.where(stray, to[rank], i)
    M = stray.sum()
    old = torch.arange(table.shape[1], device=free.device) < ((st["length"].long() + page - 1) // page)[:, None]
    table = torch.where(old, moved[table.clamp(min=0)], -1)
    given = torch.zeros_like(shared).scatter_add(0, torch.where(stray, moved, 0), torch.where(stray, shared, 0))
    shared = torch.where(hole, given, torch.where(stray, 0, shared))
    copies = torch.stack([from_, to, torch.where(from_ >= 0, page, 0)], 1)[:room]
    return {"table_out": table.int(), "shared_out": shared, "free_out": torch.where(i < n_free, P - 1 - i, -1).int(), "moved_to": moved.int(), "copies": copies.int(),
            "n_copies": M.int().reshape(1), "status": st["status"]}


_PLAIN = {"chunk": _chunk, "fork": _fork, "copy": _copy, "compact": _compact}


def run(st):
    if own:
        return _call(st)
    return _PLAIN[st["case"]["call"]](st)


# ---- the same from the definitions, in 64 bits ---------------------------------------------------------------------------

def exact(case, seed):
    if case["call"] in ("fork", "compact"):            # whole numbers
        return None
    st = prepare(case, seed)
    page = st["page"]
    if case["call"] == "copy":
        got = {k: None if st[k] is None else st[k].double() for k in ("K", "V", "logw", "bounds", "w_max")}
        for src, dst, n in st["copies"].tolist()[:case["pages"]]:
            got["K"][dst, :, :n], got["V"][dst, :, :n] = got["K"][src, :, :n].clone(), got["V"][src, :, :n].clone()
            if got["logw"] is not None:
                got["logw"][dst, :n] = got["logw"][src, :n].clone()
            if got["bounds"] is not None:
                got["bounds"][dst], got["w_max"][dst] = got["bounds"][src].clone(), got["w_max"][src].clone()
        return dict(got, status=None)
    n_qh, H, D = case["n_qh"], case["n_kvh"], case["d_h"]
    out, lse = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda"), torch.zeros(st["lse"].shape, dtype=torch.float64, device="cuda")
    group, table, starts = n_qh // H, st["table"].long(), st["start"].tolist()
    for b, (L, n) in enumerate(zip(_lengths(case), _new(case))):
        if not n:
            continue
        ids = table[b, :-(-L // page)]
        w = None if st["logw"] is None else st["logw"][ids].reshape(-1)[:L].double()
        at = slice(starts[b], starts[b] + n)
        ahead = torch.arange(L, device="cuda") > torch.arange(L - n, L, device="cuda")[:, None] if case["causal"] else None
        for h in range(n_qh):
            k, v = (X[ids, h // group].reshape(-1, D)[:L].double() for X in (st["K"], st["V"]))
            s = (st["q"][at, h].double() @ k.T) * st["scale"]
            if w is not None:
                s = s + w
            if ahead is not None:
                s = s.masked_fill(ahead, -math.inf)
            lse[at, h] = torch.logsumexp(s, 1)
            out[at, h] = torch.softmax(s, 1) @ v
    return {"out": out, "lse": lse, "status": None}


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------

def work(case):
    e, oe = 2 if case["dtype"] == "bf16" else 4, 2 if case["out"] == "bf16" else 4
    B, page, H, D, Q = case["B"], case["page"], case["n_kvh"], case["d_h"], case["n_qh"]
    pages = lambda n: -(-n // page)                    # noqa: E731
    if case["call"] == "copy":
        rows, n = sum(_copied_rows(case)), case["pages"]
        return {"bytes": 12.0 * n + rows * (4.0 * H * D * e + (8.0 if case["sizes"] else 0.0)) + (n * 2.0 * (2.0 * H * D * e + 4.0) if case["bounds"] else 0.0), "flops": 0.0}
    if case["call"] == "chunk":
        lengths, new = _lengths(case), _new(case)
        rows, seen = sum(new), sum(L for L, n in zip(lengths, new) if n)
        pairs = sum(n * L - (n * (n - 1) // 2 if case["causal"] else 0) for L, n in zip(lengths, new))
        return {"bytes": seen * (2.0 * H * D * e + (4.0 if case["sizes"] else 0.0)) + 4.0 * sum(pages(L) for L, n in zip(lengths, new) if n) +
                rows * Q * (D * (e + oe) + 4.0) + 12.0 * B, "flops": 4.0 * D * Q * pairs}
    lengths, table, extra = _holders(case)
    named = sum(pages(n) for n in lengths)
    if case["call"] == "fork":
        source, rows = _sources(case, lengths)
        # tables in and out, holders of every page that is named in and out, lengths, sources, rows and new lengths, copies
        return {"bytes": 4.0 * named + 4.0 * sum(map(pages, rows)) + 8.0 * len(extra) + 16.0 * B + 12.0 * sum(1 for n in rows if n % page), "flops": 2.0 * named}
    free = case["pages"] - len(extra)
    # the stack in and out, tables in and out, where each page went, copies and holders of what moves (about free * used / all of them)
    return {"bytes": 8.0 * free + 8.0 * named + 4.0 * case["pages"] + 24.0 * free * len(extra) / case["pages"], "flops": 2.0 * named}
