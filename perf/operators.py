"""The operators that follow the reduction while a model answers: the paged cache of keys, values and attention biases that the
reduced sequence is kept in, and the attention of one new token over it, as measurable cases.

Keys of a case
    call     "plan" (pact_cache_plan: block tables and slots of the rows that come next), "write" (pact_cache_write: rows into
             their slots, bounds of the pages' keys), "select" (pact_page_select: the pages that a query may need most), "attend"
             (pact_paged_attention)
    B, rows  requests, and cached rows of the longest one; `ragged`: the requests differ in length, one holds a single row and, from
             eight requests on, one holds none
    page     rows of a page
    n_qh, n_kvh, d_h   query heads, key heads, head width
    dtype, out         element types of the cache and the query, and of the attention's result ("bf16" or "fp32")
    new      "plan" and "write": rows that come next for every request (1: a decoding step), or 0 for whole prompts
    stride   "plan" and "write": 0 for packed new rows, else the rows that each request has room for in the input
    sizes    the cached rows carry the log of a cluster size, which the attention adds to the logits
    bounds   "write": the cache keeps bounds of its pages' keys
    keep     "select": pages to select; "attend": attend to that many selected pages only (0: to all rows)
    heads_first   order of a page's axes: key heads before rows, or rows before key heads
"""
import functools
import math
import random

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}

_BASE = {"call": "attend", "B": 1, "rows": 2500, "ragged": False, "page": 64, "n_qh": 28, "n_kvh": 4, "d_h": 128, "dtype": "bf16",
         "out": "bf16", "new": 1, "stride": 0, "sizes": True, "bounds": True, "keep": 0, "heads_first": True}


def _case(name=None, **kw):
    c = dict(_BASE, **kw)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # the bookkeeping of one decoding step of 128 chats, a few of which have ended: latency is all there is
        _case("plan_decode_128", call="plan", B=128, rows=8192, ragged=True, new=1),
        # the reduced prompts of 48 requests with many images enter a cache of small pages
        _case("plan_prompts_48", call="plan", B=48, rows=5000, ragged=True, new=0, page=16),
        # one layer's new row of 128 chats
        _case("write_decode_128", call="write", B=128, rows=8192, ragged=True, new=1, n_qh=32, n_kvh=8),
        # one layer's rows of 16 reduced prompts, as they lie in the padded output of the reduction
        _case("write_prompts_16", call="write", B=16, rows=2948, ragged=True, new=0, stride=2948, n_qh=4),
        # one short chat on a small fp32 model: the smallest call
        _case("attend_tiny_fp32", rows=212, n_qh=2, n_kvh=2, d_h=64, page=16, dtype="fp32", out="fp32"),
        # one chat about one large image after its reduction
        _case("attend_one_2500", rows=2500),
        # a batch of chats in a cache of small pages, rows before heads, the result in fp32
        _case("attend_batch_48", B=48, rows=4097, ragged=True, page=16, out="fp32", heads_first=False),
        # one very long context (hours of video)
        _case("attend_long_262144", rows=262144, n_qh=32, n_kvh=8),
        # the largest call: a full server
        _case("attend_batch_128", B=128, rows=8192, ragged=True, n_qh=32, n_kvh=8),
        # the pages that matter to the next token of two long videos
        _case("select_2x131072", call="select", B=2, rows=131072, keep=64),
        # the same for a batch on a model with more key heads and smaller pages
        _case("select_batch_32", call="select", B=32, rows=16384, ragged=True, page=32, n_qh=32, n_kvh=8, keep=128),
        # attention to the selected eighth of 32 long contexts
        _case("attend_selected_32", B=32, rows=32768, ragged=True, n_qh=32, n_kvh=8, keep=64),
    ]


# (n_qh, n_kvh, d_h) of the models a caller may bring
_MODELS = [(2, 2, 64), (14, 2, 64), (16, 4, 128), (4, 4, 128), (28, 4, 128), (32, 8, 128), (32, 8, 80)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """One more case of the same ranges."""
    call = rng.choices(["attend", "plan", "write", "select"], [50, 14, 18, 18])[0]
    n_qh, n_kvh, d_h = rng.choices(_MODELS, [1, 1, 1, 1, 3, 3, 1])[0]
    B = rng.choices([1, _log_int(rng, 2, 128)], [1, 2])[0]
    kw = {"call": call, "n_qh": n_qh, "n_kvh": n_kvh, "d_h": d_h, "B": B, "ragged": B > 1 and rng.random() < 0.8,
          "page": rng.choice([16, 32, 64, 128]), "sizes": rng.random() < 0.8, "heads_first": rng.random() < 0.7}
    if rng.random() < 0.2:
        kw.update(dtype="fp32", out="fp32")
    elif rng.random() < 0.2:
        kw["out"] = "fp32"
    most = 128 * 5120 * 8 * 128 * 2 // (B * n_kvh * d_h * (4 if kw.get("dtype") == "fp32" else 2))   # bytes of the largest case
    if call == "plan":
        kw["new"] = rng.choice([0, 1, 1, rng.randint(2, 9)])
        kw["rows"] = _log_int(rng, 2, 8192 if kw["new"] else 240000 // B)
        kw["stride"] = 0 if rng.random() < 0.5 else kw["new"] or kw["rows"] + rng.randint(0, 70)
    elif call == "write":
        kw["new"] = rng.choice([0, 1, 1, rng.randint(2, 9)])
        kw["rows"] = _log_int(rng, 2, min(8192, most) if kw["new"] else 60000 // B)
        kw["stride"] = 0 if rng.random() < 0.5 else kw["new"] or kw["rows"] + rng.randint(0, 70)
        kw["bounds"] = rng.random() < 0.7
    elif call == "select":
        kw["rows"] = _log_int(rng, 4 * kw["page"], min(131072, most))
        kw["keep"] = rng.randint(2, min(128, 3 * kw["rows"] // (4 * kw["page"])))
    else:
        kw["rows"] = _log_int(rng, 1, min(262144, most))
        kw["keep"] = rng.randint(2, 128) if rng.random() < 0.3 else 0
    return _case(**kw)


# ---- inputs ------------------------------------------------------------------------------------------------------

def _lengths(case):
    """Rows of each request: in the cache, or with new = 0 those that enter it."""
    B, rows = case["B"], case["rows"]
    if not case["ragged"]:
        return [rows] * B
    n = [max(1, rows - (rows * 3 * b) // (4 * B) - b % 7) for b in range(B)]
    n[-1] = 1
    if B >= 8:
        n[-2] = 0
    random.Random(B).shuffle(n)
    return n


def _before_and_new(case):
    """Rows that each request of a "plan" or "write" has in the cache already, and how many it gets; -1: it has ended."""
    n = _lengths(case)
    if case["new"]:
        ended = 16 if case["call"] == "plan" else len(n) + 1
        return n, [-1 if b % ended == ended - 1 else case["new"] for b in range(len(n))]
    return [21 if b % 3 == 2 else 0 for b in range(len(n))], n       # some prompts go on from an earlier turn


def _scale(case):
    return float(np.float32(1.0 / math.sqrt(case["d_h"])))


def _block_table(pages, width, n_pages, perm):
    """[B, width] page ids in the order of `perm`, -1 where a request has no page yet, and the ids that are left over."""
    table = np.full((len(pages), width), -1, np.int32)
    start = np.concatenate([[0], np.cumsum(pages)])
    for b, n in enumerate(pages):
        table[b, :n] = perm[start[b]:start[b] + n]
    return table, perm[start[-1]:n_pages]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dev = {"device": "cuda", "generator": g}
    B, page, H, D, dt = case["B"], case["page"], case["n_kvh"], case["d_h"], _TYPES[case["dtype"]]
    i32 = lambda v: torch.tensor(np.asarray(v, np.int32), device="cuda")   # noqa: E731
    st = {"case": case, "page": page, "status": i32([0])}
    adds = case["call"] in ("plan", "write")
    before, new = _before_and_new(case) if adds else (_lengths(case), [0] * B)
    after = [n + max(0, m) for n, m in zip(before, new)]
    pages_of = lambda n: [-(-v // page) for v in n]                        # noqa: E731
    width = max(1, max(pages_of(after))) + 1
    n_pages = sum(pages_of(after)) + B + 64
    perm = torch.randperm(n_pages, **dev).cpu().numpy().astype(np.int32)
    table, left = _block_table(pages_of(before if case["call"] == "plan" else after), width, n_pages, perm)
    st["table"] = torch.from_numpy(table).cuda()
    st["length"], st["new"] = i32(before), i32(new)
    packed = sum(max(0, m) for m in new)
    n_rows = B * case["stride"] if case["stride"] else packed + 5          # a captured step has room for a few rows more
    if case["call"] == "plan":
        free = np.full(n_pages, -1, np.int32)
        free[:len(left)] = left
        st.update(free=i32(free), n_free=i32([len(left)]), length_out=i32([0] * B), n_free_out=i32([0]), row_start=i32([0] * (B + 1)),
                  slot=torch.zeros(n_rows, dtype=torch.int64, device="cuda"), free0=i32(free), table0=st["table"].clone())
        return st
    shape = (n_pages, H, page, D) if case["heads_first"] else (n_pages, page, H, D)
    st["K"], st["V"] = torch.randn(shape, dtype=dt, **dev), torch.randn(shape, dtype=dt, **dev)
    # neighbouring rows of a sequence have keys alike
    st["K"].mul_(0.6).add_(torch.randn((n_pages,) + ((H, 1, D) if case["heads_first"] else (1, H, D)), dtype=dt, **dev).mul_(0.8))
    if not case["heads_first"]:
        st["K"], st["V"] = st["K"].transpose(1, 2), st["V"].transpose(1, 2)
    # most rows stand for one token, merged ones for some, as the reduction leaves them
    sizes = lambda *s: torch.log(torch.floor(1 + 0.5 * torch.rand(*s, **dev).pow(-0.7)))   # noqa: E731
    st["logw"] = sizes(n_pages, page) if case["sizes"] else None
    with_bounds = case["bounds"] if case["call"] == "write" else case["call"] == "select"
    st["bounds"] = st["w_max"] = None
    if with_bounds:                                    # over whole pages: a page that is filled up in part has looser ones
        st["bounds"] = torch.stack([st["K"].amin(2), st["K"].amax(2)], 2)
        st["w_max"] = st["logw"].amax(1) if case["sizes"] else torch.zeros(n_pages, device="cuda")
    if case["call"] == "write":
        slot = np.full(n_rows, -1, np.int64)
        at = 0
        for b, m in enumerate(new):
            p = before[b] + np.arange(m)
            first = b * case["stride"] if case["stride"] else at
            slot[first:first + m] = table[b, p // page].astype(np.int64) * page + p % page
            at += m
        st["slot"] = torch.from_numpy(slot).cuda()
        st["K_new"], st["V_new"] = torch.randn(n_rows, H, D, dtype=dt, **dev), torch.randn(n_rows, H, D, dtype=dt, **dev)
        st["logw_new"] = sizes(n_rows) if case["sizes"] else None
        return st
    st["scale"] = _scale(case)
    st["q"] = torch.randn(B, case["n_qh"], D, dtype=dt, **dev)
    if case["call"] == "select":
        st["selected"] = torch.zeros(B, H, case["keep"], dtype=torch.int32, device="cuda")
        return st
    st["out"] = torch.zeros(B, case["n_qh"], D, dtype=_TYPES[case["out"]], device="cuda")
    st["lse"] = torch.zeros(B, case["n_qh"], device="cuda")
    st["selected"] = None
    if case["keep"]:                                   # ascending, -1 behind the last; the first and the last page among them
        n = i32(pages_of(before))[:, None, None]
        at = torch.arange(width, device="cuda").expand(B, H, width)
        key = torch.rand(B, H, width, **dev)
        key = torch.where((at == 0) | (at == n - 1), 2.0, torch.where(at < n, key, -1.0))
        key, at = key.topk(min(case["keep"], width), dim=2)
        at = torch.where(key >= 0, at, 1 << 30).sort(2).values.int()
        at = torch.where(at < 1 << 30, at, -1)
        st["selected"] = torch.nn.functional.pad(at, (0, case["keep"] - at.shape[2]), value=-1)
    return st


# ---- the framework's calls ------------------------------------------------------------------------------------------

@functools.lru_cache(maxsize=None)
def _context(n_qh, n_kvh, d_h, dtype, out):
    """The context that a serving program keeps for its model."""
    from paper_2504_08966_b200 import binding as pb
    return pb.Context(n_qh * d_h, n_qh, n_kvh, d_h, _TYPES[dtype], _TYPES[out])


def _call(st):
    case = st["case"]
    ctx = _context(case["n_qh"], case["n_kvh"], case["d_h"], case["dtype"], case["out"])
    if case["call"] == "plan":
        ctx.pact_cache_plan(st["page"], st["table"], st["length"], st["new"], st["free"], st["n_free"], st["length_out"], st["n_free_out"],
                            st["row_start"], st["slot"], row_stride=case["stride"], status=st["status"])
        return {k: st[k] for k in ("table", "length_out", "free", "n_free_out", "row_start", "slot", "status")}
    cache = st.get("cache")
    if cache is None:                                  # the handle that a program keeps beside a layer's cache
        from paper_2504_08966_b200 import binding as pb
        cache = st["cache"] = pb.PagedCache(st["K"], st["V"], st["logw"], st["bounds"], st["w_max"])
    if case["call"] == "write":
        ctx.pact_cache_write(cache, st["K_new"], st["V_new"], st["logw_new"], st["slot"], status=st["status"])
        return {k: st[k] for k in ("K", "V", "logw", "bounds", "w_max", "status")}
    if case["call"] == "select":
        ctx.pact_page_select(cache, st["q"], st["table"], st["length"], st["selected"], scale=st["scale"], status=st["status"])
        return {"selected": st["selected"], "status": st["status"]}
    ctx.pact_paged_attention(cache, st["q"], st["table"], st["length"], st["out"], lse=st["lse"], selected=st["selected"], scale=st["scale"],
                             status=st["status"])
    return {"out": st["out"], "lse": st["lse"], "status": st["status"]}


# ---- the plain forms ---------------------------------------------------------------------------------------------------

def _plan(st):
    """Pages and slots of the new rows.  Free pages are a stack; ended requests (new < 0) push theirs, in the order of the requests, before
    any page is taken.  A call that asks for too much changes nothing."""
    page, stride, table, length, new = st["page"], st["case"]["stride"], st["table0"], st["length"].long(), st["new"].long()
    free, n_free, n_rows = st["free0"], st["n_free"].long(), st["slot"].numel()
    B, width = table.shape
    ended, add = new < 0, new.clamp(min=0)
    had = (length + page - 1) // page
    need = torch.where(ended, 0, (length + add + page - 1) // page - had)
    freed = torch.where(ended, had, 0)
    F, A = freed.sum(), need.sum()
    start = torch.cat([torch.zeros_like(n_free), add.cumsum(0)])
    fits = (add <= stride).all() if stride else start[-1] <= n_rows
    ok = fits & (A <= n_free + F).all() & (torch.where(ended, 0, length + add) <= width * page).all()
    j = torch.arange(width, device=table.device)
    gives = ended[:, None] & (j < had[:, None])
    at = torch.where(gives, (freed.cumsum(0) - freed)[:, None] + j + n_free, free.numel() + width * B)
    stack = torch.cat([free, torch.zeros(width * B + 1, dtype=torch.int32, device=table.device)])
    stack = stack.scatter(0, at.reshape(-1), table.reshape(-1))
    takes = ok & (j >= had[:, None]) & (j < (had + need)[:, None])
    k = (need.cumsum(0) - need)[:, None] + j - had[:, None]
    table = torch.where(takes, stack[torch.where(takes, n_free + F - 1 - k, 0)], table)
    left = torch.where(ok, n_free + F - A, n_free)
    i = torch.arange(free.numel(), device=table.device)
    free = torch.where((i >= n_free) & (i < left), stack[:free.numel()], free)
    r = torch.arange(n_rows, device=table.device)
    if stride:
        b = r // stride
        p = r - b * stride
    else:
        b = torch.searchsorted(start[1:].contiguous(), r, right=True).clamp(max=B - 1)
        p = r - start[b]
    valid = ok & (p < add[b])
    p = p + length[b]
    slot = torch.where(valid, table[b, torch.where(valid, p // page, 0)].long() * page + p % page, -1)
    return {"table": table, "length_out": torch.where(ok, torch.where(ended, 0, length + add), length).int(), "free": free,
            "n_free_out": left.int(), "row_start": torch.where(ok, start, 0).int(), "slot": slot, "status": st["status"]}


def _write(st):
    """Rows into their slots; a page whose first row is written begins new bounds, others are widened."""
    K, V, page = st["K"], st["V"], st["page"]
    rows = (st["slot"] >= 0).nonzero().squeeze(1)
    s = st["slot"][rows]
    at, r = s // page, s % page
    K_new = st["K_new"][rows]
    K[at, :, r], V[at, :, r] = K_new, st["V_new"][rows]
    w = st["logw_new"][rows] if st["logw_new"] is not None else torch.zeros(rows.numel(), device=K.device)
    if st["logw"] is not None:
        st["logw"][at, r] = w
    if st["bounds"] is not None:
        fresh = torch.zeros(K.shape[0], dtype=torch.bool, device=K.device)
        fresh[at[r == 0]] = True
        lo, hi = st["bounds"].float().unbind(2)
        inf = torch.full_like(lo[:1], math.inf)
        lo, hi = torch.where(fresh[:, None, None], inf, lo), torch.where(fresh[:, None, None], -inf, hi)
        lo.index_reduce_(0, at, K_new.float(), "amin")
        hi.index_reduce_(0, at, K_new.float(), "amax")
        st["bounds"].copy_(torch.stack([lo, hi], 2))
        st["w_max"].copy_(torch.where(fresh, -math.inf, st["w_max"]).index_reduce(0, at, w, "amax"))
    return {k: st[k] for k in ("K", "V", "logw", "bounds", "w_max", "status")}


def _select(st):
    """The first and the last page of a request and those that may hold its largest logits: for any key k of a page with bounds lo, hi
    scale q.k + logw <= scale sum_c max(q_c lo_c, q_c hi_c) + w_max.  In 64 bits: the order of the scores decides."""
    B, H, keep = st["selected"].shape
    page, width, D = st["page"], st["table"].shape[1], st["q"].shape[2]
    n = ((st["length"].long() + page - 1) // page)[:, None, None]
    at = st["table"].long().clamp(min=0)
    lo, hi = st["bounds"][at].permute(0, 2, 3, 4, 1).double().unbind(2)           # [B, H, D, width]
    q = st["q"].view(B, H, -1, D).double()
    score = (q.clamp(min=0) @ hi + q.clamp(max=0) @ lo).amax(2) * st["scale"] + st["w_max"][at][:, None].double()
    j = torch.arange(width, device=at.device)
    score = torch.where((j == 0) | (j == n - 1), math.inf, torch.where(j < n, score, -math.inf))
    order = score.sort(stable=True, dim=2, descending=True).indices[:, :, :keep]
    order = torch.where(order < n, order, width).sort(2).values
    order = torch.where(order < width, order, -1).int()
    return {"selected": torch.nn.functional.pad(order, (0, keep - order.shape[2]), value=-1), "status": st["status"]}


def _attend(st):
    """softmax(scale q.k + logw) v over the cached rows of each request, or over those of its selected pages; nothing where there are none."""
    q, K, V, page, sel = st["q"], st["K"], st["V"], st["page"], st["selected"]
    B, n_qh, D = q.shape
    H, T = K.shape[1], st["table"].shape[1]
    if sel is None:
        sel = torch.arange(T, device=q.device, dtype=torch.int32).expand(B, 1, T)
    b, h = torch.arange(B, device=q.device)[:, None, None], torch.arange(H, device=q.device)[None, :, None]
    at = st["table"][b, sel.long().clamp(min=0)].long().clamp(min=0)              # [B, H or 1, pages]
    k, v = (X[at, h].reshape(B, H, -1, D).float() for X in (K, V))
    pos = sel.long()[..., None] * page + torch.arange(page, device=q.device)
    there = ((sel >= 0)[..., None] & (pos < st["length"][:, None, None, None])).flatten(2)[:, :, None]
    s = q.view(B, H, -1, D).float() @ k.transpose(2, 3) * st["scale"]
    if st["logw"] is not None:
        s = s + st["logw"][at].flatten(2)[:, :, None]
    s = torch.where(there, s, -math.inf)
    m = s.amax(3, keepdim=True).clamp(min=-3e38)
    e = torch.exp(s - m)
    total = e.sum(3, keepdim=True)
    v = torch.where(there.transpose(2, 3), v, 0.0)
    out = (e @ v) / torch.where(total > 0, total, 1.0)
    return {"out": out.reshape(B, n_qh, D).to(st["out"].dtype), "lse": (m + torch.log(total)).reshape(B, n_qh), "status": st["status"]}


_PLAIN = {"plan": _plan, "write": _write, "select": _select, "attend": _attend}


def run(st):
    if own:
        return _call(st)
    return _PLAIN[st["case"]["call"]](st)


# ---- the same from the definitions, in 64 bits ---------------------------------------------------------------------------

def exact(case, seed):
    if case["call"] in ("plan", "select"):             # whole numbers
        return None
    st = prepare(case, seed)
    page, table = st["page"], st["table"].cpu().numpy()
    if case["call"] == "write":
        K, V = st["K"].double(), st["V"].double()
        logw = None if st["logw"] is None else st["logw"].double()
        bounds, w_max = (None, None) if st["bounds"] is None else (st["bounds"].double(), st["w_max"].double())
        before, new = _before_and_new(case)
        first = 0
        for b, m in enumerate(new):
            row = b * case["stride"] if case["stride"] else first
            first += m
            p = before[b]
            while p < before[b] + m:                   # page by page
                n = min(page - p % page, before[b] + m - p)
                at, r = int(table[b, p // page]), p % page
                src = slice(row + p - before[b], row + p - before[b] + n)
                k, v = st["K_new"][src].double().transpose(0, 1), st["V_new"][src].double().transpose(0, 1)
                K[at, :, r:r + n], V[at, :, r:r + n] = k, v
                w = torch.zeros(n, dtype=torch.float64, device="cuda") if st["logw_new"] is None else st["logw_new"][src].double()
                if logw is not None:
                    logw[at, r:r + n] = w
                if bounds is not None:
                    lo, hi, top = k.amin(1), k.amax(1), w.max()
                    if r:
                        lo, hi, top = torch.minimum(lo, bounds[at, :, 0]), torch.maximum(hi, bounds[at, :, 1]), torch.maximum(top, w_max[at])
                    bounds[at, :, 0], bounds[at, :, 1], w_max[at] = lo, hi, top
                p += n
        return {"K": K, "V": V, "logw": logw, "bounds": bounds, "w_max": w_max, "status": None}
    B, n_qh, D = st["q"].shape
    H = case["n_kvh"]
    out = torch.zeros(B, n_qh, D, dtype=torch.float64, device="cuda")
    lse = torch.full((B, n_qh), -math.inf, dtype=torch.float64, device="cuda")
    group = n_qh // H
    for b, n in enumerate(_lengths(case)):
        for h in range(H) if n else ():
            which = range(-(-n // page))
            if st["selected"] is not None:
                which = [j for j in st["selected"][b, h].tolist() if j >= 0]
            ids = torch.from_numpy(table[b, list(which)].astype(np.int64)).cuda()
            pos = (torch.tensor(list(which), device="cuda")[:, None] * page + torch.arange(page, device="cuda")).reshape(-1)
            live = pos < n
            k, v = st["K"][ids, h].reshape(-1, D)[live].double(), st["V"][ids, h].reshape(-1, D)[live].double()
            s = (st["q"][b, h * group:(h + 1) * group].double() @ k.T) * st["scale"]
            if st["logw"] is not None:
                s = s + st["logw"][ids].reshape(-1)[live].double()
            lse[b, h * group:(h + 1) * group] = torch.logsumexp(s, 1)
            out[b, h * group:(h + 1) * group] = torch.softmax(s, 1) @ v
    return {"out": out, "lse": lse, "status": None}


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------

def work(case):
    e, oe = 2 if case["dtype"] == "bf16" else 4, 2 if case["out"] == "bf16" else 4
    B, page, H, D, Q = case["B"], case["page"], case["n_kvh"], case["d_h"], case["n_qh"]
    pages = lambda n: -(-n // page)                    # noqa: E731
    if case["call"] in ("plan", "write"):
        before, new = _before_and_new(case)
        add = [max(0, m) for m in new]
        rows, room = sum(add), B * case["stride"] if case["stride"] else sum(add) + 5
        if case["call"] == "plan":
            freed = sum(pages(n) for n, m in zip(before, new) if m < 0)
            taken = sum(pages(n + m) - pages(n) for n, m in zip(before, new) if m >= 0)
            open_pages = sum(1 for n, m in zip(before, new) if m > 0 and n % page)
            # lengths and counts in, new lengths and row starts out, pages given back and taken, tables' open pages, slots out
            return {"bytes": 16.0 * B + 8.0 * freed + 8.0 * taken + 4.0 * open_pages + 8.0 * room, "flops": 4.0 * room + 8.0 * B}
        touched = sum(pages(n + m) - n // page for n, m in zip(before, add) if m)
        opened = sum(1 for n, m in zip(before, add) if m and n % page)
        # slots in; keys, values and biases in and out; bounds out, those of pages that were begun before also in
        return {"bytes": 8.0 * room + rows * (4.0 * H * D * e + (8.0 if case["sizes"] else 0.0)) +
                ((touched + opened) * (2.0 * H * D * e + 4.0) if case["bounds"] else 0.0), "flops": 2.0 * rows * H * D}
    n = _lengths(case)
    if case["call"] == "select":
        p = sum(pages(v) for v in n)
        return {"bytes": p * (2.0 * H * D * e + 8.0) + B * (Q * D * e + 4.0 + 4.0 * H * case["keep"]), "flops": 4.0 * p * Q * D}
    if case["keep"]:                                   # the last page, which may be part full, is always among the selected
        n = [v if pages(v) <= case["keep"] else (case["keep"] - 1) * page + (v - 1) % page + 1 for v in n]
    rows = sum(n)
    ids = H * case["keep"] * 4.0 * B if case["keep"] else 0.0
    return {"bytes": rows * (2.0 * H * D * e + ((H if case["keep"] else 1) * 4.0 if case["sizes"] else 0.0)) + ids + 4.0 * sum(map(pages, n)) +
            B * (Q * D * (e + oe) + 4.0 * Q + 4.0), "flops": 4.0 * rows * Q * D}
