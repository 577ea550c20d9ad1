"""The paged cache on the GPU against its plain float64 implementation (oracle/paged_oracle.py): pages and slots, rows into slots, page
selection, attention of one new token, and all of them in a row behind pact_reduce."""
import itertools

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po

pytestmark = pytest.mark.gpu

BF, F32, I32, I64 = torch.bfloat16, torch.float32, torch.int32, torch.int64


@pytest.fixture(scope="module")
def pb():
    from paper_2504_08966_b200 import binding
    return binding


_ctx = {}


def context(pb, n_qh=8, n_kvh=2, d_h=64, dtype=BF, out=None):
    key = (n_qh, n_kvh, d_h, dtype, out or dtype)
    if key not in _ctx:
        _ctx[key] = pb.Context((n_qh * d_h + 7) // 8 * 8, n_qh, n_kvh, d_h, dtype, out or dtype)
    return _ctx[key]


def i32(v):
    return torch.tensor(np.asarray(v, np.int32), device="cuda")


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


# ---- plan ----------------------------------------------------------------------------------------------------------

def plan_state(rng, B, width, page, n_pages, most_len):
    lens = [int(rng.integers(0, most_len + 1)) for _ in range(B)]
    ids = rng.permutation(n_pages)
    table, at = np.full((B, width), -7, np.int32), 0
    for b in range(B):
        n = po.pages_for(lens[b], page)
        table[b, :n] = ids[at:at + n]
        at += n
    free = np.full(n_pages, -9, np.int32)
    free[:n_pages - at] = ids[at:]
    return lens, table, free, n_pages - at


def run_plan(pb, page, table, lens, new, free, n_free, n_rows, row_stride, in_place, with_slots=True, stride=1):
    ctx = context(pb)
    t, ln, fr, nf, status = i32(table), i32(lens), i32(free), i32([n_free]), i32([0])
    n_new = torch.full((len(lens), stride), -5, dtype=I32, device="cuda")
    n_new[:, 0] = i32(new)
    ln_out, nf_out = (ln, nf) if in_place else (i32([-3] * len(lens)), i32([-3]))
    start = i32([-3] * (len(lens) + 1))
    slot = torch.full((n_rows,), -3, dtype=I64, device="cuda") if with_slots else None
    ctx.pact_cache_plan(page, t, ln, n_new[:, 0], fr, nf, ln_out, nf_out, start, slot, n_rows=None if with_slots else n_rows, row_stride=row_stride, status=status)
    torch.cuda.synchronize()
    if not in_place:
        assert ln.tolist() == list(lens) and nf.item() == n_free
    return status.item(), t.cpu().numpy(), ln_out.tolist(), fr.cpu().numpy(), nf_out.item(), start.tolist(), slot.tolist() if with_slots else None


def check_plan(got, want, free):
    st, table, lens, stack, start, slot = want
    assert got[0] == st
    assert np.array_equal(got[1], table) and got[2] == lens
    assert got[4] == len(stack) and got[3][:len(stack)].tolist() == stack
    assert np.array_equal(got[3][max(len(stack), 0):][got[3][len(stack):] != free[len(stack):]], [])   # above the new top nothing changes
    assert got[5] == start and (got[6] is None or got[6] == slot)


@pytest.mark.parametrize("B,page,most_len,most_new,row_stride", [
    (1, 16, 0, 1, 0), (1, 64, 40, 200, 0), (3, 16, 100, 1, 1), (7, 48, 300, 5, 9), (64, 16, 400, 1, 0), (130, 32, 200, 3, 0), (1500, 16, 60, 2, 0),
    (4096, 16, 20, 1, 0), (5, 1024, 5000, 2500, 0), (6, 16, 40, 2500, 2500), (6, 64, 40, 2500, 2600), (9, 16, 900, 4000, 0)])
@pytest.mark.parametrize("in_place", [False, True])
def test_plan(pb, B, page, most_len, most_new, row_stride, in_place):
    rng = np.random.default_rng(B * 7 + page + most_new)
    width = po.pages_for(most_len + most_new, page) + 1
    lens, table, free, n_free = plan_state(rng, B, width, page, B * width + 3, most_len)
    new = [-1 if rng.random() < 0.2 else 0 if rng.random() < 0.1 else int(rng.integers(1, most_new + 1)) for _ in range(B)]
    n_rows = B * row_stride if row_stride else sum(max(0, m) for m in new) + int(rng.integers(0, 40))
    want = po.plan(page, table, lens, new, free, n_free, n_rows, row_stride)
    assert want[0] == 0
    check_plan(run_plan(pb, page, table, lens, new, free, n_free, n_rows, row_stride, in_place), want, free)
    if B <= 7:
        check_plan(run_plan(pb, page, table, lens, new, free, n_free, n_rows, row_stride, in_place, with_slots=False, stride=16), want, free)


@pytest.mark.parametrize("rows", [40, 9000])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("fault", ["pages", "length", "negative", "room", "n_free", "n_free_high", "stack", "stride"])
def test_a_plan_that_cannot_be_served_changes_nothing(pb, fault, in_place, rows):
    rng = np.random.default_rng(5)
    B, page, width = 4, 16, rows // 16 + 4
    lens, table, free, n_free = plan_state(rng, B, width, page, B * width, 50)
    new, n_rows, row_stride = [rows, 1, -1, 2], rows + 3, 0
    if fault == "pages":
        n_free, lens[2] = 1, 0                         # the request that ends has none to give back
    elif fault == "length":
        lens[1] = width * page
    elif fault == "negative":
        lens[3] = -1
    elif fault == "room":
        n_rows -= 1
    elif fault == "n_free":
        n_free = -1
    elif fault == "n_free_high":
        n_free = len(free) + 1
    elif fault == "stack":
        lens[2], n_free = 50, len(free) - 1
    else:
        row_stride = rows - 1
        n_rows = B * row_stride
    want = po.plan(page, table, lens, new, free, n_free, n_rows, row_stride)
    assert want[0] == (po.NO_PAGES if fault == "pages" else po.INVALID)
    got = run_plan(pb, page, table, lens, new, free, n_free, n_rows, row_stride, in_place)
    assert got[0] == want[0] and np.array_equal(got[1], table) and got[2] == lens and np.array_equal(got[3], free) and got[4] == n_free
    assert got[5] == [0] * (B + 1) and got[6] == [-1] * n_rows


def test_plan_step_after_step_in_a_graph(pb):
    """A captured decoding step: lengths, tables and the free pages live on in the same buffers."""
    ctx, rng, B, page, width = context(pb), np.random.default_rng(1), 6, 16, 8
    lens, table, free, n_free = plan_state(rng, B, width, page, B * width, 40)
    t, ln, fr, nf, new, status = i32(table), i32(lens), i32(free), i32([n_free]), i32([1] * B), i32([0])
    start, slot = i32([0] * (B + 1)), torch.zeros(B, dtype=I64, device="cuda")
    call = lambda: ctx.pact_cache_plan(page, t, ln, new, fr, nf, ln, nf, start, slot, status=status)   # noqa: E731
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    stack = None
    for step in range(30):
        new_now = [int(x) for x in rng.choice([1, 1, 1, 2, 0, -1], B)]
        new.copy_(i32(new_now))
        want = po.plan(page, table, lens, new_now, free, n_free, B)
        g.replay()
        torch.cuda.synchronize()
        assert t.cpu().numpy().tolist() == want[1].tolist() and ln.tolist() == want[2] and slot.tolist() == want[5]
        table, lens, stack = want[1], want[2], want[3]
        free[:len(stack)] = stack
        n_free = len(stack)
        assert nf.item() == n_free and fr.tolist()[:n_free] == stack
        status.zero_()


# ---- write ---------------------------------------------------------------------------------------------------------

def cache_tensors(g, n_pages, H, page, D, dtype, heads_first=True, logw=True, bounds=True):
    shape = (n_pages, H, page, D) if heads_first else (n_pages, page, H, D)
    K, V = (torch.randn(shape, generator=g, device="cuda").to(dtype) for _ in range(2))
    if not heads_first:
        K, V = K.transpose(1, 2), V.transpose(1, 2)
    w = torch.log(torch.randint(1, 30, (n_pages, page), generator=g, device="cuda").float()) if logw else None
    b = torch.stack([K.amin(2), K.amax(2)], 2).contiguous() if bounds else None
    return K, V, w, b, (w.amax(1) if logw else torch.zeros(n_pages, device="cuda")) if bounds else None


def run_slots(rng, n_pages, page, runs):
    """Slots of `runs` (rows, first place) pieces as a plan lays them out: pages drawn without repetition, -1 between some of them."""
    ids, slot = iter(rng.permutation(n_pages)), []
    for rows, place in runs:
        at = None
        for _ in range(rows):
            if at is None or place == page:
                at, place = int(next(ids)), place if at is None else 0
            slot.append(at * page + place)
            place += 1
        if rng.random() < 0.4:
            slot += [-1] * int(rng.integers(1, 5))
    return slot


@pytest.mark.parametrize("dtype,H,D,page,heads_first,logw,bounds,runs", [
    (BF, 2, 64, 16, True, True, True, [(1, 0)]), (BF, 2, 64, 16, True, True, True, [(1, 15), (1, 0), (1, 7)] * 20), (BF, 8, 128, 64, True, True, True, [(1, 3)] * 40),
    (BF, 4, 128, 64, False, True, True, [(300, 0), (1, 5), (77, 21), (64, 0)]), (BF, 1, 8, 48, True, False, True, [(500, 7), (2, 0)]), (BF, 3, 256, 16, True, True, False, [(90, 3)]),
    (BF, 2, 80, 1024, True, True, True, [(1500, 1000), (3, 0)]), (F32, 2, 64, 16, True, True, True, [(5, 14), (40, 0), (1, 1)]), (F32, 4, 100, 32, False, False, False, [(70, 9)]),
    (F32, 1, 128, 128, True, True, True, [(4, 0), (4, 100), (200, 60)]), (BF, 4, 128, 16, True, True, True, [(5000, 3)])])
def test_write(pb, dtype, H, D, page, heads_first, logw, bounds, runs):
    rng, g = np.random.default_rng(D + page), torch.Generator(device="cuda").manual_seed(D + page)
    n_pages = sum(po.pages_for(r + p, page) for r, p in runs) + 5
    K, V, w, b, wm = cache_tensors(g, n_pages, H, page, D, dtype, heads_first, logw, bounds)
    slot = run_slots(rng, n_pages, page, runs)
    n = len(slot)
    # rows of a wider buffer, keys and values beside one another
    kv = torch.randn(n, 2, H, D, generator=g, device="cuda").to(dtype)
    K_new, V_new = kv[:, 0], kv[:, 1]
    lw = torch.randn(n, generator=g, device="cuda") if logw or bounds else None
    want = [f64(x) for x in (K, V, w, b, wm)]
    assert po.write(*want, f64(K_new), f64(V_new), f64(lw), slot, page) == 0
    ctx, status = context(pb, H, H, D, dtype), i32([0])
    ctx.pact_cache_write(pb.PagedCache(K, V, w, b, wm), K_new, V_new, lw, torch.tensor(slot, device="cuda"), status=status)
    torch.cuda.synchronize()
    assert status.item() == 0
    for x, y, what in zip((K, V, w, b, wm), want, ("K", "V", "logw", "bounds", "w_max")):
        assert (x is None and y is None) or np.array_equal(f64(x), y), what


def test_write_without_biases_and_with_bad_slots(pb):
    g = torch.Generator(device="cuda").manual_seed(3)
    K, V, w, b, wm = cache_tensors(g, 6, 2, 16, 64, BF)
    slot = [16, 17, 6 * 16, -1, 5 * 16 + 9, 1 << 40, -(1 << 40)]
    K_new, V_new = (torch.randn(7, 2, 64, generator=g, device="cuda").to(BF) for _ in range(2))
    want = [f64(x) for x in (K, V, w, b, wm)]
    assert po.write(*want, f64(K_new), f64(V_new), None, slot, 16) == po.INVALID
    ctx, status = context(pb, 2, 2, 64), i32([0])
    ctx.pact_cache_write(pb.PagedCache(K, V, w, b, wm), K_new, V_new, None, torch.tensor(slot, device="cuda"), status=status)
    assert status.item() == po.INVALID
    for x, y in zip((K, V, w, b, wm), want):
        assert np.array_equal(f64(x), y)
    ctx.pact_cache_write(pb.PagedCache(K, V, w, b, wm), K_new[:0], V_new[:0], None, torch.zeros(0, dtype=I64, device="cuda"))   # no rows: nothing to do
    assert np.array_equal(f64(K), want[0])


def test_a_cache_without_biases_takes_none(pb):
    # the attention adds nothing then, so neither may the bound of a page: with biases below 0 it would fall below the logits
    g = torch.Generator(device="cuda").manual_seed(8)
    K, V, _, b, wm = cache_tensors(g, 4, 1, 16, 64, F32, logw=False)
    rows, lw = torch.randn(40, 1, 64, generator=g, device="cuda"), -5 - torch.rand(40, generator=g, device="cuda")
    context(pb, 1, 1, 64, F32).pact_cache_write(pb.PagedCache(K, V, None, b, wm), rows, rows, lw, torch.arange(40, device="cuda"))
    assert wm.tolist() == [0, 0, 0, 0]


def test_bounds_leave_out_what_is_not_a_number(pb):
    K, V, w, b, wm = cache_tensors(torch.Generator(device="cuda").manual_seed(4), 3, 1, 16, 64, F32)
    rows = torch.randn(6, 1, 64, device="cuda")
    rows[0, 0, :5] = float("nan")
    rows[3, 0, 3:9] = float("nan")
    rows[4, 0, 20] = float("inf")
    want = np.fmin.reduce(f64(rows), 0), np.fmax.reduce(f64(rows), 0)
    context(pb, 1, 1, 64, F32).pact_cache_write(pb.PagedCache(K, V, w, b, wm), rows, rows, None, torch.arange(16, 22, device="cuda"))
    assert np.array_equal(f64(b)[1, :, 0], want[0]) and np.array_equal(f64(b)[1, :, 1], want[1])


# ---- selection -----------------------------------------------------------------------------------------------------

def tables(rng, lens, width, page, n_pages):
    ids, at = rng.permutation(n_pages), 0
    table = np.full((len(lens), width), -1, np.int32)
    for b, n in enumerate(lens):
        k = po.pages_for(n, page)
        table[b, :k] = ids[at:at + k]
        at += k
    return table


@pytest.mark.parametrize("dtype,n_qh,H,D,page,lens,n_first,n_last,n_select", [
    (BF, 4, 2, 64, 16, [200, 0, 1, 16, 500], 1, 1, 5), (BF, 7, 1, 128, 16, [3000, 2999], 0, 0, 17), (BF, 16, 2, 128, 32, [4000, 33], 2, 3, 64), (BF, 2, 2, 80, 64, [5000], 0, 4, 4),
    (BF, 10, 2, 256, 16, [700], 1, 1, 9), (BF, 3, 3, 8, 48, [9000], 1, 0, 2), (F32, 4, 2, 64, 16, [1500, 40], 1, 1, 20), (F32, 5, 1, 128, 16, [20000], 1, 1, 1000), (F32, 2, 1, 100, 16, [160, 176], 0, 0, 10),
    (BF, 8, 1, 64, 16, [16 * 9000, 100], 1, 1, 700)])
def test_select(pb, dtype, n_qh, H, D, page, lens, n_first, n_last, n_select):
    rng, g = np.random.default_rng(D), torch.Generator(device="cuda").manual_seed(D)
    width = max(po.pages_for(n, page) for n in lens) + 2
    n_pages = sum(po.pages_for(n, page) for n in lens) + 3
    K, V, w, b, wm = cache_tensors(g, n_pages, H, page, D, dtype)
    Q = torch.randn(len(lens), n_qh, D, generator=g, device="cuda").to(dtype)
    table = tables(rng, lens, width, page, n_pages)
    ctx, status = context(pb, n_qh, H, D, dtype), i32([0])
    sel = torch.full((len(lens), H, n_select), -9, dtype=I32, device="cuda")
    ctx.pact_page_select(pb.PagedCache(K, V, w, b, wm), Q, i32(table), i32(lens), sel, n_first, n_last, scale=0.125, status=status)
    want = po.select(f64(Q), f64(b), f64(wm), table, lens, page, 0.125, n_first, n_last, n_select)
    assert status.item() == 0 and np.array_equal(sel.cpu().numpy(), want)


@pytest.mark.parametrize("n,kinds,n_select", [(100, 1, 10), (1500, 1, 700), (1500, 2, 700), (1500, 3, 20), (9000, 2, 4600), (600, 5, 599)])
def test_equal_scores_go_to_the_lower_page(pb, n, kinds, n_select):
    """Pages of few kinds: hundreds of equal scores, more than are ranked by comparing them."""
    rng = np.random.default_rng(n)
    kind = rng.integers(0, kinds, n)
    D, page = 64, 16
    proto = torch.randn(kinds, 1, 2, D, device="cuda").to(BF).sort(2).values
    b = proto[torch.tensor(kind, device="cuda")].contiguous()
    K = torch.zeros(n, 1, page, D, dtype=BF, device="cuda")
    wm = torch.zeros(n, device="cuda")
    Q = torch.randn(1, 4, D, device="cuda").to(BF)
    sel = torch.zeros(1, 1, n_select, dtype=I32, device="cuda")
    table = np.arange(n, dtype=np.int32)[None]
    context(pb, 4, 1, D).pact_page_select(pb.PagedCache(K, K, None, b, wm), Q, i32(table), i32([n * page]), sel, 1, 1, scale=0.125)
    assert np.array_equal(sel.cpu().numpy(), po.select(f64(Q), f64(b), f64(wm), table, [n * page], page, 0.125, 1, 1, n_select))


def test_scores_that_differ_beyond_32_bits(pb):
    """Scores of about 1e4 that differ by 1e-5: equal in 32 bits."""
    n, D, page = 900, 64, 16
    b = torch.zeros(n, 1, 2, D, device="cuda")
    order = torch.randperm(n, device="cuda")
    b[:, 0, :, 0] = 1e4
    b[:, 0, :, 1] = (order.float() * 2.0 ** -17)[:, None]
    K = torch.zeros(n, 1, page, D, device="cuda")
    Q = torch.zeros(1, 1, D, device="cuda")
    Q[..., :2] = 1
    sel = torch.zeros(1, 1, 100, dtype=I32, device="cuda")
    context(pb, 1, 1, D, F32).pact_page_select(pb.PagedCache(K, K, None, b, torch.zeros(n, device="cuda")), Q, torch.arange(n, device="cuda", dtype=I32)[None], i32([n * page]), sel, 0, 0, scale=1.0)
    assert sel[0, 0].tolist() == sorted(order.argsort(descending=True)[:100].tolist())


@pytest.mark.parametrize("dtype,D,k_size,q_size,scale", [(F32, 64, 1e-22, 1e-20, 1.0), (BF, 64, 1e-22, 1e-20, 1.0), (BF, 128, 1e-20, 1e-18, 0.5), (F32, 128, 1.0, 1.0, 1e-43), (BF, 128, 1.0, 1.0, 1e-43), (F32, 100, 1e-25, 1e-20, 1e30)])
def test_scores_below_the_normal_numbers_of_fp32(pb, dtype, D, k_size, q_size, scale):
    """Products of about 1e-38 and far below, which fp32 holds in few bits or not at all."""
    n, page, n_select, g = 700, 16, 90, torch.Generator(device="cuda").manual_seed(D)
    b = (torch.randn(n, 1, 2, D, generator=g, device="cuda") * k_size).to(dtype).sort(2).values.contiguous()
    Q, K, wm = (torch.randn(1, 3, D, generator=g, device="cuda") * q_size).to(dtype), torch.zeros(n, 1, page, D, dtype=dtype, device="cuda"), torch.zeros(n, device="cuda")
    sel, table = torch.zeros(1, 1, n_select, dtype=I32, device="cuda"), torch.arange(n, device="cuda", dtype=I32)[None]
    context(pb, 3, 1, D, dtype).pact_page_select(pb.PagedCache(K, K, None, b, wm), Q, table, i32([n * page]), sel, 1, 1, scale=scale)
    want = po.select(f64(Q), f64(b), f64(wm), table.cpu().numpy(), [n * page], page, float(np.float32(scale)), 1, 1, n_select)
    assert np.array_equal(sel.cpu().numpy(), want)


def test_select_with_bad_pages_lengths_and_scores(pb):
    rng = np.random.default_rng(0)
    n_pages, page, D, width = 40, 16, 64, 12
    K, V, w, b, wm = cache_tensors(torch.Generator(device="cuda").manual_seed(8), n_pages, 1, page, D, BF)
    b[3, 0, 1, 2] = float("nan")                       # a page whose scores are not numbers
    b[4, 0] = float("inf")
    wm[5] = float("-inf")
    Q = torch.randn(4, 2, D, device="cuda").to(BF)
    table = rng.permutation(n_pages)[:width].astype(np.int32)[None].repeat(4, 0)
    table[0, :3] = 3, 4, 5
    table[1, 4], table[1, 6] = -1, n_pages
    ctx = context(pb, 2, 1, D)
    for lens, bad in (([width * page] * 4, True), ([width * page, 0, 100, 5], False), ([-4, 0, 100, width * page + 1], True), ([(1 << 31) - 1, 3, 3, 3], True)):
        status, sel = i32([0]), torch.full((4, 1, 6), -9, dtype=I32, device="cuda")
        ctx.pact_page_select(pb.PagedCache(K, V, w, b, wm), Q, i32(table), i32(lens), sel, 1, 1, scale=0.2, status=status)
        assert status.item() == (po.INVALID if bad else 0)
        assert np.array_equal(sel.cpu().numpy(), po.select(f64(Q), f64(b), f64(wm), table, lens, page, 0.2, 1, 1, 6))


# ---- attention -----------------------------------------------------------------------------------------------------

def attend_and_check(pb, dtype, out_dtype, n_qh, H, D, page, lens, heads_first=True, logw=True, seed=0, poison=False, mask=None, selected=None, table=None, n_pages=None,
                     scale=None, want_status=0, q_strided=False):
    rng, g = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    width = max(max(po.pages_for(max(n, 0), page) for n in lens), 1) + 1
    n_pages = n_pages or sum(po.pages_for(max(n, 0), page) for n in lens) + 2
    K, V, w, _, _ = cache_tensors(g, n_pages, H, page, D, dtype, heads_first, logw, False)
    if table is None:
        table = tables(rng, lens, width, page, n_pages)
    if mask is not None:
        mask(w, table)
    B = len(lens)
    Q = torch.randn(B, n_qh + 1 if q_strided else n_qh, D + (8 if q_strided else 0), generator=g, device="cuda").to(dtype)[:, :n_qh, :D]
    Kc, Vc = f64(K), f64(V)
    if poison:                                         # what must not be seen is not a number
        seen = np.zeros((n_pages, page), bool)
        for b, n in enumerate(lens):
            for x in po.rows_of(table[b], max(0, n), page, n_pages):
                seen[x] = w is None or float(w[x]) != -np.inf
        hide = torch.tensor(~seen, device="cuda")[:, None, :, None]
        bad = torch.tensor([float("nan"), float("inf"), float("-inf")], device="cuda").to(dtype)[torch.randint(0, 3, K.shape, device="cuda", generator=g)]
        K.copy_(torch.where(hide, bad, K))
        V.copy_(torch.where(hide, bad, V))
        if w is not None:
            w.copy_(torch.where(torch.tensor(~seen, device="cuda") & (w != float("-inf")), float("nan"), w))
    scale = D ** -0.5 if scale is None else scale
    scale = float(np.float32(scale))
    sel = None if selected is None else i32(selected)
    buf = torch.full((B, n_qh, D + 8), -5.0, device="cuda").to(out_dtype)   # rows of a wider buffer
    out, lse, status = buf[..., :D], torch.full((B, n_qh), -5.0, device="cuda"), i32([0])
    ctx = context(pb, n_qh, H, D, dtype, out_dtype)
    call = lambda: ctx.pact_paged_attention(pb.PagedCache(K, V, w), Q, i32(table), i32(lens), out, lse, sel, scale=scale, status=status)   # noqa: E731
    call()
    torch.cuda.synchronize()
    assert status.item() == want_status
    assert (buf[..., D:] == -5).all()
    wc = None if w is None else np.nan_to_num(f64(w), nan=0.0, neginf=-np.inf)
    ref, lse_ref, mag, big = po.attend(f64(Q), Kc, Vc, wc, table, lens, page, scale, selected)
    # Logits: a dot product of d_h terms in fp32 (every partial sum off by half a step, tensor cores by a whole one), the scale in 32 bits, the exponent's
    # argument rounded; probabilities: exponential 2^-21, two bf16 terms 2^-16; sums: a term per tile of 64 rows and a dozen to join, each step 2^-22 at most.
    delta = (D + 8) * 2.0 ** -23 * big
    steps = max(max(lens), 0) / 64 + 20
    tol = mag * (2 * delta + 2.0 ** -16 + 2.0 ** -20 + steps * 2.0 ** -21)[..., None] + np.abs(ref) * torch.finfo(out_dtype).eps / 2 + 1e-30
    got, got_lse = f64(out), f64(lse)
    err = np.abs(got - ref)
    assert np.isfinite(got).all() and (err <= tol).all(), (err / tol).max()
    none = lse_ref == -np.inf
    assert np.array_equal(got_lse == -np.inf, none) and not got[none].any()
    err = np.abs(got_lse[~none] - lse_ref[~none])
    assert (err <= (delta + 2.0 ** -20 + steps * 2.0 ** -21 + 2.0 ** -22 * np.abs(lse_ref, where=~none, out=np.zeros_like(lse_ref)))[~none]).all()
    first = out.clone(), lse.clone()
    call()
    assert torch.equal(out, first[0]) and torch.equal(lse, first[1])   # bitwise the same again
    return got


LENS = [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300, 1000]


@pytest.mark.parametrize("n_qh,H,D,page", [(4, 4, 64, 16), (14, 2, 64, 32), (28, 4, 128, 64), (32, 8, 128, 16), (8, 1, 256, 64), (16, 1, 128, 128), (12, 1, 80, 48), (40, 1, 64, 16), (20, 2, 192, 32),
                                           (3, 1, 8, 16), (32, 2, 256, 16), (10, 1, 168, 1024), (2, 2, 24, 80)])
@pytest.mark.parametrize("heads_first", [True, False])
def test_attention_bf16(pb, n_qh, H, D, page, heads_first):
    attend_and_check(pb, BF, F32 if heads_first else BF, n_qh, H, D, page, LENS, heads_first, logw=heads_first or D == 64, seed=D + page, q_strided=not heads_first)


@pytest.mark.parametrize("n_qh,H,D,page", [(2, 2, 64, 16), (14, 2, 64, 32), (8, 2, 128, 64), (9, 1, 100, 16), (4, 1, 96, 128), (32, 2, 32, 48), (3, 3, 4, 16), (17, 1, 128, 16)])
@pytest.mark.parametrize("heads_first", [True, False])
def test_attention_fp32(pb, n_qh, H, D, page, heads_first):
    attend_and_check(pb, F32, F32 if heads_first else BF, n_qh, H, D, page, LENS, heads_first, logw=heads_first, seed=D + page, q_strided=not heads_first)


@pytest.mark.parametrize("dtype,n_qh,H,D,page,lens", [
    (BF, 4, 1, 128, 64, [1]), (BF, 8, 8, 64, 16, [37]), (BF, 28, 4, 128, 64, [40000]), (BF, 8, 1, 128, 128, [70000, 3, 0, 12345]), (BF, 4, 4, 64, 16, [5, 0] * 150), (BF, 2, 1, 64, 16, [0, 0, 0]),
    (BF, 16, 2, 256, 32, [9000, 1, 9001]), (F32, 2, 2, 64, 16, [212]), (F32, 8, 1, 128, 64, [20000, 77]), (F32, 1, 1, 32, 16, list(range(0, 200, 3))), (BF, 8, 2, 64, 16, [(i * 37) % 200 for i in range(700)])])
def test_attention_of_few_and_many_requests(pb, dtype, n_qh, H, D, page, lens):
    attend_and_check(pb, dtype, F32, n_qh, H, D, page, lens, seed=len(lens))


@pytest.mark.parametrize("n_qh,D", [(1, 64), (8, 128), (16, 256)])
def test_fp32_results_of_bf16_rows_have_fp32_probabilities(pb, n_qh, D):
    # Two rows with logits 0 and b (queries 0), values 0 and 1: out = x / (1 + x), x = exp(b), -1 <= b < 0.  In units of 2^-22 of it: the argument b log2 e is off by
    # 2^-24 and 1.44 * 2^-25 at most, so x by 0.3; ex2 by 1; the terms of x, of which an instruction cuts each to 2^-23, by 1.5; 1 + x, its reciprocal and the product by
    # 2^-24 each, 0.75.  In all less than 4: 2^-20.  Probabilities of two bf16 terms would be off by up to 2^-16.
    B, page = 64, 16
    K = torch.zeros(B, 1, page, D, dtype=BF, device="cuda")
    V, w = K.clone(), torch.zeros(B, page, device="cuda")
    V[:, :, 1] = 1
    w[:, 1] = -torch.rand(B, generator=torch.Generator(device="cuda").manual_seed(D), device="cuda")
    out = torch.empty(B, n_qh, D, device="cuda")
    ctx = context(pb, n_qh, 1, D, BF, F32)
    ctx.pact_paged_attention(pb.PagedCache(K, V, w), torch.zeros(B, n_qh, D, dtype=BF, device="cuda"), torch.arange(B, dtype=I32, device="cuda")[:, None], i32([2] * B), out)
    x = np.exp(f64(w)[:, 1])[:, None, None]
    assert np.abs(f64(out) / (x / (1 + x)) - 1).max() <= 2.0 ** -20


@pytest.mark.parametrize("B,n_qh,D,page", [(4096, 1, 64, 16), (64, 8, 256, 16), (1000, 16, 128, 32)])
def test_bf16_results_are_rounded_once(pb, B, n_qh, D, page):
    # Two rows with logits 0 and b (queries 0), values 0 and v: out = v x / (1 + x), x = exp(b), -1 <= b < 0.  In fp32 it is good to 2^-20, as above (v x is three products of eight
    # bits by eight, exact each), so the result is off by half a bf16 step and 2^-20 at most.
    g = torch.Generator(device="cuda").manual_seed(D)
    K = torch.zeros(B, 1, page, D, dtype=BF, device="cuda")
    V, w = K.clone(), torch.zeros(B, page, device="cuda")
    V[:, 0, 1] = 1 + torch.rand(B, D, generator=g, device="cuda").to(BF)
    w[:, 1] = -torch.rand(B, generator=g, device="cuda")
    out = torch.empty(B, n_qh, D, dtype=BF, device="cuda")
    context(pb, n_qh, 1, D, BF).pact_paged_attention(pb.PagedCache(K, V, w), torch.zeros(B, n_qh, D, dtype=BF, device="cuda"), torch.arange(B, dtype=I32, device="cuda")[:, None], i32([2] * B), out)
    x = np.exp(f64(w)[:, 1])[:, None, None]
    want = f64(V)[:, :, 1] * x / (1 + x)
    half_step = 2.0 ** (np.floor(np.log2(want)) - 8)
    assert (np.abs(f64(out) - want) <= half_step + 2.0 ** -20 * want).all()


@pytest.mark.parametrize("dtype,n_qh,D", [(BF, 1, 64), (BF, 8, 128), (BF, 16, 256), (F32, 1, 64), (F32, 8, 128), (F32, 2, 100)])
@pytest.mark.parametrize("wide", [False, True])
def test_probabilities_are_fp32_on_every_route(pb, dtype, n_qh, D, wide):
    # the two rows and the 2^-20 of test_fp32_results_of_bf16_rows_have_fp32_probabilities, in tables that clusters take and in wide ones, which all CTAs share out; fp32 rows
    # have products of one rounding each, less than the three terms of bf16
    B, page = 64, 16
    g = torch.Generator(device="cuda").manual_seed(D)
    K = torch.zeros(B, 1, page, D, dtype=dtype, device="cuda")
    V, w = K.clone(), torch.zeros(B, page, device="cuda")
    V[:, :, 1] = 1
    w[:, 1] = -torch.rand(B, generator=g, device="cuda")
    out, table = torch.empty(B, n_qh, D, device="cuda"), torch.full((B, 6000 if wide else 1), -1, dtype=I32, device="cuda")
    table[:, 0] = torch.arange(B, dtype=I32, device="cuda")
    context(pb, n_qh, 1, D, dtype, F32).pact_paged_attention(pb.PagedCache(K, V, w), torch.zeros(B, n_qh, D, dtype=dtype, device="cuda"), table, i32([2] * B), out)
    x = np.exp(f64(w)[:, 1])[:, None, None]
    assert np.abs(f64(out) / (x / (1 + x)) - 1).max() <= 2.0 ** -20


@pytest.mark.parametrize("dtype,n_qh,H,D,lens,wide", [(BF, 8, 2, 64, [1000, 3, 64], False), (BF, 28, 4, 128, [5000, 17], True), (BF, 16, 1, 256, [900], True), (F32, 2, 2, 64, [700, 1], False), (F32, 8, 1, 128, [4000], True)])
def test_results_to_fp32(pb, dtype, n_qh, H, D, lens, wide):
    # Logits from the biases alone (queries 0), values of both signs.  In units of 2^-22 of sum p |v|: p as above, 1.5 in the numerator and 1.5 in the denominator (fp32 rows: less); an
    # instruction cuts its sum to 2^-23, six of them for a warp's 16 rows: 3; sums: a step per 64 rows and warp in an fp32 of its own, then three to join the warps, eight for the parts
    # that meet, off by half a step, 2^-24, each.
    rng, g, page = np.random.default_rng(D), torch.Generator(device="cuda").manual_seed(D), 16
    n_pages = sum(po.pages_for(n, page) for n in lens) + 1
    K, V, w, _, _ = cache_tensors(g, n_pages, H, page, D, dtype, bounds=False)
    w = -torch.rand(n_pages, page, generator=g, device="cuda")
    table = tables(rng, lens, 6000 if wide else max(po.pages_for(n, page) for n in lens), page, n_pages)
    Q, out = torch.zeros(len(lens), n_qh, D, dtype=dtype, device="cuda"), torch.empty(len(lens), n_qh, D, device="cuda")
    context(pb, n_qh, H, D, dtype, F32).pact_paged_attention(pb.PagedCache(K, V, w), Q, i32(table), i32(lens), out)
    ref, _, mag, _ = po.attend(f64(Q), f64(K), f64(V), f64(w), table, lens, page, 1.0)
    steps = np.array([n / 64 + 12 for n in lens])[:, None, None]
    assert (np.abs(f64(out) - ref) <= mag * (6 * 2.0 ** -22 + 2 * steps * 2.0 ** -24)).all()


@pytest.mark.parametrize("n_qh,H,D,rows", [(32, 32, 64, 1 << 17), (64, 4, 64, 1 << 20), (8, 8, 256, 1 << 18)])
def test_sums_over_many_rows_are_not_biased(pb, n_qh, H, D, rows):
    # Values of one sign, thousands of rows of one running sum.  What a sum in fp32 may be off by grows as its roundings happen to fall, and their mean over heads and columns
    # stays near 0; what is cut off towards 0 adds up.  Within 16 rows there are three instructions; each cuts its terms and its result to 2^-23 of them at most, which is 2^-21 in all.  The
    # same p are in numerator and denominator, so their errors (2^-21 each) cancel but for those of independent rows.  2^-20 leaves as much again for the mean of the roundings: a
    # sum of 500 steps is off by 2^-24 * sqrt(500) = 2^-19.5 (one standard deviation, at most), the mean over 2048 results and more by 2^-25; that of the denominators, one per head
    # but of 32 lanes and thousands of parts each, by less than 2^-22.
    P, page = 64, 64
    g = torch.Generator(device="cuda").manual_seed(D)
    K = torch.zeros(P, H, page, D, dtype=BF, device="cuda")
    V, w = 1 + torch.rand(P, H, page, D, generator=g, device="cuda").to(BF), -torch.rand(P, page, generator=g, device="cuda")
    out = torch.empty(1, n_qh, D, device="cuda")
    table = torch.arange(rows // page, dtype=I32, device="cuda")[None] % P
    context(pb, n_qh, H, D, BF, F32).pact_paged_attention(pb.PagedCache(K, V, w), torch.zeros(1, n_qh, D, dtype=BF, device="cuda"), table, i32([rows]), out)
    p = torch.exp(w.double())
    want = (torch.einsum("pr,phrc->hc", p, V.double()) / p.sum()).repeat_interleave(n_qh // H, 0)
    assert abs(((out[0].double() - want) / want).mean().item()) <= 2.0 ** -20


def _mask_some(w, table):
    g = torch.Generator(device="cuda").manual_seed(1)
    w.masked_fill_(torch.rand(w.shape, generator=g, device="cuda") < 0.5, float("-inf"))
    w[torch.tensor(table[-1][table[-1] >= 0], device="cuda").long()] = float("-inf")     # the last request: nothing is left
    if (table[0] >= 0).any():
        w[int(table[0][0]), 1:] = float("-inf")                                            # and a page with one row


@pytest.mark.parametrize("dtype,D", [(BF, 128), (BF, 64), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("masked", [False, True])
def test_rows_that_do_not_count_may_hold_anything(pb, dtype, D, masked):
    attend_and_check(pb, dtype, F32, 8, 2, D, 32, [100, 5, 64, 0, 700, 33, 90], poison=True, mask=_mask_some if masked else None, seed=D)


def test_masks_of_the_lowest_value_and_large_logits(pb):
    """The lowest float as a bias is a number: where all rows have it, they share the attention; beside others it is nothing."""
    lowest = torch.finfo(F32).min

    def some(w, table):
        w[int(table[0, 0])] = lowest
        w[int(table[1, 0]), 3:] = lowest

    got = attend_and_check(pb, F32, F32, 2, 1, 64, 16, [40, 16], mask=some, seed=3)
    assert got.any()

    # all of them: shared as by zeros (fp32 logits this low do not tell q.k apart, so q is zero here)
    K, V = torch.zeros(2, 1, 16, 64, device="cuda"), torch.randn(2, 1, 16, 64, device="cuda")
    w = torch.full((2, 16), lowest, device="cuda")
    for dtype in (F32, BF):
        out, lse = torch.zeros(1, 1, 64, device="cuda"), torch.zeros(1, 1, device="cuda")
        cache = pb.PagedCache(K.to(dtype), V.to(dtype), w)
        context(pb, 1, 1, 64, dtype, F32).pact_paged_attention(cache, torch.zeros(1, 1, 64, device="cuda", dtype=dtype), i32([[0, 1]]), i32([20]), out, lse)
        rows = cache.V.double().reshape(32, 64)[:20]
        assert ((out[0, 0].double() - rows.mean(0)).abs() <= rows.abs().mean(0) * 2.0 ** -18).all() and lse.item() == lowest
    attend_and_check(pb, BF, F32, 8, 1, 128, 64, [500, 64], scale=3.0, seed=5)            # logits of a few hundred
    attend_and_check(pb, F32, F32, 8, 1, 64, 64, [500, 64], scale=-1.0, seed=5)


def test_what_is_not_a_number_and_counts_shows(pb):
    K, V, w, _, _ = cache_tensors(torch.Generator(device="cuda").manual_seed(2), 4, 1, 16, 64, BF, True, True, False)
    K[1, 0, 3, 5] = float("nan")
    w[2, 2] = float("inf")
    Q, out, lse = torch.randn(3, 2, 64, device="cuda").to(BF), torch.zeros(3, 2, 64, device="cuda"), torch.zeros(3, 2, device="cuda")
    context(pb, 2, 1, 64, BF, F32).pact_paged_attention(pb.PagedCache(K, V, w), Q, i32([[0, 1], [2, 0], [0, 3]]), i32([32, 20, 32]), out, lse)
    assert out[0].isnan().all() and out[1].isnan().all() and torch.isfinite(out[2]).all() and lse[0].isnan().all()


@pytest.mark.parametrize("dtype,D,page", [(BF, 128, 64), (BF, 64, 16), (F32, 64, 32), (BF, 80, 128), (BF, 64, 48)])
def test_attention_over_selected_pages(pb, dtype, D, page):
    rng = np.random.default_rng(page)
    lens, H, n_select = [1000, 0, 5, 300, 64, 2222], 2, 7
    sel = np.full((len(lens), H, n_select), -1, np.int32)
    for b, n in enumerate(lens):
        k = po.pages_for(n, page)
        for h in range(H):
            m = min(k, n_select)
            sel[b, h, :m] = np.sort(rng.permutation(k)[:m])
    attend_and_check(pb, dtype, F32, 8, H, D, page, lens, selected=sel, seed=D)
    # any order, gaps, repeats and places that the request does not have
    sel[0, 0], sel[0, 1] = [3, 1, -1, 2, 3, 10000, 0], [-5, -1, 4, 4, 4, 1, 2]
    sel[3, 0] = -1
    sel[5, 1] = [1 << 30, -(1 << 31), 1, 0, 5, 2, 2]
    attend_and_check(pb, dtype, F32, 8, H, D, page, lens, selected=sel, poison=False, seed=D)
    attend_and_check(pb, dtype, F32, 8, H, D, page, lens, selected=sel[:, :, :1].copy(), seed=D)


def test_bad_pages_and_lengths(pb):
    rng, page, n_pages = np.random.default_rng(0), 16, 30
    table = rng.integers(0, n_pages, (3, 9)).astype(np.int32)
    table[0, 2], table[0, 5], table[1, 0], table[2, 8] = -1, n_pages, 1 << 30, -(1 << 31)
    for dtype in (BF, F32):
        attend_and_check(pb, dtype, F32, 4, 2, 64, page, [100, 10, 9 * page], table=table, n_pages=n_pages, want_status=po.INVALID)
        attend_and_check(pb, dtype, F32, 4, 2, 64, page, [20, -3, 0], table=np.abs(table) % n_pages, n_pages=n_pages, want_status=po.INVALID)
        attend_and_check(pb, dtype, F32, 4, 2, 64, page, [20, 9 * page + 1, 0], table=np.abs(table) % n_pages, n_pages=n_pages, want_status=po.INVALID)


def test_a_page_that_two_requests_share(pb):
    table = np.array([[0, 1, 2], [0, 1, 3], [0, 0, 0]], np.int32)
    attend_and_check(pb, BF, BF, 8, 2, 128, 64, [150, 190, 192], table=table, n_pages=4)


def test_offsets_past_32_bits(pb):
    """A cache of more than 2^32 bytes and 2^31 elements: pages at its far end, in all three calls that touch it."""
    n_pages, H, page, D = 2050, 8, 1024, 128
    if torch.cuda.mem_get_info()[0] < 14 << 30:
        pytest.skip("not enough memory")
    K, V = (torch.zeros(n_pages, H, page, D, dtype=BF, device="cuda") for _ in range(2))
    assert K.numel() > 1 << 31
    b, wm, w = torch.zeros(n_pages, H, 2, D, dtype=BF, device="cuda"), torch.zeros(n_pages, device="cuda"), torch.zeros(n_pages, page, device="cuda")
    cache = pb.PagedCache(K, V, w, b, wm)
    ctx = context(pb, H, H, D)
    ids = [n_pages - 1, 0, n_pages - 3, 7]
    n = 3 * page + 500
    g = torch.Generator(device="cuda").manual_seed(1)
    K_new, V_new = (torch.randn(n, H, D, generator=g, device="cuda").to(BF) for _ in range(2))
    p = torch.arange(n, device="cuda")
    slot = torch.tensor(ids, device="cuda")[p // page] * page + p % page
    ctx.pact_cache_write(cache, K_new, V_new, None, slot)
    assert torch.equal(K[ids].transpose(1, 2).reshape(-1, H, D)[:n], K_new) and torch.equal(V[ids].transpose(1, 2).reshape(-1, H, D)[:n], V_new)
    assert torch.equal(b[ids[0], :, 0], K_new[:page].amin(0))
    Q, out = torch.randn(1, H, D, generator=g, device="cuda").to(BF), torch.zeros(1, H, D, dtype=BF, device="cuda")
    sel = torch.zeros(1, H, 3, dtype=I32, device="cuda")
    ctx.pact_page_select(cache, Q, i32([ids]), i32([n]), sel, 0, 1)
    assert np.array_equal(sel.cpu().numpy(), po.select(f64(Q), f64(b), f64(wm), np.array([ids]), [n], page, float(np.float32(D ** -0.5)), 0, 1, 3))
    ctx.pact_paged_attention(cache, Q, i32([ids]), i32([n]), out)
    s = torch.einsum("hc,nhc->hn", Q[0].double(), K_new.double()) * D ** -0.5
    ref = torch.einsum("hn,nhc->hc", torch.softmax(s, 1), V_new.double())
    # a bf16 number has eight significant bits, so its rounding is off by up to 2^-8 of the value (half of eps = 2^-7); 2^-15: two-term probabilities
    assert ((out[0].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -15).all()


@pytest.mark.parametrize("dtype,n_qh,H,D,page", [(BF, 28, 4, 128, 64), (BF, 4, 4, 64, 16), (BF, 16, 1, 256, 32), (F32, 2, 2, 64, 16), (F32, 12, 2, 128, 64)])
@pytest.mark.parametrize("lens", [[1], [900], [64, 0, 65], [5000], [3000, 1]])
def test_short_and_wide_tables_agree(pb, dtype, n_qh, H, D, page, lens):
    """The same requests in a table as long as they need, where clusters of CTAs take them, and in one of 100000 rows, where all CTAs share them out."""
    rng, g = np.random.default_rng(7), torch.Generator(device="cuda").manual_seed(7)
    n_pages = sum(po.pages_for(n, page) for n in lens) + 1
    K, V, w, _, _ = cache_tensors(g, n_pages, H, page, D, dtype, bounds=False)
    short = tables(rng, lens, max(1, max(po.pages_for(n, page) for n in lens)), page, n_pages)
    wide = np.full((len(lens), 100000 // page), -1, np.int32)
    wide[:, :short.shape[1]] = short
    Q = torch.randn(len(lens), n_qh, D, generator=g, device="cuda").to(dtype)
    ctx, got = context(pb, n_qh, H, D, dtype, F32), []
    for table in (short, wide):
        out, lse, status = torch.full((len(lens), n_qh, D), -5.0, device="cuda"), torch.zeros(len(lens), n_qh, device="cuda"), i32([0])
        ctx.pact_paged_attention(pb.PagedCache(K, V, w), Q, i32(table), i32(lens), out, lse, status=status)
        assert status.item() == 0
        got.append((f64(out), f64(lse)))
    scale = float(np.float32(D ** -0.5))
    ref, lse_ref, mag, big = po.attend(f64(Q), f64(K), f64(V), f64(w), short, lens, page, scale)
    # the tolerance of attend_and_check
    delta, steps = (D + 8) * 2.0 ** -23 * big, max(lens) / 64 + 20
    for out, lse in got:
        assert (np.abs(out - ref) <= mag * (2 * delta + 2.0 ** -16 + 2.0 ** -20 + steps * 2.0 ** -21)[..., None] + np.abs(ref) * 2.0 ** -24 + 1e-30).all()
        none = lse_ref == -np.inf
        assert np.array_equal(lse == -np.inf, none)
        assert (np.abs(lse[~none] - lse_ref[~none]) <= (delta + 2.0 ** -20 + steps * 2.0 ** -21)[~none] + 2.0 ** -22 * np.abs(lse_ref[~none])).all()


def test_most_requests(pb):
    """As many requests as a call may have, most of them short, some empty."""
    lens = [(i * 7) % 40 for i in range(4096)]
    attend_and_check(pb, BF, F32, 2, 1, 64, 16, lens, seed=1)


def test_a_row_for_one_request_and_none_for_the_others(pb):
    attend_and_check(pb, BF, F32, 4, 2, 64, 16, [0, 0, 0, 1, 0, 0, 0, 0, 0, 0, 0, 0])
    attend_and_check(pb, F32, F32, 4, 2, 64, 16, [0] * 300 + [1])


def test_the_same_page_named_for_a_write_by_two_requests_is_not_needed(pb):
    """A page that two requests share (a common beginning) is written once; what both read is the same."""
    g = torch.Generator(device="cuda").manual_seed(1)
    K, V, w, b, wm = cache_tensors(g, 8, 2, 16, 64, BF)
    ctx, cache = context(pb, 4, 2, 64, BF, F32), pb.PagedCache(K, V, w, b, wm)
    rows = torch.randn(16, 2, 64, generator=g, device="cuda").to(BF)
    ctx.pact_cache_write(cache, rows, rows, None, torch.arange(32, 48, device="cuda"))
    Q, out = torch.randn(1, 4, 64, device="cuda").to(BF).expand(2, 4, 64).contiguous(), torch.zeros(2, 4, 64, device="cuda")
    ctx.pact_paged_attention(cache, Q, i32([[2, 5], [2, 5]]), i32([30, 30]), out)
    assert torch.equal(out[0], out[1])


def test_the_first_call_of_a_context_inside_a_capture(pb):
    g = torch.Generator(device="cuda").manual_seed(3)
    K, V, w, b, wm = cache_tensors(g, 200, 2, 16, 64, BF)
    cache = pb.PagedCache(K, V, w, b, wm)
    T, L, Q = torch.randperm(200, device="cuda").int()[None], i32([3000]), torch.randn(1, 8, 64, device="cuda").to(BF)
    want, out = torch.zeros(1, 8, 64, device="cuda"), torch.zeros(1, 8, 64, device="cuda")
    sel_want, sel = torch.zeros(1, 2, 7, dtype=I32, device="cuda"), torch.zeros(1, 2, 7, dtype=I32, device="cuda")
    old = context(pb, 8, 2, 64, BF, F32)
    old.pact_page_select(cache, Q, T, L, sel_want)
    old.pact_paged_attention(cache, Q, T, L, want)
    fresh = pb.Context(512, 8, 2, 64, BF, F32)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fresh.pact_paged_attention(cache, Q, T, L, out)          # makes the workspace ...
        fresh.pact_page_select(cache, Q, T, L, sel)
    # ... which stays, although a later call with many pages outgrows it
    wide = torch.full((64, 60000), -1, dtype=I32, device="cuda")
    fresh.pact_page_select(cache, Q.expand(64, 8, 64).contiguous(), wide, torch.zeros(64, dtype=I32, device="cuda"), torch.zeros(64, 2, 7, dtype=I32, device="cuda"))
    junk = [torch.full((1 << 20,), 7, dtype=torch.uint8, device="cuda") for _ in range(40)]
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(sel, sel_want) and all((x == 7).all() for x in junk)


def test_selection_of_infinite_and_huge_bounds(pb):
    """What fp32 cannot hold is decided in double: infinities, products beyond 1e38, many scores alike."""
    D, page, n = 64, 16, 1200
    for dtype in (F32, BF):
        g = torch.Generator(device="cuda").manual_seed(11)
        K, V, w, b, wm = cache_tensors(g, n, 2, page, D, dtype)
        b[7, 0, 1, 3] = float("inf")
        b[9, 1, 0] = float("-inf")
        b[30:40] *= 1e30
        b[600, :, 1, 5] = float("nan")
        wm[5], wm[6], wm[8] = float("inf"), float("-inf"), float("nan")
        Q = torch.randn(2, 6, D, generator=g, device="cuda").to(dtype) * 1e9
        Q[1, 2, 4] = float("nan")
        table = np.stack([np.random.default_rng(i).permutation(n).astype(np.int32) for i in range(2)])
        lens = [n * page, 700 * page - 3]
        sel = torch.zeros(2, 2, 50, dtype=I32, device="cuda")
        context(pb, 6, 2, D, dtype).pact_page_select(pb.PagedCache(K, V, w, b, wm), Q, i32(table), i32(lens), sel, 1, 1, scale=0.5)
        with np.errstate(invalid="ignore"):
            want = po.select(f64(Q), f64(b), np.nan_to_num(f64(wm), nan=-np.inf, posinf=np.inf, neginf=-np.inf), table, lens, page, 0.5, 1, 1, 50)
        assert np.array_equal(sel.cpu().numpy(), want)


@pytest.mark.parametrize("dtype,D,n", [(BF, 64, 12), (F32, 64, 12), (BF, 128, 900), (F32, 100, 300), (BF, 256, 40)])
def test_a_key_with_an_infinite_coordinate_hides_no_other_row(pb, dtype, D, n):
    """Pages written by the library; one page has the row with the largest logit and another row with an infinite key, whose own logit is minus infinity."""
    page, H, g = 16, 1, torch.Generator(device="cuda").manual_seed(D + n)
    K, V, w, b, wm = cache_tensors(g, n, H, page, D, dtype)
    ctx, cache = context(pb, 2, H, D, dtype), pb.PagedCache(K, V, w, b, wm)
    Q = torch.randn(1, 2, D, generator=g, device="cuda").to(dtype)
    Q[0, :, 5], Q[0, :, 9] = -1, 0
    rows = (torch.randn(n * page, H, D, generator=g, device="cuda") * 0.1).to(dtype)
    target = n // 2
    rows[target * page + 3, 0] = 0.5 * Q[0, 1]                # the largest logit of all
    for bad in (float("inf"), float("-inf")):
        rows[target * page + 8, 0, 9] = bad                    # 0 times it: the logit is not a number
        rows[target * page + 9, 0, 5] = float("inf")
        status, sel = i32([0]), torch.zeros(1, H, 3, dtype=I32, device="cuda")
        ctx.pact_cache_write(cache, rows, rows, None, torch.arange(n * page, device="cuda"), status=status)
        ctx.pact_page_select(cache, Q, torch.arange(n, dtype=I32, device="cuda")[None], i32([n * page]), sel, 0, 0, scale=0.2, status=status)
        logits = torch.einsum("hc,nc->nh", Q[0].double(), rows[:, 0].double()).nan_to_num(nan=float("-inf")).amax(1)
        assert logits.argmax().item() // page == target and logits.amax().isfinite()
        assert status.item() == 0 and target in sel[0, 0].tolist()
        assert np.array_equal(sel.cpu().numpy(), po.select(f64(Q), f64(b), f64(wm), np.arange(n)[None], [n * page], page, float(np.float32(0.2)), 0, 0, 3))


@pytest.mark.parametrize("dtype,D,n,n_bad,n_select", [(BF, 64, 300, 1, 40), (BF, 128, 9000, 3, 500), (F32, 64, 2000, 700, 300), (F32, 128, 9000, 40, 64), (BF, 64, 2000, 2000, 30), (BF, 64, 1500, 5, 1499)])
def test_pages_with_infinite_bounds_among_many(pb, dtype, D, n, n_bad, n_select):
    """Only their scores are formed in double; the others keep the order that they have, and infinite scores tie to the lower page."""
    rng, g, page = np.random.default_rng(n + n_bad), torch.Generator(device="cuda").manual_seed(n), 16
    K, V, w, b, wm = cache_tensors(g, n, 1, page, D, dtype)
    bad = rng.permutation(n)[:n_bad]
    at = lambda x: torch.tensor(np.ascontiguousarray(x), device="cuda")   # noqa: E731
    b[at(bad), 0, at(rng.integers(0, 2, n_bad)), at(rng.integers(0, D, n_bad))] = at(rng.choice([np.inf, -np.inf, np.nan], n_bad)).to(dtype)
    wm[at(bad[1::7])] = float("-inf")
    wm[at(bad[2::7])] = float("inf")
    Q = torch.randn(2, 3, D, generator=g, device="cuda").to(dtype)
    Q[1, :, ::2] = 0
    table = np.stack([rng.permutation(n).astype(np.int32) for _ in range(2)])
    lens, sel, status = [n * page, (n - 1) * page - 3], torch.zeros(2, 1, n_select, dtype=I32, device="cuda"), i32([0])
    context(pb, 3, 1, D, dtype).pact_page_select(pb.PagedCache(K, V, w, b, wm), Q, i32(table), i32(lens), sel, 1, 1, scale=0.5, status=status)
    want = po.select(f64(Q), f64(b), f64(wm), table, lens, page, 0.5, 1, 1, n_select)
    assert status.item() == 0 and np.array_equal(sel.cpu().numpy(), want)


# ---- as a serving program uses them --------------------------------------------------------------------------------

def test_workspace_of_a_selection(pb):
    """Eight bytes per request, key head and page for scores in double, and four for those in fp32 only where a request may have more than shared memory holds."""
    ctx = context(pb, 6, 2, 64)
    parts = ctx._L.pact_paged_workspace_bytes(ctx.handle, 1, 1)
    for B, pages, of_score in ((128, 8192, 8), (1, 60000, 12), (64, 8193, 12)):
        assert ctx._L.pact_paged_workspace_bytes(ctx.handle, B, pages) == max(parts, (B * 2 * pages * of_score + 255) // 256 * 256)


def test_captured_and_replayed_with_other_lengths_beside_eager_calls(pb):
    """Two captured graphs and eager calls of one context take turns on its workspace."""
    rng, g = np.random.default_rng(0), torch.Generator(device="cuda").manual_seed(0)
    page, H, D, n_qh, n_pages, B = 16, 2, 64, 8, 600, 5
    K, V, w, b, wm = cache_tensors(g, n_pages, H, page, D, BF)
    cache, ctx = pb.PagedCache(K, V, w, b, wm), context(pb, n_qh, H, D, BF, F32)
    table = rng.permutation(n_pages).astype(np.int32)[:B * 100].reshape(B, 100)
    T, L, Q = i32(table), i32([100] * B), torch.zeros(B, n_qh, D, dtype=BF, device="cuda")
    sel = torch.zeros(B, H, 9, dtype=I32, device="cuda")
    out, out_s, out_e = (torch.zeros(B, n_qh, D, device="cuda") for _ in range(3))
    full, sparse = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(full):
        ctx.pact_paged_attention(cache, Q, T, L, out)
    with torch.cuda.graph(sparse):
        ctx.pact_page_select(cache, Q, T, L, sel)
        ctx.pact_paged_attention(cache, Q, T, L, out_s, selected=sel)
    scale = float(np.float32(D ** -0.5))
    for lens in ([100] * B, [1600, 0, 3, 1, 999], [0] * B, [64] * B, [1600] * B):
        L.copy_(i32(lens))
        Q.copy_(torch.randn(B, n_qh, D, generator=g, device="cuda"))
        full.replay()
        sparse.replay()
        ctx.pact_paged_attention(cache, Q, T, L, out_e)
        full.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, out_e)
        want_sel = po.select(f64(Q), f64(b), f64(wm), table, lens, page, scale, 1, 1, 9)
        assert np.array_equal(sel.cpu().numpy(), want_sel)
        for o, s in ((out, None), (out_s, want_sel)):
            ref, _, mag, _ = po.attend(f64(Q), f64(K), f64(V), f64(w), table, lens, page, scale, s)
            assert (np.abs(f64(o) - ref) <= mag * 1e-3 + 1e-30).all()


def test_another_stream(pb):
    g = torch.Generator(device="cuda").manual_seed(0)
    K, V, w, b, wm = cache_tensors(g, 300, 2, 16, 64, BF)
    cache, ctx = pb.PagedCache(K, V, w, b, wm), pb.Context(512, 8, 2, 64, BF, F32)
    Q, T, L = torch.randn(1, 8, 64, device="cuda").to(BF), torch.arange(300, device="cuda", dtype=I32)[None], i32([4800])
    out, out2 = torch.zeros(1, 8, 64, device="cuda"), torch.zeros(1, 8, 64, device="cuda")
    ctx.pact_paged_attention(cache, Q, T, L, out)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        K2, V2 = K.clone(), V.clone()
        ctx.pact_paged_attention(pb.PagedCache(K2, V2, w), Q, T, L, out2)
    s.synchronize()
    assert torch.equal(out, out2)


def test_cache_behind_a_reduction(pb):
    """pact_reduce on a batch, its row counts straight from the counters into pages and slots, keys, values and log W of the reduced rows into the
    cache, then decoding steps: a row per request, attention over everything and over selected pages."""
    from paper_2504_08966_b200 import workloads
    wl = workloads.tiny()
    d, n_qh, n_kvh, d_h = wl.d, wl.n_qh, wl.n_kvh, wl.d_h
    ctx = pb.Context(d, n_qh, n_kvh, d_h, F32, F32)
    B, cap = 3, wl.images[0].H.shape[0]
    H_out, logw = torch.zeros(B, cap, d, device="cuda"), torch.zeros(B, cap, device="cuda")
    counters = torch.zeros(B, pb.N_COUNTERS, dtype=I32, device="cuda")
    ims = []
    for i in range(B):
        im = pb.device_image(wl.images[0], F32)
        im.H_out, im.logw_out, im.counters = H_out[i], logw[i], counters[i]
        ims.append(im)
    ctx.pact_reduce(ims, [pb.make_params(lam=lam, d_c=d_c) for lam, d_c in ((0.1, 0.01), (0.3, wl.d_c), (0.6, 0.02))])
    page, width, n_pages = 16, 20, 60
    K, V = torch.full((2, n_pages, n_kvh, page, d_h), float("nan"), device="cuda")
    w, b, wm = (torch.full(s, float("nan"), device="cuda") for s in ((n_pages, page), (n_pages, n_kvh, 2, d_h), (n_pages,)))
    cache = pb.PagedCache(K, V, w, b, wm)
    table, length, status = torch.full((B, width), -1, dtype=I32, device="cuda"), i32([0] * B), i32([0])
    free, n_free = torch.randperm(n_pages, device="cuda").int(), i32([n_pages])
    slot = torch.zeros(B * cap, dtype=I64, device="cuda")
    # nothing comes back to the host between the reduction and the attention
    ctx.pact_cache_plan(page, table, length, counters[:, pb.CNT["n_out"]], free, n_free, length, n_free, slot=slot, row_stride=cap, status=status)
    Wk, Wv, Wq = (torch.randn(d, n * d_h, device="cuda") / d ** 0.5 for n in (n_kvh, n_kvh, n_qh))
    k, v = (H_out @ Wk).view(-1, n_kvh, d_h), (H_out @ Wv).view(-1, n_kvh, d_h)
    ctx.pact_cache_write(cache, k, v, logw.view(-1), slot, status=status)
    n_out = counters[:, 0].tolist()
    hist = [[k.view(B, cap, n_kvh, d_h)[i, :n].double(), v.view(B, cap, n_kvh, d_h)[i, :n].double(), logw[i, :n].double()] for i, n in enumerate(n_out)]
    assert length.tolist() == n_out and len(set(n_out)) > 1
    out, lse, sel = torch.zeros(B, n_qh, d_h, device="cuda"), torch.zeros(B, n_qh, device="cuda"), torch.zeros(B, n_kvh, 3, dtype=I32, device="cuda")
    step_slot, one = torch.zeros(B, dtype=I64, device="cuda"), i32([1] * B)
    for step in range(20):
        h = torch.randn(B, d, device="cuda")
        ctx.pact_cache_plan(page, table, length, one, free, n_free, length, n_free, slot=step_slot, status=status)
        k1, v1, q = (h @ Wk).view(B, n_kvh, d_h), (h @ Wv).view(B, n_kvh, d_h), (h @ Wq).view(B, n_qh, d_h)
        ctx.pact_cache_write(cache, k1, v1, None, step_slot, status=status)
        for i in range(B):
            hist[i] = [torch.cat(x) for x in zip(hist[i], (k1[i:i + 1].double(), v1[i:i + 1].double(), torch.zeros(1, device="cuda").double()))]
        for sparse in (False, True):
            if sparse:
                ctx.pact_page_select(cache, q, table, length, sel, status=status)
            ctx.pact_paged_attention(cache, q, table, length, out, lse, selected=sel if sparse else None, status=status)
            for i, (kk, vv, ww) in enumerate(hist):
                s = torch.einsum("hgc,nhc->hgn", q[i].double().view(n_kvh, -1, d_h), kk) * d_h ** -0.5 + ww
                if sparse:
                    places = sel[i].long()
                    live = torch.zeros(n_kvh, po.pages_for(len(kk), page), dtype=torch.bool, device="cuda")
                    for j in range(n_kvh):
                        live[j, places[j][places[j] >= 0]] = True
                    assert live[:, -1].all() and live[:, 0].all()
                    s = s.masked_fill(~live.repeat_interleave(page, 1)[:, None, :len(kk)], float("-inf"))
                ref = torch.einsum("hgn,nhc->hgc", torch.softmax(s, 2), vv).view(n_qh, d_h)
                # fp32 throughout: logits of a few units good to 1e-5, sums of some hundred rows
                assert (out[i].double() - ref).abs().max() < 1e-4 and (lse[i].double() - torch.logsumexp(s, 2).view(-1)).abs().max() < 1e-4
    assert status.item() == 0
    # the requests end: every page is free again
    ctx.pact_cache_plan(page, table, length, i32([-1] * B), free, n_free, length, n_free, n_rows=0, status=status)
    assert n_free.item() == n_pages and sorted(free.tolist()) == list(range(n_pages)) and length.tolist() == [0] * B and status.item() == 0


def test_refusals_on_the_device(pb):
    """Head widths without an attention kernel; the library's own answers behind the binding's checks."""
    wide = context(pb, 2, 1, 264, BF)
    K = torch.zeros(4, 1, 16, 264, dtype=BF, device="cuda")
    with pytest.raises(pb.PactError, match="unsupported"):
        wide.pact_paged_attention(pb.PagedCache(K, K), torch.zeros(1, 2, 264, dtype=BF, device="cuda"), i32([[0]]), i32([3]), torch.zeros(1, 2, 264, dtype=BF, device="cuda"))
    ctx = context(pb, 2, 1, 64, BF)
    K = torch.zeros(4, 1, 24, 64, dtype=BF, device="cuda")
    Q = torch.zeros(1, 2, 64, dtype=BF, device="cuda")
    with pytest.raises(pb.PactError, match="invalid"):
        ctx.pact_paged_attention(pb.PagedCache(K, K), Q, i32([[0]]), i32([3]), Q.clone())
    K = torch.zeros(4, 1, 16, 64, dtype=BF, device="cuda")
    with pytest.raises(pb.PactError, match="invalid"):
        ctx.pact_page_select(pb.PagedCache(K, K), Q, i32([[0]]), i32([3]), i32([[[0]]]))
    with pytest.raises(pb.PactError, match="wanted"):
        ctx.pact_paged_attention(pb.PagedCache(K, K), Q.cpu(), i32([[0]]), i32([3]), Q.clone())


@pytest.mark.parametrize("dtype,n_qh,H,D,lens,wide", [(BF, 8, 2, 64, [3000], False), (BF, 8, 2, 128, [60000, 5, 0, 20000], True), (F32, 2, 2, 64, [212], False), (F32, 8, 1, 128, [30000, 7], True),
                                                      (BF, 16, 1, 256, [9000] * 3, True), (BF, 4, 2, 64, [700, 300] * 12, False)])
def test_waits_that_run_out(pb, dtype, n_qh, H, D, lens, wide):
    """Waits of a few polls: the call ends with its status, wherever in the ring a warp gave up, nothing outside the result is touched, and the next call is right."""
    rng, g, page = np.random.default_rng(0), torch.Generator(device="cuda").manual_seed(0), 16
    n_pages = sum(po.pages_for(n, page) for n in lens) + 1
    K, V, w, _, _ = cache_tensors(g, n_pages, H, page, D, dtype, bounds=False)
    width = 100000 // page if wide else max(po.pages_for(n, page) for n in lens)
    table = i32(tables(rng, lens, width, page, n_pages))
    ctx, cache = pb.Context(n_qh * D, n_qh, H, D, dtype, F32), pb.PagedCache(K, V, w)
    Q, L, B = torch.randn(len(lens), n_qh, D, generator=g, device="cuda").to(dtype), i32(lens), len(lens)
    want, buf, status = torch.zeros(B, n_qh, D, device="cuda"), torch.full((B + 2, n_qh, D), -5.0, device="cuda"), i32([0])
    copies = [x.clone() for x in (K, V, w)]
    ctx.pact_paged_attention(cache, Q, table, L, want, status=status)
    assert status.item() == 0
    seen = set()
    for polls in (1, 2, 1, 3, 5, 9, 20, 50, 100, 1, 0):
        ctx.set_wait_limits(barrier_polls=polls)
        buf.fill_(-5)
        status.zero_()
        ctx.pact_paged_attention(cache, Q, table, L, buf[1:-1], status=status)
        seen.add(status.item())
        assert status.item() in (0, -5) and (polls != 1 or status.item() == -5) and (polls or status.item() == 0)
        assert (buf[0] == -5).all() and (buf[-1] == -5).all()
        if status.item() == 0:
            assert torch.equal(buf[1:-1], want)
    assert seen == {0, -5} and all(torch.equal(x, y) for x, y in zip(copies, (K, V, w)))


def test_two_calls_at_once_on_two_contexts(pb):
    """Contexts have workspaces of their own."""
    g = torch.Generator(device="cuda").manual_seed(6)
    K, V, w, _, _ = cache_tensors(g, 2000, 2, 64, 128, BF, bounds=False)
    T, L = torch.randperm(2000, device="cuda").int().view(2, 1000), i32([64000, 50001])
    runs = []
    for i in range(2):
        Q = torch.randn(2, 8, 128, device="cuda", generator=g).to(BF)
        ctx, s = pb.Context(1024, 8, 2, 128, BF, F32), torch.cuda.Stream()
        alone = torch.zeros(2, 8, 128, device="cuda")
        ctx.pact_paged_attention(pb.PagedCache(K, V, w), Q, T, L, alone)
        runs.append((ctx, s, Q, alone, torch.zeros(2, 8, 128, device="cuda")))
    torch.cuda.synchronize()
    for _, (ctx, s, Q, _, out) in itertools.product(range(20), runs):
        with torch.cuda.stream(s):
            ctx.pact_paged_attention(pb.PagedCache(K, V, w), Q, T, L, out)
    torch.cuda.synchronize()
    for _, _, _, alone, out in runs:
        assert torch.equal(out, alone)
