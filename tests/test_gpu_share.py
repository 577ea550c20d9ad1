"""Pages that several requests hold, on the GPU against plain implementations (oracle/chunk_oracle.py): fork, compaction and copies of pages, and a run of them with the attention."""
import numpy as np
import pytest
import torch

from oracle import chunk_oracle as co
from oracle import paged_oracle as po
from tests.test_gpu_chunk import BF, F32, I32, context, f64, i32, pb, tolerances   # noqa: F401

pytestmark = pytest.mark.gpu


class Cache:
    """Block tables, lengths, counts and the stack of a cache, on the host."""

    def __init__(self, n_pages, B, width, page, seed=0):
        self.page, self.table = page, np.full((B, width), -1, np.int32)
        self.length, self.shared, self.stack = [0] * B, [0] * n_pages, [int(x) for x in np.random.default_rng(seed).permutation(n_pages)]

    def grow(self, b, n):
        for j in range(po.pages_for(self.length[b], self.page), po.pages_for(self.length[b] + n, self.page)):
            self.table[b, j] = self.stack.pop()
        self.length[b] += n

    def stack_buffer(self):
        return np.array(self.stack + [-7] * (len(self.shared) - len(self.stack)), np.int32)

    def fork_and_check(self, pb, ctx, source, rows=None, in_place=False, want=po.OK):
        B, P = len(self.length), len(self.shared)
        T, L, S, F, N = i32(self.table), i32(self.length), i32(self.shared), i32(self.stack_buffer()), i32([len(self.stack)])
        T2, L2 = torch.full_like(T, -9), torch.full_like(L, -9)
        S2, F2, N2 = (S, F, N) if in_place else (torch.full_like(x, -9) for x in (S, F, N))
        copies, n_copies, status = i32(np.full((B, 3), -9)), i32([-9]), i32([0])
        before = [x.clone() for x in (T, L, S, F, N)]
        ctx.pact_cache_fork(self.page, T, L, i32(source), S, F, N, T2, L2, S2, F2, N2, copies, n_copies, rows=None if rows is None else i32(rows), status=status)
        r = co.fork(self.page, self.table, self.length, source, rows, self.shared, self.stack_buffer(), len(self.stack))
        assert status.item() == r[0] == want
        assert L2.tolist() == r[2] and S2.tolist() == r[3] and N2.item() == len(r[4]) and F2.tolist()[:len(r[4])] == r[4]
        for b, pages in enumerate(r[1]):
            assert T2[b].tolist() == pages + [-9] * (self.table.shape[1] - len(pages))
        assert copies.tolist() == r[5] + [[-1, -1, 0]] * (B - len(r[5])) and n_copies.item() == len(r[5])
        # behind the new top the stack keeps what it had, unless pages that were freed and handed out again lay there
        if not in_place:
            assert all(torch.equal(x, y) for x, y in zip(before, (T, L, S, F, N)))
            assert F2.tolist()[len(r[4]):] == [-9] * (P - len(r[4]))
        else:
            assert torch.equal(F[len(r[4]):], before[3][len(r[4]):])
        self.length, self.shared, self.stack = r[2], r[3], r[4]
        self.table = np.full_like(self.table, -1)
        for b, pages in enumerate(r[1]):
            self.table[b, :len(pages)] = pages
        return r

    def compact_and_check(self, pb, ctx, in_place=False, want=po.OK, extra=0):
        B, P = len(self.length), len(self.shared)
        T, L, S, F, N = i32(self.table), i32(self.length), i32(self.shared), i32(self.stack_buffer()), i32([len(self.stack)])
        T2, S2, F2 = (T, S, F) if in_place else (torch.full_like(x, -9) for x in (T, S, F))
        n_list = max(1, P // 2) + extra
        moved, copies, n_copies, status = i32([-9] * P), i32(np.full((n_list, 3), -9)), i32([-9]), i32([0])
        ctx.pact_cache_compact(self.page, T, L, S, F, N, T2, S2, F2, moved, copies, n_copies, status=status)
        r = co.compact(self.page, self.table, self.length, self.shared, self.stack_buffer(), len(self.stack))
        assert status.item() == r[0] == want
        assert S2.tolist() == r[2] and F2.tolist()[:len(r[3])] == r[3] and moved.tolist() == r[4]
        for b, pages in enumerate(r[1]):
            assert T2[b].tolist() == pages + ([-9] * (self.table.shape[1] - len(pages)) if not in_place else self.table[b, len(pages):].tolist())
        assert copies.tolist() == r[5] + [[-1, -1, 0]] * (n_list - len(r[5])) and n_copies.item() == len(r[5])
        for b, pages in enumerate(r[1]):
            self.table[b, :len(pages)] = pages
        self.shared, self.stack = r[2], r[3]
        return r


def share_context(pb):
    return context(pb, 4, 2, 64)


@pytest.mark.parametrize("B,width,page,P", [(1, 1, 16, 1), (1, 9, 16, 30), (7, 5, 32, 50), (33, 40, 16, 1500), (129, 17, 64, 2500), (1030, 3, 16, 4000)])
def test_generations_of_forks(pb, B, width, page, P):
    """Random requests go on with others, end, are cut, grow and are compacted, over and over; every state is the plain implementation's."""
    rng, c = np.random.default_rng(B), Cache(P, B, width, page)
    for b in range(B):
        c.grow(b, int(rng.integers(0, width * page + 1)) if P > B * width else min(width * page, page * (P // B)) if b % 2 == 0 else 0)
    for step in range(8):
        source = rng.integers(-1, B, B) if step % 3 else np.where(rng.random(B) < 0.6, np.arange(B), rng.integers(-1, B, B))
        rows = None
        if step % 2:
            have = np.array([c.length[s] if s >= 0 else 0 for s in source])
            rows = np.where(rng.random(B) < 0.3, have // page * page, np.floor(rng.random(B) * (have + 1))).astype(int)
        want = co.fork(page, c.table, c.length, source, rows, c.shared, c.stack_buffer(), len(c.stack))[0]
        assert want in (po.OK, po.NO_PAGES)
        c.fork_and_check(pb, share_context(pb), source, rows, in_place=bool(step & 2), want=want)
        if step in (2, 5):
            c.compact_and_check(pb, share_context(pb), in_place=step == 5, extra=step)
        for b in range(B):
            # further rows go onto pages of the request's own: those that others hold are full
            n = min(int(rng.integers(0, 2 * page)), width * page - c.length[b])
            if po.pages_for(c.length[b] + n, page) - po.pages_for(c.length[b], page) <= len(c.stack):
                c.grow(b, n)
    c.fork_and_check(pb, share_context(pb), [-1] * B)
    assert sorted(c.stack) == list(range(P)) and not any(c.shared)


def test_many_requests_and_long_tables(pb):
    c = Cache(70000, 4096, 16, 16)
    for b in range(4096):
        c.grow(b, (b * 31) % 257)
    rng = np.random.default_rng(1)
    c.fork_and_check(pb, share_context(pb), rng.integers(0, 4096, 4096))
    c.compact_and_check(pb, share_context(pb))
    c = Cache(9000, 3, 4000, 16)
    c.grow(0, 63999)
    c.fork_and_check(pb, share_context(pb), [0, 0, 0], [63999, 63990, 16 * 2500 + 1])
    c.compact_and_check(pb, share_context(pb))


def test_a_hold_of_the_programs_own(pb):
    """A prompt that the program keeps: its pages stay when the last request that has them ends, and a page that ends in part is copied."""
    c = Cache(20, 3, 4, 16)
    c.grow(0, 40)
    kept = c.table[0, :3].copy()
    for p in kept:
        c.shared[p] += 1
    c.fork_and_check(pb, share_context(pb), [0, 0, -1])             # both end in the third page, which the program holds: two copies
    assert set(kept[:2]) <= set(c.table[0]) and kept[2] not in c.table[:2]
    c.fork_and_check(pb, share_context(pb), [-1, -1, -1])
    assert not set(kept) & set(c.stack) and len(c.stack) == 17 and all(c.shared[p] == 0 for p in kept)


def test_what_cannot_be_served_changes_nothing(pb):
    ctx = share_context(pb)

    def fresh(n_pages=12):
        c = Cache(n_pages, 3, 4, 16, seed=4)
        c.grow(0, 40)
        c.grow(2, 20)
        return c

    for in_place in (False, True):
        c = fresh(5)                                                 # no page is free: two requests that end in one page need one
        c.fork_and_check(pb, ctx, [0, 0, 2], in_place=in_place, want=po.NO_PAGES)
        c.fork_and_check(pb, ctx, [0, 0, -1], in_place=in_place)       # with the pages of one that ends there is room
        for source, rows in (([0, 3, 2], None), ([0, -2, 2], None), ([0, 0, 2], [40, 41, 20]), ([0, 0, 2], [40, -1, 20]), ([0, 1, 2], [40, 1, 20])):
            fresh().fork_and_check(pb, ctx, source, rows, in_place=in_place, want=po.INVALID)
        for place, page in (((0, 1), 12), ((2, 0), -1), ((2, 1), 1 << 30), ((0, 0), -(1 << 31))):
            c = fresh()
            c.table[place] = page
            c.fork_and_check(pb, ctx, [0, 0, 2], in_place=in_place, want=po.INVALID)
        for length in (-1, 65, 1 << 30):
            c = fresh()
            c.length[1] = length
            c.fork_and_check(pb, ctx, [0, 0, 2], in_place=in_place, want=po.INVALID)
        c = fresh()
        c.table[2, 0] = c.table[0, 0]                                  # two requests on a page that one holds
        c.fork_and_check(pb, ctx, [0, 0, 2], in_place=in_place, want=po.INVALID)
        c = fresh()
        c.shared[c.table[0, 0]] = -1
        c.fork_and_check(pb, ctx, [0, 0, 2], in_place=in_place, want=po.INVALID)
    # a number of free pages that cannot be
    for n in (-1, 13, 1 << 30):
        c = fresh()
        T, L, S, F = i32(c.table), i32(c.length), i32(c.shared), i32(c.stack_buffer())
        T2, L2, S2, F2, N2, C, M, status = T.clone(), L.clone(), S.clone(), F.clone(), i32([0]), i32(np.zeros((3, 3))), i32([0]), i32([0])
        ctx.pact_cache_fork(16, T, L, i32([0, 0, 2]), S, F, i32([n]), T2, L2, S2, F2, N2, C, M, status=status)
        assert status.item() == po.INVALID and N2.item() == n and M.item() == 0 and all(torch.equal(x, y) for x, y in ((T, T2), (L, L2), (S, S2), (F, F2)))
        status.zero_()
        moved, C = i32([0] * 12), i32(np.zeros((6, 3)))
        ctx.pact_cache_compact(16, T, L, S, F, i32([n]), T2, S2, F2, moved, C, M, status=status)
        assert status.item() == po.INVALID and M.item() == 0 and moved.tolist() == list(range(12)) and all(torch.equal(x, y) for x, y in ((T, T2), (S, S2), (F, F2)))
    for bad in ("twice", -1, 12):
        c = fresh()
        c.stack[1] = c.stack[0] if bad == "twice" else bad
        c.compact_and_check(pb, ctx, want=po.INVALID)
    c = fresh()                                                      # what can be moved is; entries that are no pages stay
    c.table[0, 1], c.length[2] = 99, -5
    c.compact_and_check(pb, ctx, want=po.INVALID)


@pytest.mark.parametrize("P", [1, 31, 32, 33, 1000, 70001])
@pytest.mark.parametrize("free", [0.0, 0.5, 0.97, 1.0])
def test_compaction(pb, P, free):
    rng = np.random.default_rng(P)
    n_free = int(round(P * free))
    ids = [int(x) for x in rng.permutation(P)]
    c = Cache(P, 5, 100, 16)
    c.stack, used = ids[:n_free], ids[n_free:]
    c.shared = [int(x) if p in set(used) else 0 for p, x in enumerate(rng.integers(0, 3, P))] if P < 2000 else [0] * P
    for b in range(5):
        mine = used[b * 80:b * 80 + 80]
        c.table[b, :len(mine)] = mine
        c.length[b] = len(mine) * 16 - (3 if mine else 0)
    r = c.compact_and_check(pb, share_context(pb), extra=P % 3)
    assert sorted(c.stack) == list(range(P - n_free, P)) and len(r[5]) <= P // 2
    assert not c.compact_and_check(pb, share_context(pb))[5]            # once more: nothing moves


@pytest.mark.parametrize("dtype,H,D,page", [(BF, 2, 64, 16), (BF, 4, 128, 64), (F32, 1, 4, 16), (F32, 3, 100, 48), (BF, 1, 8, 1024), (BF, 2, 256, 16)])
@pytest.mark.parametrize("bounds", [False, True])
def test_copies(pb, dtype, H, D, page, bounds):
    g, P = torch.Generator(device="cuda").manual_seed(0), 40
    for heads_first in (True, False):
        shape = (P, H, page, D) if heads_first else (P, page, H, D)
        kv = [torch.randn(shape, generator=g, device="cuda").to(dtype) for _ in range(2)]
        K, V = kv if heads_first else (x.transpose(1, 2) for x in kv)
        w = torch.randn(P, page, generator=g, device="cuda") if bounds or heads_first else None
        bd = (torch.randn(P, H, 2, D, generator=g, device="cuda").to(dtype), torch.randn(P, generator=g, device="cuda")) if bounds else (None, None)
        entries = [[0, 1, page], [2, 3, 1], [2, 4, page - 1], [5, 6, 0], [-1, 7, 5], [8, P - 1, 7], [P, 9, 3], [10, P, 3], [11, -1, 3], [12, 13, page + 1], [14, 14, 3], [15, 16, -4], [17, 18, 9], [19, 20, page]]
        for n, status_want in ((None, -1), (6, 0), (len(entries) - 1, -1), (0, 0), (-3, 0), (1000, -1)):
            kc, vc, wc, bc = K.clone(), V.clone(), w, bd
            if not heads_first:
                kc, vc = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (K, V))
            wc = None if w is None else w.clone()
            bc = tuple(None if x is None else x.clone() for x in bd)
            status = i32([0])
            context(pb, H, H, D, dtype).pact_page_copy(pb.PagedCache(kc, vc, wc, *bc), i32(entries), n_copies=None if n is None else i32([n]), status=status)
            kr, vr, wr, br = K.clone(), V.clone(), None if w is None else w.clone(), tuple(None if x is None else x.clone() for x in bd)
            for a, b, rows in entries[:len(entries) if n is None else min(max(n, 0), len(entries))]:
                if a < 0 or rows <= 0 or a >= P or not 0 <= b < P or rows > page or a == b:
                    continue
                for x in (kr, vr):
                    x[b, :, :rows] = x[a, :, :rows]
                if wr is not None:
                    wr[b, :rows] = wr[a, :rows]
                for x in br:
                    if x is not None:
                        x[b] = x[a]
            assert status.item() == status_want and torch.equal(kc, kr) and torch.equal(vc, vr) and (w is None or torch.equal(wc, wr))
            assert all(x is None or torch.equal(x, y) for x, y in zip(bc, br))


def test_copies_far_away_and_none(pb):
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("not enough memory")
    K, V = (torch.zeros(2050, 8, 1024, 128, dtype=BF, device="cuda") for _ in range(2))
    K[2047, 7, 1000:], V[0, 3, 5] = 1, 2
    ctx, cache = context(pb, 8, 8, 128), pb.PagedCache(K, V)
    ctx.pact_page_copy(cache, i32([[2047, 2049, 1024], [0, 2048, 6]]))
    assert torch.equal(K[2049], K[2047]) and torch.equal(V[2048, :, :6], V[0, :, :6]) and not V[2049].any() and not K[2048].any() and not K[2046].any()
    ctx.pact_page_copy(cache, i32(np.zeros((0, 3))))


def test_captured_and_replayed(pb):
    """The stages of a search over beams in one graph: fork, copies, other states at every replay; in place beside eager calls on another workspace."""
    page, P, B, width, ctx = 16, 300, 6, 12, pb.Context(256, 4, 2, 64, BF, BF)
    g = torch.Generator(device="cuda").manual_seed(0)
    K, V, w = torch.randn(P, 2, page, 64, generator=g, device="cuda").to(BF), torch.randn(P, 2, page, 64, generator=g, device="cuda").to(BF), torch.randn(P, page, generator=g, device="cuda")
    T, L, src = i32(np.full((B, width), -1)), i32([0] * B), i32([0] * B)
    S, F, N = i32([0] * P), i32(list(range(P))), i32([P])
    T2, L2, copies, n_copies, status = torch.full_like(T, -1), torch.zeros_like(L), i32(np.zeros((B, 3))), i32([0]), i32([0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.pact_cache_fork(page, T, L, src, S, F, N, T2, L2, S, F, N, copies, n_copies, status=status)
        ctx.pact_page_copy(pb.PagedCache(K, V, w), copies, n_copies, status=status)
    c, rng = Cache(P, B, width, page), np.random.default_rng(0)
    c.grow(0, 50)
    k, v, bias = f64(K), f64(V), f64(w)
    for step in range(6):
        source = np.zeros(B, int) if step == 0 else rng.integers(0, B, B)
        for x, y in ((T, c.table), (L, c.length), (src, source), (S, c.shared), (F, c.stack_buffer()), (N, [len(c.stack)])):
            x.copy_(i32(y))
        graph.replay()
        r = c.fork_and_check(pb, ctx, source)
        assert status.item() == 0 and L2.tolist() == r[2] and S.tolist() == r[3] and F.tolist()[:len(r[4])] == r[4] and N.item() == len(r[4])
        for a, b, rows in r[5]:
            k[b, :, :rows], v[b, :, :rows], bias[b, :rows] = k[a, :, :rows], v[a, :, :rows], bias[a, :rows]
        assert np.array_equal(f64(K), k) and np.array_equal(f64(V), v) and np.array_equal(f64(w), bias)
        for b in range(B):
            c.grow(b, int(rng.integers(1, 20)) if c.length[b] < 150 else 0)


@pytest.mark.parametrize("dtype,out", [(BF, BF), (F32, F32)])
def test_a_prompt_its_samples_and_their_ends(pb, dtype, out):
    """All of it as it is used: two prompts by plan, write and attention of their tokens; the first goes on as three samples, which decode with tokens of their own; one of them and the
    second prompt end; the cache is compacted; drafted tokens are looked at and cut.  Every result is that of contiguous keys and values that the test keeps itself."""
    g, page, P, H, D, n_qh, B, width = torch.Generator(device="cuda").manual_seed(2), 16, 40, 2, 64, 6, 4, 10
    ctx = pb.Context(n_qh * D, n_qh, H, D, dtype, out)
    K, V = (torch.full((P, H, page, D), float("nan"), device="cuda").to(dtype) for _ in range(2))
    cache = pb.PagedCache(K, V, torch.full((P, page), float("nan"), device="cuda"))
    T, L, S, F, N = i32(np.full((B, width), -1)), i32([0] * B), i32([0] * P), i32(list(range(P))), i32([P])
    held = [None] * B                                                # keys, values, biases of each request
    scale = float(np.float32(D ** -0.5))

    def tokens(n_new):
        nonlocal T, L
        rows, status, n = sum(n_new), i32([0]), i32(n_new)
        start, slot, L2 = i32([0] * (B + 1)), torch.zeros(rows, dtype=torch.int64, device="cuda"), torch.zeros_like(L)
        ctx.pact_cache_plan(page, T, L, n, F, N, L2, N, row_start=start, slot=slot, status=status)
        k, v, q = (torch.randn(rows, h, D, generator=g, device="cuda").to(dtype) for h in (H, H, n_qh))
        w = torch.randn(rows, generator=g, device="cuda")
        ctx.pact_cache_write(cache, k, v, w, slot, status=status)
        o, lse = torch.full((rows, n_qh, D), -5.0, device="cuda").to(out), torch.zeros(rows, n_qh, device="cuda")
        ctx.pact_chunk_attention(cache, q, T, L2, n, o, row_start=start, lse=lse, status=status)
        L = L2
        assert status.item() == 0
        at = 0
        for b, m in enumerate(n_new):
            if m:
                new = [f64(x[at:at + m]) for x in (k, v, w)]
                held[b] = new if held[b] is None else [np.concatenate(x) for x in zip(held[b], new)]
                kk, vv, ww = held[b]
                one = len(ww)
                _, ref, lref, mag, big = co.attend(f64(q[at:at + m]), kk.transpose(1, 0, 2)[None], vv.transpose(1, 0, 2)[None], ww[None], np.zeros((1, 1), int), [one], [m], [0], one, scale, True, m)
                tol, tol_lse = tolerances(ref, mag, big, D, one, dtype, out)
                assert (np.abs(f64(o[at:at + m]) - ref) <= tol).all() and (np.abs(f64(lse[at:at + m]) - lref) <= tol_lse + 2.0 ** -22 * np.abs(lref)).all()
            at += m

    def fork(source, rows=None):
        nonlocal T, L, held
        T2, L2, copies, n, status = torch.full_like(T, -1), torch.zeros_like(L), i32(np.zeros((B, 3))), i32([0]), i32([0])
        ctx.pact_cache_fork(page, T, L, i32(source), S, F, N, T2, L2, S, F, N, copies, n, rows=None if rows is None else i32(rows), status=status)
        ctx.pact_page_copy(cache, copies, n, status=status)
        assert status.item() == 0
        T, L = T2, L2
        held = [None if s < 0 or held[s] is None else [x[:None if rows is None else rows[b]] for x in held[s]] for b, s in enumerate(source)]
        return n.item()

    def compact():
        moved, copies, n, status = i32([0] * P), i32(np.zeros((P // 2, 3))), i32([0]), i32([0])
        ctx.pact_cache_compact(page, T, L, S, F, N, T, S, F, moved, copies, n, status=status)
        ctx.pact_page_copy(cache, copies, n, status=status)
        assert status.item() == 0
        return n.item()

    tokens([0, 70, 37, 0])                       # two prompts
    assert fork([1, 1, 2, 1]) == 2               # the first goes on three times; one keeps the last page
    free = N.item()
    assert free == P - 5 - 3 - 2
    for _ in range(12):
        tokens([1, 1, 1, 1])                     # each decodes
    assert fork([0, 1, -1, -1]) == 0             # one sample and the second prompt end
    tokens([3, 1, 0, 0])
    assert compact() > 0
    tokens([5, 5, 9, 0])                         # drafted tokens, and a new prompt in an old place
    have = [int(x) for x in L]
    fork([0, 1, 2, -1], [have[0] - 4, have[1] - 2, have[2], 0])     # of which some are kept
    tokens([1, 1, 1, 0])
    fork([-1] * B)
    assert N.item() == P and sorted(F.tolist()) == list(range(P)) and not S.any()


def test_refusals_on_the_device(pb):
    ctx = share_context(pb)
    c = Cache(12, 3, 4, 16)
    T, L, S, F, N = i32(c.table), i32(c.length), i32(c.shared), i32(c.stack_buffer()), i32([12])
    rest = S.clone(), F.clone(), N.clone(), i32(np.zeros((3, 3))), i32([0])
    with pytest.raises(pb.PactError, match="invalid"):
        ctx.pact_cache_fork(16, T, L, i32([0] * 3), S, F, N, T, L.clone(), *rest)        # tables in place
    with pytest.raises(pb.PactError, match="invalid"):
        ctx.pact_cache_fork(16, T, L, i32([0] * 3), S, F, N, T.clone(), L, *rest)
    with pytest.raises(pb.PactError, match="wanted"):
        ctx.pact_cache_fork(16, T, L, i32([0] * 2), S, F, N, T.clone(), L.clone(), *rest)
    with pytest.raises(pb.PactError, match="invalid"):
        ctx.pact_cache_compact(16, T, L, S, F, N, T, S, F, i32([0] * 12), i32(np.zeros((5, 3))), i32([0]))   # a list that may be too short
