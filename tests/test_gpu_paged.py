"""The paged key/value cache through the C ABI: slot maps bit for bit, appended tokens, attention of
chunks and single tokens over the pages against the fp64 oracle, and a serving loop of all three."""

from types import SimpleNamespace

import numpy as np
import pytest
import torch

import oracle.attention as oa
import paper_2002_07062_amd as bsm
from attention_util import U, forward_bound, to64

pytestmark = pytest.mark.gpu

NAN = float("nan")


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Cache:
    """Pages in no order, NaN wherever no token of a request lies."""

    def __init__(self, kv_len, page, hk, d, seed=0, extra=3, layout="page_first"):
        g = torch.Generator().manual_seed(seed)
        counts = [-(-n // page) for n in kv_len]
        n_pages = sum(counts) + extra
        shape = (n_pages, page, hk, d)
        if layout == "heads_first":   # (pages, heads, page, dim)
            self.k, self.v = (torch.full((n_pages, hk, page, d), NAN, dtype=torch.bfloat16).transpose(1, 2) for _ in "kv")
        elif layout == "shifted":     # off every 16-byte boundary
            n = int(np.prod(shape))
            self.k, self.v = (torch.full((n + 5,), NAN, dtype=torch.bfloat16)[3:3 + n].view(shape) for _ in "kv")
        else:
            self.k, self.v = (torch.full(shape, NAN, dtype=torch.bfloat16) for _ in "kv")
        order = torch.randperm(n_pages, generator=g).tolist()
        self.table = torch.full((len(kv_len), max(counts, default=0) + 2), -1, dtype=torch.int32)
        self.tokens = []              # (k, v) of every request, (kv_len, hk, d) fp64
        for b, n in enumerate(kv_len):
            pages = [order.pop() for _ in range(counts[b])]
            self.table[b, :counts[b]] = torch.tensor(pages, dtype=torch.int32)
            mine = []
            for x in (self.k, self.v):
                t = torch.randn((n, hk, d), generator=g).to(torch.bfloat16)
                for j in range(n):
                    x[pages[j // page], j % page] = t[j]
                mine.append(to64(t))
            self.tokens.append(mine)
        if layout == "shifted":
            n = int(np.prod(shape))
            out = []
            for x in (self.k, self.v):
                y = torch.full((n + 5,), NAN, dtype=torch.bfloat16, device="cuda")
                y[3:3 + n] = x.reshape(-1).cuda()
                out.append(y[3:3 + n].view(shape))
            self.k, self.v = out
        else:
            self.k, self.v = self.k.cuda(), self.v.cuda()
        self.table = self.table.cuda()


def _check(o, q, cache, new, kv_len, group, scale, window=0):
    at = 0
    for b, n in enumerate(new):
        k, v = cache.tokens[b]
        for h in range(q.shape[1]):
            qq = to64(q[at:at + n, h])
            ref, lse, p = oa.forward(qq, k[:, h // group], v[:, h // group], scale, True, window)
            tol, _ = forward_bound(qq, k[:, h // group], v[:, h // group], scale, True, window, p, lse, ref)
            err = np.abs(to64(o[at:at + n, h]) - ref)
            assert (err <= tol).all(), f"request {b} head {h}: worst excess {(err - tol).max():.3e} at {np.argwhere(~(err <= tol))[:4].tolist()}"
        at += n


# new tokens, kv_len, page, query heads, kv heads, head dim, window, layout
CASES = [
    ([1], [1], 16, 1, 1, 64, 0, "page_first"),
    ([1, 1, 1], [5, 64, 200], 16, 8, 2, 128, 0, "page_first"),
    ([1, 1], [3000, 31], 16, 4, 4, 64, 0, "page_first"),       # pieces of the key axis
    ([1, 1], [3000, 700], 24, 8, 1, 128, 0, "page_first"),
    ([1, 2, 1], [1500, 90, 0], 1, 4, 2, 80, 0, "page_first"),  # a page per token; a request without keys
    ([3, 1, 4], [700, 65, 4], 7, 6, 2, 96, 0, "heads_first"),
    ([33, 1, 100], [33, 513, 400], 16, 4, 2, 64, 0, "page_first"),
    ([130, 1, 0, 64], [900, 2000, 77, 64], 64, 8, 2, 128, 0, "page_first"),
    ([60, 20], [30, 20], 32, 2, 2, 128, 0, "shifted"),         # rows before the first key
    ([1, 1, 50], [1000, 20, 300], 16, 4, 1, 64, 100, "page_first"),
    ([1, 2], [2500, 2049], 128, 2, 1, 128, 1, "heads_first"),
    ([9, 5], [300, 400], 16, 5, 5, 8, 64, "shifted"),
    ([1, 1], [600, 601], 16, 64, 1, 64, 0, "page_first"),      # a group of 64
    ([300], [1800], 16, 3, 1, 128, 500, "page_first"),
]


def _name(c):
    return "-".join(str(x) for x in c).replace(" ", "")


@pytest.mark.parametrize("case", CASES, ids=_name)
def test_paged_attention_matches_the_oracle(case):
    new, kv_len, page, hq, hk, d, window, layout = case
    cache = Cache(kv_len, page, hk, d, 3, layout=layout)
    g = torch.Generator().manual_seed(4)
    tokens = sum(new)
    q = (2 * torch.randn((tokens + 2, hq, d), generator=g)).to(torch.bfloat16).cuda()
    o = torch.full_like(q, NAN)
    start = i32([0] + list(np.cumsum(new)))
    scale = float(np.float32(d ** -0.5))
    seen = []
    for max_q, max_kv in ((max(new), max(kv_len)), (max(new), None), (max(new) + 40, 64)):
        o.fill_(NAN)
        bsm.bsm_attention_paged(q, cache.k, cache.v, cache.table, start, i32(kv_len), o, max_q=max_q, max_kv=max_kv, window=window)
        torch.cuda.synchronize()
        _check(o, q, cache, new, kv_len, hq // hk, scale, window)
        assert torch.isnan(o[tokens:]).all(), "rows behind the last request were written"


@pytest.mark.parametrize("batch", [3, 40])
def test_mixed_batches_in_pieces(batch):
    """Chunks of many sizes beside single tokens and requests without any, over keys long enough for
    pieces, some starting before the window of their rows."""
    rng = np.random.default_rng(batch)
    new = [int(rng.choice([0, 1, 2, 7, 30, 70, 140])) for _ in range(batch)]
    new[0], new[-1] = 200, 1
    kv_len = [n + int(rng.integers(0, 2600)) for n in new]
    cache = Cache(kv_len, 16, 2, 64, 15)
    g = torch.Generator().manual_seed(16)
    q = (2 * torch.randn((sum(new), 6, 64), generator=g)).to(torch.bfloat16).cuda()
    for window in (0, 900):
        o = torch.full_like(q, NAN)
        bsm.bsm_attention_paged(q, cache.k, cache.v, cache.table, i32([0] + list(np.cumsum(new))), i32(kv_len), o,
                                max_q=max(new), max_kv=max(kv_len), window=window)
        torch.cuda.synchronize()
        _check(o, q, cache, new, kv_len, 3, 0.125, window)


@pytest.mark.parametrize("chunk,window", [(1, 0), (1, 700), (45, 0)])
def test_paged_attention_of_hundreds_of_requests(chunk, window):
    """More requests than a workgroup has threads, most of them short, some long, some without new
    tokens, one with a chunk of its own."""
    rng = np.random.default_rng(chunk)
    new = rng.integers(0, 3, 300).tolist()
    kv_len = [int(rng.integers(n, 40)) for n in new]
    for b in (0, 17, 255, 256, 299):
        kv_len[b] = int(rng.integers(1100, 2300))
    new[256], new[299] = chunk, 1
    cache = Cache(kv_len, 16, 1, 64, 5)
    g = torch.Generator().manual_seed(6)
    q = (2 * torch.randn((sum(new), 2, 64), generator=g)).to(torch.bfloat16).cuda()
    o = torch.full_like(q, NAN)
    bsm.bsm_attention_paged(q, cache.k, cache.v, cache.table, i32([0] + list(np.cumsum(new))), i32(kv_len), o,
                            max_q=max(new), max_kv=max(kv_len), window=window)
    torch.cuda.synchronize()
    _check(o, q, cache, new, kv_len, 2, 0.125, window)


@pytest.mark.parametrize("stride,pages", [((1 << 32) + 128, [1, 0]), (1 << 31, [2, 0])])
def test_pages_past_32_bits(stride, pages):
    """Pages that lie more than 2^32 elements apart, written and read (a single token, a chunk)."""
    page, hk, d, n_pages = 32, 2, 64, max(pages) + 1
    buffer = torch.empty((n_pages - 1) * stride + 2 * page * hk * d, dtype=torch.bfloat16, device="cuda")
    k_cache, v_cache = (torch.as_strided(buffer, (n_pages, page, hk, d), (stride, hk * d, d, 1), x * page * hk * d) for x in (0, 1))
    k_cache.fill_(NAN)
    v_cache.fill_(NAN)
    g = torch.Generator().manual_seed(12)
    n = 55
    k, v = (torch.randn((n, hk, d), generator=g).to(torch.bfloat16).cuda() for _ in "kv")
    slots = torch.tensor([pages[j // page] * page + j % page for j in range(n)], device="cuda")
    bsm.bsm_cache_append(k, v, slots, k_cache, v_cache)
    assert torch.equal(k_cache[pages[1], :n - page], k[page:]) and torch.equal(v_cache[pages[0]], v[:page])
    cache = SimpleNamespace(tokens=[[to64(k), to64(v)]])
    for new in (1, 50):
        q = (2 * torch.randn((new, 4, d), generator=g)).to(torch.bfloat16).cuda()
        o = torch.full_like(q, NAN)
        bsm.bsm_attention_paged(q, k_cache, v_cache, i32([pages]), i32([0, new]), i32([n]), o, max_q=new)
        torch.cuda.synchronize()
        _check(o, q, cache, [new], [n], 2, 0.125)


def test_long_requests_are_shared():
    """Few rows over many keys go to several workgroups, whose parts need a workspace."""
    assert bsm.bsm_attention_paged_workspace(4, 4, 8, 8, 64, 1, 1024) == 0
    for batch, keys in ((1, 1537), (4, 4096), (64, 32768)):
        assert bsm.bsm_attention_paged_workspace(batch, batch, 8, 8, 64, 1, keys) > 0
    # a chunk beside many single tokens takes parts of its own rows, not of as many for each request
    for batch in (2, 200, 2000):
        assert bsm.bsm_attention_paged_workspace(batch, batch + 4096, 8, 1, 64, 4096, 8192) < 400 << 20


def test_bounds_keep_bad_lengths_and_pages_inside():
    """Entries that name no page read as zeros, lengths past the table count up to it, starts past
    the tokens are clamped, rows past max_q are left alone."""
    cache = Cache([64, 64], 16, 1, 64, 9)
    table = cache.table[:, :4].contiguous()
    table[0, 1] = -7
    table[0, 2] = 1 << 30
    g = torch.Generator().manual_seed(5)
    q = torch.randn((4, 1, 64), generator=g).to(torch.bfloat16).cuda()
    o = torch.full_like(q, NAN)
    bsm.bsm_attention_paged(q, cache.k, cache.v, table, i32([0, 3, 9]), i32([64, 1 << 30]), o, max_q=2)
    torch.cuda.synchronize()
    for x in cache.tokens[0]:
        x[16:48] = 0
    qq = to64(q[:3, 0])
    for at, n, b in ((0, 3, 0), (3, 1, 1)):
        k, v = (x[:, 0] for x in cache.tokens[b])
        qq = to64(q[at:at + n, 0])
        ref, lse, p = oa.forward(qq, k, v, 0.125, True)
        tol, _ = forward_bound(qq, k, v, 0.125, True, 0, p, lse, ref)
        err = np.abs(to64(o[at:at + n, 0]) - ref)[:2]
        assert (err <= tol[:2]).all()
    assert torch.isnan(o[2]).all(), "a row past max_q was written"


def test_paged_attention_replays_with_new_lengths():
    """A captured call whose lengths, table and chunk starts change between replays."""
    cache = Cache([900, 40, 300], 16, 2, 64, 21)
    g = torch.Generator().manual_seed(6)
    q = torch.randn((8, 4, 64), generator=g).to(torch.bfloat16).cuda()
    o = torch.full_like(q, NAN)
    start, kv, table = i32([0, 1, 2, 3]), i32([900, 40, 300]), cache.table.clone()
    ws = torch.empty(bsm.bsm_attention_paged_workspace(3, 8, 4, 2, 64, 4, 900), dtype=torch.uint8, device="cuda")

    def call(w, out):
        bsm.bsm_attention_paged(q, cache.k, cache.v, table, start, kv, out, max_q=4, max_kv=900, workspace=w)

    call(ws, o)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(ws, o)
    order = [0, 1, 2]
    for new, lens, perm in (([1, 1, 1], [900, 40, 300], [0, 1, 2]), ([4, 1, 3], [40, 300, 900], [1, 2, 0]),
                            ([1, 4, 0], [299, 77, 0], [2, 0, 1])):
        start.copy_(i32([0] + list(np.cumsum(new))))
        kv.copy_(i32(lens))
        table.copy_(cache.table[perm])
        o.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        eager = torch.full_like(q, NAN)
        call(None, eager)
        torch.cuda.synchronize()
        assert torch.equal(o.view(torch.int16), eager.view(torch.int16))
        at = 0
        for b, n in enumerate(new):
            for h in range(4):
                k, v = (x[:lens[b], h // 2] for x in cache.tokens[perm[b]])
                qq = to64(q[at:at + n, h])
                ref, lse, p = oa.forward(qq, k, v, 0.125, True)
                tol, _ = forward_bound(qq, k, v, 0.125, True, 0, p, lse, ref)
                assert (np.abs(to64(o[at:at + n, h]) - ref) <= tol).all()
            at += n
    del graph, order


# ---------------------------------------------------------------------------------------- slots
def _slots(cached, fresh, page, n_pages, table, free, n_free, n_slots):
    b = len(cached)
    t = i32(table).view(b, -1) if b else torch.empty((0, 4), dtype=torch.int32, device="cuda")
    q_start, kv_len = torch.full((b + 3,), -5, dtype=torch.int32, device="cuda"), torch.full((b + 2,), -5, dtype=torch.int32, device="cuda")
    slots, taken = torch.full((n_slots,), -9, dtype=torch.int64, device="cuda"), i32([-5, -5, -5])
    bsm.bsm_cache_slots(i32(cached), i32(fresh), page, n_pages, t, i32(free), i32([n_free]), q_start, kv_len, slots, taken)
    torch.cuda.synchronize()
    ref = oa.slots(cached, fresh, page, n_pages, np.asarray(table).reshape(b, t.shape[1]), free, n_free, n_slots)
    assert q_start[:b + 1].tolist() == ref[0]
    assert kv_len[:b].tolist() == ref[1]
    assert np.array_equal(t.cpu().numpy(), ref[2])
    assert np.array_equal(slots.cpu().numpy(), ref[3])
    assert taken.tolist() == ref[4] + [-5]
    assert (q_start[b + 1:] == -5).all() and (kv_len[b:] == -5).all()


@pytest.mark.parametrize("seed", range(12))
def test_slots_of_random_steps(seed):
    rng = np.random.default_rng(seed)
    b = int(rng.choice([0, 1, 3, 255, 256, 257, 700]))
    page = int(rng.choice([1, 3, 16, 64]))
    hi = int(rng.choice([1, 2, 40, 300]))
    cached, fresh = rng.integers(0, 5 * page + 2, b), rng.integers(0, hi + 1, b)
    if seed % 3 == 0 and b:
        cached[rng.integers(0, b)] = -4
        fresh[rng.integers(0, b)] = -1
    cached, fresh = cached.tolist(), fresh.tolist()
    need = sum(-(-(max(c, 0) + max(f, 0)) // page) + -(-max(c, 0) // page) for c, f in zip(cached, fresh))
    n_pages = need + 10
    width = max([-(-(max(c, 0) + max(f, 0)) // page) for c, f in zip(cached, fresh)], default=0) + 1
    if seed % 4 == 1:
        width = max(1, width // 2)
    table = rng.integers(0, n_pages, (b, width))
    free = rng.permutation(n_pages).tolist()
    if seed % 4 == 2:
        table[rng.integers(0, max(b, 1), 5) % max(b, 1), 0] = n_pages if b else 0
        free[:3] = [-1, n_pages, 2**31 - 1]
    n_free = n_pages if seed % 2 == 0 else need // 4
    total = sum(max(f, 0) for f in fresh)
    _slots(cached, fresh, page, n_pages, table.tolist(), free, n_free, total + 70 if seed % 5 else max(0, total - 3))


def test_slots_bounds():
    _slots([0, 0], [4, 4], 4, 8, [[-1], [-1]], [], 0, 8)                       # an empty free list
    _slots([0, 0], [4, 4], 4, 8, [[-1], [-1]], [3], 1000, 8)                   # n_free past the list
    _slots([2**31 - 1, 5], [2**31 - 1, 1], 4, 8, [[1, 2], [3, 4]], [0], 1, 4)  # lengths near 2^31
    _slots([0], [0], 4, 8, [[-1]], [0], 1, 0)


# --------------------------------------------------------------------------------------- append
@pytest.mark.parametrize("tokens,page,hk,d,layout", [
    (1, 16, 1, 8, "page_first"), (77, 16, 2, 64, "page_first"), (300, 24, 8, 128, "page_first"),
    (50, 7, 3, 96, "heads_first"), (33, 1, 1, 40, "shifted"), (9001, 16, 8, 128, "page_first")])
def test_append_writes_the_slots_and_nothing_else(tokens, page, hk, d, layout):
    g = torch.Generator().manual_seed(tokens)
    n_pages = -(-tokens // page) + 4
    cache = Cache([], page, hk, d, extra=n_pages, layout=layout)
    slots = torch.randperm(n_pages * page, generator=g)[:tokens].cuda()
    slots[tokens // 2] = -1
    slots[tokens // 3] = n_pages * page
    fused = torch.randn((tokens, 2 * hk, d), generator=g).to(torch.bfloat16).cuda()
    k, v = fused[:, :hk], fused[:, hk:]
    bsm.bsm_cache_append(k, v, slots, cache.k, cache.v)
    torch.cuda.synchronize()
    for x, y in ((k, cache.k), (v, cache.v)):
        want = torch.full((n_pages * page, hk, d), NAN, dtype=torch.bfloat16, device="cuda")
        ok = (slots >= 0) & (slots < n_pages * page)
        want[slots[ok]] = x[ok]
        assert torch.equal(want.view(torch.int16), y.contiguous().view(-1, hk, d).view(torch.int16))


# ---------------------------------------------------------------------------------- all together
def test_a_serving_loop():
    """Prompts in chunks, then single tokens: every step takes its slots, writes its keys and values
    and attends over the pages; the outputs are those of the whole sequences so far."""
    g = torch.Generator().manual_seed(77)
    hq, hk, d, page, n_pages, width = 4, 2, 64, 16, 64, 12
    k_cache, v_cache = (torch.full((n_pages, page, hk, d), NAN, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    table = torch.full((3, width), -1, dtype=torch.int32, device="cuda")
    free = torch.randperm(n_pages, generator=g).to(torch.int32).cuda()
    cached = i32([0, 0, 0])
    history = [[], [], []]
    steps = [[40, 7, 0], [40, 1, 100], [13, 1, 1], [1, 1, 1], [1, 1, 1], [0, 1, 16]]
    for fresh in steps:
        t = sum(fresh)
        qkv = torch.randn((t, hq + 2 * hk, d), generator=g).to(torch.bfloat16).cuda()
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        q_start, kv_len = torch.empty(4, dtype=torch.int32, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda")
        slots, taken = torch.empty(t, dtype=torch.int64, device="cuda"), i32([0, 0])
        bsm.bsm_cache_slots(cached, i32(fresh), page, n_pages, table, free, i32([free.numel()]), q_start, kv_len, slots, taken)
        bsm.bsm_cache_append(k, v, slots, k_cache, v_cache)
        o = torch.full((t, hq, d), NAN, dtype=torch.bfloat16, device="cuda")
        bsm.bsm_attention_paged(q, k_cache, v_cache, table, q_start, kv_len, o, max_q=max(fresh))
        torch.cuda.synchronize()
        pages, refused = taken.tolist()
        assert refused == 0
        free = free[pages:].contiguous()
        cached = kv_len
        at = 0
        for b, n in enumerate(fresh):
            history[b].append((to64(k[at:at + n]), to64(v[at:at + n])))
            kk, vv = (np.concatenate([x[i] for x in history[b]]) for i in (0, 1))
            for h in range(hq):
                qq = to64(q[at:at + n, h])
                ref, lse, p = oa.forward(qq, kk[:, h // 2], vv[:, h // 2], 0.125, True)
                tol, _ = forward_bound(qq, kk[:, h // 2], vv[:, h // 2], 0.125, True, 0, p, lse, ref)
                assert (np.abs(to64(o[at:at + n, h]) - ref) <= tol).all()
            at += n
    assert U == 2.0 ** -8


def test_a_refused_request_comes_out_empty():
    """The free list holds pages for the first request only: the second has no slots, its rows of the
    output are zeros, and the cache holds nothing of it."""
    hk, d, page = 1, 64, 16
    k_cache, v_cache = (torch.full((4, page, hk, d), NAN, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    table = torch.full((2, 4), -1, dtype=torch.int32, device="cuda")
    q_start, kv_len = torch.empty(3, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    slots, taken = torch.empty(40, dtype=torch.int64, device="cuda"), i32([0, 0])
    bsm.bsm_cache_slots(i32([0, 0]), i32([20, 20]), page, 4, table, i32([2, 0, 1]), i32([3]), q_start, kv_len, slots, taken)
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn((40, 1, d), generator=g).to(torch.bfloat16).cuda() for _ in "qkv")
    bsm.bsm_cache_append(k, v, slots, k_cache, v_cache)
    o = torch.full_like(q, NAN)
    bsm.bsm_attention_paged(q, k_cache, v_cache, table, q_start, kv_len, o, max_q=20)
    torch.cuda.synchronize()
    assert taken.tolist() == [2, 1] and kv_len.tolist() == [20, 0] and (slots[20:] == -1).all()
    assert (o[20:] == 0).all() and torch.isfinite(o[:20].float()).all()
    assert torch.isnan(k_cache[[1, 3]]).all()


# few rows, tiles, both; some rows see nothing (more new tokens than keys)
@pytest.mark.parametrize("window", [2**31 - 1, 2**31 - 40])
@pytest.mark.parametrize("new,kv_len", [([9, 5], [3, 5]), ([60, 20], [30, 20]), ([100, 6, 1], [70, 2, 40])])
def test_the_largest_windows_hide_nothing(new, kv_len, window):
    cache = Cache(kv_len, 16, 2, 64, 31)
    g = torch.Generator().manual_seed(32)
    q = (2 * torch.randn((sum(new), 4, 64), generator=g)).to(torch.bfloat16).cuda()
    o = torch.full_like(q, NAN)
    bsm.bsm_attention_paged(q, cache.k, cache.v, cache.table, i32([0] + list(np.cumsum(new))), i32(kv_len), o,
                            max_q=max(new), max_kv=max(kv_len), window=window)
    torch.cuda.synchronize()
    _check(o, q, cache, new, kv_len, 2, 0.125)


@pytest.mark.parametrize("batch,chunk,hq,hk", [(300, 4096, 64, 8), (512, 2048, 64, 8), (512, 4096, 32, 8), (512, 8192, 32, 8),
                                               (257, 8192, 64, 8), (2000, 4096, 16, 2), (2000, 4096, 64, 8)])
def test_hundreds_of_requests_beside_a_long_chunk_are_taken(batch, chunk, hq, hk):
    """What a call launches decides whether it is too large, not a join that it does not need."""
    assert bsm.bsm_attention_paged_workspace(batch, batch + chunk, hq, hk, 128, chunk, 2 * chunk) < 1 << 30
    with pytest.raises(bsm.BsmError, match="too large"):
        bsm.bsm_attention_paged_workspace(1 << 20, (1 << 20) + chunk, hq, hk, 128, chunk, 2 * chunk)


def test_hundreds_of_requests_beside_a_chunk():
    """300 requests, 64/8 heads, room for a chunk of 4096: single tokens, one chunk, some without any."""
    rng = np.random.default_rng(8)
    new = rng.integers(0, 2, 300).tolist()
    new[0], new[255], new[256], new[280], new[299] = 1, 3, 1, 150, 40
    kv_len = [n + int(rng.integers(0, 30)) for n in new]
    kv_len[255], kv_len[256] = 700, 1300
    cache = Cache(kv_len, 16, 8, 64, 33)
    g = torch.Generator().manual_seed(34)
    q = torch.full((4096 + 300, 64, 64), NAN, dtype=torch.bfloat16)
    q[:sum(new)] = (2 * torch.randn((sum(new), 64, 64), generator=g)).to(torch.bfloat16)
    q = q.cuda()
    o = torch.full_like(q, NAN)
    start = [0] + [int(x) for x in np.cumsum(new)]
    bsm.bsm_attention_paged(q, cache.k, cache.v, cache.table, i32(start), i32(kv_len), o, max_q=4096, max_kv=8192)
    torch.cuda.synchronize()
    assert torch.isfinite(o[:start[-1]].float()).all() and torch.isnan(o[start[-1]:]).all()
    for b in (0, 1, 100, 255, 256, 280, 298, 299):
        rows, one = slice(start[b], start[b + 1]), SimpleNamespace(tokens=[cache.tokens[b]])
        _check(o[rows], q[rows], one, [new[b]], [kv_len[b]], 8, 0.125)


@pytest.mark.parametrize("form", ["pages", "rows", "heads", "halves", "heads_first"])
def test_keys_and_values_in_one_tensor(form):
    """The cache's k and v as views of one tensor, in every way that they interleave."""
    n_pages, page, hk, d = 9, 16, 2, 64
    shape = {"pages": (n_pages, 2, page, hk, d), "rows": (n_pages, page, 2, hk, d), "heads": (n_pages, page, hk, 2, d),
             "halves": (2, n_pages, page, hk, d), "heads_first": (n_pages, hk, 2, page, d)}[form]
    x = torch.full(shape, NAN, dtype=torch.bfloat16, device="cuda")
    k_cache, v_cache = x.unbind({"pages": 1, "rows": 2, "heads": 3, "halves": 0, "heads_first": 2}[form])
    if form == "heads_first":
        k_cache, v_cache = k_cache.transpose(1, 2), v_cache.transpose(1, 2)
    g = torch.Generator().manual_seed(35)
    k, v = (torch.randn((100, hk, d), generator=g).to(torch.bfloat16).cuda() for _ in "kv")
    slots = torch.randperm(n_pages * page, generator=g)[:100].cuda()
    bsm.bsm_cache_append(k, v, slots, k_cache, v_cache)
    torch.cuda.synchronize()
    for cache, y in ((k_cache, k), (v_cache, v)):
        assert torch.equal(cache[slots // page, slots % page], y)
    assert int(torch.isfinite(x.float()).sum()) == 2 * 100 * hk * d


@pytest.mark.parametrize("device", [-1, 64, 2**31 - 1])
def test_a_workspace_for_no_device_is_refused(device):
    with pytest.raises(bsm.BsmError) as e:
        bsm.bsm_attention_paged_workspace(4, 4, 8, 8, 64, 1, 4096, device=device)
    assert e.value.status == bsm.BSM_ERR_INVALID_ARG and "device" in e.value.message
    assert bsm.load().hipGetLastError() == 0, "left for the next call that looks"


@pytest.mark.parametrize("new", [[1, 1], [1, 40]])
def test_no_bound_on_the_keys(new):
    """max_kv of 0 stands for the table's width, as None does, in the workspace too."""
    kv_len = [2500, 300]
    cache = Cache(kv_len, 16, 1, 64, 37)
    g = torch.Generator().manual_seed(38)
    q = torch.randn((sum(new), 1, 64), generator=g).to(torch.bfloat16).cuda()
    outs = []
    for max_kv in (0, None):
        o = torch.full_like(q, NAN)
        bsm.bsm_attention_paged(q, cache.k, cache.v, cache.table, i32([0, 1, sum(new)]), i32(kv_len), o, max_q=max(new), max_kv=max_kv)
        torch.cuda.synchronize()
        _check(o, q, cache, new, kv_len, 1, 0.125)
        outs.append(o)
    assert torch.equal(*outs)


@pytest.mark.parametrize("name", ["max_q", "max_kv", "window"])
def test_arguments_past_32_bits_are_refused(name):
    """A bound of 2^32 is not one of 0, which would leave o as it is without a word."""
    cache = Cache([40], 16, 1, 64, 39)
    q = torch.ones((1, 1, 64), dtype=torch.bfloat16, device="cuda")
    args = dict(max_q=1, max_kv=40, window=0)
    for x in (2**32, 2**32 + 1, 2**31, -2**32 + 1):
        with pytest.raises(ValueError, match=f"{name} .*32 bits"):
            bsm.bsm_attention_paged(q, cache.k, cache.v, cache.table, i32([0, 1]), i32([40]), torch.empty_like(q), **{**args, name: x})
    with pytest.raises(ValueError, match="page_size .*32 bits"):
        bsm.bsm_cache_slots(i32([0]), i32([1]), 2**32 + 16, 8, i32([[0]]), i32([1]), i32([1]), i32([0, 0]), i32([0]),
                            torch.empty(1, dtype=torch.int64, device="cuda"), i32([0, 0]))


def test_slots_of_idle_requests():
    """A request without new tokens keeps its cache when an earlier one's tokens go past the slots."""
    _slots([1, 2, 7, 0], [3, 4, 0, 1], 4, 12, [[4, -1], [5, -1], [6, 7], [-1, -1]], [8, 9], 2, 6)
    _slots([9] * 300, [5] + [0] * 299, 4, 12, [[1, 2, 3, 4]] * 300, [8, 9], 2, 3)
    _slots([0, 4, 9], [1, 0, 0], 4, 12, [[1], [2], [3]], [8, 9], 2, 0)  # the last one's pages do not fit


# new tokens and query heads of a kv head: up to 16 rows, up to 32, tiles beside up to 16 and up to 32, tiles alone
ROWS = {"16": ([1, 2], 4), "32": ([5, 3], 4), "tiles+16": ([40, 3], 4), "tiles+32": ([3, 1], 20), "tiles": ([40], 4)}


@pytest.mark.parametrize("layout", ["page_first", "shifted"])
@pytest.mark.parametrize("keys", [[300, 77], [2600, 1900]], ids=["short", "long"])  # whole, and in shares or pieces
@pytest.mark.parametrize("rows", list(ROWS))
@pytest.mark.parametrize("d", [40, 64, 72, 96, 104, 128])
def test_every_kernel_matches_the_oracle(d, rows, keys, layout):
    new, group = ROWS[rows]
    kv_len = keys[:len(new)]
    cache = Cache(kv_len, 16, 2, d, 41, layout=layout)
    g = torch.Generator().manual_seed(42)
    q = (2 * torch.randn((sum(new), 2 * group, d), generator=g)).to(torch.bfloat16).cuda()
    o = torch.full_like(q, NAN)
    n = bsm.bsm_attention_paged_workspace(len(new), sum(new), 2 * group, 2, d, max(new), max(kv_len))
    assert (n > 0) == (keys[0] > 300 or "tiles" in rows)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")  # NaN
    bsm.bsm_attention_paged(q, cache.k, cache.v, cache.table, i32([0] + list(np.cumsum(new))), i32(kv_len), o, max_q=max(new),
                            max_kv=max(kv_len), workspace=ws)
    torch.cuda.synchronize()
    _check(o, q, cache, new, kv_len, group, float(np.float32(d ** -0.5)))


@pytest.mark.parametrize("d", [64, 96, 128])
def test_pieces_of_many_tiles(d):
    """Tiles that fill the compute units in a few pieces: a workgroup joins 16 rows of one."""
    cache = Cache([2600], 16, 8, d, 43)
    g = torch.Generator().manual_seed(44)
    q = (2 * torch.randn((512, 32, d), generator=g)).to(torch.bfloat16).cuda()
    o = torch.full_like(q, NAN)
    bsm.bsm_attention_paged(q, cache.k, cache.v, cache.table, i32([0, 512]), i32([2600]), o, max_q=512, max_kv=2600)
    torch.cuda.synchronize()
    assert torch.isfinite(o.float()).all()
    for h in (0, 5, 7):
        one = SimpleNamespace(tokens=[[x[:, h:h + 1] for x in cache.tokens[0]]])
        _check(o[:, 4 * h + 1:4 * h + 2], q[:, 4 * h + 1:4 * h + 2], one, [512], [2600], 1, float(np.float32(d ** -0.5)))


@pytest.mark.parametrize("new", [[1, 2], [40, 1]])
def test_joins_of_more_parts_than_a_wave_has_lanes(new):
    """40000 keys of one kv head: 79 shares of single tokens, 157 pieces of a chunk's tile."""
    kv_len = [40000, 600]
    cache = Cache(kv_len, 64, 1, 64, 45)
    g = torch.Generator().manual_seed(46)
    q = (2 * torch.randn((sum(new), 2, 64), generator=g)).to(torch.bfloat16).cuda()
    o = torch.full_like(q, NAN)
    bsm.bsm_attention_paged(q, cache.k, cache.v, cache.table, i32([0, new[0], sum(new)]), i32(kv_len), o, max_q=max(new), max_kv=40000)
    torch.cuda.synchronize()
    _check(o, q, cache, new, kv_len, 2, 0.125)


def test_mixed_batches_on_two_streams_and_replayed():
    """A chunk beside single tokens, four kernels a call: on two streams at once with workspaces of their own,
    and captured, replayed with other lengths between eager calls."""
    lens = [[1700, 900, 2500], [2500, 1700, 900]]
    cache = Cache([2500, 1700, 900], 16, 2, 64, 47)
    tables = [cache.table[[1, 2, 0]].contiguous(), cache.table]
    g = torch.Generator().manual_seed(48)
    q = [(2 * torch.randn((70, 6, 64), generator=g)).to(torch.bfloat16).cuda() for _ in "ab"]
    new = [[1, 60, 3], [50, 1, 1]]
    starts, kv = [i32([0] + list(np.cumsum(n))) for n in new], [i32(x) for x in lens]
    n = bsm.bsm_attention_paged_workspace(3, 70, 6, 2, 64, 60, 2500)
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in "ab"]
    out = [torch.full_like(x, NAN) for x in q]
    streams = [torch.cuda.Stream() for _ in "ab"]
    torch.cuda.synchronize()

    def call(i, o, w, **k):
        bsm.bsm_attention_paged(q[i], cache.k, cache.v, tables[i], starts[i], kv[i], o, max_q=60, max_kv=2500, workspace=w, **k)

    def check(i, o):
        order = [1, 2, 0] if i == 0 else [0, 1, 2]
        one = SimpleNamespace(tokens=[cache.tokens[b] for b in order])
        _check(o, q[i], one, new[i], lens[i], 3, 0.125)

    for _ in range(5):
        for i in (0, 1):
            call(i, out[i], ws[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in (0, 1):
        check(i, out[i])
    # captured with the first batch's arrays, which then hold either batch
    o, mine = torch.full_like(q[0], NAN), [x.clone() for x in (q[0], tables[0], starts[0], kv[0])]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bsm.bsm_attention_paged(mine[0], cache.k, cache.v, *mine[1:], o, max_q=60, max_kv=2500, workspace=ws[0])
    for i in (1, 0, 1):
        for x, y in zip(mine, (q[i], tables[i], starts[i], kv[i])):
            x.copy_(y)
        o.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o.view(torch.int16)[:sum(new[i])], out[i].view(torch.int16)[:sum(new[i])])
        eager = torch.full_like(o, NAN)
        call(i, eager, ws[1])
        torch.cuda.synchronize()
        assert torch.equal(o.view(torch.int16), eager.view(torch.int16))


@pytest.mark.parametrize("window", [0, 1, 25, 100])
@pytest.mark.parametrize("new,kv_len", [([1], [1000]), ([1, 3], [3001, 130]), ([10, 1], [300, 2600]), ([50], [700])])
def test_how_far_a_hidden_nan_reaches(new, kv_len, window):
    """NaN in every value whose block of 64 keys no row sees (the table may still hold pages that a window
    has left behind): the results keep their bits."""
    cache = Cache(kv_len, 16, 1, 64, 49)
    g = torch.Generator().manual_seed(50)
    q = (2 * torch.randn((sum(new), 2, 64), generator=g)).to(torch.bfloat16).cuda()
    outs = []
    for _ in range(2):
        o = torch.full_like(q, NAN)
        bsm.bsm_attention_paged(q, cache.k, cache.v, cache.table, i32([0] + list(np.cumsum(new))), i32(kv_len), o, max_q=max(new),
                                max_kv=max(kv_len), window=window)
        torch.cuda.synchronize()
        outs.append(o.view(torch.int16))
        for b, n in enumerate(kv_len):
            blocks = oa.seen(new[b], n, True, window).any(0)
            for key in range(n):
                if not blocks[key // 64 * 64:key // 64 * 64 + 64].any():
                    cache.v[cache.table[b, key // 16], key % 16] = NAN
    assert torch.equal(*outs)
