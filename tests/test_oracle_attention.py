"""Pins of the fp64 attention oracle, and the library's refusals of bad attention calls, which come
before any HIP call (no GPU here)."""

import ctypes
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import oracle.attention as oa
import paper_2002_07062_amd as bsm
from attention_util import FORMS, kernels_of
from paper_2002_07062_amd import attention as att

TOPO = dict(n_xcd=8)


# ------------------------------------------------------------------------------------ oracle
@pytest.mark.parametrize("n,m,causal,window", [(7, 7, False, 0), (7, 7, True, 0), (5, 12, True, 0),
                                               (12, 5, True, 0), (9, 9, True, 3), (4, 11, True, 6), (1, 1, True, 1)])
def test_oracle_matches_float64_autograd(n, m, causal, window):
    g = torch.Generator().manual_seed(n * m)
    q, k, v, do = (torch.randn((r, 6), generator=g, dtype=torch.float64) for r in (n, m, m, n))
    mask = torch.tensor([[not causal or (j <= i + m - n and (window == 0 or j > i + m - n - window))
                          for j in range(m)] for i in range(n)])
    live = mask.any(1)
    args = [x.clone().requires_grad_() for x in (q, k, v)]
    s = (args[0] @ args[1].T) * 0.4
    p = torch.softmax(s[live].masked_fill(~mask[live], -torch.inf), 1)
    o = torch.zeros((n, 6), dtype=torch.float64)
    o = o.index_put((live.nonzero()[:, 0],), p @ args[2])
    o.backward(do)
    mine, lse, _ = oa.forward(q, k, v, 0.4, causal, window)
    np.testing.assert_allclose(mine, o.detach(), atol=1e-13)
    assert np.array_equal(lse == -np.inf, ~live.numpy())
    for got, x in zip(oa.backward(q, k, v, mine, lse, do, 0.4, causal, window), args):
        np.testing.assert_allclose(got, x.grad if x.grad is not None else 0, atol=1e-12)


def test_oracle_by_hand():
    """Two keys with scores 0 and ln 3: weights 1/4 and 3/4."""
    q, k, v = np.array([[1.0]]), np.array([[0.0], [np.log(3)]]), np.array([[4.0], [8.0]])
    o, lse, p = oa.forward(q, k, v, 1.0)
    np.testing.assert_allclose(p, [[0.25, 0.75]])
    np.testing.assert_allclose(o, [[7.0]])
    np.testing.assert_allclose(lse, [np.log(4)])


def test_oracle_slots_by_hand():
    """Pages of 4: request 0 fills its page and takes one, 1 is new and takes two, 2 finds none left,
    3 needs none."""
    table = [[9, -1, -1], [-1, -1, -1], [-1, -1, -1], [5, -1, -1]]
    q_start, kv_len, out, slots, taken = oa.slots([3, 0, 0, 1], [2, 5, 1, 2], 4, 12, table, [7, 2, 11, 3], 3, 12)
    assert q_start == [0, 2, 7, 8, 10] and kv_len == [5, 5, 0, 3] and taken == [3, 1]
    assert out.tolist() == [[9, 7, -1], [2, 11, -1], [-1, -1, -1], [5, -1, -1]]
    assert slots.tolist() == [39, 28, 8, 9, 10, 11, 44, -1, 21, 22, -1, -1]


# -------------------------------------------------------------------------------------- plans
def _status(fn, *a, **k):
    try:
        fn(*a, **k)
    except bsm.BsmError as e:
        return e.status, e.message
    return bsm.BSM_OK, ""


def _plan(q_len=(4, 5), kv_len=None, **k):
    args = dict(heads_q=4, heads_kv=2, head_dim=64, topology=TOPO, device=-1)
    args.update(k)
    return bsm.bsm_attention_plan_create(list(q_len), kv_len if kv_len is None else list(kv_len), **args)


@pytest.mark.parametrize("kwargs,status,msg", [
    (dict(heads_q=5), "INVALID_ARG", "multiple"),
    (dict(heads_kv=0), "INVALID_ARG", "multiple"),
    (dict(heads_q=0, heads_kv=1), "INVALID_ARG", "multiple"),
    (dict(head_dim=0), "INVALID_ARG", "head_dim"),
    (dict(head_dim=60), "UNSUPPORTED", "head_dim"),
    (dict(head_dim=136), "UNSUPPORTED", "head_dim"),
    (dict(window=4), "INVALID_ARG", "causal"),
    (dict(window=-1, causal=True), "INVALID_ARG", "window"),
    (dict(q_len=(4, -1)), "INVALID_ARG", "lengths"),
    (dict(kv_len=(4, 2**30 + 1)), "INVALID_ARG", "lengths"),
    (dict(q_start=[0, -2]), "INVALID_ARG", "first rows"),
    (dict(schedule=9), "INVALID_ARG", "schedule"),
    (dict(topology=None), "INVALID_ARG", "topology"),
    (dict(topology=dict(n_xcd=17)), "INVALID_ARG", "n_xcd"),
    (dict(device=-2), "INVALID_ARG", "device"),
    (dict(q_len=[2**30] * 8, heads_q=256, heads_kv=256), "INVALID_ARG", "too many"),
])
def test_plan_refusals(kwargs, status, msg):
    st, m = _status(_plan, **kwargs)
    assert st == getattr(bsm, "BSM_ERR_" + status), m
    assert msg in m


def test_plan_python_checks():
    with pytest.raises(ValueError):
        _plan(q_len=(4, 5), kv_len=(4,))
    with pytest.raises(ValueError):
        _plan(q_len=(2**31,))


@pytest.mark.parametrize("q_len,kv_len,causal,window", [
    ([7, 300, 0], [7, 300, 12], False, 0), ([7, 300, 1], [9, 512, 40], True, 0), ([30, 5], [10, 0], True, 0),
    ([300, 40], [300, 90], True, 17), ([300], [20], True, 5), ([5], [300], True, 100)])
def test_plan_stats(q_len, kv_len, causal, window):
    p = _plan(q_len, kv_len, causal=causal, window=window)
    d = bsm.bsm_attention_plan_describe(p)
    assert d["pairs"] == sum(int(oa.seen(n, m, causal, window).sum()) for n, m in zip(q_len, kv_len))
    assert d["q_units"] == 4 * sum(-(-n // 64) for n in q_len)  # little work: units of 64 rows
    assert d["kv_units"] >= 2 * sum(-(-m // 128) for m in kv_len)  # some in parts
    assert d["lse_elems"] == 4 * sum(q_len) and d["workspace_bytes"] >= 16 * sum(q_len)
    one = bsm.bsm_attention_plan_describe(_plan(q_len, kv_len, causal=causal, window=window, topology=dict(n_xcd=8, n_cu=1)))
    assert one["q_units"] == 4 * sum(-(-n // 128) for n in q_len)
    assert one["kv_units"] in [2 * sum(-(-m // n) for m in kv_len) for n in (128, 64)]
    assert one["workspace_bytes"] == 16 * sum(q_len)
    assert (d["total_q"], d["total_kv"], d["causal"], d["window"]) == (sum(q_len), sum(kv_len), causal, window)


@pytest.mark.parametrize("q_len,kv_len,parted", [([4096], [4096], True), ([4096] * 64, [4096] * 64, False),
                                                 ([9], [4096], False),
                                                 # causal: the last 130 queries alone see keys, 3 steps of 64 by 2 heads
                                                 ([8192, 30], [130, 30], False)])
def test_plan_parts_of_few_keys(q_len, kv_len, parted):
    """Units that alone would keep few compute units busy are cut into parts, within bounds of the
    work table and the workspace."""
    whole, halves = (2 * sum(-(-m // n) for m in kv_len) for n in (128, 64))
    for n_cu in (0, 64, 256):
        d = bsm.bsm_attention_plan_describe(_plan(q_len, kv_len, causal=True, topology=dict(n_xcd=8, n_cu=n_cu)))
        slots = 2 * (n_cu or 256)  # head dimension 64: two workgroups on a compute unit
        assert d["workspace_bytes"] <= 16 * sum(q_len) + 2 * slots * 128 * 1024
        assert d["kv_units"] <= halves + 2 * slots
        if not parted or n_cu != 64:
            assert (d["kv_units"] not in (whole, halves)) == parted
    # parts of dq: few queries of many keys
    assert bsm.bsm_attention_plan_describe(_plan([9], [4096]))["workspace_bytes"] > 16 * 9
    assert bsm.bsm_attention_plan_describe(_plan([4096] * 64))["workspace_bytes"] == 16 * 4096 * 64
    st, m = _status(_plan, topology=dict(n_xcd=8, n_cu=-1))
    assert st == bsm.BSM_ERR_INVALID_ARG and "n_cu" in m


@pytest.mark.parametrize("q_len,dim,causal,rows", [
    ([512] * 32, 64, False, 128), ([4096] * 16, 128, True, 128), ([4096], 64, True, 64), ([4096], 128, True, 64),
    ([700] * 4, 96, False, 64), ([], 64, False, 64)])
def test_plan_rows_of_query_units(q_len, dim, causal, rows):
    d = bsm.bsm_attention_plan_describe(_plan(q_len, head_dim=dim, causal=causal))
    assert d["q_units"] == 4 * sum(-(-n // rows) for n in q_len)


def test_plan_allocation_failure(monkeypatch):
    monkeypatch.setenv("BSM_TEST_ALLOC_FAIL", "host")
    assert _status(_plan)[0] == bsm.BSM_ERR_OOM
    monkeypatch.delenv("BSM_TEST_ALLOC_FAIL")
    _plan().destroy()


def test_empty_batch_plans():
    for q_len in ([], [0, 0]):
        d = bsm.bsm_attention_plan_describe(_plan(q_len))
        assert d["q_units"] == 0 and d["workspace_bytes"] == 0
    assert att._load().bsm_attention_plan_destroy(None) == bsm.BSM_ERR_INVALID_ARG


# ----------------------------------------------------------------- refusals of paged cache calls
def _heads(at, row=256, head=64, seq=0):
    return ctypes.byref(att.bsm_heads(at, seq, row, head))


def _cache(**k):
    a = dict(k=1 << 30, v=1 << 31, n_pages=8, page_stride=16 * 128, row_stride=128, head_stride=64, page_size=16, heads=2,
             head_dim=64, reserved=0)
    a.update(k)
    return ctypes.byref(att.bsm_cache(**a))


def _paged(cache=None, q=None, o=None, table=1 << 40, width=4, q_start=1 << 41, kv_len=1 << 42, batch=2, tokens=6, heads_q=4,
           max_q=3, max_kv=60, window=0, scale=0.125, ws=1 << 43, ws_bytes=1 << 30):
    return att._load().bsm_attention_paged(cache or _cache(), q or _heads(1 << 44), o or _heads(1 << 45), table, width, q_start,
                                           kv_len, batch, tokens, heads_q, max_q, max_kv, window, scale, ws, ws_bytes, None)


@pytest.mark.parametrize("kwargs,status,msg", [
    (dict(cache=_cache(head_dim=20)), "UNSUPPORTED", "head_dim"),
    (dict(cache=_cache(page_size=0)), "INVALID_ARG", "pages"),
    (dict(cache=_cache(n_pages=-1)), "INVALID_ARG", "pages"),
    (dict(cache=_cache(k=0)), "INVALID_ARG", "NULL"),
    (dict(cache=_cache(k=(1 << 30) + 1)), "INVALID_ARG", "aligned"),
    (dict(cache=_cache(row_stride=-8)), "INVALID_ARG", "strides"),
    (dict(heads_q=3), "INVALID_ARG", "multiple"),
    (dict(width=-1), "INVALID_ARG", "width"),
    (dict(width=2**27), "INVALID_ARG", "2^30"),
    (dict(window=-1), "INVALID_ARG", "window"),
    (dict(scale=0.0), "INVALID_ARG", "scale"),
    (dict(scale=float("nan")), "INVALID_ARG", "scale"),
    (dict(batch=-1), "INVALID_ARG", "batch"),
    (dict(tokens=-1), "INVALID_ARG", "tokens"),
    (dict(max_q=-1), "INVALID_ARG", "max_q"),
    (dict(max_kv=2**30 + 1), "INVALID_ARG", "max_kv"),
    (dict(q=_heads(None)), "INVALID_ARG", "NULL"),
    (dict(o=_heads(1 << 45, row=128)), "INVALID_ARG", "overlap"),
    (dict(o=_heads(1 << 45, head=0)), "INVALID_ARG", "overlap"),
    (dict(o=_heads(1 << 44)), "ALIAS", "overlaps"),
    (dict(o=_heads((1 << 30) + 64)), "ALIAS", "overlaps"),
    (dict(o=_heads((1 << 40) + 8)), "ALIAS", "overlaps"),
    (dict(table=None), "INVALID_ARG", "NULL"),
    (dict(q_start=None), "INVALID_ARG", "NULL"),
])
def test_paged_refusals(kwargs, status, msg):
    st = _paged(**kwargs)
    assert st == getattr(bsm, "BSM_ERR_" + status), bsm.bsm_last_error()
    assert msg in bsm.bsm_last_error()


def test_paged_calls_without_work_touch_no_gpu():
    for k in (dict(batch=0), dict(tokens=0, q=_heads(None), o=_heads(None)), dict(max_q=0)):
        assert _paged(**k) == bsm.BSM_OK


def _slots(cached=1 << 30, fresh=1 << 31, batch=4, page_size=16, n_pages=64, table=1 << 32, width=8, free=1 << 33, cap=32,
           n_free=1 << 34, q_start=1 << 35, kv_len=1 << 36, slots=1 << 37, n_slots=10, taken=1 << 38):
    return att._load().bsm_cache_slots(cached, fresh, batch, page_size, n_pages, table, width, free, cap, n_free, q_start, kv_len,
                                       slots, n_slots, taken, None)


@pytest.mark.parametrize("kwargs,status,msg", [
    (dict(batch=-1), "INVALID_ARG", "batch"),
    (dict(page_size=0), "INVALID_ARG", "page_size"),
    (dict(width=-1), "INVALID_ARG", "width"),
    (dict(width=2**27), "INVALID_ARG", "2^30"),
    (dict(cap=-1), "INVALID_ARG", "free_cap"),
    (dict(n_slots=-1), "INVALID_ARG", "n_slots"),
    (dict(cached=None), "INVALID_ARG", "NULL"),
    (dict(table=None), "INVALID_ARG", "NULL"),
    (dict(n_free=None), "INVALID_ARG", "NULL"),
    (dict(slots=None), "INVALID_ARG", "NULL"),
    (dict(slots=(1 << 37) + 4), "INVALID_ARG", "aligned"),
    (dict(fresh=(1 << 31) + 2), "INVALID_ARG", "aligned"),
    (dict(kv_len=1 << 30), "ALIAS", "input"),
    (dict(q_start=(1 << 33) + 64), "ALIAS", "input"),
    (dict(taken=(1 << 32) + 32), "ALIAS", "outputs"),
])
def test_slots_refusals(kwargs, status, msg):
    st = _slots(**kwargs)
    assert st == getattr(bsm, "BSM_ERR_" + status), bsm.bsm_last_error()
    assert msg in bsm.bsm_last_error()


def _append(cache=None, k=None, v=None, slots=1 << 40, tokens=6):
    return att._load().bsm_cache_append(cache or _cache(), k or _heads(1 << 44, 128), v or _heads(1 << 45, 128), slots, tokens, None)


@pytest.mark.parametrize("kwargs,status,msg", [
    (dict(cache=_cache(page_stride=0)), "INVALID_ARG", "overlap"),
    (dict(cache=_cache(row_stride=64)), "INVALID_ARG", "overlap"),
    (dict(cache=_cache(v=1 << 30)), "ALIAS", "same place"),
    (dict(tokens=-1), "INVALID_ARG", "tokens"),
    (dict(k=_heads((1 << 44) + 1, 128)), "INVALID_ARG", "aligned"),
    (dict(v=_heads(None, 128)), "INVALID_ARG", "NULL"),
    (dict(k=_heads((1 << 30) + 32, 128)), "ALIAS", "overlaps"),
    (dict(slots=(1 << 31) + 16), "ALIAS", "overlaps"),
    (dict(slots=None), "INVALID_ARG", "NULL"),
    (dict(slots=(1 << 40) + 4), "INVALID_ARG", "aligned"),
])
def test_append_refusals(kwargs, status, msg):
    st = _append(**kwargs)
    assert st == getattr(bsm, "BSM_ERR_" + status), bsm.bsm_last_error()
    assert msg in bsm.bsm_last_error()


def test_append_without_tokens_touches_no_gpu():
    assert _append(tokens=0, k=_heads(None), v=_heads(None), slots=None) == bsm.BSM_OK
    assert _append(cache=_cache(n_pages=0, k=0, v=0)) == bsm.BSM_OK


def test_host_only_plans_do_not_run():
    p = _plan()
    st = att._load().bsm_attention_execute(p.handle, *[_heads(1 << (40 + i)) for i in range(4)], None, 0.125, None)
    assert st == bsm.BSM_ERR_UNSUPPORTED


@pytest.mark.parametrize("cache,offset", [
    ({}, 64), ({}, 8), ({}, 128), ({}, 2048), ({}, -64), ({}, 3 * 2048 + 64),
    (dict(page_stride=2 * 2048), 1024), (dict(page_stride=2 * 2048), 2048 - 8), (dict(row_stride=256, page_stride=16 * 256), 64),
    (dict(row_stride=256, page_stride=16 * 256), 8 * 256), (dict(head_stride=128, row_stride=256, page_stride=16 * 256), 32),
])
def test_caches_on_top_of_each_other_are_refused(cache, offset):
    """v lies `offset` elements behind k, in it."""
    at = 1 << 30
    assert _append(cache=_cache(k=at, v=at + 2 * offset, **cache)) == bsm.BSM_ERR_ALIAS
    assert "overlap" in bsm.bsm_last_error()


def test_a_workspace_for_no_device_is_refused():
    st, m = _status(bsm.bsm_attention_paged_workspace, 4, 4, 8, 8, 64, 1, 4096, device=-1)
    assert st == bsm.BSM_ERR_INVALID_ARG and "device" in m


@pytest.mark.parametrize("name", ["heads_q", "heads_kv", "head_dim", "window", "device"])
@pytest.mark.parametrize("beyond", [2**32, -2**32, 2**31])
def test_plan_arguments_past_32_bits_are_refused(name, beyond):
    """Not cut off to the value that is left of them, here a good one."""
    good = dict(heads_q=4, heads_kv=2, head_dim=64, window=0, device=-1)[name]
    with pytest.raises(ValueError, match=f"{name} .*32 bits"):
        _plan(**{"causal": True, name: good + beyond if beyond != 2**31 else beyond})


@pytest.mark.parametrize("name", ["heads_q", "heads_kv", "head_dim", "max_q", "max_kv", "device"])
def test_workspace_arguments_past_32_bits_are_refused(name):
    args = dict(heads_q=8, heads_kv=8, head_dim=64, max_q=1, max_kv=1024, device=0)
    args[name] += 2**32
    with pytest.raises(ValueError, match=f"{name} .*32 bits"):
        bsm.bsm_attention_paged_workspace(4, 4, **args)


@pytest.mark.parametrize("name", ["table", "q_start", "kv_len"])
@pytest.mark.parametrize("off", [1, 2])
def test_paged_arrays_off_their_alignment_are_refused(name, off):
    assert _paged(**{name: (1 << 40) + off}) == bsm.BSM_ERR_INVALID_ARG
    assert "aligned" in bsm.bsm_last_error()


def test_oracle_slots_of_idle_requests_by_hand():
    """Room for 6 tokens: request 1's go past it, and with them 3's; 0 and 2 keep what they have, 2 without
    asking for anything."""
    table = [[4, -1], [5, -1], [6, 7], [-1, -1]]
    q_start, kv_len, out, slots, taken = oa.slots([1, 2, 7, 0], [3, 4, 0, 1], 4, 12, table, [8, 9], 2, 6)
    assert kv_len == [4, 0, 7, 0] and q_start == [0, 3, 6, 6, 6] and taken == [0, 2]
    assert out.tolist() == table and slots.tolist() == [17, 18, 19, -1, -1, -1]


def test_every_kernel_of_sequences_has_a_tested_batch():
    """Heads up to 64 have units of 64 and 128 rows of either kind, with steps of 128 keys in the smaller
    query units of few; longer heads have units of 128 keys only. Units of the gradient may have parts."""
    want = set()
    for d in (64, 96, 128):
        queries = [(128, 64), (64, 64)] + ([(64, 128)] if d == 64 else [])
        want |= {("forward", d, rows, step, False) for rows, step in queries}
        want |= {("dq", d, rows, step, parts) for rows, step in queries for parts in (False, True)}
        want |= {("dk and dv", d, rows, 64, parts) for rows in ((128, 64) if d == 64 else (128,)) for parts in (False, True)}
    have = set()
    for q_len, kv_len, hq, hk, d, causal, window, n_cu in FORMS:
        p = _plan(q_len, kv_len, heads_q=hq, heads_kv=hk, head_dim=d, causal=causal, window=window, topology=dict(n_xcd=8, n_cu=n_cu))
        have |= kernels_of(d, bsm.bsm_attention_plan_describe(p)["forms"])
    assert have == want


@pytest.mark.parametrize("scale", [3e38, float(np.nextafter(np.float32(2.0 ** 127), np.float32(np.inf))), float("inf"), -1.0])
def test_scales_whose_exponents_have_no_room_are_refused(scale):
    assert _paged(scale=scale) == bsm.BSM_ERR_INVALID_ARG
    assert "scale" in bsm.bsm_last_error()


def test_streams_of_other_devices_are_refused():
    stream = SimpleNamespace(cuda_stream=1234, device_index=1)
    assert att._stream(1, stream) == 1234 and att._stream(0, 5678) == 5678
    with pytest.raises(ValueError, match="cuda:1.*cuda:0"):
        att._stream(0, stream)


@pytest.mark.parametrize("window", [2**31 - 1, 2**30 + 1, 2**30, 2**30 - 1])
def test_the_largest_windows_hide_nothing(window):
    d = bsm.bsm_attention_plan_describe(_plan([100, 5], [50, 700], causal=True, window=window))
    assert d["window"] == window and d["pairs"] == sum(int(oa.seen(n, m, True).sum()) for n, m in ((100, 50), (5, 700)))
