"""Attention of ragged sequences and its gradient against the fp64 oracle, through the C ABI."""

import numpy as np
import pytest
import torch

import paper_2002_07062_amd as bsm
from attention_util import FORMS, Batch, check_backward, check_forward, kernels_of

pytestmark = pytest.mark.gpu

# q_len, kv_len (None: the same), query heads, kv heads, head dim, causal, window, layout
CASES = [
    ([1], None, 1, 1, 64, False, 0, "packed"),
    ([64, 64], None, 2, 2, 64, False, 0, "packed"),
    ([31, 32, 33, 1], None, 2, 1, 64, True, 0, "packed"),
    ([63, 64, 65, 127, 128, 129], None, 2, 2, 128, True, 0, "packed"),
    ([200, 77], None, 4, 2, 128, False, 0, "fused"),
    ([300, 1, 150], None, 4, 1, 64, True, 0, "fused"),
    ([5, 130], [90, 333], 2, 2, 80, True, 0, "packed"),      # a prefix before the queries
    ([130, 40], [70, 40], 2, 1, 64, True, 0, "packed"),      # more queries than keys: rows that see nothing
    ([17, 0, 20], [40, 30, 0], 2, 2, 64, False, 0, "packed"),  # no queries; no keys
    ([17, 0, 20], [40, 30, 0], 3, 3, 128, True, 0, "shifted"),
    ([200, 90], None, 2, 2, 64, True, 1, "packed"),          # every row sees itself alone
    ([300, 129], [310, 200], 2, 1, 128, True, 70, "packed"),
    ([100, 260], None, 3, 3, 8, True, 33, "packed"),
    ([100, 37], None, 2, 2, 24, False, 0, "padded"),
    ([66, 150], [150, 151], 8, 2, 96, True, 0, "padded"),
    ([140, 33], None, 4, 4, 72, True, 0, "heads_first"),
    ([64, 129], [200, 64], 6, 2, 120, False, 0, "heads_first"),
    ([95, 96, 97], None, 5, 1, 40, True, 64, "shifted"),
    ([513], None, 1, 1, 128, True, 0, "packed"),
]


def _name(c):
    return "-".join(str(x) for x in (c[0], c[1] or "", *c[2:])).replace(" ", "")


def _batch(case, seed=3):
    q_len, kv_len, hq, hk, d, _, _, layout = case
    return Batch(q_len, kv_len or q_len, hq, hk, d, layout, seed)


def _run(batch, causal, window, schedule="balanced", scale=None, lse=True, n_cu=0):
    plan = bsm.bsm_attention_plan_create(**batch.plan_args(causal, window, schedule), topology=dict(n_cu=n_cu) if n_cu else None)
    o = batch.empty("q")
    rows = torch.full((batch.hq, sum(batch.q_len)), 7.0, device="cuda") if lse else None
    bsm.bsm_attention_execute(plan, batch.q, batch.k, batch.v, o, lse=rows, scale=scale)
    torch.cuda.synchronize()
    return plan, o, rows


# planned for one compute unit the work is not cut into halves and parts, for all of them it is
@pytest.mark.parametrize("n_cu", [0, 1])
@pytest.mark.parametrize("case", CASES, ids=_name)
def test_forward_matches_the_oracle(case, n_cu):
    batch, scale = _batch(case), 1 / np.sqrt(case[4])
    plan, o, lse = _run(batch, case[5], case[6], n_cu=n_cu)
    check_forward(batch, o, lse, float(np.float32(scale)), case[5], case[6])
    plan.destroy()


@pytest.mark.parametrize("n_cu", [0, 1])
@pytest.mark.parametrize("case", CASES, ids=_name)
def test_backward_matches_the_oracle(case, n_cu):
    batch, scale = _batch(case, 5), float(np.float32(1 / np.sqrt(case[4])))
    plan, o, lse = _run(batch, case[5], case[6], n_cu=n_cu)
    dout = batch.operand("q")
    dq, dk, dv = batch.empty("q"), batch.empty("kv"), batch.empty("kv")
    bsm.bsm_attention_backward(plan, batch.q, batch.k, batch.v, o, lse, dout, dq, dk, dv)
    torch.cuda.synchronize()
    check_backward(batch, o, lse, dout, dq, dk, dv, scale, case[5], case[6])
    plan.destroy()


@pytest.mark.parametrize("case", [CASES[3], CASES[5], CASES[11]], ids=_name)
def test_schedules_and_repeats_give_the_same_bits(case):
    batch = _batch(case, 7)
    dout = batch.operand("q")
    seen = []
    for schedule in ("balanced", "xcd", "rr", "balanced"):
        plan, o, lse = _run(batch, case[5], case[6], schedule)
        grads = [batch.empty("q"), batch.empty("kv"), batch.empty("kv")]
        bsm.bsm_attention_backward(plan, batch.q, batch.k, batch.v, o, lse, dout, *grads)
        torch.cuda.synchronize()
        seen.append([x.contiguous().view(torch.int16) for x in (o, *grads)] + [lse.view(torch.int32)])
        plan.destroy()
    for other in seen[1:]:
        for x, y in zip(seen[0], other):
            assert torch.equal(x, y)


# few keys for many query rows, or the reverse: several workgroups share a unit
PARTED = [
    ([2048], None, 2, 1, 128, True, 0, "packed"),
    ([1500], [1100], 4, 1, 64, False, 0, "shifted"),
    ([1030, 0, 31, 700], [1500, 9, 0, 40], 4, 1, 80, True, 0, "padded"),
    ([1700, 40], None, 8, 1, 96, True, 300, "fused"),
    ([4000], [1], 1, 1, 40, False, 0, "heads_first"),
    ([3, 40], [3000, 900], 2, 1, 64, True, 0, "packed"),     # few queries: several share a row's keys
    ([150], [1600], 3, 1, 128, False, 0, "shifted"),
    ([70, 1], [2000, 700], 2, 2, 96, True, 1500, "padded"),
]


@pytest.mark.parametrize("case", PARTED, ids=_name)
def test_gradients_of_few_rows(case):
    batch, scale = _batch(case, 9), float(np.float32(1 / np.sqrt(case[4])))
    plan, o, lse = _run(batch, case[5], case[6])
    assert plan.workspace_bytes > 4 * lse.numel() + 16  # there are parts
    dout = batch.operand("q")
    seen = []
    for schedule in ("balanced", "xcd", "rr"):
        plan = bsm.bsm_attention_plan_create(**batch.plan_args(case[5], case[6], schedule))
        dq, dk, dv = batch.empty("q"), batch.empty("kv"), batch.empty("kv")
        ws = torch.full((plan.workspace_bytes,), 255, dtype=torch.uint8, device="cuda")  # NaN
        bsm.bsm_attention_backward(plan, batch.q, batch.k, batch.v, o, lse, dout, dq, dk, dv, workspace=ws)
        torch.cuda.synchronize()
        check_backward(batch, o, lse, dout, dq, dk, dv, scale, case[5], case[6])
        seen.append([x.contiguous().view(torch.int16) for x in (dq, dk, dv)])
    assert all(torch.equal(x, y) for other in seen[1:] for x, y in zip(seen[0], other))


@pytest.mark.parametrize("scale", [1e-3, 1.0, 8.0])
def test_scales(scale):
    """Flat rows, and rows that one key takes almost whole (scores of several hundred)."""
    batch = Batch([150, 70], [150, 90], 2, 1, 64, "packed", 11, sigma=1.0)
    plan, o, lse = _run(batch, True, 0, scale=scale)
    check_forward(batch, o, lse, float(np.float32(scale)), True)
    dout = batch.operand("q")
    grads = [batch.empty("q"), batch.empty("kv"), batch.empty("kv")]
    bsm.bsm_attention_backward(plan, batch.q, batch.k, batch.v, o, lse, dout, *grads, scale=scale)
    check_backward(batch, o, lse, dout, *grads, float(np.float32(scale)), True)
    plan.destroy()


def test_rising_scores_move_the_reference():
    """Keys whose scores grow by steps of 1 to 40 along the sequence, so that a row's reference
    moves at some tiles and not at others."""
    batch = Batch([80], [700], 1, 1, 64, "packed", 13, sigma=0.0)
    j = torch.arange(700, dtype=torch.float32)
    batch.q[:, 0, 0] = torch.linspace(0.25, 4.0, 80).to(torch.bfloat16).cuda()
    batch.k[:, 0] = 0
    batch.k[:, 0, 0] = (j // 64 * torch.linspace(0.1, 10, 700)).to(torch.bfloat16).cuda()
    plan, o, lse = _run(batch, False, 0, scale=1.0)
    check_forward(batch, o, lse, 1.0, False)
    plan.destroy()


def test_scores_of_infinity():
    """Scores of -inf take no weight, a row of nothing else is zero, +inf or NaN makes its row NaN;
    other rows keep their values."""
    batch = Batch([40], [70], 1, 1, 64, "packed", 17)
    inf = float("inf")
    batch.q[:, 0, 0] = 1.0
    batch.k[:, 0, 0] = 0.0
    batch.k[5, 0] = 0.0
    batch.k[5, 0, 0] = -inf            # -inf for every query
    plan, o, lse = _run(batch, False, 0)
    check = Batch([40], [69], 1, 1, 64, "packed", 17)
    keep = [j for j in range(70) if j != 5]
    check.q, check.k, check.v = batch.q, batch.k[keep], batch.v[keep]
    check_forward(check, o, lse, 0.125, False)
    batch.k[:, 0] = 0.0
    batch.k[:, 0, 0] = -inf
    plan, o, lse = _run(batch, False, 0)
    assert (o == 0).all() and (lse == -inf).all()
    batch.k[:, 0, 0] = 0.0
    batch.k[9, 0, 0] = inf             # +inf where q > 0, -inf where q < 0
    batch.q[::2, 0, 0] = -1.0
    plan, o, lse = _run(batch, False, 0)
    assert torch.isnan(o[1::2]).all() and torch.isnan(lse[0, 1::2]).all()
    assert torch.isfinite(o[::2].float()).all()


def test_rows_that_see_nothing_take_no_gradient_whatever_they_hold():
    batch = Batch([100], [60], 2, 1, 64, "packed", 19)
    plan, o, lse = _run(batch, True, 0)
    dout = batch.operand("q")
    dout[:40] = float("nan")
    batch.q[:40] = float("inf")
    o[:40] = float("nan")
    grads = [batch.empty("q"), batch.empty("kv"), batch.empty("kv")]
    bsm.bsm_attention_backward(plan, batch.q, batch.k, batch.v, o, lse, dout, *grads)
    torch.cuda.synchronize()
    assert (grads[0][:40] == 0).all()
    check_backward(batch, o, lse, dout, *grads, 0.125, True)
    plan.destroy()


def test_gradients_match_differences():
    """Central differences of the fp64 forward pass along random directions."""
    import oracle.attention as oa
    batch = Batch([37], [50], 2, 1, 64, "packed", 23, sigma=1.0)
    plan, o, lse = _run(batch, True, 0)
    dout = batch.operand("q")
    grads = [batch.empty("q"), batch.empty("kv"), batch.empty("kv")]
    bsm.bsm_attention_backward(plan, batch.q, batch.k, batch.v, o, lse, dout, *grads)
    q, k, v, do = (x.double().cpu().numpy() for x in (batch.q, batch.k, batch.v, dout))
    got = [x.double().cpu().numpy() for x in grads]

    def loss(q, k, v):
        return sum((oa.forward(q[:, h], k[:, 0], v[:, 0], 0.125, True)[0] * do[:, h]).sum() for h in range(2))

    rng = np.random.default_rng(1)
    for i, x in enumerate((q, k, v)):
        d = rng.standard_normal(x.shape)
        step = 1e-5
        args = [[q, k, v], [q, k, v]]
        args[0][i], args[1][i] = x + step * d, x - step * d
        want = (loss(*args[0]) - loss(*args[1])) / (2 * step)
        # errors of the gradients' elements are independent roundings of about 2^-8, four deviations
        tol = 4 * 2 ** -8 * np.sqrt(((got[i] * d) ** 2).sum()) + 1e-3 * abs(want)
        assert abs((got[i] * d).sum() - want) <= tol
    plan.destroy()


def test_a_fused_gradient_tensor():
    """dq, dk and dv as views of one tensor, like q, k and v."""
    batch = Batch([90, 61], [90, 61], 4, 2, 64, "fused", 29)
    plan, o, lse = _run(batch, True, 0)
    dout = batch.operand("q")
    x = torch.full((151, 8, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    dq, dk, dv = x[:, :4], x[:, 4:6], x[:, 6:]
    bsm.bsm_attention_backward(plan, batch.q, batch.k, batch.v, o, lse, dout, dq, dk, dv)
    check_backward(batch, o, lse, dout, dq, dk, dv, 0.125, True)
    plan.destroy()


def test_shared_keys_and_values():
    """Two sequences that read the same keys, and heads that read one by a stride of 0; their
    gradients are refused in the shared rows and right in rows of their own."""
    g = torch.Generator().manual_seed(31)
    q = torch.randn((60, 4, 64), generator=g).to(torch.bfloat16).cuda()
    kv = torch.randn((50, 1, 64), generator=g).to(torch.bfloat16).cuda()
    wide = kv.expand(-1, 2, -1)
    plan = bsm.bsm_attention_plan_create([30, 30], [50, 50], heads_q=4, heads_kv=2, head_dim=64, kv_start=[0, 0])
    o, lse = torch.empty_like(q), torch.empty((4, 60), device="cuda")
    bsm.bsm_attention_execute(plan, q, wide, wide, o, lse=lse)
    batch = Batch([30, 30], [50, 50], 4, 2, 64, "packed", 1)
    batch.q = q
    batch.k = batch.v = torch.cat([wide, wide]).contiguous()
    check_forward(batch, o, lse, 0.125, False)
    dk = torch.empty((50, 2, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(bsm.BsmError) as e:
        bsm.bsm_attention_backward(plan, q, wide, wide, o, lse, q, torch.empty_like(q), dk, torch.empty_like(dk))
    assert e.value.status == bsm.BSM_ERR_INVALID_ARG
    own = bsm.bsm_attention_plan_create([30, 30], [50, 50], heads_q=4, heads_kv=2, head_dim=64)
    dout = batch.operand("q")
    grads = [batch.empty("q"), batch.empty("kv"), batch.empty("kv")]
    bsm.bsm_attention_backward(own, q, batch.k, batch.v, o, lse, dout, *grads)
    check_backward(batch, o, lse, dout, *grads, 0.125, False)


@pytest.mark.parametrize("stride,rows", [((1 << 24) - 8, 290), (45_000_000, 100)])
def test_rows_past_32_bits(stride, rows):
    """Operands and gradients whose rows are up to 2^32 elements and more from the first."""
    batch = Batch([rows], [rows], 1, 1, 64, "packed", 53)
    far = [torch.empty((rows - 1) * stride + 4 * 64, dtype=torch.bfloat16, device="cuda") for _ in range(3)]

    def view(buffer, x):
        return torch.as_strided(far[buffer], (rows, 1, 64), (stride, 64, 1), 64 * x)

    q, k, v, dout = (view(0, x) for x in range(4))
    o, dq, dk, dv = view(1, 0), view(2, 0), view(2, 1), view(2, 2)
    for x, y in zip((q, k, v), (batch.q, batch.k, batch.v)):
        x.copy_(y)
    dout.copy_(batch.operand("q"))
    plan = bsm.bsm_attention_plan_create([rows], heads_q=1, head_dim=64, causal=True)
    lse = torch.empty((1, rows), device="cuda")
    with pytest.raises(bsm.BsmError) as e:  # an output between the operands' rows
        bsm.bsm_attention_execute(plan, q, k, v, dout)
    assert e.value.status == bsm.BSM_ERR_ALIAS
    bsm.bsm_attention_execute(plan, q, k, v, o, lse=lse)
    bsm.bsm_attention_backward(plan, q, k, v, o, lse, dout, dq, dk, dv)
    torch.cuda.synchronize()
    check_forward(batch, o, lse, 0.125, True)
    check_backward(batch, o, lse, dout, dq, dk, dv, 0.125, True)
    plan.destroy()


def test_two_streams_with_their_own_workspaces():
    batches = [Batch([300, 120], [300, 120], 4, 2, 128, "packed", s) for s in (41, 42)]
    plan, _, _ = _run(batches[0], True, 0)
    streams = [torch.cuda.Stream() for _ in batches]
    outs = []
    for batch in batches:
        outs.append([batch.empty("q"), torch.empty((4, 420), device="cuda"), batch.operand("q"),
                     batch.empty("q"), batch.empty("kv"), batch.empty("kv"),
                     torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda")])
    torch.cuda.synchronize()
    for batch, st, (o, lse, dout, dq, dk, dv, ws) in zip(batches, streams, outs):
        bsm.bsm_attention_execute(plan, batch.q, batch.k, batch.v, o, lse=lse, stream=st)
        bsm.bsm_attention_backward(plan, batch.q, batch.k, batch.v, o, lse, dout, dq, dk, dv, workspace=ws, stream=st)
    torch.cuda.synchronize()
    scale = float(np.float32(128 ** -0.5))
    for batch, (o, lse, dout, dq, dk, dv, _) in zip(batches, outs):
        check_forward(batch, o, lse, scale, True)
        check_backward(batch, o, lse, dout, dq, dk, dv, scale, True)
    plan.destroy()


def test_a_captured_step_replays():
    """Forward and backward in one captured graph, replayed after new inputs, with eager work in
    between: every replay equals the eager result bit for bit."""
    batch = Batch([130, 77], [130, 77], 4, 2, 64, "packed", 43)
    plan = bsm.bsm_attention_plan_create(**batch.plan_args(True))
    o, lse, dout = batch.empty("q"), torch.empty((4, 207), device="cuda"), batch.operand("q")
    grads = [batch.empty("q"), batch.empty("kv"), batch.empty("kv")]

    def step(ws=None):
        bsm.bsm_attention_execute(plan, batch.q, batch.k, batch.v, o, lse=lse)
        bsm.bsm_attention_backward(plan, batch.q, batch.k, batch.v, o, lse, dout, *grads, workspace=ws)

    step()
    torch.cuda.synchronize()
    ws = torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(ws)
    for _ in range(3):
        for x in (batch.q, batch.k, batch.v, dout):
            x.copy_(torch.randn(x.shape, generator=batch.gen).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (o, lse, *grads)]
        step()
        torch.cuda.synchronize()
        for x, y in zip(got, (o, lse, *grads)):
            assert torch.equal(x, y)
    del graph
    plan.destroy()


# "no limit" as a window: the largest numbers, beside rows that see nothing (more queries than keys)
@pytest.mark.parametrize("n_cu", [0, 1])
@pytest.mark.parametrize("window", [2**31 - 1, 2**31 - 40, 2**30 + 1])
@pytest.mark.parametrize("q_len,kv_len,d", [([100], [50], 64), ([300, 40, 9], [131, 10, 9], 128), ([1500], [1100], 64)])
def test_the_largest_windows_hide_nothing(q_len, kv_len, d, window, n_cu):
    batch, scale = Batch(q_len, kv_len, 2, 1, d, "packed", 59), float(np.float32(d ** -0.5))
    plan, o, lse = _run(batch, True, window, n_cu=n_cu)
    check_forward(batch, o, lse, scale, True)
    dout = batch.operand("q")
    grads = [batch.empty("q"), batch.empty("kv"), batch.empty("kv")]
    bsm.bsm_attention_backward(plan, batch.q, batch.k, batch.v, o, lse, dout, *grads)
    torch.cuda.synchronize()
    check_backward(batch, o, lse, dout, *grads, scale, True)
    plan.destroy()


@pytest.mark.parametrize("order", [(1, 0, 2), (2, 0, 1), (1, 2, 0), (2, 1, 0)], ids=["rows-batch-heads", "heads-batch-rows", "rows-heads-batch", "heads-rows-batch"])
def test_batches_inside_rows_or_heads(order):
    """(batch, rows, heads, dim) operands and results whose sequences do not follow each other in memory:
    dimension order[i] of the tensor is the i-th outermost."""
    batch = Batch([40, 77, 5], [90, 77, 33], 4, 2, 64, "padded", 61)

    def laid(x):
        y = torch.full([x.shape[i] for i in order] + [64], float("nan"), dtype=torch.bfloat16, device="cuda")
        back = [order.index(i) for i in range(3)]
        return y.permute(*back, 3).copy_(x)

    batch.q, batch.k, batch.v = (laid(x) for x in (batch.q, batch.k, batch.v))
    o, dq, dk, dv = (laid(batch.empty(x)) for x in ("q", "q", "kv", "kv"))
    dout, lse = laid(batch.operand("q")), torch.empty((4, 122), device="cuda")
    plan = bsm.bsm_attention_plan_create(**batch.plan_args(True))
    bsm.bsm_attention_execute(plan, batch.q, batch.k, batch.v, o, lse=lse)
    bsm.bsm_attention_backward(plan, batch.q, batch.k, batch.v, o, lse, dout, dq, dk, dv)
    torch.cuda.synchronize()
    check_forward(batch, o, lse, 0.125, True)
    check_backward(batch, o, lse, dout, dq, dk, dv, 0.125, True)
    for bad in ((512, 64), (64, 64)):  # heads or sequences on top of each other
        with pytest.raises(bsm.BsmError, match="overlap each other"):
            bsm.bsm_attention_execute(plan, batch.q, batch.k, batch.v, torch.as_strided(o, o.shape, (64, *bad, 1)))
    plan.destroy()


def _one_tensor(layout, n=70, hq=2, hk=2, d=64):
    """Two sequences of n rows: starts, and dq, dk, dv as views of one tensor, which comes last."""
    def nan(*shape):
        return torch.full(shape, float("nan"), dtype=torch.bfloat16, device="cuda")

    w = hq + 2 * hk
    if layout == "heads":           # beside each other in a row
        x = nan(2 * n, w, d)
        return None, None, x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:], x
    if layout == "inside heads":
        x = nan(2 * n, hq, 3, d)
        return None, None, x[:, :, 0], x[:, :, 1], x[:, :, 2], x
    if layout == "thirds":
        x = nan(3, 2 * n, hq, d)
        return None, None, x[0], x[1], x[2], x
    if layout == "padded":
        x = nan(2, n + 3, w, d)
        return 0, 0, x[:, :, :hq], x[:, :, hq:hq + hk], x[:, :, hq + hk:], x
    if layout == "heads first":
        x = nan(2, w, n, d)
        t = x.transpose(1, 2)
        return 0, 0, t[:, :, :hq], t[:, :, hq:hq + hk], t[:, :, hq + hk:], x
    if layout == "rows first":
        x = nan(n, 2, w, d)
        t = x.transpose(0, 1)
        return 0, 0, t[:, :, :hq], t[:, :, hq:hq + hk], t[:, :, hq + hk:], x
    x = nan(6 * n, hq, d)           # "blocks": a sequence's three after the other
    return [0, 3 * n], [0, 3 * n], x[:4 * n], x[n:5 * n], x[2 * n:], x


@pytest.mark.parametrize("layout,hq,hk", [("heads", 4, 2), ("inside heads", 2, 2), ("thirds", 2, 2), ("padded", 6, 3),
                                          ("heads first", 4, 1), ("rows first", 2, 2), ("blocks", 2, 2)])
def test_gradients_as_views_of_one_tensor(layout, hq, hk):
    batch = Batch([70, 70], [70, 70], hq, hk, 64, "packed", 67)
    plan, o, lse = _run(batch, True, 0)
    dout = batch.operand("q")
    want = [batch.empty("q"), batch.empty("kv"), batch.empty("kv")]
    bsm.bsm_attention_backward(plan, batch.q, batch.k, batch.v, o, lse, dout, *want)
    q_start, kv_start, *grads, x = _one_tensor(layout, hq=hq, hk=hk)
    plan = bsm.bsm_attention_plan_create([70, 70], heads_q=hq, heads_kv=hk, head_dim=64, causal=True, q_start=q_start, kv_start=kv_start)

    def rows(t, b):
        return t[b, :70] if t.dim() == 4 else t[(q_start or [0, 70])[b]:][:70]

    def laid(t, like):
        y = torch.zeros_like(like)
        for b in (0, 1):
            rows(y, b).copy_(t[70 * b:70 * b + 70])
        return y

    dq, dk, dv = grads
    bsm.bsm_attention_backward(plan, laid(batch.q, dq), laid(batch.k, dk), laid(batch.v, dv), laid(o, dq), lse, laid(dout, dq), dq, dk, dv)
    torch.cuda.synchronize()
    for mine, ref in zip(grads, want):
        for b in (0, 1):
            assert torch.equal(rows(mine, b), ref[70 * b:70 * b + 70])
    for b in (0, 1):
        for t in grads:
            rows(t, b).fill_(float("nan"))
    assert torch.isnan(x).all()


def test_gradients_on_top_of_each_other_are_refused():
    batch = Batch([70, 70], [70, 70], 2, 2, 64, "packed", 71)
    plan, o, lse = _run(batch, True, 0)
    dout = batch.operand("q")
    x = torch.full((300, 6, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    flat, apart = x.view(-1), batch.empty("kv")

    def at(first, row=6 * 64, head=64):
        return torch.as_strided(flat, (140, 2, 64), (row, head, 1), first)

    def call(dq, dk, dv):
        bsm.bsm_attention_backward(plan, batch.q, batch.k, batch.v, o, lse, dout, dq, dk, dv)

    bad = [(at(0), at(0)), (at(0), at(64)), (at(64), at(0)), (at(0), at(8)), (at(0), at(6 * 64)), (at(0), at(20 * 6 * 64 + 64)),
           (at(0), at(320)), (at(0), at(128, row=4 * 64)), (at(0, head=128), at(128, head=128)), (at(0, row=128), at(128 * 139, row=128))]
    for one, two in bad:
        for dq, dk, dv in ((one, two, apart), (one, apart, two), (apart, one, two)):
            with pytest.raises(bsm.BsmError, match="two gradients overlap") as e:
                call(dq, dk, dv)
            assert e.value.status == bsm.BSM_ERR_ALIAS
    torch.cuda.synchronize()
    assert torch.isnan(x).all()
    call(at(0), at(128), at(256))
    call(at(256), at(0, head=128), at(64, head=128))  # every other head
    call(at(0, row=128), at(128 * 140, row=128), apart)
    plan.destroy()


def test_an_error_of_another_call_is_not_reported():
    """The thread's last error belongs to whoever made it: a call after it succeeds and leaves it there."""
    hip = bsm.load()  # the runtime that the library is linked to
    batch = Batch([200, 40], [200, 40], 2, 1, 64, "packed", 73)
    plan = bsm.bsm_attention_plan_create(**batch.plan_args(True))
    o, lse, dout = batch.empty("q"), torch.empty((2, 240), device="cuda"), batch.operand("q")
    grads = [batch.empty("q"), batch.empty("kv"), batch.empty("kv")]
    ws = torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda")
    cache = [torch.zeros((16, 16, 1, 64), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    slots = torch.empty(240, dtype=torch.int64, device="cuda")
    table, lengths, zeros, free, n_free, start, kv, taken = (
        torch.tensor(x, dtype=torch.int32, device="cuda")
        for x in ([[0] * 13] * 2, [200, 40], [0, 0], list(range(16)), [16], [0] * 3, [0] * 2, [0] * 2))
    o2 = torch.empty((240, 2, 64), dtype=torch.bfloat16, device="cuda")
    ws2 = torch.empty(bsm.bsm_attention_paged_workspace(2, 240, 2, 1, 64, 200, 200), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    assert hip.hipGetLastError() == 0
    assert hip.hipSetDevice(1 << 20) != 0
    try:
        bsm.bsm_attention_execute(plan, batch.q, batch.k, batch.v, o, lse=lse)
        bsm.bsm_attention_backward(plan, batch.q, batch.k, batch.v, o, lse, dout, *grads, workspace=ws)
        bsm.bsm_cache_slots(zeros, lengths, 16, 16, table, free, n_free, start, kv, slots, taken)
        bsm.bsm_cache_append(batch.k, batch.v, slots, *cache)
        bsm.bsm_attention_paged(batch.q, *cache, table, start, kv, o2, max_q=200, max_kv=200, workspace=ws2)
    finally:
        left = hip.hipGetLastError()
    assert left != 0
    torch.cuda.synchronize()
    check_forward(batch, o, lse, 0.125, True)
    check_forward(batch, o2, None, 0.125, True)
    check_backward(batch, o, lse, dout, *grads, 0.125, True)
    plan.destroy()


@pytest.mark.parametrize("layout", ["packed", "shifted"])
@pytest.mark.parametrize("case", FORMS, ids=_name)
def test_every_kernel_matches_the_oracle(case, layout):
    q_len, kv_len, hq, hk, d, causal, window, n_cu = case
    batch, scale = Batch(q_len, kv_len, hq, hk, d, layout, 79), float(np.float32(d ** -0.5))
    plan, o, lse = _run(batch, causal, window, n_cu=n_cu)
    print(sorted(kernels_of(d, bsm.bsm_attention_plan_describe(plan)["forms"])))
    check_forward(batch, o, lse, scale, causal, window)
    dout = batch.operand("q")
    grads = [batch.empty("q"), batch.empty("kv"), batch.empty("kv")]
    ws = torch.full((plan.workspace_bytes,), 255, dtype=torch.uint8, device="cuda")  # NaN
    bsm.bsm_attention_backward(plan, batch.q, batch.k, batch.v, o, lse, dout, *grads, workspace=ws)
    torch.cuda.synchronize()
    check_backward(batch, o, lse, dout, *grads, scale, causal, window)
    plan.destroy()


def test_the_largest_scale():
    """Scores of 0 stay equal, others leave one key."""
    batch = Batch([3], [40], 1, 1, 64, "packed", 83)
    batch.q[:] = 0
    batch.q[1, 0, 0], batch.q[2, 0, 0] = 1.0, -1.0
    batch.k[:] = 0
    batch.k[7, 0, 0] = 2.0 ** -100
    plan, o, lse = _run(batch, False, 0, scale=2.0 ** 127)
    check_forward(batch, o, lse, 2.0 ** 127, False)
    plan.destroy()


@pytest.mark.parametrize("n_cu", [0, 1])
@pytest.mark.parametrize("q_len,kv_len,d,window", [(200, 263, 64, 0), (200, 263, 128, 40), (300, 300, 96, 100), (150, 90, 64, 0)])
def test_how_far_a_hidden_nan_reaches(q_len, kv_len, d, window, n_cu):
    """A NaN at a row or key: what shares no visible pair of its blocks (32 rows, 64 keys) keeps its bits."""
    import oracle.attention as oa
    seen = oa.seen(q_len, kv_len, True, window)
    rows, keys = np.arange(q_len), np.arange(kv_len)
    # pairs (block of rows, block of keys) some of which are visible
    near = np.zeros((-(-q_len // 32), -(-kv_len // 64)), bool)
    np.logical_or.at(near, (rows[:, None] // 32, keys[None, :] // 64), seen)

    def run(batch, dout):
        plan, o, lse = _run(batch, True, window, n_cu=n_cu)
        grads = [batch.empty("q"), batch.empty("kv"), batch.empty("kv")]
        bsm.bsm_attention_backward(plan, batch.q, batch.k, batch.v, o, lse, dout, *grads)
        torch.cuda.synchronize()
        plan.destroy()
        return [x.view(torch.int16).cpu().numpy() for x in (o, *grads)]

    batch = Batch([q_len], [kv_len], 2, 1, d, "packed", 89)
    dout = batch.operand("q")
    clean = run(batch, dout)
    for key in (0, 70, kv_len - 1):
        kept = batch.v[key].clone()
        batch.v[key] = float("nan")
        got = run(batch, dout)
        batch.v[key] = kept
        far = ~near[rows // 32, key // 64]
        for x, y in zip(got[:2], clean[:2]):  # o and dq
            assert np.array_equal(x[far], y[far])
    for row in (0, 100, q_len - 1):
        for x in (batch.q, dout):
            kept = x[row].clone()
            x[row] = float("nan")
            got = run(batch, dout)
            x[row] = kept
            far = ~near[row // 32, keys // 64]
            for a, b in zip(got[2:], clean[2:]):  # dk and dv
                assert np.array_equal(a[far], b[far])
            others = np.arange(q_len) != row
            for a, b in zip(got[:2], clean[:2]):
                assert np.array_equal(a[others], b[others])
