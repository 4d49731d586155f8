"""Helpers of the attention tests: operands in every layout, and how far bf16 results may be from
the fp64 oracle.

Bounds, from the operations alone (u = 2^-8, half a step of bf16; e = 2^-24, of fp32).  A score is
an fp32 sum of d exact products, in any order, times two rounded factors: off by at most
a = 2 (d + 2) e scale sum|q||k|.  Its exponential, taken from a difference of numbers of size at
most |s| + |ref|, is off by a relative a + 4 e (|s| + |ref| + 4).  P (and dS) are rounded to bf16
once, u relative; a product over m rows adds 2 m e of its absolute sum; the result is rounded once
more, u of its value."""

from __future__ import annotations

import numpy as np
import torch

import oracle.attention as oa

U, E = 2.0 ** -8, 2.0 ** -24


def to64(t: torch.Tensor) -> np.ndarray:
    return t.detach().to("cpu").double().numpy()


def exp_error(q, k, scale, ref):
    """Relative error of every probability of one head whose exponents are taken from `ref` (rows)."""
    d = q.shape[1]
    s = np.abs(q @ k.T) * scale
    a = 2 * (d + 2) * E * scale * (np.abs(q) @ np.abs(k).T)
    r = np.where(np.isfinite(ref), np.abs(ref), 0.0)[:, None]
    return a + 4 * E * (s + r + 4)


def forward_bound(q, k, v, scale, causal, window, p, lse, o):
    """|o - oracle| per element, and |lse - oracle| per row."""
    m = k.shape[0]
    # the row's sum carries the errors of all its terms, so each weight does twice
    rel = exp_error(q, k, scale, lse) * p
    worst = rel.sum(axis=1, keepdims=True)
    av = np.abs(v)
    err = (rel + p * (worst + 4 * m * E)) @ av + U * (p @ av)
    lse_err = worst[:, 0] + 2 * m * E + 8 * E * (np.abs(np.where(np.isfinite(lse), lse, 0.0)) + 1)
    return 1.01 * err + U * np.abs(o) + 1e-30, 1.01 * lse_err


def backward_bound(q, k, v, o, lse, dout, scale, causal, window, dq, dk, dv):
    n, m, d = q.shape[0], k.shape[0], q.shape[1]
    mask = oa.seen(n, m, causal, window) & np.isfinite(lse)[:, None]
    s = (q @ k.T) * scale
    p = np.where(mask, np.exp(np.where(mask, s - np.where(np.isfinite(lse), lse, 0.0)[:, None], 0.0)), 0.0)
    rel = exp_error(q, k, scale, lse)
    dp, delta = dout @ v.T, (dout * o).sum(axis=1, keepdims=True)
    ds = np.abs(p * (dp - delta))
    # dP and delta are fp32 sums of d products, their difference rounds once more
    dp_err = 2 * (d + 2) * E * (np.abs(dout) @ np.abs(v).T + (np.abs(dout) * np.abs(o)).sum(axis=1, keepdims=True))
    ds_err = p * dp_err * (1 + rel) + ds * (rel + 2 * E)
    total = ds_err + U * (ds + ds_err)
    sums = lambda w, x, r: (w * (1 + 2 * r * E) + 0) @ np.abs(x)  # noqa: E731
    b_dq = scale * (sums(total, k, m) + 2 * m * E * (ds @ np.abs(k)))
    b_dk = scale * (sums(total.T, q, n) + 2 * n * E * (ds.T @ np.abs(q)))
    pe = p * (rel + U * (1 + rel))
    b_dv = sums(pe.T, dout, n) + 2 * n * E * (p.T @ np.abs(dout))
    return b_dq, b_dk, b_dv


# Batches that between them run every kernel of the forward pass and of the gradient, each as
# (q_len, kv_len, query heads, kv heads, head dim, causal, window, compute units to plan for); in the
# layouts "packed" (tiles go straight to LDS) and "shifted" (through registers).
FORMS = [
    ([368, 111, 50], [201, 41, 502], 4, 2, 96, True, 312, 1),
    ([31, 84, 198], [2440, 3602, 3687], 2, 2, 40, True, 287, 6),
    ([33, 14, 498], [997, 1289, 1453], 1, 1, 128, True, 110, 2),
    ([90, 159, 314], [887, 1815, 1245], 2, 1, 64, True, 695, 12),
    ([26, 357, 38], [2945, 1633, 621], 2, 1, 72, True, 543, 24),
    ([46, 446, 36], [2256, 988, 1695], 2, 1, 128, True, 252, 24),
    ([302, 497, 202], [64, 314, 1081], 4, 2, 40, True, 302, 24),
    ([376, 140, 235], [1294, 2642, 94], 2, 1, 40, False, 0, 24),
    ([34, 141, 171], [2088, 1178, 2246], 1, 1, 104, True, 544, 24),
    ([352, 13, 233], [215, 1398, 1066], 2, 1, 96, True, 610, 24),
    ([89, 50, 122], [1357, 60, 58], 2, 2, 104, True, 874, 8),
    ([264, 244, 341], [161, 1385, 68], 1, 1, 96, True, 880, 8),
    ([240, 64, 36], [562, 5346, 3987], 3, 1, 64, False, 0, 8),
    ([167, 65], [828, 11128], 3, 3, 64, False, 0, 3),
]


def kernels_of(head_dim, forms):
    """The kernels that a plan of these forms runs, as (pass, padded head dimension, rows of a unit, keys
    of a step, parts)."""
    d = 64 if head_dim <= 64 else 96 if head_dim <= 96 else 128
    half_forward, half_dq, half_keys, long_steps, dq_parts, key_parts = (bool(forms & 1 << i) for i in range(6))
    return {("forward", d, 64 if half_forward else 128, 128 if half_forward and long_steps else 64, False),
            ("dq", d, 64 if half_dq else 128, 128 if half_dq and long_steps else 64, dq_parts),
            ("dk and dv", d, 64 if half_keys else 128, 64, key_parts)}


class Batch:
    """Sequences in one layout on the GPU. layouts: packed (tokens, heads, dim); fused (q, k, v
    views of one tensor; needs q_len == kv_len); padded (batch, rows, heads, dim); heads_first
    (batch, heads, rows, dim) passed transposed; shifted (packed, first element off every 16-byte
    boundary, and a gap of NaN rows between sequences)."""

    def __init__(self, q_len, kv_len, hq, hk, d, layout="packed", seed=0, sigma=2.0, device="cuda"):
        self.q_len, self.kv_len, self.hq, self.hk, self.d = list(q_len), list(kv_len), hq, hk, d
        self.layout, self.device = layout, device
        self.gen = torch.Generator().manual_seed(seed)
        b = len(q_len)
        if layout in ("padded", "heads_first"):
            self.q_start = self.kv_start = 0
            sq, sk = max(q_len) + 3, max(kv_len) + 5
            self.q_at, self.kv_at = [0] * b, [0] * b
            self.q_shape = (b, sq, hq, d) if layout == "padded" else (b, hq, sq, d)
            self.kv_shape = (b, sk, hk, d) if layout == "padded" else (b, hk, sk, d)
        else:
            gap = 2 if layout == "shifted" else 0
            self.q_at = [int(x) for x in np.cumsum([0] + [n + gap for n in q_len])[:-1]]
            self.kv_at = [int(x) for x in np.cumsum([0] + [n + gap for n in kv_len])[:-1]]
            self.q_start = self.q_at if gap else None
            self.kv_start = self.kv_at if gap else None
            self.q_shape = (sum(q_len) + gap * b, hq, d)
            self.kv_shape = (sum(kv_len) + gap * b, hk, d)
        if layout == "fused":
            assert self.q_len == self.kv_len
            x = torch.randn((sum(q_len), hq + 2 * hk, d), generator=self.gen)
            x[:, :hq] *= sigma
            x = x.to(torch.bfloat16).to(device)
            self.q, self.k, self.v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
        else:
            self.q = self.operand("q", sigma)
            self.k, self.v = self.operand("kv"), self.operand("kv")

    def empty(self, kind, fill=float("nan")):
        shape = self.q_shape if kind == "q" else self.kv_shape
        n = int(np.prod(shape))
        if self.layout == "shifted":
            x = torch.full((n + 9,), fill, dtype=torch.bfloat16).to(self.device)[3:3 + n].view(shape)
        else:
            x = torch.full(shape, fill, dtype=torch.bfloat16, device=self.device)
        return x.transpose(1, 2) if self.layout == "heads_first" else x

    def operand(self, kind, sigma=1.0):
        """N(0, sigma^2) in the sequences' rows, NaN everywhere else."""
        x = self.empty(kind)
        for b in range(len(self.q_len)):
            r = self.rows(x, b, kind)
            r.copy_((sigma * torch.randn(r.shape, generator=self.gen)).to(torch.bfloat16))
        return x

    def rows(self, x, b, kind):
        """(rows, heads, dim) view of sequence b."""
        n = (self.q_len if kind == "q" else self.kv_len)[b]
        at = (self.q_at if kind == "q" else self.kv_at)[b]
        return x[b, :n] if x.dim() == 4 else x[at:at + n]

    def untouched(self, x, kind) -> bool:
        """Everything outside the sequences still has the NaN it was filled with."""
        y = x.clone()
        for b in range(len(self.q_len)):
            self.rows(y, b, kind).fill_(float("nan"))
        return bool(torch.isnan(y).all())

    def plan_args(self, causal, window=0, schedule="balanced"):
        return dict(q_len=self.q_len, kv_len=self.kv_len, heads_q=self.hq, heads_kv=self.hk,
                    head_dim=self.d, causal=causal, window=window, q_start=self.q_start,
                    kv_start=self.kv_start, schedule=schedule)


def check_forward(batch: Batch, o, lse, scale, causal, window=0):
    at, g = 0, batch.hq // batch.hk
    for b, n in enumerate(batch.q_len):
        q, k, v, got = (to64(batch.rows(x, b, kind)) for x, kind in
                        ((batch.q, "q"), (batch.k, "kv"), (batch.v, "kv"), (o, "q")))
        for h in range(batch.hq):
            ref, ref_lse, p = oa.forward(q[:, h], k[:, h // g], v[:, h // g], scale, causal, window)
            tol, tol_lse = forward_bound(q[:, h], k[:, h // g], v[:, h // g], scale, causal, window, p, ref_lse, ref)
            err = np.abs(got[:, h] - ref)
            assert (err <= tol).all(), f"sequence {b} head {h}: worst excess {(err - tol).max():.3e} at {np.argwhere(~(err <= tol))[:4].tolist()}"
            if lse is not None:
                mine = to64(lse)[h, at:at + n]
                dead = np.isinf(ref_lse)
                assert np.array_equal(mine == -np.inf, dead), f"sequence {b} head {h}: rows that see nothing"
                err = np.abs(mine[~dead] - ref_lse[~dead])
                assert (err <= tol_lse[~dead]).all(), f"sequence {b} head {h}: lse off by {err.max():.3e}"
        at += n
    assert batch.untouched(o, "q"), "rows outside the sequences were written"


def check_backward(batch: Batch, o, lse, dout, dq, dk, dv, scale, causal, window=0):
    at, g = 0, batch.hq // batch.hk
    for b, n in enumerate(batch.q_len):
        q, k, v, oo, do, gq, gk, gv = (to64(batch.rows(x, b, kind)) for x, kind in (
            (batch.q, "q"), (batch.k, "kv"), (batch.v, "kv"), (o, "q"), (dout, "q"), (dq, "q"), (dk, "kv"), (dv, "kv")))
        for hk in range(batch.hk):
            sums = [np.zeros(k[:, 0].shape) for _ in range(4)]  # dk, dv and their bounds
            for h in range(hk * g, hk * g + g):
                row = to64(lse)[h, at:at + n]
                # rows that see nothing count as zeros, whatever they hold
                dead = np.isinf(row)[:, None]
                args = [np.where(dead, 0.0, x) for x in (q[:, h], oo[:, h], do[:, h])]
                ref = oa.backward(args[0], k[:, hk], v[:, hk], args[1], row, args[2], scale, causal, window)
                bound = backward_bound(args[0], k[:, hk], v[:, hk], args[1], row, args[2], scale, causal, window, *ref)
                tol = 1.01 * bound[0] + U * np.abs(ref[0]) + 1e-30
                err = np.abs(gq[:, h] - ref[0])
                assert (err <= tol).all(), f"sequence {b} head {h}: dq, worst excess {(err - tol).max():.3e} at {np.argwhere(~(err <= tol))[:4].tolist()}"
                for i, x in enumerate((ref[1], ref[2], bound[1], bound[2])):
                    sums[i] += x
            for name, got, ref, bound in (("dk", gk[:, hk], sums[0], sums[2]), ("dv", gv[:, hk], sums[1], sums[3])):
                tol = 1.02 * bound + U * np.abs(ref) + 1e-30
                err = np.abs(got - ref)
                assert (err <= tol).all(), f"sequence {b} kv head {hk}: {name}, worst excess {(err - tol).max():.3e} at {np.argwhere(~(err <= tol))[:4].tolist()}"
        at += n
    for x, kind in ((dq, "q"), (dk, "kv"), (dv, "kv")):
        assert batch.untouched(x, kind), "rows outside the sequences were written"
