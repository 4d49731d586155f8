"""fp64 attention of one head, its gradient, and the paged cache's bookkeeping, in plain numpy.

Masks, probabilities and gradients are formed in full from the definitions; nothing here shares
code with the library."""

from __future__ import annotations

import numpy as np


def seen(n: int, m: int, causal: bool, window: int = 0) -> np.ndarray:
    """(n, m) truth values: query row i, at position i + m - n, sees key j."""
    j = np.arange(m)[None, :]
    p = (np.arange(n) + m - n)[:, None]
    s = np.ones((n, m), bool)
    if causal:
        s &= j <= p
        if window > 0:
            s &= j > p - window
    return s


def forward(q, k, v, scale, causal=False, window=0):
    """o (n, d), lse (n) and probabilities (n, m) of q (n, d) over k and v (m, d), all fp64. Rows
    that see nothing, or only scores of -inf: o = 0, lse = -inf."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    n, m = q.shape[0], k.shape[0]
    s = np.where(seen(n, m, causal, window), (q @ k.T) * scale, -np.inf)
    top = s.max(axis=1, initial=-np.inf)
    ref = np.where(top == -np.inf, 0.0, top)
    e = np.exp(s - ref[:, None])
    total = e.sum(axis=1)
    with np.errstate(divide="ignore"):
        lse = np.where(total == 0, -np.inf, ref + np.log(total))
    p = e / np.where(total == 0, 1.0, total)[:, None]
    return p @ v, lse, p


def backward(q, k, v, o, lse, dout, scale, causal=False, window=0):
    """dq, dk, dv of one head from the saved o and lse."""
    q, k, v, o, dout = (np.asarray(x, np.float64) for x in (q, k, v, o, dout))
    n, m = q.shape[0], k.shape[0]
    mask = seen(n, m, causal, window) & np.isfinite(lse)[:, None]
    s = (q @ k.T) * scale
    p = np.where(mask, np.exp(np.where(mask, s - np.where(np.isfinite(lse), lse, 0.0)[:, None], 0.0)), 0.0)
    ds = p * (dout @ v.T - (dout * o).sum(axis=1, keepdims=True))
    return scale * ds @ k, scale * ds.T @ q, p.T @ dout


def slots(cached, fresh, page_size, n_pages, table, free_pages, n_free, n_slots):
    """What a step's lengths give, request by request: q_start, kv_len, table, slots, taken."""
    table = np.array(table, copy=True)
    width = table.shape[1]
    q_start, kv_len = [0], []
    out = np.full(n_slots, -1, np.int64)
    n_free = max(0, min(int(n_free), len(free_pages)))
    at = 0        # pages that the requests so far ask for
    taken = refused = tokens = 0
    for b, (c, f) in enumerate(zip(cached, fresh)):
        c, f = max(0, int(c)), max(0, int(f))
        held, full = -(-c // page_size), -(-(c + f) // page_size)
        need = 0 if full > width else full - held
        ok = full <= width and (f == 0 or tokens + f <= n_slots) and (need == 0 or at + need <= n_free)
        if ok:
            for i in range(need):
                page = int(free_pages[at + i])
                table[b, held + i] = page if 0 <= page < n_pages else -1
            for t in range(f):
                place = c + t
                page = int(table[b, place // page_size])
                if 0 <= page < n_pages:
                    out[tokens + t] = page * page_size + place % page_size
            if need:
                taken = at + need
        else:
            refused += 1
        at += need
        tokens += f
        q_start.append(min(tokens, n_slots))
        kv_len.append(c + f if ok else 0)
    return q_start, kv_len, table, out, [taken, refused]
