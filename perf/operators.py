"""Performance cases of the attention operators: one pass over ragged sequences, its gradient,
and the paged key/value cache (slot maps, writing new tokens, attention over the pages).

A case is a plain dict.  `listed()` names the standing ones, `draw(rng)` makes one more of the
same ranges, `prepare` makes what a program holds before the call, `run` is one pass: with
`own` through the library's entry points, else in elementary torch operations in fp32, rounded
once at the end.  `work` is what a pass cannot do without, `exact` its outputs in fp64.

Five operators:
  attention  o and the rows' log-sum-exp of packed sequences (shared key/value heads, causal
             and sliding-window masks, operands as views of one fused projection or apart)
  backward   dq, dk, dv from the saved output and log-sum-exp
  paged      a chunk of new tokens of every request over its cached pages (1 token: decode)
  slots      block tables and the slot of every new token, from the requests' lengths
  append     new keys and values written to their slots
"""

import math
import random

import torch

own = False

SIGMA = 3.0  # scaled scores are drawn from about N(0, 9), as in workloads.py


# ------------------------------------------------------------------------------------ cases
def _sequences(name, op, batch, lo, hi, heads_q, heads_kv, dim, causal, window=0, extra=0,
               fused=False, schedule="balanced", geometry=1):
    """`batch` sequences of lo..hi queries (log-uniform); each has up to `extra` more keys than
    queries (a prefix that was computed before).  fused: q, k, v are views of one tensor."""
    return {"name": name, "op": op, "batch": batch, "lo": lo, "hi": hi, "heads_q": heads_q,
            "heads_kv": heads_kv, "dim": dim, "causal": causal, "window": window,
            "extra": extra, "fused": fused, "schedule": schedule, "geometry": geometry}


def _requests(name, op, batch, new_lo, new_hi, kv_lo, kv_hi, heads_q, heads_kv, dim, page,
              window=0, decodes=0.0, short=False, geometry=1):
    """`batch` requests with kv_lo..kv_hi cached tokens and new_lo..new_hi new ones (both
    log-uniform); a share `decodes` of them has one new token.  short: the free list holds too
    few pages for all of them."""
    return {"name": name, "op": op, "batch": batch, "new_lo": new_lo, "new_hi": new_hi,
            "kv_lo": kv_lo, "kv_hi": kv_hi, "heads_q": heads_q, "heads_kv": heads_kv,
            "dim": dim, "page": page, "window": window, "decodes": decodes, "short": short,
            "geometry": geometry}


def listed():
    return [
        # the smallest call: a few short sequences, where the launch counts
        _sequences("attention_small", "attention", 2, 64, 64, 8, 8, 64, False),
        # an unpadded encoder batch: 32 sequences of any length up to 512, 12 heads
        _sequences("attention_varlen_bert", "attention", 32, 16, 512, 12, 12, 64, False,
                   fused=True),
        # a decoder's training or prompt batch at head dimension 128, 4 query heads per kv head
        _sequences("attention_causal_long", "attention", 4, 4096, 4096, 32, 8, 128, True),
        # gradient of the headline workload's layer: 384 slices of 512 x 512
        _sequences("backward_bert", "backward", 32, 512, 512, 12, 12, 64, False),
        # gradient of a decoder's packed batch: lengths that are no multiple of anything
        _sequences("backward_causal_ragged", "backward", 6, 700, 4001, 32, 8, 128, True,
                   fused=True),
        # decode: one token per request over caches of 1k to 32k tokens
        _requests("paged_decode", "paged", 64, 1, 1, 1024, 32768, 32, 8, 128, 16),
        # chunked prompts: 512 new tokens of each request behind what is cached
        _requests("paged_chunk", "paged", 8, 512, 512, 1000, 8000, 32, 8, 128, 64),
        # the smallest decode step, where the launch counts
        _requests("paged_small", "paged", 4, 1, 1, 100, 1000, 16, 2, 64, 16),
        # a decode step's slots
        _requests("slots_decode", "slots", 256, 1, 1, 100, 8000, 1, 1, 8, 16),
        # slots of a batch of new prompts
        _requests("slots_prompts", "slots", 64, 100, 4096, 1, 2000, 1, 1, 8, 16),
        # a decode step's keys and values
        _requests("append_decode", "append", 256, 1, 1, 100, 2000, 8, 8, 128, 16),
        # a prompt batch's keys and values
        _requests("append_prompts", "append", 16, 512, 2048, 1, 2000, 8, 8, 128, 64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    case = _draw(rng)
    del case["name"]
    return case


def _draw(rng):
    op = rng.choice(["attention", "attention", "backward", "backward", "paged", "paged", "slots",
                     "append"])
    geometry = rng.randrange(1, 1 << 30)
    dim = rng.choice([32, 64, 64, 80, 96, 128, 128])
    heads_kv = rng.choice([1, 2, 4, 8])
    heads_q = heads_kv * rng.choice([1, 1, 2, 3, 4, 8])
    if op in ("attention", "backward"):
        hi = _log_int(rng, 32, 4200)
        lo = max(1, _log_int(rng, 8, hi))
        # at most the work of the largest listed case
        batch = _log_int(rng, 1, max(1, min(64, 80_000_000 // (hi * (hi + 64)))))
        most = 5.0e11 / (dim * (4 if op == "attention" else 10))
        while batch * heads_q * hi * (hi + 300) > min(most, 1.0e9) and batch > 1:
            batch = (batch + 1) // 2
        if batch * heads_q * hi * (hi + 300) > min(most, 1.0e9):
            heads_q = heads_kv
        causal = rng.random() < 0.6
        window = _log_int(rng, 16, 2048) if causal and rng.random() < 0.3 else 0
        extra = _log_int(rng, 1, 300) if rng.random() < 0.3 else 0
        return _sequences("", op, batch, lo, hi, heads_q, heads_kv, dim, causal, window, extra,
                          rng.random() < 0.5, rng.choice(["balanced", "balanced", "xcd", "rr"]),
                          geometry)
    page = rng.choice([8, 16, 16, 32, 64, 128, 1, 24])
    if op == "paged":
        kv_hi = _log_int(rng, 64, 32768)
        kv_lo = max(1, kv_hi // rng.choice([1, 4, 32]))
        new_hi = rng.choice([1, 1, 2, 5, _log_int(rng, 8, 1024)])
        batch = _log_int(rng, 1, max(1, min(128, 300_000 // kv_hi)))
        while batch * new_hi * (kv_hi + new_hi) * heads_q > 1.0e9:
            new_hi = max(1, new_hi // 2)
        window = _log_int(rng, 64, 4096) if rng.random() < 0.25 else 0
        return _requests("", op, batch, 1 if rng.random() < 0.5 else new_hi, new_hi, kv_lo,
                         kv_hi, heads_q, heads_kv, dim, page, window,
                         rng.choice([0.0, 0.5]), False, geometry)
    batch = _log_int(rng, 1, 1024)
    new_hi = 1 if rng.random() < 0.5 else max(1, min(4096, _log_int(rng, 2, 100_000) // batch))
    return _requests("", op, batch, 1, new_hi, 1, _log_int(rng, 16, 4000 if op == "slots" else
                                                           1 + 250_000 // batch),
                     heads_q, heads_kv, dim if op == "append" else 8, page, 0, 0.0,
                     op == "slots" and rng.random() < 0.25, geometry)


# --------------------------------------------------------------------------------- geometry
def _sequence_lengths(case):
    rng = random.Random(case["geometry"])
    q = [_log_int(rng, case["lo"], case["hi"]) for _ in range(case["batch"])]
    kv = [n + (rng.randint(0, case["extra"]) if case["extra"] else 0) for n in q]
    return q, kv


def _request_lengths(case):
    rng = random.Random(case["geometry"])
    cached = [_log_int(rng, case["kv_lo"], case["kv_hi"]) for _ in range(case["batch"])]
    new = [1 if rng.random() < case["decodes"] else _log_int(rng, case["new_lo"], case["new_hi"])
           for _ in range(case["batch"])]
    return cached, new


def _visible(n, m, causal, window):
    """Query/key pairs that the mask leaves, for n queries at the end of m >= n keys."""
    if not causal:
        return n * m
    first, last = m - n + 1, m  # keys up to the first and the last query
    if window == 0 or window >= last:
        return n * (first + last) // 2
    if window <= first:
        return n * window
    return (window - first) * (first + window - 1) // 2 + (last - window + 1) * window


def work(case):
    hq, hk, d = case["heads_q"], case["heads_kv"], case["dim"]
    if case["op"] in ("attention", "backward"):
        q, kv = _sequence_lengths(case)
        tq, tk = sum(q), sum(kv)
        pairs = sum(_visible(a, b, case["causal"], case["window"]) for a, b in zip(q, kv))
        if case["op"] == "attention":
            return {"bytes": 2 * d * (2 * tq * hq + 2 * tk * hk) + 4 * tq * hq,
                    "flops": 4 * d * hq * pairs}
        return {"bytes": 2 * d * (4 * tq * hq + 4 * tk * hk) + 4 * tq * hq,
                "flops": 10 * d * hq * pairs}
    cached, new = _request_lengths(case)
    t = sum(new)
    pages = [-(-(c + n) // case["page"]) for c, n in zip(cached, new)]
    if case["op"] == "paged":
        w = case["window"]
        read = sum(min(c + n, w + n - 1) if w else c + n for c, n in zip(cached, new))
        pairs = sum(_visible(n, c + n, True, w) for c, n in zip(cached, new))
        return {"bytes": 4 * d * (t * hq + read * hk) + 4 * sum(pages), "flops": 4 * d * hq * pairs}
    if case["op"] == "slots":
        fresh = sum(p - -(-c // case["page"]) for p, c in zip(pages, cached))
        return {"bytes": 16 * case["batch"] + 8 * t + 8 * fresh, "flops": 0}
    return {"bytes": 8 * t * hk * d + 8 * t, "flops": 0}


# ---------------------------------------------------------------------------------- prepare
def _normal(gen, shape, sigma=1.0):
    x = torch.randn(shape, generator=gen, device="cuda")
    return (x * sigma if sigma != 1.0 else x).to(torch.bfloat16)


def _starts(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["op"] in ("attention", "backward"):
        return _prepare_sequences(case, gen)
    return _prepare_requests(case, gen, seed)


def _prepare_sequences(case, gen):
    q_len, kv_len = _sequence_lengths(case)
    hq, hk, d = case["heads_q"], case["heads_kv"], case["dim"]
    tq, tk = sum(q_len), sum(kv_len)
    if case["fused"] and tq == tk:
        # the fused projection's output: q, k and v heads of a token side by side
        qkv = torch.randn((tq, hq + 2 * hk, d), generator=gen, device="cuda")
        qkv[:, :hq] *= SIGMA
        qkv = qkv.to(torch.bfloat16)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    else:
        q = _normal(gen, (tq, hq, d), SIGMA)
        k, v = _normal(gen, (tk, hk, d)), _normal(gen, (tk, hk, d))
    s = {"case": case, "q_len": q_len, "kv_len": kv_len, "q": q, "k": k, "v": v,
         "scale": 1.0 / math.sqrt(d), "o": torch.empty((tq, hq, d), dtype=q.dtype, device="cuda"),
         "lse": torch.empty((hq, tq), dtype=torch.float32, device="cuda")}
    if case["op"] == "backward":
        # what the forward pass left behind, and the gradient that comes in
        s["o"], s["lse"] = _plain_attention(s)
        s["do"] = _normal(gen, (tq, hq, d))
        s["dq"] = torch.empty((tq, hq, d), dtype=q.dtype, device="cuda")
        s["dk"] = torch.empty((tk, hk, d), dtype=q.dtype, device="cuda")
        s["dv"] = torch.empty((tk, hk, d), dtype=q.dtype, device="cuda")
    if own:
        import paper_2002_07062_amd as bsm

        s["plan"] = bsm.bsm_attention_plan_create(
            q_len, kv_len, heads_q=hq, heads_kv=hk, head_dim=d, causal=case["causal"],
            window=case["window"], schedule=case["schedule"], device=0)
    return s


def _prepare_requests(case, gen, seed):
    rng = random.Random(seed)
    cached, new = _request_lengths(case)
    page, hq, hk, d = case["page"], case["heads_q"], case["heads_kv"], case["dim"]
    held = [-(-c // page) for c in cached]                        # pages before the step
    full = [-(-(c + n) // page) for c, n in zip(cached, new)]     # pages after it
    n_pages = sum(full) + 8
    width = max(full) + 2
    order = list(range(n_pages))
    rng.shuffle(order)  # pages come back to the free list in no order
    order_t = torch.tensor(order, dtype=torch.int32, device="cuda")
    before = case["op"] == "slots"
    counts = torch.tensor(held if before else full, device="cuda")
    at = torch.cumsum(counts, 0) - counts
    column = torch.arange(width, device="cuda")
    index = (at[:, None] + column).clamp(max=n_pages - 1)
    table = torch.where(column < counts[:, None], order_t[index], -1).to(torch.int32)
    s = {"case": case, "cached": torch.tensor(cached, dtype=torch.int32, device="cuda"),
         "new": torch.tensor(new, dtype=torch.int32, device="cuda"), "table": table,
         "tokens": sum(new), "n_pages": n_pages}
    if case["op"] == "slots":
        taken = sum(held)
        free = order_t[taken:].contiguous()
        if case["short"]:
            free = free[: max(1, (sum(full) - taken) // 2)].contiguous()
        s["free"] = free
        s["n_free"] = torch.tensor([free.numel()], dtype=torch.int32, device="cuda")
        s["q_start"] = torch.empty(len(new) + 1, dtype=torch.int32, device="cuda")
        s["kv_len"] = torch.empty(len(new), dtype=torch.int32, device="cuda")
        s["slots"] = torch.empty(sum(new), dtype=torch.int64, device="cuda")
        s["taken"] = torch.empty(2, dtype=torch.int32, device="cuda")
        return s
    s["k_cache"] = _normal(gen, (n_pages, page, hk, d))
    s["v_cache"] = _normal(gen, (n_pages, page, hk, d))
    if case["op"] == "append":
        s["k"], s["v"] = _normal(gen, (sum(new), hk, d)), _normal(gen, (sum(new), hk, d))
        s["slots"] = _plain_token_slots(s)
        return s
    s["q"] = _normal(gen, (sum(new), hq, d), SIGMA)
    s["o"] = torch.empty_like(s["q"])
    s["scale"] = 1.0 / math.sqrt(d)
    s["q_start"] = torch.tensor(_starts(new), dtype=torch.int32, device="cuda")
    s["kv_len"] = s["cached"] + s["new"]
    # what a serving loop knows on the host: bounds on the chunk and on the cached length
    s["max_q"], s["max_kv"] = max(new), max(c + n for c, n in zip(cached, new))
    if own:
        import paper_2002_07062_amd as bsm

        s["workspace"] = torch.empty(
            bsm.bsm_attention_paged_workspace(len(new), sum(new), hq, hk, d, s["max_q"],
                                              s["max_kv"], device=0),
            dtype=torch.uint8, device="cuda")
    return s


# -------------------------------------------------------------------------------------- run
def run(s):
    op = s["case"]["op"]
    if own:
        return _OWN[op](s)
    return _PLAIN[op](s)


def _own_attention(s):
    import paper_2002_07062_amd as bsm

    bsm.bsm_attention_execute(s["plan"], s["q"], s["k"], s["v"], s["o"], lse=s["lse"],
                              scale=s["scale"])
    return {"o": s["o"], "lse": s["lse"]}


def _own_backward(s):
    import paper_2002_07062_amd as bsm

    bsm.bsm_attention_backward(s["plan"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["do"],
                               s["dq"], s["dk"], s["dv"], scale=s["scale"])
    return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}


def _own_paged(s):
    import paper_2002_07062_amd as bsm

    bsm.bsm_attention_paged(s["q"], s["k_cache"], s["v_cache"], s["table"], s["q_start"],
                            s["kv_len"], s["o"], max_q=s["max_q"], max_kv=s["max_kv"],
                            window=s["case"]["window"], scale=s["scale"],
                            workspace=s["workspace"])
    return {"o": s["o"]}


def _own_slots(s):
    import paper_2002_07062_amd as bsm

    bsm.bsm_cache_slots(s["cached"], s["new"], s["case"]["page"], s["n_pages"], s["table"],
                        s["free"], s["n_free"], s["q_start"], s["kv_len"], s["slots"],
                        s["taken"])
    return {"q_start": s["q_start"], "kv_len": s["kv_len"], "table": s["table"],
            "slots": s["slots"], "taken": s["taken"]}


def _own_append(s):
    import paper_2002_07062_amd as bsm

    bsm.bsm_cache_append(s["k"], s["v"], s["slots"], s["k_cache"], s["v_cache"])
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}


_OWN = {"attention": _own_attention, "backward": _own_backward, "paged": _own_paged,
        "slots": _own_slots, "append": _own_append}


# ------------------------------------------------------------------------------- plain forms
def _padded(lengths):
    """Token index of every (sequence, place), the places that hold a token, and (sequence,
    place) of every token, for sequences packed one after the other."""
    n = torch.tensor(lengths, device="cuda")
    at = torch.cumsum(n, 0) - n
    place = torch.arange(max(lengths), device="cuda")
    live = place < n[:, None]
    index = (at[:, None] + place).clamp(max=sum(lengths) - 1)
    return n, index, live


def _heads(x, index):
    """(tokens, heads, dim) -> fp32 (sequences, heads, places, dim), padded."""
    return x[index].float().transpose(1, 2).contiguous()


def _mask(q_n, kv_n, q_places, kv_places, causal, window):
    """(sequences, q places, kv places): which keys a query sees."""
    j = torch.arange(kv_places, device="cuda")
    position = torch.arange(q_places, device="cuda") + (kv_n - q_n)[:, None]
    seen = (j < kv_n[:, None])[:, None, :].expand(-1, q_places, -1)
    if causal:
        seen = seen & (j <= position[:, :, None])
    if window:
        seen = seen & (j > position[:, :, None] - window)
    return seen


def _plain_scores(s):
    """fp32 scores (sequences, kv heads, group, q places, kv places), -inf where masked, with
    the padded operands and the index of the tokens."""
    case = s["case"]
    q_n, q_index, q_live = _padded(s["q_len"])
    kv_n, kv_index, kv_live = _padded(s["kv_len"])
    b, hq, hk = len(s["q_len"]), case["heads_q"], case["heads_kv"]
    q, k, v = _heads(s["q"], q_index), _heads(s["k"], kv_index), _heads(s["v"], kv_index)
    sq, sk, d = q.shape[2], k.shape[2], q.shape[3]
    q = q.view(b, hk, hq // hk * sq, d)
    scores = (torch.matmul(q, k.transpose(2, 3)) * s["scale"]).view(b, hk, hq // hk, sq, sk)
    seen = _mask(q_n, kv_n, sq, sk, case["causal"], case["window"])
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    return scores, q, k, v, q_index, q_live, kv_index, kv_live


def _plain_attention(s):
    scores, q, k, v, _, q_live, _, _ = _plain_scores(s)
    b, hk, g, sq, sk = scores.shape
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(torch.isinf(top), 0.0, top))
    total = p.sum(-1, keepdim=True)
    lse = (torch.log(total) + top).view(b, hk * g, sq)
    o = torch.matmul(p.view(b, hk, g * sq, sk), v).view(b, hk, g, sq, -1)
    o = torch.where(total > 0, o / total, 0.0).view(b, hk * g, sq, -1).transpose(1, 2)
    return o[q_live].to(s["q"].dtype), lse.transpose(1, 2)[q_live].t().contiguous()


def _plain_backward(s):
    scores, q, k, v, q_index, q_live, _, kv_live = _plain_scores(s)
    b, hk, g, sq, sk = scores.shape
    d = q.shape[3]
    do = _heads(s["do"], q_index).view(b, hk, g * sq, d)
    do = do * q_live[:, None, None, :].expand(-1, hk, g, -1).reshape(b, hk, g * sq, 1)
    o = _heads(s["o"], q_index).view(b, hk, g * sq, d)
    lse = s["lse"].t()[q_index].transpose(1, 2).reshape(b, hk, g, sq, 1)
    p = torch.exp(scores - torch.where(torch.isinf(lse), 0.0, lse)).view(b, hk, g * sq, sk)
    p = p * q_live[:, None, None, :].expand(-1, hk, g, -1).reshape(b, hk, g * sq, 1)
    dv = torch.matmul(p.transpose(2, 3), do)
    ds = p * (torch.matmul(do, v.transpose(2, 3)) - (do * o).sum(-1, keepdim=True))
    dq = (torch.matmul(ds, k) * s["scale"]).view(b, hk * g, sq, d).transpose(1, 2)
    dk = (torch.matmul(ds.transpose(2, 3), q) * s["scale"]).transpose(1, 2)
    t = s["q"].dtype
    return {"dq": dq[q_live].to(t), "dk": dk[kv_live].to(t),
            "dv": dv.transpose(1, 2)[kv_live].to(t)}


def _plain_forward(s):
    o, lse = _plain_attention(s)
    return {"o": o, "lse": lse}


def _plain_paged(s):
    case = s["case"]
    page, hq, hk = case["page"], case["heads_q"], case["heads_kv"]
    kv_n, start = s["kv_len"].long(), s["q_start"].long()
    q_n, b = start[1:] - start[:-1], s["kv_len"].numel()
    j = torch.arange(s["max_kv"], device="cuda")
    row = s["table"].long().clamp(min=0)[:, j // page] * page + j % page
    k = s["k_cache"].view(-1, hk, case["dim"])[row].float().transpose(1, 2).contiguous()
    v = s["v_cache"].view(-1, hk, case["dim"])[row].float().transpose(1, 2).contiguous()
    i = torch.arange(s["max_q"], device="cuda")
    q_live = i < q_n[:, None]
    q_index = (start[:-1, None] + i).clamp(max=s["tokens"] - 1)
    q = _heads(s["q"], q_index).view(b, hk, hq // hk * s["max_q"], case["dim"])
    scores = torch.matmul(q, k.transpose(2, 3)) * s["scale"]
    seen = _mask(q_n, kv_n, s["max_q"], s["max_kv"], True, case["window"])
    scores = scores.view(b, hk, hq // hk, s["max_q"], -1)
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(torch.isinf(top), 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(b, hk, -1, s["max_kv"]), v).view(b, hk, hq // hk, s["max_q"], -1)
    o = torch.where(total > 0, o / total, 0.0).view(b, hq, s["max_q"], -1).transpose(1, 2)
    return {"o": o[q_live].to(s["q"].dtype)}


def _plain_token_slots(s):
    """The slot of every new token of requests whose table holds all their pages."""
    new, page = s["new"].long(), s["case"]["page"]
    end = torch.cumsum(new, 0)
    t = torch.arange(s["tokens"], device="cuda")
    b = torch.searchsorted(end, t, right=True)
    place = s["cached"].long()[b] + t - (end - new)[b]
    return s["table"].long()[b, place // page] * page + place % page


def _plain_slots(s):
    page, table = s["case"]["page"], s["table"]
    cached, new = s["cached"].long(), s["new"].long()
    held, full = (cached + page - 1) // page, (cached + new + page - 1) // page
    fits = full <= table.shape[1]
    need = torch.where(fits, full - held, 0)
    end = torch.cumsum(need, 0)
    granted = fits & ((end <= s["n_free"]) | (need == 0))
    column = torch.arange(table.shape[1], device="cuda")
    fresh = (column >= held[:, None]) & (column < full[:, None]) & granted[:, None]
    rank = ((end - need)[:, None] + column - held[:, None]).clamp(0, s["free"].numel() - 1)
    table.copy_(torch.where(fresh, s["free"][rank], table))
    stop = torch.cumsum(new, 0)
    t = torch.arange(s["tokens"], device="cuda")
    b = torch.searchsorted(stop, t, right=True).clamp(max=new.numel() - 1)
    place = cached[b] + t - (stop - new)[b]
    slot = table[b, (place // page).clamp(max=table.shape[1] - 1)].long() * page + place % page
    taken = torch.where(granted & (need > 0), end, 0).amax()
    return {"q_start": torch.nn.functional.pad(stop, (1, 0)).int(),
            "kv_len": torch.where(granted, cached + new, 0).int(), "table": table,
            "slots": torch.where(granted[b], slot, -1),
            "taken": torch.stack([taken, (~granted).sum()]).int()}


def _plain_append(s):
    hk, d = s["case"]["heads_kv"], s["case"]["dim"]
    s["k_cache"].view(-1, hk, d)[s["slots"]] = s["k"]
    s["v_cache"].view(-1, hk, d)[s["slots"]] = s["v"]
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}


_PLAIN = {"attention": _plain_forward, "backward": _plain_backward, "paged": _plain_paged,
          "slots": _plain_slots, "append": _plain_append}


# ------------------------------------------------------------------------------------ exact
def _exact_probabilities(q, k, scale, causal, window, lse=None):
    """fp64 of one head: probabilities (n, m) and log-sum-exp (n) of n queries at the end of m
    keys; with `lse` the probabilities that belong to it."""
    n, m = q.shape[0], k.shape[0]
    x = (q @ k.t()) * scale
    if causal:
        p = torch.arange(m - n, m, device=q.device)[:, None]
        j = torch.arange(m, device=q.device)[None, :]
        hidden = j > p
        if window:
            hidden = hidden | (j <= p - window)
        x = x.masked_fill(hidden, -math.inf)
    if lse is None:
        lse = torch.logsumexp(x, 1)
    return torch.exp(x - lse[:, None]), lse


def exact(case, seed):
    global own
    if case["op"] == "slots":
        return None  # whole numbers
    mine, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = mine
    if case["op"] == "append":
        out = {}
        for x in ("k", "v"):
            cache = s[x + "_cache"].double()
            page, place = s["slots"] // case["page"], s["slots"] % case["page"]
            out[x + "_cache"] = cache.index_put((page, place), s[x].double())
        return out
    hq, hk, scale = case["heads_q"], case["heads_kv"], s["scale"]
    g = hq // hk
    if case["op"] == "paged":
        o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        at = s["q_start"].tolist()
        for b, m in enumerate(s["kv_len"].tolist()):
            pages = s["table"][b, : -(-m // case["page"])].long()
            keys = s["k_cache"][pages].flatten(0, 1)[:m].double()
            values = s["v_cache"][pages].flatten(0, 1)[:m].double()
            for h in range(hq):
                q = s["q"][at[b]:at[b + 1], h].double()
                p, _ = _exact_probabilities(q, keys[:, h // g], scale, True, case["window"])
                o[at[b]:at[b + 1], h] = p @ values[:, h // g]
        return {"o": o}
    aq, ak = _starts(s["q_len"]), _starts(s["kv_len"])
    names = ("o",) if case["op"] == "attention" else ("dq", "dk", "dv")
    like = {"o": "q", "dq": "q", "dk": "k", "dv": "v"}
    out = {x: torch.zeros(s[like[x]].shape, dtype=torch.float64, device="cuda") for x in names}
    if case["op"] == "attention":
        out["lse"] = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    for b in range(case["batch"]):
        i, j = slice(aq[b], aq[b + 1]), slice(ak[b], ak[b + 1])
        for h in range(hq):
            q, k, v = s["q"][i, h].double(), s["k"][j, h // g].double(), s["v"][j, h // g].double()
            if case["op"] == "attention":
                p, lse = _exact_probabilities(q, k, scale, case["causal"], case["window"])
                out["o"][i, h], out["lse"][h, i] = p @ v, lse
                continue
            p, _ = _exact_probabilities(q, k, scale, case["causal"], case["window"],
                                        s["lse"][h, i].double())
            do, o = s["do"][i, h].double(), s["o"][i, h].double()
            ds = p * (do @ v.t() - (do * o).sum(1, keepdim=True))
            out["dq"][i, h] = ds @ k * scale
            out["dk"][j, h // g] += ds.t() @ q * scale
            out["dv"][j, h // g] += p.t() @ do
    return out
