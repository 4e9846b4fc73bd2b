"""What the speed of the operators for language models is judged on: attention with a sliding window and sinks, its gradient,
attention of new tokens over a paged cache, and the call that writes new tokens into that cache.

A case is one call.  With `own` false it is computed by elementary torch operations in 32 bits, with `own` true by the
package's tensor-level entry points.

Everywhere query i of N stands at position i + M - N of M, and key j is visible to position p when j <= p and either
p - j < window (0: no window) or j < sinks.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"


# ------------------------------------------------------------------------------------------------ cases
def _window(op, batch, heads, kv_heads, N, M, d, window, sinks):
    return {"op": op, "batch": batch, "heads": heads, "kv_heads": kv_heads, "N": N, "M": M, "d": d, "window": window, "sinks": sinks}


def _paged(op, seqs, new_lo, new_hi, long_chunks, ctx_lo, ctx_hi, heads, kv_heads, d, page, window, sinks):
    """`seqs` sequences with new_lo .. new_hi new tokens each (the first `long_chunks` of them have new_hi) behind ctx_lo ..
    ctx_hi older ones."""
    return {"op": op, "seqs": seqs, "new_lo": new_lo, "new_hi": new_hi, "long_chunks": long_chunks, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi,
            "heads": heads, "kv_heads": kv_heads, "d": d, "page": page, "window": window, "sinks": sinks}


def listed():
    table = {
        # the smallest call: one short sequence, all latency
        "window_small": _window("window", 1, 4, 4, 64, 64, 64, 32, 4),
        # sizes that come from data: a second part of a sequence, nothing a multiple of anything
        "window_odd": _window("window", 3, 12, 4, 1777, 2500, 64, 333, 17),
        # a long sequence through a layer with a window, four query heads to a key head
        "window_8192": _window("window", 1, 32, 8, 8192, 8192, 128, 1024, 4),
        # training steps: odd sizes, a layer with a window, and plain causal attention with a key head for each query head
        "grad_odd": _window("grad", 3, 12, 4, 1777, 1777, 64, 333, 17),
        "grad_window_4096": _window("grad", 2, 32, 8, 4096, 4096, 128, 1024, 4),
        "grad_causal_4096": _window("grad", 4, 16, 16, 4096, 4096, 128, 0, 0),
        # serving: one user's next token after a short text, all latency
        "paged_one": _paged("paged", 1, 1, 1, 0, 130, 130, 8, 2, 64, 16, 0, 0),
        # the next token of 64 users, texts of 1000 to 8000 tokens
        "paged_decode_64": _paged("paged", 64, 1, 1, 0, 1000, 8000, 32, 8, 128, 16, 0, 0),
        # a batch in which one user's text is read in (a chunk of 1024 tokens) while seven others get their next token
        "paged_mixed": _paged("paged", 8, 1, 1024, 1, 2000, 7000, 32, 8, 128, 16, 0, 0),
        # chunks of ragged lengths through a layer with a window and sinks
        "paged_window": _paged("paged", 24, 1, 300, 0, 0, 5000, 16, 4, 128, 64, 1024, 4),
        # the cache's side of a decoding step and of reading texts in
        "append_decode_64": _paged("append", 64, 1, 1, 0, 1000, 8000, 32, 8, 128, 16, 0, 0),
        "append_chunks": _paged("append", 24, 1, 2000, 4, 0, 3000, 32, 8, 128, 16, 0, 0),
    }
    return [dict(case, name=name) for name, case in table.items()]


MOST_FLOPS = 6.8e11                   # of a drawn case: about those of grad_causal_4096


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["window", "window", "grad", "grad", "decode", "decode", "chunks", "chunks", "append"])
    d = rng.choice([64, 128])
    while True:
        kv_heads = rng.choice([1, 2, 4, 8, 16])
        heads = kv_heads * rng.choice([1, 1, 2, 3, 4, 8])
        window = rng.choice([0, 0, _log_int(rng, 16, 4096)])
        sinks = rng.choice([0, 0, 1, 4, rng.randint(1, 200)]) if window else 0
        if kind in ("window", "grad"):
            M = _log_int(rng, 1 if kind == "window" else 16, 8192)
            N = M if rng.random() < 0.6 else max(1, min(M, _log_int(rng, 1, M)))
            batch = rng.choice([1, 1, 2, 3, 4])
            if heads > 64 or 4.0 * batch * heads * N * M > 8.6e9:      # the plain form holds all scores
                continue
            case = _window(kind, batch, heads, kv_heads, N, M, d, window, sinks)
            if work(case)["flops"] <= MOST_FLOPS:
                return case
            continue
        page = rng.choice([16, 16, 32, 64, 128])
        if heads > 64:
            continue
        if kind == "append":
            seqs = _log_int(rng, 1, 64)
            hi = _log_int(rng, 1, 2000)
            return _paged("append", seqs, 1, hi, 0, 0, _log_int(rng, 1, 4000), heads, kv_heads, d, page, window, sinks)
        ctx = _log_int(rng, 16, 16384)
        seqs = _log_int(rng, 1, 64)
        hi = 1 if kind == "decode" else _log_int(rng, 2, 1024)
        # scores of the plain form, and its copies of keys and values
        if 4.0 * seqs * heads * hi * (ctx + hi) > 8.6e9 or 8.0 * seqs * (ctx + hi) * kv_heads * d > 2.9e9:
            continue
        case = _paged("paged", seqs, 1, hi, 0, ctx // 4, ctx, heads, kv_heads, d, page, window, sinks)
        if work(case)["flops"] <= MOST_FLOPS:
            return case


# ------------------------------------------------------------------------------------------------ inputs
def _lengths(case):
    """New tokens and older ones of every sequence; the same for every seed, so that work() counts what run() does."""
    import random
    rng = random.Random(case["seqs"] * 7919 + case["ctx_hi"])
    new, old = [], []
    for b in range(case["seqs"]):
        new.append(case["new_hi"] if b < case["long_chunks"] else
                   1 if case["long_chunks"] else rng.randint(case["new_lo"], case["new_hi"]))
        old.append(rng.randint(case["ctx_lo"], case["ctx_hi"]))
    return new, old


def _normal(shape, gen):
    return torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.0, generator=gen)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    d, heads, kv = case["d"], case["heads"], case["kv_heads"]
    if case["op"] in ("window", "grad"):
        b, N, M = case["batch"], case["N"], case["M"]
        state = {"case": case, "Q": _normal((b, heads, N, d), gen), "K": _normal((b, kv, M, d), gen), "V": _normal((b, kv, M, d), gen)}
        if case["op"] == "grad":      # what the forward pass left, and the gradient that arrives
            state["O"], state["lse"] = _plain_window(state)
            state["dO"] = _normal((b, heads, N, d), gen)
        return state
    new, old = _lengths(case)
    page, seqs = case["page"], case["seqs"]
    total = [n + o for n, o in zip(new, old)]
    need = [-(-t // page) for t in total]
    pages = sum(need) + 3
    # pages in the order in which a pool hands them out after a while: any
    order = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32).tolist()
    table, at = [], 0
    for n in need:
        table.append(order[at:at + n] + [0] * (max(need) - n))
        at += n
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    whole = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    state = {"case": case, "K_cache": _normal((pages, kv, page, d), gen), "V_cache": _normal((pages, kv, page, d), gen),
             "table": whole(table), "lengths": whole(total), "starts": whole(starts), "max_new": max(new), "longest": max(total)}
    if case["op"] == "append":
        state["K"], state["V"] = _normal((starts[-1], kv, d), gen), _normal((starts[-1], kv, d), gen)
    else:
        state["Q"] = _normal((starts[-1], heads, d), gen)
    return state


# ------------------------------------------------------------------------------------------------ the plain forms
def _visible(p, j, window, sinks):
    seen = j <= p
    return seen & ((p - j < window) | (j < sinks)) if window else seen


def _weights(scores, seen):
    """exp(scores - lse) over the visible keys, and lse; rows that see nothing: zeros and -inf."""
    scores = scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    e = scores.sub_(torch.where(top.isinf(), 0.0, top)).exp_()
    total = e.sum(-1, keepdim=True)
    return e.div_(torch.where(total == 0, 1.0, total)), (top + total.log()).squeeze(-1)


def _grouped(x, kv):
    """(batch, heads, N, d) as (batch, kv, group * N, d)."""
    b, heads, N, d = x.shape
    return x.reshape(b, kv, heads // kv * N, d)


def _seen_rows(case):
    """(N, M): what every query sees."""
    N, M = case["N"], case["M"]
    p = torch.arange(N, device=DEV)[:, None] + (M - N)
    return _visible(p, torch.arange(M, device=DEV)[None, :], case["window"], case["sinks"])


def _plain_window(state):
    case = state["case"]
    b, heads, kv, N, M = case["batch"], case["heads"], case["kv_heads"], case["N"], case["M"]
    K, V = state["K"].float(), state["V"].float()
    S = torch.matmul(_grouped(state["Q"].float() / math.sqrt(case["d"]), kv), K.transpose(-1, -2))
    P, lse = _weights(S.view(b, heads, N, M), _seen_rows(case))
    O = torch.matmul(P.view(b, kv, heads // kv * N, M), V)
    return O.view(b, heads, N, -1).to(torch.bfloat16), lse


def _plain_grad(state):
    case = state["case"]
    b, heads, kv, N, M, d = case["batch"], case["heads"], case["kv_heads"], case["N"], case["M"], case["d"]
    Q, dO = _grouped(state["Q"].float(), kv), _grouped(state["dO"].float(), kv)
    K, V = state["K"].float(), state["V"].float()
    D = (state["dO"].float() * state["O"].float()).sum(-1, keepdim=True)
    P = torch.matmul(Q / math.sqrt(d), K.transpose(-1, -2)).view(b, heads, N, M)
    seen = _seen_rows(case)
    P = P.sub_(torch.where(state["lse"].isinf(), 0.0, state["lse"])[..., None]).masked_fill_(~seen, -math.inf).exp_()
    dV = torch.matmul(P.view(b, kv, -1, M).transpose(-1, -2), dO)
    dS = torch.matmul(dO, V.transpose(-1, -2)).view(b, heads, N, M).sub_(D).mul_(P)
    dS = dS.view(b, kv, -1, M)
    dQ = torch.matmul(dS, K) / math.sqrt(d)
    dK = torch.matmul(dS.transpose(-1, -2), Q) / math.sqrt(d)
    return dQ.view(b, heads, N, d).to(torch.bfloat16), dK.to(torch.bfloat16), dV.to(torch.bfloat16)


def _tokens(state, count):
    """Sequence and index within it of every new token."""
    t = torch.arange(count, device=DEV)
    seq = torch.searchsorted(state["starts"][1:].long(), t, right=True)
    return seq, t - state["starts"].long()[seq]


def _plain_paged(state):
    case = state["case"]
    heads, kv, d, page, seqs = case["heads"], case["kv_heads"], case["d"], case["page"], case["seqs"]
    Q, most, longest = state["Q"], state["max_new"], state["longest"]
    j = torch.arange(longest, device=DEV)
    at = state["table"].long()[:, j // page]                                    # (seqs, longest)
    K = state["K_cache"][at, :, j % page].float().transpose(1, 2)                # (seqs, kv, longest, d)
    V = state["V_cache"][at, :, j % page].float().transpose(1, 2)
    starts, lengths = state["starts"].long(), state["lengths"].long()
    i = torch.arange(most, device=DEV)
    rows = (starts[:-1, None] + i).clamp_(max=Q.shape[0] - 1)
    Qp = (Q[rows].float() / math.sqrt(d)).transpose(1, 2)                        # (seqs, heads, most, d)
    p = (lengths - (starts[1:] - starts[:-1]))[:, None] + i                      # positions
    seen = _visible(p[:, None, :, None], j, case["window"], case["sinks"]) & (j < lengths[:, None, None, None])
    S = torch.matmul(_grouped(Qp, kv), K.transpose(-1, -2)).view(seqs, heads, most, longest)
    P, _ = _weights(S, seen)
    O = torch.matmul(P.view(seqs, kv, -1, longest), V).view(seqs, heads, most, d)
    seq, index = _tokens(state, Q.shape[0])
    return O[seq, :, index].to(torch.bfloat16)


def _plain_append(state):
    page = state["case"]["page"]
    seq, index = _tokens(state, state["K"].shape[0])
    starts = state["starts"].long()
    p = state["lengths"].long()[seq] - (starts[seq + 1] - starts[seq]) + index
    at = state["table"].long()[seq, p // page]
    state["K_cache"][at, :, p % page] = state["K"]
    state["V_cache"][at, :, p % page] = state["V"]
    return state["K_cache"], state["V_cache"]


# ------------------------------------------------------------------------------------------------ the framework's calls
def _own(state):
    import paper_2511_09987_amd as lib
    case = state["case"]
    mask = {"window": case["window"] or None, "sinks": case["sinks"]}
    if case["op"] == "window":
        return lib.recurrence_attention_window(state["Q"], state["K"], state["V"], **mask)
    if case["op"] == "grad":
        return lib.recurrence_attention_window_grad(state["Q"], state["K"], state["V"], state["O"], state["lse"], state["dO"], **mask)
    cache = state["K_cache"], state["V_cache"], state["table"], state["lengths"], state["starts"]
    if case["op"] == "paged":
        return lib.recurrence_attention_paged(state["Q"], *cache, max_new=state["max_new"], **mask)
    lib.cache_append(state["K"], state["V"], *cache)
    return state["K_cache"], state["V_cache"]


def run(state):
    if own:
        return _own(state)
    return {"window": _plain_window, "grad": _plain_grad, "paged": _plain_paged, "append": _plain_append}[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------ work
def _sees(p, window, sinks):
    """How many keys position p sees."""
    if p < 0:
        return 0
    if not window or p < window:
        return p + 1
    return window + min(sinks, p - window + 1)


def work(case):
    d, heads, kv = case["d"], case["heads"], case["kv_heads"]
    if case["op"] in ("window", "grad"):
        b, N, M = case["batch"], case["N"], case["M"]
        pairs = b * heads * sum(_sees(i + M - N, case["window"], case["sinks"]) for i in range(N))
        q, k = b * heads * N * d * 2, b * kv * M * d * 2
        if case["op"] == "window":
            return {"bytes": 2 * q + 2 * k + b * heads * N * 4, "flops": 4 * d * pairs}
        return {"bytes": 4 * q + 4 * k + b * heads * N * 4, "flops": 10 * d * pairs}
    new, old = _lengths(case)
    tokens = sum(new)
    if case["op"] == "append":
        return {"bytes": tokens * kv * d * 2 * 2 * 2, "flops": 0}
    pairs = keys = 0
    for n, o in zip(new, old):
        pairs += heads * sum(_sees(o + i, case["window"], case["sinks"]) for i in range(n))
        keys += _sees(o, case["window"], case["sinks"]) + n - 1 if case["window"] else o + n
    return {"bytes": tokens * heads * d * 2 * 2 + keys * kv * d * 2 * 2, "flops": 4 * d * pairs}


# ------------------------------------------------------------------------------------------------ 64-bit results
def _exact_rows(q, k, v, first, window, sinks):
    """Softmax-weighted sums of v (M, d) for queries q (N, d) at positions first, first + 1, .., and the logarithms of the sums."""
    N, M = q.shape[0], k.shape[0]
    pos = torch.arange(first, first + N, device=DEV).view(N, 1)
    key = torch.arange(M, device=DEV).view(1, M)
    hidden = key > pos
    if window:
        hidden |= (key <= pos - window) & (key >= sinks)
    s = (q @ k.T) * (q.shape[1] ** -0.5)
    s[hidden] = -math.inf
    lse = torch.logsumexp(s, dim=1)
    w = torch.exp(s - torch.where(torch.isneginf(lse), torch.zeros_like(lse), lse)[:, None])
    return w, w @ v, lse


def exact(case, seed):
    state = prepare(case, seed)
    d, G, window, sinks = case["d"], case["heads"] // case["kv_heads"], case["window"], case["sinks"]
    if case["op"] in ("window", "grad"):
        Q, K, V = (state[x].double() for x in ("Q", "K", "V"))
        b, heads, N, M = case["batch"], case["heads"], case["N"], case["M"]
        if case["op"] == "window":
            O, lse = torch.empty_like(Q), torch.empty(Q.shape[:3], dtype=torch.float64, device=DEV)
            for x in range(b):
                for h in range(heads):
                    _, O[x, h], lse[x, h] = _exact_rows(Q[x, h], K[x, h // G], V[x, h // G], M - N, window, sinks)
            return O, lse
        dQ, dK, dV, dO = torch.empty_like(Q), torch.zeros_like(K), torch.zeros_like(V), state["dO"].double()
        for x in range(b):
            for h in range(heads):
                g = h // G
                w, o, _ = _exact_rows(Q[x, h], K[x, g], V[x, g], M - N, window, sinks)
                ds = w * (dO[x, h] @ V[x, g].T - (dO[x, h] * o).sum(1, keepdim=True)) * d ** -0.5
                dQ[x, h] = ds @ K[x, g]
                dK[x, g] += ds.T @ Q[x, h]
                dV[x, g] += w.T @ dO[x, h]
        return dQ, dK, dV
    new, old = _lengths(case)
    page, at = case["page"], 0
    out = torch.empty(state["Q"].shape, dtype=torch.float64, device=DEV) if case["op"] == "paged" else None
    K_cache, V_cache = state["K_cache"].double(), state["V_cache"].double()
    for x, (n, o) in enumerate(zip(new, old)):
        used = state["table"][x, :-(-(n + o) // page)].long()
        if out is None:
            for t in range(n):
                where = used[(o + t) // page]
                K_cache[where, :, (o + t) % page] = state["K"][at + t].double()
                V_cache[where, :, (o + t) % page] = state["V"][at + t].double()
        else:
            for g in range(case["kv_heads"]):
                k, v = (c[used, g].reshape(-1, d)[:n + o] for c in (K_cache, V_cache))
                for h in range(g * G, g * G + G):
                    out[at:at + n, h] = _exact_rows(state["Q"][at:at + n, h].double(), k, v, o, window, sinks)[1]
        at += n
    return (K_cache, V_cache) if out is None else out
