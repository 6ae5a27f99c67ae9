"""Language-model operators of the attention library as its users call them, for timing and comparing.

Five operators: attention with a causal sliding window and a few first tokens
that stay visible (forward, and backward for training), storing new keys and
values in a paged cache, attention of one new token per sequence over that
cache, and shortening the cache to its most attended tokens.  With ``own`` false
``run`` computes them from elementary torch operations in 32 bits, rounded once
at the end; with ``own`` true it makes the library's calls.  ``exact`` evaluates
the definitions in 64 bits.

Fields of a case
  op      "prefill" (window forward with L), "train" (window forward, then
          backward), "append", "decode", "evict"
  dtype   of q, k, v and of the results; cache: "16" (the same type) or "int8"
          (codes and one fp32 scale per token and head, max|x| / 127)
  B, Hq, Hkv, N, D   sequences, query heads, key/value heads, tokens, head dimension.
          N: prefill, train: tokens per row of the batch; append: tokens per call
          and sequence; decode, evict: the longest cached sequence
  ragged  sequences of differing lengths (else all N)
  window  keys a query sees, its own token among them (0: all before it); sinks:
          first tokens that every query sees
  page    tokens per page; budget, first, last (evict): tokens kept, and how many
          of them are the sequence's first and last ones
  weights (decode) attention weights are added up for the eviction
"""
import math

import numpy as np
import torch

own = False

BASE = {"op": "decode", "B": 1, "Hq": 32, "Hkv": 8, "N": 1024, "D": 128, "dtype": "bf16", "cache": "16", "ragged": False,
        "window": 0, "sinks": 0, "page": 64, "weights": False, "budget": 0, "first": 0, "last": 0}


def _case(**kw):
    c = dict(BASE)
    c.update(kw)
    return c


def listed():
    return [
        # the smallest decode call: one short sequence, an odd length, small pages; latency is all there is
        _case(name="decode_b1n77d64_fp16", Hq=8, Hkv=2, N=77, D=64, dtype="fp16", page=16),
        # a serving batch of ordinary lengths under a sliding window with sinks
        _case(name="decode_b32n6000_window", B=32, N=6000, ragged=True, window=4096, sinks=4),
        # one very long sequence: the work has to be split over its length
        _case(name="decode_b1n131072", N=131072, page=128),
        # an 8-bit cache of a larger ragged batch whose weights are added up for the eviction
        _case(name="decode_b48n8000_int8_weights", B=48, Hkv=4, N=8000, cache="int8", ragged=True, page=32, weights=True),
        # prompts stored in the 8-bit cache, right-padded batch
        _case(name="append_b4n4096_int8", op="append", B=4, N=4096, cache="int8", ragged=True, page=32),
        # one new token of every sequence of a batch
        _case(name="append_b128n1", op="append", B=128, N=1),
        # a long prompt with the window that long-context models use
        _case(name="prefill_b1n32768_window", op="prefill", N=32768, window=4096, sinks=4),
        # a padded batch of short odd prompts, one key head per query head
        _case(name="prefill_b4n1237d64_fp16", op="prefill", B=4, Hq=24, Hkv=24, N=1237, D=64, dtype="fp16", ragged=True,
              window=256, sinks=1),
        # one attention layer of a training step with a window and sinks
        _case(name="train_b1n8192_window", op="train", N=8192, window=1024, sinks=16),
        # a small batch trained with plain causal attention, odd length, fp16
        _case(name="train_b2n1000d64_fp16", op="train", B=2, Hq=12, Hkv=4, N=1000, D=64, dtype="fp16"),
        # a batch brought back to its budget; some sequences are still within it
        _case(name="evict_b16n5000", op="evict", B=16, N=5000, ragged=True, budget=2048, first=4, last=256),
        # one long context halved twice
        _case(name="evict_b1n65536", op="evict", N=65536, page=128, budget=16384, first=16, last=4096),
    ]


def draw(rng):
    logu = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    while True:
        op = rng.choice(["decode", "decode", "decode", "prefill", "prefill", "train", "train", "append", "evict"])
        Hkv = rng.choice([1, 2, 4, 8, 8, 12, 16])
        Hq = Hkv * rng.choice([1, 2, 3, 4, 4, 7, 8, 16])
        c = _case(op=op, Hq=Hq, Hkv=Hkv, D=rng.choice([128, 128, 64]), dtype=rng.choice(["bf16", "bf16", "fp16"]),
                  ragged=rng.random() < 0.6, page=rng.choice([16, 16, 32, 64, 128, 256, 24]))
        if Hq > 64:
            continue
        paged = op in ("decode", "append", "evict")
        c["B"] = logu(1, 128 if paged else 8)
        c["N"] = logu(1, {"decode": 131072, "append": 8192, "evict": 65536, "prefill": 32768, "train": 16384}[op])
        if paged:
            c["cache"] = rng.choice(["16", "16", "int8"])
        if op in ("decode", "prefill", "train") and rng.random() < 0.7:
            c["window"] = logu(16, 8192)
            c["sinks"] = rng.choice([0, 0, 1, 4, 16, 100])
        if op == "decode":
            c["weights"] = rng.random() < 0.3
        if op == "evict":
            if c["N"] < 8:
                continue
            c["budget"] = max(4, int(c["N"] * rng.uniform(0.1, 0.9)))
            c["first"] = rng.choice([0, min(4, c["budget"] // 4)])
            c["last"] = int(c["budget"] * rng.uniform(0.0, 0.5))
        w, n = work(c), c["B"] * c["N"] * c["D"] * 2
        if w["bytes"] < 6e8 and n * Hkv < 2 ** 28 and n * Hq < (2 ** 40 if paged else 2 ** 29) and w["flops"] < 2e12 \
                and c["B"] * Hq * c["N"] < 2 ** 26:
            return c


# ---------------------------------------------------------------- sizes
def _lens(case):
    """The sequences' lengths (in an order of the seed's): all N, or spread from an eighth of N to N."""
    B, N = case["B"], case["N"]
    if not case["ragged"]:
        return [N] * B
    return [max(1, N - (N * 7 * i) // (8 * B)) for i in range(B)]


def _pairs(n, case):
    """(query, key) pairs that n tokens of one sequence see, and the keys that the last of them sees."""
    i = np.arange(n, dtype=np.int64)
    w = case["window"] or n
    seen = np.minimum(i + 1, w) + np.minimum(case["sinks"], np.maximum(0, i + 1 - w))
    return float(seen.sum()), int(seen[-1]) if n else 0


def _row_bytes(case):
    """Bytes of one token's key or value in the cache."""
    return case["D"] + 4 if case["cache"] == "int8" else 2 * case["D"]


def work(case):
    B, Hq, Hkv, D, lens = case["B"], case["Hq"], case["Hkv"], case["D"], _lens(case)
    tokens, op = sum(lens), case["op"]
    if op in ("prefill", "train"):
        pairs = sum(_pairs(n, case)[0] for n in lens)
        byts = 2 * D * (2 * Hq + 2 * Hkv) * tokens + 4 * Hq * tokens
        if op == "train":                                # dO, and dQ, dK, dV
            byts += 2 * D * (2 * Hq + 2 * Hkv) * tokens
        return {"bytes": byts, "flops": (14.0 if op == "train" else 4.0) * D * Hq * pairs}
    if op == "append":
        return {"bytes": Hkv * tokens * 2 * (2 * D + _row_bytes(case)), "flops": 2.0 * Hkv * tokens * D}
    if op == "decode":
        seen = sum(_pairs(n, case)[1] for n in lens)
        byts = 2 * Hkv * seen * _row_bytes(case) + B * Hq * (4 * D + 4) + (8 * Hkv * seen if case["weights"] else 0)
        return {"bytes": byts, "flops": 4.0 * D * Hq * seen}
    kept = sum(min(n, case["budget"]) for n in lens)
    return {"bytes": Hkv * (4 * tokens + kept * (4 * _row_bytes(case) + 8)), "flops": float(Hkv * tokens)}


# ---------------------------------------------------------------- inputs
def _quantized(x):
    """Codes and scales of an 8-bit cache: s = max|x| / 127 per token and head, codes round(x * (1 / s)), ties to even."""
    x = x.float()
    s = x.abs().amax(-1)
    s = s / torch.full_like(s, 127)                      # (divided by a number, torch would multiply by its reciprocal)
    r = torch.where(s > 0, 1 / s, torch.zeros_like(s))
    return torch.round(x * r[..., None]).to(torch.int8), s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    B, Hq, Hkv, N, D, page = (case[x] for x in ("B", "Hq", "Hkv", "N", "D", "page"))
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float16
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")
    order = torch.randperm(B, generator=g, device="cuda")
    lens = torch.tensor(_lens(case), dtype=torch.int32, device="cuda")[order].contiguous()
    s = {"case": case, "lens": lens}
    # keys carry a per-channel offset that their tokens share, as keys of trained models do
    if case["op"] in ("prefill", "train"):
        s["q"], s["v"] = rand(B, Hq, N, D).to(dt), rand(B, Hkv, N, D).to(dt)
        s["k"] = (rand(B, Hkv, N, D) + rand(B, Hkv, 1, D)).to(dt)
        if case["op"] == "train":
            s["dout"] = rand(B, Hq, N, D).to(dt)
        return s
    # paged: every sequence has pages for its longest length (append: after 100 tokens that it may hold already);
    # the last page belongs to none
    longest = N + 100 if case["op"] == "append" else N
    M = -(-longest // page)
    M2 = -(-case["budget"] // page) if case["op"] == "evict" else 0
    P = B * (M + M2) + 1
    pages = torch.randperm(P - 1, generator=g, device="cuda").to(torch.int32)
    s["table"] = pages[:B * M].view(B, M).contiguous()
    s["new_table"] = pages[B * M:].view(B, M2).contiguous()
    k, v = (rand(P, Hkv, page, D) for _ in range(2))
    k += rand(1, Hkv, 1, D)
    s["k_scale"] = s["v_scale"] = None
    if case["cache"] == "int8":
        (s["k_cache"], s["k_scale"]), (s["v_cache"], s["v_scale"]) = _quantized(k), _quantized(v)
    else:
        s["k_cache"], s["v_cache"] = k.to(dt), v.to(dt)
    if case["op"] == "append":
        s["k"], s["v"] = (rand(B, Hkv, N, D).to(dt) for _ in range(2))
        s["pos"] = torch.randint(0, 101, (B,), generator=g, device="cuda").to(torch.int32)
    if case["op"] == "decode":
        s["q"] = rand(B, Hq, D).to(dt)
    if case["weights"] or case["op"] == "evict":
        # weights of heavy-tailed size: few tokens draw most of the attention
        s["weights"] = torch.exp(3 * rand(B, Hkv, M * page) - 6)
        # ... and some that no query has attended to, all equal
        s["weights"] *= torch.rand((B, Hkv, M * page), generator=g, device="cuda") < 0.9
    return s


# ---------------------------------------------------------------- the operators in plain form
def _visible(i, j, n, window, sinks):
    """Which keys j the queries i of a sequence of n tokens see."""
    w = (j <= i) & (j < n)
    return w & ((j > i - window) | (j < sinks)) if window else w


def _softmax(x):
    """Weights and log-sum-exp of the last axis; rows of -inf alone have weights 0 and -inf."""
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - m.clamp_min(torch.finfo(x.dtype).min))
    t = e.sum(-1, keepdim=True)
    return e / torch.where(t > 0, t, 1.0), (m + torch.log(t))[..., 0]


BLOCK = 1024   # queries whose scores are held at a time


def _blocks(case, n):
    """Query ranges and the keys that each can see: the sinks' and the window's, as index ranges."""
    w, s = case["window"] or n, case["sinks"]
    for i0 in range(0, n, BLOCK):
        i1 = min(n, i0 + BLOCK)
        lo = max(0, i0 - w + 1)
        yield i0, i1, min(s, lo), lo


def _plain_window(st):
    """Forward of all blocks of queries, in 32 bits; returns what a backward needs too."""
    c = st["case"]
    B, Hq, Hkv, N, D = (c[x] for x in ("B", "Hq", "Hkv", "N", "D"))
    q = st["q"].float().view(B, Hkv, Hq // Hkv, N, D)
    k, v = st["k"].float()[:, :, None], st["v"].float()[:, :, None]
    at = torch.arange(N, device=q.device)
    n = st["lens"].view(B, 1, 1, 1, 1)
    inside = at.view(N, 1) < n                           # rows behind a sequence's end stay zero
    o, lse, parts = torch.empty_like(q), torch.empty_like(q[..., 0]), []
    grads = "dout" in st
    if grads:
        do = torch.where(inside, st["dout"].float().view_as(q), 0.0)
        dq, dk, dv = torch.empty_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for i0, i1, s, lo in _blocks(c, N):
        j = torch.cat([at[:s], at[lo:i1]])
        kj, vj = torch.cat([k[..., :s, :], k[..., lo:i1, :]], -2), torch.cat([v[..., :s, :], v[..., lo:i1, :]], -2)
        see = _visible(at[i0:i1, None], j, n, c["window"], c["sinks"]) & inside[..., i0:i1, :]
        qi = q[..., i0:i1, :]
        p, lse[..., i0:i1] = _softmax(torch.where(see, qi @ kj.transpose(-1, -2) / math.sqrt(D), -math.inf))
        o[..., i0:i1, :] = p @ vj
        if grads:
            g = do[..., i0:i1, :]
            ds = p * (g @ vj.transpose(-1, -2) - (g * o[..., i0:i1, :]).sum(-1, keepdim=True)) / math.sqrt(D)
            dq[..., i0:i1, :] = ds @ kj
            for t, x in ((dk, ds.transpose(-1, -2) @ qi), (dv, p.transpose(-1, -2) @ g)):
                x = x.sum(2, keepdim=True)
                t[..., :s, :] += x[..., :s, :]
                t[..., lo:i1, :] += x[..., s:, :]
    dt = st["q"].dtype
    out = [o.view(B, Hq, N, D).to(dt), lse.view(B, Hq, N)]
    if grads:
        out += [dq.view(B, Hq, N, D).to(dt), dk[:, :, 0].to(dt), dv[:, :, 0].to(dt)]
    return tuple(out)


def _values(cache, scale):
    return cache if scale is None else cache.float() * scale[..., None]


def _caches(st):
    """The cache as the values it stands for, without the page that belongs to no sequence."""
    return _values(st["k_cache"], st["k_scale"])[:-1], _values(st["v_cache"], st["v_scale"])[:-1]


def _plain_append(st):
    c = st["case"]
    N, page, last = c["N"], c["page"], st["k_cache"].shape[0] - 1
    t = torch.arange(N, device="cuda")
    at = st["pos"].long()[:, None] + t
    real = t < st["lens"][:, None]
    to = torch.where(real, st["table"].long().gather(1, (at // page).clamp(max=st["table"].shape[1] - 1)), last)
    for x, cache, scale in ((st["k"], st["k_cache"], st["k_scale"]), (st["v"], st["v_cache"], st["v_scale"])):
        x = x.transpose(1, 2)                            # [B, N, Hkv, D]
        if scale is not None:
            x, sc = _quantized(x)
            scale[to, :, at % page] = sc
        cache[to, :, at % page] = x
    return _caches(st)


def _gathered(cache, scale, table):
    """[B, Hkv, positions, D] in 32 bits."""
    x = cache[table.long()].float()
    if scale is not None:
        x = x * scale[table.long()][..., None]
    B, M, H, page, D = x.shape
    return x.transpose(1, 2).reshape(B, H, M * page, D)


def _plain_decode(st):
    c = st["case"]
    B, Hq, Hkv, D = (c[x] for x in ("B", "Hq", "Hkv", "D"))
    k, v = (_gathered(st[x + "_cache"], st[x + "_scale"], st["table"]) for x in "kv")
    n = st["lens"].view(B, 1, 1, 1)
    see = _visible(n - 1, torch.arange(k.shape[2], device="cuda"), n, c["window"], c["sinks"])
    q = st["q"].float().view(B, Hkv, Hq // Hkv, D)
    p, lse = _softmax(torch.where(see, q @ k.transpose(-1, -2) / math.sqrt(D), -math.inf))
    o = p @ torch.where(see.view(B, 1, -1, 1), v, 0.0)
    out = [o.view(B, Hq, D).to(st["q"].dtype), lse.view(B, Hq)]
    if c["weights"]:
        out.append(st["weights"] + p.sum(2))
    return tuple(out)


def _plain_evict(st):
    c = st["case"]
    B, Hkv, page, budget = (c[x] for x in ("B", "Hkv", "page", "budget"))
    w, last = st["weights"], st["k_cache"].shape[0] - 1
    L = w.shape[-1]
    j, n = torch.arange(L, device="cuda"), st["lens"].long().view(B, 1, 1)
    new = n.clamp(max=budget)
    # the heaviest come first, ties with the lowest index first; the first and last tokens before them
    fixed = (j < c["first"]) | (j >= n - c["last"])
    key = torch.where(j < n, torch.where(fixed, math.inf, w), -math.inf)
    top = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :budget]
    slot = torch.arange(top.shape[-1], device="cuda")
    kept = torch.sort(torch.where(slot < new, top, L), dim=-1).values
    real = slot < new
    src = torch.where(real, kept, 0)
    h = torch.arange(Hkv, device="cuda").view(1, Hkv, 1)
    b = torch.arange(B, device="cuda").view(B, 1, 1)
    sp = st["table"].long()[b, src // page]
    dp = torch.where(real, st["new_table"].long()[b, slot // page], last)
    for x in ("k_cache", "v_cache", "k_scale", "v_scale"):
        if st[x] is not None:
            st[x][dp, h, slot % page] = st[x][sp, h, src % page]
    nw = torch.zeros((B, Hkv, st["new_table"].shape[1] * page), device="cuda")
    nw[..., :len(slot)] = torch.where(real, w.gather(-1, src), 0.0)
    full = torch.full((B, Hkv, budget), -1, dtype=torch.int32, device="cuda")
    full[..., :len(slot)] = torch.where(real, kept, -1)
    return (new.view(B).to(torch.int32), nw, full) + _caches(st)


def run(st):
    c = st["case"]
    if own:
        from paper_2505_11594_amd import binding as bd
        win = dict(window=c["window"] or None, sinks=c["sinks"])
        scales = dict(k_scale=st.get("k_scale"), v_scale=st.get("v_scale"))
        if c["op"] in ("prefill", "train"):
            lens = st["lens"] if c["ragged"] else None
            o, lse = bd.sage_attn_window_fwd(st["q"], st["k"], st["v"], lens=lens, **win)
            if c["op"] == "prefill":
                return o, lse
            return (o, lse) + tuple(bd.sage_attn_window_bwd(st["q"], st["k"], st["v"], o, lse, st["dout"], lens=lens, **win))
        if c["op"] == "append":
            bd.sage_kv_append(st["k"], st["v"], st["k_cache"], st["v_cache"], st["table"], st["pos"],
                              counts=st["lens"] if c["ragged"] else None, **scales)
            return _caches(st)
        if c["op"] == "decode":
            w = st["weights"].clone() if c["weights"] else None
            o, lse = bd.sage_attn_paged_decode(st["q"], st["k_cache"], st["v_cache"], st["table"], st["lens"], weights=w,
                                               **win, **scales)
            return (o, lse, w) if c["weights"] else (o, lse)
        return tuple(bd.sage_kv_evict(st["k_cache"], st["v_cache"], st["table"], st["lens"], st["weights"], st["new_table"],
                                      c["budget"], keep_first=c["first"], keep_last=c["last"], **scales)) + _caches(st)
    if c["op"] in ("prefill", "train"):
        return _plain_window(st)
    return {"append": _plain_append, "decode": _plain_decode, "evict": _plain_evict}[c["op"]](st)


# ---------------------------------------------------------------- the definitions in 64 bits
def _exact_window(st):
    """Dense masked attention, one sequence and head at a time, the gradients by differentiating it."""
    c = st["case"]
    B, Hq, Hkv, N, D = (c[x] for x in ("B", "Hq", "Hkv", "N", "D"))
    grads = c["op"] == "train"
    z = lambda *s: torch.zeros(s, dtype=torch.float64, device="cuda")
    o, lse = z(B, Hq, N, D), z(B, Hq, N) - math.inf
    dq, dk, dv = z(B, Hq, N, D), z(B, Hkv, N, D), z(B, Hkv, N, D)
    for b, n in enumerate(st["lens"].tolist()):
        for h in range(Hq):
            q, k, v = (st[x][b, hh, :n].double().requires_grad_(grads) for x, hh in (("q", h), ("k", h * Hkv // Hq), ("v", h * Hkv // Hq)))
            for r0 in range(0, n, 8192):
                i = torch.arange(r0, min(n, r0 + 8192), device="cuda")[:, None]
                j = torch.arange(int(i[-1]) + 1, device="cuda")
                hidden = j > i
                if c["window"]:
                    hidden = hidden | ((i - j >= c["window"]) & (j >= c["sinks"]))
                x = ((q[r0:r0 + 8192] @ k[:len(j)].T) * D ** -0.5).masked_fill(hidden, -math.inf)
                y = torch.softmax(x, -1) @ v[:len(j)]
                if grads:
                    y.backward(st["dout"][b, h, r0:r0 + 8192][:len(i)].double())
                o[b, h, r0:r0 + len(i)] = y.detach()
                lse[b, h, r0:r0 + len(i)] = torch.logsumexp(x.detach(), -1)
            if grads:
                dq[b, h, :n] = q.grad
                dk[b, h * Hkv // Hq, :n] += k.grad
                dv[b, h * Hkv // Hq, :n] += v.grad
    return (o, lse, dq, dk, dv) if grads else (o, lse)


def _exact_rows(st, x, b, h, n):
    """The first n cached rows of one sequence and head in 64 bits."""
    page = st["case"]["page"]
    ids = st["table"][b, :-(-n // page)].long()
    r = st[x + "_cache"][ids, h].double()
    if st[x + "_scale"] is not None:
        r = r * st[x + "_scale"][ids, h].double()[..., None]
    return r.reshape(-1, r.shape[-1])[:n]


def _exact_decode(st):
    c = st["case"]
    B, Hq, Hkv, D = (c[x] for x in ("B", "Hq", "Hkv", "D"))
    o = torch.zeros((B, Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device="cuda")
    w = st["weights"].double() if c["weights"] else None
    G = Hq // Hkv
    for b, n in enumerate(st["lens"].tolist()):
        near = torch.arange(n, device="cuda") >= (n - c["window"] if c["window"] else 0)
        near[:c["sinks"]] = True
        for h in range(Hkv):
            x = st["q"][b, h * G:(h + 1) * G].double() @ _exact_rows(st, "k", b, h, n).T * D ** -0.5
            x = x.masked_fill(~near, -math.inf)
            p = torch.softmax(x, -1)
            o[b, h * G:(h + 1) * G] = p @ _exact_rows(st, "v", b, h, n)
            lse[b, h * G:(h + 1) * G] = torch.logsumexp(x, -1)
            if w is not None:
                w[b, h, :n] += p.sum(0)
    return (o, lse) if w is None else (o, lse, w)


def _exact_append(st):
    page, pos, table = st["case"]["page"], st["pos"].tolist(), st["table"].tolist()
    out = []
    for x in "kv":
        c = _values(st[x + "_cache"], st[x + "_scale"]).double()
        for b, n in enumerate(st["lens"].tolist()):
            rows = st[x][b, :, :n].double()              # [Hkv, n, D]
            if st[x + "_scale"] is not None:             # the codes follow their 32-bit definition
                codes, s = _quantized(st[x][b, :, :n])
                rows = codes.double() * s.double()[..., None]
            t = 0
            while t < n:                                 # up to the end of a page at a time
                at = pos[b] + t
                m = min(n - t, page - at % page)
                c[table[b][at // page], :, at % page:at % page + m] = rows[:, t:t + m]
                t += m
        out.append(c[:-1])
    return tuple(out)


def _exact_evict(st):
    c = st["case"]
    B, Hkv, page, budget = (c[x] for x in ("B", "Hkv", "page", "budget"))
    weights = st["weights"].cpu().numpy()
    lens, table, new_table = st["lens"].tolist(), st["table"].cpu().numpy(), st["new_table"].cpu().numpy()
    kept = np.full((B, Hkv, budget), -1, dtype=np.int32)
    nw = np.zeros((B, Hkv, new_table.shape[1] * page))
    caches = [_values(st[x + "_cache"], st[x + "_scale"]).double() for x in "kv"]
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int64)).cuda()
    for b, n in enumerate(lens):
        for h in range(Hkv):
            keep = np.arange(n)
            if n > budget:
                mid = np.arange(c["first"], n - c["last"])
                order = np.lexsort((mid, -weights[b, h, mid].astype(np.float64)))
                mid = mid[order[:budget - c["first"] - c["last"]]]
                keep = np.sort(np.concatenate([np.arange(c["first"]), mid, np.arange(n - c["last"], n)]))
            m = np.arange(len(keep))
            kept[b, h, m], nw[b, h, m] = keep, weights[b, h, keep]
            sp, so, dp, do = (dev(x) for x in (table[b, keep // page], keep % page, new_table[b, m // page], m % page))
            for x in caches:
                x[dp, h, do] = x[sp, h, so]
    return (torch.tensor([min(n, budget) for n in lens], dtype=torch.int32), torch.from_numpy(nw), torch.from_numpy(kept),
            caches[0][:-1], caches[1][:-1])


def exact(case, seed):
    if case["op"] in ("prefill", "train") and case["B"] * case["Hq"] * float(case["N"]) ** 2 > 6e10:
        return None
    st = prepare(case, seed)
    if case["op"] in ("prefill", "train"):
        return _exact_window(st)
    return {"append": _exact_append, "decode": _exact_decode, "evict": _exact_evict}[case["op"]](st)
