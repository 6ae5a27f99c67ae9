"""64-bit definitions of the window attention, the paged cache and one-token
attention, on whatever device their inputs are, and the error bounds of the kernels.

Bounds.  u = eps / 2 of the 16-bit type (bf16 2^-8, fp16 2^-11) and f = 2^-24.  A
score is a sum of D exact products in fp32: off by at most e = (D + 4) f |q|.|k| /
sqrt(D) (the scale and the base change included).  A probability is then off by a
relative 2 e (its own score and the sum's) + 2 (n + 64) f (n-term sums, exp2), and by
u where it is rounded to 16 bits for the product with V, whose sum adds n f."""
import math


def f64(t):
    return t.double()


def visible(i, j, n, window, sinks):
    w = (j <= i) & (j < n)
    return w if window is None else w & ((j > i - window) | (j < sinks))


def window_attention(q, k, v, window, sinks, n, dout=None, u=0.0):
    """One sequence and head: q, k, v [N, D] in 64 bits.  Returns a dict with o, lse, p,
    the score's error bound e and, with dout, the gradients and bounds of their errors
    before the last rounding (u: the 16-bit type's)."""
    import torch
    N, D = q.shape
    at = torch.arange(N, device=q.device)
    see = visible(at[:, None], at[None, :], n, window, sinks) & (at[:, None] < n)
    q, k, v = q.clone(), k.clone(), v.clone()
    q[n:], k[n:], v[n:] = 0, 0, 0
    s = torch.where(see, q @ k.T / math.sqrt(D), -math.inf)
    m = s.amax(-1, keepdim=True).clamp_min(-1e300)
    x = torch.exp(s - m)
    l = x.sum(-1, keepdim=True)
    p = x / torch.where(l > 0, l, 1.0)
    e = (D + 4) * 2.0 ** -24 * torch.where(see, q.abs() @ k.abs().T, 0.0).amax(-1, keepdim=True) / math.sqrt(D)
    r = {"o": p @ v, "lse": (m + torch.log(l))[:, 0], "p": p, "e": e, "av": p @ v.abs(), "see": see}
    if dout is None:
        return r
    # Gradients and their bounds.  P: relative rho (as for O), and u where it meets dO.  dP: D exact
    # products.  delta: O is off by o_bound.  dS = P (dP - delta): both errors, and u for its rounding
    # (in fp16 its power of two leaves at most 2^-38 max|dO| max|V| of underflow).  Sums of N terms.
    g = dout.clone()
    g[n:] = 0
    f, rd = 2.0 ** -24, 1 / math.sqrt(D)
    rho = 2 * e + 2 * (N + 64) * f
    dp, delta = g @ v.T, (g * r["o"]).sum(-1, keepdim=True)
    ds = p * (dp - delta)
    e_dp = (D + 4) * f * (g.abs() @ v.abs().T)
    e_delta = (g.abs() * o_bound(r, n, u)).sum(-1, keepdim=True) + (D + 4) * f * (g.abs() * r["o"].abs()).sum(-1, keepdim=True)
    low = 2.0 ** -38 * float(g.norm(dim=-1).max() * v.norm(dim=-1).max()) if n else 0.0
    e_ds = (rho + u) * ds.abs() + (1 + u) * p * (e_dp + e_delta) + torch.where(see, low, 0.0)
    r["dq"], r["dk"], r["dv"] = ds @ k * rd, ds.T @ q * rd, p.T @ g
    # dQ_i = sum_j dS_ij (K_j - c) for any c, as sum_j dS_ij = 0: the kernel's is the sum over its
    # rounded dS, off by sum_j e_ij |K_j - c|.  Its c is the mean of the last 64-key tile that the
    # workgroup of 128 queries reads.
    edq = torch.zeros_like(r["dq"])
    for q0 in range(0, n, 128):
        last = min(q0 + 128, n)
        tile = k[(last - 1) // 64 * 64:min(n, (last - 1) // 64 * 64 + 64)]
        c, rows = tile.mean(0, keepdim=True), slice(q0, last)
        edq[rows] = e_ds[rows] @ (k - c).abs() + (N + 64) * f * (ds[rows].abs() @ (k.abs() + c.abs()))
    r["edq"] = edq * rd
    r["edk"] = (e_ds + N * f * ds.abs()).T @ q.abs() * rd
    r["edv"] = ((rho + u + N * f) * p).T @ g.abs()
    return r


def unit(dtype):
    import torch
    return torch.finfo(dtype).eps / 2


def o_bound(r, n, u, up=None):
    """Bound of |O - o| per element: P's error against the sum of p |v|, and O's own rounding."""
    up = u if up is None else up
    rel = up + 2 * r["e"] + 2 * (n + 64) * 2.0 ** -24 + n * 2.0 ** -24
    t = rel * r["av"]
    return t + u * (r["o"].abs() + t) + 1e-30


def lse_bound(r, n):
    return r["e"][:, 0] + (n + 64) * 2.0 ** -24 + 2.0 ** -21 * r["lse"].abs().nan_to_num(0, 0, 0) + 2.0 ** -21


def cache_rows(cache, scale, table_row, h, n):
    """The first n rows of one sequence and head in 64 bits, and which of them have a page."""
    import torch
    P, _, page, D = cache.shape
    rows, has = [], []
    for j in range(n):
        pid = int(table_row[j // page])
        ok = 0 <= pid < P
        has.append(ok)
        x = cache[pid, h, j % page].double() if ok else torch.zeros(D, dtype=torch.float64, device=cache.device)
        if ok and scale is not None:
            x = x * scale[pid, h, j % page].double()
        rows.append(x)
    if not rows:
        return torch.zeros((0, D), dtype=torch.float64, device=cache.device), torch.zeros(0, dtype=torch.bool)
    return torch.stack(rows), torch.tensor(has, device=cache.device)


def decode_attention(q, kr, vr, has, window, sinks):
    """One sequence and key head: q [G, D], rows [n, D] in 64 bits."""
    import torch
    n, D = kr.shape
    if n == 0:
        z = q.new_zeros
        return {"o": z(q.shape), "lse": z(q.shape[0]) - math.inf, "p": z((q.shape[0], 0)), "e": z((q.shape[0], 1)),
                "av": z(q.shape)}
    see = visible(n - 1, torch.arange(n, device=q.device), n, window, sinks) & has
    s = torch.where(see, q @ kr.T / math.sqrt(D), -math.inf)
    m = s.amax(-1, keepdim=True).clamp_min(-1e300)
    x = torch.exp(s - m)
    l = x.sum(-1, keepdim=True)
    p = x / torch.where(l > 0, l, 1.0)
    vr = torch.where(see[:, None], vr, 0.0)
    e = (D + 4) * 2.0 ** -24 * torch.where(see, q.abs() @ kr.abs().T, 0.0).amax(-1, keepdim=True) / math.sqrt(D)
    return {"o": p @ vr, "lse": (m + torch.log(l))[:, 0], "p": p, "e": e, "av": p @ vr.abs()}


def quantized(x):
    """Codes and scales of 8-bit cache rows (their 32-bit definition).  Divided by a tensor:
    torch multiplies by the reciprocal where the divisor is a number."""
    import torch
    x = x.float()
    s = x.abs().amax(-1)
    s = s / torch.full_like(s, 127)
    s = torch.where(s >= 2.0 ** -126, s, 0.0)
    r = torch.where(s > 0, 1 / s, 0.0)
    return torch.round(x * r[..., None]).to(torch.int8), s


def kept_tokens(w, n, budget, first, last):
    """Which of n cached tokens an eviction keeps, by its definition (w: numpy, one head)."""
    import numpy as np
    if n <= budget:
        return np.arange(n)
    mid = np.arange(first, n - last)
    key = np.where(np.isnan(w[mid]), -np.inf, w[mid].astype(np.float64))
    # NaN below -inf
    order = sorted(range(len(mid)), key=lambda i: (-key[i], bool(np.isnan(w[mid[i]])), mid[i]))
    pick = mid[np.array(order[:budget - first - last], dtype=np.int64)]
    return np.sort(np.concatenate([np.arange(first), pick, np.arange(n - last, n)]).astype(np.int64))
