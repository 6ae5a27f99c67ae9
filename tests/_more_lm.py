"""64-bit definitions of the norms with rotation, rows in MXFP4 and page tables, on whatever device
their inputs are, and the error bounds of the kernels.

Bounds of the norms with rotation.  f = 2^-24, u = eps / 2 of the 16-bit type.  A sum of D squares is 8
FMAs and 4 additions deep: off by 12 f, its root by 6 f and 2 f of its own, two products more: y is off by
12 f.  A sine or cosine is off by 6 f (series, the angle's rounding) and by the angle's own error, at most
|p| 2^-50 (three roundings of 2^-53 of |p f|, f <= 1, and 2 pi): with the rotation's two roundings z is off
by (24 f + |p| 2^-50) (|y_a| + |y_b|), and by u |z| for its rounding.
Backward: with g' = |dz_a| + |dz_b| the pairs of dz are off by (8 f + |p| 2^-50) g'; in dx = r u - x r^3
mean(u x) the first term is off by that and 16 f, the second by 12 f for its sum, 36 f for r^3 (12 f each),
and products: together below 64 f of S = r g' |w| + |x| r^3 mean(g' |w| |x|).  dw: (24 f + rows f) of the sum
of g' |x| r over its rows (no chain of additions is longer)."""
import numpy as np

import _lm


def angles(inv_freq, p):
    return p.double()[..., None] * inv_freq.double()


def pair(x, R, pairs):
    return (x[..., 0:R:2], x[..., 1:R:2]) if pairs else (x[..., :R // 2], x[..., R // 2:R])


def rotated(x, th, pairs, sign=1.0):
    """x [..., D] turned by th [..., R / 2]."""
    import torch
    R = 2 * th.shape[-1]
    a, b = pair(x, R, pairs)
    c, s = torch.cos(th), sign * torch.sin(th)
    out = x.clone()
    oa, ob = pair(out, R, pairs)
    oa[...], ob[...] = a * c - b * s, b * c + a * s
    return out


def both(x, R, pairs):
    """|a| + |b| in both places of a pair, |x| elsewhere."""
    x = x.abs()
    a, b = pair(x, R, pairs)
    out = x.clone()
    oa, ob = pair(out, R, pairs)
    oa[...], ob[...] = a + b, a + b
    return out


def norm_rope(x, w, th, pairs, eps, live):
    """x [B, H, N, D], th [B, 1, N, R / 2], live [B, 1, N, 1] in 64 bits: y and z."""
    import torch
    y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * w
    return y, torch.where(live, rotated(y, th, pairs), 0.0)


def norm_rope_bound(y, z, R, pairs, p, u, live):
    import torch
    t = (24 * 2.0 ** -24 + p.abs().double()[:, None, :, None] * 2.0 ** -50) * both(y, R, pairs)
    return torch.where(live, t + u * (z.abs() + t) + 2.0 ** -25, 0.0)


def norm_rope_grads(x, w, th, pairs, eps, live, dz, p, u):
    """Gradients by their formulas, and bounds: dx, dw, tx, tw."""
    import torch
    f, R, D = 2.0 ** -24, 2 * th.shape[-1], x.shape[-1]
    x, dz = torch.where(live, x, 1.0), torch.where(live, dz, 0.0)
    r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    g = rotated(dz, th, pairs, -1.0)
    ud = g * w
    dx = r * ud - x * r ** 3 * (ud * x).mean(-1, keepdim=True)
    dw = (g * x * r).sum((0, 1, 2))
    far = p.abs().double()[:, None, :, None] * 2.0 ** -50
    g2 = both(dz, R, pairs)
    size = r * g2 * w.abs() + x.abs() * r ** 3 * (g2 * w.abs() * x.abs()).mean(-1, keepdim=True)
    tx = (64 * f + far) * size
    rows = x.numel() // D
    tw = ((24 * f + rows * f + far) * g2 * x.abs() * r).sum((0, 1, 2)) + 1e-30
    return dx, dw, torch.where(live, tx + u * (dx.abs() + tx) + 2.0 ** -25, 0.0), tw


# ---------------------------------------------------------------- MXFP4 rows
VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def fp4_rows(x):
    """Codes and scale bytes of rows by their definition, in numpy: x [..., D] float64."""
    x = x.reshape(x.shape[:-1] + (-1, 32))
    top = np.abs(x).max(-1)
    e = np.full(top.shape, -127)
    for k in range(127, -128, -1):                       # the smallest e with 6 * 2^e >= max|x|
        e = np.where(6 * 2.0 ** k >= top, k, e)
    y = np.abs(x) / 2.0 ** e[..., None].astype(np.float64)
    v = np.array(VALUES)
    d = np.abs(y[..., None] - v)
    c = d.argmin(-1)                                     # ties: the even code of the two
    tie = (c < 7) & (np.take_along_axis(d, np.minimum(c + 1, 7)[..., None], -1)[..., 0] == d.min(-1))
    c = np.where(tie & (c % 2 == 1), c + 1, c)
    c = c + 8 * np.signbit(x)
    c = c.reshape(c.shape[:-2] + (-1,)).astype(np.uint8)
    return c[..., 0::2] | c[..., 1::2] << 4, (e + 127).astype(np.uint8)


def fp4_values(codes, scale):
    """The rows that codes and scales (torch) stand for, in 64 bits."""
    import torch
    v = torch.tensor(VALUES + [-x for x in VALUES], dtype=torch.float64, device=codes.device)
    x = v[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()]
    return x * torch.exp2(scale.double() - 127).repeat_interleave(32, -1)


def fp4_decode(q, kr, vr, has, window, sinks):
    """As _lm.decode_attention, with this kernel's bounds: an fp16 q enters in two parts, whose D products each are added
    up, and the scale's product; P in two bf16 parts (2^-16)."""
    D = q.shape[-1]
    r = _lm.decode_attention(q, kr, vr, has, window, sinks)
    r["e"] = r["e"] * (2 * D + 8) / (D + 4)
    return r


# ---------------------------------------------------------------- page tables
def plan(table, lens, counts, free, n_free, page, T):
    """sage_kv_plan by its definition, one request at a time (numpy, copies): table, lens, free, n_free,
    granted, starts, pos, slots."""
    table, lens, free = table.copy(), lens.copy(), free.copy()
    S, M = table.shape
    F = len(free)
    n = max(0, min(int(n_free[0]), F))
    for s in range(S):
        lens[s] = max(0, min(int(lens[s]), M * page))
        if counts[s] < 0:
            for x in table[s, :-(-int(lens[s]) // page)]:
                if n < F:
                    free[n] = x
                    n += 1
            table[s], lens[s] = -1, 0
    granted, starts = np.zeros(S, np.int32), np.zeros(S + 1, np.int32)
    pos, slots = np.zeros(T, np.int32), np.full(T, -1, np.int64)
    pages = tokens = total = 0
    left = n
    for s in range(S):
        c, had = int(counts[s]), int(lens[s])
        if c > 0 and had + c <= M * page:
            held, top = -(-had // page), -(-(had + c) // page)
            pages += top - held
            tokens += c
            if (top == held or pages <= n) and tokens <= T:
                for m in range(held, top):
                    left -= 1
                    table[s, m] = free[left]
                for i in range(c):
                    pos[total + i] = had + i
                    slots[total + i] = int(table[s, (had + i) // page]) * page + (had + i) % page
                granted[s], lens[s] = c, had + c
                total += c
        starts[s + 1] = total
    return table, lens, free, np.array([left], np.int32), granted, starts, pos, slots
