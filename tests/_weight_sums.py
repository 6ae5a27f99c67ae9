"""The bound on the weights' gradients of the norms with rotation, by the additions that a term goes through.

f = 2^-24.  A term g x r of a row: g, the pairs of dz turned back, is off by (8 f + |p| 2^-50) (|dz_a| + |dz_b|); r by
6 f (half of the 12 f of its sum of squares), f for the mean with eps and 2 f of its own; x r by f: together below
24 f + |p| 2^-50 of g' |x| r, with g' = |dz_a| + |dz_b|.  The sum: a lane adds its rows one after another, 64 / (D / 8)
lanes and 4 waves are added in pairs, and of the workgroups' sums 64 chains, these in pairs again.  Each addition
rounds by f of a sum that is at most that of its terms' sizes, so that all of them together are off by f times the
number of additions that a term goes through, times the sum of g' |x| r."""
import _more_lm as mo


def cdiv(a, b):
    return -(-a // b)


def additions(B, Hq, Hkv, N, D):
    """The most additions on a term's way into dq_weight, and into dk_weight."""
    rows = 512 // D                                      # that a wave takes in a step
    sq, sk, tokens, split = cdiv(Hq, rows), cdiv(Hkv, rows), B * N, 1
    while split * 2 <= sq + sk and tokens * split < 4096:        # waves that share a token
        split *= 2
    blocks = min(1024, cdiv(tokens * split, 4))
    passes = cdiv(tokens * split, 4 * blocks)            # tokens of a wave
    pairs = {128: 2, 64: 3}[D] + 2
    return [passes * cdiv(s, split) + pairs + cdiv(blocks, 64) + 6 for s in (sq, sk)]


def make(case, device):
    """Inputs of a case of test_gpu_more_lm.ROPES: q, k, weights, inv_freq, positions, live rows, gradients, keywords."""
    import torch
    B, Hq, Hkv, N, D, R, pairs, dtype, at, lens, packed, weights = case
    dt = {"bf16": torch.bfloat16, "fp16": torch.float16}[dtype]
    g = torch.Generator(device=device).manual_seed(11 + N + 5 * D + R)
    rn = lambda *s: torch.randn(s, generator=g, device=device)
    ints = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g, device=device).to(torch.int32)
    q, k = rn(B, Hq, N, D).to(dt), (rn(B, Hkv, N, D) + rn(1, Hkv, 1, D)).to(dt)
    dq, dk = rn(B, Hq, N, D).to(dt), rn(B, Hkv, N, D).to(dt)
    w = [1 + 0.3 * rn(D) for _ in range(2)]
    inv = (10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64, device=device) / max(R, 1))).float()
    pos = {"0": None, "start": ints(0, 200000, B), "each": ints(-50, 5000, B, N), "far": ints(2 ** 30, 2 ** 31 - 1000 - N, B)}[at]
    p = torch.arange(N, device=device).expand(B, N)
    if pos is not None:
        p = pos.long() if pos.dim() == 2 else p + pos.long()[:, None]
    n = torch.full((B,), N, device=device) if lens is None else torch.tensor(lens, device=device)
    live = (torch.arange(N, device=device) < n[:, None])[:, None, :, None]
    kw = dict(pos=pos, lens=None if lens is None else n.to(torch.int32), eps=1e-5, interleaved=pairs)
    return q, k, w, inv, p, live, dq, dk, kw


def weight_gradients(case, q, k, w, inv, p, live, dq, dk):
    """For q and for k: every row's terms [rows, D] in 64 bits (their sum is the gradient), and its bound."""
    import torch
    B, Hq, Hkv, N, D, R, pairs = case[:7]
    f, out = 2.0 ** -24, []
    th = mo.angles(inv, p)[:, None]
    far = p.abs().double()[:, None, :, None] * 2.0 ** -50
    for x, dz, depth in zip((q, k), (dq, dk), additions(B, Hq, Hkv, N, D)):
        x, dz = torch.where(live, x.double(), 1.0), torch.where(live, dz.double(), 0.0)
        r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-5)
        terms = (mo.rotated(dz, th, pairs, -1.0) * x * r).flatten(0, 2)
        tol = (((24 + depth) * f + far) * mo.both(dz, R, pairs) * x.abs() * r).sum((0, 1, 2)) + 1e-30
        out.append((terms, tol))
    return out
