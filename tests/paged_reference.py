"""Plain 64-bit forms of the paged-cache operators, on the CPU, and the error their kernels may make."""
import math

import torch

TOP = {torch.float8_e4m3fn: 448.0, torch.int8: 127.0}
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # one rounding, relative


def quantise(x, kind):
    """Rows as (values kept, scale or None); the scale and the quotient are rounded to fp32, the code to nearest even."""
    x = x.double()
    if kind not in TOP:
        return x, None
    scale = (x.abs().amax(-1) / TOP[kind]).float().double()
    scale = torch.where(scale < 2.0 ** -100, torch.full_like(scale, 2.0 ** -100), scale)
    y = (x / scale[..., None]).float().double().clamp(-TOP[kind], TOP[kind])
    if kind == torch.int8:
        return y.round(), scale
    unit = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)      # a quarter of a step is never a border
    return (y / unit).round() * unit, scale


def norm_rope(x, w, positions, inv_freq, eps, interleaved):
    """(value, error bound) of the normed and rotated rows x [T, H, d]."""
    y = x.double()
    if w is not None:
        y = y / (y.square().mean(-1, keepdim=True) + eps).sqrt() * w.double()
    R = 2 * inv_freq.numel()
    angle = positions.double()[:, None, None] * inv_freq.double()
    cos, sin = angle.cos(), angle.sin()
    z, size = y.clone(), y.abs()
    ia = torch.arange(0, R, 2) if interleaved else torch.arange(R // 2)
    ib = ia + (1 if interleaved else R // 2)
    a, b = y[..., ia], y[..., ib]
    z[..., ia], z[..., ib] = a * cos - b * sin, b * cos + a * sin
    size[..., ia] = size[..., ib] = a.abs() + b.abs()
    # fp32 steps: the mean square (8 + 4 additions, halved by the root), root and quotient (2^-23 each),
    # two products; the angle reduced to half turns in fp32 (pi 2^-25), sinpi / cospi (2^-23), and the
    # rotation's three operations: together below 24 half steps of |a| + |b|
    return z, size * 24 * 2.0 ** -24 + z.abs() * HALF_STEP[x.dtype]


def attention(q, k, v, dtype, scale=None, kind=None):
    """One sequence: q [Hq, d], k and v [Hkv, n, d] in 64 bits. Returns (out, lse, out bound, lse bound)."""
    Hq, d = q.shape
    H, n = k.shape[:2]
    if n == 0:
        return torch.zeros(Hq, d, dtype=torch.float64), torch.full((Hq,), -math.inf, dtype=torch.float64), torch.zeros(Hq, d), torch.zeros(Hq)
    scale = d ** -0.5 if scale is None else scale
    q = q.double().view(H, -1, d)
    s = torch.einsum("hgd,hnd->hgn", q, k) * scale
    p = torch.softmax(s, -1)
    out, lse = torch.einsum("hgn,hnd->hgd", p, v), torch.logsumexp(s, -1)
    # a logit: d products and additions in fp32, then three factors (scale, row scale, log2 e) and the difference from the
    # maximum; fp32 operands lose 2^-23 to their three bf16 parts, which the first term's slack of two covers
    es = (2 * d * 2.0 ** -24 * torch.einsum("hgd,hnd->hgn", q.abs(), k.abs()).amax(-1) * abs(scale) + 6 * 2.0 ** -24 * s.abs().amax(-1)).unsqueeze(-1)
    # a probability: its logit's error, exp2 (2^-22), up to n additions to the sum in chains of n/16 or fewer and rescalings;
    # its parts for the product: 2^-16 for bf16 outputs, 2^-22 for fp32. Of an 8-bit cache (kind) and bf16 outputs it is one
    # fp16 number: half a step, 2^-11 of it, or, below fp16's normal range, of 2^-24 in units of 2^-8 (the kernel gives a
    # probability of 1 at the largest value scale the weight 2^8), per key and times the largest value
    ep = 2 * es + 2.0 ** -21 + (n / 16 + 40) * 2.0 ** -24
    single = dtype == torch.bfloat16 and kind in TOP
    parts = 2.0 ** -11 if single else 2.0 ** -16 if dtype == torch.bfloat16 else 2.0 ** -22
    weight = torch.einsum("hgn,hnd->hgd", p, v.abs())
    bound = weight * (ep + parts) + out.abs() * HALF_STEP[dtype]
    if single:
        bound = bound + n * 2.0 ** -33 * v.abs().amax((1, 2))[:, None, None]
    return out.view(Hq, d), lse.view(Hq), bound.view(Hq, d), (ep.squeeze(-1) + lse.abs() * 2.0 ** -22).view(Hq)


def page_bounds(k, page):
    """[pages, H, 2, d] of one sequence's keys [n, H, d]: smallest and largest value per dimension; NaN does not count."""
    rows = []
    for i in range(0, k.shape[0], page):
        x = k[i:i + page].double()
        rows.append(torch.stack([x.nan_to_num(nan=math.inf, posinf=math.inf, neginf=-math.inf).amin(0),
                                 x.nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf).amax(0)], 1))
    return torch.stack(rows) if rows else torch.zeros(0, k.shape[1], 2, k.shape[2], dtype=torch.float64)


def choose(q, bounds, sink, recent, top):
    """Pages of one sequence for every KV head, a list of ascending lists: q [Hq, d], bounds [pages, H, 2, d]."""
    count, H = bounds.shape[:2]
    q = q.double().view(H, -1, q.shape[-1])
    chosen = []
    for h in range(H):
        if count <= sink + recent + top:
            chosen.append(list(range(count)))
            continue
        e = bounds[:, h].double()
        score = torch.maximum(q[h][None] * e[:, 0, None], q[h][None] * e[:, 1, None]).sum((1, 2)).tolist()
        middle = sorted(range(sink, count - recent), key=lambda i: (0 if score[i] != score[i] else 1, -score[i] if score[i] == score[i] else 0, i))
        chosen.append(sorted(list(range(sink)) + middle[:top] + list(range(count - recent, count))))
    return chosen
