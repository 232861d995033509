"""Plain 64-bit forms of the operators on packed rows, and bounds on what their arithmetic in fewer bits may be off by.

Bounds count a rounding as half a step: 2^-8 of the value for bf16, 2^-24 for fp32."""
import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 0.0}   # of a stored output (fp32 outputs: in the arithmetic's share)
U = 2.0 ** -24
DTYPES = [torch.bfloat16, torch.float32]


def d64(t):
    return t.detach().cpu().double()


def frequencies(w, theta, scaling, factor, low, high, original_len):
    """Radians per position of the w / 2 pairs of one axis, by the definitions in the header."""
    out = []
    base = theta * factor ** (w / (w - 2)) if scaling == "ntk" and w > 2 else theta
    for i in range(w // 2):
        f = base ** (-2.0 * i / w)
        if scaling == "linear":
            f /= factor
        elif scaling == "ramp_turns":
            keep = min(max((original_len * f / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
            f = f * keep + f / factor * (1 - keep)
        elif scaling == "ramp_index":
            index = lambda n: w * math.log(original_len / (2 * math.pi * n)) / (2 * math.log(theta))
            a, b = max(math.floor(index(high)), 0), min(math.ceil(index(low)), w - 1)
            keep = 1 - min(max((i - a) / max(b - a, 1e-3), 0.0), 1.0)
            f = f * keep + f / factor * (1 - keep)
        out.append(f)
    return torch.tensor(out, dtype=torch.float64)


def rope(x, pos, head_dim, axes, layout, theta, scaling="none", factor=1.0, low=1.0, high=32.0, original_len=1, magnitude=1.0):
    """(turned rows, bound on an fp32 evaluation) in 64 bits; x [tokens, heads * head_dim], pos [tokens, n_axes]."""
    x = d64(x)
    y = x.reshape(x.shape[0], -1, head_dim).clone()
    bound = torch.zeros_like(y)
    pos = pos.cpu().double().reshape(x.shape[0], len(axes))
    at = 0
    for a, w in enumerate(axes):
        ang = pos[:, a, None] * frequencies(w, theta, scaling, factor, low, high, original_len)
        c, s = (magnitude * torch.cos(ang))[:, None], (magnitude * torch.sin(ang))[:, None]
        first = torch.arange(at, at + w, 2) if layout == "interleaved" else torch.arange(at, at + w // 2)
        second = first + 1 if layout == "interleaved" else first + w // 2
        p, q = y[..., first].clone(), y[..., second].clone()
        y[..., first], y[..., second] = p * c - q * s, p * s + q * c
        # the fraction of a turn rounded to 32 bits (2^-26 turns, 2^-23.3 rad), sine and cosine within two units, two
        # products and a sum: below 8 roundings of the pair's size
        bound[..., first] = bound[..., second] = 8 * U * magnitude * (p.abs() + q.abs())
        at += w
    return y.reshape(x.shape), bound.reshape(x.shape)


def attention(q, k, v, head_dim, last, scale=None, present=None):
    """One sequence in 64 bits: q [n, H * dh], k, v [m, Hk * dh]; query i sees keys 0 .. last[i] - 1 that are `present`.
    Returns out, lse, bound_bf16, bound_f32, bound_lse: what the arithmetic may be off by, without the output's own rounding."""
    q, k, v = (d64(t).reshape(t.shape[0], t.shape[1] // head_dim, head_dim) for t in (q, k, v))
    n, H, m, Hk = q.shape[0], q.shape[1], k.shape[0], k.shape[1]
    scale = 1 / math.sqrt(head_dim) if scale is None else scale
    out, mag = torch.zeros(n, H, head_dim, dtype=torch.float64), torch.zeros(n, H, head_dim, dtype=torch.float64)
    lse, size = torch.full((n, H), -math.inf, dtype=torch.float64), torch.zeros(n, H, dtype=torch.float64)
    if n and m:
        seen = torch.arange(m)[None] < last[:, None]
        if present is not None:
            seen = seen & present[None]
        some = seen.any(1)
        used = seen.any(0)   # rows that no query sees may hold anything
        k, v = torch.where(used[:, None, None], k, 0.0), torch.where(used[:, None, None], v, 0.0)
        for h in range(H):
            kh, vh = k[:, h * Hk // H], v[:, h * Hk // H]
            s = (q[:, h] @ kh.T * scale).masked_fill(~seen, -math.inf)
            lse[:, h] = torch.logsumexp(s, 1)
            p = torch.exp(s - lse[:, h, None].masked_fill(~some[:, None], 0.0))
            out[:, h], mag[:, h] = p @ vh, p @ vh.abs()
            size[:, h] = (q[:, h].abs() @ kh.abs().T * scale).masked_fill(~seen, 0.0).amax(1)
    # a score: dh products and sums; its exponent: a multiply-add and the hardware's 2^x (2^-22 relative); both a weight and the
    # denominator carry it.  The sums over keys: m roundings each.
    score = (head_dim + 8) * U * size + 2.0 ** -21
    rel = (2 * score + 2 * (m + 8) * U)[..., None]
    shape = (n, H * head_dim)
    return out.reshape(shape), lse, ((rel + 2.0 ** -8) * mag).reshape(shape), (rel * mag).reshape(shape), score + (m + 8) * U


def norm(x, kind, w, b, eps):
    if kind == "none":
        return x, torch.ones(x.shape[0], 1, dtype=torch.float64), torch.zeros(x.shape[0], 1, dtype=torch.float64)
    mean = x.mean(1, keepdim=True) if kind == "layer" else torch.zeros(x.shape[0], 1, dtype=torch.float64)
    r = 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + eps)
    y = (x - mean) * r
    y = y if w is None else y * d64(w)
    return y if b is None else y + d64(b), r, mean


def norm_residual(y, x, seg, post=("none", None, None, 0.0), pre=("none", None, None, 0.0), gate=None, gate_tanh=False, x_scale=1.0,
                  scale=None, shift=None):
    """(x', h, bound of x', bound of h before its own rounding); seg: sequence of each row, or None for shared vectors."""
    pick = lambda t, one: torch.full((1, x.shape[1]), one, dtype=torch.float64) if t is None else d64(t)[seg] if seg is not None else d64(t)[None]
    x = d64(x) * x_scale
    big = x.abs()
    if y is not None:
        yn, r, mean = norm(d64(y), *post)
        g = pick(gate, 1.0)
        g = torch.tanh(g) if gate_tanh else g
        bias = 0.0 if post[2] is None else d64(post[2]).abs()
        w = 1.0 if post[1] is None else d64(post[1]).abs()
        x = x + g * yn
        # sums of at most 64 rounded terms in a lane and the tree above them, then a handful of roundings per element; a mean
        # that is off moves every element by its own size
        big = big + g.abs() * (yn.abs() + bias + (r * mean.abs() * w if post[0] == "layer" else 0.0))
    e_x = 96 * U * big
    n, r, mean = norm(x, *pre)
    w = torch.ones(1, x.shape[1], dtype=torch.float64) if pre[1] is None else d64(pre[1])[None].abs()
    b = torch.zeros_like(w) if pre[2] is None else d64(pre[2])[None].abs()
    sc, sh = pick(scale, 0.0), pick(shift, 0.0)
    h = n * (1 + sc) + sh
    plain = (x - mean) * r
    lift = r * (e_x + e_x.mean(1, keepdim=True)) + plain.abs() * r * e_x.amax(1, keepdim=True)
    e_h = (1 + sc).abs() * w * (lift + 96 * U * (plain.abs() + r * mean.abs())) + 8 * U * ((1 + sc).abs() * (b + plain.abs() * w) + sh.abs())
    return x, h, e_x, e_h


def check(got, want, bound, what):
    """Every element within its bound; NaN and infinities only where the reference has them."""
    got = d64(got)
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    bad = ~same & ~((got - want).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[0].tolist(), float(got[bad][0]), float(want[bad][0]), float(bound.expand_as(want)[bad][0]))


def stored(bound, want, dtype):
    """The arithmetic's bound and the rounding to the type it is stored in."""
    return bound + HALF_STEP[dtype] * (want.abs() + bound) + 1e-30
