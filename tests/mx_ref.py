"""Plain 64-bit forms of the operators around a cache in 8 or 4 bits, and bounds on what their arithmetic in 32 bits may be off by."""
import math
import random

import torch

import requests_ref as R
from paper_2405_14430_amd import KvMxPages, pf_kv_mx_row_bytes

U = R.U
FORMATS = ["e4m3", "e2m1"]
TOP = {"e4m3": 448.0, "e2m1": 6.0}
RANGE = {"e4m3": (-117, 119), "e2m1": (-125, 125)}
# all magnitudes, in the order of their codes
MAGNITUDES = {"e4m3": [m / 8 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)][:-1],
              "e2m1": [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]}


def blocks(dh):
    return (dh + 31) // 32


def encode(x, fmt):
    """x [..., dh] in 64 bits -> codes [..., dh] (one to an element), exponent bytes [..., blocks], as int64."""
    grid = torch.tensor(MAGNITUDES[fmt], dtype=torch.float64)
    half = len(grid) + (fmt == "e4m3")         # the sign's place: 7f is no number
    lo, hi = RANGE[fmt]
    codes, exps = torch.zeros(x.shape, dtype=torch.int64), []
    for b in range(0, x.shape[-1], 32):
        y = x[..., b:b + 32]
        most = y.abs().amax(-1)
        bad = ~torch.isfinite(y).all(-1)
        e = torch.full(most.shape, lo, dtype=torch.int64)
        for k in range(lo, hi):                # the least exponent under which the largest fits
            e = torch.where((most > TOP[fmt] * 2.0 ** k) & (e == k), k + 1, e)
        z = (y.abs() / torch.exp2(e.double())[..., None]).clamp(max=TOP[fmt])
        below = (torch.searchsorted(grid, z.nan_to_num(0.0).contiguous(), right=True) - 1).clamp(max=len(grid) - 2)
        down, up = z - grid[below], grid[below + 1] - z
        code = below + ((up < down) | ((up == down) & (below % 2 == 1))).long()
        code = code + half * torch.signbit(y).long()
        codes[..., b:b + 32] = torch.where(bad[..., None], 0, code)
        exps.append(torch.where(bad, 255, e + 127))
    return codes, torch.stack(exps, -1)


def packed(codes, fmt, dh):
    """Rows of bytes as the pages hold them."""
    rows = torch.zeros(*codes.shape[:-1], pf_kv_mx_row_bytes(fmt, dh), dtype=torch.int64)
    if fmt == "e4m3":
        rows[..., :dh] = codes
    else:
        rows[..., :dh // 2] = codes[..., 0::2] + 16 * codes[..., 1::2]
    return rows.to(torch.uint8)


def decode(rows, exps, fmt, dh):
    """Rows of bytes and exponents (uint8) -> [..., dh] in 64 bits; values past the largest bf16 number are infinities."""
    rows, exps = rows.cpu().long(), exps.cpu().long()
    codes = rows if fmt == "e4m3" else torch.stack((rows % 16, rows // 16), -1).flatten(-2)
    codes = codes[..., :dh]
    grid = torch.tensor(MAGNITUDES[fmt] + [math.nan] * (fmt == "e4m3"), dtype=torch.float64)
    e = exps.repeat_interleave(32, -1)[..., :dh]
    v = grid[codes % len(grid)] * torch.exp2(e.double() - 127)
    v = torch.where(v >= 2.0 ** 128, math.inf, v)
    v = torch.where(e == 255, math.nan, v)
    return torch.where(codes >= len(grid), -v, v)


def head_norm(x, dh, kind, w, b, eps):
    """x [tokens, heads * dh] -> (normed, bound on an fp32 evaluation)."""
    x = R.d64(x).unflatten(1, (-1, dh))
    if kind == "none":
        return x.flatten(1), torch.zeros_like(x).flatten(1)
    mean = x.mean(-1, keepdim=True) if kind == "layer" else torch.zeros(*x.shape[:-1], 1, dtype=torch.float64)
    r = 1 / torch.sqrt(((x - mean) ** 2).mean(-1, keepdim=True) + eps)
    plain = (x - mean) * r
    w = torch.ones(dh, dtype=torch.float64) if w is None else R.d64(w)
    b = torch.zeros(dh, dtype=torch.float64) if b is None else R.d64(b)
    # sums of at most 128 terms, 8 in a lane and 5 exchanges: 13 roundings each, halved for the root; mean, root, quotient, products and
    # sum behind them below 12; a mean that is off moves every element by its own error
    off = 16 * U * x.abs().mean(-1, keepdim=True) if kind == "layer" else 0.0
    return (plain * w + b).flatten(1), (w.abs() * (24 * U * plain.abs() + r * (off + 2 * U * mean.abs())) + 2 * U * b.abs()).flatten(1)


def turn(x, dh, norm, pos=None, rope=None):
    """norm = (kind, w, b, eps), rope = arguments of requests_ref.rope; returns (rows, bound without the output's rounding)."""
    y, e = head_norm(x, dh, *norm)
    if rope is None:
        return y, e
    z, bound = R.rope(y, pos, **rope)
    axes, layout, mag = rope["axes"], rope["layout"], rope.get("magnitude", 1.0)
    e = e.unflatten(1, (-1, dh)).clone()
    at = 0
    for w in axes:                             # an error of either channel of a pair reaches both
        first = torch.arange(at, at + w, 2) if layout == "interleaved" else torch.arange(at, at + w // 2)
        second = first + 1 if layout == "interleaved" else first + w // 2
        both = mag * (e[..., first] + e[..., second])
        e[..., first] = e[..., second] = both
        at += w
    return z, bound + e.flatten(1)


def make_pages(fmt, kv_heads, dh, page, need, seed=0, fill=None, spare=3, gap=0, std=1.0):
    """Pools with `need` pages per sequence in an arbitrary order, of random rows or of bytes `fill`; gap: bytes between pages (16s)."""
    n = sum(need) + spare
    order = list(range(n))
    random.Random(seed).shuffle(order)
    width = max(max(need), 1)
    table, at = [], 0
    for c in need:
        table.append(order[at:at + c] + [-1] * (width - c))
        at += c

    def pool(rows):
        flat = torch.full((n, rows[0].numel() + gap), 0xa5, dtype=torch.uint8)
        flat[:, :rows[0].numel()] = rows.flatten(1)
        return flat.cuda()[:, :rows[0].numel()].unflatten(1, rows.shape[1:])

    def both(s):
        if fill is not None:
            code = torch.full((n, kv_heads, page, pf_kv_mx_row_bytes(fmt, dh)), fill, dtype=torch.uint8)
            return pool(code), pool(torch.full((n, kv_heads, page, blocks(dh)), fill, dtype=torch.uint8))
        x = torch.randn(n, kv_heads, page, dh, generator=torch.Generator().manual_seed(s)) * std
        codes, exps = encode(x.double(), fmt)
        return pool(packed(codes, fmt, dh)), pool(exps.to(torch.uint8))

    (k, ks), (v, vs) = both(seed + 100), both(seed + 200)
    return KvMxPages(fmt, k, v, ks, vs, torch.tensor(table, dtype=torch.int32).cuda(), dh)


def slot_rows(pages, which, s, n):
    """Slots [0, n) of sequence s of "k" or "v", [n, kv_heads * head_dim] in 64 bits, and which of them have a page."""
    code, exp = getattr(pages, which).cpu(), getattr(pages, which + "_scale").cpu()
    values = decode(code, exp, pages.format, pages.head_dim)
    table = pages.table.cpu()
    out = torch.zeros(n, pages.kv_heads * pages.head_dim, dtype=torch.float64)
    have = torch.zeros(n, dtype=torch.bool)
    for t in range(min(n, pages.max_pages * pages.page_size)):
        pg = int(table[s, t // pages.page_size])
        if 0 <= pg < code.shape[0]:
            out[t], have[t] = values[pg, :, t % pages.page_size].reshape(-1), True
    return out, have
