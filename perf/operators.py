"""Operators for requests of different sizes: the calls they are timed on, and the ranges these stand for.

A program that serves images of several resolutions, and the prompts in front of them, keeps the rows of all requests
packed behind each other and the keys and values in pages.  One block of its model then makes these calls:

* `rope`    - rotary positions on packed rows (`pf_op_rope`);
* `append`  - the same rotation on q and k together with the write of k and v into the pages (`pf_op_kv_append`);
* `packed`  - attention over packed sequences (`pf_op_attention_packed`);
* `paged`   - attention of each request's new rows over its pages (`pf_op_attention_paged`);
* `norm`    - the norms, gate and residual between a branch and the next one (`pf_op_norm_residual`).

With `own` false the operators are computed in their plain form, elementary operations in 32 bits (angles in 64); with
`own` true by the library.  `exact` computes them from their definitions in 64 bits.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
ESZ = {"bf16": 2, "f32": 4}


# ---- the cases ------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one new token of each of 32 prompts: rotation of part of each head, frequencies stretched for a long context
        dict(name="rope_tokens", op="rope", dtype="bf16", tokens=32, heads=32, head_dim=128, axes="64", layout="half",
             theta=500000.0, scaling="ramp_turns", far=100000),
        # the rows of one 2048 px image behind its 512 text rows: three axes (text, row, column), interleaved pairs
        dict(name="rope_image", op="rope", dtype="bf16", tokens=16896, heads=32, head_dim=128, axes="16,56,56",
             layout="interleaved", theta=10000.0, scaling="none", far=128),
        # one new token of each of 48 prompts goes into its last page
        dict(name="append_tokens", op="append", dtype="bf16", new=",".join(["1"] * 48), first="ragged:4096", heads=32,
             kv_heads=8, head_dim=128, page=16, axes="128", layout="half", theta=1000000.0, scaling="linear"),
        # three prompts written at once by the program that a bf16 one is judged against (head size of the 1152-wide stage)
        dict(name="append_prompts_f32", op="append", dtype="f32", new="4100,1031,2047", first="zero", heads=16, kv_heads=16,
             head_dim=72, page=64, axes="72", layout="interleaved", theta=10000.0, scaling="none"),
        # short prompts of a text conditioner in fp32: all latency
        dict(name="packed_prompts_f32", op="packed", dtype="f32", q="1,7,19,77,120,33,64", k="", causal=True, heads=16,
             kv_heads=4, head_dim=64),
        # images of six resolutions in one call, head size 72, every token sees its whole image
        dict(name="packed_images", op="packed", dtype="bf16", q="4096,2304,1024,9216,1536,4080", k="", causal=False,
             heads=16, kv_heads=16, head_dim=72),
        # prompts of very different lengths, causal, four query heads to a key head
        dict(name="packed_prompts", op="packed", dtype="bf16", q="16384,8192,3001,517,128,1", k="", causal=True, heads=32,
             kv_heads=8, head_dim=128),
        # one new token of each of 64 prompts, caches from a few to 16k tokens
        dict(name="paged_tokens", op="paged", dtype="bf16", new=",".join(["1"] * 64), kv="ragged:16384", heads=32,
             kv_heads=8, head_dim=128, page=16, causal=True, lse=False),
        # one new token of a single long request
        dict(name="paged_long_token", op="paged", dtype="bf16", new="1", kv="131071", heads=16, kv_heads=2, head_dim=128,
             page=64, causal=True, lse=False),
        # a patch of 512 rows in the middle of each of four images' caches, the other rows a step old (1536-wide stage);
        # the log-sum-exp goes to a program that joins parts of a sequence
        dict(name="paged_patches", op="paged", dtype="bf16", new="512,512,512,512", kv="4250,4250,4250,4250", heads=24,
             kv_heads=24, head_dim=64, page=128, causal=False, lse=True),
        # a few rows, RMS norms on both sides and a tanh gate
        dict(name="norm_tokens", op="norm", dtype="bf16", rows="1,5,26", d=1536, post="rms", pre="rms", gate_tanh=True,
             x_scale=1.0, modulate=False),
        # the rows of four 1024 px images, LayerNorm with per-image modulation after the branch's own norm
        dict(name="norm_images_f32", op="norm", dtype="f32", rows="4096,4096,4096,4096", d=1152, post="rms", pre="layer",
             gate_tanh=False, x_scale=0.8, modulate=True),
    ]


def _ragged(rng, n, lo, hi, total):
    """n lengths spread over the logarithm of [lo, hi], with a sum of at most `total` (or one each)."""
    out = [int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))) for _ in range(n)]
    while sum(out) > total and max(out) > 1:
        i = out.index(max(out))
        out[i] = max(1, out[i] // 2)
    return out


def _text(lengths):
    return ",".join(str(x) for x in lengths)


def _heads(rng):
    kv = rng.choice([1, 2, 3, 4, 8, 16])
    group = rng.choice([1, 1, 2, 4, 7, 8])
    while kv * group > 32:
        group = max(1, group // 2)
    return kv * group, kv


def _rotation(rng, head_dim):
    kind = rng.choice(["one", "part", "two", "three"])
    if kind == "one":
        axes = [head_dim]
    elif kind == "part":
        axes = [2 * rng.randint(1, head_dim // 2)]
    elif kind == "two":
        w = head_dim // 4 * 2
        axes = [w, head_dim - w]
    else:
        w = (head_dim - 16) // 4 * 2
        axes = [16, w, head_dim - 16 - w]
    return dict(axes=_text(axes), layout=rng.choice(["interleaved", "half"]), theta=rng.choice([1e4, 1e5, 1e6]),
                scaling=rng.choice(["none", "linear", "ntk", "ramp_turns", "ramp_index"]))


def draw(rng):
    op = rng.choice(["rope", "append", "packed", "paged", "norm"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    dh = rng.choice([64, 64, 72, 80, 96, 128, 128])
    heads, kv_heads = _heads(rng)
    log_int = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if op == "rope":
        return dict(op=op, dtype=dtype, tokens=log_int(1, 16000), heads=heads, head_dim=dh, far=log_int(64, 1000000),
                    **_rotation(rng, dh))
    if op == "append":
        new = _ragged(rng, log_int(1, 48), 1, rng.choice([1, 16, 4096]), 12000)
        return dict(op=op, dtype=dtype, new=_text(new), first=rng.choice(["zero", "ragged:%d" % log_int(16, 20000)]),
                    heads=heads, kv_heads=kv_heads, head_dim=dh, page=rng.choice([16, 32, 64, 128, 256]), **_rotation(rng, dh))
    if op == "packed":
        total = 3000 if dtype == "f32" else 14000
        q = _ragged(rng, log_int(1, 24), 1, rng.choice([64, 1024, 12000]), total)
        k = [] if rng.random() < 0.6 else [log_int(1, rng.choice([200, 4000])) for _ in q]
        return dict(op=op, dtype=dtype, q=_text(q), k=_text(k), causal=rng.random() < 0.5, heads=heads, kv_heads=kv_heads,
                    head_dim=dh)
    if op == "paged":
        n = log_int(1, 64)
        new = _ragged(rng, n, 1, rng.choice([1, 1, 8, 600]), 2000)
        longest = log_int(64, 4000 if dtype == "f32" else 30000)
        kv = [max(x, log_int(1, longest)) for x in new]
        return dict(op=op, dtype=dtype, new=_text(new), kv=_text(kv), heads=heads, kv_heads=kv_heads, head_dim=dh,
                    page=rng.choice([16, 32, 64, 128, 256]), causal=rng.random() < 0.6, lse=rng.random() < 0.5)
    rows = _ragged(rng, log_int(1, 12), 1, rng.choice([4, 300, 8000]), 16000)
    d = 8 * log_int(8, 1024)
    while sum(rows) * d > 4 * 4096 * 1152:
        d = max(64, d // 16 * 8)
    return dict(op=op, dtype=dtype, rows=_text(rows), d=d, post=rng.choice(["none", "rms", "layer"]),
                pre=rng.choice(["rms", "layer"]), gate_tanh=rng.random() < 0.5, x_scale=rng.choice([1.0, 0.5]),
                modulate=rng.random() < 0.5)


# ---- inputs -----------------------------------------------------------------------------------------------------------
def _lengths(text, like=()):
    """Lengths from "a,b,c", or from "ragged:top": as many as `like`, spread over the logarithm of [1, top]."""
    if text == "zero":
        return [0] * len(like)
    if text.startswith("ragged:"):
        top = int(text[7:])
        rng = random.Random(top * 1000 + len(like))
        return [max(1, int(math.exp(rng.uniform(math.log(max(top // 256, 1)), math.log(top))))) for _ in like]
    return [int(x) for x in text.split(",")]


def _axes(case):
    return [int(x) for x in case["axes"].split(",")]


SCALING = dict(factor=8.0, low=1.0, high=4.0, original_len=8192)   # of the scaled cases


def _scaling(case):
    s = case["scaling"]
    mag = 0.1 * math.log(SCALING["factor"]) + 1.0 if s == "ramp_index" else 1.0
    return s, mag


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _cu(lengths):
    return _int32([0] + np.cumsum(lengths).tolist())


def _paged_inputs(case, gen, slots):
    """Pools with room for `slots` tokens of each sequence, pages in an arbitrary order, and the page table."""
    page, dh, hk, dt = case["page"], case["head_dim"], case["kv_heads"], DT[case["dtype"]]
    need = [(n + page - 1) // page for n in slots]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=gen, device="cuda").tolist()
    table = [[-1] * max(need) for _ in need]
    at = 0
    for s, n in enumerate(need):
        table[s][:n] = order[at:at + n]
        at += n
    k = torch.randn(n_pages, hk, page, dh, generator=gen, device="cuda", dtype=dt)
    v = torch.randn(n_pages, hk, page, dh, generator=gen, device="cuda", dtype=dt)
    return k, v, table


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DT[case["dtype"]]
    rand = lambda *shape, t=dt: torch.randn(*shape, generator=gen, device="cuda", dtype=t)
    st = dict(case=case)
    op = case["op"]
    if op in ("packed", "paged", "append"):
        h, hk, dh = case["heads"], case["kv_heads"], case["head_dim"]
    if op == "rope":
        n_axes = len(_axes(case))
        st["x"] = rand(case["tokens"], case["heads"] * case["head_dim"])
        st["pos"] = torch.randint(0, case["far"] + 1, (case["tokens"], n_axes), generator=gen, device="cuda", dtype=torch.int32)
    elif op == "append":
        new = _lengths(case["new"])
        first = _lengths(case["first"], new)
        st["qkv"] = rand(sum(new), (h + 2 * hk) * dh)
        st["k_pool"], st["v_pool"], st["table_host"] = _paged_inputs(case, gen, [f + n for f, n in zip(first, new)])
        st["new"], st["first_host"] = new, first
        slots = np.concatenate([np.arange(f, f + n) for f, n in zip(first, new)])
        # one axis: the slot itself; more: the slot as a place on a grid of 128 columns
        cols = [slots, slots // 128, slots % 128][:len(_axes(case))]
        st["pos"] = _int32(np.stack(cols, 1).tolist())
    elif op == "packed":
        nq = _lengths(case["q"])
        nk = _lengths(case["k"]) if case["k"] else nq
        st["nq"], st["nk"] = nq, nk
        st["q"], st["k"], st["v"] = rand(sum(nq), h * dh), rand(sum(nk), hk * dh), rand(sum(nk), hk * dh)
    elif op == "paged":
        new = _lengths(case["new"])
        kv = [max(n, m) for n, m in zip(new, _lengths(case["kv"], new))]
        st["new"], st["kv"] = new, kv
        # causal: the new tokens end the cache; full: a patch anywhere in it
        st["first_host"] = [m - n if case["causal"] else (m - n) // 2 for n, m in zip(new, kv)]
        st["q"] = rand(sum(new), h * dh)
        st["k_pool"], st["v_pool"], st["table_host"] = _paged_inputs(case, gen, kv)
    else:
        rows, d = _lengths(case["rows"]), case["d"]
        n = sum(rows)
        st["rows"] = rows
        st["y"], st["x"] = rand(n, d), rand(n, d, t=torch.float32)
        st["gate"] = rand(len(rows), d, t=torch.float32) * 0.5
        st["scale"] = rand(len(rows), d, t=torch.float32) * 0.3 if case["modulate"] else None
        st["shift"] = rand(len(rows), d, t=torch.float32) * 0.3 if case["modulate"] else None
        for side in ("post", "pre"):
            kind = case[side]
            st[side + "_w"] = (1.0 + 0.2 * rand(d, t=torch.float32)).to(dt) if kind != "none" else None
            st[side + "_b"] = (0.2 * rand(d, t=torch.float32)).to(dt) if kind == "layer" else None
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    st["own"] = own
    op = case["op"]
    if "table_host" in st:
        st["table"] = _int32(st["table_host"])
        st["first"] = _int32(st["first_host"])
        st["cu"] = _cu(st["new"])
    if op == "packed":
        st["cu_q"], st["cu_k"] = _cu(st["nq"]), _cu(st["nk"])
    if op == "paged":
        st["kv_len"] = _int32(st["kv"])
    if op == "norm":
        st["cu"] = _cu(st["rows"])
    if own:   # the handles a user's program keeps
        import paper_2405_14430_amd as pf
        st["pf"] = pf
        if op in ("rope", "append"):
            s, mag = _scaling(case)
            st["rope"] = pf.make_rope(_axes(case), layout=case["layout"], theta=case["theta"], scaling=s, magnitude=mag, **SCALING)
        if "table" in st:
            st["pages"] = pf.KvPages(st["k_pool"], st["v_pool"], st["table"])
        if op == "norm":
            for side in ("post", "pre"):
                st[side] = None if case[side] == "none" else pf.make_norm(case[side], st[side + "_w"], st[side + "_b"], eps=1e-6)
    return st


# ---- the library's operators ----------------------------------------------------------------------------------------------
def _run_own(st):
    c, pf = st["case"], st["pf"]
    op = c["op"]
    if op == "rope":
        return pf.pf_op_rope(st["x"], st["rope"], st["pos"], c["head_dim"])
    if op == "append":
        dh, h, hk = c["head_dim"], c["heads"], c["kv_heads"]
        q, k, v = st["qkv"].split((h * dh, hk * dh, hk * dh), dim=1)
        q_out = pf.pf_op_kv_append(st["pages"], k, v, st["cu"], st["first"], rope=st["rope"], pos=st["pos"], q=q)
        return q_out, st["k_pool"], st["v_pool"]
    if op == "packed":
        return pf.pf_op_attention_packed(st["q"], st["k"], st["v"], st["cu_q"], st["cu_k"], c["head_dim"], causal=c["causal"])
    if op == "paged":
        return pf.pf_op_attention_paged(st["q"], st["pages"], st["cu"], st["first"], st["kv_len"], causal=c["causal"],
                                        want_lse=c["lse"])
    return pf.pf_op_norm_residual(st["y"], st["x"], post=st["post"], pre=st["pre"], gate=st["gate"],
                                  gate_tanh=c["gate_tanh"], x_scale=c["x_scale"], scale=st["scale"], shift=st["shift"],
                                  cu=st["cu"])


# ---- the plain form --------------------------------------------------------------------------------------------------------
def _frequencies(width, theta, scaling):
    """Radians per position of the pairs of one axis (numpy, 64 bits)."""
    f, lo, hi, n0 = SCALING["factor"], SCALING["low"], SCALING["high"], SCALING["original_len"]
    i = np.arange(width // 2, dtype=np.float64)
    if scaling == "ntk" and width > 2:
        theta = theta * f ** (width / (width - 2))
    w = theta ** (-2.0 * i / width)
    if scaling == "linear":
        return w / f
    if scaling == "ramp_turns":      # pairs that turn often over the original length keep their frequency
        keep = np.clip((n0 * w / (2 * np.pi) - lo) / (hi - lo), 0, 1)
        return w * (keep + (1 - keep) / f)
    if scaling == "ramp_index":      # the same between two pair indexes
        at = lambda turns: width * math.log(n0 / (2 * math.pi * turns)) / (2 * math.log(theta))
        a, b = max(math.floor(at(hi)), 0), min(math.ceil(at(lo)), width - 1)
        r = np.clip((i - a) / max(b - a, 1e-3), 0, 1)
        return w * ((1 - r) + r / f)
    return w


def _plain_rope(x, pos, case, n_heads):
    """x [rows, n_heads * head_dim] of any type, rotated in 32 bits; angles in 64."""
    dh = case["head_dim"]
    scaling, mag = _scaling(case)
    y = x.float().reshape(x.shape[0], n_heads, dh).clone()
    at = 0
    for a, w in enumerate(_axes(case)):
        f = torch.from_numpy(_frequencies(w, case["theta"], scaling)).to(x.device)
        ang = pos[:, a].double()[:, None] * f
        cos, sin = (torch.cos(ang) * mag).float()[:, None], (torch.sin(ang) * mag).float()[:, None]
        part = y[:, :, at:at + w]
        if case["layout"] == "interleaved":
            p, q = part[..., 0::2].clone(), part[..., 1::2].clone()
            part[..., 0::2], part[..., 1::2] = p * cos - q * sin, p * sin + q * cos
        else:
            p, q = part[..., :w // 2].clone(), part[..., w // 2:].clone()
            part[..., :w // 2], part[..., w // 2:] = p * cos - q * sin, p * sin + q * cos
        at += w
    return y.reshape(x.shape).to(x.dtype)


def _plain_attention(q, k, v, heads, kv_heads, dh, last):
    """One sequence: q [n, heads*dh], k and v [m, kv_heads*dh]; query i sees keys [0, last[i]].  Out in 32 bits, and the
    log of the softmax denominators."""
    n, m, g = q.shape[0], k.shape[0], heads // kv_heads
    out = torch.zeros(n, heads, dh, device=q.device)
    lse = torch.full((n, heads), -math.inf, device=q.device)
    if n == 0 or m == 0:
        return out.reshape(n, heads * dh), lse
    hidden = torch.arange(m, device=q.device)[None, :] > last[:, None]
    empty = last < 0
    qf, kf, vf = (t.float().reshape(t.shape[0], -1, dh) for t in (q, k, v))
    for h in range(heads):
        s = torch.matmul(qf[:, h], kf[:, h // g].t().contiguous()) * (1.0 / math.sqrt(dh))
        s = s.masked_fill(hidden, -math.inf)
        top = s.amax(1, keepdim=True).masked_fill(empty[:, None], 0.0)
        p = torch.exp(s - top)
        total = p.sum(1, keepdim=True)
        out[:, h] = torch.matmul(p, vf[:, h // g].contiguous()) / total.masked_fill(empty[:, None], 1.0)
        lse[:, h] = (top + torch.log(total))[:, 0]
    return out.reshape(n, heads * dh), lse


def _gathered(st, pool, s):
    """Keys or values of sequence s of a paged pool, [kv_len, kv_heads * head_dim]."""
    page, m = st["case"]["page"], st["kv"][s]
    ids = st["table"][s, :(m + page - 1) // page].long()
    rows = pool[ids].permute(0, 2, 1, 3).reshape(len(ids) * page, -1)
    return rows[:m]


def _plain_norm(x, kind, w, b, eps=1e-6):
    if kind == "none":
        return x
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    x = x / torch.sqrt((x * x).mean(1, keepdim=True) + eps)
    x = x * w.float()
    return x if b is None else x + b.float()


def _run_plain(st):
    c = st["case"]
    op = c["op"]
    if op == "rope":
        return _plain_rope(st["x"], st["pos"], c, c["heads"])
    if op == "append":
        dh, h, hk, page = c["head_dim"], c["heads"], c["kv_heads"], c["page"]
        q, k, v = st["qkv"].split((h * dh, hk * dh, hk * dh), dim=1)
        q, k = _plain_rope(q, st["pos"], c, h), _plain_rope(k, st["pos"], c, hk)
        for s, n in enumerate(st["new"]):
            at = sum(st["new"][:s])
            slot = torch.arange(n, device=q.device) + st["first"][s]
            ids, rows = st["table"][s][slot // page].long(), slot % page
            st["k_pool"][ids, :, rows] = k[at:at + n].reshape(n, hk, dh)
            st["v_pool"][ids, :, rows] = v[at:at + n].reshape(n, hk, dh)
        return q, st["k_pool"], st["v_pool"]
    if op == "packed":
        outs, aq, ak = [], 0, 0
        for n, m in zip(st["nq"], st["nk"]):
            last = torch.arange(n, device="cuda") + (m - n) if c["causal"] else torch.full((n,), m - 1, device="cuda")
            outs.append(_plain_attention(st["q"][aq:aq + n], st["k"][ak:ak + m], st["v"][ak:ak + m], c["heads"],
                                         c["kv_heads"], c["head_dim"], last)[0])
            aq, ak = aq + n, ak + m
        return torch.cat(outs).to(st["q"].dtype)
    if op == "paged":
        outs, lses, at = [], [], 0
        for s, n in enumerate(st["new"]):
            m = st["kv"][s]
            last = torch.arange(n, device="cuda") + st["first"][s] if c["causal"] else torch.full((n,), m - 1, device="cuda")
            o, l = _plain_attention(st["q"][at:at + n], _gathered(st, st["k_pool"], s), _gathered(st, st["v_pool"], s),
                                    c["heads"], c["kv_heads"], c["head_dim"], last)
            outs.append(o)
            lses.append(l)
            at += n
        out = torch.cat(outs).to(st["q"].dtype)
        return (out, torch.cat(lses)) if c["lse"] else out
    seg = torch.repeat_interleave(torch.arange(len(st["rows"]), device="cuda"), torch.diff(st["cu"]).long())
    gate = torch.tanh(st["gate"]) if c["gate_tanh"] else st["gate"]
    x = c["x_scale"] * st["x"] + gate[seg] * _plain_norm(st["y"].float(), c["post"], st["post_w"], st["post_b"])
    h = _plain_norm(x, c["pre"], st["pre_w"], st["pre_b"])
    if c["modulate"]:
        h = h * (1.0 + st["scale"][seg]) + st["shift"][seg]
    return x, h.to(st["y"].dtype)


def run(state):
    return _run_own(state) if state["own"] else _run_plain(state)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------
def work(case):
    op, e = case["op"], ESZ[case["dtype"]]
    if op == "rope":
        n = case["tokens"] * case["heads"] * case["head_dim"]
        return {"bytes": 2 * n * e + 4 * case["tokens"] * len(_axes(case)), "flops": 3 * n}
    if op == "append":
        t = sum(_lengths(case["new"]))
        h, hk, dh = case["heads"], case["kv_heads"], case["head_dim"]
        return {"bytes": 2 * t * (h + 2 * hk) * dh * e + 4 * t * len(_axes(case)), "flops": 3 * t * (h + hk) * dh}
    if op in ("packed", "paged"):
        h, hk, dh = case["heads"], case["kv_heads"], case["head_dim"]
        if op == "packed":
            nq = _lengths(case["q"])
            nk = _lengths(case["k"]) if case["k"] else nq
            seqs = [(n, m, m - n) for n, m in zip(nq, nk)]
        else:
            nq = _lengths(case["new"])
            seqs = [(n, max(n, m), max(n, m) - n) for n, m in zip(nq, _lengths(case["kv"], nq))]
        pairs = keys = 0
        for n, m, first in seqs:
            if case["causal"]:   # query i sees first + i + 1 keys, none if that is not positive
                a = max(first + 1, 0)
                pairs += (a + first + n) * (first + n - a + 1) // 2 if first + n >= a else 0
                keys += max(min(m, first + n), 0)
            else:
                pairs += n * m
                keys += m if n else 0
        rows = sum(nq)
        extra = 4 * rows * h if case.get("lse") else 0
        return {"bytes": 2 * rows * h * dh * e + 2 * keys * hk * dh * e + extra, "flops": 4 * pairs * h * dh}
    n, d = sum(_lengths(case["rows"])), case["d"]
    return {"bytes": n * d * (2 * e + 8) + 4 * d * len(_lengths(case["rows"])) * (3 if case["modulate"] else 1), "flops": 12 * n * d}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------
def _exact_rotation(x, pos, case):
    """x [rows, heads, head_dim] in 64 bits: each pair as a complex number times m e^(i angle)."""
    scaling, mag = _scaling(case)
    cols, at = [], 0
    for a, w in enumerate(_axes(case)):
        part = x[:, :, at:at + w]
        z = part.reshape(*part.shape[:2], w // 2, 2) if case["layout"] == "interleaved" else \
            part.reshape(*part.shape[:2], 2, w // 2).transpose(2, 3)
        z = torch.complex(z[..., 0].contiguous(), z[..., 1].contiguous())
        f = torch.tensor(_frequencies(w, case["theta"], scaling).tolist(), dtype=torch.float64, device=x.device)
        ang = torch.outer(pos[:, a].to(torch.float64), f)
        z = z * torch.polar(torch.full_like(ang, mag), ang)[:, None, :]
        pair = (z.real, z.imag)
        cols.append(torch.stack(pair, -1).flatten(2) if case["layout"] == "interleaved" else torch.cat(pair, -1))
        at += w
    cols.append(x[:, :, at:])
    return torch.cat(cols, -1)


def _exact_attention(q, k, v, first):
    """q [n, H, d], k and v [m, Hk, d] in 64 bits; query i sees keys up to first + i (first None: all)."""
    n, H, d = q.shape
    m, hk = k.shape[0], k.shape[1]
    out, lse = torch.zeros_like(q), torch.full((n, H), -math.inf, dtype=torch.float64, device=q.device)
    for h in range(H):
        kh, vh = k[:, h * hk // H], v[:, h * hk // H]
        for a in range(0, n, 2048):
            b = min(n, a + 2048)
            top = m if first is None else min(m, first + b)
            if top <= 0:
                continue
            s = q[a:b, h] @ kh[:top].t() / math.sqrt(d)
            if first is not None:
                i = torch.arange(a, b, device=q.device)[:, None]
                s.masked_fill_(torch.arange(top, device=q.device)[None] > i + first, -math.inf)
            l = torch.logsumexp(s, 1)
            lse[a:b, h] = l
            w = torch.exp(s - torch.where(torch.isinf(l), torch.zeros_like(l), l)[:, None])
            out[a:b, h] = w @ vh[:top]
    return out.reshape(n, H * d), lse


def exact(case, seed):
    st = _inputs(case, seed)
    op = case["op"]
    if op == "rope":
        x = st["x"].double().reshape(case["tokens"], case["heads"], case["head_dim"])
        return _exact_rotation(x, st["pos"], case).reshape(st["x"].shape)
    if op in ("append", "packed", "paged"):
        H, hk, dh = case["heads"], case["kv_heads"], case["head_dim"]
    if op == "append":
        page, t = case["page"], sum(st["new"])
        x = st["qkv"].double().reshape(t, H + 2 * hk, dh)
        rot = _exact_rotation(x[:, :H + hk], st["pos"], case)
        pages, rows = [], []
        for s, (f, n) in enumerate(zip(st["first_host"], st["new"])):
            for slot in range(f, f + n):
                pages.append(st["table_host"][s][slot // page])
                rows.append(slot % page)
        pages, rows = torch.tensor(pages, device="cuda"), torch.tensor(rows, device="cuda")
        kp, vp = st["k_pool"].double(), st["v_pool"].double()
        kp[pages, :, rows], vp[pages, :, rows] = rot[:, H:], x[:, H + hk:]
        return rot[:, :H].reshape(t, H * dh), kp, vp
    if op in ("packed", "paged"):
        outs, lses = [], []
        q = st["q"].double().reshape(-1, H, dh)
        aq = ak = 0
        for s, n in enumerate(st["nq"] if op == "packed" else st["new"]):
            if op == "packed":
                m = st["nk"][s]
                k, v = (st[x][ak:ak + m].double().reshape(m, hk, dh) for x in ("k", "v"))
                first = m - n
                ak += m
            else:
                m, page = st["kv"][s], case["page"]
                ids = torch.tensor(st["table_host"][s], device="cuda")[torch.arange(m, device="cuda") // page]
                at = torch.arange(m, device="cuda") % page
                k, v = st["k_pool"][ids, :, at].double(), st["v_pool"][ids, :, at].double()
                first = st["first_host"][s]
            o, l = _exact_attention(q[aq:aq + n], k, v, first if case["causal"] else None)
            outs.append(o)
            lses.append(l)
            aq += n
        return (torch.cat(outs), torch.cat(lses)) if case.get("lse") else torch.cat(outs)
    d = case["d"]

    def normed(x, side):
        if case[side] == "none":
            return x
        mean = x.mean(-1, keepdim=True) if case[side] == "layer" else 0.0
        y = (x - mean) * torch.rsqrt(((x - mean) ** 2).sum(-1, keepdim=True) / d + 1e-6) * st[side + "_w"].double()
        return y + st[side + "_b"].double() if st[side + "_b"] is not None else y

    xs, hs, at = [], [], 0
    for i, n in enumerate(st["rows"]):
        g = st["gate"][i].double()
        x = case["x_scale"] * st["x"][at:at + n].double() + (torch.tanh(g) if case["gate_tanh"] else g) * \
            normed(st["y"][at:at + n].double(), "post")
        h = normed(x, "pre")
        if case["modulate"]:
            h = h * (1 + st["scale"][i].double()) + st["shift"][i].double()
        xs.append(x)
        hs.append(h)
        at += n
    return torch.cat(xs), torch.cat(hs)
