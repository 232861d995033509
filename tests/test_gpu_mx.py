"""The operators around a cache in 8 or 4 bits against their plain 64-bit forms (tests/mx_ref.py)."""
import ctypes as C
import math

import pytest
import torch

import mx_ref as M
import requests_ref as R
from paper_2405_14430_amd import (KvMxPages, KvPages, PfError, load_library, make_norm, make_rope, pf_op_attention_mx, pf_op_attention_paged,
                                  pf_op_kv_append_mx, pf_op_kv_read_mx, pf_op_qk_norm_rope)
from test_gpu_requests import BF16, CANARY, F32, PAGED, ROPES, cu, dev, ints, make, rope_args, wide

pytestmark = pytest.mark.gpu


def norm_of(kind, dh, dtype, seed, eps=1e-5):
    """(norm for the call, arguments for the plain form)"""
    if kind == "none":
        return None, ("none", None, None, 0.0)
    w = (1 + 0.3 * dev(dh, dtype=F32, seed=seed)).to(dtype) if kind != "rms-bare" else None
    b = (0.3 * dev(dh, dtype=F32, seed=seed + 1)).to(dtype) if kind in ("layer", "rms-bias") else None
    kind = kind.split("-")[0]
    return make_norm(kind, w, b, eps=eps), (kind, w, b, eps)


def positions(rows, r, far=4096, seed=1):
    return torch.randint(-far, far + 1, (rows, len(r["axes"])), generator=torch.Generator().manual_seed(seed), dtype=torch.int32).cuda()


# ---- norm and rotation -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("tokens,heads,kv_heads,q_kind,k_kind", [(1, 1, 1, "rms", "rms"), (37, 5, 2, "layer", "rms-bare"),
                                                                 (130, 7, 7, "rms-bias", "none"), (4099, 3, 1, "rms", "layer")])
@pytest.mark.parametrize("r", ROPES, ids=lambda r: f"{r['axes']}-{r['layout']}")
def test_qk_norm_rope(r, tokens, heads, kv_heads, q_kind, k_kind, dtype):
    dh = r["head_dim"]
    x = wide(tokens, (heads + kv_heads) * dh, dtype, seed=tokens)
    q, k = x.split((heads * dh, kv_heads * dh), dim=1)
    pos = positions(tokens, r)
    (qn, q_plain), (kn, k_plain) = norm_of(q_kind, dh, dtype, 7), norm_of(k_kind, dh, dtype, 9)
    out = torch.full((tokens, heads * dh + 8), CANARY, dtype=dtype, device="cuda")
    q_out, k_out = pf_op_qk_norm_rope(q, k, dh, q_norm=qn, k_norm=kn, rope=make(r), pos=pos, q_out=out[:, :heads * dh])
    for got, src, plain, what in ((q_out, q, q_plain, "q"), (k_out, k, k_plain, "k")):
        want, bound = M.turn(src, dh, plain, pos, rope_args(r))
        R.check(got, want, R.stored(bound, want, dtype), what)
    assert (out[:, heads * dh:] == CANARY).all()
    # one side alone, and in place
    alone, none = pf_op_qk_norm_rope(q, None, dh, q_norm=qn, rope=make(r), pos=pos)
    assert none is None and torch.equal(alone, q_out)
    none, alone = pf_op_qk_norm_rope(None, k, dh, k_norm=kn, rope=make(r), pos=pos)
    assert none is None and torch.equal(alone, k_out)
    pf_op_qk_norm_rope(q, k, dh, q_norm=qn, k_norm=kn, rope=make(r), pos=pos, q_out=q, k_out=k)
    assert torch.equal(q, q_out) and torch.equal(k, k_out)


@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("dh", [8, 40, 64, 72, 80, 96, 104, 120, 128])
def test_norm_without_rotation(dh, dtype):
    q, k = wide(21, 3 * dh, dtype, 1), dev(21, 2 * dh, dtype=dtype, seed=2)
    k[3], k[4, :dh] = 0.0, 3.0            # a row of zeros, a head without variance
    (qn, q_plain), (kn, k_plain) = norm_of("rms", dh, dtype, 3), norm_of("layer", dh, dtype, 5)
    for got, src, plain in zip(pf_op_qk_norm_rope(q, k, dh, q_norm=qn, k_norm=kn), (q, k), (q_plain, k_plain)):
        want, bound = M.turn(src, dh, plain)
        R.check(got, want, R.stored(bound, want, dtype), plain[0])
    got = pf_op_qk_norm_rope(q, k, dh)    # nothing asked for: the rows themselves
    assert torch.equal(got[0], q) and torch.equal(got[1], k)


def test_channels_behind_the_axes_keep_to_themselves():
    """Infinities and NaN behind the axes pass, and reach no other channel, without a norm."""
    x = dev(4, 64, dtype=F32)
    x[:, 40], x[:, 63] = math.inf, math.nan
    for layout in ("interleaved", "half"):
        r = dict(axes=(10,), head_dim=64, layout=layout, theta=1e4)
        pos = ints(5, -7, 0, 1)
        want, bound = R.rope(x, pos, **r)
        R.check(pf_op_qk_norm_rope(x, None, 64, rope=make(r), pos=pos)[0], want, bound + 1e-30, layout)


# ---- the way into the pages and back --------------------------------------------------------------------------------------------
def check_written(pages, which, s, first, rows, dh):
    """Slots first .. of sequence s hold exactly what `rows` [n, kv_heads * dh] (their type's values) are coded as, padding zero."""
    codes, exps = M.encode(R.d64(rows).unflatten(1, (-1, dh)), pages.format)
    want = M.packed(codes, pages.format, dh)
    code, exp, table = getattr(pages, which).cpu(), getattr(pages, which + "_scale").cpu(), pages.table.cpu()
    for i in range(rows.shape[0]):
        pg, at = int(table[s, (first + i) // pages.page_size]), (first + i) % pages.page_size
        assert torch.equal(exp[pg, :, at].long(), exps[i]), (which, s, i)
        assert torch.equal(code[pg, :, at], want[i]), (which, s, i)


APPENDS = [
    # page, heads, kv_heads, new, first, rotation, norms
    (16, 8, 2, [1] * 5, [0, 15, 16, 31, 40], 0, "rms"),
    (32, 4, 4, [33, 0, 7, 64], [5, 3, 30, 0], 3, "none"),
    (64, 6, 3, [130, 1], [0, 200], 6, "layer"),
    (256, 0, 1, [300], [17], 4, "rms"),
    (16, 3, 1, [4200, 50], [0, 7], 5, "rms-bias"),
    (16, 2, 5, [40], [3], 7, "rms"),
    (32, 1, 2, [40, 3], [3, 9], 8, "layer"),
    (1024, 5, 3, [9], [1020], 10, "rms"),
]


@pytest.mark.parametrize("fmt", M.FORMATS)
@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("page,heads,kv_heads,new,first,ri,kind", APPENDS)
def test_append(page, heads, kv_heads, new, first, ri, kind, dtype, fmt):
    """The pages get exactly the codes of the rows that pf_op_qk_norm_rope gives, of v's rows, and nothing else; the way back is exact."""
    r = ROPES[ri]
    dh = r["head_dim"]
    tokens, lead, tail = sum(new), 2, 3
    rows = lead + tokens + tail
    pages = M.make_pages(fmt, kv_heads, dh, page, [(f + n + page - 1) // page for f, n in zip(first, new)], fill=0x5b, gap=48)
    qkv = dev(rows, (heads + 2 * kv_heads) * dh, dtype=dtype, seed=3)
    q, k, v = qkv.split((heads * dh, kv_heads * dh, kv_heads * dh), dim=1)
    q = q if heads else None
    pos = positions(rows, r, 500)
    (qn, _), (kn, _) = norm_of(kind, dh, dtype, 7), norm_of(kind, dh, dtype, 9)
    want_q, want_k = pf_op_qk_norm_rope(q, k, dh, q_norm=qn, k_norm=kn, rope=make(r), pos=pos)
    q_out = torch.full((rows, heads * dh), CANARY, dtype=dtype, device="cuda") if heads else None
    got = pf_op_kv_append_mx(pages, k, v, cu(new, lead), ints(*first), k_norm=kn, rope=make(r), pos=pos, q=q, q_norm=qn, q_out=q_out)
    written = torch.zeros(pages.k.shape[0], page, dtype=torch.bool)
    at = lead
    for s, (n, f) in enumerate(zip(new, first)):
        check_written(pages, "k", s, f, want_k[at:at + n], dh)
        check_written(pages, "v", s, f, v[at:at + n], dh)
        for t in range(f, f + n):
            written[int(pages.table[s, t // page]), t % page] = True
        at += n
    for pool in (pages.k, pages.v, pages.k_scale, pages.v_scale):
        assert (pool.cpu().permute(0, 2, 1, 3)[~written] == 0x5b).all()
    if heads:
        assert torch.equal(got[lead:at], want_q[lead:at]) and (got[:lead] == CANARY).all() and (got[at:] == CANARY).all()
    else:
        assert got is None
    for out in R.DTYPES:
        k_back, v_back = (torch.full((rows, kv_heads * dh + 8), CANARY, dtype=out, device="cuda") for _ in range(2))
        cut = slice(0, kv_heads * dh)
        pf_op_kv_read_mx(pages, cu(new, lead), ints(*first), rows, out, k_out=k_back[:, cut], v_out=v_back[:, cut])
        at = lead
        for s, (n, f) in enumerate(zip(new, first)):
            for back, which in ((k_back, "k"), (v_back, "v")):
                assert torch.equal(R.d64(back[at:at + n, cut]), M.slot_rows(pages, which, s, f + n)[0][f:]), (which, s, out)
            at += n
        for back in (k_back, v_back):
            assert (back[:lead] == CANARY).all() and (back[at:] == CANARY).all() and (back[:, kv_heads * dh:] == CANARY).all()


def hard_rows(dtype):
    """Rows of 72 channels with what a code can go wrong at: zeros, infinities, NaN, ties, both ends of the range, one large channel."""
    x = torch.randn(40, 72, generator=torch.Generator().manual_seed(5))
    x[0] = 0.0
    x[1, 5], x[2, 40], x[3, 71], x[4] = math.inf, -math.inf, math.nan, math.nan
    x[5, :32] = torch.arange(32) * 14.0 + 3.5              # ties of e4m3 among them, largest 437.5
    x[6, :32] = torch.linspace(-6, 6, 32)
    x[7, :8] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])   # every tie of e2m1
    x[7, 8:32] = 0.0
    x[8], x[9] = x[8] * 2.0 ** -130, x[9] * 2.0 ** 126
    x[10, :32], x[11, :32] = 3.38e38, -3.38e38
    x[12], x[12, 3] = x[12] * 1e-3, 1e4
    x[13, :32], x[14, :32] = 448.0, 6.0
    x[15, 0], x[15, 1:32] = 448.0 + 2, 1.0                  # just past the largest: the next exponent
    x[16, 0], x[16, 1:32] = 6.03125, 1.0
    x[17] = -0.0
    x[18, 64:] = torch.tensor([1.0, -2.0, 3.0, -4.0, 5.0, -6.0, 7.0, -8.0])
    x[19, :32] = 2.0 ** -126
    x[20, 0], x[20, 1:32] = 1.0, 2.0 ** -10                 # e4m3: a tie between the smallest number and none
    return x.to(dtype)


@pytest.mark.parametrize("fmt", M.FORMATS)
@pytest.mark.parametrize("dtype", R.DTYPES)
def test_append_of_hard_rows(dtype, fmt):
    x = hard_rows(dtype).cuda()
    pages = M.make_pages(fmt, 1, 72, 16, [3], fill=0x5b)
    pf_op_kv_append_mx(pages, x, x.flip(0).contiguous(), cu([40]), ints(0))
    check_written(pages, "k", 0, 0, x, 72)
    check_written(pages, "v", 0, 0, x.flip(0), 72)
    k, v = pf_op_kv_read_mx(pages, cu([40]), ints(0), 40, dtype)
    want = M.slot_rows(pages, "k", 0, 40)[0]
    assert torch.equal(R.d64(k).nan_to_num(7.5), want.nan_to_num(7.5)) and torch.equal(k.isnan().cpu(), want.isnan())
    fine = torch.isfinite(x)
    assert not torch.isfinite(k[1, :32]).any() and torch.isfinite(k[1, 32:]).all() and torch.isfinite(k[fine.all(1)]).all()


@pytest.mark.parametrize("fmt", M.FORMATS)
@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("dh", range(8, 136, 8))
def test_append_of_blocks_of_every_length(dh, dtype, fmt):
    """A block's largest number, an infinity or a NaN in each unit of eight channels in turn: all codes of the block go by it, also where the last
    block of a head has one, two or three units."""
    units, heads = dh // 8, 5
    x = torch.randn(4 * units, heads, dh, generator=torch.Generator().manual_seed(dh))
    for u in range(units):
        x[u, :, 8 * u + u % 8] = -300.0
        x[units + u, ::2, 8 * u + 7 - u % 8] = 2.0 ** 40
        x[2 * units + u, u % heads, 8 * u + 3] = math.inf
        x[3 * units + u, u % heads, 8 * u + 5] = math.nan
    x = x.flatten(1).to(dtype)
    k, v = x.cuda(), x.flip(0).contiguous().cuda()
    n = len(x)
    pages = M.make_pages(fmt, heads, dh, 16, [(n + 15) // 16], fill=0x5b)
    pf_op_kv_append_mx(pages, k, v, cu([n]), ints(0))
    check_written(pages, "k", 0, 0, k, dh)
    check_written(pages, "v", 0, 0, v, dh)


@pytest.mark.parametrize("fmt", M.FORMATS)
def test_every_bf16_value_is_coded_and_read_back(fmt):
    """All finite bf16 numbers, alone in their blocks and beside a large one."""
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(BF16)
    x = x[torch.isfinite(x)]
    rows = torch.zeros(len(x), 64, dtype=BF16)
    rows[:, 0] = rows[:, 33] = x
    rows[:, 32] = 100.0
    rows = rows.cuda()
    pages = M.make_pages(fmt, 1, 64, 1024, [(len(x) + 1023) // 1024], fill=0)
    pf_op_kv_append_mx(pages, rows, rows, cu([len(x)]), ints(0))
    codes, exps = M.encode(R.d64(rows).unflatten(1, (1, 64)), fmt)
    want = M.packed(codes, fmt, 64)
    ids = pages.table[0].long()
    for pool in (pages.k, pages.v):
        assert torch.equal(pool[ids].transpose(1, 2).reshape(-1, 1, want.shape[-1])[:len(x)].cpu(), want)
    assert torch.equal(pages.k_scale[ids].transpose(1, 2).reshape(-1, 1, 2)[:len(x)].cpu().long(), exps)
    k, _ = pf_op_kv_read_mx(pages, cu([len(x)]), ints(0), len(x), BF16)
    assert torch.equal(R.d64(k), M.decode(want, exps.to(torch.uint8), fmt, 64).flatten(1))


@pytest.mark.parametrize("fmt", M.FORMATS)
def test_rows_without_a_place(fmt):
    """Negative slots, slots past the table and table entries that are no page: nothing is written, and zeros are read."""
    pages = M.make_pages(fmt, 1, 64, 16, [2, 2, 2], fill=0x5b)
    t = pages.table
    t[1, 0], t[1, 1] = -5, pages.k.shape[0]
    k, v = dev(60, 64, seed=1), dev(60, 64, seed=2)
    first = ints(-4, 6, 2 ** 31 - 5)
    pf_op_kv_append_mx(pages, k, v, cu([20, 20, 20]), first)
    check_written(pages, "k", 0, 0, k[4:20], 64)
    keep = torch.ones(pages.k.shape[0], dtype=torch.bool)
    keep[int(t[0, 0])] = False
    for pool in (pages.k, pages.v, pages.k_scale, pages.v_scale):
        assert (pool[keep.cuda()] == 0x5b).all()
    assert (pages.k[int(t[0, 1])] == 0x5b).all()
    k_back, v_back = pf_op_kv_read_mx(pages, cu([20, 20, 20]), first, 60, F32)
    assert torch.equal(R.d64(k_back[4:20]), M.slot_rows(pages, "k", 0, 16)[0])
    for back in (k_back, v_back):
        assert (back[:4] == 0).all() and (back[20:] == 0).all()


@pytest.mark.parametrize("fmt", M.FORMATS)
@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("tokens,kv_heads,dh", [(1, 1, 8), (37, 3, 72), (1, 40, 128), (1500, 8, 64), (2047, 1, 40), (2048, 5, 128), (3001, 40, 72),
                                                (5003, 1, 64)])
def test_read_of_one_side(tokens, kv_heads, dh, dtype, fmt):
    """k alone and v alone: what the read of both gives, and nothing where no row belongs to a sequence."""
    page = 64
    pages = M.make_pages(fmt, kv_heads, dh, page, [(tokens + page - 1) // page + 1], spare=1)
    if tokens > page:
        pages.table[0, 1] = -1
    where = (cu([tokens], 2), ints(5), tokens + 5, dtype)
    new = lambda: torch.full((tokens + 5, kv_heads * dh), CANARY, dtype=dtype, device="cuda")
    k, v = pf_op_kv_read_mx(pages, *where, k_out=new(), v_out=new())
    for s, which in ((k, "k"), (v, "v")):
        assert torch.equal(R.d64(s[2:2 + min(tokens, 50)]), M.slot_rows(pages, which, 0, min(tokens, 50) + 5)[0][5:])
    alone, none = pf_op_kv_read_mx(pages, *where, k_out=new(), want_v=False)
    assert none is None and torch.equal(alone, k)
    none, alone = pf_op_kv_read_mx(pages, *where, v_out=new(), want_k=False)
    assert none is None and torch.equal(alone, v)
    assert not torch.equal(k, v) and all((x[:2] == CANARY).all() and (x[-3:] == CANARY).all() for x in (k, v))
    alone, none = pf_op_kv_read_mx(pages, *where, want_v=False)
    assert none is None and torch.equal(alone[2:-3], k[2:-3])
    for wrong in (dict(want_k=False, want_v=False), dict(want_k=False, k_out=new()), dict(want_v=False, v_out=new())):
        with pytest.raises(PfError) as e:
            pf_op_kv_read_mx(pages, *where, **wrong)
        assert e.value.status == -1


@pytest.mark.parametrize("fmt", M.FORMATS)
def test_read_of_every_code_under_every_power(fmt):
    """All bytes of codes under all bytes of exponents, also those that append never writes: infinities past the largest number, numbers below the
    smallest normal one, NaN."""
    codes = torch.arange(256).view(-1, 1, 64) if fmt == "e4m3" else (torch.arange(64) % 16).view(1, 1, 64)
    rows = len(codes) * 256
    code = M.packed(codes, fmt, 64).repeat(256, 1, 1)
    exp = torch.arange(256).to(torch.uint8).repeat_interleave(len(codes)).view(-1, 1, 1).repeat(1, 1, 2)
    pool = lambda t: t.unflatten(0, (-1, 16)).transpose(1, 2).contiguous().cuda()
    pages = KvMxPages(fmt, pool(code), pool(code), pool(exp), pool(exp), torch.arange(rows // 16).int().cuda()[None], 64)
    want = M.decode(code, exp, fmt, 64).flatten(1)
    for dtype in R.DTYPES:
        for got in pf_op_kv_read_mx(pages, cu([rows]), ints(0), rows, dtype):
            got, near = R.d64(got), R.d64(want.to(dtype))
            assert torch.equal(got.isnan(), near.isnan()) and torch.equal(got.nan_to_num(7.5), near.nan_to_num(7.5))
            assert torch.equal(torch.signbit(got)[~got.isnan()], torch.signbit(near)[~got.isnan()])


# ---- attention ---------------------------------------------------------------------------------------------------------------
MANY = [
    # as PAGED, with rows for the kernels of many rows
    (128, 4, 2, 64, [600, 900], [500, 0], None, True),
    (64, 6, 6, 32, [1100, 40], [0, 0], [1300, 700], False),
    (72, 4, 4, 16, [900], [333], None, True),
    (96, 8, 2, 128, [700], [0], None, True),
    (80, 4, 4, 64, [800, 1], [0, 3], [1000, 5], False),
    (128, 8, 1, 16, [3], [5000], None, True),
    (40, 2, 1, 16, [33, 70], [10, 90], None, True),
]


@pytest.mark.parametrize("fmt", M.FORMATS)
@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("dh,heads,kv_heads,page,new,first,kv,causal", PAGED + MANY)
def test_attention(dh, heads, kv_heads, page, new, first, kv, causal, dtype, fmt):
    kv = [f + n for f, n in zip(first, new)] if kv is None else kv
    lead = 1
    pages = M.make_pages(fmt, kv_heads, dh, page, [(n + page - 1) // page for n in kv], gap=16)
    used = torch.zeros(pages.k.shape[0], page, dtype=torch.bool)       # the rest is not read: NaN
    for s, n in enumerate(kv):
        for t in range(n):
            used[int(pages.table[s, t // page]), t % page] = True
    for pool in (pages.k, pages.v, pages.k_scale, pages.v_scale):
        pool.permute(0, 2, 1, 3)[~used.cuda()] = 255
    tq = sum(new) + lead + 2
    q = wide(tq, heads * dh, dtype, 4)
    out = torch.full((tq, heads * dh), CANARY, dtype=dtype, device="cuda")
    got, lse = pf_op_attention_mx(q, pages, cu(new, lead), ints(*first), ints(*kv), causal=causal, out=out, want_lse=True)
    at = lead
    for s, n in enumerate(new):
        k, have = M.slot_rows(pages, "k", s, kv[s])
        v, _ = M.slot_rows(pages, "v", s, kv[s])
        last = (torch.arange(n) + first[s] + 1).clamp(max=kv[s]) if causal else torch.full((n,), kv[s])
        want, want_lse, b16, b32, bl = R.attention(q[at:at + n], k, v, dh, last, present=have)
        R.check(got[at:at + n], want, R.stored(b16 if dtype == BF16 else b32, want, dtype), ("out", s))
        R.check(lse[at:at + n], want_lse, bl + 4 * R.U * want_lse.abs().nan_to_num(posinf=0.0), ("lse", s))
        at += n
    assert (got[:lead] == CANARY).all() and (got[at:] == CANARY).all()


@pytest.mark.parametrize("fmt", M.FORMATS)
@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("new,causal", [([1, 1], True), ([40, 150], False), ([40, 150], True)])
def test_attention_missing_pages_and_long_lengths(new, causal, dtype, fmt):
    pages = M.make_pages(fmt, 2, 64, 16, [14, 14])
    t = pages.table
    t[0, 3], t[0, 4], t[1, 0], t[1, 13] = -1, pages.k.shape[0], -2 ** 31, 2 ** 31 - 1
    first, m = [200 - new[0], 224 - new[1]], 224
    q = dev(sum(new), 4 * 64, dtype=dtype, seed=2)
    got = pf_op_attention_mx(q, pages, cu(new), ints(*first), ints(10 ** 9, 14 * 16), causal=causal)
    at = 0
    for s, n in enumerate(new):
        k, have = M.slot_rows(pages, "k", s, m)
        v, _ = M.slot_rows(pages, "v", s, m)
        last = (torch.arange(n) + first[s] + 1).clamp(max=m) if causal else torch.full((n,), m)
        want, _, b16, b32, _ = R.attention(q[at:at + n], k, v, 64, last, present=have)
        R.check(got[at:at + n], want, R.stored(b16 if dtype == BF16 else b32, want, dtype), s)
        at += n
    pages.table.fill_(-1)
    got, lse = pf_op_attention_mx(q, pages, cu(new), ints(*first), ints(m, m), causal=causal, want_lse=True)
    assert (got == 0).all() and (lse == -math.inf).all()


def decoded_pages(pages, dtype):
    values = lambda which: M.decode(getattr(pages, which), getattr(pages, which + "_scale"), pages.format, pages.head_dim).to(dtype).cuda()
    return KvPages(values("k"), values("v"), pages.table)


@pytest.mark.parametrize("fmt", M.FORMATS)
@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("dh,heads,kv_heads,new,first", [(64, 2, 2, [70], [40]), (128, 8, 1, [5], [300]), (128, 4, 2, [900], [30]),
                                                         (96, 8, 8, [600], [0]), (72, 3, 1, [33, 9], [0, 500])])
def test_attention_over_anything_that_the_mask_hides(dh, heads, kv_heads, new, first, dtype, fmt):
    """Bytes of any value, NaN blocks and powers that overflow among them, in slots from the first row's on: they reach the rows that see
    them, as over pages of rows, and no others."""
    kv = [f + n for f, n in zip(first, new)]
    pages = M.make_pages(fmt, kv_heads, dh, 16, [(n + 15) // 16 for n in kv])
    g = torch.Generator().manual_seed(3)
    for s, (f, n) in enumerate(zip(first, new)):
        for t in range(f, f + n):
            pg, at = int(pages.table[s, t // 16]), t % 16
            kind = int(torch.randint(0, 12, (1,), generator=g))
            if kind == 0:        # a NaN block in v
                pages.v_scale[pg, :, at, 0] = 255
            elif kind == 1:      # finite codes that a large power takes past the largest bf16 number
                pages.v_scale[pg, :, at, -1] = 254
            elif kind == 2 and fmt == "e4m3":
                pages.v[pg, :, at, 3], pages.v[pg, 0, at, 5] = 0x7f, 0xff
            elif kind == 3 and t > f + n // 2:
                pages.k_scale[pg, :, at] = 255
    q = dev(sum(new), heads * dh, dtype=dtype, seed=9)
    got, lse = pf_op_attention_mx(q, pages, cu(new), ints(*first), ints(*kv), causal=True, want_lse=True)
    want, want_lse = pf_op_attention_paged(q, decoded_pages(pages, dtype), cu(new), ints(*first), ints(*kv), causal=True, want_lse=True)
    for a, b, rel in ((got, want, 2.0 ** -6 if dtype == BF16 else 1e-4), (lse, want_lse, 1e-4)):
        assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.isinf(), b.isinf())
        ok = torch.isfinite(b)
        assert ok.any() and not ok.all()
        assert torch.equal(a[b.isinf()], b[b.isinf()])
        assert ((a[ok] - b[ok]).abs() <= rel * (b[ok].abs() + 1)).all()


SAME = [
    # type, head_dim, heads, kv_heads, page, new lengths, first slots, causal, kernel, in chunks
    (BF16, 64, 4, 4, 16, [100, 3, 0, 41], [2000, 0, 5, 17], True, "attn_rows_kernel<bf16,64,1,4>", True),
    (BF16, 128, 8, 2, 64, [9, 60], [300, 70], True, "attn_rows_kernel<bf16,128,1,4>", False),
    (BF16, 72, 16, 2, 16, [40], [0], True, "attn_rows_kernel<bf16,96,1,4>", False),
    (BF16, 56, 4, 4, 32, [800, 330, 0], [3300, 11, 5], False, "attn_rows_kernel<bf16,64,4,1>", True),
    (BF16, 64, 16, 16, 32, [2500, 500, 7], [0, 300, 2], True, "attn_rows_wide_kernel<64,4>", False),
    (BF16, 72, 32, 4, 16, [777, 240, 13], [100, 0, 330], False, "attn_rows_wide_kernel<96,5>", False),
    (BF16, 96, 16, 4, 128, [1500, 90], [33, 0], True, "attn_rows_wide_kernel<96,6>", False),
    (BF16, 128, 14, 2, 64, [700, 77], [1300, 0], True, "attn_rows_wide_kernel<128,8>", True),
    (F32, 96, 8, 1, 16, [1, 2, 5], [2990, 0, 700], True, "attn_rows_kernel<float,96,1,4>", True),
    (F32, 64, 4, 4, 32, [90, 3], [0, 77], False, "attn_rows_kernel<float,64,1,4>", False),
    (F32, 72, 32, 4, 16, [777, 240, 13], [100, 0, 330], True, "attn_rows_kernel<float,96,4,1>", False),
]


@pytest.mark.parametrize("fmt", M.FORMATS)
@pytest.mark.parametrize("dtype,dh,heads,kv_heads,page,new,first,causal,name,chunks", SAME, ids=lambda v: v if isinstance(v, str) else None)
def test_kernels_of_pages_of_rows_give_the_same_bits(dtype, dh, heads, kv_heads, page, new, first, causal, name, chunks, fmt):
    """The tile, key and wide kernels over pages of few bits: bit for bit what they give over pages of rows that hold the decoded values, with pages
    missing, and bytes of all kinds where the causal mask hides them from some rows."""
    kv = [f + n for f, n in zip(first, new)]
    pages = M.make_pages(fmt, kv_heads, dh, page, [(n + page - 1) // page for n in kv])
    if kv[0] > 4 * page:
        pages.table[0, 1] = -1
    g = torch.Generator().manual_seed(3)
    for t in torch.randint(first[0], kv[0], (9,), generator=g).tolist() if causal else ():
        pg, at = int(pages.table[0, t // page]), t % page
        if pg >= 0:
            pages.v_scale[pg, :, at, 0] = 254 + t % 2
    sizes = (sum(new), len(new), heads, kv_heads, dh, pages.max_pages * page)
    lib, code, n = load_library(), int(dtype == BF16), [C.c_int(), C.c_int()]
    names = [lib.pf_attention_mx_kernel_name(code, int(fmt == "e2m1"), *sizes, C.byref(n[0])),
             lib.pf_attention_rows_kernel_name(code, *sizes, C.byref(n[1]))]
    assert names[0] == names[1] == name.encode() and n[0].value == n[1].value and (n[0].value > 1) == chunks, (names, n)
    q = wide(sum(new), heads * dh, dtype, 4)
    args = (cu(new), ints(*first), ints(*kv))
    got = pf_op_attention_mx(q, pages, *args, causal=causal, want_lse=True)
    want = pf_op_attention_paged(q, decoded_pages(pages, dtype), *args, causal=causal, want_lse=True)
    for a, b in zip(got, want):
        assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a[~a.isnan()], b[~b.isnan()])
        assert not b.isnan().all()
