"""Every kernel of the attention over packed rows and pages, whole and in chunks, at sizes that choose it: against the 64-bit form on
some of the heads, with infinities and NaN where the causal mask hides them from most rows."""
import ctypes as C
import math
import random

import pytest
import torch

import requests_ref as R
from paper_2405_14430_amd import KvPages, load_library, pf_op_attention_packed, pf_op_attention_paged

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32

KERNELS = [
    # type, head_dim, rows, sequences, heads, kv_heads, keys, kernel, in chunks
    (BF16, 64, 520, 3, 32, 4, 173, "attn_rows_kernel<bf16,64,4,1>", False),
    (BF16, 64, 1030, 3, 4, 4, 4000, "attn_rows_kernel<bf16,64,4,1>", True),
    (BF16, 40, 777, 1, 32, 4, 777, "attn_rows_kernel<bf16,64,4,1>", False),
    (BF16, 72, 1500, 3, 16, 16, 500, "attn_rows_kernel<bf16,96,4,1>", False),
    (BF16, 96, 300, 3, 24, 24, 4000, "attn_rows_kernel<bf16,96,4,1>", True),
    (BF16, 128, 777, 3, 24, 24, 259, "attn_rows_kernel<bf16,128,4,1>", False),
    (BF16, 120, 777, 1, 4, 4, 4000, "attn_rows_kernel<bf16,128,4,1>", True),
    (F32, 64, 1030, 3, 32, 4, 343, "attn_rows_kernel<float,64,4,1>", False),
    (F32, 72, 1030, 3, 32, 4, 343, "attn_rows_kernel<float,96,4,1>", False),
    (F32, 128, 1030, 3, 32, 4, 343, "attn_rows_kernel<float,128,4,1>", False),
    (F32, 64, 4100, 1, 8, 8, 4000, "attn_rows_kernel<float,64,4,1>", True),
    (BF16, 64, 2050, 3, 16, 16, 683, "attn_rows_wide_kernel<64,4>", False),
    (BF16, 64, 4100, 1, 4, 4, 2000, "attn_rows_wide_kernel<64,4>", True),
    (BF16, 40, 300, 3, 32, 4, 4000, "attn_rows_wide_kernel<64,4>", True),
    (BF16, 72, 1030, 3, 32, 4, 343, "attn_rows_wide_kernel<96,5>", False),
    (BF16, 72, 1500, 1, 4, 4, 4000, "attn_rows_wide_kernel<96,5>", True),
    (BF16, 96, 777, 1, 24, 24, 777, "attn_rows_wide_kernel<96,6>", False),
    (BF16, 96, 2050, 3, 4, 4, 2000, "attn_rows_wide_kernel<96,6>", True),
    (BF16, 128, 4100, 1, 8, 8, 1000, "attn_rows_wide_kernel<128,8>", False),
    (BF16, 128, 777, 3, 14, 2, 2000, "attn_rows_wide_kernel<128,8>", True),
    (BF16, 64, 5, 3, 8, 2, 3000, "attn_rows_kernel<bf16,64,1,4>", True),
    (BF16, 72, 60, 1, 6, 3, 900, "attn_rows_kernel<bf16,96,1,4>", True),
    (BF16, 72, 60, 1, 6, 3, 500, "attn_rows_kernel<bf16,96,1,4>", False),
    (BF16, 128, 33, 3, 14, 2, 3000, "attn_rows_kernel<bf16,128,1,4>", True),
    (F32, 64, 300, 1, 8, 8, 700, "attn_rows_kernel<float,64,1,4>", True),
    (F32, 64, 300, 1, 8, 8, 400, "attn_rows_kernel<float,64,1,4>", False),
    (BF16, 128, 60, 3, 8, 2, 170, "attn_rows_kernel<bf16,128,1,4>", False),
    (F32, 96, 3, 3, 8, 1, 3000, "attn_rows_kernel<float,96,1,4>", True),
    (F32, 128, 70, 3, 8, 2, 2500, "attn_rows_kernel<float,128,1,4>", True),
]
ids = lambda k: f"{k[7]}{'-chunks' if k[8] else ''}-{k[1]}"


def rand(*shape, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g).to(dtype).cuda()


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def starts(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return ints(out)


def shares(total, parts):
    return [total] if parts == 1 else [total // 2, 1, total - total // 2 - 1]


def kernel_name(dtype, rows, seqs, heads, kv_heads, dh, keys):
    n = C.c_int()
    name = load_library().pf_attention_rows_kernel_name(int(dtype == BF16), rows, seqs, heads, kv_heads, dh, keys, C.byref(n))
    return name.decode(), n.value > 1


def plant(k, v, m, dh):
    """An infinity and a NaN among the last values of a sequence of m keys, and a NaN key near its end (rows [m, kv_heads * dh])."""
    if m < 16:
        return
    v.view(v.shape[0], -1, dh)[m - 13, :, 3] = math.inf
    v.view(v.shape[0], -1, dh)[m - 11, :, 5] = math.nan
    k.view(k.shape[0], -1, dh)[m - 2] = math.nan


def check_sequence(out, lse, q, k, v, heads, kv_heads, dh, last, planted, dtype, what):
    """out, q [n, heads * dh], k, v [m, kv_heads * dh] of one sequence, on the CPU."""
    m = k.shape[0]
    clean = lambda t: torch.where(torch.isfinite(t), t, 0.0)
    for h in sorted({0, heads // 2, heads - 1}):
        g = h * kv_heads // heads
        col = slice(h * dh, h * dh + dh)
        want, want_lse, b16, b32, bl = R.attention(q[:, col], clean(k[:, g * dh:g * dh + dh]), clean(v[:, g * dh:g * dh + dh]), dh, last)
        got, bound = out[:, col].clone(), R.stored(b16 if dtype == BF16 else b32, want, dtype)
        if planted and m >= 16:
            want[last > m - 13, 3] = math.inf
            want[last > m - 11, 5] = math.nan
            want[last > m - 2] = math.nan
            want_lse[last > m - 2] = math.nan
        R.check(got, want, bound, (what, h))
        R.check(lse[:, h:h + 1], want_lse, bl + 4 * R.U * want_lse.abs().nan_to_num(posinf=0.0), (what, h, "lse"))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("case", KERNELS, ids=ids)
def test_packed(case, causal):
    dtype, dh, rows, seqs, heads, kv_heads, keys, name, chunks = case
    nq, nk = shares(rows, seqs), shares(keys, seqs)[::-1]
    assert kernel_name(dtype, rows, seqs, heads, kv_heads, dh, keys) == (name, chunks)
    q, k, v = rand(rows, heads * dh, dtype=dtype, seed=1), rand(keys, kv_heads * dh, dtype=dtype, seed=2), rand(keys, kv_heads * dh, dtype=dtype, seed=3)
    at = 0
    for m in nk if causal else ():
        plant(k[at:at + m], v[at:at + m], m, dh)
        at += m
    out, lse = pf_op_attention_packed(q, k, v, starts(nq), starts(nk), dh, causal=causal, want_lse=True)
    out, lse, q, k, v = (R.d64(t) for t in (out, lse, q, k, v))
    a = b = 0
    for n, m in zip(nq, nk):
        last = (torch.arange(n) + m - n + 1).clamp(min=0) if causal else torch.full((n,), m)
        check_sequence(out[a:a + n], lse[a:a + n], q[a:a + n], k[b:b + m], v[b:b + m], heads, kv_heads, dh, last, causal, dtype, (n, m))
        a, b = a + n, b + m


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("case", KERNELS, ids=ids)
def test_paged(case, causal):
    dtype, dh, rows, seqs, heads, kv_heads, keys, name, chunks = case
    page = 16
    capacity = (keys + page - 1) // page
    new = shares(rows, seqs)
    kv = [keys] if seqs == 1 else [keys - 3, max(keys // 3, 1), keys]
    assert kernel_name(dtype, rows, seqs, heads, kv_heads, dh, capacity * page)[0] == name
    order = list(range(seqs * capacity + 2))
    random.Random(7).shuffle(order)
    table = [order[s * capacity:(s + 1) * capacity] for s in range(seqs)]
    kp = rand(len(order), kv_heads, page, dh, dtype=dtype, seed=4)
    vp = rand(len(order), kv_heads, page, dh, dtype=dtype, seed=5)
    pages = KvPages(kp, vp, ints(table))
    rows_of = lambda pool, s, m: pool[torch.tensor(table[s])].permute(0, 2, 1, 3).reshape(capacity * page, kv_heads * dh)[:m]
    kc, vc = kp.cpu(), vp.cpu()
    ks, vs = [rows_of(kc, s, m) for s, m in enumerate(kv)], [rows_of(vc, s, m) for s, m in enumerate(kv)]
    for s, m in enumerate(kv):
        if causal:
            plant(ks[s], vs[s], m, dh)
            for t in range(max(m - 13, 0), m):
                kp[table[s][t // page], :, t % page] = ks[s][t].view(kv_heads, dh).cuda()
                vp[table[s][t // page], :, t % page] = vs[s][t].view(kv_heads, dh).cuda()
        for t in range(m, capacity * page):
            kp[table[s][t // page], :, t % page] = math.nan
            vp[table[s][t // page], :, t % page] = math.nan
    q = rand(rows, heads * dh, dtype=dtype, seed=6)
    first = [m - n for n, m in zip(new, kv)]
    out, lse = pf_op_attention_paged(q, pages, starts(new), ints(first), ints(kv), causal=causal, want_lse=True)
    out, lse, q = (R.d64(t) for t in (out, lse, q))
    a = 0
    for s, (n, m) in enumerate(zip(new, kv)):
        last = (torch.arange(n) + first[s] + 1).clamp(min=0) if causal else torch.full((n,), m)
        check_sequence(out[a:a + n], lse[a:a + n], q[a:a + n], R.d64(ks[s]), R.d64(vs[s]), heads, kv_heads, dh, last, causal, dtype, (s, n, m))
        a += n


@pytest.mark.parametrize("dtype,dh,rows,heads,keys", [(BF16, 128, 300, 8, 700), (BF16, 128, 777, 24, 259), (BF16, 64, 2050, 16, 2050)])
def test_scores_that_are_not_finite_reach_their_rows_only(dtype, dh, rows, heads, keys):
    """A query with a NaN or an infinity spoils its own row and head, log-sum-exp included, and nothing else."""
    q, k, v = (rand(n, heads * dh, dtype=dtype, seed=i) for i, n in enumerate((rows, keys, keys)))
    q[7, 3], q[9, dh + 1] = math.nan, math.inf
    ref, ref_lse = pf_op_attention_packed(torch.where(torch.isfinite(q), q, 0), k, v, starts([rows]), starts([keys]), dh, want_lse=True)
    out, lse = pf_op_attention_packed(q, k, v, starts([rows]), starts([keys]), dh, want_lse=True)
    assert torch.isnan(out[7, :dh]).all() and torch.isnan(out[9, dh:2 * dh]).all() and torch.isnan(lse[7, 0]) and torch.isnan(lse[9, 1])
    out[7, :dh], ref[7, :dh], out[9, dh:2 * dh], ref[9, dh:2 * dh] = 0, 0, 0, 0
    lse[7, 0], ref_lse[7, 0], lse[9, 1], ref_lse[9, 1] = 0, 0, 0, 0
    # other rows: the same sums, but the wide kernel may form a shared step's weights anew with another reference, which moves each by its
    # rounding: 2 * 2^-8 of sum p |v| (below 1.2 over hundreds of unit normal keys), and the output by its own, below 2^-8 at |out| < 1
    assert (out.float() - ref.float()).abs().max() <= 2.0 ** -7 * 1.2 + 2.0 ** -8 and (lse - ref_lse).abs().max() <= 1e-5


@pytest.mark.parametrize("dtype,rows,keys,chunks", [(BF16, 1, 240, False), (BF16, 1, 4096, True), (BF16, 1, 16384, True), (F32, 5, 4096, True)])
def test_values_whose_weight_underflows_reach_the_row(dtype, rows, keys, chunks):
    """An infinity and a NaN among the values of keys far below the row's best one, exp(-400) of its weight: the row is not finite there,
    in one chunk as in many, and what it would be elsewhere."""
    dh = 64
    name, cut = kernel_name(dtype, rows, 1, 1, 1, dh, keys)
    assert cut == chunks, name
    q, k, v = rand(rows, dh, dtype=dtype, seed=1), rand(keys, dh, dtype=dtype, seed=2), rand(keys, dh, dtype=dtype, seed=3)
    q[:, 0] = 16.0
    k[:, 0] = 0.0
    k[keys - 100:, 0] = 200.0                      # 16 * 200 / sqrt(64) = 400
    want, _, b16, b32, _ = R.attention(q, k, v, dh, torch.full((rows,), keys))
    v[20, 3], v[keys // 3, 5] = math.inf, math.nan
    out = R.d64(pf_op_attention_packed(q, k, v, starts([rows]), starts([keys]), dh))
    assert not torch.isfinite(out[:, [3, 5]]).any()
    out[:, [3, 5]] = want[:, [3, 5]]
    R.check(out, want, R.stored(b16 if dtype == BF16 else b32, want, dtype), "out")
