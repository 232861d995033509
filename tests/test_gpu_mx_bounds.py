"""Pages of 8 or 4 bits with wrong lengths, slots and page numbers on the device: wrong rows at most, nothing outside the arrays (see
test_gpu_requests_bounds.py, whose guarded arrays these are: codes and exponents have 255 around them, exponents of NaN)."""
import ctypes as C
import random

import pytest
import torch

import mx_ref as M
from paper_2405_14430_amd import (KvMxPages, load_library, make_norm, make_rope, pf_kv_mx_row_bytes, pf_op_attention_mx, pf_op_kv_append_mx,
                                  pf_op_kv_read_mx, pf_op_qk_norm_rope)
from test_gpu_requests_bounds import BF16, F32, LOW, TOP, Guarded, rand, work_space, wrong_starts

pytestmark = pytest.mark.gpu

ATTENTION = [
    # type, head_dim, rows, sequences, heads, kv_heads, keys, kernel, in chunks
    (BF16, 64, 39, 3, 4, 4, 3000, "attn_rows_few_kernel<64>", True),
    (BF16, 64, 40, 3, 4, 4, 3000, ("attn_rows_kernel<bf16,64,1,4>", "attn_rows_few_kernel<64>"), True),   # by format
    (BF16, 72, 3, 3, 16, 1, 3000, "attn_rows_few_kernel<96>", True),
    (BF16, 128, 60, 70, 8, 2, 170, "attn_rows_few_kernel<128>", False),
    (BF16, 128, 33, 3, 14, 2, 3000, "attn_rows_kernel<bf16,128,1,4>", True),
    (BF16, 64, 1030, 3, 4, 4, 4000, "attn_rows_kernel<bf16,64,4,1>", True),
    (BF16, 72, 1030, 3, 32, 4, 343, "attn_rows_wide_kernel<96,5>", False),
    (BF16, 128, 777, 3, 14, 2, 2000, "attn_rows_wide_kernel<128,8>", True),
    (F32, 96, 3, 3, 8, 1, 3000, "attn_rows_kernel<float,96,1,4>", True),
    (F32, 72, 1030, 3, 32, 4, 343, "attn_rows_kernel<float,96,4,1>", False),
]
ids = lambda k: f"{k[7] if isinstance(k[7], str) else 'by-format'}{'-chunks' if k[8] else ''}"


def some_bytes(fmt, n_pages, kv_heads, page, dh, seed):
    """Codes and exponents of numbers below 2^5 of either format."""
    g = torch.Generator().manual_seed(seed)
    code = torch.randint(0, 256, (n_pages, kv_heads, page, pf_kv_mx_row_bytes(fmt, dh)), generator=g, dtype=torch.uint8)
    exp = torch.randint(118, 123, (n_pages, kv_heads, page, M.blocks(dh)), generator=g, dtype=torch.uint8)
    return (code & 0xf7 if fmt == "e4m3" else code).cuda(), exp.cuda()


def guarded_pages(g, fmt, n_pages, kv_heads, page, dh, table, fixed=True):
    """(pages, the four pools)"""
    pools = []
    for seed in (1, 2):
        for t in some_bytes(fmt, n_pages, kv_heads, page, dh, seed) if fixed else \
                [torch.full_like(t, 0x5b) for t in some_bytes(fmt, n_pages, kv_heads, page, dh, seed)]:
            pools.append(g.of(t, 255, fixed=fixed))
    return KvMxPages(fmt, pools[0], pools[2], pools[1], pools[3], table, dh), pools


def wrong_table(g, rng, n, width, n_pages, good):
    return g.ints([[rng.choice([rng.randrange(good)] * 3 + [LOW, -1, n_pages, TOP]) for _ in range(width)] for _ in range(n)])


@pytest.mark.parametrize("fmt", M.FORMATS)
@pytest.mark.parametrize("case", ATTENTION, ids=ids)
def test_attention_of_wrong_lengths(case, fmt):
    dtype, dh, rows, seqs, heads, kv_heads, keys, name, chunks = case
    lib, page, n_pages = load_library(), 16, 9
    name = name if isinstance(name, str) else name[M.FORMATS.index(fmt)]
    width = (keys + page - 1) // page
    n = C.c_int()
    sizes = (int(dtype == BF16), int(fmt == "e2m1"), rows, seqs, heads, kv_heads, dh, width * page)
    assert (lib.pf_attention_mx_kernel_name(*sizes, C.byref(n)).decode(), n.value > 1) == (name, chunks)
    ws_bytes = lib.pf_op_attention_mx_ws_bytes(*sizes)
    rng = random.Random(5)
    for i, cu_q in enumerate(wrong_starts(seqs, rows, 3)):
        g = Guarded()
        q = g.of(rand(rows, heads * dh, dtype=dtype, seed=1))
        pages, _ = guarded_pages(g, fmt, n_pages, kv_heads, page, dh, wrong_table(g, rng, seqs, width, n_pages, n_pages))
        kv = g.ints([rng.choice([LOW, -1, 0, 5, keys, width * page + 1, TOP]) for _ in range(seqs)])
        first = g.ints([rng.choice([LOW, -7, 0, 5, keys, TOP]) for _ in range(seqs)])
        out, lse, ws, cq = g.out(rows, heads * dh, dtype=dtype), g.out(rows, heads, dtype=F32), work_space(g, ws_bytes), g.ints(cu_q)
        print(name, i, flush=True)
        for causal in (0, 1):
            st = lib.pf_op_attention_mx(int(dtype == BF16), q.data_ptr(), heads * dh, pages.ref, cq.data_ptr(), first.data_ptr(), kv.data_ptr(),
                                        rows, heads, 0.0, causal, out.data_ptr(), heads * dh, lse.data_ptr(), ws.data_ptr(), ws_bytes,
                                        torch.cuda.current_stream().cuda_stream)
            assert st == 0
            torch.cuda.synchronize()
            g.check((i, causal))
            assert torch.isfinite(out).all() and not torch.isnan(lse).any(), (i, causal)


@pytest.mark.parametrize("fmt", M.FORMATS)
@pytest.mark.parametrize("case", ATTENTION, ids=ids)
def test_attention_clips_starts_and_lengths(case, fmt):
    """Starts below 0 and behind the last row, lengths below 0 and past the table's end: what the clipped ones give."""
    dtype, dh, rows, seqs, heads, kv_heads, keys, _, _ = case
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    cut = lambda v, top: [min(max(x, 0), top) for x in v]
    cu_q = [-5] + sorted(random.Random(rows).randint(0, rows) for _ in range(seqs - 2)) + [rows + 1, TOP]
    q = rand(rows, heads * dh, dtype=dtype, seed=1)
    page, width = 16, (keys + 15) // 16
    (k, ks), (v, vs) = (some_bytes(fmt, width, kv_heads, page, dh, s) for s in (7, 8))
    pages = KvMxPages(fmt, k, v, ks, vs, torch.arange(width, dtype=torch.int32, device="cuda").repeat(seqs, 1), dh)
    kv = [[LOW, keys // 2, width * page + 1, TOP, -1][s % 5] for s in range(seqs)]
    first = ints([max(keys - rows, 0)] * seqs)
    for causal in (False, True):
        a = pf_op_attention_mx(q, pages, ints(cu_q), first, ints(kv), causal=causal, want_lse=True)
        b = pf_op_attention_mx(q, pages, ints(cut(cu_q, rows)), first, ints(cut(kv, width * page)), causal=causal, want_lse=True)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("fmt", M.FORMATS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,seqs,heads,dh", [(60, 5, 4, 64), (60, 70, 40, 72), (5000, 3, 1, 128), (5000, 3, 9, 40)])
def test_append_and_read_of_wrong_lengths(rows, seqs, heads, dh, dtype, fmt):
    kv_heads, page, width, n_pages = 2, 16, 4, 12
    rope = make_rope((dh,), layout="half")
    rng = random.Random(6)
    for i, cu in enumerate(wrong_starts(seqs, rows, 4)):
        g = Guarded()
        q, k, v = (g.of(rand(rows, h * dh, dtype=dtype, seed=s)) for s, h in enumerate((heads, kv_heads, kv_heads)))
        # pages 8 .. 11 are nobody's
        pages, pools = guarded_pages(g, fmt, n_pages, kv_heads, page, dh, wrong_table(g, rng, seqs, width, n_pages, 8), fixed=False)
        first, pos = g.ints([rng.choice([LOW, -7, 0, 5, 63, TOP]) for _ in range(seqs)]), g.ints(list(range(rows)))
        q_out, k_back, v_back = (g.out(rows, h * dh, dtype=dtype) for h in (heads, kv_heads, kv_heads))
        cu, norm = g.ints(cu), make_norm("rms")
        print(rows, seqs, heads, dh, i, flush=True)
        pf_op_kv_append_mx(pages, k, v, cu, first, k_norm=norm, rope=rope, pos=pos, q=q, q_norm=norm, q_out=q_out)
        torch.cuda.synchronize()
        g.check(i)
        assert all((p[8:] == 0x5b).all() for p in pools) and all((p != 255).all() for p in pools[1::2]) and torch.isfinite(q_out).all()
        pf_op_kv_read_mx(pages, cu, first, rows, dtype, k_out=k_back, v_out=v_back)
        torch.cuda.synchronize()
        g.check((i, "read"))
        assert torch.isfinite(k_back).all() and torch.isfinite(v_back).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tokens,heads,kv_heads,dh", [(1, 1, 1, 8), (33, 7, 3, 72), (1030, 40, 2, 128), (5, 200, 33, 40)])
def test_norm_and_rotation_stay_within_their_rows(tokens, heads, kv_heads, dh, dtype):
    g = Guarded()
    q, k = (g.of(rand(tokens, h * dh, dtype=dtype, seed=s)) for s, h in enumerate((heads, kv_heads)))
    w, b = (g.of(rand(dh, dtype=dtype, seed=s)) for s in (3, 4))
    q_out, k_out = (g.out(tokens, h * dh, dtype=dtype) for h in (heads, kv_heads))
    pos = g.ints(list(range(tokens)))
    pf_op_qk_norm_rope(q, k, dh, q_norm=make_norm("layer", w, b), k_norm=make_norm("rms", w), rope=make_rope((dh,), layout="interleaved"),
                       pos=pos, q_out=q_out, k_out=k_out)
    torch.cuda.synchronize()
    g.check("norm")
    assert torch.isfinite(q_out).all() and torch.isfinite(k_out).all() and (q_out != 77).any(1).all() and (k_out != 77).any(1).all()


@pytest.mark.parametrize("fmt", M.FORMATS)
def test_append_of_two_rows_for_one_slot(fmt):
    """Two sequences over the same page: slots of one row hold it, those of two hold the bytes of either, unit by unit."""
    dh, kv_heads, page = 128, 8, 64
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    k, v = (rand(100, kv_heads * dh, dtype=BF16, seed=s) for s in (1, 2))

    def append(cu, first, rows):
        p = KvMxPages.zeros(fmt, 1, kv_heads, page, dh, ints(*[0] * (len(cu) - 1)).view(-1, 1))
        pf_op_kv_append_mx(p, k[rows], v[rows], ints(*cu), ints(*first))
        return p
    both = append((0, 60, 100), (0, 20), slice(0, 100))
    one, other = append((0, 60), (0,), slice(0, 60)), append((0, 40), (20,), slice(60, 100))
    for pool in ("k", "v", "k_scale", "v_scale"):
        x, a, b = (getattr(p, pool) for p in (both, one, other))
        assert torch.equal(x[:, :, :20], a[:, :, :20]) and (x[:, :, 60:] == 0).all()
        assert ((x == a) | (x == b))[:, :, 20:60].all()
