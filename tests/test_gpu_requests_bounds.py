"""Wrong lengths, slots and pages on the device: wrong rows at most, nothing outside the arrays.  Every array lies in the middle of a larger
one whose ends must stay as they were; inputs have NaN in theirs, so that a row read from there would show in a result.  Starts and lengths
that are only too large or too small are clipped, and then the rows are right."""
import ctypes as C
import math
import random

import pytest
import torch

from paper_2405_14430_amd import (KvPages, load_library, make_norm, make_rope, pf_op_attention_packed, pf_op_attention_paged, pf_op_kv_append,
                                  pf_op_norm_residual)

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
LOW, TOP = -2 ** 31, 2 ** 31 - 1
CANARY = 77.0


class Guarded:
    """Tensors between ends of 64 KiB elements each; `check` says that the ends, and tensors named as inputs, are as they were."""

    def __init__(self):
        self.all = []

    def of(self, t, ends=math.nan, fixed=True):
        n = 1 << 16
        flat = torch.full((t.numel() + 2 * n,), ends, dtype=t.dtype, device="cuda")
        flat[n:n + t.numel()] = t.reshape(-1)
        self.all.append((flat, flat.clone(), t.numel(), fixed))
        return flat[n:n + t.numel()].view(t.shape)

    def out(self, *shape, dtype):
        return self.of(torch.full(shape, CANARY, dtype=dtype, device="cuda"), CANARY, fixed=False)

    def ints(self, values):
        return self.of(torch.tensor(values, dtype=torch.int32, device="cuda"), 1)

    def check(self, what):
        n = 1 << 16
        same = lambda a, b: torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        for i, (now, was, size, fixed) in enumerate(self.all):
            assert same(now[:n], was[:n]) and same(now[n + size:], was[n + size:]), (what, i, "ends")
            assert not fixed or same(now, was), (what, i, "input")


def rand(*shape, dtype, seed):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def wrong_starts(n, rows, seed):
    """cu of n sequences over `rows` rows, wrong in several ways."""
    rng = random.Random(seed)
    some = lambda lo, hi: [rng.randint(lo, hi) for _ in range(n + 1)]
    return [sorted(some(0, rows), reverse=True), some(-3, rows + 3), some(LOW, TOP), [LOW] * n + [TOP], [TOP] + [LOW] * n,
            [rng.choice([LOW, -1, 0, rows, rows + 1, TOP]) for _ in range(n + 1)], [rows + 5] * (n + 1), [-9] * (n + 1)]


ATTENTION = [
    # type, head_dim, rows, sequences, heads, kv_heads, keys, kernel, in chunks
    (BF16, 64, 520, 3, 32, 4, 173, "attn_rows_kernel<bf16,64,4,1>", False),
    (BF16, 64, 1030, 3, 4, 4, 4000, "attn_rows_kernel<bf16,64,4,1>", True),
    (F32, 72, 1030, 3, 32, 4, 343, "attn_rows_kernel<float,96,4,1>", False),
    (BF16, 72, 1030, 3, 32, 4, 343, "attn_rows_wide_kernel<96,5>", False),
    (BF16, 128, 777, 3, 14, 2, 2000, "attn_rows_wide_kernel<128,8>", True),
    (BF16, 128, 33, 3, 14, 2, 3000, "attn_rows_kernel<bf16,128,1,4>", True),
    (BF16, 128, 60, 70, 8, 2, 170, "attn_rows_kernel<bf16,128,1,4>", False),
    (F32, 96, 3, 3, 8, 1, 3000, "attn_rows_kernel<float,96,1,4>", True),
]
ids = lambda k: f"{k[7]}{'-chunks' if k[8] else ''}"


def plan(dtype, rows, seqs, heads, kv_heads, dh, keys):
    lib, n = load_library(), C.c_int()
    sizes = (int(dtype == BF16), rows, seqs, heads, kv_heads, dh, keys)
    return lib.pf_attention_rows_kernel_name(*sizes, C.byref(n)).decode(), n.value > 1, lib.pf_op_attention_rows_ws_bytes(*sizes)


def work_space(g, size):
    return g.of(torch.zeros(max(size // 4, 4), device="cuda"), CANARY, fixed=False)


@pytest.mark.parametrize("case", ATTENTION, ids=ids)
def test_packed_attention_of_wrong_lengths(case):
    dtype, dh, rows, seqs, heads, kv_heads, keys, name, chunks = case
    lib = load_library()
    kernel, cut, ws_bytes = plan(dtype, rows, seqs, heads, kv_heads, dh, keys)
    assert (kernel, cut) == (name, chunks)
    for i, (cu_q, cu_k) in enumerate(zip(wrong_starts(seqs, rows, 1), wrong_starts(seqs, keys, 2)[::-1])):
        for causal in (0, 1):
            g = Guarded()
            q, k, v = (g.of(rand(n, h * dh, dtype=dtype, seed=s)) for s, (n, h) in enumerate(((rows, heads), (keys, kv_heads), (keys, kv_heads))))
            out, lse, ws = g.out(rows, heads * dh, dtype=dtype), g.out(rows, heads, dtype=F32), work_space(g, ws_bytes)
            cq, ck = g.ints(cu_q), g.ints(cu_k)
            print(name, i, causal, flush=True)
            st = lib.pf_op_attention_packed(int(dtype == BF16), q.data_ptr(), heads * dh, k.data_ptr(), kv_heads * dh, v.data_ptr(), kv_heads * dh,
                                            cq.data_ptr(), ck.data_ptr(), seqs, rows, keys, heads, kv_heads, dh, 0.0, causal, out.data_ptr(),
                                            heads * dh, lse.data_ptr(), ws.data_ptr(), ws_bytes, torch.cuda.current_stream().cuda_stream)
            assert st == 0
            torch.cuda.synchronize()
            g.check((i, causal))
            assert torch.isfinite(out).all() and not torch.isnan(lse).any(), (i, causal)


@pytest.mark.parametrize("case", ATTENTION, ids=ids)
def test_paged_attention_of_wrong_lengths(case):
    dtype, dh, rows, seqs, heads, kv_heads, keys, name, chunks = case
    lib, page = load_library(), 16
    width = (keys + page - 1) // page
    kernel, _, ws_bytes = plan(dtype, rows, seqs, heads, kv_heads, dh, width * page)
    assert kernel == name
    rng = random.Random(5)
    n_pages = 9
    for i, cu_q in enumerate(wrong_starts(seqs, rows, 3)):
        g = Guarded()
        q = g.of(rand(rows, heads * dh, dtype=dtype, seed=1))
        k, v = (g.of(rand(n_pages, kv_heads, page, dh, dtype=dtype, seed=s)) for s in (2, 3))
        table = g.ints([[rng.choice([rng.randrange(n_pages)] * 3 + [LOW, -1, n_pages, TOP]) for _ in range(width)] for _ in range(seqs)])
        kv = g.ints([rng.choice([LOW, -1, 0, 5, keys, width * page + 1, TOP]) for _ in range(seqs)])
        first = g.ints([rng.choice([LOW, -7, 0, 5, keys, TOP]) for _ in range(seqs)])
        out, lse, ws, cq = g.out(rows, heads * dh, dtype=dtype), g.out(rows, heads, dtype=F32), work_space(g, ws_bytes), g.ints(cu_q)
        pages = KvPages(k, v, table)
        print(name, i, flush=True)
        for causal in (0, 1):
            st = lib.pf_op_attention_paged(int(dtype == BF16), q.data_ptr(), heads * dh, pages.ref, cq.data_ptr(), first.data_ptr(), kv.data_ptr(), rows,
                                           heads, 0.0, causal, out.data_ptr(), heads * dh, lse.data_ptr(), ws.data_ptr(), ws_bytes,
                                           torch.cuda.current_stream().cuda_stream)
            assert st == 0
            torch.cuda.synchronize()
            g.check((i, causal))
            assert torch.isfinite(out).all() and not torch.isnan(lse).any(), (i, causal)


@pytest.mark.parametrize("case", ATTENTION, ids=ids)
def test_attention_clips_starts_and_lengths(case):
    """Starts below 0 and behind the last row, lengths below 0 and past the table's end: what the clipped ones give."""
    dtype, dh, rows, seqs, heads, kv_heads, keys, _, _ = case
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    cut = lambda v, top: [min(max(x, 0), top) for x in v]
    inner = lambda n: sorted(random.Random(n).randint(0, n) for _ in range(seqs - 2))
    cu_q, cu_k = [-5] + inner(rows) + [rows + 1, TOP], [LOW] + inner(keys) + [keys + 100, keys + 200]
    q, k, v = (rand(n, h * dh, dtype=dtype, seed=s) for s, (n, h) in enumerate(((rows, heads), (keys, kv_heads), (keys, kv_heads))))
    page, width = 16, (keys + 15) // 16
    pages = KvPages(*(rand(width, kv_heads, page, dh, dtype=dtype, seed=s) for s in (7, 8)),
                    torch.arange(width, dtype=torch.int32, device="cuda").repeat(seqs, 1))
    kv = [[LOW, keys // 2, width * page + 1, TOP, -1][s % 5] for s in range(seqs)]
    first = ints([max(keys - rows, 0)] * seqs)
    for causal in (False, True):
        a = pf_op_attention_packed(q, k, v, ints(cu_q), ints(cu_k), dh, causal=causal, want_lse=True)
        b = pf_op_attention_packed(q, k, v, ints(cut(cu_q, rows)), ints(cut(cu_k, keys)), dh, causal=causal, want_lse=True)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        a = pf_op_attention_paged(q, pages, ints(cu_q), first, ints(kv), causal=causal, want_lse=True)
        b = pf_op_attention_paged(q, pages, ints(cut(cu_q, rows)), first, ints(cut(kv, width * page)), causal=causal, want_lse=True)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,seqs,heads", [(60, 5, 4), (60, 70, 40), (5000, 3, 1), (5000, 3, 9)])
def test_append_of_wrong_lengths(rows, seqs, heads, dtype):
    dh, kv_heads, page, width, n_pages = 64, 2, 16, 4, 12
    rope = make_rope((dh,), layout="half")
    rng = random.Random(6)
    for i, cu in enumerate(wrong_starts(seqs, rows, 4)):
        g = Guarded()
        q, k, v = (g.of(rand(rows, h * dh, dtype=dtype, seed=s)) for s, h in enumerate((heads, kv_heads, kv_heads)))
        # pages 8 .. 11 are nobody's
        kp, vp = (g.out(n_pages, kv_heads, page, dh, dtype=dtype) for _ in range(2))
        table = g.ints([[rng.choice([rng.randrange(8)] * 3 + [LOW, -1, n_pages, TOP]) for _ in range(width)] for _ in range(seqs)])
        first, pos = g.ints([rng.choice([LOW, -7, 0, 5, 63, TOP]) for _ in range(seqs)]), g.ints(list(range(rows)))
        q_out = g.out(rows, heads * dh, dtype=dtype)
        print(rows, seqs, heads, i, flush=True)
        pf_op_kv_append(KvPages(kp, vp, table), k, v, g.ints(cu), first, rope=rope, pos=pos, q=q, q_out=q_out)
        torch.cuda.synchronize()
        g.check(i)
        assert (kp[8:] == CANARY).all() and (vp[8:] == CANARY).all() and all(torch.isfinite(t).all() for t in (kp, vp, q_out))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,seqs,d", [(7, 3, 520), (300, 70, 1152), (5000, 3, 72), (9, 2, 8192)])
def test_norm_of_wrong_lengths(rows, seqs, d, dtype):
    for i, cu in enumerate(wrong_starts(seqs, rows, 5)):
        g = Guarded()
        x, y = g.of(rand(rows, d, dtype=F32, seed=1)), g.of(rand(rows, d, dtype=dtype, seed=2))
        gate, scale = g.of(rand(seqs, d, dtype=F32, seed=3)), g.of(rand(seqs, d, dtype=F32, seed=4))
        x_out, h = g.out(rows, d, dtype=F32), g.out(rows, d, dtype=dtype)
        print(rows, seqs, d, i, flush=True)
        pf_op_norm_residual(y, x, post=make_norm("rms"), pre=make_norm("layer"), gate=gate, scale=scale, cu=g.ints(cu), x_out=x_out, h_out=h)
        torch.cuda.synchronize()
        g.check(i)
        assert torch.isfinite(x_out).all() and torch.isfinite(h).all()
        done = (x_out != CANARY).any(1)
        assert torch.equal(done, (h != CANARY).any(1))
        if i == 3:                          # one sequence of all rows behind empty ones
            want = pf_op_norm_residual(y, x, post=make_norm("rms"), pre=make_norm("layer"), gate=gate[seqs - 1], scale=scale[seqs - 1])
            assert torch.equal(x_out, want[0]) and torch.equal(h, want[1])
        if i in (6, 7):                     # all behind the rows, or in front (starts that decrease give some sequence's rows)
            assert not done.any()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_append_of_two_rows_for_one_slot(dtype):
    """Two sequences over the same page: every element is that of one of the rows, and slots of one row have it."""
    dh, kv_heads, page = 128, 8, 64
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    k, v = (rand(100, kv_heads * dh, dtype=dtype, seed=s) for s in (1, 2))
    pages = KvPages(*(torch.full((1, kv_heads, page, dh), CANARY, dtype=dtype, device="cuda") for _ in range(2)), ints(0, 0).view(2, 1))
    pf_op_kv_append(pages, k, v, ints(0, 60, 100), ints(0, 20))
    for pool, rows in ((pages.k, k), (pages.v, v)):
        got = pool[0].transpose(0, 1).reshape(page, kv_heads * dh)
        assert torch.equal(got[:20], rows[:20]) and (got[60:] == CANARY).all()
        assert ((got[20:60] == rows[20:60]) | (got[20:60] == rows[60:])).all()
