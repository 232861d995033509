"""The operators around a cache in 8 or 4 bits as a program uses them: one after the other, captured, on two streams, over long caches and
calls of many rows."""
import random

import pytest
import torch

import mx_ref as M
import requests_ref as R
from paper_2405_14430_amd import KvMxPages, make_norm, make_rope, pf_op_attention_mx, pf_op_kv_append_mx, pf_op_kv_read_mx, pf_op_qk_norm_rope
from test_gpu_requests import BF16, CANARY, F32, cu, dev, ints

pytestmark = pytest.mark.gpu
POOLS = ("k", "v", "k_scale", "v_scale")


class Layer:
    """A projected row [q, k, v] goes into the cache and over it."""

    def __init__(self, dtype, fmt, heads=8, kv_heads=2, dh=128, page=16):
        self.dtype, self.fmt, self.heads, self.kv_heads, self.dh, self.page = dtype, fmt, heads, kv_heads, dh, page
        weight = lambda seed: (1 + 0.3 * dev(dh, dtype=F32, seed=seed)).to(dtype)
        self.q_norm, self.k_norm = make_norm("rms", weight(7), eps=1e-5), make_norm("rms", weight(9), eps=1e-5)
        self.q_plain = ("rms", weight(7), None, 1e-5)
        self.rope_args = dict(axes=(dh,), head_dim=dh, layout="half", theta=1e4)
        self.rope = make_rope((dh,), layout="half", theta=1e4)

    def rows(self, n, seed):
        return dev(n, (self.heads + 2 * self.kv_heads) * self.dh, dtype=self.dtype, seed=seed)

    def split(self, x):
        return x.split((self.heads * self.dh, self.kv_heads * self.dh, self.kv_heads * self.dh), 1)

    def cache(self, lengths, seed=0):
        return M.make_pages(self.fmt, self.kv_heads, self.dh, self.page, [(n + self.page - 1) // self.page for n in lengths], seed=seed, fill=0)

    def run(self, x, pages, cu_rows, first, kv_len, pos, out=None, causal=True):
        q, k, v = self.split(x)
        q = pf_op_kv_append_mx(pages, k, v, cu_rows, first, k_norm=self.k_norm, rope=self.rope, pos=pos, q=q, q_norm=self.q_norm)
        return q, pf_op_attention_mx(q, pages, cu_rows, first, kv_len, causal=causal, out=out)


@pytest.mark.parametrize("fmt", M.FORMATS)
@pytest.mark.parametrize("dtype", R.DTYPES)
def test_prompts_then_tokens(dtype, fmt):
    """Two prompts, the second in two parts, then single tokens: every row's attention is that of its turned q over the values that stand for
    the turned k and the v of all rows before it."""
    L = Layer(dtype, fmt)
    total = [70, 45]
    pages = L.cache(total)
    rows = [L.rows(n, seed=20 + s) for s, n in enumerate(total)]
    want_q = []
    for s, n in enumerate(total):           # the turned rows from the operator beside, which is held to its plain form elsewhere
        q, k, _ = L.split(rows[s])
        want_q.append(pf_op_qk_norm_rope(q, k, L.dh, q_norm=L.q_norm, k_norm=L.k_norm, rope=L.rope, pos=torch.arange(n).int().cuda()[:, None]))
        want, bound = M.turn(q, L.dh, L.q_plain, torch.arange(n).int()[:, None], L.rope_args)
        R.check(want_q[s][0], want, R.stored(bound, want, dtype), s)
    done = [0, 0]
    for step in [(60, 20), (0, 15)] + [(1, 1)] * 10:
        first = list(done)
        x = torch.cat([rows[s][done[s]:done[s] + n] for s, n in enumerate(step)])
        pos = torch.cat([torch.arange(done[s], done[s] + n) for s, n in enumerate(step)]).int().cuda()[:, None]
        done = [d + n for d, n in zip(done, step)]
        q, got = L.run(x, pages, cu(step), ints(*first), ints(*done), pos)
        at = 0
        for s, n in enumerate(step):
            assert torch.equal(q[at:at + n], want_q[s][0][first[s]:done[s]])
            k, v = (M.slot_rows(pages, p, s, done[s])[0] for p in ("k", "v"))
            for values, src in ((k, want_q[s][1]), (v, L.split(rows[s])[2])):
                codes, exps = M.encode(R.d64(src[:done[s]]).unflatten(1, (-1, L.dh)), fmt)
                assert torch.equal(values, M.decode(M.packed(codes, fmt, L.dh), exps, fmt, L.dh).flatten(1)), (step, s)
            want, _, b16, b32, _ = R.attention(q[at:at + n], k, v, L.dh, torch.arange(first[s], done[s]) + 1)
            R.check(got[at:at + n], want, R.stored(b16 if dtype == BF16 else b32, want, dtype), (step, s))
            at += n


@pytest.mark.parametrize("fmt", M.FORMATS)
@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("most", [5, 100])
def test_a_captured_layer_replays_with_other_lengths(most, dtype, fmt):
    """One graph serves every step of a growing batch.  Each replay equals the eager calls, which run between the replays."""
    L = Layer(dtype, fmt)
    caches = [L.cache([3000, 700], seed=1) for _ in range(2)]
    x = L.rows(most, seed=0)
    st = dict(cu_rows=cu([most - 2, 1]), first=ints(50, 3), kv_len=ints(48 + most, 4), pos=torch.zeros(most, 1, dtype=torch.int32, device="cuda"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        L.run(x, caches[0], **st)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for p in POOLS:
        getattr(caches[0], p).zero_()
    out = torch.empty(most, L.heads * L.dh, dtype=dtype, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.run(x, caches[0], out=out, **st)
    rng = random.Random(1)
    for i in range(7):
        x.copy_(L.rows(most, seed=30 + i))
        a = rng.choice([0, 1, rng.randint(0, most), most])
        lens = (a, rng.randint(0, most - a))
        first = [rng.choice([0, 400 * i, 2900]), 100 * i]
        st["cu_rows"].copy_(cu(lens))
        st["first"].copy_(ints(*first))
        st["kv_len"].copy_(ints(first[0] + lens[0], first[1] + lens[1]))
        st["pos"].copy_(torch.randint(0, 4000, (most, 1), generator=torch.Generator().manual_seed(i), dtype=torch.int32))
        out.fill_(CANARY)
        g.replay()
        torch.cuda.synchronize()
        want = torch.full_like(out, CANARY)
        L.run(x, caches[1], out=want, **st)
        n = sum(lens)
        assert (out[n:] == CANARY).all() and torch.equal(out, want), (i, lens)
        assert all(torch.equal(getattr(caches[0], p), getattr(caches[1], p)) for p in POOLS), i


@pytest.mark.parametrize("fmt", M.FORMATS)
@pytest.mark.parametrize("dtype", R.DTYPES)
def test_two_streams_at_once(dtype, fmt):
    """Calls of one kind on two streams share nothing."""
    work = [(dev(2, 8 * 128, dtype=dtype, seed=i), M.make_pages(fmt, 2, 128, 16, [200], seed=i)) for i in range(2)]
    lens, first, kv = cu([2]), ints(3100), ints(3102)

    def run(q, pages):
        rows = pf_op_kv_read_mx(pages, lens, first, 2, dtype)
        return (pf_op_attention_mx(q, pages, lens, first, kv), *rows, pf_op_qk_norm_rope(q, rows[0], 128, q_norm=make_norm("rms"))[0])
    want = [run(*w) for w in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    got = [[], []]
    for _ in range(20):
        for i, (w, s) in enumerate(zip(work, streams)):
            with torch.cuda.stream(s):
                got[i].append(run(*w))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for g in got[i] for a, b in zip(g, want[i]))


@pytest.mark.parametrize("fmt", M.FORMATS)
@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("seqs,heads,kv_heads,dh,longest", [(150, 8, 2, 128, 700), (70, 32, 1, 64, 60), (130, 4, 4, 72, 2600), (65, 5, 5, 40, 33)])
def test_attention_of_many_short_sequences(seqs, heads, kv_heads, dh, longest, dtype, fmt):
    """More sequences than a wave has lanes, of 0 to 3 rows over caches from none to long ones; a run of empty sequences among them."""
    rng = random.Random(seqs)
    new = [0 if 20 <= s < 90 and seqs > 100 else rng.choice([0, 1, 1, 1, 2, 3]) for s in range(seqs)]
    kv = [rng.choice([0, n, rng.randint(n, longest)]) for n in new]
    first = [m - n for m, n in zip(kv, new)]
    pages = M.make_pages(fmt, kv_heads, dh, 16, [(m + 15) // 16 for m in kv], seed=2)
    values = {p: M.decode(getattr(pages, p), getattr(pages, p + "_scale"), fmt, dh) for p in ("k", "v")}
    slots = lambda p, s: values[p][pages.table[s].cpu().clamp(min=0).long()].transpose(1, 2).reshape(-1, kv_heads * dh)[:kv[s]]
    lead, tq = 1, sum(new) + 3
    q = dev(tq, heads * dh, dtype=dtype, seed=4)
    for causal in (True, False):
        out = torch.full_like(q, CANARY)
        got, lse = pf_op_attention_mx(q, pages, cu(new, lead), ints(*first), ints(*kv), causal=causal, out=out, want_lse=True)
        at = lead
        for s, n in enumerate(new):
            if n:
                k, v = slots("k", s), slots("v", s)
                last = (torch.arange(n) + first[s] + 1).clamp(0, kv[s]) if causal else torch.full((n,), kv[s])
                want, want_lse, b16, b32, bl = R.attention(q[at:at + n], k, v, dh, last)
                R.check(got[at:at + n], want, R.stored(b16 if dtype == BF16 else b32, want, dtype), ("out", s))
                R.check(lse[at:at + n], want_lse, bl + 4 * R.U * want_lse.abs().nan_to_num(posinf=0.0), ("lse", s))
            at += n
        assert (got[:lead] == CANARY).all() and (got[at:] == CANARY).all()


@pytest.mark.parametrize("fmt", M.FORMATS)
@pytest.mark.parametrize("seqs,heads,kv_heads,dh", [(8192, 32, 32, 64), (8192, 64, 16, 64), (9001, 17, 17, 8)])
def test_many_tokens_over_a_wide_table(seqs, heads, kv_heads, dh, fmt):
    """Thousands of single tokens with room for 131072 keys each, of which few are there: taken as over pages of rows."""
    page, pool = 1024, 5
    pages = M.make_pages(fmt, kv_heads, dh, page, [pool], spare=0)
    kv = torch.arange(seqs) * 7 % 61
    pages = KvMxPages(fmt, pages.k, pages.v, pages.k_scale, pages.v_scale, (torch.arange(seqs * 128) % (pool + 1)).int().view(seqs, 128).cuda(), dh)
    q = dev(seqs, heads * dh, seed=3)
    lens, kv_len = torch.arange(seqs + 1).int().cuda(), kv.int().cuda()
    got = pf_op_attention_mx(q, pages, lens, kv_len - 1, kv_len)
    assert (got[kv.cuda() == 0] == 0).all()
    for s in (1, 2, 8, 700, 4095, 4096, seqs - 2, seqs - 1):
        n = int(kv[s])
        k, have = M.slot_rows(pages, "k", s, n)
        v, _ = M.slot_rows(pages, "v", s, n)
        want, _, b16, _, _ = R.attention(q[s:s + 1], k, v, dh, torch.tensor([n]), present=have)
        R.check(got[s:s + 1], want, R.stored(b16, want, BF16), s)


@pytest.mark.parametrize("fmt", M.FORMATS)
def test_as_many_sequences_as_over_pages_of_rows(fmt):
    """2^20 tokens of 16 query heads to a key head: bit for bit what calls of 4096 of them give."""
    part, times, heads, kv_heads, dh, page, pool = 4096, 256, 128, 8, 8, 16, 7
    small = M.make_pages(fmt, kv_heads, dh, page, [pool], spare=0)
    i = torch.arange(part * times, device="cuda") % part
    table, kv = (i % (pool + 1)).int()[:, None], (i % 17).int()
    q = dev(part, heads * dh, seed=3)

    def run(q, n):
        pages = KvMxPages(fmt, small.k, small.v, small.k_scale, small.v_scale, table[:n], dh)
        return pf_op_attention_mx(q, pages, torch.arange(n + 1).int().cuda(), kv[:n] - 1, kv[:n])
    want, got = run(q, part), run(q.repeat(times, 1), part * times)
    assert torch.equal(got.view(times, part, -1), want.expand(times, -1, -1)) and want.isfinite().all() and (want != 0).any()


@pytest.mark.parametrize("fmt", M.FORMATS)
@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("rows", [2, 40, 700])
def test_results_do_not_change_from_call_to_call(rows, dtype, fmt):
    pages = M.make_pages(fmt, 2, 128, 64, [60, 20])
    q = dev(rows, 8 * 128, dtype=dtype, seed=4)
    run = lambda: pf_op_attention_mx(q, pages, cu([rows - 1, 1]), ints(3800 - rows, 1200), ints(3800 - 1, 1201), want_lse=True)
    want = run()
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(run(), want))


@pytest.mark.parametrize("fmt", M.FORMATS)
def test_pages_far_apart(fmt):
    """Pages whose offsets pass 2^32 bytes, written and read."""
    kv_heads, dh, page, n_pages = 2, 64, 16, 6
    near = KvMxPages.zeros(fmt, n_pages, kv_heads, page, dh, ints(5, 0, 4, 1, 3, 2).view(2, 3))

    def far(t):
        flat = torch.empty(n_pages, 2 ** 30, dtype=torch.uint8, device="cuda")
        return flat[:, :t[0].numel()].unflatten(1, t.shape[1:]).fill_(0)
    new, first = [40, 30], [3, 10]
    q, k, v = dev(70, 4 * dh, seed=1), dev(70, kv_heads * dh, seed=2), dev(70, kv_heads * dh, seed=3)
    results = []
    for pages in (near, KvMxPages(fmt, far(near.k), far(near.v), far(near.k_scale), far(near.v_scale), near.table, dh)):
        pf_op_kv_append_mx(pages, k, v, cu(new), ints(*first))
        rows = pf_op_attention_mx(q, pages, cu(new), ints(*first), ints(43, 40))
        tokens = pf_op_attention_mx(q[:2], pages, cu([1, 1]), ints(42, 39), ints(43, 40))
        full = pf_op_attention_mx(q.float(), pages, cu(new), ints(*first), ints(43, 40), causal=False)
        results.append((*(getattr(pages, p).clone() for p in POOLS), rows, tokens, full, *pf_op_kv_read_mx(pages, cu(new), ints(*first), 70, F32)))
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_rows_far_apart():
    """Rows whose offsets pass 2^31 elements: what packed rows give, bit for bit."""
    n, heads, kv_heads, dh, far = 515, 4, 2, 64, 2 ** 22

    def spread(x):
        return torch.empty(n, far, dtype=x.dtype, device="cuda")[:, :x.shape[1]].copy_(x)
    q, k, v = dev(n, heads * dh, seed=1), dev(n, kv_heads * dh, seed=2), dev(n, kv_heads * dh, seed=3)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")[:, None]
    rope, norm, table = make_rope((dh,), theta=1e4, layout="half"), make_norm("rms"), torch.arange(33, dtype=torch.int32, device="cuda")[None]
    turned = pf_op_qk_norm_rope(q, k, dh, q_norm=norm, k_norm=norm, rope=rope, pos=pos)
    got = pf_op_qk_norm_rope(spread(q), spread(k), dh, q_norm=norm, k_norm=norm, rope=rope, pos=pos, q_out=spread(q), k_out=spread(k))
    assert all(torch.equal(a, b) for a, b in zip(got, turned))
    pages = [KvMxPages.zeros("e4m3", 33, kv_heads, 16, dh, table) for _ in range(2)]
    pf_op_kv_append_mx(pages[0], k, v, cu([n]), ints(2), k_norm=norm, rope=rope, pos=pos)
    pf_op_kv_append_mx(pages[1], spread(k), spread(v), cu([n]), ints(2), k_norm=norm, rope=rope, pos=pos)
    assert all(torch.equal(getattr(pages[0], p), getattr(pages[1], p)) for p in POOLS)
    back = pf_op_kv_read_mx(pages[0], cu([n]), ints(2), n, BF16)
    got = pf_op_kv_read_mx(pages[0], cu([n]), ints(2), n, BF16, k_out=spread(k), v_out=spread(v))
    assert all(torch.equal(a, b) for a, b in zip(got, back))
    for rows in (n, 3):
        args = (pages[0], cu([rows]), ints(517 - rows), ints(517))
        assert torch.equal(pf_op_attention_mx(spread(q)[:rows], *args, out=spread(q)[:rows]), pf_op_attention_mx(q[:rows], *args))


@pytest.mark.parametrize("fmt", M.FORMATS)
@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("n,heads,kv_heads,dh,page", [(2 ** 22 + 5, 1, 1, 8, 1024), (140001, 16, 8, 64, 64), (60013, 5, 16, 72, 256)])
def test_large_calls_equal_their_parts(n, heads, kv_heads, dh, page, dtype, fmt):
    """More rows than a launch takes, and more bytes than the caches hold: bit for bit what calls of a part of the rows give."""
    x = dev(4099, (heads + 2 * kv_heads) * dh, dtype=dtype, seed=1).repeat(n // 4099 + 1, 1)[:n]
    q, k, v = x.split((heads * dh, kv_heads * dh, kv_heads * dh), 1)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")[:, None]
    step = 2 ** 20 + 3 if n > 2 ** 22 else 9001
    parts = [slice(i, min(i + step, n)) for i in range(0, n, step)]
    rope, norm = make_rope((dh,), layout="half"), make_norm("rms")
    kw = dict(q_norm=norm, k_norm=norm, rope=rope)
    got = pf_op_qk_norm_rope(q, k, dh, pos=pos, **kw)
    want = [pf_op_qk_norm_rope(q[p], k[p], dh, pos=pos[p], **kw) for p in parts]
    assert all(torch.equal(g, torch.cat([w[i] for w in want])) for i, g in enumerate(got))
    del want
    table = torch.randperm((n + page - 1) // page, generator=torch.Generator().manual_seed(3)).int().cuda()[None]
    caches = [KvMxPages.zeros(fmt, table.shape[1], kv_heads, page, dh, table) for _ in range(2)]
    assert torch.equal(pf_op_kv_append_mx(caches[0], k, v, cu([n]), ints(0), pos=pos, q=q, **kw), got[0])
    for p in parts:
        pf_op_kv_append_mx(caches[1], k[p], v[p], cu([p.stop - p.start]), ints(p.start), k_norm=norm, rope=rope, pos=pos[p])
    assert all(torch.equal(getattr(caches[0], p), getattr(caches[1], p)) for p in POOLS)
    back = pf_op_kv_read_mx(caches[0], cu([n]), ints(0), n, dtype)
    for p in parts:
        some = pf_op_kv_read_mx(caches[0], cu([p.stop - p.start]), ints(p.start), p.stop - p.start, dtype)
        assert all(torch.equal(a, b[p]) for a, b in zip(some, back))


@pytest.mark.parametrize("fmt", M.FORMATS)
@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("dh", range(8, 136, 8))
def test_a_layer_of_every_head_size(dh, dtype, fmt):
    """Normed and turned rows into the pages and attention over these, tokens and prompts: every head size, rotation of a part of the channels and of
    axes of odd halves, either pair layout."""
    heads, kv_heads, page = 6, 3, 16
    layout = "half" if dh % 16 else "interleaved"
    axes = [(dh,), (dh // 2 - dh // 2 % 2, 2), (max(dh // 4 * 2 - 2, 2),)][dh // 8 % 3]
    args = dict(axes=axes, head_dim=dh, layout=layout, theta=1e4)
    rope = make_rope(axes, layout=layout, theta=1e4)
    w = (1 + 0.3 * dev(dh, dtype=F32, seed=7)).to(dtype)
    norm, plain = make_norm("rms", w, eps=1e-5), ("rms", w, None, 1e-5)
    for new, first in (([1, 2, 1], [40, 0, 129]), ([70, 1], [9, 200])):
        n, kv = sum(new), [a + b for a, b in zip(new, first)]
        pages = M.make_pages(fmt, kv_heads, dh, page, [(m + page - 1) // page for m in kv], seed=1)
        q, k, v = (dev(n, h * dh, dtype=dtype, seed=s) for s, h in enumerate((heads, kv_heads, kv_heads)))
        pos = torch.randint(-300, 300, (n, len(axes)), generator=torch.Generator().manual_seed(2), dtype=torch.int32).cuda()
        k_turned = pf_op_qk_norm_rope(None, k, dh, k_norm=norm, rope=rope, pos=pos)[1]
        want, bound = M.turn(k, dh, plain, pos, args)
        R.check(k_turned, want, R.stored(bound, want, dtype), "k")
        q = pf_op_kv_append_mx(pages, k, v, cu(new), ints(*first), k_norm=norm, rope=rope, pos=pos, q=q, q_norm=norm, q_out=q)
        want, bound = M.turn(dev(n, heads * dh, dtype=dtype, seed=0), dh, plain, pos, args)
        R.check(q, want, R.stored(bound, want, dtype), "q")
        got = pf_op_attention_mx(q, pages, cu(new), ints(*first), ints(*kv))
        at = 0
        for s, m in enumerate(new):
            rows = {}
            for which, src in (("k", k_turned), ("v", v)):
                rows[which] = M.slot_rows(pages, which, s, kv[s])[0]
                codes, exps = M.encode(R.d64(src[at:at + m]).unflatten(1, (-1, dh)), fmt)
                assert torch.equal(rows[which][first[s]:], M.decode(M.packed(codes, fmt, dh), exps, fmt, dh).flatten(1)), (which, s)
            want, _, b16, b32, _ = R.attention(q[at:at + m], rows["k"], rows["v"], dh, torch.arange(first[s], kv[s]) + 1)
            R.check(got[at:at + m], want, R.stored(b16 if dtype == BF16 else b32, want, dtype), s)
            at += m
