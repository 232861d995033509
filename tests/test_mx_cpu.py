"""Host side of the operators around a cache in 8 or 4 bits: sizes, refusals and no-ops of the C entry points (nothing is launched, so the
pointers need not be real), and the binding's checks."""
import ctypes as C
import math

import pytest
import torch

from paper_2405_14430_amd import binding as B
from test_requests_cpu import CONFIG, DTYPE, NULL, P, SHAPE, WORKSPACE, call, lib, rope64  # noqa: F401


def norm(kind=1, eps=1e-6, weight=P, bias=None):
    return C.byref(B.PfNorm(kind=kind, eps=eps, weight=weight, bias=bias))


BAD_NORMS = [(dict(kind=3), CONFIG), (dict(kind=-1), CONFIG), (dict(eps=-1.0), CONFIG), (dict(eps=math.nan), CONFIG),
             (dict(kind=0), CONFIG), (dict(weight=P + 8), SHAPE), (dict(bias=P + 4), SHAPE)]


def test_row_bytes(lib):
    sizes = lambda fmt: [lib.pf_kv_mx_row_bytes(fmt, d) for d in (8, 16, 24, 32, 40, 64, 72, 80, 96, 104, 128)]
    assert sizes(0) == [16, 16, 32, 32, 48, 64, 80, 80, 96, 112, 128]
    assert sizes(1) == [16, 16, 16, 16, 32, 32, 48, 48, 48, 64, 64]
    for fmt, d in ((2, 64), (-1, 64), (0, 0), (0, 4), (0, 136), (1, 100), (0, -8)):
        assert lib.pf_kv_mx_row_bytes(fmt, d) == 0
    for fmt, d in (("e3m2", 64), ("e4m3", 12), ("e4m3", 0), ("e2m1", 1 << 40)):
        with pytest.raises(B.PfError):
            B.pf_kv_mx_row_bytes(fmt, d)


TURN = dict(dtype=1, q=P, ldq=256, q_norm=None, q_out=2 * P, ldqo=256, heads=4, k=P, ldk=128, k_norm=None, k_out=2 * P, ldko=128,
            kv_heads=2, rope=None, pos=P, tokens=5, dh=64, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), SHAPE), (dict(heads=-1), SHAPE), (dict(kv_heads=65537), SHAPE), (dict(dtype=2), DTYPE), (dict(q=None), NULL),
    (dict(q_out=None), NULL), (dict(k=None), NULL), (dict(k_out=None), NULL), (dict(pos=None), NULL), (dict(dh=60), SHAPE),
    (dict(dh=136), SHAPE), (dict(dh=0), SHAPE), (dict(ldq=255), SHAPE), (dict(ldq=260), SHAPE), (dict(ldqo=248), SHAPE), (dict(ldk=120), SHAPE),
    (dict(ldko=132), SHAPE), (dict(q=P + 8), SHAPE), (dict(k_out=2 * P + 4), SHAPE), (dict(pos=P + 2), SHAPE), (dict(q_out=P, ldqo=264), SHAPE),
    (dict(k_out=P, ldko=136), SHAPE), (dict(tokens=(1 << 24) + 1), SHAPE), (dict(dh=32), CONFIG),
    (dict(tokens=0, q=None, k=None, q_out=None, k_out=None, pos=None), 0), (dict(heads=0, kv_heads=0, q=None, k=None), 0),
])
def test_turn_refuses(lib, change, status):
    assert call(lib, "pf_op_qk_norm_rope", dict(TURN, rope=rope64()), change) == status
    if status:
        assert lib.pf_last_error(None)


@pytest.mark.parametrize("side", ["q_norm", "k_norm"])
@pytest.mark.parametrize("bad,status", BAD_NORMS)
def test_bad_norms_are_refused(lib, bad, status, side):
    pg = pages()
    assert call(lib, "pf_op_qk_norm_rope", TURN, {side: norm(**bad)}) == status
    assert call(lib, "pf_op_kv_append_mx", dict(APPEND, pages=C.byref(pg)), {side: norm(**bad)}) == status


def pages(**kw):
    f = dict(k=P, v=2 * P, k_scale=P, v_scale=P, k_page_stride=2 * 16 * 64, v_page_stride=2 * 16 * 64, k_scale_stride=2 * 16 * 2,
             v_scale_stride=64, table=P, format=0, n_pages=10, page_size=16, kv_heads=2, head_dim=64, n_seqs=3, max_pages=4)
    f.update(kw)
    return B.PfKvMxPages(**f)


BAD_PAGES = [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(k_scale=None), NULL), (dict(v_scale=None), NULL), (dict(table=None), NULL),
    (dict(format=2), DTYPE), (dict(format=-1), DTYPE), (dict(page_size=24), SHAPE), (dict(page_size=8), SHAPE),
    (dict(page_size=2048, k_page_stride=1 << 20, v_page_stride=1 << 20, k_scale_stride=1 << 20, v_scale_stride=1 << 20), SHAPE),
    (dict(kv_heads=0), SHAPE), (dict(kv_heads=65537), SHAPE), (dict(head_dim=12), SHAPE),
    (dict(head_dim=136, k_page_stride=1 << 20, v_page_stride=1 << 20, k_scale_stride=1 << 20, v_scale_stride=1 << 20), SHAPE),
    (dict(n_seqs=-1), SHAPE), (dict(n_seqs=(1 << 30) + 1), SHAPE), (dict(max_pages=0), SHAPE), (dict(n_pages=0), SHAPE),
    (dict(k_page_stride=2047), SHAPE), (dict(v_page_stride=2056), SHAPE), (dict(k_page_stride=2032), SHAPE), (dict(k=P + 8), SHAPE),
    (dict(k_scale_stride=63), SHAPE), (dict(v_scale_stride=0), SHAPE), (dict(k_page_stride=1 << 60), SHAPE), (dict(v_scale_stride=1 << 60), SHAPE),
    (dict(head_dim=72), SHAPE),       # rows of 80 bytes
]
APPEND = dict(dtype=1, pages=None, k=P, ldk=128, k_norm=None, v=P, ldv=128, cu=P, first=P, tokens=7, rope=None, pos=P, q=P, ldq=256,
              q_norm=None, q_out=2 * P, ldqo=256, heads=4, stream=None)
READ = dict(dtype=1, pages=None, cu=P, first=P, tokens=7, k_out=P, ldk=128, v_out=2 * P, ldv=128, stream=None)
ATTEND = dict(dtype=1, q=P, ldq=256, pages=None, cu_q=P, first=P, kv_len=P, total_q=9, heads=4, scale=0.0, causal=1, out=2 * P, ldo=256,
              lse=None, ws=None, ws_bytes=0, stream=None)


@pytest.mark.parametrize("bad,status", BAD_PAGES)
def test_bad_pages_are_refused(lib, bad, status):
    pg = pages(**bad)
    d = 2 * pg.head_dim
    assert call(lib, "pf_op_kv_append_mx", dict(APPEND, pages=C.byref(pg)), dict(ldk=d, ldv=d, ldq=2 * d, ldqo=2 * d)) == status
    assert call(lib, "pf_op_kv_read_mx", dict(READ, pages=C.byref(pg)), dict(ldk=d, ldv=d)) == status
    assert call(lib, "pf_op_attention_mx", dict(ATTEND, pages=C.byref(pg)), dict(ldq=2 * d, ldo=2 * d)) == status


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), SHAPE), (dict(heads=-1), SHAPE), (dict(dtype=9), DTYPE), (dict(pages=None), NULL), (dict(k=None), NULL),
    (dict(v=None), NULL), (dict(cu=None), NULL), (dict(first=None), NULL), (dict(pos=None), NULL), (dict(q=None), NULL),
    (dict(q_out=None), NULL), (dict(heads=0), SHAPE), (dict(ldk=120), SHAPE), (dict(ldv=132), SHAPE), (dict(ldq=255), SHAPE),
    (dict(ldqo=128), SHAPE), (dict(k=P + 2), SHAPE), (dict(pos=P + 1), SHAPE), (dict(q_out=P, ldqo=512), SHAPE),
    (dict(tokens=(1 << 24) + 1), SHAPE), (dict(tokens=0, k=None, v=None, cu=None, first=None, pages=None), 0),
])
def test_append_refuses(lib, change, status):
    pg = pages()
    assert call(lib, "pf_op_kv_append_mx", dict(APPEND, pages=C.byref(pg), rope=rope64()), change) == status


def test_append_checks_its_rotation(lib):
    pg = pages(head_dim=32)
    sizes = dict(ldk=64, ldv=64, ldq=128, ldqo=128, rope=rope64())     # 64 channels to turn, heads of 32
    assert call(lib, "pf_op_kv_append_mx", dict(APPEND, pages=C.byref(pg)), sizes) == CONFIG


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), SHAPE), (dict(dtype=5), DTYPE), (dict(pages=None), NULL), (dict(cu=None), NULL), (dict(first=None), NULL),
    (dict(k_out=None, v_out=None), NULL), (dict(ldk=120), SHAPE), (dict(ldv=129), SHAPE), (dict(k_out=P + 8), SHAPE),
    (dict(v_out=P + 4), SHAPE), (dict(tokens=(1 << 24) + 1), SHAPE), (dict(tokens=0, cu=None, pages=None), 0),
])
def test_read_refuses(lib, change, status):
    pg = pages()
    assert call(lib, "pf_op_kv_read_mx", dict(READ, pages=C.byref(pg)), change) == status


@pytest.mark.parametrize("change,status", [
    (dict(total_q=-1), SHAPE), (dict(dtype=3), DTYPE), (dict(pages=None), NULL), (dict(q=None), NULL), (dict(cu_q=None), NULL),
    (dict(kv_len=None), NULL), (dict(first=None), NULL), (dict(out=None), NULL), (dict(heads=3), SHAPE), (dict(heads=0), SHAPE),
    (dict(ldq=128), SHAPE), (dict(ldo=250), SHAPE), (dict(q=P + 8), SHAPE), (dict(lse=P + 2), SHAPE), (dict(scale=math.nan), SHAPE),
    (dict(scale=math.inf), SHAPE), (dict(total_q=1 << 30), SHAPE), (dict(total_q=0, q=None, out=None, pages=None), 0),
])
def test_attention_refuses(lib, change, status):
    pg = pages()
    assert call(lib, "pf_op_attention_mx", dict(ATTEND, pages=C.byref(pg)), change) == status


def test_attention_asks_for_its_workspace(lib):
    pg = pages(n_pages=5000, max_pages=4096, n_seqs=1)
    sizes = (1, 0, 1, 1, 4, 2, 64, 4096 * 16)
    need = lib.pf_op_attention_mx_ws_bytes(*sizes)
    n = C.c_int()
    assert need > 0 and lib.pf_attention_mx_kernel_name(*sizes, C.byref(n)) and n.value > 1
    base = dict(ATTEND, pages=C.byref(pg), total_q=1)
    assert call(lib, "pf_op_attention_mx", base, {}) == WORKSPACE
    assert call(lib, "pf_op_attention_mx", base, dict(ws=P, ws_bytes=need - 1)) == WORKSPACE
    assert call(lib, "pf_op_attention_mx", base, dict(ws=P + 4, ws_bytes=need)) == WORKSPACE
    for bad in ((2, 0, 1, 1, 4, 2, 64, 4096), (1, 2, 1, 1, 4, 2, 64, 4096), (1, 0, 0, 1, 4, 2, 64, 4096), (1, 0, 1, 1, 4, 3, 64, 4096),
                (1, 0, 1, 1, 4, 2, 60, 4096), (1, 0, 1, 1, 4, 2, 64, 0), (1, 0, 1, 1, 4, 2, 64, 1 << 31)):
        assert lib.pf_op_attention_mx_ws_bytes(*bad) == 0 and lib.pf_attention_mx_kernel_name(*bad, None) == b""


def test_binding_refuses_host_tensors_and_wrong_formats(lib):
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)
    table = torch.zeros(1, 2, dtype=torch.int32)
    with pytest.raises(B.PfError) as e:
        B.KvMxPages("e5m2", u8(2, 1, 16, 64), u8(2, 1, 16, 64), u8(2, 1, 16, 2), u8(2, 1, 16, 2), table, 64)
    assert e.value.status == DTYPE
    with pytest.raises(B.PfError) as e:
        B.KvMxPages("e4m3", u8(2, 1, 16, 64), u8(2, 1, 16, 64), u8(2, 1, 16, 2), u8(2, 1, 16, 2), table, 64)
    assert e.value.status == SHAPE and "cpu" in str(e.value)
    with pytest.raises(B.PfError) as e:
        B.pf_op_qk_norm_rope(torch.zeros(3, 64), None, 64)
    assert e.value.status == SHAPE
    with pytest.raises(B.PfError) as e:
        B.pf_op_qk_norm_rope(None, None, 64)
    assert e.value.status == NULL


@pytest.mark.parametrize("fmt", [0, 1])
def test_workspace_of_tokens_is_bounded_whatever_the_table_holds(lib, fmt):
    """Partial results of at most 65536 tiles of 16 rows: a table with room for long caches costs no more than that, and none where there are more tiles."""
    n = C.c_int()
    for heads, kv_heads, dh in ((32, 8, 128), (24, 24, 64), (16, 1, 72), (128, 8, 128)):
        for tokens in (1, 5, 64, 256, 1024, 8192, 100000):
            for keys in (16, 1000, 4096, 16384, 131072, 1 << 20, (1 << 31) - 4096):
                sizes = (1, fmt, tokens, tokens, heads, kv_heads, dh, keys)
                need = lib.pf_op_attention_mx_ws_bytes(*sizes)
                name = lib.pf_attention_mx_kernel_name(*sizes, C.byref(n))
                assert b"few" in name and 1 <= n.value <= 256, sizes
                assert need == (0 if n.value == 1 else n.value * tokens * heads * (dh + 2) * 4), sizes
                assert need <= 65536 * 16 * (dh + 2) * 4 and n.value <= max(65536 // (tokens * kv_heads), 1), sizes
    assert lib.pf_op_attention_mx_ws_bytes(1, fmt, 8192, 8192, 32, 8, 128, 131072) == 0
