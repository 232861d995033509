"""Host side of the operators on packed rows: rotation tables, refusals and no-ops of the C entry points (nothing is launched, so the
pointers need not be real), and the binding's checks of tensors."""
import ctypes as C
import math
import os

import pytest
import torch

import requests_ref as R
from paper_2405_14430_amd import binding as B

P = 1 << 20   # stands for a device address, 16-byte aligned
NULL, CONFIG, SHAPE, DTYPE, WORKSPACE = -1, -2, -3, -4, -7


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2405_14430_amd.build import build
        build()
    return B.load_library()


@pytest.mark.parametrize("axes", [(64,), (128,), (2,), (16, 56, 56), (36, 36)])
@pytest.mark.parametrize("scaling,kw", [
    ("none", {}), ("linear", dict(factor=8.0)), ("ntk", dict(factor=4.0)),
    ("ramp_turns", dict(factor=8.0, low=1.0, high=4.0, original_len=8192)),
    ("ramp_index", dict(factor=16.0, low=1.0, high=32.0, original_len=4096)),
    ("ramp_index", dict(factor=2.0, low=50.0, high=60.0, original_len=64)),      # the whole ramp below pair 0
])
def test_rope_frequencies(lib, axes, scaling, kw):
    rope = B.make_rope(axes, theta=1e4, scaling=scaling, **kw)
    full = dict(factor=1.0, low=1.0, high=32.0, original_len=1)
    full.update(kw)
    want = torch.cat([R.frequencies(w, 1e4, scaling, **full) for w in axes])
    got = torch.tensor(list(rope.turns), dtype=torch.float64) * 2 * math.pi
    assert (got[:len(want)] / want - 1).abs().max() < 1e-13 and (got[len(want):] == 0).all()
    assert list(rope.axis_dim) == list(axes) + [0] * (3 - len(axes))


@pytest.mark.parametrize("kw", [
    dict(axis_dims=()), dict(axis_dims=(2, 2, 2, 2)), dict(axis_dims=(3,)), dict(axis_dims=(0,)), dict(axis_dims=(130,)),
    dict(axis_dims=(64, 64, 2)), dict(theta=1.0), dict(theta=math.inf), dict(theta=math.nan), dict(layout="split"),
    dict(scaling="cubic"), dict(scaling="linear", factor=0.5), dict(scaling="ntk", factor=math.nan),
    dict(scaling="ramp_turns", factor=2.0, low=4.0, high=4.0, original_len=100),
    dict(scaling="ramp_turns", factor=2.0, low=0.0, high=4.0, original_len=100),
    dict(scaling="ramp_index", factor=2.0, original_len=0), dict(magnitude=0.0), dict(magnitude=math.nan), dict(magnitude=math.inf),
])
def test_rope_init_refuses(lib, kw):
    kw = dict(dict(axis_dims=(64,)), **kw)
    with pytest.raises(B.PfError) as e:
        B.make_rope(**kw)
    assert e.value.status == CONFIG and str(e.value)


def rope64():
    return C.byref(B.make_rope((64,)))


def call(lib, name, base, change):
    args = dict(base)
    assert set(change) <= set(args)
    args.update(change)
    return getattr(lib, name)(*args.values())


ROPE = dict(dtype=1, rope=None, pos=P, x=P, ldx=256, out=2 * P, ldo=256, tokens=5, heads=4, dh=64, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), SHAPE), (dict(dtype=2), DTYPE), (dict(pos=None), NULL), (dict(x=None), NULL), (dict(out=None), NULL),
    (dict(heads=0), SHAPE), (dict(dh=60), SHAPE), (dict(dh=136), SHAPE), (dict(ldx=255), SHAPE), (dict(ldx=260), SHAPE),
    (dict(ldo=248), SHAPE), (dict(x=P + 8), SHAPE), (dict(out=P, ldo=264), SHAPE), (dict(dh=32, heads=8), CONFIG),
    (dict(tokens=0, x=None, out=None, pos=None), 0), (dict(pos=P + 2), SHAPE),
])
def test_rope_refuses(lib, change, status):
    assert call(lib, "pf_op_rope", dict(ROPE, rope=rope64()), change) == status
    if status:
        assert lib.pf_last_error(None)


def test_rope_checks_its_rotation(lib):
    assert call(lib, "pf_op_rope", ROPE, {}) == NULL
    for field, value in (("n_axes", 0), ("n_axes", 4), ("layout", 7), ("magnitude", math.nan)):
        r = B.make_rope((64,))
        setattr(r, field, value)
        assert call(lib, "pf_op_rope", dict(ROPE, rope=C.byref(r)), {}) == CONFIG, field
    r = B.make_rope((64,))
    r.axis_dim[0] = 63
    assert call(lib, "pf_op_rope", dict(ROPE, rope=C.byref(r)), {}) == CONFIG


def pages(**kw):
    f = dict(k=P, v=2 * P, k_page_stride=2 * 16 * 64, v_page_stride=2 * 16 * 64, table=P, n_pages=10, page_size=16, kv_heads=2,
             head_dim=64, n_seqs=3, max_pages=4)
    f.update(kw)
    return B.PfKvPages(**f)


BAD_PAGES = [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(table=None), NULL), (dict(page_size=24), SHAPE), (dict(page_size=8), SHAPE),
    (dict(page_size=2048, k_page_stride=1 << 20, v_page_stride=1 << 20), SHAPE), (dict(kv_heads=0), SHAPE), (dict(head_dim=12), SHAPE),
    (dict(head_dim=256, k_page_stride=1 << 20, v_page_stride=1 << 20), SHAPE), (dict(n_seqs=-1), SHAPE), (dict(max_pages=0), SHAPE),
    (dict(n_pages=0), SHAPE), (dict(k_page_stride=2047), SHAPE), (dict(v_page_stride=2052), SHAPE), (dict(k=P + 4), SHAPE),
    (dict(k_page_stride=1 << 60), SHAPE),
]
APPEND = dict(dtype=1, pages=None, k=P, ldk=128, v=P, ldv=128, cu=P, first=P, tokens=7, rope=None, pos=P, q=P, ldq=256, q_out=2 * P,
              ldqo=256, heads=4, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), SHAPE), (dict(heads=-1), SHAPE), (dict(dtype=9), DTYPE), (dict(k=None), NULL), (dict(v=None), NULL),
    (dict(cu=None), NULL), (dict(first=None), NULL), (dict(pos=None), NULL), (dict(q=None), NULL), (dict(q_out=None), NULL),
    (dict(heads=0), SHAPE), (dict(ldk=120), SHAPE), (dict(ldv=132), SHAPE), (dict(ldq=255), SHAPE), (dict(ldqo=128), SHAPE),
    (dict(k=P + 2), SHAPE), (dict(q_out=P, ldqo=512), SHAPE), (dict(tokens=0, k=None, v=None, cu=None, first=None), 0),
])
def test_append_refuses(lib, change, status):
    pg = pages()
    assert call(lib, "pf_op_kv_append", dict(APPEND, pages=C.byref(pg), rope=rope64()), change) == status


PACKED = dict(dtype=1, q=P, ldq=256, k=P, ldk=128, v=P, ldv=128, cu_q=P, cu_k=P, n_seqs=3, total_q=50, total_k=60, heads=4, kv_heads=2,
              dh=64, scale=0.0, causal=1, out=2 * P, ldo=256, lse=None, ws=None, ws_bytes=0, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(n_seqs=-1), SHAPE), (dict(total_q=-1), SHAPE), (dict(total_k=-2), SHAPE), (dict(dtype=3), DTYPE), (dict(q=None), NULL),
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(cu_q=None), NULL), (dict(cu_k=None), NULL), (dict(out=None), NULL),
    (dict(heads=3), SHAPE), (dict(heads=0), SHAPE), (dict(kv_heads=0), SHAPE), (dict(dh=4), SHAPE), (dict(dh=192), SHAPE),
    (dict(ldq=128), SHAPE), (dict(ldo=250), SHAPE), (dict(ldk=(1 << 20) + 8), SHAPE), (dict(ldv=100), SHAPE), (dict(scale=math.nan), SHAPE),
    (dict(scale=math.inf), SHAPE), (dict(lse=P + 2), SHAPE), (dict(total_q=1 << 30), SHAPE), (dict(v=P + 8), SHAPE),
    (dict(n_seqs=0, cu_q=None, cu_k=None), 0), (dict(total_q=0, q=None, out=None), 0),
])
def test_packed_refuses(lib, change, status):
    assert call(lib, "pf_op_attention_packed", PACKED, change) == status


PAGED = dict(dtype=1, q=P, ldq=256, pages=None, cu_q=P, first=P, kv_len=P, total_q=9, heads=4, scale=0.0, causal=1, out=2 * P, ldo=256,
             lse=None, ws=None, ws_bytes=0, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(total_q=-1), SHAPE), (dict(dtype=-1), DTYPE), (dict(q=None), NULL), (dict(cu_q=None), NULL), (dict(first=None), NULL),
    (dict(kv_len=None), NULL), (dict(out=None), NULL), (dict(heads=5), SHAPE), (dict(ldq=8), SHAPE), (dict(out=P + 8), SHAPE),
    (dict(total_q=0, q=None), 0),
])
def test_paged_refuses(lib, change, status):
    pg = pages()
    assert call(lib, "pf_op_attention_paged", dict(PAGED, pages=C.byref(pg)), change) == status


def test_scales_that_overflow_in_base_2_are_refused(lib):
    pg = pages()
    for scale in (3e38, 2.4e38, math.nan, math.inf):
        assert call(lib, "pf_op_attention_packed", PACKED, dict(scale=scale)) == SHAPE
        assert call(lib, "pf_op_attention_paged", dict(PAGED, pages=C.byref(pg)), dict(scale=scale)) == SHAPE
    for scale in (2e38, 0.0, -3e38):     # (stop at the workspace)
        assert call(lib, "pf_op_attention_packed", PACKED, dict(scale=scale, total_k=1 << 20)) == WORKSPACE


@pytest.mark.parametrize("change,status", BAD_PAGES)
def test_bad_pages_are_refused(lib, change, status):
    pg = pages(**change)
    assert call(lib, "pf_op_kv_append", dict(APPEND, pages=C.byref(pg), rope=rope64()), {}) == status
    assert call(lib, "pf_op_attention_paged", dict(PAGED, pages=C.byref(pg)), {}) == status
    assert call(lib, "pf_op_attention_paged", PAGED, {}) == NULL
    assert call(lib, "pf_op_kv_append", APPEND, {}) == NULL


def test_capacity_past_32_bits_is_refused(lib):
    pg = pages(max_pages=1 << 28)
    assert call(lib, "pf_op_attention_paged", dict(PAGED, pages=C.byref(pg)), {}) == SHAPE


def test_calls_without_rows_may_pass_null_for_everything(lib):
    none = lambda base: {k: None for k in base if base[k] == P or base[k] == 2 * P or base[k] == 3 * P or k in ("pages", "rope", "post", "pre")}
    for name, base, rows in (("pf_op_rope", ROPE, "tokens"), ("pf_op_kv_append", APPEND, "tokens"), ("pf_op_attention_packed", PACKED, "total_q"),
                             ("pf_op_attention_paged", PAGED, "total_q"), ("pf_op_norm_residual", NORM, "rows")):
        change = none(base)
        assert not any(v == P for v in dict(base, **change).values())
        assert call(lib, name, base, dict(change, **{rows: 0})) == 0, name
        assert call(lib, name, base, change) == NULL, name


@pytest.mark.parametrize("kw", [dict(axis_dims=(2 ** 32 + 64,)), dict(axis_dims=(64 - 2 ** 32,)),
                                dict(scaling="ramp_turns", factor=2.0, original_len=2 ** 32 + 4096)])
def test_rope_numbers_past_32_bits_are_refused(lib, kw):
    with pytest.raises(B.PfError) as e:
        B.make_rope(**dict(dict(axis_dims=(64,)), **kw))
    assert e.value.status == CONFIG


@pytest.mark.parametrize("n_seqs", [2 ** 30 + 1, 2 ** 31 - 64, 2 ** 31 - 1])
def test_more_sequences_than_the_search_counts_are_refused(lib, n_seqs):
    pg = pages(n_seqs=n_seqs)
    assert call(lib, "pf_op_kv_append", dict(APPEND, pages=C.byref(pg), rope=rope64()), {}) == SHAPE
    assert call(lib, "pf_op_attention_paged", dict(PAGED, pages=C.byref(pg)), {}) == SHAPE
    assert call(lib, "pf_op_attention_packed", PACKED, dict(n_seqs=n_seqs)) == SHAPE
    assert call(lib, "pf_op_norm_residual", NORM, dict(n_seqs=n_seqs)) == SHAPE


def test_rows_past_the_documented_ones_are_refused(lib):
    pg, n = pages(), 2 ** 24 + 1
    assert call(lib, "pf_op_rope", dict(ROPE, rope=rope64()), dict(tokens=n)) == SHAPE
    assert call(lib, "pf_op_kv_append", dict(APPEND, pages=C.byref(pg), rope=rope64()), dict(tokens=n)) == SHAPE
    assert call(lib, "pf_op_norm_residual", NORM, dict(rows=n)) == SHAPE
    # 2^24 workgroups of 32 rows, two key heads with two query heads each
    assert call(lib, "pf_op_attention_packed", PACKED, dict(total_q=2 ** 27, total_k=1)) == SHAPE
    assert call(lib, "pf_op_attention_paged", dict(PAGED, pages=C.byref(pg)), dict(total_q=2 ** 27)) == SHAPE


def test_keys_past_what_32_bits_can_round_up_are_refused(lib):
    most = 2 ** 31 - 4096
    for n, status in ((most, WORKSPACE), (most + 1, SHAPE), (2 ** 31 - 1, SHAPE)):
        assert call(lib, "pf_op_attention_packed", PACKED, dict(total_k=n)) == status, n
    for max_pages, status in ((most // 16, WORKSPACE), (most // 16 + 1, SHAPE)):
        pg = pages(max_pages=max_pages)
        assert call(lib, "pf_op_attention_paged", dict(PAGED, pages=C.byref(pg)), {}) == status, max_pages
    assert lib.pf_op_attention_rows_ws_bytes(1, 50, 3, 4, 2, 64, most) > 0 and lib.pf_attention_rows_kernel_name(1, 50, 3, 4, 2, 64, most, None)
    assert lib.pf_op_attention_rows_ws_bytes(1, 50, 3, 4, 2, 64, most + 1) == 0
    assert lib.pf_attention_rows_kernel_name(1, 50, 3, 4, 2, 64, most + 1, None) == b""


def test_workspace_bytes(lib):
    f = lib.pf_op_attention_rows_ws_bytes
    for bad in ((2, 1, 1, 4, 2, 64, 10), (1, 0, 1, 4, 2, 64, 10), (1, 1, 0, 4, 2, 64, 10), (1, 1, 1, 5, 2, 64, 10),
                (1, 1, 1, 4, 2, 60, 10), (1, 1, 1, 4, 2, 64, 0)):
        assert f(*bad) == 0
    # a launch that fills the chip with query rows needs none, whatever the keys
    assert f(1, 1 << 20, 4, 8, 8, 64, 1 << 20) == 0


NORM = dict(dtype=1, y=P, ldy=512, post=None, gate=P, gate_stride=512, tanh=1, x_scale=1.0, x=P, ldx=512, x_out=2 * P, ldxo=512, pre=None,
            shift=P, scale=P, mod_stride=512, h=3 * P, ldh=512, cu=P, n_seqs=2, rows=8, d=512, stream=None)


def norm(kind=1, eps=1e-6, weight=P, bias=None):
    return C.byref(B.PfNorm(kind=kind, eps=eps, weight=weight, bias=bias))


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), SHAPE), (dict(n_seqs=-1), SHAPE), (dict(dtype=2), DTYPE), (dict(x=None), NULL), (dict(x_out=None, h=None), NULL),
    (dict(d=4), SHAPE), (dict(d=12), SHAPE), (dict(d=8200), SHAPE), (dict(ldx=511), SHAPE), (dict(ldy=514), SHAPE), (dict(ldxo=8), SHAPE),
    (dict(ldh=510), SHAPE), (dict(x=P + 8), SHAPE), (dict(y=P + 4), SHAPE), (dict(gate=P + 4), SHAPE), (dict(gate_stride=5), SHAPE),
    (dict(mod_stride=2), SHAPE), (dict(x_out=P, ldxo=1024), SHAPE), (dict(h=P, ldh=1024), SHAPE),
    (dict(rows=0, x=None, x_out=None, h=None), 0), (dict(n_seqs=0), 0),
])
def test_norm_refuses(lib, change, status):
    assert call(lib, "pf_op_norm_residual", dict(NORM, post=norm(), pre=norm()), change) == status


@pytest.mark.parametrize("bad,status", [(dict(kind=3), CONFIG), (dict(kind=-1), CONFIG), (dict(eps=-1.0), CONFIG), (dict(eps=math.nan), CONFIG),
                                        (dict(weight=P + 4), SHAPE), (dict(bias=P + 2), SHAPE), (dict(kind=0), CONFIG)])
def test_norm_refuses_bad_norms(lib, bad, status):
    assert call(lib, "pf_op_norm_residual", dict(NORM, post=norm(**bad)), {}) == status
    assert call(lib, "pf_op_norm_residual", dict(NORM, pre=norm(**bad)), {}) == status


def test_binding_refuses_tensors_that_are_not_on_a_gpu(lib):
    x, i = torch.zeros(4, 64), torch.zeros(4, 1, dtype=torch.int32)
    rope = B.make_rope((64,))
    for f in (lambda: B.pf_op_rope(x, rope, i, 64),
              lambda: B.KvPages(torch.zeros(2, 1, 16, 64), torch.zeros(2, 1, 16, 64), torch.zeros(1, 1, dtype=torch.int32)),
              lambda: B.pf_op_attention_packed(x, x, x, i[:2, 0], i[:2, 0], 64),
              lambda: B.pf_op_norm_residual(x, x),
              lambda: B.make_norm("rms", torch.zeros(64))):
        with pytest.raises(B.PfError):
            f()
    with pytest.raises(B.PfError):
        B.make_norm("batch")


def test_reference_attention_of_a_row_that_sees_nothing():
    """The 64-bit forms themselves: an empty row is zero with log-sum-exp -inf, and NaN behind the mask does not reach it."""
    q, k, v = torch.randn(3, 8), torch.randn(4, 8), torch.full((4, 8), math.nan)
    v[0] = 1.0
    out, lse, *_ = R.attention(q, k, v, 8, torch.tensor([0, 1, 1]))
    assert (out[0] == 0).all() and lse[0] == -math.inf and (out[1:] - 1).abs().max() < 1e-15


def test_reference_attention_equals_torch():
    q, k, v = torch.randn(5, 16, dtype=torch.float64), torch.randn(9, 8, dtype=torch.float64), torch.randn(9, 8, dtype=torch.float64)
    out = R.attention(q, k, v, 8, torch.arange(5) + 5)[0]
    mask = torch.arange(9)[None] < (torch.arange(5) + 5)[:, None]
    for h in range(2):
        want = torch.nn.functional.scaled_dot_product_attention(q[None, None, :, 8 * h:8 * h + 8], k[None, None], v[None, None], attn_mask=mask)[0, 0]
        assert (out[:, 8 * h:8 * h + 8] - want).abs().max() < 1e-14


LISTING = """
_Zkernel:                               ; @_Zkernel
; %bb.0:
\tv_accvgpr_write_b32 a0, 0
\ts_and_saveexec_b64 s[0:1], vcc
\ts_cbranch_execz .LBB0_2
; %bb.1:
\tv_accvgpr_write_b32 a1, v3
{in_branch}
.LBB0_2:                                ; %join
{in_front}
\ts_or_b64 exec, exec, s[0:1]
\tv_accvgpr_read_b32 v4, a0
\ts_cbranch_execz .LBB0_3
{behind}
.LBB0_3:
\ts_endpgm
\t.amdhsa_kernel _Zkernel
"""


def test_build_refuses_register_moves_in_front_of_activated_lanes():
    from paper_2405_14430_amd import build as bld
    listing = lambda **kw: LISTING.format(**dict(dict(in_branch="", in_front="", behind=""), **kw))
    bld._check_moves("attn_rows.hip", listing())
    bld._check_moves("attn_rows.hip", listing(in_branch="\tv_accvgpr_write_b32 a2, v5", in_front="\tv_mov_b32_e32 v1, v2"))
    for bad in (dict(in_front="\tv_accvgpr_write_b32 a2, v5"), dict(in_front="\tv_accvgpr_read_b32 v5, a2 ; saved"),
                dict(in_branch="\tv_accvgpr_write_b32 a2, v5\n\ts_xor_b64 exec, exec, s[2:3]"),
                dict(behind="\ts_mov_b64 exec, -1"), dict(behind="\ts_or_saveexec_b64 s[2:3], -1")):
        with pytest.raises(RuntimeError, match="_Zkernel"):
            bld._check_moves("attn_rows.hip", listing(**bad))
    with pytest.raises(RuntimeError):
        bld._check_moves("attn_rows.hip", "")
