"""ctypes binding of libpfstage.so: argument marshalling only.

Function names mirror include/pfstage.h.  torch is used for device memory and streams;
every arithmetic step runs inside the library's HIP kernels.  Loading fails loudly when the
library has not been built (python paper_2405_14430_amd/build.py, or __graft_entry__.build()).
"""
from __future__ import annotations

import ctypes as C
import functools
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpfstage.so")

PF_F32, PF_BF16 = 0, 1
PF_PATH_AUTO, PF_PATH_SIMT, PF_PATH_AUTO_PRESCALED_Q = 0, 1, 2
KERNEL_CLASSES = ["modulation", "ln_modulate", "gemm_qkv", "kv_scatter", "attention", "attn_combine",
                  "gemm_out", "gemm_xattn", "xattn", "gemm_up", "gemm_down", "copy"]
STATUS = {0: "PF_OK", -1: "PF_ERR_NULL", -2: "PF_ERR_CONFIG", -3: "PF_ERR_SHAPE", -4: "PF_ERR_DTYPE",
          -5: "PF_ERR_STATE", -6: "PF_ERR_RANGE", -7: "PF_ERR_WORKSPACE", -8: "PF_ERR_DEVICE"}


class PfConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("kind", "dtype", "n_layers", "hidden", "n_heads", "head_dim", "mlp_dim",
                                          "seq_img", "n_patches", "text_len", "cross_dim", "grid_h", "grid_w")] + \
               [("ln_eps", C.c_float), ("rope_theta", C.c_float), ("gelu_tanh", C.c_int32), ("kernel_path", C.c_int32), ("batch", C.c_int32),
                ("qk_norm", C.c_int32), ("joint_rope", C.c_int32), ("txt_pre_only_last", C.c_int32)]


class PfLayerWeights(C.Structure):
    pass


_W_FIELDS = ["w_mod", "b_mod", "w_qkv", "b_qkv", "w_o", "b_o", "w_up", "b_up", "w_down", "b_down",
             "xattn_wq", "xattn_bq", "xattn_wkv", "xattn_bkv", "xattn_wo", "xattn_bo", "q_norm_w", "k_norm_w"]
PfLayerWeights._fields_ = [(n, C.c_void_p) for n in _W_FIELDS] + [("txt", C.POINTER(PfLayerWeights))]


class PfCond(C.Structure):
    _fields_ = [("cond", C.c_void_p), ("text", C.c_void_p), ("text_out", C.c_void_p), ("same_cond", C.c_int32)]


class PfKvView(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("rows", C.c_int32), ("rows_padded", C.c_int32),
                ("text_rows", C.c_int32), ("elem_bytes", C.c_int32),
                ("k_row_stride", C.c_int64), ("k_head_stride", C.c_int64), ("k_col_stride", C.c_int64),
                ("v_row_stride", C.c_int64), ("v_head_stride", C.c_int64), ("v_col_stride", C.c_int64)]


EXPORTS = ["pf_stage_kv_bytes", "pf_stage_workspace_bytes", "pf_stage_create", "pf_kv_init",
           "pf_stage_patch_forward", "pf_kv_view", "pf_xattn_kv_view", "pf_stage_attention_plan", "pf_stage_qkv_plan", "pf_stage_set_stream",
           "pf_stage_profile",
           "pf_stage_profile_read", "pf_stage_destroy", "pf_status_str", "pf_last_error", "pf_op_modulation",
           "pf_op_ln_modulate", "pf_op_gemm", "pf_op_kv_scatter", "pf_op_attention_ws_bytes", "pf_op_attention", "pf_attention_kernel_name", "pf_probe_mfma_loop",
           "pf_gemm_tile_count", "pf_gemm_tile_map", "pf_gemm_read_ahead", "pf_op_gemm_tile", "pf_static_scratch_bytes", "pf_op_attention_static", "pf_gemm_kernel_name", "pf_gemm_qkv_kernel_name", "pf_op_axpy", "pf_kv_view_image", "pf_op_axpby",
           "pf_rope_init", "pf_op_rope", "pf_op_kv_append", "pf_op_attention_rows_ws_bytes", "pf_op_attention_packed",
           "pf_op_attention_paged", "pf_op_norm_residual", "pf_attention_rows_kernel_name"]

PF_ROPE_MAX_AXES, PF_ROPE_MAX_PAIRS = 3, 64
ROPE_LAYOUTS = {"interleaved": 0, "half": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "ramp_turns": 3, "ramp_index": 4}
NORM_KINDS = {"none": 0, "rms": 1, "layer": 2}


class PfRopeConfig(C.Structure):
    _fields_ = [("layout", C.c_int32), ("n_axes", C.c_int32), ("axis_dim", C.c_int32 * PF_ROPE_MAX_AXES), ("theta", C.c_float),
                ("scaling", C.c_int32), ("factor", C.c_float), ("low", C.c_float), ("high", C.c_float),
                ("original_len", C.c_int32), ("magnitude", C.c_float)]


class PfRope(C.Structure):
    _fields_ = [("layout", C.c_int32), ("n_axes", C.c_int32), ("axis_dim", C.c_int32 * PF_ROPE_MAX_AXES),
                ("magnitude", C.c_float), ("turns", C.c_double * PF_ROPE_MAX_PAIRS)]


class PfKvPages(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_page_stride", C.c_int64), ("v_page_stride", C.c_int64),
                ("table", C.c_void_p), ("n_pages", C.c_int32), ("page_size", C.c_int32), ("kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("n_seqs", C.c_int32), ("max_pages", C.c_int32)]


class PfNorm(C.Structure):
    _fields_ = [("kind", C.c_int32), ("eps", C.c_float), ("weight", C.c_void_p), ("bias", C.c_void_p)]


_lib = None


def load_library():
    """dlopen libpfstage.so and declare the prototypes.  Raises if the library is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it first (python paper_2405_14430_amd/build.py). "
                           "There is no fallback path.")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, f32, sz = C.c_void_p, C.c_int, C.c_int64, C.c_float, C.c_size_t
    lib.pf_stage_kv_bytes.restype = sz
    lib.pf_stage_kv_bytes.argtypes = [C.POINTER(PfConfig)]
    lib.pf_stage_workspace_bytes.restype = sz
    lib.pf_stage_workspace_bytes.argtypes = [C.POINTER(PfConfig)]
    lib.pf_stage_create.restype = i32
    lib.pf_stage_create.argtypes = [C.POINTER(PfConfig), C.POINTER(PfLayerWeights), vp, sz, vp, sz, vp, C.POINTER(vp)]
    lib.pf_kv_init.restype = i32
    lib.pf_kv_init.argtypes = [vp, vp, C.POINTER(PfCond), vp]
    lib.pf_stage_patch_forward.restype = i32
    lib.pf_stage_patch_forward.argtypes = [vp, vp, C.POINTER(PfCond), i32, vp]
    lib.pf_kv_view.restype = i32
    lib.pf_kv_view.argtypes = [vp, i32, C.POINTER(PfKvView)]
    lib.pf_xattn_kv_view.restype = i32
    lib.pf_xattn_kv_view.argtypes = [vp, i32, C.POINTER(PfKvView)]
    lib.pf_kv_view_image.restype = i32
    lib.pf_kv_view_image.argtypes = [vp, i32, i32, i32, C.POINTER(PfKvView)]
    lib.pf_stage_attention_plan.restype = i32
    lib.pf_stage_attention_plan.argtypes = [vp, i32, i32, C.POINTER(C.c_int), C.POINTER(sz), C.POINTER(sz)]
    lib.pf_stage_qkv_plan.restype = i32
    lib.pf_stage_qkv_plan.argtypes = [vp, i32, i32, C.POINTER(C.c_int), C.POINTER(C.c_int), C.POINTER(C.c_int)]
    lib.pf_stage_set_stream.restype = i32
    lib.pf_stage_set_stream.argtypes = [vp, vp]
    lib.pf_stage_profile.restype = i32
    lib.pf_stage_profile.argtypes = [vp, i32]
    lib.pf_stage_profile_read.restype = i32
    lib.pf_stage_profile_read.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_int64)]
    lib.pf_stage_destroy.restype = None
    lib.pf_stage_destroy.argtypes = [vp]
    lib.pf_status_str.restype = C.c_char_p
    lib.pf_status_str.argtypes = [i32]
    lib.pf_last_error.restype = C.c_char_p
    lib.pf_last_error.argtypes = [vp]
    lib.pf_op_modulation.restype = i32
    lib.pf_op_modulation.argtypes = [i32, vp, vp, vp, vp, i32, i32, i32, vp]
    lib.pf_op_ln_modulate.restype = i32
    lib.pf_op_ln_modulate.argtypes = [i32, vp, i64, vp, vp, f32, vp, i64, i32, i32, i32, vp]
    lib.pf_op_gemm.restype = i32
    lib.pf_op_gemm.argtypes = [i32, i32, vp, i64, vp, i64, vp, vp, i64, i32, i32, i32, i32, i32, i32, vp, vp, i64,
                               vp, i64, vp]
    lib.pf_op_kv_scatter.restype = i32
    lib.pf_op_kv_scatter.argtypes = [i32, vp, i64, vp, vp, i32, i32, i32, i32, i32, i32, i32, i32, f32, vp, vp, f32, vp]
    lib.pf_attention_kernel_name.restype = C.c_char_p
    lib.pf_attention_kernel_name.argtypes = [i32, i32, i32, i32, i32]
    lib.pf_probe_mfma_loop.restype = i32
    lib.pf_probe_mfma_loop.argtypes = [vp, i32, i32, C.POINTER(C.c_double), vp]
    lib.pf_op_attention_ws_bytes.restype = sz
    lib.pf_op_attention_ws_bytes.argtypes = [i32, i32, i32, i32]
    lib.pf_op_attention.restype = i32
    lib.pf_op_attention.argtypes = [i32, i32, vp, i64, vp, vp, i32, i32, i32, i32, vp, i64, i32, i32, vp, sz, vp]
    lib.pf_static_scratch_bytes.restype = sz
    lib.pf_static_scratch_bytes.argtypes = []
    lib.pf_op_attention_static.restype = i32
    lib.pf_op_attention_static.argtypes = [i32, i32, vp, i64, vp, vp, i32, i32, i32, i32, vp, i64, i32, i32, vp]
    lib.pf_gemm_kernel_name.restype = C.c_char_p
    lib.pf_gemm_kernel_name.argtypes = [i32, i32, i32, i32, i32]
    lib.pf_gemm_qkv_kernel_name.restype = C.c_char_p
    lib.pf_gemm_qkv_kernel_name.argtypes = [i32, i32, i32, i32]
    lib.pf_op_axpy.restype = i32
    lib.pf_op_axpy.argtypes = [vp, vp, f32, vp, i64, vp]
    lib.pf_op_axpby.restype = i32
    lib.pf_op_axpby.argtypes = [vp, vp, f32, f32, vp, i64, vp]
    lib.pf_gemm_tile_count.restype = i32
    lib.pf_gemm_tile_count.argtypes = []
    lib.pf_gemm_tile_map.restype = i32
    lib.pf_gemm_tile_map.argtypes = [i32, i32, i32, i32, C.c_uint, C.POINTER(C.c_uint), C.POINTER(i32), C.POINTER(i32)]
    lib.pf_gemm_read_ahead.restype = i32
    lib.pf_gemm_read_ahead.argtypes = [i32, i32, i32]
    lib.pf_op_gemm_tile.restype = i32
    lib.pf_op_gemm_tile.argtypes = [i32] + lib.pf_op_gemm.argtypes
    lib.pf_rope_init.restype = i32
    lib.pf_rope_init.argtypes = [C.POINTER(PfRopeConfig), C.POINTER(PfRope)]
    lib.pf_op_rope.restype = i32
    lib.pf_op_rope.argtypes = [i32, C.POINTER(PfRope), vp, vp, i64, vp, i64, i32, i32, i32, vp]
    lib.pf_op_kv_append.restype = i32
    lib.pf_op_kv_append.argtypes = [i32, C.POINTER(PfKvPages), vp, i64, vp, i64, vp, vp, i32, C.POINTER(PfRope), vp, vp, i64,
                                    vp, i64, i32, vp]
    lib.pf_op_attention_rows_ws_bytes.restype = sz
    lib.pf_op_attention_rows_ws_bytes.argtypes = [i32, i32, i32, i32, i32, i32, i64]
    lib.pf_attention_rows_kernel_name.restype = C.c_char_p
    lib.pf_attention_rows_kernel_name.argtypes = [i32, i32, i32, i32, i32, i32, i64, C.POINTER(i32)]
    lib.pf_op_attention_packed.restype = i32
    lib.pf_op_attention_packed.argtypes = [i32, vp, i64, vp, i64, vp, i64, vp, vp, i32, i32, i32, i32, i32, i32, f32, i32, vp,
                                           i64, vp, vp, sz, vp]
    lib.pf_op_attention_paged.restype = i32
    lib.pf_op_attention_paged.argtypes = [i32, vp, i64, C.POINTER(PfKvPages), vp, vp, vp, i32, i32, f32, i32, vp, i64, vp, vp,
                                          sz, vp]
    lib.pf_op_norm_residual.restype = i32
    lib.pf_op_norm_residual.argtypes = [i32, vp, i64, C.POINTER(PfNorm), vp, i64, i32, f32, vp, i64, vp, i64, C.POINTER(PfNorm),
                                        vp, vp, i64, vp, i64, vp, i32, i32, i32, vp]
    _lib = lib
    return lib


class PfError(RuntimeError):
    def __init__(self, status, msg=""):
        self.status = status
        super().__init__(f"{STATUS.get(status, status)}: {msg}")


def make_config(cfg, kernel_path=PF_PATH_AUTO, n_layers=None):
    return PfConfig(kind=cfg["kind"], dtype=PF_BF16 if cfg["dtype"] == "bf16" else PF_F32,
                    n_layers=cfg["n_layers"] if n_layers is None else n_layers, hidden=cfg["hidden"],
                    n_heads=cfg["n_heads"], head_dim=cfg["head_dim"], mlp_dim=cfg["mlp_dim"],
                    seq_img=cfg["seq_img"], n_patches=cfg["n_patches"], text_len=cfg.get("text_len", 0),
                    cross_dim=cfg.get("cross_dim", 0), grid_h=cfg["grid_h"], grid_w=cfg["grid_w"],
                    ln_eps=cfg.get("ln_eps", 1e-6), rope_theta=cfg.get("rope_theta", 1e4),
                    gelu_tanh=cfg.get("gelu_tanh", 1), kernel_path=kernel_path, batch=cfg.get("batch", 1),
                    qk_norm=cfg.get("qk_norm", 0), joint_rope=cfg.get("joint_rope", 0),
                    txt_pre_only_last=cfg.get("txt_pre_only_last", 0))


def torch_dtype(cfg):
    return torch.bfloat16 if cfg["dtype"] == "bf16" else torch.float32


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream_ptr(stream=None):
    s = torch.cuda.current_stream() if stream is None else stream
    return C.c_void_p(s.cuda_stream)


def to_device(a, dtype, device="cuda"):
    """numpy float32 array (values already representable in dtype) -> device tensor of dtype."""
    return torch.from_numpy(np.ascontiguousarray(a)).to(device=device, dtype=dtype)


class Stage:
    """Owns the device memory of one stage (weights, K/V buffer, workspace) and forwards calls to the library."""

    def __init__(self, cfg, layers, kernel_path=PF_PATH_AUTO, device="cuda", stream=None):
        self.lib = load_library()
        self.cfg = dict(cfg)
        self.device = device
        self.dt = torch_dtype(cfg)
        self.c = make_config(cfg, kernel_path, n_layers=len(layers))
        self.n = cfg["seq_img"] // cfg["n_patches"]
        self.d = cfg["hidden"]
        self.T = cfg.get("text_len", 0)
        self.joint = cfg["kind"] in (2, 3)
        self._keep = []
        arr = (PfLayerWeights * len(layers))()
        self._txt = (PfLayerWeights * len(layers))()
        for i, w in enumerate(layers):
            self._fill(arr[i], w)
            if "txt" in w:
                self._fill(self._txt[i], w["txt"])
                arr[i].txt = C.pointer(self._txt[i])
        self._layers = arr
        kvb = self.lib.pf_stage_kv_bytes(C.byref(self.c))
        wsb = self.lib.pf_stage_workspace_bytes(C.byref(self.c))
        if kvb == 0:
            raise PfError(-2, "invalid configuration")
        self.kv = torch.zeros(kvb, dtype=torch.uint8, device=device)
        self.ws = torch.empty(wsb, dtype=torch.uint8, device=device)
        self.h = C.c_void_p()
        st = self.lib.pf_stage_create(C.byref(self.c), arr, _ptr(self.kv), kvb, _ptr(self.ws), wsb,
                                      _stream_ptr(stream), C.byref(self.h))
        if st != 0:
            raise PfError(st, self.lib.pf_last_error(None).decode())

    def _fill(self, dst, w):
        for name in _W_FIELDS:
            if name in w:
                t = to_device(w[name], self.dt, self.device)
                self._keep.append(t)
                setattr(dst, name, t.data_ptr())

    def _check(self, st):
        if st != 0:
            raise PfError(st, self.lib.pf_last_error(self.h).decode())

    def _cond(self, cond, text, text_out, same_cond=False):
        return PfCond(cond=None if cond is None else cond.data_ptr(), text=None if text is None else text.data_ptr(),
                      text_out=None if text_out is None else text_out.data_ptr(), same_cond=int(bool(same_cond)))

    def kv_init(self, x_prev=None, cond=None, text=None, want_output=False):
        """x_prev/cond/text: device tensors (x_prev, cond, joint text: float32; kind-1 text: stage dtype).  A stage with
        batch B > 1 takes every array with a leading image axis of length B."""
        y = torch.empty_like(x_prev) if (want_output and x_prev is not None) else None
        tout = torch.empty_like(text) if (want_output and self.joint and text is not None and x_prev is not None) else None
        pc = self._cond(cond, text, tout)
        self._check(self.lib.pf_kv_init(self.h, _ptr(x_prev), C.byref(pc), _ptr(y)))
        return (y, tout) if want_output else None

    def patch_forward(self, x_patch, cond, p, text=None, out=None, text_out=None, same_cond=False):
        """same_cond: `cond` has the values of this stage's previous call (the other patches of the same diffusion
        step): the stage reuses its modulation vectors instead of deriving them again."""
        y = torch.empty_like(x_patch) if out is None else out
        if self.joint and text is not None and text_out is None:
            text_out = torch.empty_like(text)
        pc = self._cond(cond, text if self.joint else None, text_out, same_cond)
        self._check(self.lib.pf_stage_patch_forward(self.h, _ptr(x_patch), C.byref(pc), int(p), _ptr(y)))
        return (y, text_out) if (self.joint and text is not None) else y

    def _view(self, layer, image, cross):
        v = PfKvView()
        self._check(self.lib.pf_kv_view_image(self.h, layer, image, int(cross), C.byref(v)))
        typed = self.kv.view(self.dt)
        H, dh, esz = self.cfg["n_heads"], self.cfg["head_dim"], v.elem_bytes
        ko = (v.k - self.kv.data_ptr()) // esz
        vo = (v.v - self.kv.data_ptr()) // esz
        K = typed.as_strided((v.rows, H, dh), (v.k_row_stride, v.k_head_stride, v.k_col_stride), ko)
        V = typed.as_strided((v.rows, H, dh), (v.v_row_stride, v.v_head_stride, v.v_col_stride), vo)
        return K, V, v

    def kv_view(self, layer, image=0):
        """(K, V) as strided [rows, H, dh] tensor views into the caller-owned buffer, plus the raw view struct."""
        return self._view(layer, image, False)

    def xattn_kv_view(self, layer, image=0):
        return self._view(layer, image, True)

    def set_stream(self, stream):
        self._check(self.lib.pf_stage_set_stream(self.h, _stream_ptr(stream)))

    def profile(self, enable):
        self._check(self.lib.pf_stage_profile(self.h, int(enable)))

    def profile_read(self):
        ms = (C.c_double * len(KERNEL_CLASSES))()
        cnt = (C.c_int64 * len(KERNEL_CLASSES))()
        self._check(self.lib.pf_stage_profile_read(self.h, ms, cnt))
        return {k: (ms[i], cnt[i]) for i, k in enumerate(KERNEL_CLASSES)}

    def destroy(self):
        if self.h:
            self.lib.pf_stage_destroy(self.h)
            self.h = C.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


# ---- single-operator wrappers (device tensors in, device tensors out) ---------------------------------------
def _dt_code(t):
    return PF_BF16 if t.dtype == torch.bfloat16 else PF_F32


def _ok(st):
    if st != 0:
        raise PfError(st)


def pf_op_modulation(w, b, c, table_mode=False):
    lib = load_library()
    out_dim = w.numel() if table_mode else w.shape[0]
    in_dim = w.shape[-1]
    mod = torch.empty(out_dim, dtype=torch.float32, device=w.device)
    _ok(lib.pf_op_modulation(_dt_code(w), _ptr(w), _ptr(b), _ptr(c), _ptr(mod), out_dim, in_dim, int(table_mode),
                             _stream_ptr()))
    return mod


def pf_op_ln_modulate(x, shift, scale, eps, dtype, normalize=True):
    lib = load_library()
    rows, d = x.shape
    out = torch.empty(rows, d, dtype=dtype, device=x.device)
    _ok(lib.pf_op_ln_modulate(PF_BF16 if dtype == torch.bfloat16 else PF_F32, _ptr(x), x.stride(0), _ptr(shift),
                              _ptr(scale), eps, _ptr(out), out.stride(0), rows, d, int(normalize), _stream_ptr()))
    return out


def pf_op_gemm(A, W, bias, epilogue=0, gelu_from=None, gelu_tanh=1, gate=None, R=None, want_copy=False,
               path=PF_PATH_AUTO, tile=0):
    """epilogue 0 -> dtype [M,N]; epilogue 1 -> (float32 [M,N] new residual, optional dtype copy).
    tile > 0 goes through pf_op_gemm_tile (one tile configuration of the bf16 kernel, this launch only)."""
    lib = load_library()
    M, K = A.shape
    N = W.shape[0]
    if epilogue == 0:
        Cc = torch.empty(M, N, dtype=A.dtype, device=A.device)
        C2 = None
    else:
        Cc = torch.empty(M, N, dtype=torch.float32, device=A.device)
        C2 = torch.empty(M, N, dtype=A.dtype, device=A.device) if want_copy else None
    args = (_dt_code(A), path, _ptr(A), A.stride(0), _ptr(W), W.stride(0), _ptr(bias), _ptr(Cc),
            Cc.stride(0), M, N, K, epilogue, N if gelu_from is None else gelu_from, gelu_tanh, _ptr(gate),
            _ptr(R), 0 if R is None else R.stride(0), _ptr(C2), 0 if C2 is None else C2.stride(0), _stream_ptr())
    _ok(lib.pf_op_gemm_tile(int(tile), *args) if tile else lib.pf_op_gemm(*args))
    return Cc if epilogue == 0 else (Cc, C2)


def pf_op_kv_scatter(qkv, kbuf, vtbuf, rows_padded, n_heads, head_dim, row0, rope=False, tok0=-1, grid_w=1,
                     theta=1e4, q_norm_w=None, k_norm_w=None, norm_eps=1e-6):
    lib = load_library()
    _ok(lib.pf_op_kv_scatter(_dt_code(qkv), _ptr(qkv), qkv.stride(0), _ptr(kbuf), _ptr(vtbuf), rows_padded, n_heads,
                             head_dim, row0, qkv.shape[0], int(rope), tok0, grid_w, theta, _ptr(q_norm_w),
                             _ptr(k_norm_w), norm_eps, _stream_ptr()))


def pf_op_attention(q, kbuf, vtbuf, kv_rows, rows_padded, n_heads, head_dim, splits=1, path=PF_PATH_AUTO):
    lib = load_library()
    nq = q.shape[0]
    out = torch.empty(nq, n_heads * head_dim, dtype=q.dtype, device=q.device)
    wsb = lib.pf_op_attention_ws_bytes(nq, n_heads, head_dim, splits)
    ws = torch.empty(max(wsb, 16), dtype=torch.uint8, device=q.device)
    _ok(lib.pf_op_attention(_dt_code(q), path, _ptr(q), q.stride(0), _ptr(kbuf), _ptr(vtbuf), kv_rows, rows_padded,
                            n_heads, head_dim, _ptr(out), out.stride(0), nq, splits, _ptr(ws), wsb, _stream_ptr()))
    return out


def pf_op_attention_static(q, kbuf, vtbuf, kv_rows, rows_padded, n_heads, head_dim, out, splits=1, path=PF_PATH_AUTO):
    """pf_op_attention through the entry point that allocates nothing: `out` is the caller's, the split partials go into
    the library's static scratch array."""
    lib = load_library()
    st = lib.pf_op_attention_static(_dt_code(q), path, _ptr(q), q.stride(0), _ptr(kbuf), _ptr(vtbuf), kv_rows, rows_padded,
                                    n_heads, head_dim, _ptr(out), out.stride(0), q.shape[0], splits, _stream_ptr())
    if st != 0:
        raise PfError(st, lib.pf_last_error(None).decode())
    return out


def probe_mfma_tflops(workgroups=512, iters=4000):
    """TFLOP/s of a register-only bf16 MFMA loop on the current device and stream (measured ceiling of the matrix pipes)."""
    lib = load_library()
    out = torch.empty(workgroups * 256, dtype=torch.float32, device="cuda")
    fl = C.c_double()
    _ok(lib.pf_probe_mfma_loop(_ptr(out), workgroups, 50, C.byref(fl), _stream_ptr()))      # warm-up
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    _ok(lib.pf_probe_mfma_loop(_ptr(out), workgroups, iters, C.byref(fl), _stream_ptr()))
    e1.record()
    e1.synchronize()
    return fl.value / (e0.elapsed_time(e1) * 1e-3) / 1e12


def pf_op_axpy(x, y, alpha, out=None):
    lib = load_library()
    out = torch.empty_like(x) if out is None else out
    _ok(lib.pf_op_axpy(_ptr(x), _ptr(y), float(alpha), _ptr(out), x.numel(), _stream_ptr()))
    return out


def pf_op_axpby(x, y, a, b, out=None):
    lib = load_library()
    out = torch.empty_like(x) if out is None else out
    _ok(lib.pf_op_axpby(_ptr(x), _ptr(y), float(a), float(b), _ptr(out), x.numel(), _stream_ptr()))
    return out


# ---- operators on packed rows: requests of different sizes in one call -----------------------------------------------------
# Rows of all sequences stand behind each other, cu [n_seqs + 1] (int32, device) says where each one's begin.  Tensors have to
# be on one GPU; the work goes to that GPU's current stream.
_DT = {torch.float32: PF_F32, torch.bfloat16: PF_BF16}


# Sizes pass the C boundary as 32-bit ints, and ctypes drops what does not fit: they are looked at before.
def _too_large(what, *sizes):
    raise PfError(-3, f"{what}: sizes {sizes}, one is past 2^31 - 1")


def _raise(st):
    raise PfError(st, load_library().pf_last_error(None).decode())


def _rows(name, t, dtype=None, device=None):
    """A 2-d tensor of rows as the kernels read them: any row stride, channels next to each other."""
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise PfError(-3, f"{name}: rows of contiguous channels are needed, got shape {tuple(t.shape)}, strides {t.stride()}")
    return _plain(name, t, dtype, device)


def _plain(name, t, dtype=None, device=None):
    if not t.is_cuda:
        raise PfError(-3, f"{name}: is on {t.device}, a GPU tensor is needed")
    if device is not None and t.device != device:
        raise PfError(-3, f"{name}: is on {t.device}, the call's other tensors on {device}")
    if dtype is not None and t.dtype != dtype:
        raise PfError(-4, f"{name}: is {t.dtype}, {dtype} is needed")
    if t.dtype not in _DT and dtype is None:
        raise PfError(-4, f"{name}: {t.dtype} is neither float32 nor bfloat16")
    return t


def _ints(name, t, shape, device):
    """An int32 tensor of lengths, positions or pages, contiguous and of the given shape."""
    _plain(name, t, torch.int32, device)
    if tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise PfError(-3, f"{name}: shape {tuple(t.shape)}, a contiguous {tuple(shape)} is needed")
    return t


def _vectors(name, t, d, n_seqs, index, device):
    """float [d], or [n_seqs, d] for a call with sequences; returns the stride between sequences and the address."""
    if t is None:
        return 0, None
    shape = (d,) if n_seqs is None else (n_seqs, d)
    if not (t.dtype is torch.float32 and t.get_device() == index and t.shape == shape and t.stride(-1) == 1):
        _plain(name, t, torch.float32, device)
        raise PfError(-3, f"{name}: shape {tuple(t.shape)}, strides {t.stride()}, contiguous vectors {shape} are needed")
    return 0 if n_seqs is None or n_seqs == 1 else t.stride(0), t.data_ptr()


def _ld(t):
    # the stride of a single row (or of none) may be anything: rows are then as far apart as they are wide
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 8)


# The checks above say what is wrong; a call of a few microseconds first asks these, which only say whether all is well.
def _good_rows(t, dtype, index):
    return t.dtype is dtype and t.get_device() == index and t.dim() == 2 and t.stride(1) == 1


def _good_ints(t, shape, index):
    return t.dtype is torch.int32 and t.get_device() == index and t.shape == shape and t.is_contiguous()


def _launch(index, fn, *args):
    """Calls a C entry point, whose last argument is the stream, on GPU `index` and its current stream."""
    if torch._C._cuda_getDevice() == index:
        st = fn(*args, torch._C._cuda_getCurrentRawStream(index))
    else:
        with torch.cuda.device(index):
            st = fn(*args, torch._C._cuda_getCurrentRawStream(index))
    if st != 0:
        _raise(st)


def _like(t, dtype=None):
    return torch.empty_like(t, dtype=dtype, memory_format=torch.contiguous_format)


def make_rope(axis_dims, layout="interleaved", theta=1e4, scaling="none", factor=1.0, low=1.0, high=32.0, original_len=1,
              magnitude=1.0):
    """A rotation for pf_op_rope / pf_op_kv_append (pf_rope_init): made once, used by every call."""
    if layout not in ROPE_LAYOUTS or scaling not in ROPE_SCALINGS:
        raise PfError(-2, f"rope: layout {layout!r}, scaling {scaling!r}")
    dims = [int(w) for w in axis_dims]
    if any(not -2 ** 31 <= n < 2 ** 31 for n in (*dims, original_len)):
        raise PfError(-2, f"rope: axis_dims {dims}, original_len {original_len}")
    c = PfRopeConfig(layout=ROPE_LAYOUTS[layout], n_axes=len(dims), theta=theta, scaling=ROPE_SCALINGS[scaling], factor=factor,
                     low=low, high=high, original_len=original_len, magnitude=magnitude)
    c.axis_dim[:min(len(dims), PF_ROPE_MAX_AXES)] = dims[:PF_ROPE_MAX_AXES]
    rope = PfRope()
    st = load_library().pf_rope_init(C.byref(c), C.byref(rope))
    if st != 0:
        _raise(st)
    return rope


def _heads(name, t, head_dim):
    if head_dim < 1 or t.shape[1] % head_dim:
        raise PfError(-3, f"{name}: rows of {t.shape[1]} channels are no whole heads of {head_dim}")
    return t.shape[1] // head_dim


def _positions(rope, pos, tokens, index, device):
    n = rope.n_axes
    if not (_good_ints(pos, (tokens, n), index) or (n == 1 and _good_ints(pos, (tokens,), index))):
        _ints("pos", pos, (tokens,) if pos.dim() == 1 and n == 1 else (tokens, n), device)


def pf_op_rope(x, rope, pos, head_dim, out=None):
    """x [tokens, heads * head_dim] with every head turned by its row's position(s); pos int32 [tokens, n_axes] (or [tokens] for
    one axis).  out may be x."""
    index, dt = x.get_device(), _DT.get(x.dtype)
    if index < 0 or dt is None or not _good_rows(x, x.dtype, index):
        _rows("x", x)
    tokens, width = x.shape
    if (tokens | width) >> 31:
        _too_large("x", tokens, width)
    heads = _heads("x", x, head_dim)
    _positions(rope, pos, tokens, index, x.device)
    if out is None:
        out, ldo = _like(x), width
    else:
        ldo = _ld(_out("out", out, x.shape, x.dtype, x.device))
    _launch(index, (_lib or load_library()).pf_op_rope, dt, C.byref(rope), pos.data_ptr(), x.data_ptr(), _ld(x), out.data_ptr(), ldo,
            tokens, heads, head_dim)
    return out


def _out(name, t, shape, dtype, device):
    _rows(name, t, dtype, device)
    if tuple(t.shape) != tuple(shape):
        raise PfError(-3, f"{name}: shape {tuple(t.shape)}, {tuple(shape)} is needed")
    return t


class KvPages:
    """Keys and values in pages: k and v [n_pages, kv_heads, page_size, head_dim] (pages any distance apart, a page contiguous),
    table int32 [n_seqs, max_pages] of page numbers (those outside [0, n_pages): no page).  Holds the tensors it was given;
    their contents, the table's among them, may change between calls."""

    def __init__(self, k, v, table):
        for name, t in (("k", k), ("v", v)):
            _plain(name, t, None if t is k else k.dtype, k.device)
            if t.dim() != 4 or t.shape != k.shape or not (t.shape[0] == 0 or t[0].is_contiguous()):
                raise PfError(-3, f"{name} pages: shape {tuple(t.shape)}, strides {t.stride()}")
        if table.dim() != 2:
            raise PfError(-3, f"table: shape {tuple(table.shape)}, [n_seqs, max_pages] is needed")
        _ints("table", table, table.shape, k.device)
        self.k, self.v, self.table = k, v, table
        n, self.kv_heads, self.page_size, self.head_dim = k.shape
        block = self.kv_heads * self.page_size * self.head_dim
        self.n_seqs, self.max_pages = table.shape
        if (n | self.kv_heads | self.page_size | self.head_dim | self.n_seqs | self.max_pages) >> 31:
            _too_large("pages", *k.shape, *table.shape)
        self.device, self.index = k.device, k.get_device()
        self.c = PfKvPages(k=k.data_ptr(), v=v.data_ptr(), k_page_stride=k.stride(0) if n > 1 else block,
                           v_page_stride=v.stride(0) if n > 1 else block, table=table.data_ptr(), n_pages=n,
                           page_size=self.page_size, kv_heads=self.kv_heads, head_dim=self.head_dim, n_seqs=self.n_seqs,
                           max_pages=self.max_pages)
        self.ref = C.byref(self.c)


def pf_op_kv_append(pages, k, v, cu, first, rope=None, pos=None, q=None, q_out=None):
    """Writes rows of k and v [tokens, kv_heads * head_dim] into the pages, row cu[s] + i of sequence s into slot first[s] + i, k
    turned by `rope` on the way; returns q turned likewise (None without q)."""
    dt, dev, index = pages.k.dtype, pages.device, pages.index
    if not (_good_rows(k, dt, index) and _good_rows(v, dt, index) and v.shape == k.shape and
            _good_ints(cu, (pages.n_seqs + 1,), index) and _good_ints(first, (pages.n_seqs,), index)):
        _rows("k", k, dt, dev)
        _out("v", v, k.shape, dt, dev)
        _ints("cu", cu, (pages.n_seqs + 1,), dev)
        _ints("first", first, (pages.n_seqs,), dev)
    tokens, width = k.shape
    if tokens >> 31:
        _too_large("k", tokens, width)
    if width != pages.kv_heads * pages.head_dim:
        raise PfError(-3, f"k: rows of {width} channels for {pages.kv_heads} heads of {pages.head_dim}")
    if rope is not None:
        if pos is None:
            raise PfError(-1, "pos")
        _positions(rope, pos, tokens, index, dev)
    if q is None:
        if q_out is not None:
            raise PfError(-1, "q_out without q")
        q_args = (None, 0, None, 0, 0)
    else:
        if not _good_rows(q, dt, index):
            _rows("q", q, dt, dev)
        if q.shape[0] != tokens:
            raise PfError(-3, f"q: {q.shape[0]} rows, k has {tokens}")
        if q.shape[1] >> 31:
            _too_large("q", *q.shape)
        heads = _heads("q", q, pages.head_dim)
        if q_out is None:
            q_out, ldo = _like(q), heads * pages.head_dim
        else:
            ldo = _ld(_out("q_out", q_out, q.shape, dt, dev))
        q_args = (q.data_ptr(), _ld(q), q_out.data_ptr(), ldo, heads)
    _launch(index, (_lib or load_library()).pf_op_kv_append, _DT[dt], pages.ref, k.data_ptr(), _ld(k), v.data_ptr(), _ld(v),
            cu.data_ptr(), first.data_ptr(), tokens, None if rope is None else C.byref(rope),
            None if rope is None else pos.data_ptr(), *q_args)
    return q_out


@functools.lru_cache(maxsize=1024)
def _rows_ws_bytes(*sizes):
    return load_library().pf_op_attention_rows_ws_bytes(*sizes)


def _attention_buffers(q, heads, kv_heads, head_dim, n_seqs, max_kv, out, want_lse):
    """out, lse, and (address of out, its row stride, address of lse, workspace, its bytes) for the call."""
    if out is None:
        out, ldo = _like(q), heads * head_dim
    else:
        ldo = _ld(_out("out", out, q.shape, q.dtype, q.device))
    lse = torch.empty(q.shape[0], heads, dtype=torch.float32, device=q.device) if want_lse else None
    n = _rows_ws_bytes(_DT[q.dtype], q.shape[0], n_seqs, heads, kv_heads, head_dim, max_kv)
    ws = torch.empty(n, dtype=torch.uint8, device=q.device) if n else None
    return out, lse, ws, (out.data_ptr(), ldo, None if lse is None else lse.data_ptr(), None if ws is None else ws.data_ptr(), n)


def pf_op_attention_packed(q, k, v, cu_q, cu_k, head_dim, causal=False, scale=None, out=None, want_lse=False):
    """Attention of packed sequences: q [total_q, heads * head_dim], k and v [total_k, kv_heads * head_dim], cu_q and cu_k int32
    [n_seqs + 1].  causal: the last query of a sequence sees all its keys, the one before all but one, ...  Returns out, or
    (out, lse) with lse float [total_q, heads]; rows of no sequence are not written."""
    index, dt = q.get_device(), q.dtype
    n_seqs = cu_q.shape[0] - 1 if cu_q.dim() == 1 else -1
    if not (index >= 0 and dt in _DT and n_seqs >= 0 and _good_rows(q, dt, index) and _good_rows(k, dt, index) and
            _good_rows(v, dt, index) and v.shape == k.shape and _good_ints(cu_q, (n_seqs + 1,), index) and
            _good_ints(cu_k, (n_seqs + 1,), index)):
        _rows("q", q)
        _rows("k", k, dt, q.device)
        _out("v", v, k.shape, dt, q.device)
        if n_seqs < 0:
            raise PfError(-3, f"cu_q: shape {tuple(cu_q.shape)}, [n_seqs + 1] is needed")
        _ints("cu_q", cu_q, (n_seqs + 1,), q.device)
        _ints("cu_k", cu_k, (n_seqs + 1,), q.device)
    if (q.shape[0] | q.shape[1] | k.shape[0] | k.shape[1] | n_seqs) >> 31:
        _too_large("q, k, sequences", *q.shape, *k.shape, n_seqs)
    heads, kv_heads = _heads("q", q, head_dim), _heads("k", k, head_dim)
    if scale is not None and not scale > 0:
        raise PfError(-3, f"scale: {scale}")
    out, lse, ws, tail = _attention_buffers(q, heads, kv_heads, head_dim, n_seqs, max(k.shape[0], 1), out, want_lse)
    _launch(index, (_lib or load_library()).pf_op_attention_packed, _DT[dt], q.data_ptr(), _ld(q), k.data_ptr(), _ld(k),
            v.data_ptr(), _ld(v), cu_q.data_ptr(), cu_k.data_ptr(), n_seqs, q.shape[0], k.shape[0], heads, kv_heads, head_dim,
            0.0 if scale is None else scale, int(causal), *tail)
    return (out, lse) if want_lse else out


def pf_op_attention_paged(q, pages, cu_q, first, kv_len, causal=True, scale=None, out=None, want_lse=False):
    """Attention of new rows q [total_q, heads * head_dim], cu_q[s] .. cu_q[s + 1] those of sequence s from its slot first[s] on,
    over slots [0, kv_len[s]) of the pages; causal: row i sees slots up to first[s] + i.  first may be None if not causal.
    Returns out, or (out, lse) with lse float [total_q, heads]; rows of no sequence are not written."""
    index, dt = pages.index, pages.k.dtype
    if not (_good_rows(q, dt, index) and _good_ints(cu_q, (pages.n_seqs + 1,), index) and
            _good_ints(kv_len, (pages.n_seqs,), index) and (first is None or _good_ints(first, (pages.n_seqs,), index))):
        _rows("q", q, dt, pages.device)
        _ints("cu_q", cu_q, (pages.n_seqs + 1,), pages.device)
        _ints("kv_len", kv_len, (pages.n_seqs,), pages.device)
        if first is not None:
            _ints("first", first, (pages.n_seqs,), pages.device)
    if (q.shape[0] | q.shape[1]) >> 31:
        _too_large("q", *q.shape)
    heads = _heads("q", q, pages.head_dim)
    if scale is not None and not scale > 0:
        raise PfError(-3, f"scale: {scale}")
    out, lse, ws, tail = _attention_buffers(q, heads, pages.kv_heads, pages.head_dim, pages.n_seqs,
                                            pages.max_pages * pages.page_size, out, want_lse)
    _launch(index, (_lib or load_library()).pf_op_attention_paged, _DT[dt], q.data_ptr(), _ld(q), pages.ref, cu_q.data_ptr(),
            None if first is None else first.data_ptr(), kv_len.data_ptr(), q.shape[0], heads, 0.0 if scale is None else scale,
            int(causal), *tail)
    return (out, lse) if want_lse else out


class Norm:
    """A norm over rows for pf_op_norm_residual (make_norm)."""

    def __init__(self, kind, weight, bias, eps):
        if kind not in NORM_KINDS:
            raise PfError(-2, f"norm: kind {kind!r}")
        self.weight, self.bias = weight, bias
        for name, t in (("weight", weight), ("bias", bias)):
            if t is not None and (t.dim() != 1 or not _plain("norm " + name, t).is_contiguous()):
                raise PfError(-3, f"norm {name}: shape {tuple(t.shape)}, a contiguous [d] is needed")
        self.c = PfNorm(kind=NORM_KINDS[kind], eps=eps, weight=None if weight is None else weight.data_ptr(),
                        bias=None if bias is None else bias.data_ptr())
        self.ref = C.byref(self.c)
        self.key = None      # (type, GPU, width) of the last call that the vectors fitted

    def check(self, side, dtype, device, d):
        for t in (self.weight, self.bias):
            if t is not None and tuple(_plain(side + " norm", t, dtype, device).shape) != (d,):
                raise PfError(-3, f"{side} norm: {tuple(t.shape)}, ({d},) is needed")
        self.key = (dtype, device.index, d)


def make_norm(kind, weight=None, bias=None, eps=1e-6):
    """kind "rms" or "layer", weight and bias [d] in the type of the branch or None."""
    return Norm(kind, weight, bias, eps)


def pf_op_norm_residual(y, x, post=None, pre=None, gate=None, gate_tanh=False, x_scale=1.0, scale=None, shift=None, cu=None,
                        x_out=None, h_out=None, dtype=None, want_h=True):
    """x_out = x_scale * x + g(gate) * post(y), h = pre(x_out) * (1 + scale) + shift; returns (x_out, h).  x float [rows, d], y and h
    in `dtype` (y's; without a branch, y None, it has to be given).  gate / scale / shift float [d], or [n_seqs, d] with cu
    int32 [n_seqs + 1].  want_h False: only the residual (h None)."""
    index, dev = x.get_device(), x.device
    if index < 0 or not _good_rows(x, torch.float32, index):
        _rows("x", x, torch.float32)
    rows, d = x.shape
    if y is None:
        y_args = (None, 0)
    else:
        dtype = y.dtype if dtype is None else dtype
        if not (_good_rows(y, dtype, index) and y.shape == x.shape):
            _out("y", y, x.shape, dtype, dev)
        y_args = (y.data_ptr(), _ld(y))
    if dtype not in _DT:
        raise PfError(-4, f"dtype {dtype}")
    if post is not None and post.key != (dtype, index, d):
        post.check("post", dtype, dev, d)
    if pre is not None and pre.key != (dtype, index, d):
        pre.check("pre", dtype, dev, d)
    n_seqs = None
    if cu is not None:
        if cu.dim() != 1 or cu.shape[0] < 1:
            raise PfError(-3, f"cu: shape {tuple(cu.shape)}, [n_seqs + 1] is needed")
        n_seqs = cu.shape[0] - 1
        if not _good_ints(cu, (n_seqs + 1,), index):
            _ints("cu", cu, (n_seqs + 1,), dev)
    if (rows | d | (n_seqs or 0)) >> 31:
        _too_large("x, sequences", rows, d, n_seqs)
    gs, g_at = _vectors("gate", gate, d, n_seqs, index, dev)
    ms, sc_at = _vectors("scale", scale, d, n_seqs, index, dev)
    ms2, sh_at = _vectors("shift", shift, d, n_seqs, index, dev)
    if scale is not None and shift is not None and ms != ms2:
        raise PfError(-3, f"scale and shift: {ms} and {ms2} elements between sequences")
    if x_out is None:
        x_out, ldxo = _like(x), d
    else:
        ldxo = _ld(_out("x_out", x_out, x.shape, torch.float32, dev))
    if not want_h:
        h_args = (None, 0)
    elif h_out is None:
        h_out = _like(x, dtype)
        h_args = (h_out.data_ptr(), d)
    else:
        h_args = (h_out.data_ptr(), _ld(_out("h_out", h_out, x.shape, dtype, dev)))
    _launch(index, (_lib or load_library()).pf_op_norm_residual, _DT[dtype], *y_args, None if post is None else post.ref, g_at, gs,
            int(gate_tanh), x_scale, x.data_ptr(), _ld(x), x_out.data_ptr(), ldxo, None if pre is None else pre.ref, sh_at,
            sc_at, max(ms, ms2), *h_args, None if cu is None else cu.data_ptr(), n_seqs or 0, rows, d)
    return x_out, h_out if want_h else None
