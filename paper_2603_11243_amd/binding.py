"""ctypes binding of the C ABI in include/ssd.h: argument marshalling only.

Torch is used for device memory (tensors own the buffers, `data_ptr()` is what crosses the ABI)
and for the stream handle.  Every computation happens inside libssd.so.
"""
import ctypes as C
import os
import struct
from typing import Optional, Sequence

import numpy as np
import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libssd.so")

SSD_F32, SSD_BF16, SSD_F16, SSD_E4M3, SSD_I8 = 0, 1, 2, 3, 4
_DTYPE_CODE = {torch.float32: SSD_F32, torch.bfloat16: SSD_BF16}
_KV_CODE = {torch.float32: SSD_F32, torch.bfloat16: SSD_BF16, torch.float16: SSD_F16}
_PAGE_CODE = {**_KV_CODE, torch.float8_e4m3fn: SSD_E4M3, torch.int8: SSD_I8}
_STATUS = {0: "SSD_OK", -1: "SSD_EINVAL", -2: "SSD_ESHAPE", -3: "SSD_EWORKSPACE", -4: "SSD_EHIP",
           -5: "SSD_EUNSUPPORTED"}

EXPORTS = ["ssd_create", "ssd_destroy", "ssd_workspace_bytes", "ssd_set_workspace", "ssd_last_error",
           "ssd_profile_select", "ssd_profile_read", "ssd_measure_mfma_ceiling", "ssd_measure_hbm_read", "ctc_gate", "verify_forward", "accept_prefix",
           "verify_forward_kv", "ssd_kv_cache_bytes", "ssd_set_kv_cache", "ssd_ar_workspace_bytes", "ar_fallback",
           "ssd_gate_grid", "ssd_accept_grid", "ssd_plan_batches", "ssd_set_ctc_head", "ctc_head_gate", "ssd_device_flags",
           "ctc_gate_noalloc", "ssd_inexact_weights", "ssd_select_unconfident", "ssd_gather_i32", "ssd_set_qformer", "qformer_pool",
           "ssd_kv_cache_view", "ssd_tree_workspace_bytes", "tree_attention", "tree_path", "ssd_evict_workspace_bytes", "kv_evict",
           "ssd_verify_tree_workspace_bytes", "verify_tree", "accept_tree", "kv_write_pages", "kv_read_pages", "ssd_paged_workspace_bytes",
           "paged_attention"]

PROF_OFF, PROF_ALL = -2, -1
PROF_CLASSES = ["gate", "gemm_qkv", "attention", "gemm_o", "gemm_gate_up", "gemm_down", "lmhead_accept", "other",
                "ar_fallback", "ctc_head_gate", "qformer_pool"]


class SsdError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"{_STATUS.get(code, code)}: {msg}")
        self.code = code


class ModelCfgC(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_q_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("d_ff", C.c_int32), ("vocab", C.c_int32),
                ("rms_eps", C.c_float), ("rope_theta", C.c_float), ("dtype", C.c_int32),
                ("max_positions", C.c_int32), ("operand", C.c_int32)]


class WeightsC(C.Structure):
    _fields_ = [("embed", C.c_void_p)] + \
               [(n, C.POINTER(C.c_void_p)) for n in ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down",
                                                      "norm_attn", "norm_mlp")] + \
               [("norm_final", C.c_void_p), ("lm_head", C.c_void_p)]


class KvViewC(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("slots", C.c_int64), ("slot_stride", C.c_int64), ("head_stride", C.c_int64),
                ("layer_stride", C.c_int64), ("n_layers", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32)]


def load_library() -> C.CDLL:
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2603_11243_amd.build` "
                          "(there is no fallback path)")
    lib = C.CDLL(_LIB_PATH)
    vp, i32, i64, f32 = C.c_void_p, C.c_int, C.c_int64, C.c_float
    lib.ssd_create.argtypes = [C.POINTER(vp), C.POINTER(ModelCfgC), C.POINTER(WeightsC), vp]
    lib.ssd_create.restype = i32
    lib.ssd_destroy.argtypes = [vp]
    lib.ssd_destroy.restype = None
    lib.ssd_workspace_bytes.argtypes = [vp, i64, i64, i64, i64]
    lib.ssd_workspace_bytes.restype = C.c_size_t
    lib.ssd_set_workspace.argtypes = [vp, vp, C.c_size_t]
    lib.ssd_set_workspace.restype = i32
    lib.ssd_last_error.argtypes = [vp]
    lib.ssd_last_error.restype = C.c_char_p
    lib.ssd_profile_select.argtypes = [vp, i32]
    lib.ssd_profile_select.restype = i32
    lib.ssd_profile_read.argtypes = [vp, vp, vp]
    lib.ssd_profile_read.restype = i32
    lib.ssd_measure_mfma_ceiling.argtypes = [vp, i32, vp, vp]
    lib.ssd_measure_mfma_ceiling.restype = i32
    lib.ssd_measure_hbm_read.argtypes = [vp, vp, C.c_size_t, i32, vp]
    lib.ssd_measure_hbm_read.restype = i32
    lib.ctc_gate.argtypes = [vp, vp, i32, vp, i32, i32, i32, f32, vp, vp, vp, vp, vp, vp]
    lib.ctc_gate.restype = i32
    lib.verify_forward.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, vp]
    lib.verify_forward.restype = i32
    lib.accept_prefix.argtypes = [vp, vp, vp, vp, i32, f32, vp, vp, vp, vp]
    lib.accept_prefix.restype = i32
    lib.verify_forward_kv.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, vp, vp]
    lib.verify_forward_kv.restype = i32
    lib.ssd_kv_cache_bytes.argtypes = [vp, i64]
    lib.ssd_kv_cache_bytes.restype = C.c_size_t
    lib.ssd_set_kv_cache.argtypes = [vp, vp, C.c_size_t, i64]
    lib.ssd_set_kv_cache.restype = i32
    lib.ssd_ar_workspace_bytes.argtypes = [vp, i32, i32]
    lib.ssd_ar_workspace_bytes.restype = C.c_size_t
    lib.ar_fallback.argtypes = [vp, i32, vp, vp, vp, i32, vp]
    lib.ar_fallback.restype = i32
    lib.ssd_gate_grid.argtypes = [vp, vp, i32, vp, i32, vp]
    lib.ssd_gate_grid.restype = i32
    lib.ssd_accept_grid.argtypes = [vp, vp, vp, i32, vp, i32, vp, vp]
    lib.ssd_accept_grid.restype = i32
    lib.ssd_plan_batches.argtypes = [vp, i32, i64, i32, vp, vp, vp]
    lib.ssd_plan_batches.restype = i32
    lib.ssd_device_flags.argtypes = [vp, vp]
    lib.ssd_device_flags.restype = i32
    lib.ssd_set_ctc_head.argtypes = [vp, vp, vp, i32, i32]
    lib.ssd_set_ctc_head.restype = i32
    lib.ctc_head_gate.argtypes = [vp, vp, vp, i32, i32, f32, vp, vp, vp, vp, vp, vp]
    lib.ctc_head_gate.restype = i32
    lib.ctc_gate_noalloc.argtypes = [vp, vp, i32, vp, i32, i64, i32, i32, f32, vp, vp, vp, vp, C.c_char_p, C.c_size_t]
    lib.ctc_gate_noalloc.restype = i32
    lib.ssd_select_unconfident.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.ssd_select_unconfident.restype = i32
    lib.ssd_set_qformer.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32]
    lib.ssd_set_qformer.restype = i32
    lib.qformer_pool.argtypes = [vp, vp, vp, i32, vp, vp]
    lib.qformer_pool.restype = i32
    lib.ssd_gather_i32.argtypes = [vp, vp, vp, i32, vp]
    lib.ssd_gather_i32.restype = i32
    lib.ssd_kv_cache_view.argtypes = [vp, vp, i64, vp]
    lib.ssd_kv_cache_view.restype = i32
    lib.ssd_tree_workspace_bytes.argtypes = [vp, i32, i32, i32, i64, i64]
    lib.ssd_tree_workspace_bytes.restype = C.c_size_t
    lib.tree_attention.argtypes = [vp, vp, i64, i32, vp, i32, vp, vp, vp, vp, f32, vp, vp, vp]
    lib.tree_attention.restype = i32
    lib.tree_path.argtypes = [vp, vp, i32, vp, vp, f32, vp, vp, vp]
    lib.tree_path.restype = i32
    lib.ssd_evict_workspace_bytes.argtypes = [vp, i32, i32, i64, i64]
    lib.ssd_evict_workspace_bytes.restype = C.c_size_t
    lib.kv_evict.argtypes = [vp, vp, vp, i32, vp, vp, vp, i32, i32, vp, vp, vp, vp]
    lib.kv_evict.restype = i32
    lib.ssd_verify_tree_workspace_bytes.argtypes = [vp, i64, i64]
    lib.ssd_verify_tree_workspace_bytes.restype = C.c_size_t
    lib.verify_tree.argtypes = [vp, vp, i32, vp, vp, vp, vp, vp, vp, vp]
    lib.verify_tree.restype = i32
    lib.accept_tree.argtypes = [vp, vp, vp, i32, vp, vp, f32, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.accept_tree.restype = i32
    lib.kv_write_pages.argtypes = [vp, vp, vp, vp, i32, vp, vp]
    lib.kv_write_pages.restype = i32
    lib.kv_read_pages.argtypes = [vp, vp, vp, vp, vp, vp, i32]
    lib.kv_read_pages.restype = i32
    lib.ssd_paged_workspace_bytes.argtypes = [vp, i32, i32, i32, i64, i32, i64]
    lib.ssd_paged_workspace_bytes.restype = C.c_size_t
    lib.paged_attention.argtypes = [vp, vp, i32, i64, i32, i32, vp, vp, f32, vp, vp]
    lib.paged_attention.restype = i32
    lib.ssd_inexact_weights.argtypes = [vp]
    lib.ssd_inexact_weights.restype = i64
    return lib


_lib = None


def lib() -> C.CDLL:
    global _lib
    if _lib is None:
        _lib = load_library()
    return _lib


# What a small call costs is mostly the host: the arguments below are plain ints and bytes, which the argtypes take as pointers (of a gate
# call's 8 us of Python 1.1 went to one array's .ctypes and 0.7 to c_void_p objects; bytes of 1025 prefix sums are copied in 0.2).
def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous()
    return t.data_ptr()


def _host_i32(a: Sequence[int]) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


def _host_call_i32(a: Sequence[int]) -> np.ndarray:
    """_host_i32 that leaves an array as it is which needs nothing: what small calls pass four of (0.6 us each)."""
    return a if type(a) is np.ndarray and a.dtype == np.int32 and a.flags.c_contiguous else _host_i32(a)


def _host_arg(a: np.ndarray):
    """Argument for an array that the call reads before it returns: a copy of a few words (0.1 us), the address of many."""
    return a.tobytes() if a.size <= 1024 else a.ctypes.data


def _at(t: torch.Tensor, device) -> bool:
    return t.device == device or (device.index is None and t.device.type == device.type)


def _on(device, dtype, **tensors):
    """Tensors that a call reads or writes as contiguous memory of its device: ValueError names the one that is not."""
    for name, t in tensors.items():
        if t is not None and (t.dtype != dtype or not t.is_contiguous() or not _at(t, device)):
            raise ValueError(f"{name} must be a contiguous {dtype} tensor on {device}")


_KV_VIEW = struct.Struct("=QQqqqqiiii")          # ssd_kv_view


def _kv_view(device, k: torch.Tensor, v: torch.Tensor):
    """(ssd_kv_view as bytes, slots, layers, K/V heads, head_dim) of k and v [slots, K/V heads, head_dim], or with a dimension of layers before; any
    strides but the last."""
    shape, st, sv, code = k.shape, k.stride(), v.stride(), _KV_CODE.get(k.dtype)
    if shape != v.shape or len(shape) not in (3, 4) or k.dtype is not v.dtype or code is None or not _at(k, device) or k.device != v.device:
        raise ValueError(f"k and v must be alike: [layers,] slots, K/V heads, head_dim, float16, bfloat16 or float32, on {device}")
    n, H, hd = shape[-3:]
    L = shape[0] if len(shape) == 4 else 1
    if n > 1 and H > 1 and L == 1 and st == sv:
        ss, hs, one = st[-3:]
        ls = 0
    else:
        def strides(t):                                      # of dimensions of one entry: as if the rows lay close together
            ss, hs = t[-3], t[-2] if H > 1 else hd
            return ss if n > 1 else max(hd, hs * (H - 1) + hd), hs, t[0] if L > 1 else 0
        (ss, hs, ls), one = strides(st), st[-1]
        if strides(sv) != (ss, hs, ls) or hd > 1 and sv[-1] != one:
            raise ValueError("k and v must have the same strides")
    if one != 1 and hd > 1:
        raise ValueError("the elements of a row of k and v must be consecutive")
    return _KV_VIEW.pack(k.data_ptr(), v.data_ptr(), n, ss, hs, ls, L, H, hd, code), n, L, H, hd


_KV_PAGES = struct.Struct("=QQQQqiiiiixxxx")     # ssd_kv_pages
_PAGE_TABLE = struct.Struct("=QqQii")            # ssd_page_table


class KvPages:
    """K/V rows in pages (ssd_kv_pages): k and v [layers, pages, K/V heads, rows of a page, head_dim], float16, bfloat16 or float32, or float8_e4m3fn or int8 with
    k_scale and v_scale [layers, pages, K/V heads, rows of a page] float32; contiguous, on one device; one layer may come without its dimension."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None):
        code = _PAGE_CODE.get(k.dtype)
        if k.shape != v.shape or k.dim() not in (4, 5) or k.dtype is not v.dtype or code is None or k.device != v.device or not k.is_contiguous() or not v.is_contiguous():
            raise ValueError("k and v must be alike and contiguous: [layers,] pages, K/V heads, rows of a page, head_dim")
        if (k_scale is not None) != (k.element_size() == 1) or (k_scale is None) != (v_scale is None):
            raise ValueError("pages of 8-bit types have k_scale and v_scale, others none")
        if k_scale is not None:
            _on(k.device, torch.float32, k_scale=k_scale, v_scale=v_scale)
            if k_scale.shape != k.shape[:-1] or v_scale.shape != k.shape[:-1]:
                raise ValueError("k_scale and v_scale must be [layers,] pages, K/V heads, rows of a page")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.device, self.dtype, self._index = k.device, k.dtype, k.get_device()
        self.n_pages, self.n_kv_heads, self.page_rows, self.head_dim = k.shape[-4:]
        self.n_layers = k.shape[0] if k.dim() == 5 else 1
        self._view = _KV_PAGES.pack(k.data_ptr(), v.data_ptr(), 0 if k_scale is None else k_scale.data_ptr(), 0 if v_scale is None else v_scale.data_ptr(), self.n_pages,
                                    self.page_rows, self.n_layers, self.n_kv_heads, self.head_dim, code)
        self._layers = {}

    def layer(self, l: int) -> "KvPages":
        """The pages of one layer, the same memory."""
        if l not in self._layers:
            if not 0 <= l < self.n_layers:
                raise IndexError(f"layer {l} of {self.n_layers}")
            parts = (self.k, self.v, self.k_scale, self.v_scale)
            self._layers[l] = KvPages(*(t if t is None or self.k.dim() == 4 else t[l] for t in parts))
        return self._layers[l]

    @staticmethod
    def empty(n_pages: int, page_rows: int, n_kv_heads: int, head_dim: int, dtype: torch.dtype, n_layers: int = 1, device="cuda:0") -> "KvPages":
        """Pages allocated through torch, their contents not defined."""
        shape = (n_layers, n_pages, n_kv_heads, page_rows, head_dim)
        k, v = (torch.empty(shape, dtype=dtype, device=device) for _ in range(2))
        scales = [torch.empty(shape[:-1], dtype=torch.float32, device=device) for _ in range(2)] if k.element_size() == 1 else []
        return KvPages(k, v, *scales)


class Context:
    """Owns one ssd_ctx.  `weights` is the dict layout of workloads.make_model_weights (device tensors)."""

    def __init__(self, model_cfg=None, weights: Optional[dict] = None, device="cuda:0", stream=None,
                 max_positions: int = 1024, operand: str = "f16"):
        self._lib = lib()
        self.device = torch.device(device)
        self.cfg = model_cfg
        self._keep = []               # tensors whose storage the library reads in place
        self._ws, self._reserved = None, []           # the workspace; all that reserve allocated
        self._h = C.c_void_p()
        torch.cuda.set_device(self.device)
        self._index = torch.cuda.current_device()
        st = stream if stream is not None else torch.cuda.current_stream(self.device)
        self.stream, self._raw_stream = st, st.cuda_stream
        cfg_p, w_p = None, None
        if model_cfg is not None:
            m = model_cfg
            self.dtype = {"bf16": torch.bfloat16, "f32": torch.float32}[m.dtype]
            # h_verify is an activation buffer between verify_forward and accept_prefix: the MFMA operand type for
            # bf16-stored models (IEEE half by default, bfloat16 with operand="bf16"), fp32 otherwise
            self.operand = operand
            self.act_dtype = torch.float32 if m.dtype == "f32" else {"f16": torch.float16, "bf16": torch.bfloat16}[operand]
            cfg_c = ModelCfgC(m.n_layers, m.d_model, m.n_q_heads, m.n_kv_heads, m.head_dim, m.d_ff, m.vocab,
                              m.rms_eps, m.rope_theta, _DTYPE_CODE[self.dtype], max_positions,
                              {"f16": 0, "bf16": 1}[operand])
            w_c = WeightsC()

            def dev(t):
                t = t.to(self.device).contiguous()
                assert t.dtype == self.dtype
                self._keep.append(t)
                return t.data_ptr()

            w_c.embed = dev(weights["embed"])
            w_c.lm_head = dev(weights["lm_head"])
            w_c.norm_final = dev(weights["norm_final"])
            arrays = []
            for name in ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down", "norm_attn", "norm_mlp"):
                arr = (C.c_void_p * m.n_layers)(*[dev(L[name]) for L in weights["layers"]])
                arrays.append(arr)
                setattr(w_c, name, C.cast(arr, C.POINTER(C.c_void_p)))
            cfg_p, w_p = C.byref(cfg_c), C.byref(w_c)
        rc = self._lib.ssd_create(C.byref(self._h), cfg_p, w_p, C.c_void_p(st.cuda_stream))
        if rc != 0:
            raise SsdError(rc, "ssd_create failed")

    def close(self):
        if self._h:
            self._lib.ssd_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc):
        if rc != 0:
            raise SsdError(rc, self._lib.ssd_last_error(self._h).decode())

    def workspace_bytes(self, max_frames=0, max_tokens=0, max_verify_rows=0, max_utts=0) -> int:
        return int(self._lib.ssd_workspace_bytes(self._h, max_frames, max_tokens, max_verify_rows, max_utts))

    def reserve(self, max_frames=0, max_tokens=0, max_verify_rows=0, max_utts=0, ar_utts=0, ar_steps=0, tree_nodes=0, tree_utts=0,
                tree_heads=None, evict_rows=0, evict_utts=0, evict_heads=None, paged_utts=0, paged_new=1, paged_ctx=0, paged_heads=None):
        """Allocates (through torch) and hands over a workspace big enough for the given maxima.  tree_nodes, tree_utts: tree_path, with
        tree_heads (query heads, K/V heads, head_dim) tree_attention, and for a context with a model verify_tree and accept_tree;
        evict_rows (kept by all utterances), evict_utts and evict_heads (layers, K/V heads): kv_evict.  paged_utts, paged_new (tokens of an utterance),
        paged_ctx (longest context) and paged_heads (query heads, K/V heads, head_dim): paged_attention.  A workspace that is too small is replaced by one
        at least a quarter larger and kept as long as this object: calls that were captured, or still run on the context's stream, use it."""
        n = self.workspace_bytes(max_frames, max_tokens, max_verify_rows, max_utts)
        if ar_utts and ar_steps:
            n = max(n, int(self._lib.ssd_ar_workspace_bytes(self._h, ar_utts, ar_steps)))
        if tree_utts:
            n = max(n, int(self._lib.ssd_tree_workspace_bytes(self._h, *(tree_heads or (0, 0, 0)), tree_nodes, tree_utts)),
                    int(self._lib.ssd_verify_tree_workspace_bytes(self._h, tree_nodes, tree_utts)))
        if evict_utts:
            n = max(n, int(self._lib.ssd_evict_workspace_bytes(self._h, *evict_heads, evict_rows, evict_utts)))
        if paged_utts:
            n = max(n, int(self._lib.ssd_paged_workspace_bytes(self._h, *paged_heads, paged_utts, paged_new, paged_ctx)))
        if self._ws is None or self._ws.numel() < n:
            last = self._reserved[-1].numel() if self._reserved else 0
            if last < n:                                     # (all of them together: five times the last at most)
                self._reserved.append(torch.empty(max(n, last * 5 // 4), dtype=torch.uint8, device=self.device))
            self.set_workspace(self._reserved[-1])

    def set_workspace(self, buf: Optional[torch.Tensor]):
        """buf is used from here on, and held until the next; calls that were captured with it need it longer, which is the caller's to see to."""
        self._ws = buf
        self._check(self._lib.ssd_set_workspace(self._h, _ptr(buf), 0 if buf is None else buf.numel()))

    def inexact_weights(self) -> int:
        """Weight values whose conversion to the matrix-core operand type was not exact (0 for ordinary tensors)."""
        return int(self._lib.ssd_inexact_weights(self._h))

    def device_flags(self) -> int:
        """Sticky flags raised by kernels since the last call (waits for the stream); 1 = a token id was clamped,
        2 = an activation left the half range and was stored saturated (or a log-likelihood was not finite), 4 = a page number,
        length or slot was out of range and left out.  Refused while the stream is captured."""
        f = C.c_int32(0)
        self._check(self._lib.ssd_device_flags(self._h, C.byref(f)))
        return int(f.value)

    def profile_select(self, kernel_class):
        k = PROF_CLASSES.index(kernel_class) if isinstance(kernel_class, str) else kernel_class
        self._check(self._lib.ssd_profile_select(self._h, k))

    def profile_read(self) -> dict:
        ms = np.zeros(len(PROF_CLASSES), dtype=np.float32)
        n = np.zeros(len(PROF_CLASSES), dtype=np.int32)
        self._check(self._lib.ssd_profile_read(self._h, ms.ctypes.data, n.ctypes.data))
        return {name: (float(ms[i]), int(n[i])) for i, name in enumerate(PROF_CLASSES)}

    def measure_mfma_ceiling(self, iters: int = 20000):
        t, g = C.c_float(), C.c_float()
        self._check(self._lib.ssd_measure_mfma_ceiling(self._h, iters, C.byref(t), C.byref(g)))
        return float(t.value), float(g.value)

    def measure_hbm_read(self, buf: torch.Tensor, iters: int = 5) -> float:
        g = C.c_float()
        self._check(self._lib.ssd_measure_hbm_read(self._h, buf.data_ptr(), buf.numel() * buf.element_size(), iters, C.byref(g)))
        return float(g.value)

    # ---- the three calls -------------------------------------------------------------------

    def ctc_gate(self, logits: torch.Tensor, cu_frames, blank_id: int, tau_ctc: float,
                 want_frames: bool = False, out: Optional[dict] = None) -> dict:
        cu = _host_i32(cu_frames)
        B, n_rows, V = len(cu) - 1, int(logits.shape[0]), int(logits.shape[1])
        dev = self.device
        if out is None:
            out = {"max_entropy": torch.empty(max(B, 0), dtype=torch.float32, device=dev),
                   "gate_pass": torch.empty(max(B, 0), dtype=torch.uint8, device=dev),
                   "draft_ctc": torch.empty(n_rows, dtype=torch.int32, device=dev),
                   "draft_len": torch.empty(max(B, 0), dtype=torch.int32, device=dev)}
            if want_frames:
                out["frame_entropy"] = torch.empty(n_rows, dtype=torch.float32, device=dev)
                out["frame_argmax"] = torch.empty(n_rows, dtype=torch.int32, device=dev)
        self._check(self._lib.ctc_gate(self._h, _ptr(logits), _DTYPE_CODE[logits.dtype], cu.tobytes(), B, V,
                                       blank_id, tau_ctc, _ptr(out.get("frame_entropy")),
                                       _ptr(out.get("frame_argmax")), _ptr(out["max_entropy"]),
                                       _ptr(out["gate_pass"]), _ptr(out["draft_ctc"]), _ptr(out["draft_len"])))
        return out

    def set_ctc_head(self, w_ctc: torch.Tensor, bias: Optional[torch.Tensor] = None):
        """Output layer of the CTC encoder: w_ctc [V_ctc, d_enc] bf16, bias [V_ctc] fp32 (both on the device)."""
        if w_ctc.dtype != torch.bfloat16 or not w_ctc.is_contiguous():
            raise ValueError("w_ctc must be a contiguous bfloat16 tensor")
        if bias is not None and (bias.dtype != torch.float32 or bias.numel() != w_ctc.shape[0]):
            raise ValueError("bias must be float32 [V_ctc]")
        self._check(self._lib.ssd_set_ctc_head(self._h, _ptr(w_ctc), _ptr(bias), int(w_ctc.shape[0]), int(w_ctc.shape[1])))
        self._head_shape = (int(w_ctc.shape[0]), int(w_ctc.shape[1]))

    def ctc_head_gate(self, enc_h: torch.Tensor, cu_frames, blank_id: int, tau_ctc: float,
                      want_frames: bool = False) -> dict:
        cu = _host_i32(cu_frames)
        B, n_rows = len(cu) - 1, int(enc_h.shape[0])
        if enc_h.dtype != torch.bfloat16 or not enc_h.is_contiguous():
            raise ValueError("enc_h must be a contiguous bfloat16 tensor")
        shape = getattr(self, "_head_shape", None)
        if shape is not None and int(enc_h.shape[1]) != shape[1]:
            raise ValueError(f"enc_h has {enc_h.shape[1]} columns, the output layer expects {shape[1]}")
        dev = self.device
        out = {"max_entropy": torch.empty(max(B, 0), dtype=torch.float32, device=dev),
               "gate_pass": torch.empty(max(B, 0), dtype=torch.uint8, device=dev),
               "draft_ctc": torch.empty(n_rows, dtype=torch.int32, device=dev),
               "draft_len": torch.empty(max(B, 0), dtype=torch.int32, device=dev)}
        if want_frames:
            out["frame_entropy"] = torch.empty(n_rows, dtype=torch.float32, device=dev)
            out["frame_argmax"] = torch.empty(n_rows, dtype=torch.int32, device=dev)
        self._check(self._lib.ctc_head_gate(self._h, _ptr(enc_h), cu.tobytes(), B, blank_id, tau_ctc,
                                            _ptr(out.get("frame_entropy")), _ptr(out.get("frame_argmax")),
                                            _ptr(out["max_entropy"]), _ptr(out["gate_pass"]),
                                            _ptr(out["draft_ctc"]), _ptr(out["draft_len"])))
        return out

    def select_unconfident(self, sel, cu_frames, draft_len_host, draft_ctc: torch.Tensor, ctc_to_llm: Optional[torch.Tensor],
                           speech_all: Optional[torch.Tensor], cu_speech_all, prompt_all: torch.Tensor, cu_prompt_all,
                           out: Optional[dict] = None, d_model: Optional[int] = None, dtype=None) -> dict:
        """ssd_select_unconfident: packed verification inputs of the utterances `sel` (host indices).  `out` may
        hold preallocated, large-enough `speech`, `prompt`, `draft_ids` tensors (their leading parts are written).
        speech_all may be None when cu_speech_all is all zero (no speech rows are moved); then d_model and dtype
        have to be given."""
        sel, cuf, dl = _host_i32(sel), _host_i32(cu_frames), _host_i32(draft_len_host)
        cs, cp = _host_i32(cu_speech_all), _host_i32(cu_prompt_all)
        n, B = len(sel), len(cuf) - 1
        d = int(speech_all.shape[1]) if speech_all is not None else int(d_model)
        sdt = speech_all.dtype if speech_all is not None else dtype
        nS = int((cs[sel + 1] - cs[sel]).sum()); nP = int((cp[sel + 1] - cp[sel]).sum()); nU = int(dl[sel].sum())
        if out is None:
            out = {"speech": torch.empty((nS, d), dtype=sdt, device=self.device),
                   "prompt": torch.empty(nP, dtype=torch.int32, device=self.device),
                   "draft_ids": torch.empty(nU, dtype=torch.int32, device=self.device)}
        assert out["speech"].shape[0] >= nS and out["prompt"].numel() >= nP and out["draft_ids"].numel() >= nU
        cso, cpo, cdo = (np.empty(n + 1, dtype=np.int32) for _ in range(3))
        V = 0 if ctc_to_llm is None else int(ctc_to_llm.numel())
        self._check(self._lib.ssd_select_unconfident(
            self._h, B, n, sel.tobytes(), cuf.tobytes(), dl.tobytes(), _ptr(draft_ctc), _ptr(ctc_to_llm), V,
            _ptr(speech_all), cs.tobytes(), _ptr(prompt_all), cp.tobytes(), d, _DTYPE_CODE[sdt],
            _ptr(out["speech"]) if nS else None, _ptr(out["prompt"]) if nP else None, _ptr(out["draft_ids"]) if nU else None,
            cso.ctypes.data, cpo.ctypes.data, cdo.ctypes.data))
        return {"speech": out["speech"][:nS], "prompt": out["prompt"][:nP], "draft_ids": out["draft_ids"][:nU],
                "cu_speech": cso, "cu_prompt": cpo, "cu_draft": cdo}

    def gather_i32(self, src: torch.Tensor, idx, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """out[i] = src[idx[i]] on the device (ssd_gather_i32); idx is a host array."""
        ix = _host_i32(idx)
        if out is None:
            out = torch.empty(len(ix), dtype=torch.int32, device=self.device)
        self._check(self._lib.ssd_gather_i32(self._h, _ptr(src), ix.tobytes(), len(ix), _ptr(out)))
        return out

    def set_qformer(self, q_proj: torch.Tensor, w_k: torch.Tensor, w_v: torch.Tensor, w_o: torch.Tensor, n_heads: int,
                    window: int = 15):
        """Projector windows (ssd_set_qformer): q_proj [n_q, d_h], w_k / w_v [d_h, d_enc], w_o [d_out, d_h], all bf16."""
        for t in (q_proj, w_k, w_v, w_o):
            if t.dtype != torch.bfloat16 or not t.is_contiguous():
                raise ValueError("projector weights must be contiguous bfloat16 tensors")
        n_q, d_h = int(q_proj.shape[0]), int(q_proj.shape[1])
        d_enc, d_out = int(w_k.shape[1]), int(w_o.shape[0])
        self._check(self._lib.ssd_set_qformer(self._h, _ptr(q_proj), _ptr(w_k), _ptr(w_v), _ptr(w_o), n_q, n_heads, d_h,
                                              d_enc, d_out, window))
        self._qformer = (n_q, d_enc, d_out, window)

    def qformer_pool(self, enc_h: torch.Tensor, cu_frames, out: Optional[torch.Tensor] = None):
        """Encoder frames -> acoustic embeddings (qformer_pool).  Returns (speech_emb [sum S, d_out] bf16, cu_speech)."""
        n_q, d_enc, d_out, window = self._qformer
        if enc_h.dtype != torch.bfloat16 or not enc_h.is_contiguous() or int(enc_h.shape[1]) != d_enc:
            raise ValueError("enc_h must be a contiguous bfloat16 tensor with d_enc columns")
        cu = _host_i32(cu_frames)
        B = len(cu) - 1
        n_rows = n_q * int((-(-np.diff(cu) // window)).sum())
        if out is None:
            out = torch.empty((n_rows, d_out), dtype=torch.bfloat16, device=self.device)
        cu_s = np.empty(B + 1, dtype=np.int32)
        self._check(self._lib.qformer_pool(self._h, _ptr(enc_h), cu.tobytes(), B, _ptr(out), cu_s.ctypes.data))
        return out[:n_rows], cu_s

    def verify_forward(self, speech_emb: torch.Tensor, cu_speech, prompt_ids: torch.Tensor, cu_prompt,
                       draft_ids: torch.Tensor, cu_draft, out: Optional[torch.Tensor] = None,
                       kv_start=None) -> torch.Tensor:
        """kv_start (host ints, one per utterance): also store keys/values in the K/V cache (verify_forward_kv)."""
        cs, cp, cd = _host_i32(cu_speech), _host_i32(cu_prompt), _host_i32(cu_draft)
        Bv = len(cd) - 1
        if out is None:
            out = torch.empty((int(cd[-1]), self.cfg.d_model), dtype=self.act_dtype, device=self.device)
        if kv_start is None:
            self._check(self._lib.verify_forward(self._h, _ptr(speech_emb), cs.tobytes(), _ptr(prompt_ids),
                                                 cp.tobytes(), _ptr(draft_ids), cd.tobytes(), Bv, _ptr(out)))
        else:
            ks = _host_i32(kv_start)
            self._check(self._lib.verify_forward_kv(self._h, _ptr(speech_emb), cs.tobytes(), _ptr(prompt_ids),
                                                    cp.tobytes(), _ptr(draft_ids), cd.tobytes(), Bv,
                                                    ks.tobytes(), _ptr(out)))
        return out

    def gate_grid(self, max_entropy: torch.Tensor, taus_ctc) -> torch.Tensor:
        t = np.ascontiguousarray(np.asarray(taus_ctc, dtype=np.float32))
        B = int(max_entropy.numel())
        out = torch.empty((len(t), B), dtype=torch.uint8, device=self.device)
        self._check(self._lib.ssd_gate_grid(self._h, _ptr(max_entropy), B, t.ctypes.data, len(t), _ptr(out)))
        return out

    def accept_grid(self, draft_logp: torch.Tensor, cu_draft, taus_slm) -> dict:
        t = np.ascontiguousarray(np.asarray(taus_slm, dtype=np.float32))
        cd = _host_i32(cu_draft)
        Bv = len(cd) - 1
        out = {"accept_len": torch.empty((len(t), Bv), dtype=torch.int32, device=self.device),
               "all_accepted": torch.empty((len(t), Bv), dtype=torch.uint8, device=self.device)}
        self._check(self._lib.ssd_accept_grid(self._h, _ptr(draft_logp), cd.tobytes(), Bv, t.ctypes.data, len(t),
                                              _ptr(out["accept_len"]), _ptr(out["all_accepted"])))
        return out

    def set_kv_cache(self, slots: int):
        """Allocates (through torch) a K/V cache of `slots` rows per layer and attaches it."""
        n = int(self._lib.ssd_kv_cache_bytes(self._h, slots))
        self._kv = torch.empty(n, dtype=torch.uint8, device=self.device)
        self._check(self._lib.ssd_set_kv_cache(self._h, _ptr(self._kv), n, slots))

    def ar_fallback(self, kv_start, ctx_len, first_tok: torch.Tensor, n_steps: int,
                    out: Optional[torch.Tensor] = None) -> torch.Tensor:
        ks, cl = _host_i32(kv_start), _host_i32(ctx_len)
        Br = len(ks)
        if out is None:
            out = torch.empty((n_steps, Br), dtype=torch.int32, device=self.device)
        self._check(self._lib.ar_fallback(self._h, Br, ks.tobytes(), cl.tobytes(), _ptr(first_tok), n_steps, _ptr(out)))
        return out

    # ---- trees of drafted tokens over cached rows ----------------------------------------------

    def tree_attention(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, kv_start, ctx_len, cu_nodes, parent, scale: Optional[float] = None,
                       out: Optional[torch.Tensor] = None, mass: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention of the nodes of trees (tree_attention): q [nodes, query heads, head_dim] (any stride between nodes) over k, v [slots, K/V heads,
        head_dim] (any strides but the last).  Returns out [nodes, query heads, head_dim]; mass [K/V heads, slots] collects the rows' weights, lse
        [nodes, query heads] takes the log-sum-exps (both fp32, optional).  scale: 1 / sqrt(head_dim) unless given."""
        ks, cl, cn, pa = _host_call_i32(kv_start), _host_call_i32(ctx_len), _host_call_i32(cu_nodes), _host_call_i32(parent)
        B, dev = len(cn) - 1, self.device
        view, slots, _, H, hd = _kv_view(dev, k, v)
        N, Hq, q_hd = q.shape
        q_stride, head_stride, one = q.stride()
        if len(k.shape) != 3 or q.dtype is not k.dtype or q.device != k.device or q_hd != hd or (one != 1 and hd > 1) or (Hq > 1 and head_stride != hd):
            raise ValueError("q must be [nodes, query heads, head_dim] in the type of k and v, the heads of a node consecutive, k and v of one layer")
        if len(ks) != B or len(cl) != B or len(pa) != N or (B >= 0 and cn[-1] != N):
            raise ValueError("kv_start, ctx_len, cu_nodes, parent and q do not fit together")
        if out is None:
            out = q.new_empty((N, Hq, hd))
        else:
            _on(dev, q.dtype, out=out)
            if out.numel() != N * Hq * hd:
                raise ValueError("out has the wrong size")
        if mass is not None or lse is not None:
            _on(dev, torch.float32, mass=mass, lse=lse)
            if (lse is not None and lse.numel() != N * Hq) or (mass is not None and mass.numel() != H * slots):
                raise ValueError("lse or mass has the wrong size")
        self._check(self._lib.tree_attention(self._h, q.data_ptr(), q_stride if N > 1 else Hq * hd, Hq, view, B, _host_arg(ks), _host_arg(cl), _host_arg(cn),
                                             _host_arg(pa), hd ** -0.5 if scale is None else scale, out.data_ptr(), None if lse is None else lse.data_ptr(),
                                             None if mass is None else mass.data_ptr()))
        return out

    def tree_path(self, node_logp: torch.Tensor, cu_nodes, parent, tau: float, out: Optional[dict] = None) -> dict:
        """Accepted path of every tree (tree_path)."""
        cn, pa = _host_call_i32(cu_nodes), _host_call_i32(parent)
        B, N, dev = len(cn) - 1, len(pa), self.device
        if node_logp.dtype is not torch.float32 or not node_logp.is_contiguous() or not _at(node_logp, dev):
            raise ValueError(f"node_logp must be a contiguous float32 tensor on {dev}")
        if B < 0 or node_logp.numel() != N or cn[-1] != N:
            raise ValueError("cu_nodes, parent and node_logp do not fit together")
        if out is None:
            i32 = torch.int32
            out = {"accept_len": node_logp.new_empty(B, dtype=i32), "accept_node": node_logp.new_empty(B, dtype=i32), "path": node_logp.new_empty(N, dtype=i32)}
        else:
            _on(dev, torch.int32, **out)
            if out["accept_len"].numel() < B or out["accept_node"].numel() < B or out["path"].numel() < N:
                raise ValueError("accept_len, accept_node or path is too small")
        self._check(self._lib.tree_path(self._h, node_logp.data_ptr(), B, _host_arg(cn), _host_arg(pa), tau, out["accept_len"].data_ptr(),
                                        out["accept_node"].data_ptr(), out["path"].data_ptr()))
        return out

    def kv_evict(self, k: torch.Tensor, v: torch.Tensor, mass: torch.Tensor, kv_start, ctx_len, keep, n_first: int, n_recent: int,
                 k_out: torch.Tensor, v_out: torch.Tensor, out_start, mass_out: Optional[torch.Tensor] = None,
                 want_rows: bool = False) -> Optional[torch.Tensor]:
        """Copies the rows of largest weight to another cache (kv_evict): k, v [layers, slots, K/V heads, head_dim], mass [layers, K/V heads, slots].
        Returns the numbers of the kept rows [layers, K/V heads, kept rows] if they are wanted."""
        ks, cl, kp, to_at = _host_call_i32(kv_start), _host_call_i32(ctx_len), _host_call_i32(keep), _host_call_i32(out_start)
        view, slots, L, H, _ = _kv_view(self.device, k, v)
        to, to_slots, _, _, _ = _kv_view(self.device, k_out, v_out)
        if not len(ks) == len(cl) == len(kp) == len(to_at):
            raise ValueError("kv_start, ctx_len, keep and out_start must be of one length")
        _on(self.device, torch.float32, mass=mass, mass_out=mass_out)
        if mass.numel() != L * H * slots or (mass_out is not None and mass_out.numel() != L * H * to_slots):
            raise ValueError("mass or mass_out has the wrong size")
        rows = None
        if want_rows:
            rows = torch.empty((L, H, int(np.minimum(kp, cl).clip(0).sum())), dtype=torch.int32, device=self.device)
        self._check(self._lib.kv_evict(self._h, view, mass.data_ptr(), len(ks), _host_arg(ks), _host_arg(cl), _host_arg(kp), n_first, n_recent, to,
                                       _host_arg(to_at), _ptr(mass_out), _ptr(rows)))
        return rows

    def kv_tensors(self, buf: Optional[torch.Tensor] = None, slots: int = 0):
        """(k, v) [layers, slots, K/V heads, head_dim] of the attached K/V cache, or of a uint8 tensor laid out for `slots` slots (ssd_kv_cache_view)."""
        view = KvViewC()
        if buf is not None:
            _on(self.device, torch.uint8, buf=buf)
            if buf.numel() < self.kv_cache_bytes(slots):
                raise ValueError("buf is smaller than a K/V cache of so many slots")
        self._check(self._lib.ssd_kv_cache_view(self._h, _ptr(buf), slots, C.byref(view)))
        flat = (self._kv if buf is None else buf).view(self.act_dtype)
        shape = (view.n_layers, view.slots, view.n_kv_heads, view.head_dim)
        stride = (view.layer_stride, view.slot_stride, view.head_stride, 1)
        return tuple(flat.as_strided(shape, stride, flat.storage_offset() + (p - flat.data_ptr()) // flat.element_size()) for p in (view.k, view.v))

    def kv_cache_bytes(self, slots: int) -> int:
        return int(self._lib.ssd_kv_cache_bytes(self._h, slots))

    def attach_kv_cache(self, buf: torch.Tensor, slots: int):
        """Attaches a uint8 tensor of kv_cache_bytes(slots) bytes as K/V cache."""
        _on(self.device, torch.uint8, buf=buf)
        self._check(self._lib.ssd_set_kv_cache(self._h, _ptr(buf), buf.numel(), slots))
        self._kv = buf

    def verify_tree(self, node_ids: torch.Tensor, cu_nodes, parent, kv_start, ctx_len, pos0=None, kv_mass: Optional[torch.Tensor] = None,
                    out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The decoder pass over the nodes of trees with the attached K/V cache (verify_tree); returns h_tree."""
        cn, pa, ks, cl = _host_i32(cu_nodes), _host_i32(parent), _host_i32(kv_start), _host_i32(ctx_len)
        p0 = None if pos0 is None else _host_i32(pos0)
        B, N = len(cn) - 1, len(pa)
        _on(self.device, torch.int32, node_ids=node_ids)
        _on(self.device, torch.float32, kv_mass=kv_mass)
        if int(cn[-1]) != N or node_ids.numel() != N or len(ks) != B or len(cl) != B or (p0 is not None and len(p0) != B):
            raise ValueError("cu_nodes, parent, node_ids, kv_start, ctx_len and pos0 do not fit together")
        self._check_kv_mass(kv_mass)
        if out is None:
            out = torch.empty((N, self.cfg.d_model), dtype=self.act_dtype, device=self.device)
        else:
            _on(self.device, self.act_dtype, out=out)
            if out.numel() != N * self.cfg.d_model:
                raise ValueError("out has the wrong size")
        self._check(self._lib.verify_tree(self._h, _ptr(node_ids), B, cn.tobytes(), pa.tobytes(), ks.tobytes(), cl.tobytes(),
                                          None if p0 is None else p0.tobytes(), _ptr(kv_mass), _ptr(out)))
        return out

    def _check_kv_mass(self, kv_mass):
        if kv_mass is None:
            return
        view = KvViewC()
        self._check(self._lib.ssd_kv_cache_view(self._h, None, 0, C.byref(view)))
        if kv_mass.numel() != view.n_layers * view.n_kv_heads * view.slots:
            raise ValueError("kv_mass must be [layers, K/V heads, slots of the attached cache]")

    def accept_tree(self, h_tree: torch.Tensor, node_ids: torch.Tensor, cu_nodes, parent, tau_slm: float, kv_start=None, ctx_len=None,
                    kv_mass: Optional[torch.Tensor] = None) -> dict:
        """Acceptance over the trees of verify_tree (accept_tree); with kv_start the accepted rows move behind the context."""
        cn, pa = _host_i32(cu_nodes), _host_i32(parent)
        ks, cl = (None, None) if kv_start is None else (_host_i32(kv_start), _host_i32(ctx_len))
        B, N, dev = len(cn) - 1, len(pa), self.device
        _on(dev, torch.int32, node_ids=node_ids)
        _on(dev, self.act_dtype, h_tree=h_tree)
        _on(dev, torch.float32, kv_mass=kv_mass)
        if int(cn[-1]) != N or node_ids.numel() != N or h_tree.numel() != N * self.cfg.d_model or (ks is not None and not len(ks) == len(cl) == B):
            raise ValueError("cu_nodes, parent, node_ids, h_tree, kv_start and ctx_len do not fit together")
        if ks is not None:
            self._check_kv_mass(kv_mass)
        out = {"node_logp": torch.empty(N, dtype=torch.float32, device=dev), "greedy_tok": torch.empty(N, dtype=torch.int32, device=dev),
               "accept_len": torch.empty(max(B, 0), dtype=torch.int32, device=dev), "accept_node": torch.empty(max(B, 0), dtype=torch.int32, device=dev),
               "path": torch.empty(N, dtype=torch.int32, device=dev)}
        self._check(self._lib.accept_tree(self._h, _ptr(h_tree), _ptr(node_ids), B, cn.tobytes(), pa.tobytes(), tau_slm, None if ks is None else ks.tobytes(),
                                          None if cl is None else cl.tobytes(), _ptr(kv_mass) if ks is not None else None, _ptr(out["node_logp"]),
                                          _ptr(out["greedy_tok"]), _ptr(out["accept_len"]), _ptr(out["accept_node"]), _ptr(out["path"])))
        return out

    # ---- K/V rows in pages -----------------------------------------------------------------------

    def _page_table(self, pages: KvPages, page_table: torch.Tensor, ctx_len: torch.Tensor, max_ctx: Optional[int]):
        """(ssd_page_table, utterances) of page_table [B, entries] and ctx_len [B], both int32 on the device.  (An attribute of a tensor is 0.1 us, its shape 0.25.)"""
        i32, index = torch.int32, self._index
        if page_table.dtype is not i32 or ctx_len.dtype is not i32 or page_table.get_device() != index or ctx_len.get_device() != index or pages._index != index:
            raise ValueError(f"page_table and ctx_len must be int32 tensors on the device of the context, {self.device}, and the pages be there")
        B = ctx_len.numel()
        if page_table.dim() != 2 or ctx_len.dim() != 1 or not ctx_len.is_contiguous():
            raise ValueError("page_table must be [utterances, entries], ctx_len [utterances] and contiguous")
        rows, entries = page_table.shape
        stride, one = page_table.stride()
        if rows != B or (one != 1 and entries > 1):
            raise ValueError("page_table and ctx_len must be of as many utterances, the entries of an utterance consecutive")
        most = min(entries * pages.page_rows, 1 << 30)
        if max_ctx is None:
            max_ctx = most
        elif max_ctx > most:
            raise ValueError(f"a table of {entries} entries holds {most} rows an utterance, not {max_ctx}")
        return _PAGE_TABLE.pack(page_table.data_ptr(), stride if B > 1 else max(entries, 1), ctx_len.data_ptr(), B, max_ctx), B

    def _move_pages(self, write, pages, page_table, ctx_len, k, v, start, n_rows, max_rows, max_ctx):
        table, B = self._page_table(pages, page_table, ctx_len, max_ctx)
        view, slots, _, _, _ = _kv_view(self.device, k, v)
        for t in (start, n_rows):
            if t is not None and (t.dtype is not torch.int32 or t.get_device() != self._index or t.numel() != B or not t.is_contiguous()):
                raise ValueError(f"start and n_rows must be contiguous int32 tensors of an entry an utterance on {self.device}")
        if max_rows is None:
            if start is not None or n_rows is not None or B == 0 or slots % B:
                raise ValueError("max_rows is needed where not every utterance has the same number of slots, one behind the other")
            max_rows = slots // B
        s, n = None if start is None else start.data_ptr(), None if n_rows is None else n_rows.data_ptr()
        rc = self._lib.kv_write_pages(self._h, view, s, n, max_rows, pages._view, table) if write else self._lib.kv_read_pages(self._h, pages._view, table, view, s, n, max_rows)
        if rc:
            self._check(rc)

    def kv_write_pages(self, pages: KvPages, page_table: torch.Tensor, ctx_len: torch.Tensor, k: torch.Tensor, v: torch.Tensor, start: Optional[torch.Tensor] = None,
                       n_rows: Optional[torch.Tensor] = None, max_rows: Optional[int] = None, max_ctx: Optional[int] = None):
        """Rows of k, v [layers, slots, K/V heads, head_dim] (one layer also without its dimension; any strides but the last) to the pages of their utterances
        (kv_write_pages), quantised where the pages are of 8 bits: the last n_rows[b] of the ctx_len[b] rows of utterance b are the slots from start[b] on.  Tensors of the
        device (int32): page_table [utterances, entries], ctx_len, start, n_rows.  Without start and n_rows the slots belong to the utterances in equal parts."""
        self._move_pages(True, pages, page_table, ctx_len, k, v, start, n_rows, max_rows, max_ctx)

    def kv_read_pages(self, pages: KvPages, page_table: torch.Tensor, ctx_len: torch.Tensor, k: torch.Tensor, v: torch.Tensor, start: Optional[torch.Tensor] = None,
                      n_rows: Optional[torch.Tensor] = None, max_rows: Optional[int] = None, max_ctx: Optional[int] = None):
        """The way back (kv_read_pages): the same arguments; k and v are written."""
        self._move_pages(False, pages, page_table, ctx_len, k, v, start, n_rows, max_rows, max_ctx)

    def paged_attention(self, q: torch.Tensor, pages: KvPages, page_table: torch.Tensor, ctx_len: torch.Tensor, max_ctx: Optional[int] = None,
                        scale: Optional[float] = None, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention of the newest tokens over the pages of their utterances (paged_attention): q [utterances, query heads, head_dim], or [utterances, tokens, query heads,
        head_dim] (any stride between tokens).  ctx_len counts the new tokens; max_ctx: the longest context the launch is made for (what page_table holds unless
        given).  Returns out in the shape of q; lse [.., query heads] takes the log-sum-exps (float32, optional).  scale: 1 / sqrt(head_dim) unless given."""
        table, B = self._page_table(pages, page_table, ctx_len, max_ctx)
        st, code, index = q.stride(), _KV_CODE.get(q.dtype), self._index
        if len(st) == 4:
            n, n_new, Hq, hd = q.shape
            step, q_stride, head, one = st
            if n_new == 1:
                q_stride = step
            elif n > 1 and n_new > 1 and step != n_new * q_stride:
                raise ValueError("tokens of q must lie at equal distances")
        elif len(st) == 3:
            (n, Hq, hd), n_new = q.shape, 1
            q_stride, head, one = st
        else:
            raise ValueError("q must be [utterances, [tokens,] query heads, head_dim]")
        if n != B or hd != pages.head_dim or code is None or q.get_device() != index or (one != 1 and hd > 1) or (head != hd and Hq > 1):
            raise ValueError("q must be float16, bfloat16 or float32 on the device of the pages, with their head_dim, a token of each utterance, the heads of a token consecutive")
        if n * n_new <= 1:
            q_stride = Hq * hd
        if out is None:
            out = self._like(q)
        elif out.dtype is not q.dtype or out.get_device() != index or not out.is_contiguous() or out.numel() != q.numel():
            raise ValueError("out must be contiguous, of the type, the size and the device of q")
        if lse is not None and (lse.dtype is not torch.float32 or lse.get_device() != index or not lse.is_contiguous() or lse.numel() != n * n_new * Hq):
            raise ValueError("lse must be a contiguous float32 tensor of an entry a token and query head on the device of q")
        rc = self._lib.paged_attention(self._h, q.data_ptr(), code, q_stride, Hq, n_new, pages._view, table, hd ** -0.5 if scale is None else scale, out.data_ptr(),
                                       None if lse is None else lse.data_ptr())
        if rc:
            self._check(rc)
        return out

    def _like(self, t) -> torch.Tensor:
        """A contiguous tensor like t that the context's stream writes first: of that stream, so that memory in use on the current one is not given out again."""
        if torch._C._cuda_getCurrentRawStream(self._index) == self._raw_stream:
            return torch.empty_like(t, memory_format=torch.contiguous_format)
        with torch.cuda.stream(self.stream):
            return torch.empty_like(t, memory_format=torch.contiguous_format)

    def accept_prefix(self, h_verify: torch.Tensor, draft_ids: torch.Tensor, cu_draft, tau_slm: float,
                      want_greedy: bool = False, out: Optional[dict] = None) -> dict:
        cd = _host_i32(cu_draft)
        Bv, Mv = len(cd) - 1, int(cd[-1])
        dev = self.device
        if out is None:
            out = {"draft_logp": torch.empty(Mv, dtype=torch.float32, device=dev),
                   "accept_len": torch.empty(max(Bv, 0), dtype=torch.int32, device=dev),
                   "all_accepted": torch.empty(max(Bv, 0), dtype=torch.uint8, device=dev)}
            if want_greedy:
                out["greedy_tok"] = torch.empty(Mv, dtype=torch.int32, device=dev)
        self._check(self._lib.accept_prefix(self._h, _ptr(h_verify), _ptr(draft_ids), cd.tobytes(), Bv, tau_slm,
                                            _ptr(out["draft_logp"]), _ptr(out["accept_len"]),
                                            _ptr(out["all_accepted"]), _ptr(out.get("greedy_tok"))))
        return out


NOALLOC_MAX_FRAMES = 262144


def ctc_gate_noalloc(logits: torch.Tensor, cu_frames_dev: torch.Tensor, blank_id: int, tau_ctc: float, out: dict,
                     stream=None) -> dict:
    """ctc_gate_noalloc: every buffer is the caller's (`out` holds max_entropy, gate_pass, draft_ctc, draft_len;
    cu_frames_dev is an int32 device tensor of B+1 prefix sums); the call itself allocates nothing."""
    st = stream if stream is not None else torch.cuda.current_stream(logits.device)
    B, n_frames, V = int(cu_frames_dev.numel()) - 1, int(logits.shape[0]), int(logits.shape[1])
    assert cu_frames_dev.dtype == torch.int32
    err = C.create_string_buffer(256)
    rc = lib().ctc_gate_noalloc(st.cuda_stream, _ptr(logits), _DTYPE_CODE[logits.dtype], _ptr(cu_frames_dev), B,
                                n_frames, V, blank_id, tau_ctc, _ptr(out["max_entropy"]), _ptr(out["gate_pass"]),
                                _ptr(out["draft_ctc"]), _ptr(out["draft_len"]), err, len(err))
    if rc != 0:
        raise SsdError(rc, err.value.decode())
    return out


def plan_batches(lengths, max_tokens: int, padded: bool = False):
    """Host-only batch planner (ssd_plan_batches): returns a list of index arrays, one per batch."""
    L = _host_i32(lengths)
    n = len(L)
    order = np.empty(n, dtype=np.int32)
    start = np.empty(n + 1, dtype=np.int32)
    nb = C.c_int32()
    rc = lib().ssd_plan_batches(L.ctypes.data, n, int(max_tokens), int(padded), order.ctypes.data, start.ctypes.data,
                                C.byref(nb))
    if rc != 0:
        raise SsdError(rc, "ssd_plan_batches: bad argument")
    return [order[start[k]:start[k + 1]].copy() for k in range(nb.value)]
