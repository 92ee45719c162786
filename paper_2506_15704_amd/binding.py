"""ctypes binding of liblfps.so: same names as the C ABI, argument marshalling only.

Every array argument is a torch tensor living on the GPU (PyTorch is used for device memory
and streams, nothing else); its dtype/shape/contiguity are checked here and its data pointer
is handed to the library.  There is no fallback: if the shared library is missing the import
of this module fails.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "liblfps.so")

LFPS_F32, LFPS_BF16, LFPS_F16 = 0, 1, 2
_KV_DTYPES = {"f32": (LFPS_F32, torch.float32), "bf16": (LFPS_BF16, torch.bfloat16), "f16": (LFPS_F16, torch.float16)}
LFPS_OK, LFPS_EINVAL, LFPS_ECAP, LFPS_EHIP, LFPS_ENOMEM = 0, -1, -2, -3, -4
LFPS_FLAG_CAND_OVERFLOW = 1
LFPS_FLAG_TABLE_FULL = 2
LFPS_FLAG_Q_RANGE = 4
LFPS_FLAG_PAGES_FULL = 8
N_KERNELS = 24
NOALLOC_MAX_SCORES = 2097152


class LfpsError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"liblfps error {code}: {msg}")
        self.code = code


class lfps_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "batch", "n_q_heads", "n_kv_heads", "head_dim", "kv_dtype", "max_seq_len", "max_k",
        "radius", "n_recent", "n_sink", "cand_cap", "device", "table_mode")] + [
        ("table_decay", ctypes.c_float), ("table_a", ctypes.c_float), ("k_fp8", ctypes.c_int32),
        ("v_fp8", ctypes.c_int32)]


class lfps_kv(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64), ("stride_n", ctypes.c_int64),
                ("seq_lens", ctypes.c_void_p), ("block_table", ctypes.c_void_p),
                ("block_size", ctypes.c_int32), ("block_table_stride", ctypes.c_int32),
                ("n_blocks", ctypes.c_int32)]


class lfps_rotary(ctypes.Structure):
    _fields_ = [("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("inv_freq", ctypes.c_void_p), ("pair_axis", ctypes.c_void_p),
                ("eps", ctypes.c_float), ("rotary_dim", ctypes.c_int32), ("n_axes", ctypes.c_int32), ("interleaved", ctypes.c_int32)]


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2506_15704_amd.build` "
            "(there is no CPU fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    P, I32, VP = ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p
    sig = {
        "lfps_create": (ctypes.c_int, [ctypes.POINTER(lfps_config), ctypes.POINTER(P)]),
        "lfps_destroy": (ctypes.c_int, [P]),
        "lfps_last_error": (ctypes.c_char_p, [P]),
        "lfps_workspace_bytes": (ctypes.c_int, [ctypes.POINTER(lfps_config), ctypes.POINTER(ctypes.c_int64)]),
        "lfps_host_device_pointer": (ctypes.c_int, [VP, ctypes.POINTER(VP)]),
        "lfps_cand_cap": (I32, [P]),
        "lfps_candidates": (ctypes.c_int, [P, VP, VP, VP, VP, VP, VP]),
        "lfps_score_topk": (ctypes.c_int, [P, VP, ctypes.POINTER(lfps_kv), VP, VP, VP, VP, VP, VP, VP]),
        "lfps_sparse_attn": (ctypes.c_int, [P, VP, ctypes.POINTER(lfps_kv), VP, VP, VP, VP, VP]),
        "lfps_step": (ctypes.c_int, [P, VP, ctypes.POINTER(lfps_kv), VP, VP, VP, VP, VP, VP]),
        "lfps_sparse_attn_noalloc": (ctypes.c_int, [ctypes.POINTER(lfps_config), VP, ctypes.POINTER(lfps_kv), VP, VP, VP, VP]),
        "lfps_full_attn_decode": (ctypes.c_int, [P, VP, ctypes.POINTER(lfps_kv), VP, VP]),
        "lfps_exact_topk": (ctypes.c_int, [P, VP, ctypes.POINTER(lfps_kv), VP, VP, VP, VP]),
        "lfps_poll_status": (ctypes.c_int, [P, ctypes.POINTER(I32), VP]),
        "lfps_poll_rescored": (ctypes.c_int, [P, ctypes.POINTER(I32), VP]),
        "lfps_timing_enable": (ctypes.c_int, [P, I32]),
        "lfps_timing_read": (ctypes.c_int, [P, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(I32), VP]),
        "lfps_kernel_name": (ctypes.c_char_p, [I32]),
        "lfps_calib_copy": (ctypes.c_int, [VP, VP, ctypes.c_int64, VP]),
        "lfps_set_filter": (ctypes.c_int, [P, I32]),
        "lfps_reset_history": (ctypes.c_int, [P, VP]),
        "lfps_copy_cand_count": (ctypes.c_int, [P, VP, VP]),
        "lfps_tables_init": (ctypes.c_int, [P, VP, I32, ctypes.POINTER(lfps_kv), VP]),
        "lfps_tables_import": (ctypes.c_int, [P, VP, VP, VP, VP]),
        "lfps_tables_export": (ctypes.c_int, [P, VP, VP, VP, VP]),
        "lfps_table_candidates": (ctypes.c_int, [P, VP, VP, VP, VP]),
        "lfps_table_update": (ctypes.c_int, [P, VP, VP, VP, VP, VP]),
        "lfps_table_step": (ctypes.c_int, [P, VP, ctypes.POINTER(lfps_kv), VP, VP, VP, VP, VP]),
        "lfps_priors": (ctypes.c_int, [P, VP, ctypes.POINTER(lfps_kv), VP, VP, VP, VP]),
        "lfps_head_sparsity": (ctypes.c_int, [P, VP, ctypes.POINTER(lfps_kv), VP, VP, I32, ctypes.c_float, VP, VP, VP]),
        "lfps_append": (ctypes.c_int, [P, VP, VP, ctypes.c_int64, VP, I32, ctypes.POINTER(lfps_kv), VP]),
        "lfps_prompt_attn": (ctypes.c_int, [P, VP, ctypes.c_int64, VP, I32, ctypes.POINTER(lfps_kv), VP, VP]),
        "lfps_rotate_append": (ctypes.c_int, [P, ctypes.POINTER(lfps_rotary), VP, VP, VP, ctypes.c_int64, VP, VP, I32, ctypes.POINTER(lfps_kv), VP,
                                              I32, VP]),
        "lfps_window_attn": (ctypes.c_int, [P, VP, ctypes.c_int64, VP, I32, ctypes.POINTER(lfps_kv), I32, I32, VP, VP]),
        "lfps_window_attn_decode": (ctypes.c_int, [P, VP, ctypes.POINTER(lfps_kv), I32, I32, VP, VP]),
        "lfps_attn_mass": (ctypes.c_int, [P, VP, ctypes.c_int64, VP, I32, ctypes.POINTER(lfps_kv), VP, ctypes.c_float, VP, VP]),
        "lfps_full_attn_mass_decode": (ctypes.c_int, [P, VP, ctypes.POINTER(lfps_kv), VP, ctypes.c_float, VP, VP, VP]),
        "lfps_evict": (ctypes.c_int, [P, ctypes.POINTER(lfps_kv), VP, VP, I32, I32, ctypes.POINTER(lfps_kv), VP, VP, VP, VP]),
        "lfps_prefix_attn_decode": (ctypes.c_int, [P, VP, ctypes.POINTER(lfps_kv), VP, VP, I32, VP, VP]),
        "lfps_pages_workspace_bytes": (ctypes.c_int, [I32, ctypes.POINTER(ctypes.c_int64)]),
        "lfps_pages_update": (ctypes.c_int, [P, ctypes.POINTER(lfps_kv), VP, VP, VP, VP, VP, VP, VP, ctypes.c_int64, VP]),
        "lfps_pages_compact": (ctypes.c_int, [P, ctypes.POINTER(lfps_kv), VP, VP, VP, VP, VP, VP, ctypes.c_int64, VP]),
        "lfps_pages_copy": (ctypes.c_int, [P, ctypes.POINTER(lfps_kv), VP, I32, VP]),
        "lfps_table_step_gated": (ctypes.c_int, [P, VP, ctypes.POINTER(lfps_kv), VP, VP, VP, VP, I32, ctypes.c_float,
                                                 VP, VP, VP, VP, VP]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    return lib


_lib = _load()


def kernel_names():
    return [_lib.lfps_kernel_name(i).decode() for i in range(N_KERNELS)]


def workspace_bytes(**cfg) -> int:
    c = lfps_config(**cfg)
    out = ctypes.c_int64(0)
    rc = _lib.lfps_workspace_bytes(ctypes.byref(c), ctypes.byref(out))
    if rc != LFPS_OK:
        raise LfpsError(rc, _lib.lfps_last_error(None).decode())
    return out.value


def _cache_ptr(t: torch.Tensor) -> int:
    """Address of a cache tensor for the kernels: a GPU tensor's own, or for a pinned host tensor (a host-resident
    cache) the address at which the device sees it."""
    if t.is_cuda:
        return t.data_ptr()
    if not t.is_pinned():
        raise TypeError("a cache tensor must live on the GPU or in pinned host memory")
    dev = ctypes.c_void_p(None)
    rc = _lib.lfps_host_device_pointer(t.data_ptr(), ctypes.byref(dev))
    if rc != LFPS_OK:
        raise LfpsError(rc, _lib.lfps_last_error(None).decode())
    return dev.value


def _ptr(t: Optional[torch.Tensor], dtype, shape, name: str, device) -> Optional[int]:
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.device != device:
        raise TypeError(f"{name}: expected a tensor on {device}")
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected dtype {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    return t.data_ptr()


def _token_rows(t: torch.Tensor, dtype, heads: int, name: str, device):
    """[tokens, heads, D] rows with any stride between tokens -> (address, stride between tokens)."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.device != device:
        raise TypeError(f"{name}: expected a tensor on {device}")
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected dtype {dtype}, got {t.dtype}")
    if t.dim() != 3 or t.shape[1] != heads or t.shape[2] != 128:
        raise ValueError(f"{name}: expected [tokens, {heads}, 128], got {tuple(t.shape)}")
    if t.shape[0] and (t.stride(2) != 1 or (heads > 1 and t.stride(1) != 128)):
        raise ValueError(f"{name}: the heads of a token must be contiguous")
    return t.data_ptr(), int(t.stride(0)) if t.shape[0] > 1 else heads * 128


def pages_workspace_bytes(n_blocks: int) -> int:
    out = ctypes.c_int64(0)
    rc = _lib.lfps_pages_workspace_bytes(int(n_blocks), ctypes.byref(out))
    if rc != LFPS_OK:
        raise LfpsError(rc, _lib.lfps_last_error(None).decode())
    return out.value


def lfps_calib_copy(dst: torch.Tensor, src: torch.Tensor):
    """Plain device copy with exactly known traffic (src.nbytes read, the same written)."""
    if not (dst.is_cuda and src.is_cuda and dst.is_contiguous() and src.is_contiguous()):
        raise TypeError("lfps_calib_copy: contiguous GPU tensors expected")
    nbytes = src.numel() * src.element_size()
    if nbytes != dst.numel() * dst.element_size():
        raise ValueError("lfps_calib_copy: size mismatch")
    rc = _lib.lfps_calib_copy(dst.data_ptr(), src.data_ptr(), nbytes, torch.cuda.current_stream(src.device).cuda_stream)
    if rc != LFPS_OK:
        raise LfpsError(rc, "lfps_calib_copy")


class Lfps:
    """A liblfps context.  Methods mirror the C entry points one to one."""

    def __init__(self, batch: int, n_q_heads: int = 32, n_kv_heads: int = 8, head_dim: int = 128,
                 kv_dtype: str = "bf16", max_seq_len: int = 0, max_k: int = 0, radius: int = 0,
                 n_recent: int = 1, n_sink: int = 0, cand_cap: int = 0, device: int = 0,
                 table_mode: bool = False, table_decay: float = 0.95, table_a: float = 0.2, k_fp8: bool = False,
                 v_fp8: bool = False):
        if kv_dtype not in _KV_DTYPES:
            raise ValueError(f"kv_dtype must be one of {sorted(_KV_DTYPES)} (got {kv_dtype!r})")
        self.cfg = lfps_config(batch, n_q_heads, n_kv_heads, head_dim,
                               _KV_DTYPES[kv_dtype][0], max_seq_len, max_k,
                               radius, n_recent, n_sink, cand_cap, device, int(bool(table_mode)),
                               float(table_decay), float(table_a), int(bool(k_fp8)), int(bool(v_fp8)))
        self.kv_torch_dtype = _KV_DTYPES[kv_dtype][1]
        self.k_torch_dtype = torch.float8_e4m3fn if k_fp8 else self.kv_torch_dtype
        self.v_torch_dtype = torch.float8_e4m3fn if v_fp8 else self.kv_torch_dtype
        self.device = torch.device("cuda", device)
        self._ctx = ctypes.c_void_p(None)
        rc = _lib.lfps_create(ctypes.byref(self.cfg), ctypes.byref(self._ctx))
        if rc != LFPS_OK:
            raise LfpsError(rc, _lib.lfps_last_error(None).decode())
        self.B, self.Hq, self.Hkv, self.D = batch, n_q_heads, n_kv_heads, head_dim
        self.kmax, self.Lcap = max_k, max_seq_len
        self.cand_cap = int(_lib.lfps_cand_cap(self._ctx))

    # ------------------------------------------------------------------ plumbing
    def close(self):
        if self._ctx:
            _lib.lfps_destroy(self._ctx)
            self._ctx = ctypes.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc: int):
        if rc != LFPS_OK:
            raise LfpsError(rc, _lib.lfps_last_error(self._ctx).decode())

    def _stream(self) -> int:
        return torch.cuda.current_stream(self.device).cuda_stream

    def kv_view(self, K: torch.Tensor, V: Optional[torch.Tensor], seq_lens: torch.Tensor) -> lfps_kv:
        """View of a [B, Hkv, Lcap', D] cache (any strides with a contiguous last dim); K and V on the GPU, or in
        pinned host memory for a host-resident cache (rows are then fetched over the host link)."""
        for name, t in (("K", K), ("V", V)):
            if t is None:
                continue
            want = self.k_torch_dtype if name == "K" else self.v_torch_dtype
            if not (t.is_cuda or t.is_pinned()) or t.dtype != want or t.dim() != 4:
                raise TypeError(f"{name}: expected a 4-d {want} tensor on the GPU (or in pinned host memory)")
            if t.shape[0] != self.B or t.shape[1] != self.Hkv or t.shape[3] != self.D or t.stride(3) != 1:
                raise ValueError(f"{name}: expected [B={self.B}, Hkv={self.Hkv}, rows, D={self.D}] with unit channel stride")
            if t.shape[2] < self.Lcap:
                raise ValueError(f"{name}: holds {t.shape[2]} rows per head, fewer than max_seq_len={self.Lcap}")
        if V is not None and V.stride() != K.stride():
            raise ValueError("K and V must share strides")
        sl = _ptr(seq_lens, torch.int32, (self.B,), "seq_lens", self.device)
        view = lfps_kv(_cache_ptr(K), _cache_ptr(V) if V is not None else None,
                       K.stride(0), K.stride(1), K.stride(2), sl, None, 0, 0, 0)
        view._keep = (K, V, seq_lens)   # the struct holds raw pointers: keep their tensors alive with it
        return view

    def paged_kv_view(self, K: torch.Tensor, V: Optional[torch.Tensor], block_table: torch.Tensor,
                      seq_lens: torch.Tensor) -> lfps_kv:
        """View of a paged cache: K, V are pools [n_blocks, Hkv, block_size, D] (any strides with a
        contiguous last dim, e.g. a permuted [n_blocks, block_size, Hkv, D]); block_table [B, max_blocks]
        int32 names the pool block of every logical block of a request."""
        for name, t in (("K", K), ("V", V)):
            if t is None:
                continue
            want = self.k_torch_dtype if name == "K" else self.v_torch_dtype
            if not t.is_cuda or t.dtype != want or t.dim() != 4:
                raise TypeError(f"{name}: expected a 4-d {want} tensor on the GPU")
            if t.shape[1] != self.Hkv or t.shape[3] != self.D or t.stride(3) != 1:
                raise ValueError(f"{name}: expected [n_blocks, Hkv={self.Hkv}, block_size, D={self.D}] with unit channel stride")
        if V is not None and (V.stride() != K.stride() or V.shape != K.shape):
            raise ValueError("K and V pools must share shape and strides")
        if (not block_table.is_cuda or block_table.dtype != torch.int32 or block_table.dim() != 2
                or block_table.shape[0] != self.B or block_table.stride(1) != 1):
            raise ValueError(f"block_table: expected an int32 [B={self.B}, max_blocks] tensor on the GPU with unit column stride")
        sl = _ptr(seq_lens, torch.int32, (self.B,), "seq_lens", self.device)
        view = lfps_kv(K.data_ptr(), V.data_ptr() if V is not None else None,
                       K.stride(0), K.stride(1), K.stride(2), sl, block_table.data_ptr(),
                       int(K.shape[2]), int(block_table.stride(0)), int(K.shape[0]))
        view._keep = (K, V, seq_lens, block_table)
        return view

    # ------------------------------------------------------------------ entry points
    def lfps_candidates(self, prev_topk, k, seq_lens, cand, cand_count):
        d = self.device
        self._check(_lib.lfps_candidates(
            self._ctx, _ptr(prev_topk, torch.int32, (self.B, self.Hq, self.kmax), "prev_topk", d),
            _ptr(k, torch.int32, (self.B,), "k", d), _ptr(seq_lens, torch.int32, (self.B,), "seq_lens", d),
            _ptr(cand, torch.int32, (self.B, self.Hkv, self.cand_cap), "cand", d),
            _ptr(cand_count, torch.int32, (self.B, self.Hkv), "cand_count", d), self._stream()))

    def lfps_score_topk(self, q, kv: lfps_kv, cand, cand_count, k, topk_idx, topk_score=None, cand_score=None):
        d = self.device
        self._check(_lib.lfps_score_topk(
            self._ctx, _ptr(q, torch.float32, (self.B, self.Hq, self.D), "q", d), ctypes.byref(kv),
            _ptr(cand, torch.int32, (self.B, self.Hkv, self.cand_cap), "cand", d),
            _ptr(cand_count, torch.int32, (self.B, self.Hkv), "cand_count", d),
            _ptr(k, torch.int32, (self.B,), "k", d),
            _ptr(topk_idx, torch.int32, (self.B, self.Hq, self.kmax), "topk_idx", d),
            _ptr(topk_score, torch.float32, (self.B, self.Hq, self.kmax), "topk_score", d),
            _ptr(cand_score, torch.float32, (self.B, self.Hq, self.cand_cap), "cand_score", d), self._stream()))

    def lfps_sparse_attn(self, q, kv: lfps_kv, idx, idx_score, k, out):
        d = self.device
        self._check(_lib.lfps_sparse_attn(
            self._ctx, _ptr(q, torch.float32, (self.B, self.Hq, self.D), "q", d), ctypes.byref(kv),
            _ptr(idx, torch.int32, (self.B, self.Hq, self.kmax), "idx", d),
            _ptr(idx_score, torch.float32, (self.B, self.Hq, self.kmax), "idx_score", d),
            _ptr(k, torch.int32, (self.B,), "k", d),
            _ptr(out, torch.float32, (self.B, self.Hq, self.D), "out", d), self._stream()))

    def lfps_sparse_attn_noalloc(self, q, kv: lfps_kv, idx, k, out):
        """The context-free, allocation-free S4 (scores recomputed into the library's static array), called with
        this context's configuration."""
        d = self.device
        rc = _lib.lfps_sparse_attn_noalloc(
            ctypes.byref(self.cfg), _ptr(q, torch.float32, (self.B, self.Hq, self.D), "q", d), ctypes.byref(kv),
            _ptr(idx, torch.int32, (self.B, self.Hq, self.kmax), "idx", d), _ptr(k, torch.int32, (self.B,), "k", d),
            _ptr(out, torch.float32, (self.B, self.Hq, self.D), "out", d), self._stream())
        if rc != LFPS_OK:
            raise LfpsError(rc, _lib.lfps_last_error(None).decode())

    def lfps_step(self, q, kv: lfps_kv, prev_topk, k, topk_idx, out, topk_score=None):
        d = self.device
        self._check(_lib.lfps_step(
            self._ctx, _ptr(q, torch.float32, (self.B, self.Hq, self.D), "q", d), ctypes.byref(kv),
            _ptr(prev_topk, torch.int32, (self.B, self.Hq, self.kmax), "prev_topk", d),
            _ptr(k, torch.int32, (self.B,), "k", d),
            _ptr(topk_idx, torch.int32, (self.B, self.Hq, self.kmax), "topk_idx", d),
            _ptr(topk_score, torch.float32, (self.B, self.Hq, self.kmax), "topk_score", d),
            _ptr(out, torch.float32, (self.B, self.Hq, self.D), "out", d), self._stream()))

    def lfps_full_attn_decode(self, q, kv: lfps_kv, out):
        d = self.device
        self._check(_lib.lfps_full_attn_decode(
            self._ctx, _ptr(q, torch.float32, (self.B, self.Hq, self.D), "q", d), ctypes.byref(kv),
            _ptr(out, torch.float32, (self.B, self.Hq, self.D), "out", d), self._stream()))

    def lfps_exact_topk(self, q, kv: lfps_kv, k, topk_idx, topk_score=None):
        d = self.device
        self._check(_lib.lfps_exact_topk(
            self._ctx, _ptr(q, torch.float32, (self.B, self.Hq, self.D), "q", d), ctypes.byref(kv),
            _ptr(k, torch.int32, (self.B,), "k", d),
            _ptr(topk_idx, torch.int32, (self.B, self.Hq, self.kmax), "topk_idx", d),
            _ptr(topk_score, torch.float32, (self.B, self.Hq, self.kmax), "topk_score", d), self._stream()))

    # ------------------------------------------------------------------ score tables
    def lfps_tables_init(self, q_hist, kv: lfps_kv):
        """q_hist: [s, B, Hq, D] (or [B, Hq, D] for one query), most recent query first."""
        if q_hist.dim() == 3:
            q_hist = q_hist.unsqueeze(0)
        s = int(q_hist.shape[0])
        self._check(_lib.lfps_tables_init(
            self._ctx, _ptr(q_hist, torch.float32, (s, self.B, self.Hq, self.D), "q_hist", self.device), s,
            ctypes.byref(kv), self._stream()))

    def lfps_tables_import(self, phi_ver, phi_sla, seq_lens):
        d, shp = self.device, (self.B, self.Hq, self.Lcap)
        self._check(_lib.lfps_tables_import(
            self._ctx, _ptr(phi_ver, torch.float32, shp, "phi_ver", d), _ptr(phi_sla, torch.float32, shp, "phi_sla", d),
            _ptr(seq_lens, torch.int32, (self.B,), "seq_lens", d), self._stream()))

    def lfps_tables_export(self, phi_ver, phi_sla, seq_lens):
        d, shp = self.device, (self.B, self.Hq, self.Lcap)
        self._check(_lib.lfps_tables_export(
            self._ctx, _ptr(phi_ver, torch.float64, shp, "phi_ver", d), _ptr(phi_sla, torch.float64, shp, "phi_sla", d),
            _ptr(seq_lens, torch.int32, (self.B,), "seq_lens", d), self._stream()))

    def lfps_table_candidates(self, seq_lens, cand, cand_count):
        d = self.device
        self._check(_lib.lfps_table_candidates(
            self._ctx, _ptr(seq_lens, torch.int32, (self.B,), "seq_lens", d),
            _ptr(cand, torch.int32, (self.B, self.Hkv, self.cand_cap), "cand", d),
            _ptr(cand_count, torch.int32, (self.B, self.Hkv), "cand_count", d), self._stream()))

    def lfps_table_update(self, idx, idx_score, k, seq_lens):
        d = self.device
        self._check(_lib.lfps_table_update(
            self._ctx, _ptr(idx, torch.int32, (self.B, self.Hq, self.kmax), "idx", d),
            _ptr(idx_score, torch.float32, (self.B, self.Hq, self.kmax), "idx_score", d),
            _ptr(k, torch.int32, (self.B,), "k", d), _ptr(seq_lens, torch.int32, (self.B,), "seq_lens", d),
            self._stream()))

    def lfps_table_step(self, q, kv: lfps_kv, k, topk_idx, out, topk_score=None):
        d = self.device
        self._check(_lib.lfps_table_step(
            self._ctx, _ptr(q, torch.float32, (self.B, self.Hq, self.D), "q", d), ctypes.byref(kv),
            _ptr(k, torch.int32, (self.B,), "k", d),
            _ptr(topk_idx, torch.int32, (self.B, self.Hq, self.kmax), "topk_idx", d),
            _ptr(topk_score, torch.float32, (self.B, self.Hq, self.kmax), "topk_score", d),
            _ptr(out, torch.float32, (self.B, self.Hq, self.D), "out", d), self._stream()))

    # ------------------------------------------------------------------ head sparsity bypass
    def lfps_priors(self, q, kv: lfps_kv, kbar, vbar, sigma2_hat):
        d = self.device
        self._check(_lib.lfps_priors(
            self._ctx, _ptr(q, torch.float32, (self.B, self.Hq, self.D), "q", d), ctypes.byref(kv),
            _ptr(kbar, torch.float32, (self.B, self.Hkv, self.D), "kbar", d),
            _ptr(vbar, torch.float32, (self.B, self.Hkv, self.D), "vbar", d),
            _ptr(sigma2_hat, torch.float32, (self.B, self.Hq), "sigma2_hat", d), self._stream()))

    def lfps_head_sparsity(self, q, kv: lfps_kv, kbar, sigma2_hat, n_local, eps, rho, gate):
        d = self.device
        self._check(_lib.lfps_head_sparsity(
            self._ctx, _ptr(q, torch.float32, (self.B, self.Hq, self.D), "q", d), ctypes.byref(kv),
            _ptr(kbar, torch.float32, (self.B, self.Hkv, self.D), "kbar", d),
            _ptr(sigma2_hat, torch.float32, (self.B, self.Hq), "sigma2_hat", d), int(n_local), float(eps),
            _ptr(rho, torch.float32, (self.B, self.Hq), "rho", d),
            _ptr(gate, torch.int32, (self.B, self.Hq), "gate", d), self._stream()))

    def lfps_table_step_gated(self, q, kv: lfps_kv, k, kbar, vbar, sigma2_hat, n_local, eps, topk_idx, out,
                              topk_score=None, gate_out=None):
        d = self.device
        self._check(_lib.lfps_table_step_gated(
            self._ctx, _ptr(q, torch.float32, (self.B, self.Hq, self.D), "q", d), ctypes.byref(kv),
            _ptr(k, torch.int32, (self.B,), "k", d),
            _ptr(kbar, torch.float32, (self.B, self.Hkv, self.D), "kbar", d),
            _ptr(vbar, torch.float32, (self.B, self.Hkv, self.D), "vbar", d),
            _ptr(sigma2_hat, torch.float32, (self.B, self.Hq), "sigma2_hat", d), int(n_local), float(eps),
            _ptr(topk_idx, torch.int32, (self.B, self.Hq, self.kmax), "topk_idx", d),
            _ptr(topk_score, torch.float32, (self.B, self.Hq, self.kmax), "topk_score", d),
            _ptr(out, torch.float32, (self.B, self.Hq, self.D), "out", d),
            _ptr(gate_out, torch.int32, (self.B, self.Hq), "gate_out", d), self._stream()))

    # ------------------------------------------------------------------ prompts, forks and pages
    def lfps_append(self, k_new, v_new, cu, kv: lfps_kv):
        """k_new, v_new: [tokens, Hkv, D] of kv_dtype, packed (slices of one fused projection: equal token strides); the cache
        behind the view is written."""
        d = self.device
        pk, sk = _token_rows(k_new, self.kv_torch_dtype, self.Hkv, "k_new", d)
        pv, sv = _token_rows(v_new, self.kv_torch_dtype, self.Hkv, "v_new", d)
        if k_new.shape != v_new.shape or sk != sv:
            raise ValueError("k_new and v_new must share shape and token stride")
        if k_new.shape[0] == 0:
            return
        self._check(_lib.lfps_append(self._ctx, pk, pv, sk, _ptr(cu, torch.int32, (self.B + 1,), "cu", d), int(k_new.shape[0]),
                                     ctypes.byref(kv), self._stream()))

    def lfps_prompt_attn(self, q, cu, kv: lfps_kv, out):
        """q: [tokens, Hq, D] of kv_dtype, packed, any stride between tokens; out: the same shape and type, contiguous."""
        d = self.device
        pq, sq = _token_rows(q, self.kv_torch_dtype, self.Hq, "q", d)
        po = _ptr(out, self.kv_torch_dtype, tuple(q.shape), "out", d)
        if q.shape[0] == 0:
            return
        self._check(_lib.lfps_prompt_attn(self._ctx, pq, sq, _ptr(cu, torch.int32, (self.B + 1,), "cu", d), int(q.shape[0]),
                                          ctypes.byref(kv), po, self._stream()))

    # ------------------------------------------------------------------ a cache of bounded length
    def rotary(self, inv_freq=None, q_weight=None, k_weight=None, eps: float = 0.0, pair_axis=None, n_axes: int = 1,
               interleaved: bool = False) -> lfps_rotary:
        """How lfps_rotate_append norms and turns heads: inv_freq [rotary_dim / 2] fp32 (None: nothing is turned), weights [D] fp32 (None: no
        norm), pair_axis [rotary_dim / 2] int32."""
        d, half = self.device, 0 if inv_freq is None else int(inv_freq.shape[0])
        rot = lfps_rotary(_ptr(q_weight, torch.float32, (self.D,), "q_weight", d), _ptr(k_weight, torch.float32, (self.D,), "k_weight", d),
                          _ptr(inv_freq, torch.float32, (half,), "inv_freq", d), _ptr(pair_axis, torch.int32, (half,), "pair_axis", d),
                          float(eps), 2 * half, int(n_axes), int(bool(interleaved)))
        rot._keep = (q_weight, k_weight, inv_freq, pair_axis)
        return rot

    def lfps_rotate_append(self, rot: lfps_rotary, q, k_new, v_new, positions, cu, kv: lfps_kv, q_out):
        """q, k_new, v_new: [tokens, heads, D] of kv_dtype, packed (slices of one fused projection: equal token strides); positions: [n_axes, tokens]
        int32, [tokens] for one axis, or None (the cache rows: not after an eviction); q_out: [tokens, Hq, D], fp32 or kv_dtype.  The
        cache behind the view is written."""
        d, T = self.device, int(q.shape[0])
        pq, sq = _token_rows(q, self.kv_torch_dtype, self.Hq, "q", d)
        pk, sk = _token_rows(k_new, self.kv_torch_dtype, self.Hkv, "k_new", d)
        pv, sv = _token_rows(v_new, self.kv_torch_dtype, self.Hkv, "v_new", d)
        if k_new.shape[0] != T or v_new.shape[0] != T or (T > 1 and not sq == sk == sv):
            raise ValueError("q, k_new and v_new must share tokens and token stride")
        if positions is not None and positions.dim() == 1:
            positions = positions.unsqueeze(0)
        pp = _ptr(positions, torch.int32, (rot.n_axes, T), "positions", d)
        if q_out.dtype not in (torch.float32, self.kv_torch_dtype):
            raise TypeError(f"q_out: expected dtype torch.float32 or {self.kv_torch_dtype}, got {q_out.dtype}")
        po = _ptr(q_out, q_out.dtype, tuple(q.shape), "q_out", d)
        if T == 0:
            return
        self._check(_lib.lfps_rotate_append(
            self._ctx, ctypes.byref(rot), pq, pk, pv, max(sq, sk, sv), pp, _ptr(cu, torch.int32, (self.B + 1,), "cu", d), T, ctypes.byref(kv), po,
            LFPS_F32 if q_out.dtype == torch.float32 else self.cfg.kv_dtype, self._stream()))

    def lfps_window_attn(self, q, cu, kv: lfps_kv, window: int, n_sink: int, out):
        """Arguments as lfps_prompt_attn's; a token sees the newest `window` rows up to its own and the first n_sink."""
        d = self.device
        pq, sq = _token_rows(q, self.kv_torch_dtype, self.Hq, "q", d)
        po = _ptr(out, self.kv_torch_dtype, tuple(q.shape), "out", d)
        if q.shape[0] == 0:
            return
        self._check(_lib.lfps_window_attn(self._ctx, pq, sq, _ptr(cu, torch.int32, (self.B + 1,), "cu", d), int(q.shape[0]), ctypes.byref(kv),
                                          int(window), int(n_sink), po, self._stream()))

    def lfps_window_attn_decode(self, q, kv: lfps_kv, window: int, n_sink: int, out):
        d = self.device
        self._check(_lib.lfps_window_attn_decode(
            self._ctx, _ptr(q, torch.float32, (self.B, self.Hq, self.D), "q", d), ctypes.byref(kv), int(window), int(n_sink),
            _ptr(out, torch.float32, (self.B, self.Hq, self.D), "out", d), self._stream()))

    def lfps_attn_mass(self, q, cu, kv: lfps_kv, mass, held=None, decay: float = 1.0):
        """q: [tokens, Hq, D] of kv_dtype, packed: the requests' newest tokens; mass: [B, Hkv, max_seq_len] fp32; held: [B] rows that have a weight
        already (None: mass is written whole)."""
        d = self.device
        pq, sq = _token_rows(q, self.kv_torch_dtype, self.Hq, "q", d)
        self._check(_lib.lfps_attn_mass(
            self._ctx, pq, sq, _ptr(cu, torch.int32, (self.B + 1,), "cu", d), int(q.shape[0]), ctypes.byref(kv),
            _ptr(held, torch.int32, (self.B,), "held", d), float(decay), _ptr(mass, torch.float32, (self.B, self.Hkv, self.Lcap), "mass", d),
            self._stream()))

    def lfps_full_attn_mass_decode(self, q, kv: lfps_kv, mass, out, held=None, decay: float = 1.0):
        d = self.device
        self._check(_lib.lfps_full_attn_mass_decode(
            self._ctx, _ptr(q, torch.float32, (self.B, self.Hq, self.D), "q", d), ctypes.byref(kv), _ptr(held, torch.int32, (self.B,), "held", d),
            float(decay), _ptr(mass, torch.float32, (self.B, self.Hkv, self.Lcap), "mass", d),
            _ptr(out, torch.float32, (self.B, self.Hq, self.D), "out", d), self._stream()))

    def lfps_evict(self, kv: lfps_kv, mass, budget, n_sink: int, n_recent: int, mass_out, kept, lens_out, to: Optional[lfps_kv] = None):
        """mass, mass_out [B, Hkv, max_seq_len] fp32, kept the same in int32, budget and lens_out [B] int32; to: the view that receives the kept rows
        (None: in place, the cache behind kv is written)."""
        d, shape = self.device, (self.B, self.Hkv, self.Lcap)
        self._check(_lib.lfps_evict(
            self._ctx, ctypes.byref(kv), _ptr(mass, torch.float32, shape, "mass", d), _ptr(budget, torch.int32, (self.B,), "budget", d), int(n_sink),
            int(n_recent), None if to is None else ctypes.byref(to), _ptr(mass_out, torch.float32, shape, "mass_out", d),
            _ptr(kept, torch.int32, shape, "kept", d), _ptr(lens_out, torch.int32, (self.B,), "lens_out", d), self._stream()))

    def lfps_prefix_attn_decode(self, q, kv: lfps_kv, group_start, prefix_len, out):
        d, n = self.device, int(prefix_len.shape[0])
        self._check(_lib.lfps_prefix_attn_decode(
            self._ctx, _ptr(q, torch.float32, (self.B, self.Hq, self.D), "q", d), ctypes.byref(kv),
            _ptr(group_start, torch.int32, (n + 1,), "group_start", d), _ptr(prefix_len, torch.int32, (n,), "prefix_len", d), n,
            _ptr(out, torch.float32, (self.B, self.Hq, self.D), "out", d), self._stream()))

    def pages_workspace(self, n_blocks: int) -> torch.Tensor:
        """Working memory for lfps_pages_update and lfps_pages_compact on a pool of n_blocks."""
        return torch.empty(pages_workspace_bytes(n_blocks), dtype=torch.uint8, device=self.device)

    def lfps_pages_update(self, kv: lfps_kv, parent, new_lens, table_out, lens_out, copies, work, held=None):
        d, B = self.device, self.B
        self._check(_lib.lfps_pages_update(
            self._ctx, ctypes.byref(kv), _ptr(parent, torch.int32, (B,), "parent", d), _ptr(new_lens, torch.int32, (B,), "new_lens", d),
            _ptr(held, torch.int32, (kv.n_blocks,), "held", d),
            _ptr(table_out, torch.int32, (B, kv.block_table_stride), "table_out", d), _ptr(lens_out, torch.int32, (B,), "lens_out", d),
            _ptr(copies, torch.int32, (B, 3), "copies", d), _ptr(work, torch.uint8, (work.numel(),), "work", d), work.numel(),
            self._stream()))

    def lfps_pages_compact(self, kv: lfps_kv, table_out, moves, block_map, n_live, work, held=None):
        d, n = self.device, kv.n_blocks
        self._check(_lib.lfps_pages_compact(
            self._ctx, ctypes.byref(kv), _ptr(held, torch.int32, (n,), "held", d),
            _ptr(table_out, torch.int32, (self.B, kv.block_table_stride), "table_out", d),
            _ptr(moves, torch.int32, (n // 2, 3), "moves", d), _ptr(block_map, torch.int32, (n,), "block_map", d),
            _ptr(n_live, torch.int32, (1,), "n_live", d), _ptr(work, torch.uint8, (work.numel(),), "work", d), work.numel(),
            self._stream()))

    def lfps_pages_copy(self, kv: lfps_kv, copies):
        n = int(copies.shape[0])
        p = _ptr(copies, torch.int32, (n, 3), "copies", self.device)
        if n:
            self._check(_lib.lfps_pages_copy(self._ctx, ctypes.byref(kv), p, n, self._stream()))

    def lfps_set_filter(self, on: bool):
        self._check(_lib.lfps_set_filter(self._ctx, int(bool(on))))

    def lfps_reset_history(self):
        self._check(_lib.lfps_reset_history(self._ctx, self._stream()))

    def lfps_copy_cand_count(self, dst):
        self._check(_lib.lfps_copy_cand_count(
            self._ctx, _ptr(dst, torch.int32, (self.B, self.Hkv), "dst", self.device), self._stream()))

    def lfps_poll_status(self) -> int:
        flags = ctypes.c_int32(0)
        self._check(_lib.lfps_poll_status(self._ctx, ctypes.byref(flags), self._stream()))
        return flags.value

    def lfps_poll_rescored(self) -> int:
        n = ctypes.c_int32(0)
        self._check(_lib.lfps_poll_rescored(self._ctx, ctypes.byref(n), self._stream()))
        return n.value

    def lfps_timing_enable(self, on: bool):
        self._check(_lib.lfps_timing_enable(self._ctx, int(bool(on))))

    def lfps_timing_read(self):
        """-> {kernel name: (total ms, launches)} since the last read."""
        ms = (ctypes.c_float * N_KERNELS)()
        n = (ctypes.c_int32 * N_KERNELS)()
        self._check(_lib.lfps_timing_read(self._ctx, ms, n, self._stream()))
        return {name: (float(ms[i]), int(n[i])) for i, name in enumerate(kernel_names())}
