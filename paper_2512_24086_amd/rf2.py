"""Thin ctypes binding of librf2.so: same names as the C ABI, argument marshalling only.

PyTorch supplies device memory and streams; every step of the layer runs in the HIP
kernels of the library.  There is no fallback: if librf2.so is missing, loading raises.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "librf2.so")

RF2_OK = 0
RF2_ERR_INVALID_ARG, RF2_ERR_UNSUPPORTED, RF2_ERR_ALLOC, RF2_ERR_HIP, RF2_ERR_TOO_LARGE = -1, -2, -3, -4, -5
RF2_BUDGET_GLOBAL, RF2_BUDGET_ROW_INCL_SINK, RF2_BUDGET_ROW_PLUS_SINK = 0, 1, 2
RF2_LAYOUT_BHND, RF2_LAYOUT_BNHD = 0, 1
RF2_SELECT_TOPN, RF2_SELECT_CDF = 0, 1
RF2_DTYPE_BF16, RF2_DTYPE_F16 = 0, 1
RF2_PAGED_BAD_LENGTH, RF2_PAGED_SEQ_FULL, RF2_PAGED_TOKENS_FULL, RF2_PAGED_POOL_FULL = 1, 2, 4, 8


class rf2_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "heads", "head_dim", "T", "H", "W", "wt", "wh", "ww",
                                         "block", "sink_frames", "sink_at_end")] + \
               [("sparsity", C.c_float), ("budget_mode", C.c_int32), ("qkv_layout", C.c_int32), ("text_tokens", C.c_int32),
                ("select_mode", C.c_int32), ("cdf_threshold", C.c_float), ("block_k", C.c_int32)]


class rf2_info(C.Structure):
    _fields_ = [("N", C.c_int64), ("N_pad", C.c_int64), ("n_blocks", C.c_int32), ("last_block_valid", C.c_int32),
                ("sink_block_begin", C.c_int32), ("sink_block_end", C.c_int32), ("k_row", C.c_int32),
                ("k_sel", C.c_int32), ("wt", C.c_int32), ("wh", C.c_int32), ("ww", C.c_int32),
                ("kept_pairs_per_head", C.c_int64), ("achieved_sparsity", C.c_double),
                ("workspace_bytes", C.c_int64), ("block_k", C.c_int32), ("n_blocks_k", C.c_int32),
                ("last_block_valid_k", C.c_int32), ("sink_block_begin_k", C.c_int32), ("sink_block_end_k", C.c_int32),
                ("N_pad_k", C.c_int64)]


class rf2_paged_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("heads", "kv_heads", "head_dim", "page", "n_pages", "max_seqs", "max_pages",
                                         "max_tokens", "dtype", "causal")] + [("scale", C.c_float)]


class rf2_paged_info(C.Structure):
    _fields_ = [("cache_elements", C.c_int64), ("workspace_bytes", C.c_int64)]


# symbol -> (restype, argtypes); also the list of exports the tests check
SIGNATURES = {
    "rf2_plan_create": (C.c_int, [C.POINTER(rf2_config), C.POINTER(C.c_void_p)]),
    "rf2_plan_destroy": (C.c_int, [C.c_void_p]),
    "rf2_plan_info": (C.c_int, [C.c_void_p, C.POINTER(rf2_info)]),
    "rf2_plan_perm": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "rf2_permute": (C.c_int, [C.c_void_p] * 10),
    "rf2_predict_mask": (C.c_int, [C.c_void_p] * 9),
    "rf2_block_sparse_attn": (C.c_int, [C.c_void_p] * 9),
    "rf2_block_sparse_attn_unpermuted": (C.c_int, [C.c_void_p] * 9),
    "rf2_unpermute": (C.c_int, [C.c_void_p] * 4),
    "rf2_paged_plan_create": (C.c_int, [C.POINTER(rf2_paged_config), C.POINTER(C.c_void_p)]),
    "rf2_paged_plan_destroy": (C.c_int, [C.c_void_p]),
    "rf2_paged_plan_info": (C.c_int, [C.c_void_p, C.POINTER(rf2_paged_info)]),
    "rf2_paged_append": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32] + [C.c_void_p] * 11),
    "rf2_paged_release": (C.c_int, [C.c_void_p, C.c_int32] + [C.c_void_p] * 9),
    "rf2_paged_store": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64] + [C.c_void_p] * 4),
    "rf2_paged_attn": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_int64] + [C.c_void_p] * 9),
    "rf2_measure_peaks": (C.c_int, [C.POINTER(C.c_double), C.POINTER(C.c_double), C.c_void_p]),
    "rf2_measure_sustained_mfma": (C.c_int, [C.c_double, C.POINTER(C.c_double), C.c_void_p]),
    "rf2_probe_xcd_mapping": (C.c_int, [C.POINTER(C.c_int32), C.POINTER(C.c_int32), C.POINTER(C.c_int32), C.c_void_p]),
    "rf2_probe_xcd_mapping_static": (C.c_int, [C.c_int32, C.c_void_p, C.c_void_p]),
    "rf2_strerror": (C.c_char_p, [C.c_int]),
    "rf2_version": (C.c_int, []),
}

_lib = None


def lib() -> C.CDLL:
    """Loads librf2.so (built beforehand by paper_2512_24086_amd.build); raises if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2512_24086_amd.build` "
                               "(there is no fallback implementation)")
        _lib = C.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(_lib, name)
            fn.restype, fn.argtypes = res, args
    return _lib


class Rf2Error(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {lib().rf2_strerror(code).decode()} ({code})")


def _check(code: int, where: str) -> None:
    if code != RF2_OK:
        raise Rf2Error(code, where)


def _ptr(t):
    """Address of a tensor, or None (the argument types of SIGNATURES turn both into a void*)."""
    if t is None:
        return None
    assert t.is_contiguous(), "tensors handed to librf2 must be contiguous"
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def rf2_measure_peaks(stream=None):
    """(bf16 MFMA-loop TFLOP/s, copy-kernel GB/s) measured on the current device."""
    mfma, copy = C.c_double(0.0), C.c_double(0.0)
    _check(lib().rf2_measure_peaks(C.byref(mfma), C.byref(copy), _stream(stream)), "rf2_measure_peaks")
    return mfma.value, copy.value


def rf2_measure_sustained_mfma(seconds, stream=None):
    """bf16 MFMA TFLOP/s sustained for `seconds` on pseudo-random operands (the power-limited ceiling)."""
    out = C.c_double(0.0)
    _check(lib().rf2_measure_sustained_mfma(C.c_double(seconds), C.byref(out), _stream(stream)),
           "rf2_measure_sustained_mfma")
    return out.value


def rf2_probe_xcd_mapping(stream=None):
    """(workgroups on the XCD of their residue class g % 8, workgroups launched, XCD of workgroup 0)."""
    agree, total, first = C.c_int32(0), C.c_int32(0), C.c_int32(-1)
    _check(lib().rf2_probe_xcd_mapping(C.byref(agree), C.byref(total), C.byref(first), _stream(stream)),
           "rf2_probe_xcd_mapping")
    return agree.value, total.value, first.value


def rf2_probe_xcd_mapping_static(n_launch, result, stream=None):
    """Allocation-free probe: leaves (agreeing workgroups, XCD of workgroup 0) in `result` (device int32[2])."""
    _check(lib().rf2_probe_xcd_mapping_static(C.c_int32(n_launch), _ptr(result), _stream(stream)),
           "rf2_probe_xcd_mapping_static")


class Plan:
    """Owner of an rf2_plan*; methods carry the names of the C entry points."""

    def __init__(self, *, batch, heads, head_dim, T, H, W, block, sparsity, sink_frames=0, sink_at_end=1,
                 window=(0, 0, 0), budget_mode=RF2_BUDGET_GLOBAL, qkv_layout=RF2_LAYOUT_BHND, text_tokens=0,
                 cdf_threshold=None, block_k=0):
        self.cfg = rf2_config(batch, heads, head_dim, T, H, W, window[0], window[1], window[2], block,
                              sink_frames, int(sink_at_end), float(sparsity), budget_mode, qkv_layout, text_tokens,
                              RF2_SELECT_TOPN if cdf_threshold is None else RF2_SELECT_CDF,
                              0.0 if cdf_threshold is None else float(cdf_threshold), block_k)
        self._h = C.c_void_p(0)
        _check(lib().rf2_plan_create(C.byref(self.cfg), C.byref(self._h)), "rf2_plan_create")
        self.info = rf2_info()
        _check(lib().rf2_plan_info(self._h, C.byref(self.info)), "rf2_plan_info")

    def close(self):
        if self._h:
            lib().rf2_plan_destroy(self._h)
            self._h = C.c_void_p(0)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- host tables -------------------------------------------------------------------
    def rf2_plan_perm(self):
        import numpy as np
        perm = np.empty(self.info.N, dtype=np.int32)
        inv = np.empty(self.info.N, dtype=np.int32)
        _check(lib().rf2_plan_perm(self._h, perm.ctypes.data, inv.ctypes.data), "rf2_plan_perm")
        return perm, inv

    # -- buffers (allocation only) -----------------------------------------------------------
    def alloc(self, device="cuda", dense_mask=False, scores=False, lse=False):
        c, i = self.cfg, self.info
        bh = (c.batch, c.heads)
        bf = dict(dtype=torch.bfloat16, device=device)
        buf = dict(
            qp=torch.empty(*bh, i.N_pad, c.head_dim, **bf),
            kp=torch.empty(*bh, i.n_blocks_k, i.block_k // 64, c.head_dim // 8, 64, 8, **bf),
            vp=torch.empty(*bh, i.n_blocks_k, i.block_k // 64, 8, c.head_dim, 8, **bf),
            qbar=torch.empty(*bh, i.n_blocks, c.head_dim, dtype=torch.float32, device=device),
            kbar=torch.empty(*bh, i.n_blocks_k, c.head_dim, dtype=torch.float32, device=device),
            blk_idx=torch.empty(*bh, i.n_blocks, i.k_row, dtype=torch.int32, device=device),
            blk_cnt=torch.empty(*bh, i.n_blocks, dtype=torch.int32, device=device),
            op=torch.empty(*bh, i.N_pad, c.head_dim, **bf),
            o=(torch.empty(c.batch, i.N, c.heads, c.head_dim, **bf) if c.qkv_layout == RF2_LAYOUT_BNHD
               else torch.empty(*bh, i.N, c.head_dim, **bf)))
        if dense_mask:
            buf["mask_dense"] = torch.empty(*bh, i.n_blocks, i.n_blocks_k, dtype=torch.uint8, device=device)
        if scores:
            buf["scores"] = torch.empty(*bh, i.n_blocks, i.n_blocks_k, dtype=torch.float32, device=device)
        if lse:
            buf["lse"] = torch.empty(*bh, i.N_pad, dtype=torch.float32, device=device)
        return buf

    # -- the four calls --------------------------------------------------------------------
    def rf2_permute(self, q, k, v, qp, kp, vp, qbar=None, kbar=None, stream=None):
        _check(lib().rf2_permute(self._h, _ptr(q), _ptr(k), _ptr(v), _ptr(qp), _ptr(kp), _ptr(vp), _ptr(qbar),
                                 _ptr(kbar), _stream(stream)), "rf2_permute")

    def rf2_predict_mask(self, qbar, kbar, blk_idx, blk_cnt, mask_dense=None, scores=None, workspace=None,
                         stream=None):
        _check(lib().rf2_predict_mask(self._h, _ptr(qbar), _ptr(kbar), _ptr(blk_idx), _ptr(blk_cnt),
                                      _ptr(mask_dense), _ptr(scores), _ptr(workspace), _stream(stream)),
               "rf2_predict_mask")

    def rf2_block_sparse_attn(self, qp, kp, vp, blk_idx, blk_cnt, op, lse=None, stream=None):
        _check(lib().rf2_block_sparse_attn(self._h, _ptr(qp), _ptr(kp), _ptr(vp), _ptr(blk_idx), _ptr(blk_cnt),
                                           _ptr(op), _ptr(lse), _stream(stream)), "rf2_block_sparse_attn")

    def rf2_block_sparse_attn_unpermuted(self, qp, kp, vp, blk_idx, blk_cnt, o, lse=None, stream=None):
        _check(lib().rf2_block_sparse_attn_unpermuted(self._h, _ptr(qp), _ptr(kp), _ptr(vp), _ptr(blk_idx),
                                                      _ptr(blk_cnt), _ptr(o), _ptr(lse), _stream(stream)),
               "rf2_block_sparse_attn_unpermuted")

    def rf2_unpermute(self, op, o, stream=None):
        _check(lib().rf2_unpermute(self._h, _ptr(op), _ptr(o), _stream(stream)), "rf2_unpermute")

    def layer_fused(self, q, k, v, buf, stream=None):
        """The whole layer with the inverse permutation fused into the attention epilogue; returns buf['o']."""
        stream = torch.cuda.current_stream() if stream is None else stream
        self.rf2_permute(q, k, v, buf["qp"], buf["kp"], buf["vp"], buf["qbar"], buf["kbar"], stream)
        self.rf2_predict_mask(buf["qbar"], buf["kbar"], buf["blk_idx"], buf["blk_cnt"], buf.get("mask_dense"),
                              buf.get("scores"), None, stream)
        self.rf2_block_sparse_attn_unpermuted(buf["qp"], buf["kp"], buf["vp"], buf["blk_idx"], buf["blk_cnt"],
                                              buf["o"], None, stream)
        return buf["o"]

    def layer(self, q, k, v, buf, stream=None):
        """The whole layer, in order; returns buf['o']."""
        stream = torch.cuda.current_stream() if stream is None else stream
        self.rf2_permute(q, k, v, buf["qp"], buf["kp"], buf["vp"], buf["qbar"], buf["kbar"], stream)
        self.rf2_predict_mask(buf["qbar"], buf["kbar"], buf["blk_idx"], buf["blk_cnt"], buf.get("mask_dense"),
                              buf.get("scores"), None, stream)
        self.rf2_block_sparse_attn(buf["qp"], buf["kp"], buf["vp"], buf["blk_idx"], buf["blk_cnt"], buf["op"],
                                   buf.get("lse"), stream)
        self.rf2_unpermute(buf["op"], buf["o"], stream)
        return buf["o"]


# (of torch's two ways to the current stream the one that makes no object of it: 0.1 us in place of 2.8)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _arg(t, what, dtype, numel, device):
    """Address of a contiguous tensor of `numel` elements of `dtype` on the plan's device."""
    if t.dtype is not dtype or t.numel() != numel or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{what}: expected {numel} contiguous elements of {dtype} on device {device}, got "
                         f"{tuple(t.shape)} of {t.dtype} on {t.device}, strides {t.stride()}")
    return t.data_ptr()


def _rows(t, what, dtype, shape, device):
    """Address of a [tokens, heads, head_dim] tensor whose rows may be further apart than they are long, and how far."""
    tokens, heads, dim = t.shape if t.dim() == 3 else (0, 0, 0)
    stride = t.stride()
    if (t.dim() != 3 or (tokens, heads, dim) != shape or t.dtype is not dtype or t.get_device() != device
            or (tokens > 0 and (stride[2] != 1 or (heads > 1 and stride[1] != dim)))):
        raise ValueError(f"{what}: expected {shape} of {dtype} on device {device}, heads and channels dense, got "
                         f"{tuple(t.shape)} of {t.dtype} on {t.device}, strides {stride}")
    return t.data_ptr(), stride[0] if tokens > 1 else heads * dim


class PagedPlan:
    """Owner of an rf2_paged_plan*: a paged cache of keys and values and the attention of new tokens over it.

    The caller owns every tensor; `alloc` makes those that live as long as the cache, `alloc_step` those of a step.  A step:

        plan.rf2_paged_append(seq_len, new_len, free_pages, n_free, block_table, seq_len, n_free, cu_new, slots, status)
        for every layer:
            plan.rf2_paged_store(k, v, slots, k_cache, v_cache)
            plan.rf2_paged_attn(q, k_cache, v_cache, block_table, seq_len, cu_new, workspace, o)

    n_seqs is the length of new_len (or done, or seq_len), n_tokens that of slots (or q): both may change from call to
    call up to max_seqs and max_tokens, and rows behind the last new token are padding.
    """

    def __init__(self, *, heads, kv_heads, head_dim, page, n_pages, max_seqs, max_pages, max_tokens, dtype=torch.bfloat16,
                 causal=True, scale=None):
        if dtype not in (torch.bfloat16, torch.float16):
            raise ValueError(f"dtype: expected torch.bfloat16 or torch.float16, got {dtype}")
        self.dtype = dtype
        self.cfg = rf2_paged_config(heads, kv_heads, head_dim, page, n_pages, max_seqs, max_pages, max_tokens,
                                    RF2_DTYPE_F16 if dtype is torch.float16 else RF2_DTYPE_BF16, int(causal),
                                    0.0 if scale is None else float(scale))
        self._h = C.c_void_p(0)
        _check(lib().rf2_paged_plan_create(C.byref(self.cfg), C.byref(self._h)), "rf2_paged_plan_create")
        self.info = rf2_paged_info()
        _check(lib().rf2_paged_plan_info(self._h, C.byref(self.info)), "rf2_paged_plan_info")
        self.device = torch.cuda.current_device() if torch.cuda.is_available() else -1

    def close(self):
        if self._h:
            lib().rf2_paged_plan_destroy(self._h)
            self._h = C.c_void_p(0)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- buffers (allocation and the state of an empty cache) ---------------------------------
    def alloc(self, device="cuda"):
        """The cache of one layer and the tables, empty: every page on the stack, page 0 on top.  (Further layers need
        a k_cache and a v_cache each; tables, lengths and the stack are shared by all.)"""
        c = self.cfg
        ints = dict(dtype=torch.int32, device=device)
        tiles = (c.n_pages, c.kv_heads, c.page // 32)
        return dict(
            k_cache=torch.empty(*tiles, c.head_dim // 8, 32, 8, dtype=self.dtype, device=device),
            v_cache=torch.empty(*tiles, 4, c.head_dim, 8, dtype=self.dtype, device=device),
            block_table=torch.full((c.max_seqs, c.max_pages), -1, **ints),
            seq_len=torch.zeros(c.max_seqs, **ints),
            free_pages=torch.arange(c.n_pages - 1, -1, -1, **ints),
            n_free=torch.full((1,), c.n_pages, **ints),
            status=torch.zeros(1, **ints),
            workspace=self.alloc_workspace(device))

    def alloc_workspace(self, device="cuda"):
        return torch.empty(self.info.workspace_bytes, dtype=torch.uint8, device=device)

    def alloc_step(self, n_seqs, n_tokens, device="cuda"):
        c = self.cfg
        return dict(cu_new=torch.empty(n_seqs + 1, dtype=torch.int32, device=device),
                    slots=torch.empty(n_tokens, dtype=torch.int32, device=device),
                    o=torch.empty(n_tokens, c.heads, c.head_dim, dtype=self.dtype, device=device))

    # -- the calls -----------------------------------------------------------------------------
    def _stream(self, stream):
        return _raw_stream(self.device) if stream is None else stream.cuda_stream

    def rf2_paged_append(self, seq_len, new_len, free_pages, n_free, block_table, seq_len_out, n_free_out, cu_new, slots, status,
                         stream=None):
        c, dev, i32 = self.cfg, self.device, torch.int32
        n_seqs, n_tokens = new_len.numel(), slots.numel()
        _check(lib().rf2_paged_append(
            self._h, n_seqs, n_tokens, _arg(seq_len, "seq_len", i32, n_seqs, dev), _arg(new_len, "new_len", i32, n_seqs, dev),
            _arg(free_pages, "free_pages", i32, c.n_pages, dev), _arg(n_free, "n_free", i32, 1, dev),
            _arg(block_table, "block_table", i32, n_seqs * c.max_pages, dev),
            _arg(seq_len_out, "seq_len_out", i32, n_seqs, dev), _arg(n_free_out, "n_free_out", i32, 1, dev),
            _arg(cu_new, "cu_new", i32, n_seqs + 1, dev), _arg(slots, "slots", i32, n_tokens, dev),
            _arg(status, "status", i32, 1, dev), self._stream(stream)), "rf2_paged_append")

    def rf2_paged_release(self, done, seq_len, block_table, free_pages, n_free, seq_len_out, n_free_out, status, stream=None):
        c, dev, i32 = self.cfg, self.device, torch.int32
        n_seqs = done.numel()
        _check(lib().rf2_paged_release(
            self._h, n_seqs, _arg(done, "done", torch.bool if done.dtype is torch.bool else torch.uint8, n_seqs, dev),
            _arg(seq_len, "seq_len", i32, n_seqs, dev), _arg(block_table, "block_table", i32, n_seqs * c.max_pages, dev),
            _arg(free_pages, "free_pages", i32, c.n_pages, dev), _arg(n_free, "n_free", i32, 1, dev),
            _arg(seq_len_out, "seq_len_out", i32, n_seqs, dev), _arg(n_free_out, "n_free_out", i32, 1, dev),
            _arg(status, "status", i32, 1, dev), self._stream(stream)), "rf2_paged_release")

    def rf2_paged_store(self, k, v, slots, k_cache, v_cache, stream=None):
        c, dev, size = self.cfg, self.device, self.info.cache_elements
        n_tokens = slots.numel()
        shape = (n_tokens, c.kv_heads, c.head_dim)
        _check(lib().rf2_paged_store(
            self._h, n_tokens, *_rows(k, "k", self.dtype, shape, dev), *_rows(v, "v", self.dtype, shape, dev),
            _arg(slots, "slots", torch.int32, n_tokens, dev), _arg(k_cache, "k_cache", self.dtype, size, dev),
            _arg(v_cache, "v_cache", self.dtype, size, dev), self._stream(stream)), "rf2_paged_store")

    def rf2_paged_attn(self, q, k_cache, v_cache, block_table, seq_len, cu_new, workspace, o, lse=None, stream=None):
        c, dev, size, i32 = self.cfg, self.device, self.info.cache_elements, torch.int32
        n_seqs, n_tokens = seq_len.numel(), q.shape[0]
        _check(lib().rf2_paged_attn(
            self._h, n_seqs, n_tokens, *_rows(q, "q", self.dtype, (n_tokens, c.heads, c.head_dim), dev),
            _arg(k_cache, "k_cache", self.dtype, size, dev), _arg(v_cache, "v_cache", self.dtype, size, dev),
            _arg(block_table, "block_table", i32, n_seqs * c.max_pages, dev), _arg(seq_len, "seq_len", i32, n_seqs, dev),
            _arg(cu_new, "cu_new", i32, n_seqs + 1, dev),
            _arg(workspace, "workspace", torch.uint8, self.info.workspace_bytes, dev),
            _arg(o, "o", self.dtype, n_tokens * c.heads * c.head_dim, dev),
            None if lse is None else _arg(lse, "lse", torch.float32, n_tokens * c.heads, dev), self._stream(stream)),
            "rf2_paged_attn")
