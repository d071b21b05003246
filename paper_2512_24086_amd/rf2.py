"""Thin ctypes binding of librf2.so: same names as the C ABI, argument marshalling only.

PyTorch supplies device memory and streams; every step of the layer runs in the HIP
kernels of the library.  There is no fallback: if librf2.so is missing, loading raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "librf2.so")

RF2_OK = 0
RF2_ERR_INVALID_ARG, RF2_ERR_UNSUPPORTED, RF2_ERR_ALLOC, RF2_ERR_HIP, RF2_ERR_TOO_LARGE = -1, -2, -3, -4, -5
RF2_BUDGET_GLOBAL, RF2_BUDGET_ROW_INCL_SINK, RF2_BUDGET_ROW_PLUS_SINK = 0, 1, 2
RF2_LAYOUT_BHND, RF2_LAYOUT_BNHD = 0, 1
RF2_SELECT_TOPN, RF2_SELECT_CDF = 0, 1
RF2_DTYPE_BF16, RF2_DTYPE_F16, RF2_DTYPE_F32 = 0, 1, 2
RF2_NORM_NONE, RF2_NORM_RMS = 0, 1
RF2_ROPE_PAIRS, RF2_ROPE_HALVES = 0, 1
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


class rf2_rope_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("heads", "kv_heads", "head_dim", "dtype", "weight_dtype", "norm")] + \
               [("eps", C.c_float), ("pairing", C.c_int32), ("axes", C.c_int32), ("axis_dim", C.c_int32 * 4), ("theta", C.c_double)]


class rf2_rope_info(C.Structure):
    _fields_ = [("workspace_bytes", C.c_int64)]


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
    "rf2_rope_plan_create": (C.c_int, [C.POINTER(rf2_rope_config), C.c_void_p, C.POINTER(C.c_void_p)]),
    "rf2_rope_plan_destroy": (C.c_int, [C.c_void_p]),
    "rf2_rope_plan_info": (C.c_int, [C.c_void_p, C.POINTER(rf2_rope_info)]),
    "rf2_rope_apply": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_int64] + [C.c_void_p] * 3),
    "rf2_rope_backward": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_int64] + [C.c_void_p] * 6),
    "rf2_permute_rope": (C.c_int, [C.c_void_p] * 6 + [C.c_int64] + [C.c_void_p] * 10),
    "rf2_paged_store_rope": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32] + [C.c_void_p, C.c_int64] * 3 + [C.c_void_p] * 8 + [C.c_int64, C.c_void_p]),
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
        self._shape = (batch, self.info.N, heads, head_dim) if qkv_layout == RF2_LAYOUT_BNHD else (batch, heads, self.info.N, head_dim)

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

    def rf2_permute_rope(self, rope, q, k, v, pos, qp, kp, vp, qbar=None, kbar=None, wq=None, wk=None, wq_text=None, wk_text=None, stream=None):
        """rf2_permute of q and k normalised and rotated by a RopePlan; pos is [N, axes] or [batch, N, axes], text tokens behind the grid's.  q, k and v
        are laid out as this plan's qkv_layout says, whatever the RopePlan's own layout is."""
        c, i, dev, bf, f32 = self.cfg, self.info, rope.device, torch.bfloat16, torch.float32
        at, step = rope._pos(pos, c.batch, i.N)
        row = c.batch * c.heads * c.head_dim
        if not q.shape == k.shape == v.shape == self._shape:
            for x, what in ((q, "q"), (k, "k"), (v, "v")):
                _not_the_other_layout(x, what, self._shape)
        _check(lib().rf2_permute_rope(
            self._h, rope._h, _arg(q, "q", bf, row * i.N, dev), _arg(k, "k", bf, row * i.N, dev), _arg(v, "v", bf, row * i.N, dev), at, step,
            rope._weight(wq, "wq"), rope._weight(wk, "wk"), None if wq_text is None else rope._weight(wq_text, "wq_text"),
            None if wk_text is None else rope._weight(wk_text, "wk_text"), _arg(qp, "qp", bf, row * i.N_pad, dev),
            _arg(kp, "kp", bf, row * i.N_pad_k, dev), _arg(vp, "vp", bf, row * i.N_pad_k, dev),
            None if qbar is None else _arg(qbar, "qbar", f32, row * i.n_blocks, dev),
            None if kbar is None else _arg(kbar, "kbar", f32, row * i.n_blocks_k, dev), _stream(stream)), "rf2_permute_rope")

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

    def layer_fused(self, q, k, v, buf, stream=None, rope=None, pos=None, weights=()):
        """The whole layer with the inverse permutation fused into the attention epilogue; returns buf['o'].  With a RopePlan, and pos and
        weights (wq, wk, wq_text, wk_text: as many as there are) as rf2_permute_rope takes them, q and k are raw projections."""
        if rope is None and (pos is not None or any(w is not None for w in weights or ())):
            raise ValueError("pos, weights: expected with rope, the RopePlan that they are for")
        stream = torch.cuda.current_stream() if stream is None else stream
        if rope is None:
            self.rf2_permute(q, k, v, buf["qp"], buf["kp"], buf["vp"], buf["qbar"], buf["kbar"], stream)
        else:
            self.rf2_permute_rope(rope, q, k, v, pos, buf["qp"], buf["kp"], buf["vp"], buf["qbar"], buf["kbar"], *weights, stream=stream)
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


def _not_the_other_layout(t, what, shape):
    """Refuses a tensor whose tokens and heads stand in each other's place of `shape`, [batch, tokens, heads, head_dim] or [batch, heads, tokens, head_dim]."""
    last = tuple(t.shape[-3:])
    if last != shape[1:] and last == (shape[2], shape[1], shape[3]):
        raise ValueError(f"{what}: expected {shape}, got {tuple(t.shape)}: tokens and heads the other way round")


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

    def rf2_paged_store_rope(self, rope, q, k, v, pos, slots, k_cache, v_cache, q_out, wq=None, wk=None, cu_new=None, stream=None):
        """rf2_paged_store of k normalised and rotated by a RopePlan, and q the same into q_out (which may be q); with cu_new, rows of q_out
        behind the last new token stay as they are."""
        c, dev, size = self.cfg, self.device, self.info.cache_elements
        n_tokens = slots.numel()
        shape, q_shape = (n_tokens, c.kv_heads, c.head_dim), (n_tokens, c.heads, c.head_dim)
        if cu_new is not None and cu_new.numel() < 1:
            raise ValueError("cu_new: expected one element at least")
        _check(lib().rf2_paged_store_rope(
            self._h, rope._h, n_tokens, *_rows(q, "q", self.dtype, q_shape, dev), *_rows(k, "k", self.dtype, shape, dev),
            *_rows(v, "v", self.dtype, shape, dev), rope._pos(pos, 1, n_tokens)[0], rope._weight(wq, "wq"), rope._weight(wk, "wk"),
            _arg(slots, "slots", torch.int32, n_tokens, dev),
            None if cu_new is None else _arg(cu_new, "cu_new", torch.int32, cu_new.numel(), dev) + 4 * (cu_new.numel() - 1),
            _arg(k_cache, "k_cache", self.dtype, size, dev), _arg(v_cache, "v_cache", self.dtype, size, dev),
            *_rows(q_out, "q_out", self.dtype, q_shape, dev), self._stream(stream)), "rf2_paged_store_rope")

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


# an rf2_rows of C: the address of the first row, and how far elements of the batch, tokens and heads are apart
_two_rows_twice, _two_rows_thrice = struct.Struct("=" + "Qqqq" * 4), struct.Struct("=" + "Qqqq" * 6)
_NO_ROWS = (0, 0, 0, 0)


class RopePlan:
    """Owner of an rf2_rope_plan*: norms of the rows of Q's and K's heads and their rotation by positions of several axes.

    `layout` says how the tensors handed over are indexed: [batch, tokens, heads, head_dim] (RF2_LAYOUT_BNHD) or
    [batch, heads, tokens, head_dim] (RF2_LAYOUT_BHND), with or without the batch; their rows may lie anywhere (parts of a joint
    projection, views), channels side by side.  pos is [tokens, axes] or [batch, tokens, axes], int32.  A plan's rotation may also ride on
    `Plan.rf2_permute_rope` and `PagedPlan.rf2_paged_store_rope`, which go by the layout of the plan that they belong to.
    """

    def __init__(self, *, heads, kv_heads, head_dim, axis_dims, theta=10000.0, inv_freq=None, pairing=RF2_ROPE_PAIRS, norm=RF2_NORM_RMS,
                 eps=1e-6, dtype=torch.bfloat16, weight_dtype=None, layout=RF2_LAYOUT_BNHD):
        codes = {torch.bfloat16: RF2_DTYPE_BF16, torch.float16: RF2_DTYPE_F16, torch.float32: RF2_DTYPE_F32}
        weight_dtype = dtype if weight_dtype is None or norm == RF2_NORM_NONE else weight_dtype
        if dtype not in (torch.bfloat16, torch.float16):
            raise ValueError(f"dtype: expected torch.bfloat16 or torch.float16, got {dtype}")
        if weight_dtype not in codes:
            raise ValueError(f"weight_dtype: expected {dtype} or torch.float32, got {weight_dtype}")
        if layout not in (RF2_LAYOUT_BHND, RF2_LAYOUT_BNHD):
            raise ValueError(f"layout: expected RF2_LAYOUT_BHND or RF2_LAYOUT_BNHD, got {layout}")
        axis_dims = [int(x) for x in axis_dims]
        if len(axis_dims) > 4:
            raise ValueError(f"axis_dims: expected at most 4, got {len(axis_dims)}")
        table = None
        if inv_freq is not None:
            inv_freq = [float(x) for x in inv_freq]
            if len(inv_freq) != sum(axis_dims) // 2:
                raise ValueError(f"inv_freq: expected {sum(axis_dims) // 2} frequencies, one for each pair, got {len(inv_freq)}")
            table = (C.c_double * max(1, len(inv_freq)))(*inv_freq)
        self.dtype, self.weight_dtype, self.layout = dtype, weight_dtype, layout
        self.cfg = rf2_rope_config(heads, kv_heads, head_dim, codes[dtype], codes[weight_dtype], norm, float(eps), pairing, len(axis_dims),
                                   (C.c_int32 * 4)(*axis_dims), float(theta))
        self._h = C.c_void_p(0)
        _check(lib().rf2_rope_plan_create(C.byref(self.cfg), table, C.byref(self._h)), "rf2_rope_plan_create")
        self.info = rf2_rope_info()
        _check(lib().rf2_rope_plan_info(self._h, C.byref(self.info)), "rf2_rope_plan_info")
        self.device = torch.cuda.current_device() if torch.cuda.is_available() else -1

    def close(self):
        if self._h:
            lib().rf2_rope_plan_destroy(self._h)
            self._h = C.c_void_p(0)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def alloc_workspace(self, device="cuda"):
        return torch.empty(self.info.workspace_bytes, dtype=torch.uint8, device=device)

    # -- arguments -----------------------------------------------------------------------------
    def _sizes(self, t):
        """Batch and tokens of a tensor of rows, and the shapes that all of Q's and all of K's have then."""
        c, shape = self.cfg, t.shape
        if self.layout == RF2_LAYOUT_BNHD:
            if len(shape) == 4:
                batch, tokens = shape[0], shape[1]
                return batch, tokens, (batch, tokens, c.heads, c.head_dim), (batch, tokens, c.kv_heads, c.head_dim)
            if len(shape) == 3:
                return 1, shape[0], (shape[0], c.heads, c.head_dim), (shape[0], c.kv_heads, c.head_dim)
        elif len(shape) == 4:
            batch, tokens = shape[0], shape[2]
            return batch, tokens, (batch, c.heads, tokens, c.head_dim), (batch, c.kv_heads, tokens, c.head_dim)
        elif len(shape) == 3:
            return 1, shape[1], (c.heads, shape[1], c.head_dim), (c.kv_heads, shape[1], c.head_dim)
        raise ValueError(f"expected rows of three or four axes, got {tuple(shape)}")

    def _rows(self, t, what, shape):
        """(address, strides of the batch, a token, a head) of a tensor of rows."""
        if t is None:
            raise ValueError(f"{what}: expected with the others of its side")
        stride = t.stride()
        if t.shape != shape or t.dtype is not self.dtype or t.get_device() != self.device or stride[-1] != 1:
            raise ValueError(f"{what}: expected {shape} of {self.dtype} on device {self.device}, channels side by side, got {tuple(t.shape)} of "
                             f"{t.dtype} on {t.device}, strides {stride}")
        if len(stride) == 4:
            return (t.data_ptr(), *stride[:3]) if self.layout == RF2_LAYOUT_BNHD else (t.data_ptr(), stride[0], stride[2], stride[1])
        return (t.data_ptr(), 0, stride[0], stride[1]) if self.layout == RF2_LAYOUT_BNHD else (t.data_ptr(), 0, stride[1], stride[0])

    def _pos(self, pos, batch, tokens):
        axes = self.cfg.axes
        if axes == 0:
            return None, 0
        shape = None if pos is None else pos.shape
        if shape == (tokens, axes):
            step = 0
        elif shape == (batch, tokens, axes):
            step = tokens * axes
        else:
            step = -1
        if step < 0 or pos.dtype is not torch.int32 or pos.get_device() != self.device or not pos.is_contiguous():
            raise ValueError(f"pos: expected contiguous {(tokens, axes)} or {(batch, tokens, axes)} of torch.int32 on device {self.device}, got "
                             + ("none" if pos is None else f"{tuple(pos.shape)} of {pos.dtype} on {pos.device}, strides {pos.stride()}"))
        return pos.data_ptr(), step

    def _weight(self, w, what, there=True):
        if (w is None) == (there and self.cfg.norm == RF2_NORM_RMS):
            raise ValueError(f"{what}: expected " + ("weights of the norm" if w is None else "none: there is no norm, or no rows that have it"))
        return None if w is None else _arg(w, what, self.weight_dtype, self.cfg.head_dim, self.device)

    def _stream(self, stream):
        return _raw_stream(self.device) if stream is None else stream.cuda_stream

    # -- the calls -----------------------------------------------------------------------------
    def rf2_rope_apply(self, q, k, pos, q_out, k_out, wq=None, wk=None, stream=None):
        """q_out and k_out from q and k (either of them may be None, with its output).  q_out may be q, k_out k."""
        if q is None and k is None:
            raise ValueError("q and k: expected one at least")
        batch, tokens, q_shape, k_shape = self._sizes(k if q is None else q)
        rows = self._rows
        at, step = self._pos(pos, batch, tokens)
        q, q_out = (_NO_ROWS, _NO_ROWS) if q is None and q_out is None else (rows(q, "q", q_shape), rows(q_out, "q_out", q_shape))
        k, k_out = (_NO_ROWS, _NO_ROWS) if k is None and k_out is None else (rows(k, "k", k_shape), rows(k_out, "k_out", k_shape))
        _check(lib().rf2_rope_apply(self._h, batch, tokens, _two_rows_twice.pack(*q, *k, *q_out, *k_out), at, step,
                                    self._weight(wq, "wq", q is not _NO_ROWS), self._weight(wk, "wk", k is not _NO_ROWS), self._stream(stream)),
               "rf2_rope_apply")

    def rf2_rope_backward(self, q, k, pos, dq_out, dk_out, dq, dk, wq=None, wk=None, dwq=None, dwk=None, workspace=None, stream=None):
        """dq, dk, dwq, dwk from q, k and the gradients of q_out and k_out.  Without a norm q and k are not read and may be None."""
        norm = self.cfg.norm == RF2_NORM_RMS
        if not norm:
            q, k = dq_out, dk_out
        if q is None and k is None:
            raise ValueError("q and k: expected one at least")
        batch, tokens, q_shape, k_shape = self._sizes(k if q is None else q)
        at, step = self._pos(pos, batch, tokens)
        with_q, with_k = not (q is None and dq_out is None and dq is None), not (k is None and dk_out is None and dk is None)
        if (dwq is None) == (norm and with_q) or (dwk is None) == (norm and with_k):
            raise ValueError("dwq, dwk: expected the gradients of the weights where there is a norm and rows that have it, and none elsewhere")
        rows, f32, d, dev = self._rows, torch.float32, self.cfg.head_dim, self.device
        qs = (rows(q, "q", q_shape), rows(dq_out, "dq_out", q_shape), rows(dq, "dq", q_shape)) if with_q else (_NO_ROWS,) * 3
        ks = (rows(k, "k", k_shape), rows(dk_out, "dk_out", k_shape), rows(dk, "dk", k_shape)) if with_k else (_NO_ROWS,) * 3
        _check(lib().rf2_rope_backward(
            self._h, batch, tokens, _two_rows_thrice.pack(*qs[0], *ks[0], *qs[1], *ks[1], *qs[2], *ks[2]), at, step, self._weight(wq, "wq", with_q),
            self._weight(wk, "wk", with_k), None if dwq is None else _arg(dwq, "dwq", f32, d, dev), None if dwk is None else _arg(dwk, "dwk", f32, d, dev),
            _arg(workspace, "workspace", torch.uint8, self.info.workspace_bytes, dev) if norm and workspace is not None else None,
            self._stream(stream)), "rf2_rope_backward")
