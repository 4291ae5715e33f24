"""ctypes binding of the 8-bit calls of libasd (include/asd8.h): K/V cache and LM head
in e4m3 with power-of-two block scales.  Argument marshalling only, as in asd.py, whose
dims, errors and streams it shares.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch

from . import asd
from .asd import Dims, VerifyArgs, _check, _lib, _ptr, _stream

KV_BLOCK, LM_BLOCK, MIN_EXP, EXP_BIAS = 32, 128, -60, 127
ASD8_W_BF16, ASD8_W_E4M3 = 0, 1
EXPORTS = ["asd8_kv_block", "asd8_kv_scales", "asd8_workspace_bytes", "asd8_kv_quantize",
           "asd8_tree_attention", "asd8_kv_compact", "asd8_lm_head_bytes", "asd8_pack_lm_head",
           "asd8_lmhead_margin", "asd8_verify_step"]

_vp = ctypes.c_void_p


class CacheArgs(ctypes.Structure):
    """asd8_cache: the device pointers of an 8-bit cache."""
    _fields_ = [("k", _vp), ("v", _vp), ("k_exp", _vp), ("v_exp", _vp)]


class VerifyArgs8(ctypes.Structure):
    """asd8_verify_args."""
    _fields_ = [("step", VerifyArgs), ("cache", CacheArgs), ("weight", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


_P, _C = ctypes.POINTER(Dims), ctypes.POINTER(CacheArgs)
_lib.asd8_kv_block.restype = ctypes.c_int32
_lib.asd8_kv_block.argtypes = [_P]
_lib.asd8_kv_scales.restype = ctypes.c_size_t
_lib.asd8_kv_scales.argtypes = [_P]
_lib.asd8_workspace_bytes.restype = ctypes.c_size_t
_lib.asd8_workspace_bytes.argtypes = [_P, ctypes.c_int32]
_lib.asd8_kv_quantize.restype = ctypes.c_int
_lib.asd8_kv_quantize.argtypes = [_P] + [_vp] * 4 + [_C, _vp, ctypes.c_size_t, _vp]
_lib.asd8_tree_attention.restype = ctypes.c_int
_lib.asd8_tree_attention.argtypes = [_P, _vp, _C] + [_vp] * 6 + [ctypes.c_int32, _vp, _vp,
                                                                 ctypes.c_size_t, _vp]
_lib.asd8_kv_compact.restype = ctypes.c_int
_lib.asd8_kv_compact.argtypes = [_P, _vp, _vp, _vp, ctypes.c_int32] + [_vp] * 4 + [
    _C, _vp, _vp, ctypes.c_size_t, _vp]
_lib.asd8_lm_head_bytes.restype = ctypes.c_size_t
_lib.asd8_lm_head_bytes.argtypes = [_P]
_lib.asd8_pack_lm_head.restype = ctypes.c_int
_lib.asd8_pack_lm_head.argtypes = [_P, _vp, _vp, ctypes.c_size_t, _vp]
_lib.asd8_lmhead_margin.restype = ctypes.c_int
_lib.asd8_lmhead_margin.argtypes = [_P] + [_vp] * 5 + [ctypes.c_int32, ctypes.c_float] + [
    _vp] * 6 + [_vp, ctypes.c_size_t, _vp]
_lib.asd8_verify_step.restype = ctypes.c_int
_lib.asd8_verify_step.argtypes = [_P, ctypes.POINTER(VerifyArgs8), _vp, ctypes.c_size_t, _vp]


def kv_block(dims: Dims) -> int:
    """Tokens that share one scale of the cache."""
    n = int(_lib.asd8_kv_block(ctypes.byref(dims)))
    if n == 0:
        raise asd.AsdError(2, "asd8_kv_block")
    return n


class Cache8:
    """An 8-bit K/V cache: e4m3 bytes `k`, `v` in the bf16 cache's layout ([B, Hkv,
    ctx_max, D], or [P, Hkv, page, D] when paged) and their blocks' scale bytes `k_exp`,
    `v_exp` ([..., blocks], exponent + 127).  Tensors that are not given are allocated."""

    def __init__(self, dims: Dims, k=None, v=None, k_exp=None, v_exp=None, device="cuda"):
        n = kv_block(dims)
        rows = dims.page_size or dims.ctx_max
        lead = (dims.num_pages if dims.page_size else dims.batch, dims.num_kv_heads)
        shape, scales = lead + (rows, dims.head_dim), lead + (-(-rows // n),)

        def tensor(t, size, name):
            if t is None:
                return torch.zeros(size, dtype=torch.uint8, device=device)
            if t.element_size() != 1 or tuple(t.shape) != size:
                raise ValueError(f"{name}: expected bytes of shape {size}, got {t.dtype} {tuple(t.shape)}")
            return t
        self.k, self.v = tensor(k, shape, "k"), tensor(v, shape, "v")
        self.k_exp, self.v_exp = tensor(k_exp, scales, "k_exp"), tensor(v_exp, scales, "v_exp")
        self.block = n
        self.args = CacheArgs(_ptr(self.k), _ptr(self.v), _ptr(self.k_exp), _ptr(self.v_exp))
        self._ref = ctypes.byref(self.args)

    def values(self, which: str) -> torch.Tensor:
        """What the cache's bytes stand for: fp32 `k` or `v`."""
        q, e = (self.k, self.k_exp) if which == "k" else (self.v, self.v_exp)
        e = e.view(torch.uint8)   # (whatever one-byte type they came in)
        scale = torch.ldexp(torch.ones_like(e, dtype=torch.float32), e.int() - EXP_BIAS)
        rows = q.shape[2]
        return q.view(torch.float8_e4m3fn).float() * scale.repeat_interleave(self.block, 2)[:, :, :rows, None]


def asd8_workspace_bytes(dims: Dims, total_nodes: int) -> int:
    n = int(_lib.asd8_workspace_bytes(ctypes.byref(dims), int(total_nodes)))
    if n == 0:
        raise asd.AsdError(2, "asd8_workspace_bytes")
    return n


def alloc_workspace(dims: Dims, total_nodes: int, device="cuda") -> torch.Tensor:
    return torch.empty(asd8_workspace_bytes(dims, total_nodes), dtype=torch.uint8, device=device)


def asd8_kv_quantize(dims, k_cache, v_cache, page_table, ctx_len, cache: Cache8, workspace, stream=None):
    _check(_lib.asd8_kv_quantize(
        ctypes.byref(dims), _ptr(k_cache), _ptr(v_cache), _ptr(page_table), _ptr(ctx_len), cache._ref,
        _ptr(workspace), workspace.numel(), _stream(stream)), "asd8_kv_quantize")


def asd8_tree_attention(dims, q, cache: Cache8, page_table, ctx_len, tree_k, tree_v, parent, cu_nodes,
                        out, workspace, stream=None):
    _check(_lib.asd8_tree_attention(
        ctypes.byref(dims), _ptr(q), cache._ref, _ptr(page_table), _ptr(ctx_len), _ptr(tree_k),
        _ptr(tree_v), _ptr(parent), _ptr(cu_nodes), parent.numel(), _ptr(out), _ptr(workspace),
        workspace.numel(), _stream(stream)), "asd8_tree_attention")


def asd8_kv_compact(dims, tree_k, tree_v, cu_nodes, total_nodes, path, path_len, ctx_len, page_table,
                    cache: Cache8, ctx_len_out, workspace, stream=None):
    _check(_lib.asd8_kv_compact(
        ctypes.byref(dims), _ptr(tree_k), _ptr(tree_v), _ptr(cu_nodes), int(total_nodes), _ptr(path),
        _ptr(path_len), _ptr(ctx_len), _ptr(page_table), cache._ref, _ptr(ctx_len_out),
        _ptr(workspace), workspace.numel(), _stream(stream)), "asd8_kv_compact")


def asd8_lm_head_bytes(dims: Dims) -> int:
    n = int(_lib.asd8_lm_head_bytes(ctypes.byref(dims)))
    if n == 0:
        raise asd.AsdError(2, "asd8_lm_head_bytes")
    return n


def asd8_pack_lm_head(dims: Dims, w: torch.Tensor, w_packed: torch.Tensor, stream=None):
    _check(_lib.asd8_pack_lm_head(ctypes.byref(dims), _ptr(w), _ptr(w_packed), w_packed.numel(),
                                  _stream(stream)), "asd8_pack_lm_head")


def pack_lm_head(dims: Dims, w: torch.Tensor, stream=None) -> torch.Tensor:
    """A new device buffer holding w (bf16 [vocab, hidden]) in 8 bits, in the LM head's
    streaming order."""
    out = torch.empty(asd8_lm_head_bytes(dims), dtype=torch.uint8, device=w.device)
    asd8_pack_lm_head(dims, w, out, stream)
    return out


def asd8_lmhead_margin(dims, hidden, w_packed, tokens, parent, cu_nodes, tau, row_max, row_argmax,
                       row_lse, l_draft, ratio, accept, workspace, stream=None):
    _check(_lib.asd8_lmhead_margin(
        ctypes.byref(dims), _ptr(hidden), _ptr(w_packed), _ptr(tokens), _ptr(parent), _ptr(cu_nodes),
        parent.numel(), float(tau), _ptr(row_max), _ptr(row_argmax), _ptr(row_lse), _ptr(l_draft),
        _ptr(ratio), _ptr(accept), _ptr(workspace), workspace.numel(), _stream(stream)),
        "asd8_lmhead_margin")


def asd8_verify_step(dims, args: VerifyArgs8, workspace, stream=None):
    _check(_lib.asd8_verify_step(ctypes.byref(dims), ctypes.byref(args), _ptr(workspace),
                                 workspace.numel(), _stream(stream)), "asd8_verify_step")


class VerifyStep8(asd.VerifyStep):
    """asd.VerifyStep on an 8-bit cache: `bind` takes cache=Cache8 in the place of k_cache
    and v_cache, and weight=ASD8_W_E4M3 where w_lm comes from pack_lm_head here."""

    def __init__(self, dims: Dims, total_nodes: int, device="cuda", attn_dtype=torch.bfloat16):
        super().__init__(dims, total_nodes, device, attn_dtype)
        self.workspace = alloc_workspace(dims, total_nodes, device)
        self.args8 = VerifyArgs8()

    def bind(self, *, cache: Cache8, weight: int = ASD8_W_E4M3, q, tree_k, tree_v, hidden, w_lm, tokens,
             parent, cu_nodes, ctx_len, tau, page_table=None, events: Optional[Sequence] = None):
        super().bind(q=q, tree_k=tree_k, tree_v=tree_v, hidden=hidden, w_lm=w_lm, tokens=tokens,
                     parent=parent, cu_nodes=cu_nodes, ctx_len=ctx_len, k_cache=None, v_cache=None,
                     tau=tau, page_table=page_table, events=events)
        self._keep.append(cache)
        self.args8.step, self.args8.cache, self.args8.weight = self.args, cache.args, int(weight)
        return self

    def run(self, stream=None):
        asd8_verify_step(self.dims, self.args8, self.workspace, stream)
        return self.out
