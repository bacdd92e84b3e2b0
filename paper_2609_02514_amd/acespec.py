"""ctypes binding of libacespec.so: the C entry points under the same names, plus a thin
marshalling helper (``Verifier``) that passes torch device tensors' pointers and the current
torch stream.  Every step of the verify path runs in the library's HIP kernels; this module
only moves pointers and sizes across the boundary.  Importing it fails loudly if the
library has not been built.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, List, Optional

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libacespec.so")

ACESPEC_OK, ACESPEC_EINVAL, ACESPEC_EUNSUPPORTED = 0, -1, -2
ACESPEC_ENOMEM, ACESPEC_EHIP, ACESPEC_EBADTREE = -3, -4, -5
ACESPEC_EBADDRAFT, ACESPEC_ENONFINITE = -6, -7
ACESPEC_F32, ACESPEC_BF16 = 0, 1

EXPORTED = ["acespec_create", "acespec_destroy", "acespec_verify_tree",
            "acespec_verify_tree_scalar_q", "acespec_verify_tail", "acespec_commit_kv",
            "acespec_last_error", "acespec_timing_enable", "acespec_timing_read",
            "acespec_timing_only", "acespec_verify_tail_noalloc", "acespec_pack_weight",
            "acespec_convert_v_cache", "acespec_quantize_kv", "acespec_dequantize_kv",
            "acespec_attention_quant", "acespec_verify_tree_quant", "acespec_commit_kv_quant",
            "acespec_share_prefix", "acespec_attention_shared", "acespec_qk_norm_rope",
            "acespec_verify_tree_shared", "acespec_fork_kv"]


class ModelDesc(C.Structure):
    _fields_ = [("n_layers", C.c_int), ("d_model", C.c_int), ("n_heads", C.c_int),
                ("n_kv_heads", C.c_int), ("head_dim", C.c_int), ("d_ff", C.c_int),
                ("vocab", C.c_int), ("rope_base", C.c_float), ("rms_eps", C.c_float),
                ("dtype", C.c_int)]


class LayerWeights(C.Structure):
    _fields_ = [("attn_norm", C.c_void_p), ("wqkv", C.c_void_p), ("wo", C.c_void_p),
                ("mlp_norm", C.c_void_p), ("w_gate_up", C.c_void_p), ("w_down", C.c_void_p)]


ACESPEC_LAYOUT_ROWS, ACESPEC_LAYOUT_PACKED = 0, 1
ACESPEC_V_TO_HEAD_DIM_MAJOR, ACESPEC_V_TO_SLOT_MAJOR = 0, 1


class Weights(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("layers", C.POINTER(LayerWeights)),
                ("final_norm", C.c_void_p), ("lm_head", C.c_void_p), ("layout", C.c_int)]


class KVCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("capacity", C.c_int),
                ("prefix_len", C.c_void_p)]


class KVQuant(C.Structure):
    _fields_ = [("blocks", C.c_void_p), ("tail_k", C.c_void_p), ("tail_v", C.c_void_p),
                ("capacity", C.c_int), ("tail_capacity", C.c_int), ("prefix_len", C.c_void_p)]


class AttnSpan(C.Structure):
    _fields_ = [("window", C.c_int), ("sinks", C.c_int)]


class KVShared(C.Structure):
    _fields_ = [("blocks", C.c_void_p), ("prefixes", C.c_int), ("capacity", C.c_int),
                ("len", C.c_void_p)]


class QKNorm(C.Structure):
    _fields_ = [("q_gain", C.c_void_p), ("k_gain", C.c_void_p)]


class Params(C.Structure):
    _fields_ = [("temperature", C.c_float), ("top_p", C.c_float), ("top_k", C.c_int)]


class Outputs(C.Structure):
    _fields_ = [("accept", C.c_void_p), ("acc_prefix_len", C.c_void_p),
                ("resample_token", C.c_void_p), ("bonus_token", C.c_void_p),
                ("topk_ids", C.c_void_p), ("topk_probs", C.c_void_p), ("path", C.c_void_p),
                ("path_len", C.c_void_p), ("next_token", C.c_void_p),
                ("sibling_hit", C.c_void_p), ("status", C.c_void_p),
                ("logits_out", C.c_void_p)]


_lib = None


def load(path: str = LIB_PATH) -> C.CDLL:
    """Loads the HIP library (raises if it is missing: there is no fallback path)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is not built; run `python -m paper_2609_02514_amd.build`")
    lib = C.CDLL(path)
    lib.acespec_create.argtypes = [C.POINTER(ModelDesc), C.c_int, C.c_int,
                                   C.POINTER(C.c_void_p)]
    lib.acespec_create.restype = C.c_int
    lib.acespec_destroy.argtypes = [C.c_void_p]
    lib.acespec_destroy.restype = None
    lib.acespec_verify_tree.argtypes = [C.c_void_p, C.POINTER(Weights), C.POINTER(KVCache),
                                        C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                        C.c_int, C.c_int, C.POINTER(Params),
                                        C.POINTER(Outputs), C.c_void_p]
    lib.acespec_verify_tree.restype = C.c_int
    lib.acespec_verify_tree_scalar_q.argtypes = lib.acespec_verify_tree.argtypes
    lib.acespec_verify_tree_scalar_q.restype = C.c_int
    lib.acespec_verify_tail.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_void_p,
                                        C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                        C.c_int, C.c_int, C.POINTER(Params),
                                        C.POINTER(Outputs), C.c_void_p]
    lib.acespec_verify_tail.restype = C.c_int
    lib.acespec_verify_tail_noalloc.argtypes = [C.POINTER(ModelDesc), C.c_void_p, C.c_int,
                                                C.c_void_p, C.c_void_p, C.c_void_p,
                                                C.c_void_p, C.c_void_p, C.c_int, C.c_int,
                                                C.POINTER(Params), C.POINTER(Outputs),
                                                C.c_void_p]
    lib.acespec_verify_tail_noalloc.restype = C.c_int
    lib.acespec_commit_kv.argtypes = [C.c_void_p, C.POINTER(KVCache), C.c_void_p, C.c_void_p,
                                      C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_void_p]
    lib.acespec_commit_kv.restype = C.c_int
    lib.acespec_pack_weight.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_void_p]
    lib.acespec_pack_weight.restype = C.c_int
    lib.acespec_convert_v_cache.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int,
                                            C.c_int, C.c_int, C.c_void_p]
    lib.acespec_convert_v_cache.restype = C.c_int
    lib.acespec_quantize_kv.argtypes = [C.c_void_p, C.POINTER(KVCache), C.POINTER(KVQuant),
                                        C.c_void_p, C.c_int, C.c_void_p, C.c_void_p]
    lib.acespec_quantize_kv.restype = C.c_int
    lib.acespec_dequantize_kv.argtypes = [C.c_void_p, C.POINTER(KVQuant), C.POINTER(KVCache),
                                          C.c_void_p, C.c_int, C.c_void_p, C.c_void_p]
    lib.acespec_dequantize_kv.restype = C.c_int
    lib.acespec_attention_quant.argtypes = [C.c_void_p, C.POINTER(KVQuant), C.c_int,
                                            C.POINTER(AttnSpan), C.c_void_p, C.c_void_p, C.c_int,
                                            C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.acespec_attention_quant.restype = C.c_int
    lib.acespec_verify_tree_quant.argtypes = [C.c_void_p, C.POINTER(Weights), C.POINTER(KVQuant),
                                              C.POINTER(AttnSpan), C.c_void_p, C.c_void_p,
                                              C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int,
                                              C.POINTER(Params), C.POINTER(Outputs), C.c_void_p]
    lib.acespec_verify_tree_quant.restype = C.c_int
    lib.acespec_commit_kv_quant.argtypes = [C.c_void_p, C.POINTER(KVQuant), C.c_void_p, C.c_void_p,
                                            C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_void_p]
    lib.acespec_commit_kv_quant.restype = C.c_int
    lib.acespec_share_prefix.argtypes = [C.c_void_p, C.POINTER(KVCache), C.c_int,
                                         C.POINTER(KVShared), C.c_void_p, C.c_void_p, C.c_void_p,
                                         C.c_void_p]
    lib.acespec_share_prefix.restype = C.c_int
    lib.acespec_attention_shared.argtypes = [C.c_void_p, C.POINTER(KVShared), C.c_void_p,
                                             C.POINTER(KVCache), C.c_int, C.c_void_p, C.c_void_p,
                                             C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.acespec_attention_shared.restype = C.c_int
    lib.acespec_qk_norm_rope.argtypes = [C.c_void_p, C.POINTER(QKNorm), C.POINTER(KVShared),
                                         C.c_void_p, C.POINTER(KVCache), C.c_int, C.c_void_p,
                                         C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_void_p,
                                         C.c_void_p]
    lib.acespec_qk_norm_rope.restype = C.c_int
    lib.acespec_verify_tree_shared.argtypes = [C.c_void_p, C.POINTER(Weights), C.POINTER(QKNorm),
                                               C.POINTER(KVShared), C.c_void_p, C.POINTER(KVCache),
                                               C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                               C.c_void_p, C.c_int, C.c_int, C.POINTER(Params),
                                               C.POINTER(Outputs), C.c_void_p]
    lib.acespec_verify_tree_shared.restype = C.c_int
    lib.acespec_fork_kv.argtypes = [C.c_void_p, C.POINTER(KVCache), C.c_int, C.POINTER(KVCache),
                                    C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.acespec_fork_kv.restype = C.c_int
    lib.acespec_last_error.argtypes = []
    lib.acespec_last_error.restype = C.c_char_p
    lib.acespec_timing_enable.argtypes = [C.c_void_p, C.c_int]
    lib.acespec_timing_enable.restype = C.c_int
    lib.acespec_timing_read.argtypes = [C.c_void_p, C.POINTER(C.c_char_p),
                                        C.POINTER(C.c_double), C.POINTER(C.c_int), C.c_int]
    lib.acespec_timing_read.restype = C.c_int
    lib.acespec_timing_only.argtypes = [C.c_void_p, C.c_char_p]
    lib.acespec_timing_only.restype = C.c_int
    _lib = lib
    return lib


# --------------------------------------------------------------------------------------
# The C entry points, same names
# --------------------------------------------------------------------------------------


def acespec_last_error() -> str:
    return load().acespec_last_error().decode()


class AcespecError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"acespec error {code}: {msg}")
        self.code = code


def _check(rc: int) -> int:
    if rc < 0:
        raise AcespecError(rc, acespec_last_error())
    return rc


def acespec_create(desc: ModelDesc, max_batch: int, max_nodes: int) -> C.c_void_p:
    ctx = C.c_void_p()
    _check(load().acespec_create(C.byref(desc), max_batch, max_nodes, C.byref(ctx)))
    return ctx


def acespec_destroy(ctx) -> None:
    load().acespec_destroy(ctx)


def acespec_verify_tree(ctx, weights: Weights, kv: KVCache, tree_tokens: int, parent_idx: int,
                        draft_q: int, uniforms: int, B: int, N: int, params: Params,
                        outputs: Outputs, stream: int) -> int:
    return _check(load().acespec_verify_tree(ctx, C.byref(weights), C.byref(kv), tree_tokens,
                                             parent_idx, draft_q, uniforms, B, N,
                                             C.byref(params), C.byref(outputs), stream))


def acespec_verify_tree_scalar_q(ctx, weights: Weights, kv: KVCache, tree_tokens: int,
                                 parent_idx: int, q_hat: int, uniforms: int, B: int, N: int,
                                 params: Params, outputs: Outputs, stream: int) -> int:
    return _check(load().acespec_verify_tree_scalar_q(ctx, C.byref(weights), C.byref(kv),
                                                      tree_tokens, parent_idx, q_hat, uniforms,
                                                      B, N, C.byref(params), C.byref(outputs),
                                                      stream))


def acespec_verify_tail(ctx, lm_head: int, lm_head_layout: int, final_norm: Optional[int],
                        hidden: int, draft_tokens: int, draft_q: int, uniforms: int, R: int,
                        chain_len: int, params: Params, outputs: Outputs, stream: int) -> int:
    return _check(load().acespec_verify_tail(ctx, lm_head, lm_head_layout, final_norm, hidden,
                                             draft_tokens, draft_q, uniforms, R, chain_len,
                                             C.byref(params), C.byref(outputs), stream))


def acespec_verify_tail_noalloc(desc: ModelDesc, lm_head: int, lm_head_layout: int,
                                final_norm: Optional[int], hidden: int, draft_tokens: int,
                                draft_q: int, uniforms: int, R: int, chain_len: int,
                                params: Params, outputs: Outputs, stream: int) -> int:
    return _check(load().acespec_verify_tail_noalloc(C.byref(desc), lm_head, lm_head_layout,
                                                     final_norm, hidden, draft_tokens, draft_q,
                                                     uniforms, R, chain_len, C.byref(params),
                                                     C.byref(outputs), stream))


def acespec_commit_kv(ctx, kv: KVCache, path: int, path_len: int, status: Optional[int], B: int,
                      N: int, new_prefix_len: int, stream: int) -> int:
    return _check(load().acespec_commit_kv(ctx, C.byref(kv), path, path_len, status, B, N,
                                           new_prefix_len, stream))


def acespec_pack_weight(src: int, dst: int, rows: int, cols: int, stream: int) -> int:
    return _check(load().acespec_pack_weight(src, dst, rows, cols, stream))


def acespec_convert_v_cache(src: int, dst: int, planes: int, capacity: int, head_dim: int,
                            dtype: int, direction: int, stream: int) -> int:
    return _check(load().acespec_convert_v_cache(src, dst, planes, capacity, head_dim, dtype,
                                                 direction, stream))


def acespec_quantize_kv(ctx, kv: KVCache, qc: KVQuant, first: Optional[int], B: int,
                        status: Optional[int], stream: int) -> int:
    return _check(load().acespec_quantize_kv(ctx, C.byref(kv), C.byref(qc), first, B, status,
                                             stream))


def acespec_dequantize_kv(ctx, qc: KVQuant, kv: KVCache, first: Optional[int], B: int,
                          status: Optional[int], stream: int) -> int:
    return _check(load().acespec_dequantize_kv(ctx, C.byref(qc), C.byref(kv), first, B, status,
                                               stream))


def acespec_attention_quant(ctx, qc: KVQuant, layer: int, span: AttnSpan, q: int,
                            parent_idx: int, B: int, N: int, out: int, status: int,
                            stream: int) -> int:
    return _check(load().acespec_attention_quant(ctx, C.byref(qc), layer, C.byref(span), q,
                                                 parent_idx, B, N, out, status, stream))


def acespec_verify_tree_quant(ctx, weights: Weights, qc: KVQuant, span: AttnSpan,
                              tree_tokens: int, parent_idx: int, draft_q: Optional[int],
                              q_hat: Optional[int], uniforms: int, B: int, N: int, params: Params,
                              outputs: Outputs, stream: int) -> int:
    return _check(load().acespec_verify_tree_quant(ctx, C.byref(weights), C.byref(qc),
                                                   C.byref(span), tree_tokens, parent_idx,
                                                   draft_q, q_hat, uniforms, B, N,
                                                   C.byref(params), C.byref(outputs), stream))


def acespec_commit_kv_quant(ctx, qc: KVQuant, path: int, path_len: int, status: Optional[int],
                            B: int, N: int, new_prefix_len: int, stream: int) -> int:
    return _check(load().acespec_commit_kv_quant(ctx, C.byref(qc), path, path_len, status, B, N,
                                                 new_prefix_len, stream))


def acespec_share_prefix(ctx, kv: KVCache, B: int, shared: KVShared, from_: int,
                         count: Optional[int], new_len: int, stream: int) -> int:
    return _check(load().acespec_share_prefix(ctx, C.byref(kv), B, C.byref(shared), from_, count,
                                              new_len, stream))


def acespec_attention_shared(ctx, shared: KVShared, prefix_of: int, kv: KVCache, layer: int, q: int,
                             parent_idx: int, B: int, N: int, out: int, status: int,
                             stream: int) -> int:
    return _check(load().acespec_attention_shared(ctx, C.byref(shared), prefix_of, C.byref(kv), layer,
                                                  q, parent_idx, B, N, out, status, stream))


def acespec_qk_norm_rope(ctx, norm: QKNorm, shared: Optional[KVShared], prefix_of: Optional[int],
                         kv: KVCache, layer: int, qkv: int, parent_idx: int, B: int, N: int, q: int,
                         status: int, stream: int) -> int:
    return _check(load().acespec_qk_norm_rope(ctx, C.byref(norm),
                                              None if shared is None else C.byref(shared), prefix_of,
                                              C.byref(kv), layer, qkv, parent_idx, B, N, q, status,
                                              stream))


def acespec_verify_tree_shared(ctx, weights: Weights, norms, shared: Optional[KVShared],
                               prefix_of: Optional[int], kv: KVCache, tree_tokens: int,
                               parent_idx: int, draft_q: Optional[int], q_hat: Optional[int],
                               uniforms: int, B: int, N: int, params: Params, outputs: Outputs,
                               stream: int) -> int:
    """norms: an array of QKNorm, one a layer, or None."""
    return _check(load().acespec_verify_tree_shared(ctx, C.byref(weights), norms,
                                                    None if shared is None else C.byref(shared),
                                                    prefix_of, C.byref(kv), tree_tokens, parent_idx,
                                                    draft_q, q_hat, uniforms, B, N, C.byref(params),
                                                    C.byref(outputs), stream))


def acespec_fork_kv(ctx, src: KVCache, src_batch: int, dst: KVCache, dst_batch: int, from_: int,
                    first: Optional[int], new_prefix_len: int, stream: int) -> int:
    return _check(load().acespec_fork_kv(ctx, C.byref(src), src_batch, C.byref(dst), dst_batch, from_,
                                         first, new_prefix_len, stream))


def acespec_timing_enable(ctx, enable: bool) -> None:
    _check(load().acespec_timing_enable(ctx, 1 if enable else 0))


def acespec_timing_only(ctx, kind: Optional[str]) -> None:
    _check(load().acespec_timing_only(ctx, kind.encode() if kind else None))


def acespec_timing_read(ctx) -> Dict[str, tuple]:
    n = 32
    names = (C.c_char_p * n)()
    ms = (C.c_double * n)()
    cnt = (C.c_int * n)()
    k = _check(load().acespec_timing_read(ctx, names, ms, cnt, n))
    return {names[i].decode(): (ms[i], cnt[i]) for i in range(k)}


# --------------------------------------------------------------------------------------
# Marshalling helper over torch device tensors
# --------------------------------------------------------------------------------------


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


class QuantCache:
    """The tensors of a KV cache in 4 bits (acespec_kv_quant): blocks [L, B, Hkv,
    capacity / 32, 34 hd] uint8, tail_k [L, B, Hkv, tail_capacity, hd] and tail_v [L, B, Hkv,
    hd, tail_capacity] in the model dtype, prefix_len [B] int32, all contiguous on one GPU.
    Shapes and types are checked here, once.  Only prefix_len can be assigned (a commit's new
    lengths; checked again); a call refuses tensors whose memory has moved since."""

    def __init__(self, blocks, tail_k, tail_v, capacity: int, tail_capacity: int, prefix_len):
        import torch
        if blocks.dim() != 5 or tail_k.dim() != 5 or tail_k.dtype not in (torch.bfloat16, torch.float32):
            raise ValueError("blocks and tail_k must have five dimensions, tail_k in bfloat16 or float32")
        L, B, Hkv, _, hd = tail_k.shape
        self.index = blocks.get_device() if blocks.is_cuda else None   # the GPU's number
        _check_tensors([("blocks", blocks, (L, B, Hkv, capacity // 32, 34 * hd), torch.uint8),
                        ("tail_k", tail_k, (L, B, Hkv, tail_capacity, hd), tail_k.dtype),
                        ("tail_v", tail_v, (L, B, Hkv, hd, tail_capacity), tail_k.dtype),
                        ("prefix_len", prefix_len, (B,), torch.int32)], self.index)
        self._fit = (L, B, Hkv, hd, ACESPEC_BF16 if tail_k.dtype == torch.bfloat16 else ACESPEC_F32)
        self._tensors = (blocks, tail_k, tail_v, prefix_len)
        self._at = (_ptr(blocks), _ptr(tail_k), _ptr(tail_v), _ptr(prefix_len))
        self._struct = KVQuant(*self._at[:3], capacity, tail_capacity, self._at[3])

    blocks = property(lambda self: self._tensors[0])
    tail_k = property(lambda self: self._tensors[1])
    tail_v = property(lambda self: self._tensors[2])
    prefix_len = property(lambda self: self._tensors[3])
    capacity = property(lambda self: self._struct.capacity)
    tail_capacity = property(lambda self: self._struct.tail_capacity)

    @prefix_len.setter
    def prefix_len(self, lengths):
        _check_tensors((("prefix_len", lengths, self.prefix_len.shape, self.prefix_len.dtype),),
                       self.index)
        self._tensors = (*self._tensors[:3], lengths)
        self._at = (*self._at[:3], _ptr(lengths))
        self._struct = KVQuant(*self._at[:3], self.capacity, self.tail_capacity, self._at[3])

    @classmethod
    def alloc(cls, L: int, B: int, Hkv: int, hd: int, capacity: int, max_nodes: int, dtype: str,
              device="cuda"):
        """An empty cache of `capacity` slots in blocks, whose tail takes trees of max_nodes
        drafted nodes."""
        import torch
        dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        cap, tail = (capacity + 31) // 32 * 32, (31 + max_nodes + 1 + 63) // 64 * 64
        return cls(torch.zeros((L, B, Hkv, cap // 32, 34 * hd), dtype=torch.uint8, device=device),
                   torch.zeros((L, B, Hkv, tail, hd), dtype=dt, device=device),
                   torch.zeros((L, B, Hkv, hd, tail), dtype=dt, device=device), cap, tail,
                   torch.zeros(B, dtype=torch.int32, device=device))

    def with_prefix(self, prefix_len) -> "QuantCache":
        """The same cache under other lengths (a commit's new_prefix_len)."""
        other = QuantCache.__new__(QuantCache)
        other.__dict__.update(self.__dict__)
        other.prefix_len = prefix_len
        return other

    def struct(self) -> KVQuant:
        b, k, v, p = self._tensors
        if (b.data_ptr(), k.data_ptr(), v.data_ptr(), p.data_ptr()) != self._at:
            moved = [n for n, t, at in zip(("blocks", "tail_k", "tail_v", "prefix_len"), self._tensors, self._at)
                     if t.data_ptr() != at]
            raise ValueError(f"the memory of {', '.join(moved)} moved after the cache was made (resize_ or set_)")
        return self._struct


class SharedPrefix:
    """The tensors of a store of shared prefixes (acespec_kv_shared): blocks [L, P, Hkv,
    capacity / 64, 128 hd] in float16 for a bf16 model and float32 for an fp32 one, len [P] int32,
    contiguous on one GPU.  Shapes and types are checked here, once.  Only len can be assigned (what
    share_prefix returned; checked again); a call refuses tensors whose memory has moved since."""

    def __init__(self, blocks, capacity: int, lengths):
        import torch
        if blocks.dim() != 5 or blocks.dtype not in (torch.float16, torch.float32):
            raise ValueError("blocks must have five dimensions, in float16 or float32")
        L, P, Hkv, _, n = blocks.shape
        self.index = blocks.get_device() if blocks.is_cuda else None   # the GPU's number
        _check_tensors((("blocks", blocks, (L, P, Hkv, capacity // 64, n // 128 * 128), blocks.dtype),
                        ("len", lengths, (P,), torch.int32)), self.index)
        self._fit = (L, Hkv, n // 128, ACESPEC_BF16 if blocks.dtype == torch.float16 else ACESPEC_F32)
        self._tensors = (blocks, lengths)
        self._at = (_ptr(blocks), _ptr(lengths))
        self._struct = KVShared(self._at[0], P, capacity, self._at[1])

    blocks = property(lambda self: self._tensors[0])
    len = property(lambda self: self._tensors[1])
    prefixes = property(lambda self: self._struct.prefixes)
    capacity = property(lambda self: self._struct.capacity)

    @len.setter
    def len(self, lengths):
        _check_tensors((("len", lengths, self._tensors[1].shape, self._tensors[1].dtype),), self.index)
        self._tensors = (self._tensors[0], lengths)
        self._at = (self._at[0], _ptr(lengths))
        self._struct = KVShared(self._at[0], self.prefixes, self.capacity, self._at[1])

    @classmethod
    def alloc(cls, L: int, P: int, Hkv: int, hd: int, capacity: int, dtype: str, device="cuda"):
        """An empty store of P prefixes of up to `capacity` slots each."""
        import torch
        cap = (capacity + 63) // 64 * 64
        return cls(torch.zeros((L, P, Hkv, cap // 64, 128 * hd), device=device,
                               dtype=torch.float16 if dtype == "bf16" else torch.float32),
                   cap, torch.zeros(P, dtype=torch.int32, device=device))

    def struct(self) -> KVShared:
        if (self._tensors[0].data_ptr(), self._tensors[1].data_ptr()) != self._at:
            raise ValueError("the memory of blocks or len moved after the store was made (resize_ or set_)")
        return self._struct


def _stream_of(index: int) -> int:
    """The current stream's handle on that GPU (the Stream object around it costs 2.5 us more)."""
    return _torch_c()._cuda_getCurrentRawStream(index)


_torch_bindings = None


def _torch_c():
    """torch._C, looked up once (an import statement in every call costs as much as a tensor's checks)."""
    global _torch_bindings
    if _torch_bindings is None:
        import torch
        _torch_bindings = torch._C
    return _torch_bindings


def _fits(t, shape, dt, index) -> bool:
    """What _check_tensors asks of one tensor."""
    return (t is not None and t.shape == shape and t.dtype is dt and t.get_device() == index and
            t.is_contiguous())


def _check_tensors(want, index):
    """Tensors whose shape, type or stride differ from what the call says would be read out of
    range.  index: the GPU's."""
    for name, t, shape, dt in want:
        if t is None or t.shape != shape or t.dtype is not dt or t.get_device() != index or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous {dt} tensor {tuple(shape)} on GPU {index} "
                             f"(got {'None' if t is None else f'{t.dtype} {tuple(t.shape)} on {t.device}'})")


def _sized(name, t, dims: int):
    """The shape of a tensor that says how large a call is."""
    if t is None or t.dim() != dims:
        raise ValueError(f"{name} must be a tensor of {dims} dimension{'s' * (dims > 1)} "
                         f"(got {'None' if t is None else tuple(t.shape)})")
    return t.shape


def _check_room(want, index):
    """Tensors of which a call uses the first n elements."""
    for name, t, n, dt in want:
        if t is None or t.numel() < n or t.dtype is not dt or t.get_device() != index or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous {dt} tensor of at least {n} elements on GPU {index} "
                             f"(got {'None' if t is None else f'{t.dtype} {tuple(t.shape)} on {t.device}'})")


class Verifier:
    """Owns a context for one model shape and turns torch tensors into ABI structs."""

    index = None   # the GPU that the context's workspace is on

    def __init__(self, L, d, H, Hkv, hd, F, V, dtype: str, max_batch: int, max_nodes: int,
                 rope_base=10000.0, rms_eps=1e-5):
        import torch
        self.desc = ModelDesc(L, d, H, Hkv, hd, F, V, rope_base, rms_eps,
                              ACESPEC_BF16 if dtype == "bf16" else ACESPEC_F32)
        self.V = V
        self.ctx = acespec_create(self.desc, max_batch, max_nodes)
        self.index = torch.cuda.current_device()
        self._kv = (L, Hkv, hd, torch.bfloat16 if dtype == "bf16" else torch.float32, torch.int32)
        self._store = (L, Hkv, hd, self.desc.dtype)   # (a struct's fields cost a lookup each in every call)
        self._heads = (H, (H + 2 * Hkv) * hd, hd)     # query heads, a projection's width, head dim
        self._keep: List = []

    @classmethod
    def for_workload(cls, w, max_batch=None, max_nodes=None):
        import synth
        n = 0 if w.tree == "tail" else len(synth.tree_parents(w)) - 1
        mb = max_batch or (w.rows if w.tree == "tail" else w.B)
        return cls(w.L, w.d, w.H, w.Hkv, w.hd, w.F, w.V, w.dtype, mb,
                   n if max_nodes is None else max_nodes, w.rope_base, w.rms_eps)

    def close(self):
        if self.ctx:
            acespec_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    DENSE = ("wqkv", "wo", "w_gate_up", "w_down")

    def pack_weights(self, W, drop_source=False):
        """A copy of W whose dense matrices (the DENSE ones of every layer and the LM head)
        are in the packed layout (acespec_pack_weight); the embedding and the norm gains
        are shared with W.  The result carries `packed = True` for weights_struct.
        drop_source: release each row-major matrix of W once it is packed (W's entries
        become None), so that a model only slightly smaller than the device fits."""
        import copy
        import torch

        def pk(t):
            out = torch.empty(t.numel(), dtype=torch.float16, device=t.device)
            acespec_pack_weight(_ptr(t), _ptr(out), t.shape[0], t.shape[1], self._stream())
            return out

        P = copy.copy(W)
        P.layers = []
        for lw in W.layers:
            P.layers.append(dict(lw, **{k: pk(lw[k]) for k in self.DENSE}))
            if drop_source:
                for k in self.DENSE:
                    lw[k] = None
        P.lm_head = pk(W.lm_head)
        if drop_source:
            W.lm_head = None
        P.packed = True
        return P

    def weights_struct(self, W) -> Weights:
        layers = (LayerWeights * max(1, len(W.layers)))()
        for i, lw in enumerate(W.layers):
            layers[i] = LayerWeights(_ptr(lw["attn_norm"]), _ptr(lw["wqkv"]), _ptr(lw["wo"]),
                                     _ptr(lw["mlp_norm"]), _ptr(lw["w_gate_up"]),
                                     _ptr(lw["w_down"]))
        self._keep.append(layers)
        layout = ACESPEC_LAYOUT_PACKED if getattr(W, "packed", False) else ACESPEC_LAYOUT_ROWS
        return Weights(_ptr(W.embed), layers, _ptr(W.final_norm), _ptr(W.lm_head), layout)

    @staticmethod
    def alloc_outputs(rows: int, sessions: int, n1: int, k: int, V: int, device,
                      keep_logits: bool = False) -> Dict:
        import torch
        i32 = dict(dtype=torch.int32, device=device)
        return dict(
            accept=torch.zeros(rows, dtype=torch.uint8, device=device),
            acc_prefix_len=torch.zeros(rows, **i32),
            resample_token=torch.zeros(rows, **i32),
            bonus_token=torch.zeros(rows, **i32),
            topk_ids=torch.zeros(rows, k, **i32),
            topk_probs=torch.zeros(rows, k, dtype=torch.float32, device=device),
            path=torch.zeros(sessions, n1, **i32),
            path_len=torch.zeros(sessions, **i32),
            next_token=torch.zeros(sessions, **i32),
            sibling_hit=torch.zeros(sessions, dtype=torch.uint8, device=device),
            status=torch.zeros(sessions, **i32),
            logits_out=(torch.zeros(rows, V, dtype=torch.float32, device=device)
                        if keep_logits else None),
        )

    @staticmethod
    def outputs_struct(o: Dict) -> Outputs:
        return Outputs(*[_ptr(o[f]) for f, _ in Outputs._fields_])

    @staticmethod
    def _stream() -> int:
        import torch
        # the handle itself: the Stream object around it costs 2.5 us more a call
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())

    def verify_tree(self, wstruct: Weights, kv_k, kv_v, capacity: int, prefix_len, tokens,
                    parents, q, u, T: float, top_p: float, k: int, outs: Dict) -> int:
        B, n1 = tokens.shape
        kv = KVCache(_ptr(kv_k), _ptr(kv_v), capacity, _ptr(prefix_len))
        return acespec_verify_tree(self.ctx, wstruct, kv, _ptr(tokens), _ptr(parents), _ptr(q),
                                   _ptr(u), B, n1 - 1, Params(T, top_p, k),
                                   self.outputs_struct(outs), self._stream())

    def verify_tree_scalar_q(self, wstruct: Weights, kv_k, kv_v, capacity: int, prefix_len,
                             tokens, parents, q_hat, u, T: float, top_p: float, k: int,
                             outs: Dict) -> int:
        B, n1 = tokens.shape
        kv = KVCache(_ptr(kv_k), _ptr(kv_v), capacity, _ptr(prefix_len))
        return acespec_verify_tree_scalar_q(self.ctx, wstruct, kv, _ptr(tokens), _ptr(parents),
                                            _ptr(q_hat), _ptr(u), B, n1 - 1, Params(T, top_p, k),
                                            self.outputs_struct(outs), self._stream())

    def commit_kv(self, kv_k, kv_v, capacity: int, prefix_len, path, path_len, status,
                  new_prefix_len) -> int:
        B, n1 = path.shape
        kv = KVCache(_ptr(kv_k), _ptr(kv_v), capacity, _ptr(prefix_len))
        return acespec_commit_kv(self.ctx, kv, _ptr(path), _ptr(path_len), _ptr(status), B,
                                 n1 - 1, _ptr(new_prefix_len), self._stream())

    def verify_tail(self, lm_head, final_norm, hidden, draft, q, u, chain_len: int, T: float,
                    top_p: float, k: int, outs: Dict, packed: bool = False) -> int:
        """packed: lm_head is the flat output of pack_weights (acespec_pack_weight)."""
        R = hidden.shape[0]
        return acespec_verify_tail(self.ctx, _ptr(lm_head),
                                   ACESPEC_LAYOUT_PACKED if packed else ACESPEC_LAYOUT_ROWS,
                                   _ptr(final_norm), _ptr(hidden), _ptr(draft), _ptr(q),
                                   _ptr(u), R, chain_len, Params(T, top_p, k),
                                   self.outputs_struct(outs), self._stream())

    def _check_quant(self, cache: QuantCache, B: int):
        import torch
        d = self.desc
        if cache.index != torch.cuda.current_device():
            raise ValueError(f"the cache is on cuda:{cache.index}, the current device and stream "
                             f"are cuda:{torch.cuda.current_device()}'s")
        if self.index not in (None, cache.index):
            raise ValueError(f"the context is on cuda:{self.index}, the cache on cuda:{cache.index}")
        if cache._fit != (d.n_layers, B, d.n_kv_heads, d.head_dim, d.dtype):
            raise ValueError(f"a cache of (layers, sessions, kv heads, head dim, dtype) {cache._fit} "
                             f"is not this model's and batch's "
                             f"{(d.n_layers, B, d.n_kv_heads, d.head_dim, d.dtype)}")

    def _check_kv(self, kv_k, kv_v, capacity: int, cache: QuantCache, lengths):
        """A cache in the model's type against one in 4 bits; lengths: (name, tensor or None)."""
        L, B, Hkv, hd, _ = cache._fit
        dt, i32 = cache.tail_k.dtype, cache.prefix_len.dtype
        _check_tensors((("kv_k", kv_k, (L, B, Hkv, capacity, hd), dt),
                        ("kv_v", kv_v, (L, B, Hkv, hd, capacity), dt)), cache.index)
        _check_tensors([(n, t, (B,), i32) for n, t in lengths if t is not None], cache.index)

    def quantize_kv(self, kv_k, kv_v, capacity: int, prefix_len, cache: QuantCache, status=None,
                    first=None) -> int:
        """kv's slots [0, prefix_len) brought to 4 bits (acespec_quantize_kv).  The cache's own
        prefix_len is not touched."""
        B = prefix_len.shape[0]
        self._check_quant(cache, B)
        self._check_kv(kv_k, kv_v, capacity, cache, (("prefix_len", prefix_len), ("status", status),
                                                     ("first", first)))
        kv = KVCache(_ptr(kv_k), _ptr(kv_v), capacity, _ptr(prefix_len))
        return acespec_quantize_kv(self.ctx, kv, cache.struct(), _ptr(first), B, _ptr(status),
                                   self._stream())

    def dequantize_kv(self, cache: QuantCache, kv_k, kv_v, capacity: int, status=None,
                      first=None) -> int:
        """Slots [first / 32 * 32, cache.prefix_len) read back into kv (acespec_dequantize_kv)."""
        B = cache.prefix_len.shape[0]
        self._check_quant(cache, B)
        self._check_kv(kv_k, kv_v, capacity, cache, (("status", status), ("first", first)))
        kv = KVCache(_ptr(kv_k), _ptr(kv_v), capacity, None)
        return acespec_dequantize_kv(self.ctx, cache.struct(), kv, _ptr(first), B, _ptr(status),
                                     self._stream())

    def attention_quant(self, cache: QuantCache, layer: int, q, parents, out, status,
                        window: int = 0, sinks: int = 0) -> int:
        """Tree attention of one layer (acespec_attention_quant): q, out [B, N+1, H, hd]."""
        B, n1 = parents.shape
        self._check_quant(cache, B)
        shape = (B, n1, self.desc.n_heads, self.desc.head_dim)
        dt, i32 = cache.tail_k.dtype, cache.prefix_len.dtype
        _check_tensors((("q", q, shape, dt), ("out", out, shape, dt), ("parents", parents, (B, n1), i32),
                        ("status", status, (B,), i32)), cache.index)
        return acespec_attention_quant(self.ctx, cache.struct(), layer, AttnSpan(window, sinks),
                                       _ptr(q), _ptr(parents), B, n1 - 1, _ptr(out), _ptr(status),
                                       self._stream())

    def verify_tree_quant(self, wstruct: Weights, cache: QuantCache, tokens, parents, q, u,
                          T: float, top_p: float, k: int, outs: Dict, window: int = 0,
                          sinks: int = 0, scalar: bool = False) -> int:
        """verify_tree over a cache in 4 bits; scalar: q is q_hat [B, N+1]."""
        B, n1 = tokens.shape
        self._check_quant(cache, B)
        self._check_step(cache.index, tokens, parents, q, u, k, outs, scalar)
        return acespec_verify_tree_quant(self.ctx, wstruct, cache.struct(), AttnSpan(window, sinks),
                                         _ptr(tokens), _ptr(parents), None if scalar else _ptr(q),
                                         _ptr(q) if scalar else None, _ptr(u), B, n1 - 1,
                                         Params(T, top_p, k), self.outputs_struct(outs),
                                         self._stream())

    def _check_step(self, index: int, tokens, parents, q, u, k: int, outs: Dict, scalar: bool):
        """A verify step's inputs and outputs (those of alloc_outputs; they may be larger)."""
        import torch
        B, n1 = tokens.shape
        rows, V = B * n1, self.desc.vocab
        i32, f32, u8 = torch.int32, torch.float32, torch.uint8
        _check_tensors((("tokens", tokens, (B, n1), i32), ("parents", parents, (B, n1), i32)), index)
        room = [("q", q, rows if scalar else rows * V, f32), ("u", u, rows * 3, f32)]
        for name, n, dt in (("accept", rows, u8), ("acc_prefix_len", rows, i32), ("resample_token", rows, i32),
                            ("bonus_token", rows, i32), ("topk_ids", rows * k, i32),
                            ("topk_probs", rows * k, f32), ("path", rows, i32), ("path_len", B, i32),
                            ("next_token", B, i32), ("sibling_hit", B, u8), ("status", B, i32)):
            room.append((name, outs[name], n, dt))
        if outs["logits_out"] is not None:
            room.append(("logits_out", outs["logits_out"], rows * V, f32))
        _check_room(room, index)

    def commit_kv_quant(self, cache: QuantCache, path, path_len, status, new_prefix_len) -> int:
        B, n1 = path.shape
        self._check_quant(cache, B)
        i32 = cache.prefix_len.dtype
        _check_tensors((("path", path, (B, n1), i32), ("path_len", path_len, (B,), i32),
                        ("new_prefix_len", new_prefix_len, (B,), i32)), cache.index)
        if status is not None:
            _check_tensors((("status", status, (B,), i32),), cache.index)
        return acespec_commit_kv_quant(self.ctx, cache.struct(), _ptr(path), _ptr(path_len),
                                       _ptr(status), B, n1 - 1, _ptr(new_prefix_len),
                                       self._stream())

    def _here(self) -> int:
        """The current GPU, which must be the context's."""
        here = _torch_c()._cuda_getDevice()   # (the context is there, and so is the GPU)
        if self.index is not None and self.index != here:
            raise ValueError(f"the context is on cuda:{self.index}, the current device and stream are "
                             f"cuda:{here}'s")
        return here

    def _check_store(self, shared: SharedPrefix, index: int):
        if shared is None:
            raise ValueError("shared must be a SharedPrefix (got None)")
        if shared.index != index:
            raise ValueError(f"the shared prefixes are on cuda:{shared.index}, the current device and "
                             f"stream are cuda:{index}'s")
        if shared._fit != self._store:
            raise ValueError(f"a store of (layers, kv heads, head dim, dtype) {shared._fit} is not this "
                             f"model's {self._store}")

    def _check_shared(self, shared: Optional[SharedPrefix], prefix_of, B: int, index: int):
        if (shared is None) != (prefix_of is None):
            raise ValueError("shared prefixes and prefix_of come together")
        if shared is not None:
            self._check_store(shared, index)
            i32 = self._kv[4]
            if not _fits(prefix_of, (B,), i32, index):
                _check_tensors((("prefix_of", prefix_of, (B,), i32),), index)

    def _check_cache(self, kv_k, kv_v, capacity: int, lengths, index: int, B: Optional[int] = None,
                     name: str = "") -> KVCache:
        """The tensors of a cache in the model's type, of B (None: len(lengths)) sessions."""
        B = _sized(name + "prefix_len", lengths, 1)[0] if B is None else B
        L, Hkv, hd, dt, i32 = self._kv
        k, v = (L, B, Hkv, capacity, hd), (L, B, Hkv, hd, capacity)
        if not (_fits(kv_k, k, dt, index) and _fits(kv_v, v, dt, index) and _fits(lengths, (B,), i32, index)):
            _check_tensors(((name + "kv_k", kv_k, k, dt), (name + "kv_v", kv_v, v, dt),
                            (name + "prefix_len", lengths, (B,), i32)), index)
        return KVCache(kv_k.data_ptr(), kv_v.data_ptr(), capacity, lengths.data_ptr())

    def share_prefix(self, kv_k, kv_v, capacity: int, prefix_len, from_, shared: SharedPrefix, new_len,
                     count=None) -> int:
        """Sessions' first slots taken over as shared prefixes (acespec_share_prefix): from_ [P] the
        sessions or -1, count [P] how many slots (None: all).  shared.len is not touched; new_len [P]
        is written."""
        index, i32 = self._here(), self._kv[4]
        self._check_store(shared, index)
        P = (shared.prefixes,)
        kv = self._check_cache(kv_k, kv_v, capacity, prefix_len, index)
        if not (_fits(from_, P, i32, index) and _fits(new_len, P, i32, index) and
                (count is None or _fits(count, P, i32, index))):
            _check_tensors([(n, t, P, i32) for n, t in (("from_", from_), ("new_len", new_len), ("count", count))
                            if n != "count" or t is not None], index)
        return acespec_share_prefix(self.ctx, kv, prefix_len.shape[0], shared.struct(), from_.data_ptr(),
                                    _ptr(count), new_len.data_ptr(), _stream_of(index))

    def attention_shared(self, shared: SharedPrefix, prefix_of, kv_k, kv_v, capacity: int, prefix_len,
                         layer: int, q, parents, out, status) -> int:
        """Tree attention of one layer behind shared prefixes (acespec_attention_shared): q, out
        [B, N+1, H, hd]."""
        B, n1 = _sized("parents", parents, 2)
        index, dt, i32 = self._here(), self._kv[3], self._kv[4]
        if shared is None:
            self._check_store(shared, index)   # (refused: only calls that can do without take None)
        self._check_shared(shared, prefix_of, B, index)
        kv = self._check_cache(kv_k, kv_v, capacity, prefix_len, index, B)
        shape = (B, n1, self._heads[0], self._heads[2])
        if not (_fits(q, shape, dt, index) and _fits(out, shape, dt, index) and
                _fits(parents, (B, n1), i32, index) and _fits(status, (B,), i32, index)):
            _check_tensors((("q", q, shape, dt), ("out", out, shape, dt), ("parents", parents, (B, n1), i32),
                            ("status", status, (B,), i32)), index)
        return acespec_attention_shared(self.ctx, shared.struct(), prefix_of.data_ptr(), kv, layer,
                                        q.data_ptr(), parents.data_ptr(), B, n1 - 1, out.data_ptr(),
                                        status.data_ptr(), _stream_of(index))

    def qk_norm_rope(self, qkv, q_gain, k_gain, kv_k, kv_v, capacity: int, prefix_len, layer: int,
                     parents, q_out, status, shared: Optional[SharedPrefix] = None,
                     prefix_of=None) -> int:
        """One layer's projection [B, N+1, (H + 2 Hkv) hd] normalised per head (gains [hd] or None),
        rotated and written to q_out [B, N+1, H, hd] and the cache (acespec_qk_norm_rope)."""
        B, n1 = _sized("parents", parents, 2)
        index, dt, i32 = self._here(), self._kv[3], self._kv[4]
        self._check_shared(shared, prefix_of, B, index)
        kv = self._check_cache(kv_k, kv_v, capacity, prefix_len, index, B)
        H, width, hd = self._heads
        wide, rows = (B, n1, width), (B, n1, H, hd)
        if not (_fits(qkv, wide, dt, index) and _fits(q_out, rows, dt, index) and
                _fits(parents, (B, n1), i32, index) and _fits(status, (B,), i32, index) and
                (q_gain is None or _fits(q_gain, (hd,), dt, index)) and
                (k_gain is None or _fits(k_gain, (hd,), dt, index))):
            _check_tensors([("qkv", qkv, wide, dt), ("q_out", q_out, rows, dt),
                            ("parents", parents, (B, n1), i32), ("status", status, (B,), i32)] +
                           [(n, t, (hd,), dt) for n, t in (("q_gain", q_gain), ("k_gain", k_gain))
                            if t is not None], index)
        return acespec_qk_norm_rope(self.ctx, QKNorm(_ptr(q_gain), _ptr(k_gain)),
                                    None if shared is None else shared.struct(), _ptr(prefix_of), kv,
                                    layer, qkv.data_ptr(), parents.data_ptr(), B, n1 - 1,
                                    q_out.data_ptr(), status.data_ptr(), _stream_of(index))

    def verify_tree_shared(self, wstruct: Weights, shared: Optional[SharedPrefix], prefix_of, kv_k, kv_v,
                           capacity: int, prefix_len, tokens, parents, q, u, T: float, top_p: float,
                           k: int, outs: Dict, norms=None, scalar: bool = False) -> int:
        """verify_tree for sessions behind shared prefixes (or None, None); norms: a (q_gain, k_gain)
        pair a layer, or None; scalar: q is q_hat [B, N+1]."""
        B, n1 = _sized("tokens", tokens, 2)
        d, index, dt, i32 = self.desc, self._here(), self._kv[3], self._kv[4]
        self._check_shared(shared, prefix_of, B, index)
        kv = self._check_cache(kv_k, kv_v, capacity, prefix_len, index, B)
        self._check_step(index, tokens, parents, q, u, k, outs, scalar)
        array = None
        if norms is not None:
            if len(norms) != d.n_layers:
                raise ValueError(f"norms has {len(norms)} entries, the model {d.n_layers} layers")
            _check_tensors([(f"norms[{l}]", t, (d.head_dim,), dt) for l, pair in enumerate(norms)
                            for t in pair if t is not None], index)
            array = (QKNorm * d.n_layers)(*[QKNorm(_ptr(a), _ptr(b)) for a, b in norms])
        return acespec_verify_tree_shared(self.ctx, wstruct, array,
                                          None if shared is None else shared.struct(), _ptr(prefix_of),
                                          kv, _ptr(tokens), _ptr(parents), None if scalar else _ptr(q),
                                          _ptr(q) if scalar else None, _ptr(u), B, n1 - 1,
                                          Params(T, top_p, k), self.outputs_struct(outs),
                                          self._stream())

    def fork_kv(self, src_k, src_v, src_capacity: int, src_len, dst_k, dst_v, dst_capacity: int, dst_len,
                from_, new_prefix_len, first=None) -> int:
        """Sessions take over others' slots [first, src_len) (acespec_fork_kv): from_ [B of dst] the
        sessions of src, or -1; src and dst may be the same tensors.  dst_len is not touched;
        new_prefix_len is written."""
        index, i32 = self._here(), self._kv[4]
        src = self._check_cache(src_k, src_v, src_capacity, src_len, index, None, "src ")
        dst = self._check_cache(dst_k, dst_v, dst_capacity, dst_len, index, None, "dst ")
        n = dst_len.shape
        if not (_fits(from_, n, i32, index) and _fits(new_prefix_len, n, i32, index) and
                (first is None or _fits(first, n, i32, index))):
            _check_tensors([(x, t, n, i32) for x, t in
                            (("from_", from_), ("new_prefix_len", new_prefix_len), ("first", first))
                            if x != "first" or t is not None], index)
        return acespec_fork_kv(self.ctx, src, src_len.shape[0], dst, n[0], from_.data_ptr(), _ptr(first),
                               new_prefix_len.data_ptr(), _stream_of(index))
