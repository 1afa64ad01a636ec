"""ctypes binding of libspecdec.so: same names as include/specdec.h, argument
marshalling only.  Every step of the path runs in the library's HIP kernels;
PyTorch appears here only as the owner of device memory and streams.

The library must have been built (python -m paper_2203_16487_amd.build); there
is no fallback of any kind: a missing library raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, Optional, Sequence

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libspecdec.so")

SPECDEC_OK = 0
SPECDEC_ERR_INVALID_ARG = -1
SPECDEC_ERR_BAD_STATE = -2
SPECDEC_ERR_TOO_LARGE = -3
SPECDEC_ERR_HIP = -4
SPECDEC_ERR_NO_DEVICE = -5
SPECDEC_VERIFIER = 0
SPECDEC_DRAFTER = 1
SPECDEC_ROW_STATS = 8
ROW_STATS = SPECDEC_ROW_STATS
SPECDEC_COUNTERS = 8
SPECDEC_OPT_SMALL_BATCH_KERNELS = 0
SPECDEC_OPT_LN_FOLD = 1
SPECDEC_OPT_RESIDENT = 2
SPECDEC_OPT_SLICED_SUBLAYERS = 3
SPECDEC_OPT_FP8_WEIGHTS = 4
SPECDEC_OPT_FP8_CROSS_KV = 5
SPECDEC_OPT_WIDE_VOCAB_TILES = 6
SPECDEC_OPT_GIVE_UP_WAITS = 7
SPECDEC_F32, SPECDEC_BF16, SPECDEC_F16 = 0, 1, 2


class specdec_model_desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("enc_layers", "dec_layers", "d_model", "n_heads", "d_ffn", "vocab",
                                         "bos_id", "eos_id", "pad_id", "mask_id")]


class specdec_limits(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("max_batch", "k_max", "max_src", "max_tgt")]


class specdec_tree_attn_desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "batch", "rows", "n_heads", "n_kv_heads", "head_dim", "capacity")] + [
        ("scale", C.c_float)] + [(n, C.c_int64 * 3) for n in ("q_stride", "k_stride", "v_stride", "out_stride")]


class specdec_cache_desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("layers", "heads", "capacity", "row_bytes")] + [
        (n, C.c_int64) for n in ("layer_stride", "seq_stride", "head_stride", "row_stride")]


EXPORTS = {
    "specdec_create": (C.c_int, [C.POINTER(C.c_void_p), C.POINTER(specdec_limits)]),
    "specdec_destroy": (None, [C.c_void_p]),
    "specdec_last_error": (C.c_char_p, [C.c_void_p]),
    "specdec_num_weights": (C.c_int, [C.POINTER(specdec_model_desc), C.POINTER(C.c_int32)]),
    "specdec_weight_shape": (C.c_int, [C.POINTER(specdec_model_desc), C.c_int32, C.POINTER(C.c_int64), C.POINTER(C.c_int64)]),
    "specdec_state_bytes": (C.c_int, [C.c_void_p, C.POINTER(C.c_size_t)]),
    "specdec_bind_state": (C.c_int, [C.c_void_p, C.c_void_p, C.c_size_t]),
    "specdec_workspace_bytes": (C.c_int, [C.c_void_p, C.POINTER(specdec_model_desc), C.POINTER(C.c_size_t)]),
    "specdec_bind_model": (C.c_int, [C.c_void_p, C.c_int, C.POINTER(specdec_model_desc), C.POINTER(C.c_void_p),
                                     C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p]),
    "specdec_begin": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p]),
    "specdec_encode": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]),
    "specdec_set_memory": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]),
    "specdec_set_stream": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]),
    "specdec_load_cache": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]),
    "specdec_prefill": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p]),
    "specdec_draft": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]),
    "specdec_bind_draft_heads": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "specdec_draft_heads": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]),
    "specdec_configure": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32]),
    "specdec_set_prefix": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]),
    "specdec_get_draft_stats": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "specdec_get_counters": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "specdec_quantize_rows": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_void_p,
                                             C.c_void_p]),
    "specdec_verify": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_float, C.c_void_p, C.c_void_p,
                                 C.c_void_p, C.c_void_p]),
    "specdec_verify_static": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_float, C.c_void_p, C.c_void_p,
                                        C.c_void_p, C.c_void_p]),
    "specdec_commit": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "specdec_rewind": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "specdec_profile_select": (C.c_int, [C.c_void_p, C.c_int32]),
    "specdec_profile_read": (C.c_int, [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_int32)]),
    "specdec_decoder_way": (C.c_int, [C.c_void_p]),
    "specdec_get_output": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]),
    "specdec_get_cache": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]),
    "specdec_get_row_stats": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "specdec_get_memory": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p]),
    "specdec_verify_tree": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]),
    "specdec_commit_tree": (C.c_int, [C.c_void_p] * 6),
    "specdec_fork": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]),
    "specdec_pass_sizes": (C.c_int, [C.c_void_p] + [C.POINTER(C.c_int32)] * 3),
    "specdec_tree_attention_bytes": (C.c_int, [C.c_void_p, C.c_void_p, C.POINTER(C.c_size_t)]),
    "specdec_tree_attention": (C.c_int, [C.c_void_p] * 10 + [C.c_size_t, C.c_void_p]),
    "specdec_tree_visible": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]),
    "specdec_sample": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int, C.c_int32, C.c_int32, C.c_int64] + [C.c_void_p] * 8),
    "specdec_fork_cache": (C.c_int, [C.c_void_p] * 4 + [C.c_int32, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]),
    "specdec_compact_cache": (C.c_int, [C.c_void_p] * 4 + [C.c_int32, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]),
}

_lib = None


def lib() -> C.CDLL:
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2203_16487_amd.build` "
                               "(there is no fallback path)")
        # PyTorch owns the device memory this binding hands over, so both must talk to ONE HIP
        # runtime: importing torch first makes its libamdhip64 the one libspecdec binds to
        # (two runtimes in one process do not see the GPU).
        import torch  # noqa: F401
        L = C.CDLL(LIB_PATH)
        for name, (res, args) in EXPORTS.items():
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        _lib = L
    return _lib


class SpecDecError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libspecdec error {code}: {msg}")
        self.code = code


def _check(ctx, rc: int):
    if rc != SPECDEC_OK:
        msg = lib().specdec_last_error(ctx).decode() if ctx else "(no context)"
        raise SpecDecError(rc, msg)


def make_desc(d) -> specdec_model_desc:
    """From any object with the fields of specdec_model_desc (e.g. synth.ModelDesc)."""
    return specdec_model_desc(*[int(getattr(d, n)) for n, _ in specdec_model_desc._fields_])


def _ptr(t) -> Optional[int]:
    """Device pointer of a torch tensor (None -> NULL)."""
    if t is None:
        return None
    assert t.is_contiguous(), "tensors handed to libspecdec must be contiguous"
    return t.data_ptr()


def _stream() -> int:
    import torch
    return torch.cuda.current_stream().cuda_stream


# ------------------------------------------------------------------------ same-name wrappers
def specdec_create(max_batch: int, k_max: int, max_src: int, max_tgt: int) -> C.c_void_p:
    ctx = C.c_void_p()
    lim = specdec_limits(max_batch, k_max, max_src, max_tgt)
    rc = lib().specdec_create(C.byref(ctx), C.byref(lim))
    if rc != SPECDEC_OK:
        raise SpecDecError(rc, "specdec_create: bad limits")
    return ctx


def specdec_destroy(ctx):
    lib().specdec_destroy(ctx)


def specdec_num_weights(desc) -> int:
    n = C.c_int32()
    _check(None, lib().specdec_num_weights(C.byref(make_desc(desc)), C.byref(n)))
    return n.value


def specdec_weight_shape(desc, idx: int):
    r, c = C.c_int64(), C.c_int64()
    _check(None, lib().specdec_weight_shape(C.byref(make_desc(desc)), idx, C.byref(r), C.byref(c)))
    return r.value, c.value


def specdec_state_bytes(ctx) -> int:
    n = C.c_size_t()
    _check(ctx, lib().specdec_state_bytes(ctx, C.byref(n)))
    return n.value


def specdec_bind_state(ctx, buf):
    _check(ctx, lib().specdec_bind_state(ctx, _ptr(buf), buf.numel() * buf.element_size()))


def specdec_workspace_bytes(ctx, desc) -> int:
    n = C.c_size_t()
    _check(ctx, lib().specdec_workspace_bytes(ctx, C.byref(make_desc(desc)), C.byref(n)))
    return n.value


def specdec_bind_model(ctx, role: int, desc, weights: Sequence, workspace):
    arr = (C.c_void_p * len(weights))(*[_ptr(w) for w in weights])
    _check(ctx, lib().specdec_bind_model(ctx, role, C.byref(make_desc(desc)), arr, len(weights), _ptr(workspace),
                                         workspace.numel() * workspace.element_size(), _stream()))


def specdec_begin(ctx, B: int, max_new: int):
    _check(ctx, lib().specdec_begin(ctx, B, max_new, _stream()))


def specdec_encode(ctx, src, src_len):
    _check(ctx, lib().specdec_encode(ctx, _ptr(src), _ptr(src_len), src.shape[1], _stream()))


def specdec_set_memory(ctx, role: int, memory, src_len):
    _check(ctx, lib().specdec_set_memory(ctx, role, _ptr(memory), _ptr(src_len), memory.shape[1], _stream()))


def specdec_set_stream(ctx, tokens, length):
    _check(ctx, lib().specdec_set_stream(ctx, _ptr(tokens), _ptr(length), tokens.shape[1] - 1, _stream()))


def specdec_load_cache(ctx, role: int, k_cache, v_cache, n):
    _check(ctx, lib().specdec_load_cache(ctx, role, _ptr(k_cache), _ptr(v_cache), _ptr(n), k_cache.shape[2], _stream()))


def specdec_prefill(ctx, role: int):
    _check(ctx, lib().specdec_prefill(ctx, role, _stream()))


def specdec_draft(ctx, k: int, draft, logits=None):
    _check(ctx, lib().specdec_draft(ctx, k, _ptr(draft), _ptr(logits), _stream()))


def specdec_bind_draft_heads(ctx, n_heads: int, w1, b1, w2, b2):
    _check(ctx, lib().specdec_bind_draft_heads(ctx, n_heads, _ptr(w1), _ptr(b1), _ptr(w2), _ptr(b2)))


def specdec_draft_heads(ctx, accept_len, k: int, draft, logits=None):
    _check(ctx, lib().specdec_draft_heads(ctx, _ptr(accept_len), k, _ptr(draft), _ptr(logits), _stream()))


def specdec_configure(ctx, option: int, value: int):
    _check(ctx, lib().specdec_configure(ctx, option, value))


def specdec_set_prefix(ctx, role: int, tokens, length, k_cache, v_cache):
    _check(ctx, lib().specdec_set_prefix(ctx, role, _ptr(tokens), _ptr(length), tokens.shape[1] - 1, _ptr(k_cache),
                                         _ptr(v_cache), _stream()))


def specdec_get_draft_stats(ctx, stats):
    _check(ctx, lib().specdec_get_draft_stats(ctx, _ptr(stats), _stream()))


def specdec_get_counters(ctx, counters):
    _check(ctx, lib().specdec_get_counters(ctx, _ptr(counters), _stream()))


def specdec_quantize_rows(ctx, w, codes, scale):
    N, K = w.shape
    _check(ctx, lib().specdec_quantize_rows(ctx, _ptr(w), N, K, _ptr(codes), _ptr(scale), _stream()))


def specdec_verify(ctx, draft, k: int, beta: int, tau: float, accept_len, next_token, logits=None):
    _check(ctx, lib().specdec_verify(ctx, _ptr(draft), k, beta, tau, _ptr(accept_len), _ptr(next_token),
                                     _ptr(logits), _stream()))


def specdec_verify_static(ctx, draft, k: int, beta: int, tau: float, accept_len, next_token, logits=None):
    _check(ctx, lib().specdec_verify_static(ctx, _ptr(draft), k, beta, tau, _ptr(accept_len), _ptr(next_token),
                                            _ptr(logits), _stream()))


def specdec_commit(ctx, accept_len, next_token, n_active=None):
    _check(ctx, lib().specdec_commit(ctx, _ptr(accept_len), _ptr(next_token), _ptr(n_active), _stream()))


def specdec_pass_sizes(ctx):
    """(sequences of the present batch, rows a sequence of the pass over trees that can be committed, the verifier's vocabulary), 0 where there is none."""
    n = [C.c_int32() for _ in range(3)]
    _check(ctx, lib().specdec_pass_sizes(ctx, *[C.byref(x) for x in n]))
    return tuple(x.value for x in n)


def specdec_verify_tree(ctx, draft, parent, logits):
    """draft, parent int32 [B, n] (None: n = 0); logits fp32 [B, n + 1, V]."""
    B, _, V = specdec_pass_sizes(ctx)
    d, z = (0, 0) if draft is None else _shape("draft", draft, 2), _shape("logits", logits, 3)
    # (without a batch or a model: by the tensors' own sizes, and the library says what is missing)
    B, n, V = B or d[0] or z[0], d[1], V or z[2]
    if n and parent is None:
        raise SpecDecError(SPECDEC_ERR_INVALID_ARG, "parent: None, with drafts")
    dp, pp = _ints("draft", draft, (B, n)), _ints("parent", parent, (B, n))
    _check(ctx, lib().specdec_verify_tree(ctx, dp, pp, n, _ints("logits", logits, (B, n + 1, V), "float32"), _on_gpu(draft, parent, logits)))


def specdec_commit_tree(ctx, token, accept_len=None, next_token=None, n_active=None):
    """token int32 [B, n + 1] of the latest specdec_verify_tree; accept_len, next_token int32 [B] or None, n_active int32 [1] or None."""
    B, T, _ = specdec_pass_sizes(ctx)
    t = _shape("token", token, 2)
    B, T = B or t[0], T or t[1]
    args = (_ints("token", token, (B, T)), _ints("accept_len", accept_len, (B,)), _ints("next_token", next_token, (B,)),
            None if n_active is None else _ints("n_active", n_active.view(-1), (1,)))
    _check(ctx, lib().specdec_commit_tree(ctx, *args, _on_gpu(token, accept_len, next_token, n_active)))


def specdec_fork(ctx, src):
    """src int32 [sequences of the new batch]."""
    n = _shape("src", src, 1)
    _check(ctx, lib().specdec_fork(ctx, _ints("src", src, n), n[0], _on_gpu(src)))


def specdec_rewind(ctx, length):
    _check(ctx, lib().specdec_rewind(ctx, _ptr(length), _stream()))


KIND = dict(none=-1, gemm_f32=0, gemm_bf16=1, gemm_qkv=2, attn=3, vocab=4, ln=5, accept=6, other=7, resident=8)


def specdec_profile_select(ctx, kind: int):
    _check(ctx, lib().specdec_profile_select(ctx, kind))


def specdec_profile_read(ctx):
    ms, n = C.c_double(), C.c_int32()
    _check(ctx, lib().specdec_profile_read(ctx, C.byref(ms), C.byref(n)))
    return ms.value, n.value


WAYS = ("launches", "gpu", "xcd", "xcd in place")   # SPECDEC_WAY_*


def specdec_decoder_way(ctx) -> str:
    return WAYS[lib().specdec_decoder_way(ctx)]


def specdec_get_output(ctx, tokens, out_len, finished=None):
    _check(ctx, lib().specdec_get_output(ctx, _ptr(tokens), tokens.shape[1], _ptr(out_len), _ptr(finished), _stream()))


def specdec_get_cache(ctx, role: int, k_cache, v_cache):
    _check(ctx, lib().specdec_get_cache(ctx, role, _ptr(k_cache), _ptr(v_cache), k_cache.shape[2], _stream()))


def specdec_get_memory(ctx, role: int, memory):
    _check(ctx, lib().specdec_get_memory(ctx, role, _ptr(memory), _stream()))


def specdec_get_row_stats(ctx, stats):
    _check(ctx, lib().specdec_get_row_stats(ctx, _ptr(stats), _stream()))


# ------------------------------------------------------------------------ operators on the caller's tensors
def _dtype(t, *allowed) -> int:
    import torch
    code = {torch.float32: SPECDEC_F32, torch.bfloat16: SPECDEC_BF16, torch.float16: SPECDEC_F16}.get(t.dtype, -1)
    if code not in allowed:
        raise SpecDecError(SPECDEC_ERR_INVALID_ARG, f"tensors of {t.dtype} are not supported here")
    return code


def _on_gpu(*tensors) -> int:
    """The current stream, if the tensors' storage is on its GPU."""
    import torch
    for t in tensors:
        if t is not None and not t.is_cuda:
            raise SpecDecError(SPECDEC_ERR_INVALID_ARG, f"a tensor is on {t.device}")
    dev = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise SpecDecError(SPECDEC_ERR_INVALID_ARG, f"a tensor is on {t.device}, the current GPU is {dev}")
    return torch._C._cuda_getCurrentRawStream(dev)   # (current_stream() makes an object: 2.7 us of a call's 9)


def _ints(name: str, t, shape, of="int32"):
    """Device pointer of a contiguous tensor of this shape and type (None -> NULL)."""
    if t is None:
        return None
    import torch
    if t.shape != shape or t.dtype is not getattr(torch, of) or not t.is_contiguous():
        raise SpecDecError(SPECDEC_ERR_INVALID_ARG, f"{name}: contiguous {of} {list(shape)} expected, not {t.dtype} {list(t.shape)}")
    return t.data_ptr()


def _shape(name: str, t, dims: int):
    """Its sizes, if it has that many dimensions."""
    if t is None or t.dim() != dims:
        raise SpecDecError(SPECDEC_ERR_INVALID_ARG, f"{name}: {dims} dimensions expected, not {None if t is None else list(t.shape)}")
    return tuple(t.shape)


def _strided(name: str, t, shape):
    if t.shape != shape or (shape[-1] > 1 and t.stride(-1) != 1):
        raise SpecDecError(SPECDEC_ERR_INVALID_ARG, f"{name}: {list(shape)} with consecutive last values expected, not {list(t.shape)}, {t.stride()}")
    return t.data_ptr()


def tree_attn_desc(q, k, v, out, scale: float) -> specdec_tree_attn_desc:
    """Sizes and strides of q, out [B, rows, heads, dim] and k, v [B, kv heads, capacity, dim] (views of any strides, last values consecutive)."""
    B, T, H, dh = q.shape
    _, Hkv, cap, _ = k.shape
    for name, t, shape in (("q", q, (B, T, H, dh)), ("k", k, (B, Hkv, cap, dh)), ("v", v, (B, Hkv, cap, dh)), ("out", out, (B, T, H, dh))):
        _strided(name, t, shape)
        if t.dtype != q.dtype:
            raise SpecDecError(SPECDEC_ERR_INVALID_ARG, f"{name} is {t.dtype}, q {q.dtype}")
    d = specdec_tree_attn_desc(_dtype(q, SPECDEC_BF16, SPECDEC_F16), B, T, H, Hkv, dh, cap, scale)
    for name, t, dims in (("q_stride", q, (0, 1, 2)), ("k_stride", k, (0, 2, 1)), ("v_stride", v, (0, 2, 1)), ("out_stride", out, (0, 1, 2))):
        # (a dimension of one has no stride: whatever the tensor says)
        setattr(d, name, (C.c_int64 * 3)(*[t.stride(i) if t.shape[i] > 1 else 0 for i in dims]))
    d._like = [(t.shape, t.stride(), t.dtype) for t in (q, k, v, out)]
    return d


def specdec_tree_attention_bytes(ctx, desc: specdec_tree_attn_desc) -> int:
    n = C.c_size_t()
    _check(ctx, lib().specdec_tree_attention_bytes(ctx, C.byref(desc), C.byref(n)))
    return n.value


def _as_described(name: str, t, like):
    """Device pointer of a tensor of the sizes, strides and type that a description was made of."""
    if t.shape != like[0] or t.stride() != like[1] or t.dtype is not like[2]:
        raise SpecDecError(SPECDEC_ERR_INVALID_ARG, f"{name}: {t.dtype} {list(t.shape)}, {t.stride()} is not what the description was made of")
    return t.data_ptr()


def specdec_tree_attention(ctx, desc, q, k, v, cached, visible, n_rows, out, workspace):
    """desc: tree_attn_desc of tensors of these sizes and strides.  visible: int64 [B, rows] (bit masks) or None; n_rows: int32 [B] or None."""
    like, B = desc._like, (desc.batch,)
    stream = _on_gpu(q, k, v, cached, visible, n_rows, out, workspace)
    _check(ctx, lib().specdec_tree_attention(
        ctx, C.byref(desc), _as_described("q", q, like[0]), _as_described("k", k, like[1]), _as_described("v", v, like[2]),
        _ints("cached", cached, B), _ints("visible", visible, (desc.batch, desc.rows), "int64"), _ints("n_rows", n_rows, B),
        _as_described("out", out, like[3]), _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(), stream))


def specdec_tree_visible(ctx, parent, visible):
    """parent int32 [B, n] -> visible int64 [B, n + 1]."""
    B, n = parent.shape
    stream = _on_gpu(parent, visible)
    _check(ctx, lib().specdec_tree_visible(ctx, _ints("parent", parent, (B, n)), B, n, _ints("visible", visible, (B, n + 1), "int64"), stream))


def specdec_sample(ctx, logits, temperature, top_k, top_p, min_p, u, token, logprob=None):
    """logits [rows, vocab] (rows of any stride); the settings [rows] or None."""
    rows, vocab = logits.shape
    stream = _on_gpu(logits, temperature, top_k, top_p, min_p, u, token, logprob)
    n = (rows,)
    _check(ctx, lib().specdec_sample(
        ctx, _strided("logits", logits, (rows, vocab)), _dtype(logits, SPECDEC_F32, SPECDEC_BF16, SPECDEC_F16), rows, vocab,
        logits.stride(0) if rows > 1 else 0, _ints("temperature", temperature, n, "float32"), _ints("top_k", top_k, n),
        _ints("top_p", top_p, n, "float32"), _ints("min_p", min_p, n, "float32"), _ints("u", u, n, "float32"), _ints("token", token, n),
        _ints("logprob", logprob, n, "float32"), stream))


def cache_desc(k, v=None) -> specdec_cache_desc:
    """Sizes and strides of k (and v, laid out alike) [layers, sequences, heads, rows, values] (views of any strides, last values consecutive)."""
    layers, B, heads, cap, dh = k.shape
    _strided("k", k, (layers, B, heads, cap, dh))
    if v is not None and (v.shape != k.shape or v.stride() != k.stride() or v.dtype != k.dtype):
        raise SpecDecError(SPECDEC_ERR_INVALID_ARG, "k and v are laid out differently")
    n = k.element_size()
    strides = [k.stride(i) * n if k.shape[i] > 1 else 0 for i in (0, 1, 2, 3)]
    d = specdec_cache_desc(layers, heads, cap, dh * n, strides[0], strides[1], strides[2], strides[3])
    d._like = (k.shape, k.stride(), k.dtype)
    return d


def _slabs(desc, k, v, B: int):
    if B > desc._like[0][1]:
        raise SpecDecError(SPECDEC_ERR_INVALID_ARG, f"{B} sequences in a cache of {desc._like[0][1]}")
    return _as_described("k", k, desc._like), None if v is None else _as_described("v", v, desc._like)


def specdec_fork_cache(ctx, desc, k, v, src, length):
    """desc: cache_desc of k (and v).  src int32 [B], B at most the cache's sequences; length int32 [sequences that src names]."""
    stream = _on_gpu(k, v, src, length)
    B, n = src.numel(), length.numel()
    kp, vp = _slabs(desc, k, v, max(B, n))
    _check(ctx, lib().specdec_fork_cache(ctx, C.byref(desc), kp, vp, B, _ints("src", src, (B,)), n, _ints("length", length, (n,)), stream))


def specdec_compact_cache(ctx, desc, k, v, first, path, count):
    """desc: cache_desc of k (and v).  path int32 [B, n], first and count int32 [B]."""
    stream = _on_gpu(k, v, first, path, count)
    B, n = path.shape
    kp, vp = _slabs(desc, k, v, B)
    _check(ctx, lib().specdec_compact_cache(ctx, C.byref(desc), kp, vp, B, _ints("first", first, (B,)), _ints("path", path, (B, n)), n,
                                            _ints("count", count, (B,)), stream))


# ------------------------------------------------------------------------ device memory holder
class Session:
    """Owns the context and the torch tensors (weights, workspaces, state) it points into.
    Allocation and pointer marshalling only."""

    def __init__(self, max_batch: int, k_max: int, max_src: int, max_tgt: int, device="cuda:0", fill: int = 0):
        """fill: byte the state and workspace buffers hold before they are bound (the header lets the
        caller pass any buffer: 0xFF makes every untouched bf16 / fp32 word a NaN)."""
        import torch
        self.torch = torch
        self.device = torch.device(device)
        self.ctx = specdec_create(max_batch, k_max, max_src, max_tgt)
        self.limits = (max_batch, k_max, max_src, max_tgt)
        self._keep = []
        self.fill = int(fill)
        self.state = torch.full((specdec_state_bytes(self.ctx),), self.fill, dtype=torch.uint8, device=self.device)
        specdec_bind_state(self.ctx, self.state)
        self.desc: Dict[int, object] = {}

    def upload_weights(self, bits: Dict[str, np.ndarray]):
        """name -> uint16 bf16 bit patterns (ABI order) -> list of device bf16 tensors."""
        torch = self.torch
        out = []
        for v in bits.values():
            t = torch.from_numpy(np.ascontiguousarray(v).view(np.int16)).to(self.device).view(torch.bfloat16)
            out.append(t)
        return out

    def bind_model(self, role: int, desc, weights: Sequence):
        torch = self.torch
        ws = torch.full((specdec_workspace_bytes(self.ctx, desc),), self.fill, dtype=torch.uint8, device=self.device)
        specdec_bind_model(self.ctx, role, desc, weights, ws)
        self._keep.append((weights, ws))
        self.desc[role] = desc
        return ws

    def i32(self, a):
        return self.torch.as_tensor(np.ascontiguousarray(a, dtype=np.int32), device=self.device)

    def bf16(self, a_f32: np.ndarray):
        """fp32 array -> device bf16 tensor (round to nearest even)."""
        return self.torch.from_numpy(np.ascontiguousarray(a_f32, dtype=np.float32)).to(self.device).to(self.torch.bfloat16).contiguous()

    def close(self):
        if self.ctx is not None:
            self.torch.cuda.synchronize(self.device)
            specdec_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
