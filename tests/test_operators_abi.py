"""The operators on a caller's tensors refuse what they cannot do, on the host and before anything is launched."""
import ctypes as C

import pytest
import torch

from paper_2203_16487_amd import binding as sd

BAD, LARGE = sd.SPECDEC_ERR_INVALID_ARG, sd.SPECDEC_ERR_TOO_LARGE
P = C.c_void_p(4096)     # (never dereferenced: every call below is refused)


@pytest.fixture
def ctx():
    c = sd.specdec_create(1, 1, 1, 1)
    yield c
    sd.specdec_destroy(c)


def attn_desc(**change):
    d = sd.specdec_tree_attn_desc(sd.SPECDEC_BF16, 2, 4, 8, 2, 64, 100, 0.125, (C.c_int64 * 3)(2048, 512, 64), (C.c_int64 * 3)(12800, 64, 6400),
                                  (C.c_int64 * 3)(12800, 64, 6400), (C.c_int64 * 3)(2048, 512, 64))
    for name, value in change.items():
        setattr(d, name, (C.c_int64 * 3)(*value) if isinstance(value, tuple) else value)
    return d


@pytest.mark.parametrize("change", [dict(dtype=0), dict(dtype=3), dict(batch=0), dict(batch=65536), dict(rows=0), dict(rows=65), dict(n_heads=0), dict(n_heads=7),
                                    dict(n_heads=1026, n_kv_heads=2), dict(n_kv_heads=0), dict(head_dim=96), dict(head_dim=0), dict(capacity=0),
                                    dict(scale=float("nan")), dict(scale=float("inf")), dict(q_stride=(2048, 512, 60)), dict(k_stride=(-8, 64, 6400)),
                                    dict(v_stride=(1 << 50, 64, 6400)), dict(out_stride=(2048, 0, 64)), dict(out_stride=(2048, 512, 32))])
def test_tree_attention_descriptions(ctx, change):
    d, n = attn_desc(**change), C.c_size_t()
    assert sd.lib().specdec_tree_attention_bytes(ctx, C.byref(d), C.byref(n)) == BAD
    assert len(sd.lib().specdec_last_error(ctx)) > 0
    assert sd.lib().specdec_tree_attention(ctx, C.byref(d), P, P, P, P, None, None, P, P, 1 << 40, None) == BAD


def test_tree_attention_pointers(ctx):
    L, d, n = sd.lib(), attn_desc(), C.c_size_t()
    assert L.specdec_tree_attention_bytes(ctx, C.byref(d), C.byref(n)) == sd.SPECDEC_OK
    assert L.specdec_tree_attention_bytes(ctx, C.byref(d), None) == BAD and L.specdec_tree_attention_bytes(ctx, None, C.byref(n)) == BAD
    assert L.specdec_tree_attention_bytes(None, C.byref(d), C.byref(n)) == BAD
    good = [P, P, P, P, None, None, P]
    for i in (0, 1, 2, 3, 6):
        args = list(good)
        args[i] = None
        assert L.specdec_tree_attention(ctx, C.byref(d), *args, P, 1 << 40, None) == BAD
        if i != 3:
            args[i] = C.c_void_p(4104)
            assert L.specdec_tree_attention(ctx, C.byref(d), *args, P, 1 << 40, None) == BAD
    big = attn_desc(capacity=1 << 20)
    assert L.specdec_tree_attention_bytes(ctx, C.byref(big), C.byref(n)) == sd.SPECDEC_OK
    if n.value:
        assert L.specdec_tree_attention(ctx, C.byref(big), *good, None, 1 << 40, None) == BAD
        assert L.specdec_tree_attention(ctx, C.byref(big), *good, C.c_void_p(4112), 1 << 40, None) == BAD
        assert L.specdec_tree_attention(ctx, C.byref(big), *good, P, n.value - 1, None) == LARGE
    assert L.specdec_tree_attention(None, C.byref(d), *good, P, 1 << 40, None) == BAD


def test_tree_visible(ctx):
    L = sd.lib()
    for args in ((None, 1, 3, P), (P, 0, 3, P), (P, 1, -1, P), (P, 1, 64, P), (P, 1, 3, None)):
        assert L.specdec_tree_visible(ctx, *args, None) == BAD
    assert L.specdec_tree_visible(None, P, 1, 3, P, None) == BAD


def test_sample(ctx):
    L = sd.lib()
    def call(logits=P, dtype=0, rows=1, vocab=10, stride=10, u=P, token=P, c=ctx):
        return L.specdec_sample(c, logits, dtype, rows, vocab, stride, None, None, None, None, u, token, None, None)
    for change in (dict(logits=None), dict(u=None), dict(token=None), dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(vocab=0), dict(vocab=(1 << 24) + 1),
                   dict(stride=-1), dict(stride=1 << 50), dict(logits=C.c_void_p(4098)), dict(logits=C.c_void_p(4097), dtype=1), dict(c=None)):
        assert call(**change) == BAD, change
    assert call(rows=0) == sd.SPECDEC_OK          # nothing to do, nothing launched


def slabs(**change):
    d = sd.specdec_cache_desc(2, 4, 100, 128, 4 * 51200, 51200, 12800, 128)
    for name, value in change.items():
        setattr(d, name, value)
    return d


@pytest.mark.parametrize("change", [dict(layers=0), dict(heads=0), dict(layers=200, heads=200), dict(capacity=0), dict(row_bytes=0), dict(row_bytes=24),
                                    dict(row_bytes=65552, row_stride=65552), dict(layer_stride=8), dict(seq_stride=-16), dict(head_stride=1 << 50),
                                    dict(row_stride=112)])
def test_cache_descriptions(ctx, change):
    d = slabs(**change)
    assert sd.lib().specdec_fork_cache(ctx, C.byref(d), P, P, 2, P, 2, P, None) == BAD
    assert sd.lib().specdec_compact_cache(ctx, C.byref(d), P, P, 2, P, P, 3, P, None) == BAD


def test_cache_moves(ctx):
    L, d, wide = sd.lib(), slabs(), slabs(row_bytes=528, row_stride=528)
    odd = C.c_void_p(4104)
    for args in ((None, P, 2, P, 2, P), (odd, P, 2, P, 2, P), (P, odd, 2, P, 2, P), (P, P, 0, P, 2, P), (P, P, 4097, P, 2, P), (P, P, 2, None, 2, P),
                 (P, P, 2, P, 0, P), (P, P, 2, P, 4097, P), (P, P, 2, P, 2, None)):
        assert L.specdec_fork_cache(ctx, C.byref(d), *args, None) == BAD, args
    vast = slabs(capacity=1 << 26, layer_stride=0)
    assert L.specdec_fork_cache(ctx, C.byref(vast), P, P, 2, P, 2, P, None) == LARGE
    assert L.specdec_fork_cache(ctx, None, P, P, 2, P, 2, P, None) == BAD and L.specdec_fork_cache(None, C.byref(d), P, P, 2, P, 2, P, None) == BAD
    for args in ((None, P, 2, P, P, 3, P), (P, odd, 2, P, P, 3, P), (P, P, 0, P, P, 3, P), (P, P, 65536, P, P, 3, P), (P, P, 2, None, P, 3, P), (P, P, 2, P, None, 3, P),
                 (P, P, 2, P, P, 0, P), (P, P, 2, P, P, 65, P), (P, P, 2, P, P, 3, None)):
        assert L.specdec_compact_cache(ctx, C.byref(d), *args, None) == BAD, args
    assert L.specdec_compact_cache(ctx, C.byref(wide), P, P, 2, P, P, 3, P, None) == BAD


def test_binding_refuses_tensors(ctx):
    """What a pointer cannot say: tensors on the host, of other shapes, types and strides."""
    q, k = torch.zeros((2, 3, 4, 64), dtype=torch.bfloat16), torch.zeros((2, 2, 50, 64), dtype=torch.bfloat16)
    for bad in ((q, k, k[:, :1], q), (q, k, k.half(), q), (q.float(), k.float(), k.float(), q.float()), (q, k[..., ::2], k[..., ::2], q), (q, k, k, q[:1]),
                (q[:1], k, k, q)):
        with pytest.raises(sd.SpecDecError) as e:
            sd.tree_attn_desc(*bad, 0.1)
        assert e.value.code == BAD
    desc = sd.tree_attn_desc(q, k, k, q.clone(), 0.1)
    assert list(desc.k_stride) == [6400, 64, 3200] and list(desc.q_stride) == [768, 256, 64]
    one = torch.zeros(2, dtype=torch.int32)
    calls = [lambda: sd.specdec_tree_attention(ctx, desc, q, k, k, one, None, None, q, None), lambda: sd.specdec_tree_visible(ctx, one.view(1, 2), one.long()),
             lambda: sd.specdec_sample(ctx, q.view(2, -1), None, None, None, None, one.float(), one),
             lambda: sd.specdec_fork_cache(ctx, sd.cache_desc(k[None]), k[None], None, one, one),
             lambda: sd.specdec_compact_cache(ctx, sd.cache_desc(k[None]), k[None], None, one, one.view(2, 1), one)]
    for call in calls:                                # (on the host)
        with pytest.raises(sd.SpecDecError) as e:
            call()
        assert e.value.code == BAD
    for bad in (one.long(), one.view(2, 1), torch.zeros(4, dtype=torch.int32)[::2]):
        with pytest.raises(sd.SpecDecError):
            sd._ints("x", bad, (2,))
    with pytest.raises(sd.SpecDecError):
        sd.cache_desc(k[None], k.transpose(1, 2).contiguous().transpose(1, 2)[None])
    with pytest.raises(sd.SpecDecError):
        sd._slabs(sd.cache_desc(k[None]), k[None, :1], None, 1)


def test_call_order_without_a_model(ctx):
    L = sd.lib()
    assert L.specdec_verify_tree(ctx, P, P, 1, P, None) == sd.SPECDEC_ERR_BAD_STATE
    assert L.specdec_commit_tree(ctx, P, None, None, None, None) == sd.SPECDEC_ERR_BAD_STATE
    assert L.specdec_fork(ctx, P, 1, None) == sd.SPECDEC_ERR_BAD_STATE
    for call in (lambda: L.specdec_verify_tree(None, P, P, 1, P, None), lambda: L.specdec_commit_tree(None, P, None, None, None, None),
                 lambda: L.specdec_fork(None, P, 1, None)):
        assert call() == BAD
