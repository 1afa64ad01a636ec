"""Operators that write refuse tensors in which the same place belongs to two rows, on the host and before anything is launched."""
import ctypes as C

import pytest

from paper_2203_16487_amd import binding as sd

BAD = sd.SPECDEC_ERR_INVALID_ARG
K, V, P = C.c_void_p(1 << 20), C.c_void_p(1 << 30), C.c_void_p(4096)     # (never dereferenced: every call below is refused)


@pytest.fixture
def ctx():
    c = sd.specdec_create(1, 1, 1, 1)
    yield c
    sd.specdec_destroy(c)


def slabs(**change):
    d = sd.specdec_cache_desc(2, 4, 100, 128, 4 * 51200, 51200, 12800, 128)      # four sequences
    for name, value in change.items():
        setattr(d, name, value)
    return d


@pytest.mark.parametrize("change,k,v", [
    (dict(layer_stride=0), K, V), (dict(seq_stride=0), K, V), (dict(head_stride=0), K, V), (dict(seq_stride=51184), K, V), (dict(layer_stride=3 * 51200), K, V),
    (dict(head_stride=128), K, V), (dict(row_stride=512, head_stride=112), K, V), (dict(), K, K), (dict(), K, C.c_void_p(K.value + 128)),
    (dict(), C.c_void_p(K.value + 128), K), (dict(seq_stride=2 * 51200, layer_stride=8 * 51200), K, C.c_void_p(K.value + 51184))])
def test_moves_in_place(ctx, change, k, v):
    d = slabs(**change)
    for kv in ((k, v), (k, None)) if change and "seq_stride" not in change else ((k, v),):
        assert sd.lib().specdec_fork_cache(ctx, C.byref(d), *kv, 4, P, 4, P, None) == BAD
        assert b"overlap" in sd.lib().specdec_last_error(ctx)
        assert sd.lib().specdec_compact_cache(ctx, C.byref(d), *kv, 4, P, P, 3, P, None) == BAD
        assert b"overlap" in sd.lib().specdec_last_error(ctx)
    assert sd.lib().specdec_fork_cache(ctx, C.byref(d), k, v, 2, P, 4, P, None) == BAD       # (sources count, too)


@pytest.mark.parametrize("stride,fine", [((2048, 512, 64), True), ((512, 1024, 64), True), ((64, 128, 512), True), ((2048, 448, 64), False), ((2048, 64, 64), False), ((1984, 512, 64), False),
                                         ((64, 2048, 512), False), ((0, 512, 64), False), ((2048, 512, 0), False)])
def test_attention_output(ctx, stride, fine):
    """Two sequences of four rows of eight heads of 64."""
    s = lambda x: (C.c_int64 * 3)(*x)
    d = sd.specdec_tree_attn_desc(sd.SPECDEC_BF16, 2, 4, 8, 2, 64, 100, 0.125, s((0, 0, 0)), s((0, 0, 0)), s((0, 0, 0)), s(stride))
    n = C.c_size_t()
    assert sd.lib().specdec_tree_attention_bytes(ctx, C.byref(d), C.byref(n)) == (sd.SPECDEC_OK if fine else BAD)
    if not fine:
        assert b"overlap" in sd.lib().specdec_last_error(ctx)
