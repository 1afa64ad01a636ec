"""Forked sequences and compacted paths against the same moves one by one, bit for bit."""
import numpy as np
import pytest
import torch

import operators_oracle as oo
from paper_2203_16487_amd import binding as sd

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = sd.specdec_create(1, 1, 1, 1)
    yield c
    sd.specdec_destroy(c)


def caches(rng, layers, B, heads, cap, values, layout):
    """k and v [layers, B, heads, cap, values] of random 16-bit patterns, NaN among them."""
    out = []
    for _ in range(2):
        shape = (layers, B, heads, cap, values) if layout == "heads" else (layers, B, cap, heads, values)
        if layout == "padded":
            shape = (layers, B + 1, cap + 3, heads + 1, values + 8)
        t = torch.tensor(rng.integers(-2 ** 15, 2 ** 15, size=shape, dtype=np.int16), device="cuda")
        if layout == "rows":
            t = t.transpose(2, 3)
        if layout == "padded":
            t = t[:, 1:, 2:cap + 2, 1:, :values].transpose(2, 3)
        out.append(t)
    return out


FORKS = [  # layers, B, heads, cap, values, layout
    (1, 1, 1, 1, 8, "heads"), (1, 2, 1, 1, 64, "heads"), (2, 3, 2, 33, 64, "rows"), (6, 32, 8, 160, 64, "heads"), (1, 7, 3, 257, 128, "padded"),
    (2, 129, 2, 70, 64, "rows"), (1, 4096, 1, 9, 64, "heads"), (1, 2, 1, 5000, 128, "rows"), (1, 5, 2, 40, 24, "heads"), (3, 1000, 1, 3, 8, "padded"),
]


@pytest.mark.parametrize("layers,B,heads,cap,values,layout", FORKS)
@pytest.mark.parametrize("kind", ["permutation", "groups", "any", "out of range", "grown"])
def test_fork(ctx, layers, B, heads, cap, values, layout, kind):
    rng = np.random.default_rng([layers, B, cap])
    k, v = caches(rng, layers, B, heads, cap, values, layout)
    n_src = B
    if kind == "permutation":
        src = rng.permutation(B)
    elif kind == "groups":
        src = np.arange(B) // 4 * 4
    elif kind == "any":
        src = rng.integers(0, B, size=B)
    elif kind == "out of range":
        src = rng.integers(-2, B + 3, size=B)
        src[0] = -2 ** 31
    else:                    # a few sequences become all
        n_src = max(1, B // 3)
        src = rng.integers(0, n_src, size=B)
    length = rng.integers(0, cap + 1, size=n_src)
    length[0] = cap
    if kind == "out of range":
        length[-1], length[n_src // 2] = -5, cap + 1000
    want = [oo.fork(t.cpu().numpy(), src, length) for t in (k, v)]
    desc = sd.cache_desc(k, v)
    args = torch.tensor(src, dtype=torch.int32, device="cuda"), torch.tensor(length, dtype=torch.int32, device="cuda")
    only = k.clone(memory_format=torch.preserve_format)
    sd.specdec_fork_cache(ctx, desc, k, v, *args)
    assert np.array_equal(k.cpu().numpy(), want[0]) and np.array_equal(v.cpu().numpy(), want[1])
    if only.stride() == k.stride():
        sd.specdec_fork_cache(ctx, desc, only, None, *args)
        assert np.array_equal(only.cpu().numpy(), want[0])


COMPACTS = [  # layers, B, heads, cap, values, layout, n
    (1, 1, 1, 1, 8, "heads", 1), (6, 1, 8, 160, 64, "heads", 6), (2, 3, 2, 70, 64, "rows", 64), (6, 128, 16, 96, 64, "heads", 7), (1, 5, 3, 90, 128, "padded", 33),
    (2, 2, 2, 80, 256, "rows", 64), (1, 300, 1, 12, 24, "heads", 12), (3, 4, 5, 40, 8, "padded", 2),
]


@pytest.mark.parametrize("layers,B,heads,cap,values,layout,n", COMPACTS)
@pytest.mark.parametrize("kind", ["path", "any", "out of range"])
def test_compact(ctx, layers, B, heads, cap, values, layout, n, kind):
    rng = np.random.default_rng([layers, B, cap, n])
    k, v = caches(rng, layers, B, heads, cap, values, layout)
    room = min(cap, 64)
    first = rng.integers(0, max(cap - room, 0) + 1, size=B)
    if kind == "path":
        path = np.stack([np.concatenate([[0], np.sort(rng.permutation(np.arange(1, room))[:n - 1]), np.zeros(n, int)])[:n] for _ in range(B)])
        count = rng.integers(0, min(n, room) + 1, size=B)
    elif kind == "any":              # in any order, and the same row twice
        path = rng.integers(0, room, size=(B, n))
        count = rng.integers(0, min(n, room) + 1, size=B)
    else:
        path = rng.integers(-3, cap + 3, size=(B, n))
        path[0, 0] = 2 ** 31 - 1
        first = rng.integers(-4, cap + 4, size=B)
        count = rng.integers(-2, n + 5, size=B)
    want = [oo.compact(t.cpu().numpy(), first, path, count) for t in (k, v)]
    desc = sd.cache_desc(k, v)
    args = [torch.tensor(a, dtype=torch.int32, device="cuda") for a in (first, path, count)]
    only = k.clone(memory_format=torch.preserve_format)
    sd.specdec_compact_cache(ctx, desc, k, v, *args)
    assert np.array_equal(k.cpu().numpy(), want[0]) and np.array_equal(v.cpu().numpy(), want[1])
    if only.stride() == k.stride():
        sd.specdec_compact_cache(ctx, desc, only, None, *args)
        assert np.array_equal(only.cpu().numpy(), want[0])


def test_offsets_beyond_32_bits(ctx):
    arena = torch.zeros((1 << 31) + (1 << 20), dtype=torch.int16, device="cuda")
    k = arena.as_strided((1, 2, 1, 40, 64), (1 << 31, (1 << 31) + 8192, 64, 64, 1))     # the second sequence 4 GiB behind the first
    k.copy_(torch.randint(-999, 999, k.shape, dtype=torch.int16, device="cuda"))
    old = k.cpu().numpy()
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    sd.specdec_fork_cache(ctx, sd.cache_desc(k), k, None, i32([1, 0]), i32([30, 40]))
    want = oo.fork(old, [1, 0], [30, 40])
    assert np.array_equal(k.cpu().numpy(), want)
    sd.specdec_compact_cache(ctx, sd.cache_desc(k), k, None, i32([0, 5]), i32([[0, 9, 4], [0, 30, 2]]), i32([2, 3]))
    assert np.array_equal(k.cpu().numpy(), oo.compact(want, [0, 5], np.array([[0, 9, 4], [0, 30, 2]]), [2, 3]))
