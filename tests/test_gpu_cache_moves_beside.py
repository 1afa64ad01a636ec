"""Moves in caches whose keys and values lie among each other: per layer, per sequence, per row, and rows of all heads beside those of something else."""
import numpy as np
import pytest
import torch

import operators_oracle as oo
from paper_2203_16487_amd import binding as sd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("order", [(0, 1, 2, 3, 4), (1, 0, 2, 3, 4), (1, 2, 0, 3, 4), (1, 2, 4, 0, 3), (2, 1, 4, 3, 0), (4, 3, 2, 1, 0)])
def test_keys_beside_values(order):
    """Dimensions k / v / other, layers, sequences, heads, rows in this order of memory."""
    ctx = sd.specdec_create(1, 1, 1, 1)
    sizes, values = (3, 2, 5, 3, 21), 24
    rng = np.random.default_rng(sum(i * 5 ** n for n, i in enumerate(order)))
    arena = torch.tensor(rng.integers(-2 ** 15, 2 ** 15, size=[sizes[i] for i in order] + [values], dtype=np.int16), device="cuda")
    both = arena.permute([order.index(i) for i in range(5)] + [5])
    k, v, other = both[0], both[1], both[2]
    src, length = [4, 0, 0, 3, 9], [20, 3, 21, 7, 21]
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    want, rest = [oo.fork(t.cpu().numpy(), src, length) for t in (k, v)], other.clone()
    sd.specdec_fork_cache(ctx, sd.cache_desc(k, v), k, v, i32(src), i32(length))
    assert np.array_equal(k.cpu().numpy(), want[0]) and np.array_equal(v.cpu().numpy(), want[1]) and torch.equal(other, rest)
    first, path, count = [0, 7, 11, 2, 5], rng.integers(0, 10, size=(5, 4)), [4, 3, 0, 1, 4]
    want = [oo.compact(t, first, path, count) for t in want]
    sd.specdec_compact_cache(ctx, sd.cache_desc(k, v), k, v, i32(first), i32(path), i32(count))
    assert np.array_equal(k.cpu().numpy(), want[0]) and np.array_equal(v.cpu().numpy(), want[1]) and torch.equal(other, rest)
    with pytest.raises(sd.SpecDecError, match="overlap"):
        sd.specdec_fork_cache(ctx, sd.cache_desc(k, k), k, k, i32(src), i32(length))
    one = k[:, :1].expand(-1, 5, -1, -1, -1)
    with pytest.raises(sd.SpecDecError, match="overlap"):
        sd.specdec_compact_cache(ctx, sd.cache_desc(one), one, None, i32(first), i32(path), i32(count))
    sd.specdec_destroy(ctx)
