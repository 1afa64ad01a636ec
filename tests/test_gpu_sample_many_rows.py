"""Drawn tokens of more rows than the GPU has compute units, on both sides of the row sizes at which another kernel takes them: against the
definition for a few dozen rows that repeat, and against the same rows in calls of few."""
import numpy as np
import pytest
import torch

import operators_oracle as oo
from paper_2203_16487_amd import binding as sd

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
INF = float("inf")


@pytest.fixture(scope="module")
def ctx():
    c = sd.specdec_create(1, 1, 1, 1)
    yield c
    sd.specdec_destroy(c)


def draw(ctx, logits, cols):
    rows = logits.shape[0]
    token = torch.full((rows,), -9, dtype=torch.int32, device="cuda")
    logprob = torch.full((rows,), 9.0, dtype=torch.float32, device="cuda")
    sd.specdec_sample(ctx, logits, *cols, token, logprob)
    return token, logprob


# 16-byte pieces of a row: at most 2048 (with the one that an unaligned row needs), at most 9216, more
SIZES = [("f32", 8188), ("f32", 8189), ("f32", 20001), ("f32", 32768), ("f32", 36860), ("f32", 36861),
         ("bf16", 16376), ("bf16", 16377), ("bf16", 32003), ("bf16", 73720), ("bf16", 73721),
         ("f16", 16376), ("f16", 16377), ("f16", 50000), ("f16", 73720), ("f16", 73721)]
# temperature, top-k, top-p, min-p
SETTINGS = [(1.0, 0, 1.0, 0.0), (0.7, 0, 1.0, 0.0), (5.0, 0, 1.0, 0.0), (1.0, 0, 0.5, 0.0), (0.8, 0, 0.9, 0.0), (1.0, 0, 0.999, 0.0), (3.0, 0, 0.9, 0.0),
            (1.0, 40, 1.0, 0.0), (1.0, 192, 1.0, 0.0), (1.0, 193, 1.0, 0.0), (1.0, 250, 0.9, 0.0), (2.0, 5000, 0.95, 0.0), (1.0, 0, 1.0, 0.02), (2.0, 0, 0.9, 0.01),
            (0.0, 0, 1.0, 0.0), (2.0, 300, 0.99, 0.001)]


def rows_of(V, gen):
    """Peaked, flat and coarse rows (many equal logits), some tokens never drawn."""
    x = 2.0 * torch.randn((len(SETTINGS), V), generator=gen, device="cuda")
    x[::2] += torch.randn((len(SETTINGS), V), generator=gen, device="cuda")[::2].clamp_(min=0).pow_(3) * 0.3
    x[3::4] = (0.4 * x[3::4]).round()
    x[:, [1, V - 1]] = -INF
    return x


@pytest.mark.parametrize("dtype,V", SIZES)
def test_against_the_definition(ctx, dtype, V):
    D, rows = len(SETTINGS), 261
    rng = np.random.default_rng(V)
    x = rows_of(V, torch.Generator(device="cuda").manual_seed(V)).to(DT[dtype])
    u = rng.random(D).astype(np.float32)
    which = np.arange(rows) % D
    cols = [np.array([s[i] for s in SETTINGS], dtype=np.int32 if i == 1 else np.float32)[which] for i in range(4)] + [u[which]]
    cols = [torch.tensor(c, device="cuda") for c in cols]
    f64 = x.double().cpu().numpy()
    want = [oo.sample_row(f64[r], float(np.float32(s[0])), s[1], float(np.float32(s[2])), float(np.float32(s[3])), float(u[r])) for r, s in enumerate(SETTINGS)]
    at = torch.tensor(which, device="cuda")
    for shift, pitch in ((0, V), (1, V + 3), (2, V + 1)):        # rows at any place
        logits = torch.zeros(rows * pitch + 8, dtype=DT[dtype], device="cuda").as_strided((rows, V), (pitch, 1), shift)
        logits.copy_(x[at])
        token, logprob = draw(ctx, logits, cols)
        got, lp = token.tolist(), logprob.double().tolist()
        for r in range(rows):
            t, l = want[r % D]
            assert got[r] == t, (r, got[r], t, SETTINGS[r % D])
            # rounded to fp32 once; the total is off by at most half a unit of 2^-38 a token
            assert lp[r] == l or abs(lp[r] - l) <= 2.0 ** -24 * abs(l) + 2.0 ** -38 * V + 1e-12, (r, lp[r], l)
        few = [draw(ctx, logits[a:a + 87], [c[a:a + 87] for c in cols]) for a in (0, 87, 174)]     # (sums are whole numbers: the same bits)
        assert torch.equal(token, torch.cat([f[0] for f in few])) and torch.equal(logprob, torch.cat([f[1] for f in few]))


@pytest.mark.parametrize("dtype,V", [("f32", 8188), ("f32", 8189), ("f32", 36860), ("bf16", 73720), ("f16", 16377), ("f16", 73721)])
@pytest.mark.parametrize("rows", [256, 257])
def test_every_place_of_a_row(ctx, dtype, V, rows):
    """Random numbers that lead to all parts of one row: the token is where the running sum of the definition's weights passes."""
    x = (0.5 * torch.randn(V, generator=torch.Generator(device="cuda").manual_seed(7), device="cuda")).to(DT[dtype])
    f64 = x.double().cpu().numpy()
    w = np.rint(np.exp(f64 - f64.max()) * oo.WEIGHT_ONE).astype(np.int64)
    sums = np.cumsum(w)
    for part in range(4):
        u = ((np.arange(rows) + 0.25 * part) / rows).astype(np.float32)
        target = np.minimum((u.astype(np.float64) * float(sums[-1])).astype(np.int64), sums[-1] - 1)
        want = np.searchsorted(sums, target, side="right")
        token, _ = draw(ctx, x.expand(rows, V), [None, None, None, None, torch.tensor(u, device="cuda")])
        # (the definition's weights are NumPy's rounded exp, the kernel's off by less than one unit: a sum by less than V, where the number falls that near)
        near = np.minimum(np.abs(target - sums[np.maximum(want - 1, 0)]), np.abs(sums[want] - target)) <= V
        differ = token.cpu().numpy() != want
        assert not np.any(differ & ~near), (part, np.flatnonzero(differ & ~near)[:5])


@pytest.mark.parametrize("rows", [(1 << 21) + 1, (1 << 23) + 5])
def test_more_rows_than_a_launch_takes(ctx, rows):
    """Short rows by the million: greedy ones against arg-max, drawn ones against the same rows in smaller calls."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((rows, 5), generator=gen, device="cuda").to(torch.bfloat16)[:, :3]
    u = torch.rand(rows, generator=gen, device="cuda")
    t = torch.rand(rows, generator=gen, device="cuda") + 0.5
    k = torch.randint(0, 4, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    token, _ = draw(ctx, x, [torch.zeros_like(t), None, None, None, u])
    greatest = x.float().amax(1, keepdim=True)
    assert torch.equal(token.long(), torch.where(x.float() == greatest, torch.arange(3, device="cuda"), 3).amin(1))
    cols = [t, k, torch.full_like(t, 0.9), torch.full_like(t, 0.05), u]
    token, logprob = draw(ctx, x, cols)
    for a in (0, (1 << 21) - 1000, (1 << 22) - 10, rows - 1500):
        a = min(a, rows - 1500)
        some, lp = draw(ctx, x[a:a + 1500], [c[a:a + 1500] for c in cols])
        assert torch.equal(token[a:a + 1500], some) and torch.equal(logprob[a:a + 1500], lp), a
