"""Drawn tokens against the definition (whole-number weights and sums), every setting and what rows can hold."""
import numpy as np
import pytest
import torch

import operators_oracle as oo
from paper_2203_16487_amd import binding as sd

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def ctx():
    c = sd.specdec_create(1, 1, 1, 1)
    yield c
    sd.specdec_destroy(c)


def settings(rng, rows, V):
    """Columns of settings, ordinary and odd ones."""
    pick = lambda values: np.array([values[int(rng.integers(len(values)))] for _ in range(rows)])
    return (pick([1.0, 0.7, 0.2, 1.5, 0.0, 30.0]).astype(np.float32), pick([0, 1, 2, 40, V - 1, V, V + 5, -3, max(V // 2, 1)]).astype(np.int32),
            pick([1.0, 0.9, 0.5, 0.05, 0.999, 0.0, 2.0]).astype(np.float32), pick([0.0, 0.0, 0.02, 0.3, 1.0]).astype(np.float32),
            pick([0.0, float(np.float32(1 - 2.0 ** -24)), *rng.random(6)]).astype(np.float32))


def check(ctx, logits, temperature, top_k, top_p, min_p, u):
    rows, V = logits.shape
    cols = [None if c is None else torch.tensor(c, device="cuda") for c in (temperature, top_k, top_p, min_p, u)]
    token = torch.full((rows,), -9, dtype=torch.int32, device="cuda")
    logprob = torch.full((rows,), 9.0, dtype=torch.float32, device="cuda")
    sd.specdec_sample(ctx, logits, *cols, token, logprob)
    bare = torch.full((rows,), -9, dtype=torch.int32, device="cuda")
    sd.specdec_sample(ctx, logits, *cols, bare)
    got, lp = token.tolist(), logprob.double().tolist()
    assert bare.tolist() == got
    x = logits.double().cpu().numpy()
    for r in range(rows):
        one = [d if c is None else c[r] for c, d in ((temperature, 1.0), (top_k, 0), (top_p, 1.0), (min_p, 0.0), (u, 0.0))]
        one = [int(one[1]) if i == 1 else float(c) for i, c in enumerate(one)]
        want, want_lp = oo.sample_row(x[r], *one)
        assert got[r] == want, (r, got[r], want, one)
        # rounded to fp32 once; the total is off by at most half a unit a token
        assert lp[r] == want_lp or abs(lp[r] - want_lp) <= 2.0 ** -24 * abs(want_lp) + 2.0 ** -38 * V + 1e-12, (r, lp[r], want_lp)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,V", [(7, 1), (7, 2), (9, 5), (5, 63), (5, 64), (5, 65), (9, 1000), (5, 1023), (5, 1025), (24, 4097), (12, 8191), (40, 32003),
                                    (8, 32768), (3, 32769), (4, 65537), (4, 131072), (2, 262147)])
def test_against_the_definition(ctx, dtype, rows, V):
    rng = np.random.default_rng([rows, V])
    gen = torch.Generator(device="cuda").manual_seed(V)
    x = 2.5 * torch.randn((rows, V + 3), generator=gen, device="cuda")
    x += torch.randn((rows, V + 3), generator=gen, device="cuda").clamp_(min=0).pow_(3) * 0.3
    for shift, pitch in ((0, V), (1, V + 3), (2, V + 1)):        # rows at any place
        flat = torch.zeros(rows * pitch + 8, dtype=DT[dtype], device="cuda")
        logits = flat.as_strided((rows, V), (pitch, 1), shift)
        logits.copy_(x[:, :V])
        check(ctx, logits, *settings(rng, rows, V))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [3, 70, 5000, 40000])
def test_rows_of_all_kinds(ctx, dtype, V):
    rng = np.random.default_rng(V)
    gen = torch.Generator(device="cuda").manual_seed(V)
    lowest = torch.finfo(DT[dtype]).min
    def filled(v):
        return torch.full((V,), v)
    base = torch.randn(V, generator=gen, device="cuda").cpu() * 3
    some = torch.rand(V, generator=gen, device="cuda").cpu() < 0.5
    some[0], some[-1] = False, True
    kinds = [filled(0.0), filled(-INF), filled(NAN), filled(lowest), filled(INF), filled(-0.0).masked_fill(some, 0.0), base.masked_fill(some, -INF),
             base.masked_fill(some, NAN), base.masked_fill(some, lowest), base.masked_fill(some, INF), base.round(), (base * 0.3).round(),
             filled(-INF).index_fill(0, torch.tensor([V - 1]), -5.0), filled(lowest).index_fill(0, torch.tensor([1]), -torch.finfo(DT[dtype]).max * -1.0),
             base * 1e4, base.sort().values, base.sort(descending=True).values, base + 1000.0]
    for _ in range(3):
        check(ctx, torch.stack(kinds).to(DT[dtype]).cuda(), *settings(rng, len(kinds), V))


@pytest.mark.parametrize("V", [4, 500, 33000])
def test_settings_out_of_range(ctx, V):
    gen = torch.Generator(device="cuda").manual_seed(V)
    odd = [(NAN, 0, 1.0, 0.0, 0.3), (-1.0, 3, 0.5, 0.0, 0.3), (INF, 0, 1.0, 0.0, 0.7), (1e-45, 0, 1.0, 0.0, 0.7), (1e-3, 0, 0.9, 0.0, 0.5),
           (1.0, -2 ** 31, 0.9, 0.0, 0.4), (1.0, 2 ** 31 - 1, 0.9, 0.0, 0.4), (1.0, 0, NAN, 0.0, 0.4), (1.0, 0, -1.0, 0.0, 0.9), (1.0, 0, INF, 0.0, 0.9),
           (1.0, 0, 1e-30, 0.0, 0.9), (1.0, 0, 1.0, NAN, 0.9), (1.0, 0, 1.0, -1.0, 0.9), (1.0, 0, 1.0, 1.0, 0.9), (1.0, 0, 1.0, 7.0, 0.9), (1.0, 0, 1.0, INF, 0.9),
           (1.0, 0, 1.0, 0.0, 1.0), (1.0, 0, 1.0, 0.0, -0.5), (1.0, 0, 1.0, 0.0, 5.0), (1.0, 0, 1.0, 0.0, NAN), (1.0, 0, 0.5, 0.0, INF)]
    logits = torch.randn((len(odd), V), generator=gen, device="cuda").round()
    cols = [np.array([o[i] for o in odd], dtype=np.int32 if i == 1 else np.float32) for i in range(5)]
    check(ctx, logits, *cols)
    check(ctx, logits, None, None, None, None, cols[4])
    check(ctx, logits, None, cols[1], None, None, cols[4])


def test_frequencies(ctx):
    """Draws with evenly spread numbers: token i as often as its share says, off by less than one place at either end of its stretch."""
    N = 4096
    x = torch.tensor([0.0, 1.0, -1.0, 2.0, -INF, 0.5], device="cuda")
    token = torch.zeros(N, dtype=torch.int32, device="cuda")
    u = ((torch.arange(N, device="cuda") + 0.5) / N).float()
    sd.specdec_sample(ctx, x.expand(N, 6), None, None, None, None, u, token)
    p = torch.softmax(x.double(), 0).cpu()
    count = torch.bincount(token.long().cpu(), minlength=6).double()
    assert bool((count - N * p).abs().max() <= 1.0) and count[4] == 0


def test_captured(ctx):
    gen = torch.Generator(device="cuda").manual_seed(1)
    rows, V = 6, 9000
    logits, u = torch.randn((rows, V), generator=gen, device="cuda"), torch.rand(rows, generator=gen, device="cuda")
    top_p = torch.full((rows,), 0.8, device="cuda")
    token, want = (torch.zeros(rows, dtype=torch.int32, device="cuda") for _ in range(2))
    sd.specdec_sample(ctx, logits, None, None, top_p, None, u, token)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sd.specdec_sample(ctx, logits, None, None, top_p, None, u, token)
    for _ in range(4):
        logits.copy_(torch.randn((rows, V), generator=gen, device="cuda"))
        u.copy_(torch.rand(rows, generator=gen, device="cuda"))
        token.fill_(-9)
        graph.replay()
        torch.cuda.synchronize()
        sd.specdec_sample(ctx, logits, None, None, top_p, None, u, want)
        assert torch.equal(token, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [700, 20000, 150001])
def test_how_many_stay(ctx, dtype, V):
    """Rows where some number of heavy tokens, equal or not, hold nearly everything; top-k and top-p end within them, at their end and beyond."""
    rng = np.random.default_rng(V)
    for spread in (0.0, 1.0):
        rows, k, p, u = [], [], [], []
        for heavy in (1, 3, 127, 128, 129, 191, 192, 193, 194, 255, 256, 511, 512, 513, 600):
            for top_k, top_p in ((0, 0.9), (0, 0.5), (heavy, 1.0), (heavy - 1, 0.9), (heavy + 1, 1.0), (192, 0.7), (193, 1.0)):
                x = (rng.standard_normal(V) - 25).astype(np.float32)
                x[rng.permutation(V)[:heavy]] = 4 + spread * rng.random(heavy)
                rows.append(x)
                k.append(top_k)
                p.append(top_p)
                u.append(rng.random())
        n = len(rows)
        logits = torch.tensor(np.stack(rows)).to(DT[dtype]).cuda()
        check(ctx, logits, np.full(n, 1, np.float32), np.array(k, np.int32), np.array(p, np.float32), None, np.array(u, np.float32))
