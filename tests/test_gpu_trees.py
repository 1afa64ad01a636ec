"""Trees of drafts and forked batches on the models: logits of every row against the oracle's decoding along the row's path, commits against
the walk written out, caches bit for bit, and the loop verify - draw - commit as a program runs it."""
import numpy as np
import pytest
import torch

import cases
import gpu_harness as gh
import operators_oracle as oo
import specdec_oracle as orc
from paper_2203_16487_amd import binding as sd
from paper_2203_16487_amd import synth

pytestmark = pytest.mark.gpu


def desc_of(d, layers=2, vocab=1003):
    return synth.ModelDesc(0, layers, d, d // 64, 4 * d, vocab, 64, 300).resolved()


def trees(rng, B, n, gaps=False):
    """Parents of rows 1 .. n, [B, n]; gaps: some rows hang on none."""
    p = np.array([[int(rng.integers(max(0, i - 5), i)) for i in range(1, n + 1)] for _ in range(B)], dtype=np.int32).reshape(B, n)
    if gaps:
        p[rng.random(p.shape) < 0.15] = -1
        p[0, 0] = 1        # itself
    return p


def path_to(parent, i):
    rows = []
    while i > 0:
        rows.append(i)
        i = int(parent[i - 1])
    return rows[::-1]


def verify_tree(ses, draft, parent, vocab):
    logits = torch.full((len(parent), parent.shape[1] + 1, vocab), float("nan"), dtype=torch.float32, device="cuda")
    if parent.shape[1]:
        sd.specdec_verify_tree(ses.ctx, ses.i32(draft), ses.i32(parent), logits)
    else:
        sd.specdec_verify_tree(ses.ctx, None, None, logits)
    return logits


def check_logits(case, parent, draft, logits, tol):
    got = logits.cpu().numpy()
    for b in range(case.B):
        masks = oo.tree_masks(parent[b].tolist())
        pending = int(case.tokens[b, case.lens[b]])
        for i in range(parent.shape[1] + 1):
            if not masks[i]:
                continue
            along = [int(draft[b, r - 1]) for r in path_to(parent[b], i)]
            want = orc.verify_onepass(case.model, case.states[b].clone(), pending, along)[-1]
            assert float(np.abs(got[b, i] - want).max()) <= tol, (b, i)


# d, B, n, source, prefix, options: one row, few rows, many; an arena that is split over workgroups
SHAPES = [
    (128, 1, 0, 9, (0, 0), {}), (128, 1, 6, 9, (3, 7), {}), (128, 5, 5, 12, (0, 20), {}), (512, 2, 10, 20, (0, 40), {}), (512, 1, 31, 20, (30, 30), {}),
    (512, 7, 9, 20, (0, 33), {}), (128, 40, 7, 12, (0, 25), {}), (128, 3, 8, 9, (0, 12), {sd.SPECDEC_OPT_LN_FOLD: 0}), (192, 9, 12, 300, (0, 40), {}),
    (512, 3, 8, 20, (5, 20), {sd.SPECDEC_OPT_SMALL_BATCH_KERNELS: 0}),
]


@pytest.mark.parametrize("d,B,n,S,j,options", SHAPES)
def test_logits(d, B, n, S, j, options):
    rng = np.random.default_rng([d, B, n])
    case = cases.make_verify_case(desc_of(d), seed=d + B + n, B=B, S=S, k=max(n, 1), beta=3, tau=1.0, len_lo=j[0], len_hi=j[1], drafts="random",
                                  ragged_src=True, std=0.06 if d <= 192 else 0.03)
    ses = gh.open_verifier(case, options=options, fill=0xFF)
    parent = trees(rng, B, n, gaps=n > 8)
    draft = rng.integers(0, case.desc.vocab, size=(B, n)).astype(np.int32)
    check_logits(case, parent, draft, verify_tree(ses, draft, parent, case.desc.vocab), 2e-2)
    ses.close()


def test_logits_of_a_long_arena():
    """An arena beyond what one workgroup takes: the attention's work is split and joined."""
    case = cases.make_verify_case(desc_of(128, layers=1, vocab=211), seed=4, B=2, S=9, k=6, beta=3, tau=1.0, len_lo=700, len_hi=1300, drafts="random", std=0.06)
    ses = gh.open_verifier(case, max_tgt=1500, fill=0xFF)
    rng = np.random.default_rng(4)
    parent, draft = trees(rng, 2, 6), rng.integers(0, 211, size=(2, 6)).astype(np.int32)
    check_logits(case, parent, draft, verify_tree(ses, draft, parent, 211), 2e-2)
    ses.close()


@pytest.mark.parametrize("options", [{sd.SPECDEC_OPT_FP8_WEIGHTS: 1}, {sd.SPECDEC_OPT_FP8_CROSS_KV: 1}])
@pytest.mark.parametrize("B,n", [(2, 9), (6, 9)])
def test_logits_of_8_bit_models(options, B, n):
    fp8 = sd.SPECDEC_OPT_FP8_WEIGHTS in options and B * (n + 1) <= 32        # (larger passes read the bf16 matrices)
    case = cases.make_verify_case(desc_of(512), seed=B, B=B, S=20, k=n, beta=3, tau=1.0, len_lo=0, len_hi=15, drafts="random", ragged_src=True, std=0.03,
                                  fp8=fp8, fp8_kv=sd.SPECDEC_OPT_FP8_CROSS_KV in options)
    ses = gh.open_verifier(case, options=options)
    rng = np.random.default_rng(B)
    parent, draft = trees(rng, B, n), rng.integers(0, case.desc.vocab, size=(B, n)).astype(np.int32)
    check_logits(case, parent, draft, verify_tree(ses, draft, parent, case.desc.vocab), 3e-2)
    ses.close()


def test_a_chain_is_a_verification_pass():
    case = cases.make_verify_case(desc_of(512), seed=3, B=4, S=20, k=9, beta=3, tau=1.0, len_lo=0, len_hi=30, drafts="random", std=0.03)
    ses = gh.open_verifier(case)
    chain = gh.gpu_verify(ses, case)["logits"]
    got = verify_tree(ses, case.drafts, np.tile(np.arange(9, dtype=np.int32), (4, 1)), case.desc.vocab).cpu().numpy()
    assert float(np.abs(got - chain).max()) <= 1e-2
    ses.close()


def cache_of(ses, desc, B, L):
    k, v = (torch.zeros((desc.dec_layers, B, L, desc.d_model), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    sd.specdec_get_cache(ses.ctx, sd.SPECDEC_VERIFIER, k, v)
    return [x.view(torch.int16).cpu().numpy() for x in (k, v)]


@pytest.mark.parametrize("B,n,max_new", [(1, 1, 40), (1, 31, 9), (5, 7, 12), (33, 12, 20), (130, 5, 7), (3, 0, 4)])
def test_commit(B, n, max_new):
    """Tokens that follow random paths, end them, lie outside of the vocabulary; EOS and caps on the way; keys / values moved bit for bit."""
    rng = np.random.default_rng([B, n])
    desc = synth.ModelDesc(0, 2, 128, 2, 256, 211, 64, 300).resolved()
    case = cases.make_verify_case(desc, seed=B + n, B=B, S=6, k=max(n, 1), beta=3, tau=1.0, len_lo=0, len_hi=9, drafts="random", ragged_src=True)
    ses = gh.open_verifier(case, max_tgt=80, max_new=max_new)
    out, done, j = [[] for _ in range(B)], [False] * B, case.lens.astype(int).copy()
    acc, nxt, m, fin, active, cnt = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in (B, B, B, B, 1, sd.SPECDEC_COUNTERS))
    toks = torch.zeros((B, 64), dtype=torch.int32, device="cuda")
    total = 0
    for turn in range(1, 5):
        parent = trees(rng, B, n, gaps=n > 5)
        draft = rng.integers(4, 12, size=(B, n)).astype(np.int32)          # (few tokens: siblings carry the same ones)
        draft[rng.random(draft.shape) < 0.08] = desc.eos_id
        token = rng.integers(4, 14, size=(B, n + 1)).astype(np.int32)
        token[rng.random(token.shape) < 0.1] = desc.eos_id
        token[rng.random(token.shape) < 0.05] = -1
        token[rng.random(token.shape) < 0.02] = desc.vocab
        verify_tree(ses, draft, parent, desc.vocab)
        L = int(j.max()) + n + 1
        before = cache_of(ses, desc, B, L)
        if turn % 2:
            sd.specdec_commit_tree(ses.ctx, ses.i32(token), acc, nxt, active)
        else:
            sd.specdec_commit_tree(ses.ctx, ses.i32(token), None, None, active)
        after = cache_of(ses, desc, B, L)
        sd.specdec_get_output(ses.ctx, toks, m, fin)
        sd.specdec_get_counters(ses.ctx, cnt)
        for b in range(B):
            masks = oo.tree_masks(parent[b].tolist())
            at, path = 0, [0]
            while True:
                t = int(token[b, at])
                on = [i for i in range(1, n + 1) if masks[i] and int(parent[b, i - 1]) == at and int(draft[b, i - 1]) == t]
                if not 0 <= t < desc.vocab or not on:
                    break
                at = on[0]
                path.append(at)
            failed = not 0 <= t < desc.vocab
            if turn % 2:
                want = (0, desc.pad_id) if done[b] else (-1, desc.pad_id) if failed else (len(path) - 1, t)
                assert (int(acc[b]), int(nxt[b])) == want, (turn, b)
            rows = np.arange(L)
            if not done[b] and not failed:
                rows[j[b]:j[b] + len(path)] = j[b] + np.array(path)
                for x in [int(draft[b, i - 1]) for i in path[1:]] + [t]:
                    out[b].append(x)
                    j[b] += 1
                    total += 1
                    if x == desc.eos_id or len(out[b]) == max_new:
                        done[b] = True
                        break
            for x, y in zip(before, after):
                assert np.array_equal(y[:, b], x[:, b][:, rows]), (turn, b)
        assert m.cpu().tolist() == [len(o) for o in out] and fin.cpu().tolist() == [int(x) for x in done]
        for b in range(B):
            assert toks[b, :len(out[b])].cpu().tolist() == out[b], b
        assert int(active) == B - sum(done) and cnt[:3].cpu().tolist() == [turn, total, sum(done)]
    ses.close()


def test_loop_of_trees_is_greedy_decoding():
    """verify_tree, sample at temperature 0, commit_tree, with trees that hold the right continuation among others: every token is the
    oracle's arg-max after the tokens before it, or within rounding of it."""
    desc = desc_of(512, vocab=500)
    B, n = 3, 8
    case = cases.make_verify_case(desc, seed=9, B=B, S=12, k=n, beta=3, tau=1.0, len_lo=2, len_hi=9, drafts="random", std=0.06, cap_extra=40)
    ses = gh.open_verifier(case, max_tgt=80)
    rng = np.random.default_rng(9)
    streams = [case.tokens[b, :case.lens[b] + 1].tolist() for b in range(B)]
    states = [st.clone() for st in case.states]
    u, zero = torch.zeros(B * (n + 1), device="cuda"), torch.zeros(B * (n + 1), device="cuda")
    token = torch.zeros((B, n + 1), dtype=torch.int32, device="cuda")
    acc, nxt = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
    kept = 0
    for turn in range(4):
        parent, draft = trees(rng, B, n), rng.integers(0, 500, size=(B, n)).astype(np.int32)
        for b in range(B):       # the oracle's own continuation along one path of the tree
            st, t = states[b].clone(), streams[b][-1]
            for r in path_to(parent[b], n):
                t = int(np.argmax(orc.dec_step(case.model, st, t)))
                draft[b, r - 1] = t
        logits = verify_tree(ses, draft, parent, 500)
        sd.specdec_sample(ses.ctx, logits.view(-1, 500), zero, None, None, None, u, token.view(-1))
        sd.specdec_commit_tree(ses.ctx, token, acc, nxt)
        for b in range(B):
            a, rows = int(acc[b]), [0]
            for _ in range(a):
                rows.append(min(i for i in range(1, n + 1) if parent[b, i - 1] == rows[-1] and draft[b, i - 1] == int(token[b, rows[-1]])))
            for x in [int(draft[b, r - 1]) for r in rows[1:]] + [int(nxt[b])]:
                z = orc.dec_step(case.model, states[b], streams[b][-1])
                assert z.max() - z[x] <= 4e-2, (turn, b)
                streams[b].append(x)
            kept += a
    assert kept >= 12            # (paths of several drafts are kept: caches were compacted)
    ses.close()


def test_loop_captured():
    """The same three calls captured once and replayed: every replay as the eager calls on the same state."""
    desc = desc_of(128, vocab=211)
    B, n = 4, 6
    case = cases.make_verify_case(desc, seed=11, B=B, S=9, k=n, beta=3, tau=1.0, len_lo=2, len_hi=9, drafts="random", std=0.08)
    rng = np.random.default_rng(11)
    parent = [trees(rng, B, n) for _ in range(5)]
    draft = [rng.integers(4, 211, size=(B, n)).astype(np.int32) for _ in range(5)]
    us = [rng.random(B * (n + 1)).astype(np.float32) for _ in range(5)]

    def run(captured):
        ses = gh.open_verifier(case, max_tgt=80)
        p, d, u = ses.i32(parent[0]), ses.i32(draft[0]), torch.tensor(us[0], device="cuda")
        logits = torch.zeros((B, n + 1, 211), dtype=torch.float32, device="cuda")
        token = torch.zeros((B, n + 1), dtype=torch.int32, device="cuda")
        acc, nxt, m = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(3))
        toks = torch.zeros((B, 60), dtype=torch.int32, device="cuda")

        def step():
            sd.specdec_verify_tree(ses.ctx, d, p, logits)
            sd.specdec_sample(ses.ctx, logits.view(-1, 211), None, None, None, None, u, token.view(-1))
            sd.specdec_commit_tree(ses.ctx, token, acc, nxt)
        if captured:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        got = []
        for i in range(5):
            p.copy_(torch.tensor(parent[i]))
            d.copy_(torch.tensor(draft[i]))
            u.copy_(torch.tensor(us[i]))
            graph.replay() if captured else step()
            torch.cuda.synchronize()
            sd.specdec_get_output(ses.ctx, toks, m)
            got.append((logits.cpu().clone(), acc.tolist(), nxt.tolist(), m.tolist(), toks.cpu().tolist()))
        ses.close()
        return got
    for a, b in zip(run(False), run(True)):
        assert torch.equal(a[0], b[0]) and a[1:] == b[1:]


@pytest.mark.parametrize("options", [{}, {sd.SPECDEC_OPT_FP8_CROSS_KV: 1}])
@pytest.mark.parametrize("B,src", [(1, [0, 0, 0, 0]), (4, [3, 2, 1, 0]), (5, [4, 4, 1]), (3, [1, -7, 99, 0, 2, 2, 1]), (40, None)])
def test_fork(B, src, options):
    """Every sequence goes on as its source would have: stream, caps, flags, self- and cross-attention keys / values."""
    rng = np.random.default_rng(B)
    src = rng.integers(0, B, size=70).tolist() if src is None else src
    N, desc, n = len(src), desc_of(128, vocab=300), 4
    case = cases.make_verify_case(desc, seed=B, B=B, S=41, k=n, beta=3, tau=1.0, len_lo=0, len_hi=30, drafts="random", ragged_src=True, std=0.08,
                                  fp8_kv=bool(options))
    ses = gh.open_verifier(case, max_batch=max(B, N), max_tgt=70, max_new=6, options=options, fill=0xFF)
    acc, nxt = ses.i32(np.zeros(B)), ses.i32(np.zeros(B))
    sd.specdec_verify(ses.ctx, ses.i32(case.drafts), n, 3, 1.0, acc, nxt)
    sd.specdec_commit(ses.ctx, ses.i32(rng.integers(0, n + 1, size=B)), ses.i32(rng.integers(0, 300, size=B)))
    def output(count):
        toks, m, fin = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((count, 70), count, count))
        sd.specdec_get_output(ses.ctx, toks, m, fin)
        return [x.cpu().numpy() for x in (toks, m, fin)]
    L = 36
    before, was = cache_of(ses, desc, B, L), output(B)
    old = verify_tree(ses, case.drafts, np.tile(np.arange(n, dtype=np.int32), (B, 1)), 300).cpu().numpy()
    rows = [int(x) + int(c) for x, c in zip(was[1], case.lens)]
    sd.specdec_fork(ses.ctx, ses.i32(src))
    from_ = [min(max(s, 0), B - 1) for s in src]
    after, now = cache_of(ses, desc, N, L), output(N)
    for x, y in zip(was, now):
        assert np.array_equal(y, x[from_])
    for x, y in zip(before, after):
        for b, a in enumerate(from_):
            assert np.array_equal(y[:, b, :rows[a]], x[:, a, :rows[a]]), b
    new = verify_tree(ses, case.drafts[from_], np.tile(np.arange(n, dtype=np.int32), (N, 1)), 300).cpu().numpy()
    assert float(np.abs(new - old[from_]).max()) <= 1e-2
    # each goes on by itself: other tokens for copies of one sequence, caps that count what the source had
    nxt2 = np.arange(N) % 290 + 5
    token = np.tile(nxt2[:, None], (1, n + 1)).astype(np.int32)
    sd.specdec_commit_tree(ses.ctx, ses.i32(token))
    toks, m, fin = output(N)
    for b, a in enumerate(from_):
        if was[2][a]:
            assert m[b] == was[1][a]
        else:
            assert m[b] > was[1][a] and toks[b, m[b] - 1] in (nxt2[b], *case.drafts[a]) and (m[b] < 6 or fin[b])
    ses.close()


def test_fork_with_a_drafter_and_an_encoder():
    """Both models' caches and memories go along, also to a larger batch; a draft of a copy is its source's."""
    vd = synth.ModelDesc(1, 2, 128, 2, 256, 211, 32, 60).resolved()
    dd = synth.ModelDesc(1, 1, 64, 1, 128, 211, 32, 60).resolved()
    ses = sd.Session(6, 4, 32, 60, fill=0xFF)
    for role, desc in ((sd.SPECDEC_VERIFIER, vd), (sd.SPECDEC_DRAFTER, dd)):
        ses.bind_model(role, desc, ses.upload_weights(synth.make_weights(desc, 3 + role, std=0.08)))
    rng = np.random.default_rng(1)
    sd.specdec_begin(ses.ctx, 2, 40)
    src = ses.i32(rng.integers(4, 210, size=(2, 20)))
    sd.specdec_encode(ses.ctx, src, ses.i32([20, 13]))
    draft, acc, nxt = ses.i32(np.zeros((2, 4))), ses.i32([0, 0]), ses.i32([0, 0])
    for _ in range(3):
        sd.specdec_draft(ses.ctx, 4, draft)
        sd.specdec_verify(ses.ctx, draft, 4, 3, 5.0, acc, nxt)
        sd.specdec_commit(ses.ctx, acc, nxt)
    sd.specdec_fork(ses.ctx, ses.i32([1, 0, 1, 1, 0]))
    mem = torch.zeros((5, 20, 128), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(sd.SpecDecError) as e:        # the memory is that of the batch that was encoded
        sd.specdec_get_memory(ses.ctx, sd.SPECDEC_VERIFIER, mem)
    assert e.value.code == sd.SPECDEC_ERR_BAD_STATE
    with pytest.raises(sd.SpecDecError):
        sd.specdec_commit(ses.ctx, acc, nxt)
    d5, l5 = ses.i32(np.zeros((5, 4))), torch.zeros((5, 4, 211), device="cuda")
    sd.specdec_draft(ses.ctx, 4, d5, l5)
    a5, n5, v5 = ses.i32(np.zeros(5)), ses.i32(np.zeros(5)), torch.zeros((5, 5, 211), device="cuda")
    sd.specdec_verify(ses.ctx, d5, 4, 3, 5.0, a5, n5, v5)
    for other in (2, 3):
        assert torch.allclose(l5[0], l5[other], atol=1e-2) and torch.allclose(v5[0], v5[other], atol=1e-2)
    assert torch.allclose(l5[1], l5[4], atol=1e-2) and torch.allclose(v5[1], v5[4], atol=1e-2)
    assert bool(torch.isfinite(l5).all() and torch.isfinite(v5).all()) and not torch.allclose(l5[0], l5[1], atol=1e-1)
    ses.close()


def test_refusals():
    case = cases.make_verify_case(desc_of(128, vocab=211), seed=2, B=2, S=9, k=3, beta=3, tau=1.0, len_lo=1, len_hi=5, drafts="random")
    ses = gh.open_verifier(case, max_batch=3)
    L, ctx = sd.lib(), ses.ctx
    d, p, t = ses.i32(case.drafts), ses.i32(np.tile(np.arange(3), (2, 1))), ses.i32(np.zeros((2, 4)))
    z = torch.zeros((2, 4, 211), device="cuda")
    bad, state, large = sd.SPECDEC_ERR_INVALID_ARG, sd.SPECDEC_ERR_BAD_STATE, sd.SPECDEC_ERR_TOO_LARGE
    assert L.specdec_verify_tree(ctx, d.data_ptr(), p.data_ptr(), 3, None, None) == bad
    assert L.specdec_verify_tree(ctx, None, p.data_ptr(), 3, z.data_ptr(), None) == bad
    assert L.specdec_verify_tree(ctx, d.data_ptr(), None, 3, z.data_ptr(), None) == bad
    assert L.specdec_verify_tree(ctx, d.data_ptr(), p.data_ptr(), -1, z.data_ptr(), None) == bad
    assert L.specdec_verify_tree(ctx, d.data_ptr(), p.data_ptr(), 4, z.data_ptr(), None) == large
    assert L.specdec_commit_tree(ctx, t.data_ptr(), None, None, None, None) == state     # nothing verified
    acc, nxt = ses.i32([0, 0]), ses.i32([5, 5])
    sd.specdec_verify(ctx, d, 3, 3, 1.0, acc, nxt)
    assert L.specdec_commit_tree(ctx, t.data_ptr(), None, None, None, None) == state     # a chain was
    sd.specdec_verify_tree(ctx, d, p, z)
    assert L.specdec_commit(ctx, acc.data_ptr(), nxt.data_ptr(), None, None) == state    # a tree was
    stats = torch.zeros((2, 4, 8), device="cuda")
    assert L.specdec_get_row_stats(ctx, stats.data_ptr(), None) == state
    assert L.specdec_commit_tree(ctx, None, None, None, None, None) == bad
    sd.specdec_rewind(ctx, ses.i32([9, 9]))
    assert L.specdec_commit_tree(ctx, t.data_ptr(), None, None, None, None) == state     # undone
    assert L.specdec_fork(ctx, None, 2, None) == bad and L.specdec_fork(ctx, t.data_ptr(), 0, None) == bad
    assert L.specdec_fork(ctx, t.data_ptr(), 4, None) == large
    sd.specdec_set_stream(ctx, ses.i32(case.tokens), ses.i32(case.lens))
    assert L.specdec_verify_tree(ctx, d.data_ptr(), p.data_ptr(), 3, z.data_ptr(), None) == state      # nothing cached
    K, V = cases.oracle_flat_cache(case, case.L_max)
    sd.specdec_load_cache(ctx, sd.SPECDEC_VERIFIER, ses.bf16(K), ses.bf16(V), ses.i32([case.lens[0], case.lens[1] - 1]))
    sd.specdec_verify_tree(ctx, d, p, z)
    sd.specdec_commit_tree(ctx, t, acc, nxt)                                                          # (one of them short of its stream)
    assert acc.tolist()[1] == -1 and nxt.tolist()[1] == case.desc.pad_id and acc.tolist()[0] >= 0
    ses.close()
