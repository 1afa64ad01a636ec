"""A verification pass that is refused leaves the pass before it as it was: what is committed afterwards are that pass's drafts."""
import numpy as np
import pytest
import torch

import cases
import gpu_harness as gh
from paper_2203_16487_amd import binding as sd
from paper_2203_16487_amd import synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tree", [True, False])
def test_refused_pass(tree):
    desc = synth.ModelDesc(0, 2, 512, 8, 2048, 1003, 64, 300).resolved()
    B, n = 2, 4
    case = cases.make_verify_case(desc, seed=6, B=B, S=9, k=n, beta=3, tau=1.0, len_lo=1, len_hi=6, drafts="random", std=0.03, fp8=True)
    ses = gh.open_verifier(case, options={sd.SPECDEC_OPT_FP8_WEIGHTS: 1})
    first = np.array([[10, 11, 12, 13], [20, 21, 22, 23]], dtype=np.int32)
    parent = np.tile(np.arange(n, dtype=np.int32), (B, 1))
    acc, nxt = ses.i32([-7, -7]), ses.i32([-7, -7])
    if tree:
        logits = torch.zeros((B, n + 1, desc.vocab), device="cuda")
        sd.specdec_verify_tree(ses.ctx, ses.i32(first), ses.i32(parent), logits)
    else:
        sd.specdec_verify(ses.ctx, ses.i32(first), n, 3, 1.0, acc, nxt)
    sd.specdec_configure(ses.ctx, sd.SPECDEC_OPT_RESIDENT, 1)
    with pytest.raises(sd.SpecDecError) as e:       # (8-bit weights in few rows: the default kernels only)
        sd.specdec_verify(ses.ctx, ses.i32(first + 100), n, 3, 1.0, acc, nxt)
    assert e.value.code == sd.SPECDEC_ERR_BAD_STATE
    sd.specdec_configure(ses.ctx, sd.SPECDEC_OPT_RESIDENT, 0)
    if tree:                                        # each row's token is the next draft, of two sequences' first two
        token = np.array([[10, 11, 40, 40, 40], [20, 21, 41, 41, 41]], dtype=np.int32)
        sd.specdec_commit_tree(ses.ctx, ses.i32(token), acc, nxt)
        assert acc.tolist() == [2, 2] and nxt.tolist() == [40, 41]
    else:
        sd.specdec_commit(ses.ctx, ses.i32([2, 2]), ses.i32([40, 41]))
    toks, m = torch.zeros((B, 20), dtype=torch.int32, device="cuda"), ses.i32([0, 0])
    sd.specdec_get_output(ses.ctx, toks, m)
    assert m.tolist() == [3, 3] and toks[:, :3].tolist() == [[10, 11, 40], [20, 21, 41]]
    ses.close()
