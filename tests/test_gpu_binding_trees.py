"""The wrappers of the passes over trees against the batch and the pass that there is: what would be read or written out of range is refused."""
import pytest
import torch

import cases
import gpu_harness as gh
from paper_2203_16487_amd import binding as sd
from paper_2203_16487_amd import synth

pytestmark = pytest.mark.gpu


def refused(what, call):
    with pytest.raises(sd.SpecDecError, match=what) as e:
        call()
    assert e.value.code == sd.SPECDEC_ERR_INVALID_ARG


def test_sizes():
    desc = synth.ModelDesc(0, 2, 128, 2, 512, 211, 64, 300).resolved()
    case = cases.make_verify_case(desc, seed=2, B=3, S=9, k=4, beta=3, tau=1.0, len_lo=1, len_hi=5, drafts="random")
    ses = gh.open_verifier(case, max_batch=5)
    ctx = ses.ctx
    assert sd.specdec_pass_sizes(ctx) == (3, 0, 211)
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")
    z = lambda *shape: torch.zeros(shape, device="cuda")
    refused("draft", lambda: sd.specdec_verify_tree(ctx, i32(2, 2), i32(2, 2), z(2, 3, 211)))       # another batch
    refused("draft", lambda: sd.specdec_verify_tree(ctx, i32(4, 2), i32(4, 2), z(4, 3, 211)))
    refused("parent", lambda: sd.specdec_verify_tree(ctx, i32(3, 2), i32(3, 1), z(3, 3, 211)))
    refused("logits", lambda: sd.specdec_verify_tree(ctx, i32(3, 2), i32(3, 2), z(3, 3, 210)))      # another vocabulary
    refused("logits", lambda: sd.specdec_verify_tree(ctx, i32(3, 2), i32(3, 2), z(3, 2, 211)))
    refused("logits", lambda: sd.specdec_verify_tree(ctx, None, None, z(2, 1, 211)))
    refused("cpu", lambda: sd.specdec_verify_tree(ctx, i32(3, 2).cpu(), i32(3, 2), z(3, 3, 211)))
    assert sd.specdec_pass_sizes(ctx) == (3, 0, 211)
    with pytest.raises(sd.SpecDecError) as e:
        sd.specdec_commit_tree(ctx, i32(3, 3))
    assert e.value.code == sd.SPECDEC_ERR_BAD_STATE                                                 # (no pass: the library says so)
    sd.specdec_verify_tree(ctx, i32(3, 2), i32(3, 2), z(3, 3, 211))
    assert sd.specdec_pass_sizes(ctx) == (3, 3, 211)
    refused("token", lambda: sd.specdec_commit_tree(ctx, i32(3, 2)))                                # another pass
    refused("token", lambda: sd.specdec_commit_tree(ctx, i32(2, 3)))
    refused("next_token", lambda: sd.specdec_commit_tree(ctx, i32(3, 3), i32(3), i32(4)))
    sd.specdec_commit_tree(ctx, i32(3, 3), i32(3), i32(3), i32(1))
    assert sd.specdec_pass_sizes(ctx) == (3, 0, 211)
    sd.specdec_verify_tree(ctx, None, None, z(3, 1, 211))
    assert sd.specdec_pass_sizes(ctx) == (3, 1, 211)
    sd.specdec_fork(ctx, i32(5))
    assert sd.specdec_pass_sizes(ctx) == (5, 0, 211)
    refused("draft", lambda: sd.specdec_verify_tree(ctx, i32(3, 2), i32(3, 2), z(3, 3, 211)))       # (the batch is another one now)
    sd.specdec_verify_tree(ctx, i32(5, 2), i32(5, 2), z(5, 3, 211))
    ses.close()
