"""The wrappers of the passes over trees and of forks refuse tensors whose sizes and types the library would misread: by their own sizes first (here,
on host tensors), then by their device, then by the batch and pass that there is (test_gpu_binding_trees.py)."""
import pytest
import torch

from paper_2203_16487_amd import binding as sd

I32 = torch.int32


@pytest.fixture
def ctx():
    c = sd.specdec_create(4, 5, 8, 20)
    yield c
    sd.specdec_destroy(c)


def refused(what, call):
    with pytest.raises(sd.SpecDecError, match=what) as e:
        call()
    assert e.value.code == sd.SPECDEC_ERR_INVALID_ARG


def test_verify_tree(ctx):
    d, p, z = torch.zeros((2, 3), dtype=I32), torch.zeros((2, 3), dtype=I32), torch.zeros((2, 4, 11))
    call = lambda a, b, c: sd.specdec_verify_tree(ctx, a, b, c)
    refused("draft", lambda: call(d.long(), p, z))
    refused("draft", lambda: call(d[0], p, z))
    refused("draft", lambda: call(torch.zeros((3, 2), dtype=I32).t(), p, z))
    refused("parent", lambda: call(None, p, z))
    refused("parent", lambda: call(d, p.long(), z))
    refused("parent", lambda: call(d, p[:, :2].contiguous(), z))
    refused("parent", lambda: call(d, p[:1], z))
    refused("parent", lambda: call(d, None, z))
    refused("logits", lambda: call(d, p, z.bfloat16()))
    refused("logits", lambda: call(d, p, z[:, :3].contiguous()))
    refused("logits", lambda: call(d, p, z[:1]))
    refused("logits", lambda: call(d, p, z.view(8, 11)))
    refused("logits", lambda: call(d, p, torch.zeros((2, 4, 22))[:, :, ::2]))
    refused("logits", lambda: call(None, None, z))
    refused("logits", lambda: call(d, p, None))
    refused("cpu", lambda: call(d, p, z))


def test_commit_tree(ctx):
    t, one = torch.zeros((2, 4), dtype=I32), torch.zeros(2, dtype=I32)
    refused("token", lambda: sd.specdec_commit_tree(ctx, t.long()))
    refused("token", lambda: sd.specdec_commit_tree(ctx, t.view(-1)))
    refused("token", lambda: sd.specdec_commit_tree(ctx, t[:, ::2]))
    refused("token", lambda: sd.specdec_commit_tree(ctx, None))
    refused("accept_len", lambda: sd.specdec_commit_tree(ctx, t, one.long()))
    refused("accept_len", lambda: sd.specdec_commit_tree(ctx, t, one[:1]))
    refused("next_token", lambda: sd.specdec_commit_tree(ctx, t, one, one.float()))
    refused("n_active", lambda: sd.specdec_commit_tree(ctx, t, one, one, torch.zeros(1, dtype=torch.int64)))
    refused("n_active", lambda: sd.specdec_commit_tree(ctx, t, None, None, torch.zeros(0, dtype=I32)))
    refused("cpu", lambda: sd.specdec_commit_tree(ctx, t, one, one, torch.zeros(1, dtype=I32)))


def test_fork(ctx):
    refused("src", lambda: sd.specdec_fork(ctx, torch.zeros(2, dtype=torch.int64)))
    refused("src", lambda: sd.specdec_fork(ctx, torch.zeros((2, 2), dtype=I32)))
    refused("src", lambda: sd.specdec_fork(ctx, torch.zeros(4, dtype=I32)[::2]))
    refused("src", lambda: sd.specdec_fork(ctx, None))
    refused("cpu", lambda: sd.specdec_fork(ctx, torch.zeros(2, dtype=I32)))


def test_sizes_without_a_batch(ctx):
    assert sd.specdec_pass_sizes(ctx) == (0, 0, 0)
    assert sd.lib().specdec_pass_sizes(ctx, None, None, None) == sd.SPECDEC_OK
    assert sd.lib().specdec_pass_sizes(None, None, None, None) == sd.SPECDEC_ERR_INVALID_ARG
