"""Operators on a caller's tensors at the largest sizes that they accept."""
import pytest
import torch

from paper_2203_16487_amd import binding as sd

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = sd.specdec_create(1, 1, 1, 1)
    yield c
    sd.specdec_destroy(c)


def test_masks_of_many_trees(ctx):
    """More trees than the threads of one grid dimension are waves."""
    B = (1 << 26) + 3
    parent = torch.zeros((B, 1), dtype=torch.int32, device="cuda")
    parent[::3] = -1
    visible = torch.zeros((B, 2), dtype=torch.int64, device="cuda")
    sd.specdec_tree_visible(ctx, parent, visible)
    assert bool((visible[:, 0] == 1).all())
    assert torch.equal(visible[:, 1], torch.where(parent[:, 0] == 0, 3, 0))


# (33 columns in a block of 64; 129 in two of 128: in all 2^26 places of columns, and a third more)
@pytest.mark.parametrize("B,H,Hkv,T", [(1024, 1024, 1024, 33), (2048, 510, 170, 43)])
def test_attention_of_many_columns(ctx, B, H, Hkv, T):
    """As many columns as batch x heads and rows allow, in an arena that is split.  Queries, keys and values are shared (strides of 0), so every head of a
    sequence has the same output: that of a call with one head."""
    gen = torch.Generator(device="cuda").manual_seed(B)
    cap, dh = 1100, 64
    q = torch.randn((1, T, 1, dh), generator=gen, device="cuda").to(torch.bfloat16)
    k, v = (torch.randn((1, 1, cap, dh), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    cached = torch.randint(0, 100, (B,), generator=gen, device="cuda", dtype=torch.int32)
    cached[::100] = cap - T
    rows = torch.randint(0, T + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)

    def call(heads, kv):
        out = torch.full((B, T, heads, dh), 7.0, dtype=torch.bfloat16, device="cuda")
        args = q.expand(B, T, heads, dh), k.expand(B, kv, cap, dh), v.expand(B, kv, cap, dh)
        desc = sd.tree_attn_desc(*args, out, 0.125)
        ws = torch.empty(sd.specdec_tree_attention_bytes(ctx, desc), dtype=torch.uint8, device="cuda")
        sd.specdec_tree_attention(ctx, desc, *args, cached, None, rows, out, ws)
        torch.cuda.synchronize()
        return out
    one = call(1, 1)
    many = call(H, Hkv)
    for b in range(0, B, 64):
        got, want = many[b:b + 64].float(), one[b:b + 64].float()
        # (another cut of the work: weights and outputs of either rounded by half a step of bf16 of what is at most the largest value)
        assert float((got - want).abs().max()) <= 2 * 2 ** -8 * 2 * float(v.float().abs().max()) * 1.02
        assert bool((got == got[:, :, :1]).all())
        assert bool((got[torch.arange(T, device="cuda")[None] >= rows[b:b + 64, None]] == 7).all())
