"""Appending chunks of so many blocks that a wavefront takes one each and the lengths move on in a launch behind (from 226 tokens that fit)."""
import numpy as np
import pytest
import torch

from oracle import quant_oracle as Q
from tests import gpu_util as U
from tests import quant_util as T
from tests import test_gpu_quant as G

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("tokens,cap", [(225, 700), (226, 700), (257, 300), (500, 700), (600, 300)])
def test_long_chunks(tokens, cap, D, dtype):
    """Both sides of the rule, heads from empty to full, counts of zero, below and above the chunk, more tokens than a cache holds."""
    G.test_append(tokens, cap, D, dtype)


@pytest.mark.parametrize("tokens", [5, 300])
def test_many_heads(tokens):
    """264 heads, more than a workgroup of the launch that moves the lengths on; some full, some asked for nothing."""
    kk = U.kk()
    g = G.gen(tokens)
    B, H, D, cap = 33, 8, 64, 400
    lay = T.layout(B, H, 1, D, "bf16")
    rng = np.random.default_rng(3)
    lens = rng.integers(0, cap + 1, (B, H))
    lens[0, :3], lens[-1, -2:] = (0, cap, cap - 1), (64, 33)
    counts = rng.integers(-2, tokens + 3, (B, H))
    counts[-1, -1] = tokens
    c = T.state(g, lay, cap, lens)
    k_t, v_t = T.rows(g, (B, H, tokens, D), "bf16", 3.0), T.rows(g, (B, H, tokens, D), "bf16", 3.0)
    take = np.minimum(np.clip(counts, 0, tokens), cap - lens)
    some = [(0, 0), (0, 1), (0, 2), (7, 3), (16, 5), (31, 7), (32, 0), (32, 6), (32, 7)]
    want = {bh: [Q.append(*x, U.to_host(t)[bh][:take[bh]]) for x, t in zip(T.head(c, *bh), (k_t, v_t))] for bh in some}
    votes, born = c.votes.clone(), c.born.clone()
    overflow = torch.zeros(1, dtype=torch.int32, device="cuda")
    kk.append_quant(lay, c, k_t, v_t, tokens, torch.from_numpy(counts.astype(np.int32)).cuda(), overflow)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(c.len.cpu().numpy(), lens + take)
    assert int(overflow) == int((np.clip(counts, 0, tokens) > take).any())
    slot = np.arange(cap)
    new = torch.from_numpy((slot >= lens[..., None]) & (slot < (lens + take)[..., None])).cuda()
    assert torch.equal(c.votes, torch.where(new, 1, votes)) and torch.equal(c.born, torch.where(new, 9, born))
    assert torch.isneginf(c.log_s[new]).all()
    for bh in some:
        G.check_head(c, *bh, *want[bh])


def test_a_chunk_equals_its_tokens_one_by_one():
    """Where every token needs no larger scale than the block's first: the same codes, however they came."""
    kk = U.kk()
    g = G.gen(77)
    lay = T.layout(1, 3, 2, 128, "bf16")
    start = T.state(g, lay, 600, [[0, 17, 64]])
    a, b, c = (G.copy_of(kk, lay, start) for _ in range(3))
    k_t, v_t = (torch.rand((1, 3, 300, 128), generator=g, device="cuda").add_(1.0).mul_(0.25).bfloat16() for _ in range(2))
    kk.append_quant(lay, a, k_t, v_t, 300)
    for i in range(300):
        kk.append_quant(lay, b, k_t[:, :, i].contiguous(), v_t[:, :, i].contiguous())
    for i in (0, 150):
        kk.append_quant(lay, c, k_t[:, :, i:i + 150].contiguous(), v_t[:, :, i:i + 150].contiguous(), 150)
    torch.cuda.synchronize()
    for o in (b, c):
        for f in a.FIELDS:
            assert torch.equal(T.bits(getattr(a, f)), T.bits(getattr(o, f))), f
