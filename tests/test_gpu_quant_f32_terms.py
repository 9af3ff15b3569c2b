"""f32 layouts keep 24 bits of weights and queries in bf16 terms: bounds that two terms of either would break."""
import numpy as np
import pytest
import torch

from oracle import quant_oracle as Q
from tests import gpu_util as U
from tests import quant_util as T

pytestmark = pytest.mark.gpu
PLANS = [(64, 4), (128, 4), (256, 8), (512, 4), (1024, 8), (0, 0)]      # one tile a wavefront, more, by plan; with splits and without


def bf16(x):
    """To nearest even, 8 significant bits."""
    return torch.tensor(x, dtype=torch.float32).bfloat16().double().numpy()


def cut(x):
    """The 8 leading bits of an f32."""
    return (np.float32(x).view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32)


def put(c, what, rows):
    codes, scales = Q.quantize(rows)
    getattr(c, what).view(torch.uint8)[0, :, :len(rows)] = torch.from_numpy(codes).cuda()
    getattr(c, what + "_scale")[0, :, :len(scales)] = torch.from_numpy(scales.astype(np.float32)).cuda()


@pytest.mark.parametrize("per,waves", PLANS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_weights(G, D, per, waves):
    """Zero queries: the weights are votes / 3, that is 1 or 1/3.  Of each channel one slot has the value 1 and all others 0, so a channel is its
    slot's weight over the sum of weights, and of two neighbours the quotient is 1/3 whatever that sum is.

    Its roundings: log2 3 a step (2^-23, of the weight ln 2 times that), log2 1 and the difference none; exp2 a step, 2^-23; three terms 2^-27;
    their sum two steps (2^-22); two divisions (2^-23): 5.3e-7.  Two terms of 1/3 are off by 2^-18 = 3.8e-6 of it."""
    bound, third = 5.3e-7, 1.0 / 3.0
    two = bf16(third) + bf16(third - bf16(third))
    assert abs(two - third) / third > 5 * bound
    kk = U.kk()
    n, cap = 300, 320
    lay = T.layout(1, 2, G, D, "f32")
    c = kk.QuantCache(lay, cap)
    slots = np.random.default_rng(D).permutation(n)[:D]
    v, votes = np.zeros((n, D)), np.full(n, 3)
    v[slots, np.arange(D)] = 1.0
    votes[slots[::2]] = 1
    assert all((votes[i:i + 32] == 3).any() for i in range(0, n, 32))     # (no tile's maximum is another)
    put(c, "v", v)
    put(c, "k", np.ones((n, D)))
    c.votes[0, :, :n] = torch.from_numpy(votes.astype(np.int32)).cuda()
    c.len.fill_(n)
    c.plan_slots_per_split, c.plan_wavefronts = per, waves
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    kk.workspace_init(ws)
    q = torch.zeros((1, 2 * G, D), device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros((1, 2 * G), device="cuda")
    kk.decode_attn_quant(lay, c, q, out, None, lse, ws)
    torch.cuda.synchronize()
    got = out[0].cpu().numpy().astype(np.float64)
    assert (np.abs(got[:, ::2] / got[:, 1::2] * 3 - 1) <= bound).all(), float(np.abs(got[:, ::2] / got[:, 1::2] * 3 - 1).max())
    assert np.abs(got[:, 1::2] * votes.sum() / 3 - 1).max() <= (n + 16) * 2.0 ** -24      # the sum of weights: a rounding an addition
    assert np.abs(lse.cpu().numpy() - np.log(votes.sum())).max() <= (n + 16) * 2.0 ** -24 + 8 * 2.0 ** -22


@pytest.mark.parametrize("per,waves", PLANS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_queries(G, D, per, waves):
    """One channel of a query is not zero and keys are powers of two of either sign, so a logit is one product and the three terms' partial
    sums are exact.  Left are the mean over the group (G - 1 additions), its factor and the product: (G + 2) 2^-24 of the mean magnitude.  Cut to two
    terms, 16 bits, a group's mean is off by more than four times that (some group's, with one query head)."""
    kk = U.kk()
    g = torch.Generator(device="cuda").manual_seed(G * D)
    n, cap, H = 300, 320, 4
    lay = T.layout(1, H, G, D, "f32")
    c = kk.QuantCache(lay, cap)
    rng = np.random.default_rng(D + G)
    keys = rng.choice([-1.0, 1.0], (n, D)) * 2.0 ** rng.integers(-5, 3, (n, D))
    put(c, "k", keys)
    put(c, "v", np.ones((n, D)))
    c.votes.fill_(1)
    c.len.fill_(n)
    c.plan_slots_per_split, c.plan_wavefronts = per, waves
    x = (1.0 + torch.rand((H * G,), generator=g, device="cuda")).cpu().numpy()
    where = rng.integers(0, D, H)                                     # (a group's queries share their channel: no cancellation in the mean)
    q = torch.zeros((1, H * G, D), device="cuda")
    for i in range(H * G):
        q[0, i, where[i // G]] = float(x[i])
    first = cut(x)
    lost = (x - first.astype(np.float64) - cut(x - first)).reshape(H, G).mean(1) / x.astype(np.float64).reshape(H, G).mean(1)
    assert lost.max() > 4 * (G + 2) * 2.0 ** -24
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    kk.workspace_init(ws)
    out, logits = torch.zeros_like(q), torch.zeros((1, H, cap), device="cuda")
    kk.decode_attn_quant(lay, c, q, out, logits, None, ws)
    torch.cuda.synchronize()
    scale = U.f32(lay.scale)
    for h in range(H):
        mean = x[h * G:(h + 1) * G].astype(np.float64).mean()
        want = scale * mean * keys[:, where[h]]
        got = logits[0, h, :n].cpu().numpy().astype(np.float64)
        assert (np.abs(got - want) <= (G + 2) * 2.0 ** -24 * np.abs(want)).all(), (h, float((np.abs(got - want) / np.abs(want)).max() * 2 ** 24))
