"""Slots of weight zero add nothing to an output, however large their values are."""
import numpy as np
import pytest
import torch

from oracle import quant_oracle as Q
from tests import gpu_util as U
from tests import quant_util as T
from tests.test_gpu_quant import gen

pytestmark = pytest.mark.gpu
SHAPES = [(1, 64, 0, 0), (1, 128, 64, 4), (2, 128, 256, 4), (4, 128, 1024, 4), (8, 64, 512, 8)]


def run(G, D, per, waves, dtype, large):
    """Slots 32 .. 63 hold values of 2^large.  In head 0 they have no votes; in head 1 a logit of -300, whose weight vanishes beside 1 in any type.
    -> per head: output, oracle, bound.  Outputs are within a rounding (2^-8 of them covers bf16) and 2^-12 of sum_i w_i |v_i|, which is what
    softmax and sums lose with room."""
    kk = U.kk()
    g = gen(91)
    lay = T.layout(1, 2, G, D, dtype)
    c = T.state(g, lay, 300, 300)
    codes, scales = Q.quantize(np.full((32, D), 2.0 ** large))
    c.v.view(torch.uint8)[0, :, 32:64] = torch.from_numpy(codes).cuda()
    c.v_scale[0, :, 1] = float(scales[0])
    c.votes[0, 0, 32:64] = 0
    kc, ks = Q.quantize(np.full((32, D), -1.0))
    c.k.view(torch.uint8)[0, 1, 32:64] = torch.from_numpy(kc).cuda()
    c.k_scale[0, 1, 1] = float(ks[0])
    q = T.rows(g, (1, 2 * G, D), dtype)
    q[0, G:] = 300.0 / D ** 0.5
    c.k.view(torch.uint8)[0, 1, :32] = 0
    c.k.view(torch.uint8)[0, 1, 64:] = 0
    c.plan_slots_per_split, c.plan_wavefronts = per, waves
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    kk.workspace_init(ws)
    out = torch.zeros_like(q)
    kk.decode_attn_quant(lay, c, q, out, None, None, ws)
    torch.cuda.synchronize()
    for h in range(2):
        with np.errstate(divide="ignore"):
            (o, lse, _), _ = T.attention(c, lay, q, 0, h)
            (kc, ks), (vc, vs) = T.head(c, 0, h)
            z = lay.scale * U.to_host(q)[0, h * G:(h + 1) * G].astype(np.float64) @ Q.values(kc, ks).T + np.log(c.votes[0, h].cpu().numpy())
        size = np.exp(z - lse[:, None]) @ np.abs(Q.values(vc, vs))
        assert size.max() < 16
        yield U.to_host(out)[0, h * G:(h + 1) * G], o, 2.0 ** -8 * np.abs(o) + 2.0 ** -12 * size


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G,D,per,waves", SHAPES)
def test_huge_values_of_weight_zero(G, D, per, waves, dtype):
    """Values of 2^121: 32 of them are 2^126, which f32 holds."""
    for got, o, bound in run(G, D, per, waves, dtype, 121):
        assert (np.abs(got - o) <= bound).all(), float(np.abs(got - o).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G,D,per,waves", SHAPES)
def test_values_whose_sum_f32_does_not_hold(G, D, per, waves, dtype):
    """Values of 2^127.  Without votes their weights are zero in any sum.  By their logits they weigh 1 each in a sum over their tile alone, whose
    maximum is theirs: 32 * 2^127 = 2^132 is beyond f32, the sum is infinite, and its share of the head, 0 times that, NaN.  So the head's output
    is right where another tile's maximum came first, and NaN, never another number, where it did not."""
    first, second = run(G, D, per, waves, dtype, 127)
    got, o, bound = first
    assert (np.abs(got - o) <= bound).all(), float(np.abs(got - o).max())
    got, o, bound = second
    assert (np.isnan(got) | (np.abs(got - o) <= bound)).all()
