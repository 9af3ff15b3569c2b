"""What is not finite shows: a NaN in a live key or an infinite query makes NaN of its heads' outputs and of lse, and of no other head's."""
import numpy as np
import pytest
import torch

from tests import gpu_util as U
from tests import quant_util as T
from tests.test_gpu_quant import ALPHA, check_head, copy_of, gen
from oracle import quant_oracle as Q

pytestmark = pytest.mark.gpu
PLANS = [(1, 64, "f32", 0, 0), (2, 128, "bf16", 0, 0), (4, 128, "bf16", 256, 8), (8, 64, "bf16", 512, 8), (4, 128, "f32", 64, 4), (1, 128, "bf16", 1024, 4),
         (8, 128, "f32", 512, 4)]


def case(G, D, dtype, per, waves, H=8):
    kk = U.kk()
    g = gen(81)
    lay = T.layout(1, H, G, D, dtype)
    c = T.state(g, lay, 700, [[600, 555, 640, 33, 700, 64, 1, 690][:H]], 2.0)
    c.plan_slots_per_split, c.plan_wavefronts = per, waves
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    kk.workspace_init(ws)
    return kk, g, lay, c, T.rows(g, (1, H * G, D), dtype), ws


def check_only(lay, c, q, out, lse, heads):
    """The query heads `heads` are NaN, out and lse; all others are what the oracle gives."""
    torch.cuda.synchronize()
    G = lay.n_q_heads // lay.n_kv_heads
    bad = torch.zeros(lay.n_q_heads, dtype=torch.bool)
    bad[heads] = True
    assert torch.equal(torch.isnan(out[0]).all(-1).cpu(), bad) and torch.equal(torch.isnan(out[0]).any(-1).cpu(), bad)
    if lse is not None:
        assert torch.equal(torch.isnan(lse[0]).cpu(), bad)
    for h in range(lay.n_kv_heads):
        clean = [i for i in range(G) if not bad[h * G + i]]
        if clean:
            qh = torch.nan_to_num(q.float(), posinf=0.0, neginf=0.0).to(q.dtype)       # (heads of a group do not see each other's queries)
            (o, _, _), (eo, _, _) = T.attention(c, lay, qh, 0, h)
            assert (np.abs(U.to_host(out)[0, h * G:(h + 1) * G] - o) <= eo)[clean].all(), h


@pytest.mark.parametrize("G,D,dtype,per,waves", PLANS)
def test_a_key_code_that_is_nan(G, D, dtype, per, waves):
    kk, g, lay, c, q, ws = case(G, D, dtype, per, waves)
    c.k.view(torch.uint8)[0, 2, 317, 5] = T.NAN_CODE
    c.k.view(torch.uint8)[0, 6, 0, D - 1] = T.NAN_CODE                # the one slot of its head
    out, lse = torch.zeros_like(q), torch.zeros((1, lay.n_q_heads), device="cuda")
    kk.decode_attn_quant(lay, c, q, out, None, lse, ws)
    check_only(lay, c, q, out, lse, [h * G + i for h in (2, 6) for i in range(G)])
    assert not ws[:64 * 1024 + 256].any()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("G,D,dtype,per,waves", PLANS)
def test_a_token_whose_key_is_not_finite(G, D, dtype, per, waves, value):
    """Its codes are NaN where it is not finite, the scale comes from the rest."""
    kk, g, lay, c, q, ws = case(G, D, dtype, per, waves)
    k_t, v_t = T.rows(g, (1, 8, D), dtype, 4.0), T.rows(g, (1, 8, D), dtype, 4.0)
    k_t[0, 1, D // 2], k_t[0, 5] = value, value                       # one element, a whole row
    before = copy_of(kk, lay, c)
    out = torch.zeros_like(q)
    kk.decode_step_quant(lay, c, q, k_t, v_t, out, None, ALPHA, None, ws)
    check_only(lay, c, q, out, None, [h * G + i for h in (1, 5) for i in range(G)])
    for h in (0, 1, 5):
        check_head(c, 0, h, *(Q.append(*x, U.to_host(t)[0, h][None]) for x, t in zip(T.head(before, 0, h), (k_t, v_t))))


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("G,D,dtype,per,waves", PLANS)
def test_a_query_that_is_not_finite(G, D, dtype, per, waves, value):
    """Keys of both signs meet it (and zeros, whose product with infinity is NaN): the sum of weights is NaN, of this query head alone."""
    kk, g, lay, c, q, ws = case(G, D, dtype, per, waves)
    q[0, G - 1, 3] = value
    q[0, 4 * G] = value
    out, lse = torch.zeros_like(q), torch.zeros((1, lay.n_q_heads), device="cuda")
    kk.decode_attn_quant(lay, c, q, out, None, lse, ws)
    check_only(lay, c, q, out, lse, [G - 1, 4 * G])


@pytest.mark.parametrize("G,D,dtype,per,waves", PLANS + [(4, 128, "bf16", 128, -1)])
def test_rows_that_are_nan(G, D, dtype, per, waves):
    """The same of a cache of rows."""
    kk, g, lay, c, q, ws = case(G, D, dtype, per, 0 if waves < 0 else waves)
    rows = kk.Cache(lay, 700)
    kk.dequantize(lay, c, rows)
    rows.plan_slots_per_split, rows.plan_wavefronts = per, waves
    rows.k[0, 2, 317, 5] = float("nan")
    q[0, 4 * G, 1] = float("inf")
    out, lse = torch.zeros_like(q), torch.zeros((1, lay.n_q_heads), device="cuda")
    kk.decode_attn(lay, rows, q, out, None, lse, ws)
    torch.cuda.synchronize()
    bad = torch.zeros(lay.n_q_heads, dtype=torch.bool)
    bad[[2 * G + i for i in range(G)] + [4 * G]] = True
    assert torch.equal(torch.isnan(out[0]).all(-1).cpu(), bad) and torch.equal(torch.isnan(out[0]).any(-1).cpu(), bad)
    assert torch.equal(torch.isnan(lse[0]).cpu(), bad)
