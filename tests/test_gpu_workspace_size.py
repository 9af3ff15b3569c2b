"""Decode calls with a forced plan take exactly the workspace that the header names, write nothing behind it and refuse a byte less."""
import pytest
import torch

from tests import gpu_util as U
from tests import quant_util as T
from tests.test_gpu_quant import ALPHA, copy_of, gen

pytestmark = pytest.mark.gpu
HEAD = 64 * 1024 + 256


@pytest.mark.parametrize("H,G,D,dtype,cap,per", [(1, 4, 128, "bf16", 300, 64), (1, 1, 64, "f32", 500, 128), (3, 2, 64, "bf16", 700, 96), (8, 4, 128, "bf16", 900, 256)])
def test_the_documented_size(H, G, D, dtype, cap, per):
    kk = U.kk()
    g = gen(95)
    lay = T.layout(1, H, G, D, dtype)
    c = T.state(g, lay, cap, cap - 5)
    rows = kk.Cache(lay, cap)
    kk.dequantize(lay, c, rows)
    q, k_t, v_t = T.rows(g, (1, H * G, D), dtype), T.rows(g, (1, H, D), dtype), T.rows(g, (1, H, D), dtype)
    for cache, attn, step in ((c, kk.decode_attn_quant, kk.decode_step_quant), (rows, kk.decode_attn, kk.decode_step)):
        cache.plan_slots_per_split = per
        step_of = 32 if cache is c or dtype == "bf16" else 64         # what `per` is rounded down to
        n_split = -(-cap // (per // step_of * step_of))
        need = HEAD + H * G * n_split * (D + 2) * 4
        room = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
        roomy = torch.zeros(1 << 24, dtype=torch.uint8, device="cuda")
        ws = room[:need]
        kk.workspace_init(ws)
        got, want = torch.zeros_like(q), torch.zeros_like(q)
        attn(lay, cache, q, got, None, None, ws)
        attn(lay, cache, q, want, None, None, roomy)
        assert torch.equal(got, want)
        out = torch.full_like(q, 7.0)
        for call in (lambda w: attn(lay, cache, q, out, None, None, w), lambda w: step(lay, cache, q, k_t, v_t, out, None, ALPHA, None, w)):
            with pytest.raises(kk.KeepKVError) as e:
                call(room[:need - 1])
            assert e.value.status == kk.ERR_WORKSPACE
        torch.cuda.synchronize()
        assert (out == 7.0).all()
        step(lay, cache, q, k_t, v_t, out, None, ALPHA, None, ws)
        torch.cuda.synchronize()
        assert (room[need:] == 0x5A).all() and torch.isfinite(out.float()).all()


def test_other_sizes_are_covered():
    """keepkv_workspace_bytes is at least what an automatic plan's formula asks for, of every smaller cache too."""
    kk = U.kk()
    lay = kk.Layout(1, 4, 1, 128, kk.BF16, 0.1)
    for cap in (100, 300, 884, 5000):
        have = kk.workspace_bytes(lay, cap, cap)
        for plan in (kk.decode_plan, kk.decode_plan_quant):
            n = plan(lay, cap)[0]
            assert n == 1 or HEAD + 4 * n * 130 * 4 <= have
