"""Caches held in 8 bits on the GPU: quantising, appending, reading back, attention and decode steps against the 64-bit oracle."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import quant_oracle as Q
from paper_2504_09936_amd import workloads as W
from tests import gpu_util as U
from tests import quant_util as T

pytestmark = pytest.mark.gpu
ALPHA = U.f32(0.9)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def check_head(c, b, h, want_k, want_v):
    """One head's codes and scales are the oracle's."""
    for (got, sc), (want, ws) in zip(T.head(c, b, h), (want_k, want_v)):
        np.testing.assert_array_equal(sc, ws)
        T.same_values(got, want)


# ------------------------------------------------------------------------------------------------ quantising, reading back
def check_quantize_and_back(lens, cap, more, D, dtype):
    kk = U.kk()
    g = gen(cap * D)
    B, H = lens.shape
    lay = T.layout(B, H, 2, D, dtype)
    src, dst = kk.Cache(lay, cap), kk.QuantCache(lay, cap + more)
    src.k.copy_(T.rows(g, src.k.shape, dtype, 8.0))
    src.v.copy_(T.rows(g, src.v.shape, dtype, 8.0) * 1e-3)
    src.len.copy_(lens)
    src.votes.random_(1, 9, generator=g)
    src.log_s.normal_(generator=g)
    src.born.random_(0, 9, generator=g)
    src.t_obs.random_(0, 9, generator=g)
    dead = (torch.arange(cap) >= lens.unsqueeze(-1)).cuda()
    src.k[dead] = float("nan")                              # dead rows are masked out, whatever they hold
    src.v[dead] = float("inf")
    for f in dst.FIELDS:
        T.bits(getattr(dst, f)).fill_(0x5A)
    before = T.raw(dst)
    kk.quantize(lay, src, dst)
    after = T.raw(dst)
    assert torch.equal(dst.len.cpu(), lens) and torch.equal(dst.t_obs, src.t_obs)
    for b in range(B):
        for h in range(H):
            n = int(lens[b, h])
            check_head(dst, b, h, Q.quantize(U.to_host(src.k)[b, h, :n]), Q.quantize(U.to_host(src.v)[b, h, :n]))
            for f in ("votes", "log_s", "born"):
                assert torch.equal(getattr(dst, f)[b, h, :n], getattr(src, f)[b, h, :n]), f
            for f in ("k", "v", "votes", "log_s", "born", "k_scale", "v_scale"):                # what is dead stays
                a, z = (x[f].view(B, H, -1)[b, h] for x in (after, before))
                live = -(-n // 32) if "scale" in f else n
                per = a.numel() // (-(-(cap + more) // 32) if "scale" in f else cap + more)
                assert torch.equal(a[live * per:], z[live * per:]), f
    back = kk.Cache(lay, cap + more + 7)
    for f in back.FIELDS:
        T.bits(getattr(back, f)).fill_(0x33)
    kk.dequantize(lay, dst, back)
    torch.cuda.synchronize()
    for b in range(B):
        for h in range(H):
            n = int(lens[b, h])
            (kc, ks), (vc, vs) = T.head(dst, b, h)
            np.testing.assert_array_equal(U.to_host(back.k)[b, h, :n], Q.values(kc, ks) if n else np.zeros((0, D)))
            np.testing.assert_array_equal(U.to_host(back.v)[b, h, :n], Q.values(vc, vs) if n else np.zeros((0, D)))
            for f in ("votes", "log_s", "born"):
                assert torch.equal(getattr(back, f)[b, h, :n], getattr(src, f)[b, h, :n]), f
            for f in ("k", "v", "votes", "log_s", "born"):
                rest = T.bits(getattr(back, f)[b, h, n:])
                assert (rest == 0x33).all(), f
    assert torch.equal(back.len, src.len) and torch.equal(back.t_obs, src.t_obs)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap,more", [(1, 0), (31, 5), (32, 0), (33, 64), (100, 3), (513, 0)])
def test_quantize_and_back(cap, more, D, dtype):
    check_quantize_and_back(torch.tensor([[0, 1, cap], [cap // 2, max(0, cap - 1), min(cap, 32)]], dtype=torch.int32), cap, more, D, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_quantize_and_back_many_heads(D, dtype):
    """More blocks than are read ahead of the lengths."""
    lens = torch.randint(0, 301, (16, 8), generator=torch.Generator().manual_seed(D), dtype=torch.int32)
    lens[0] = torch.tensor([0, 1, 31, 32, 33, 288, 299, 300])
    check_quantize_and_back(lens, 300, 9, D, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_extreme_rows(dtype):
    """Zeros, the largest and the smallest numbers of the type, infinities and NaN among others, every rounding of a block."""
    kk = U.kk()
    lay = T.layout(1, 1, 1, 64, dtype)
    cap = 32 * 8
    x = torch.zeros(cap, 64)
    x[32] = 3.3e38                                          # the largest scale
    x[33] = 1.0
    x[64] = 1e-42 if dtype == "f32" else 1e-38
    x[65, :3] = torch.tensor([1e-30, -1e-36, 0.0])
    x[96] = torch.linspace(-448, 448, 64)
    x[97, ::2] = float("inf")
    x[98, 1::2] = float("nan")
    x[99, 5] = float("-inf")
    t = torch.from_numpy(Q.VALUES[:127])                    # ties between neighbours: to the even one
    x[128:130].view(-1)[:126] = ((t[1:] + t[:-1]) / 2).float()
    x[130:132].view(-1)[:127] = -t.float()
    x[160] = 448.0
    x[192] = 449.0
    x[224] = float("nan")                                   # nothing finite
    src, dst = kk.Cache(lay, cap), kk.QuantCache(lay, cap)
    src.k.copy_(x.view(1, 1, cap, 64))
    src.v.copy_(-x.view(1, 1, cap, 64).flip(2))
    src.len.fill_(cap)
    kk.quantize(lay, src, dst)
    torch.cuda.synchronize()
    check_head(dst, 0, 0, Q.quantize(U.to_host(src.k)[0, 0]), Q.quantize(U.to_host(src.v)[0, 0]))


# ------------------------------------------------------------------------------------------------ appending
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("tokens,cap", [(1, 70), (2, 70), (33, 70), (40, 200), (150, 400)])
def test_append(tokens, cap, D, dtype):
    kk = U.kk()
    g = gen(tokens * D)
    lay = T.layout(2, 4, 1, D, dtype)
    lens = np.array([[0, 1, 31, 32], [33, 60, cap - 1, cap]])
    for counts in (None, [[tokens, 0, 1, tokens], [tokens // 2, -3, tokens + 9, tokens]]):
        c = T.state(g, lay, cap, lens)
        k_t = T.rows(g, (2, 4, tokens, D), dtype, 6.0)      # some need larger scales than the cache has
        v_t = T.rows(g, (2, 4, tokens, D), dtype, 6.0)
        k_t[0, 2] *= 1e4                                    # this one surely: old codes become subnormal and zero
        v_t[1, 0] *= 1e-4                                   # and this one surely not
        if tokens > 1:
            k_t[0, 0, 1, 3], v_t[0, 0, 0, 7] = float("inf"), float("nan")
        want = [[[Q.append(*x, U.to_host(t)[b, h, :max(0, min(tokens if counts is None else counts[b][h], tokens, cap - lens[b, h]))])
                  for x, t in zip(T.head(c, b, h), (k_t, v_t))] for h in range(4)] for b in range(2)]
        before = T.raw(c)
        overflow = torch.zeros(1, dtype=torch.int32, device="cuda")
        kk.append_quant(lay, c, k_t, v_t, tokens, None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda"), overflow)
        after = T.raw(c)
        took = 0
        for b in range(2):
            for h in range(4):
                n0, n = lens[b, h], int(c.len[b, h])
                asked = tokens if counts is None else max(0, min(tokens, counts[b][h]))
                assert n == min(cap, n0 + asked)
                took += n0 + asked - n
                check_head(c, b, h, *want[b][h])
                assert (c.votes[b, h, n0:n] == 1).all() and torch.isneginf(c.log_s[b, h, n0:n]).all() and (c.born[b, h, n0:n] == 9).all()
                for f in ("k", "v", "votes", "log_s", "born", "k_scale", "v_scale"):
                    a, z = (x[f].view(2, 4, -1)[b, h] for x in (after, before))
                    slots = -(-cap // 32) if "scale" in f else cap
                    per, live = a.numel() // slots, -(-n // 32) if "scale" in f else n
                    assert torch.equal(a[live * per:], z[live * per:]), f
                    if f in ("votes", "log_s", "born"):
                        assert torch.equal(a[:n0 * per], z[:n0 * per]), f
        assert int(overflow) == (took > 0)


# ------------------------------------------------------------------------------------------------ attention
SHAPES = [  # B, H, G, D, dtype, capacity, lengths, slots per split
    (1, 4, 1, 64, "f32", 84, [[52, 0, 1, 84]], 0),
    (1, 1, 8, 128, "bf16", 1, [[1]], 0),
    (2, 3, 2, 128, "bf16", 333, [[0, 1, 31], [32, 33, 333]], 0),
    (2, 8, 4, 128, "bf16", 884, 852, 0),
    (1, 2, 4, 64, "bf16", 5003, [[5003, 2500]], 0),
    (1, 2, 4, 64, "f32", 5003, [[65, 4999]], 128),
    (1, 3, 8, 128, "f32", 700, [[700, 64, 699]], 96),
    (1, 8, 8, 128, "bf16", 2000, 1999, 0),
    (1, 1, 1, 128, "bf16", 40000, 39990, 0),
    (3, 2, 2, 64, "bf16", 257, [[257, 256], [255, 225], [224, 223]], 64),
    (40, 8, 4, 64, "bf16", 130, 129, 0),
]


def check_attention(lay, c, q, out, logits, lse, name=""):
    """Every head, or for many heads a spread of them."""
    torch.cuda.synchronize()
    G = lay.n_q_heads // lay.n_kv_heads
    units = [(b, h) for b in range(lay.batch) for h in range(lay.n_kv_heads)]
    for b, h in units[::max(1, len(units) // 16)]:
        (o, l, x), (eo, el, ex) = T.attention(c, lay, q, b, h)
        got = U.to_host(out)[b, h * G:(h + 1) * G]
        assert (np.abs(got - o) <= eo).all(), (name, b, h, float((np.abs(got - o) / np.maximum(eo, 1e-300)).max()))
        if lse is not None:
            gl = lse[b, h * G:(h + 1) * G].cpu().numpy()
            np.testing.assert_array_equal(np.isneginf(gl), np.isneginf(l))
            fin = np.isfinite(l)
            assert (np.abs(gl[fin] - l[fin]) <= el[fin]).all(), (name, b, h)
        if logits is not None:
            gx = logits[b, h].cpu().numpy()
            assert (np.abs(gx[:len(x)] - x) <= ex).all(), (name, b, h)


@pytest.mark.parametrize("B,H,G,D,dtype,cap,lens,per", SHAPES)
def test_attention(B, H, G, D, dtype, cap, lens, per):
    kk = U.kk()
    g = gen(cap)
    lay = T.layout(B, H, G, D, dtype)
    c = T.state(g, lay, cap, lens, 2.0)
    c.plan_slots_per_split = per
    q = T.rows(g, (B, H * G, D), dtype) * 3
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda") if per else kk.new_workspace(lay, cap, cap)
    kk.workspace_init(ws)
    for hint in (0, int(c.len.max())):
        c.len_hint = hint
        out, lse = torch.full_like(q, 7.0), torch.full((B, H * G), 7.0, device="cuda")
        logits = torch.full((B, H, cap), 7.0, device="cuda")
        before = T.raw(c)
        kk.decode_attn_quant(lay, c, q, out, logits, lse, ws)
        check_attention(lay, c, q, out, logits, lse, f"hint {hint}")
        dead = torch.arange(cap, device="cuda") >= c.len.unsqueeze(-1)
        assert (logits[dead] == 7.0).all()
        for f, x in T.raw(c).items():
            assert torch.equal(x, before[f]), f
        again = torch.full_like(q, 7.0)
        kk.decode_attn_quant(lay, c, q, again, None, None, ws)
        assert torch.equal(T.bits(out), T.bits(again))
        assert not ws[:64 * 1024 + 256].any()


@pytest.mark.parametrize("G,D,dtype", [(1, 64, "f32"), (2, 128, "f32"), (4, 128, "bf16"), (8, 64, "bf16"), (1, 128, "bf16"), (2, 64, "bf16"),
                                       (4, 64, "f32"), (8, 128, "f32")])
@pytest.mark.parametrize("waves,per", [(4, 64), (4, 128), (4, 256), (8, 256), (8, 512), (4, 1024)])
def test_attention_by_plan(waves, per, G, D, dtype):
    """Every launch shape on ragged heads."""
    kk = U.kk()
    g = gen(per + waves)
    lay = T.layout(2, 4, G, D, dtype)
    cap = 1000
    c = T.state(g, lay, cap, [[1000, 999, 513, 512], [1, 0, 700, 260]], 2.0)
    c.plan_slots_per_split, c.plan_wavefronts = per, waves
    q = T.rows(g, (2, 4 * G, D), dtype) * 3
    out, lse, logits = torch.zeros_like(q), torch.zeros((2, 4 * G), device="cuda"), torch.zeros((2, 4, cap), device="cuda")
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    kk.workspace_init(ws)
    kk.decode_attn_quant(lay, c, q, out, logits, lse, ws)
    check_attention(lay, c, q, out, logits, lse)


def test_nan_in_a_live_slot_stays_in_its_head():
    kk = U.kk()
    g = gen(5)
    lay = T.layout(1, 2, 2, 64, "bf16")
    c = T.state(g, lay, 100, 90)
    c.v.view(torch.uint8)[0, 0, 40, 3] = T.NAN_CODE
    q = T.rows(g, (1, 4, 64), "bf16")
    out = torch.zeros_like(q)
    kk.decode_attn_quant(lay, c, q, out, None, None, kk.new_workspace(lay, 100, 100))
    torch.cuda.synchronize()
    assert torch.isnan(out[0, :2, 3]).all() and torch.isfinite(out[0, 2:]).all()
    assert torch.isnan(out).sum() == 2


# ------------------------------------------------------------------------------------------------ decode steps
def check_step(lay, c, before, q, k_t, v_t, out, logits, name):
    """`before`: a copy of the cache as it was.  The new state and outputs against the oracle, then `c` for the next step."""
    torch.cuda.synchronize()
    cap, G = c.capacity, lay.n_q_heads // lay.n_kv_heads
    for b in range(lay.batch):
        for h in range(lay.n_kv_heads):
            n0 = int(before.len[b, h])
            n = min(n0 + 1, cap)
            assert int(c.len[b, h]) == n, name
            new = slice(0, n - n0)
            check_head(c, b, h, *(Q.append(*x, U.to_host(t)[b, h][None][new]) for x, t in zip(T.head(before, b, h), (k_t, v_t))))
            (o, _, x), (eo, _, ex) = T.attention(c, lay, q, b, h)
            got = U.to_host(out)[b, h * G:(h + 1) * G]
            assert (np.abs(got - o) <= eo).all(), (name, b, h, float((np.abs(got - o) / np.maximum(eo, 1e-300)).max()))
            old = np.concatenate([before.log_s[b, h, :n0].cpu().numpy().astype(np.float64), np.full(n - n0, -np.inf)])
            r, er = T.ema(old, x, ALPHA)
            assert (np.abs(c.log_s[b, h, :n].cpu().numpy() - r) <= er + ex).all(), (name, b, h)
            if logits is not None:
                assert (np.abs(logits[b, h, :n].cpu().numpy() - x) <= ex).all(), (name, b, h)
            assert torch.equal(c.votes[b, h, :n0], before.votes[b, h, :n0]) and (c.votes[b, h, n0:n] == 1).all()
            assert torch.equal(c.born[b, h, :n0], before.born[b, h, :n0]) and (c.born[b, h, n0:n] == before.t_obs[b, h]).all()
            assert torch.equal(T.bits(c.log_s[b, h, n:]), T.bits(before.log_s[b, h, n:])), name
            for f in ("k", "v"):
                assert torch.equal(T.bits(getattr(c, f)[b, h, n:]), T.bits(getattr(before, f)[b, h, n:])), name
    assert torch.equal(c.t_obs, before.t_obs + 1)


def copy_of(kk, lay, c):
    o = kk.QuantCache(lay, c.capacity)
    for f in c.FIELDS:
        T.bits(getattr(o, f)).copy_(T.bits(getattr(c, f)))
    return o


@pytest.mark.parametrize("B,H,G,D,dtype,cap,lens,per,waves", [
    (1, 4, 1, 64, "f32", 84, [[52, 0, 31, 84]], 0, 0),
    (2, 4, 4, 128, "bf16", 300, [[0, 1, 31, 32], [33, 255, 299, 300]], 0, 0),
    (2, 4, 2, 64, "bf16", 300, [[64, 65, 95, 96], [127, 128, 256, 290]], 64, 4),
    (1, 8, 8, 128, "bf16", 884, [[852, 851, 863, 864, 865, 883, 884, 7]], 0, 0),
    (1, 8, 4, 128, "bf16", 1100, [[852, 1023, 1024, 1025, 255, 256, 512, 1099]], 256, 8),
    (1, 2, 1, 128, "bf16", 700, [[640, 479]], 512, 8),
    (1, 2, 4, 128, "f32", 700, [[640, 100]], 0, 0),
    (1, 2, 8, 64, "f32", 2000, [[1999, 1535]], 512, 4),
    (1, 2, 4, 128, "bf16", 2000, [[1800, 1535]], 1024, 4),
])
def test_step(B, H, G, D, dtype, cap, lens, per, waves):
    """Four steps in a row: an ordinary token, one that makes the scales grow, a tiny one, zeros."""
    kk = U.kk()
    g = gen(cap + D)
    lay = T.layout(B, H, G, D, dtype)
    c = T.state(g, lay, cap, lens, 2.0)
    c.plan_slots_per_split, c.plan_wavefronts = per, waves
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda") if per else kk.new_workspace(lay, cap, cap)
    kk.workspace_init(ws)
    overflow = torch.zeros(1, dtype=torch.int32, device="cuda")
    for i, factor in enumerate((1.0, 300.0, 1e-5, 0.0)):
        q = T.rows(g, (B, H * G, D), dtype) * 3
        k_t, v_t = T.rows(g, (B, H, D), dtype, 2.0), T.rows(g, (B, H, D), dtype) * factor
        k_t[:, 0] *= factor                                 # (K and V grow apart)
        before = copy_of(kk, lay, c)
        c.len_hint = int(c.len.max()) if i % 2 else 0
        out, logits = torch.full_like(q, 7.0), torch.full((B, H, cap), 7.0, device="cuda")
        kk.decode_step_quant(lay, c, q, k_t, v_t, out, logits if i < 2 else None, ALPHA, overflow, ws)
        check_step(lay, c, before, q, k_t, v_t, out, logits if i < 2 else None, f"step {i}")
        assert int(overflow) == int((before.len == cap).any())
        overflow.zero_()
        assert not ws[:64 * 1024 + 256].any()


@pytest.mark.parametrize("G,D,dtype,cap,per,waves", [(4, 128, "bf16", 1000, 0, 0), (1, 64, "bf16", 1000, 128, 4), (8, 128, "bf16", 1000, 256, 4),
                                                     (2, 128, "f32", 1000, 256, 4), (4, 64, "bf16", 1000, 1024, 8)])
def test_a_bound_far_above_the_lengths(G, D, dtype, cap, per, waves):
    """The caller's bound may be any number of slots too high: tiles behind the live ones are dead, their codes and scales NaN."""
    kk = U.kk()
    g = gen(61)
    lay = T.layout(1, 6, G, D, dtype)
    c = T.state(g, lay, cap, [[0, 1, 31, 64, 500, 999]], 2.0)
    c.plan_slots_per_split, c.plan_wavefronts = per, waves
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    kk.workspace_init(ws)
    q = T.rows(g, (1, 6 * G, D), dtype) * 3
    for hint in (cap, cap + 5000):
        c.len_hint = hint
        out, lse = torch.full_like(q, 7.0), torch.zeros((1, 6 * G), device="cuda")
        kk.decode_attn_quant(lay, c, q, out, None, lse, ws)
        check_attention(lay, c, q, out, None, lse)
        k_t, v_t = T.rows(g, (1, 6, D), dtype, 4.0), T.rows(g, (1, 6, D), dtype, 4.0)
        before = copy_of(kk, lay, c)
        kk.decode_step_quant(lay, c, q, k_t, v_t, out, None, ALPHA, None, ws)
        check_step(lay, c, before, q, k_t, v_t, out, None, f"hint {hint}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_a_token_that_is_not_finite(D, dtype):
    """Its codes are NaN where it is not finite, the scale comes from the rest, and its head alone is affected."""
    kk = U.kk()
    g = gen(62)
    lay = T.layout(1, 3, 2, D, dtype)
    c = T.state(g, lay, 100, [[40, 64, 41]])
    before = copy_of(kk, lay, c)
    k_t, v_t = T.rows(g, (1, 3, D), dtype, 4.0), T.rows(g, (1, 3, D), dtype, 4.0)
    v_t[0, 0, 5], v_t[0, 0, D - 1], v_t[0, 1] = float("inf"), float("nan"), float("-inf")
    q = T.rows(g, (1, 6, D), dtype)
    out = torch.zeros_like(q)
    kk.decode_step_quant(lay, c, q, k_t, v_t, out, None, ALPHA, None, kk.new_workspace(lay, 100, 100))
    torch.cuda.synchronize()
    for h in range(3):
        check_head(c, 0, h, *(Q.append(*x, U.to_host(t)[0, h][None]) for x, t in zip(T.head(before, 0, h), (k_t, v_t))))
    nan = torch.isnan(out[0]).cpu()
    want = torch.zeros_like(nan)
    want[:2, 5] = want[:2, D - 1] = True
    want[2:4] = True
    assert torch.equal(nan, want)
    live = torch.arange(100, device="cuda") < c.len.unsqueeze(-1)
    assert torch.isfinite(c.log_s[live]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales_at_the_ends_of_their_range(dtype):
    """Blocks of the smallest and of very large rows in one head, zeros among them."""
    kk = U.kk()
    lay = T.layout(1, 2, 4, 64, dtype)
    g = gen(63)
    src, c = kk.Cache(lay, 256), kk.QuantCache(lay, 256)
    k, v = torch.randn(1, 2, 256, 64, generator=g, device="cuda"), torch.randn(1, 2, 256, 64, generator=g, device="cuda")
    factor = torch.tensor([2.0 ** e for e in (-120, -100, -60, 0, 30, 90, -126, 0)], device="cuda").repeat_interleave(32)
    v *= factor[:, None]
    k *= torch.where(factor > 1, torch.ones_like(factor), factor)[:, None]
    v[0, 1, 224:] = 0
    src.k.copy_(k)
    src.v.copy_(v)
    src.votes.fill_(1)
    src.len.fill_(250)
    kk.quantize(lay, src, c)
    q = T.rows(g, (1, 8, 64), dtype)
    out, lse = torch.zeros_like(q), torch.zeros((1, 8), device="cuda")
    kk.decode_attn_quant(lay, c, q, out, None, lse, kk.new_workspace(lay, 256, 256))
    check_attention(lay, c, q, out, None, lse)
    torch.cuda.synchronize()
    for h in range(2):
        check_head(c, 0, h, Q.quantize(U.to_host(src.k)[0, h, :250]), Q.quantize(U.to_host(src.v)[0, h, :250]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("per", [0, 64])
def test_slots_without_votes(per, dtype):
    """A live slot with no votes has weight zero; a head of nothing but such slots gives what keepkv_decode_attn gives on its rows."""
    kk = U.kk()
    g = gen(71)
    lay = T.layout(1, 3, 4, 128, dtype)
    c = T.state(g, lay, 300, [[300, 290, 97]], 2.0)
    c.plan_slots_per_split = per
    c.votes[0, 0, 5:200] = 0
    c.votes[0, 1, :290] = 0
    c.votes[0, 2, 96] = 0
    q = T.rows(g, (1, 12, 128), dtype) * 3
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    kk.workspace_init(ws)
    out, lse = torch.full_like(q, 7.0), torch.full((1, 12), 7.0, device="cuda")
    kk.decode_attn_quant(lay, c, q, out, None, lse, ws)
    r = kk.Cache(lay, 300)
    kk.dequantize(lay, c, r)
    want, want_lse = torch.full_like(q, 7.0), torch.full((1, 12), 7.0, device="cuda")
    kk.decode_attn(lay, r, q, want, None, want_lse, ws)
    torch.cuda.synchronize()
    assert torch.equal(out[0, 4:8], want[0, 4:8]) and torch.equal(lse[0, 4:8], want_lse[0, 4:8])
    with np.errstate(divide="ignore"):
        for h in (0, 2):
            (o, l, _), (eo, el, _) = T.attention(c, lay, q, 0, h)
            assert (np.abs(U.to_host(out)[0, 4 * h:4 * h + 4] - o) <= eo).all(), h
            assert (np.abs(lse[0, 4 * h:4 * h + 4].cpu().numpy() - l) <= el).all(), h


@pytest.mark.parametrize("seed", range(40))
def test_random_shapes(seed):
    """Attention and two steps on a shape, lengths, a bound on them and a plan drawn at random."""
    kk = U.kk()
    rng, g = np.random.default_rng(seed), gen(1000 + seed)
    dtype, D, G = str(rng.choice(["bf16", "bf16", "f32"])), int(rng.choice([64, 128])), int(rng.choice([1, 2, 4, 8]))
    B, H = (int(x) for x in rng.integers(1, [4, 9]))
    cap = int(2 ** rng.uniform(0, 11.5))
    lay = T.layout(B, H, G, D, dtype)
    lens = np.where(rng.random((B, H)) < 0.2, rng.choice([0, 1, cap], (B, H)), rng.integers(0, cap + 1, (B, H)))
    c = T.state(g, lay, cap, lens, float(rng.choice([1.0, 2.0, 8.0])))
    if rng.random() < 0.6:
        c.plan_slots_per_split, c.plan_wavefronts = int(rng.choice([0, 64, 96, 128, 320, 512, 2048])), int(rng.choice([0, 4, 8]))
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    kk.workspace_init(ws)
    hints = [0, int(lens.max()) + 1, cap + 3]
    q = T.rows(g, (B, H * G, D), dtype, 2.0)
    out, lse, logits = torch.full_like(q, 7.0), torch.full((B, H * G), 7.0, device="cuda"), torch.full((B, H, cap), 7.0, device="cuda")
    c.len_hint = hints[seed % 3]
    kk.decode_attn_quant(lay, c, q, out, logits, lse, ws)
    check_attention(lay, c, q, out, logits, lse, f"seed {seed}")
    for i in range(2):
        k_t, v_t = T.rows(g, (B, H, D), dtype, 8.0), T.rows(g, (B, H, D), dtype, 8.0)
        before = copy_of(kk, lay, c)
        c.len_hint = hints[(seed + i) % 3]
        kk.decode_step_quant(lay, c, q, k_t, v_t, out, logits if i else None, ALPHA, None, ws)
        check_step(lay, c, before, q, k_t, v_t, out, logits if i else None, f"seed {seed} step {i}")
    assert not ws[:64 * 1024 + 256].any()


def test_one_workspace_for_caches_of_many_shapes():
    """In turn on one stream: every call leaves the control words clear for the next one."""
    kk = U.kk()
    g = gen(64)
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    ws.random_(0, 256, generator=g)
    kk.workspace_init(ws)
    for B, H, G, D, dtype, cap in [(2, 8, 4, 128, "bf16", 884), (1, 4, 1, 64, "f32", 700), (1, 8, 8, 64, "bf16", 3000), (5, 3, 2, 128, "bf16", 200),
                                   (1, 8, 4, 128, "bf16", 884)]:
        lay = T.layout(B, H, G, D, dtype)
        assert kk.workspace_bytes(lay, cap, cap) <= ws.numel()
        c = T.state(g, lay, cap, cap - 9)
        before = copy_of(kk, lay, c)
        q, k_t, v_t = T.rows(g, (B, H * G, D), dtype), T.rows(g, (B, H, D), dtype), T.rows(g, (B, H, D), dtype)
        out = torch.zeros_like(q)
        kk.decode_step_quant(lay, c, q, k_t, v_t, out, None, ALPHA, None, ws)
        check_step(lay, c, before, q, k_t, v_t, out, None, str((B, H, G, D)))
        assert not ws[:64 * 1024 + 256].any()


def test_step_equals_its_three_calls():
    kk = U.kk()
    g = gen(11)
    for dtype in ("bf16", "f32"):
        lay = T.layout(2, 4, 4, 128, dtype)
        a = T.state(g, lay, 500, [[0, 31, 32, 200], [255, 256, 499, 500]])
        b = copy_of(kk, lay, a)
        ws = kk.new_workspace(lay, 500, 500)
        for i in range(40):
            q = T.rows(g, (2, 16, 128), dtype)
            k_t, v_t = T.rows(g, (2, 4, 128), dtype, 2.0), T.rows(g, (2, 4, 128), dtype, 2.0)
            oa, ob, logits = torch.zeros_like(q), torch.zeros_like(q), torch.zeros((2, 4, 500), device="cuda")
            kk.decode_step_quant(lay, a, q, k_t, v_t, oa, None, ALPHA, None, ws)
            kk.append_quant(lay, b, k_t, v_t)
            kk.decode_attn_quant(lay, b, q, ob, logits, None, ws)
            kk.score(lay, b, logits, ALPHA)
        torch.cuda.synchronize()
        for f in a.FIELDS:
            if f == "log_s":                                # 40 updates, each off by at most 2^-20 and some steps of f32
                live = torch.arange(500, device="cuda") < a.len.unsqueeze(-1)
                assert (a.log_s - b.log_s)[live].abs().max() <= 40 * 2.0 ** -19
            else:
                assert torch.equal(T.bits(getattr(a, f)), T.bits(getattr(b, f))), f
        # the same sums in another order: within the bounds of check_attention on both sides
        check_attention(lay, a, q, oa, None, None)
        check_attention(lay, b, q, ob, None, None)


# ------------------------------------------------------------------------------------------------ as a program uses them
def test_a_run_of_them_together():
    """Prompt, first event, quantise, decode steps, back to rows, a steady event, quantise, steps: every stage against the oracle."""
    from oracle import keepkv_oracle as O
    kk = U.kk()
    w = W.CONFIGS["llama3_8b"].scaled(batch=1, context=400, period=8, window=4)
    lay = U.layout_of(w)
    K, V = W.make_cache(w, 3)
    _, big = U.new_cache(w, capacity=400, K=K, V=V)
    cap = w.budget + w.period
    ws = kk.new_workspace(lay, 400, w.budget)
    keep = torch.zeros(1, 8, w.budget, dtype=torch.int32, device="cuda")
    n_ev, dropped = torch.zeros(1, 8, dtype=torch.int32, device="cuda"), torch.zeros(1, 8, dtype=torch.int64, device="cuda")

    def event(src, dst):
        evict = torch.zeros(1, 8, src.capacity - w.budget, dtype=torch.int32, device="cuda")
        match = torch.zeros_like(evict)
        kk.select(lay, src, w.budget, w.n_sink, w.n_recent, ALPHA, keep, evict, n_ev, ws)
        kk.match(lay, src, w.budget, keep, evict, n_ev, -2.0, match, None, ws)
        kk.merge(lay, src, dst, w.budget, keep, evict, n_ev, match, ALPHA, dropped, ws)

    q_win = np.stack([W.make_query(w, 3, t - 4) for t in range(4)], axis=2)
    kk.score_window(lay, big, U.to_device(q_win, "bf16"), 4, ALPHA, -1)
    small, other = kk.Cache(lay, cap), kk.Cache(lay, cap)
    event(big, small)
    c = kk.QuantCache(lay, cap)
    kk.quantize(lay, small, c)
    out = torch.zeros(1, 32, 128, dtype=torch.bfloat16, device="cuda")
    for t in range(2 * w.period):
        q, (k_t, v_t) = U.to_device(W.make_query(w, 3, t), "bf16"), (U.to_device(x, "bf16") for x in W.make_token(w, 3, t))
        before = copy_of(kk, lay, c)
        c.len_hint = w.budget + t % w.period
        kk.decode_step_quant(lay, c, q, k_t, v_t, out, None, ALPHA, None, ws)
        check_step(lay, c, before, q, k_t, v_t, out, None, f"step {t}")
        if (t + 1) % w.period:
            continue
        # the event: selection on the codes' state gives what it gives on rows, then rows are merged and quantised
        by_codes = torch.zeros_like(keep), torch.zeros(1, 8, w.period, dtype=torch.int32, device="cuda"), torch.zeros_like(n_ev)
        kk.select(lay, c, w.budget, w.n_sink, w.n_recent, ALPHA, *by_codes, ws)
        rows = kk.Cache(lay, cap)
        kk.dequantize(lay, c, rows)
        oc = U.download(rows)
        event(rows, other)
        trace = O.compress(oc, w.budget, w.n_sink, w.n_recent, ALPHA, U.f32(-2.0), exact_any_order=True, storage_round=W.round_bf16)
        assert torch.equal(by_codes[0], keep)
        for h, (rk, _, _) in enumerate(trace):
            assert (keep[0, h].cpu().numpy() == rk).all()
        assert (other.votes[:, :, :w.budget].cpu().numpy() == oc.votes[:, :, :w.budget]).all()
        kk.quantize(lay, other, c)
        torch.cuda.synchronize()
        for h in range(8):
            check_head(c, 0, h, Q.quantize(U.to_host(other.k)[0, h, :w.budget]), Q.quantize(U.to_host(other.v)[0, h, :w.budget]))
    total = c.votes[:, :, :w.budget].sum(-1) + dropped
    assert (total == 400 + 2 * w.period).all()


def test_graph_replays_and_streams():
    """Append, step and both conversions captured; replayed with eager work between; the same on a stream of its own."""
    kk = U.kk()
    g = gen(21)
    lay = T.layout(2, 8, 4, 128, "bf16")
    cap = 600
    c = T.state(g, lay, cap, [[500, 31, 32, 0, 480, 479, 511, 512]] * 2)
    rows, back = kk.Cache(lay, cap), kk.QuantCache(lay, cap)
    ws = kk.new_workspace(lay, cap, cap)
    q = T.rows(g, (2, 32, 128), "bf16")
    k_t, v_t = T.rows(g, (2, 8, 128), "bf16", 3.0), T.rows(g, (2, 8, 128), "bf16", 3.0)
    k_n, v_n = T.rows(g, (2, 8, 5, 128), "bf16", 3.0), T.rows(g, (2, 8, 5, 128), "bf16", 3.0)
    out, out2 = torch.zeros_like(q), torch.zeros_like(q)
    start = copy_of(kk, lay, c)

    def restore():
        for f in c.FIELDS:
            T.bits(getattr(c, f)).copy_(T.bits(getattr(start, f)))

    def body():
        kk.decode_step_quant(lay, c, q, k_t, v_t, out, None, ALPHA, None, ws)
        kk.append_quant(lay, c, k_n, v_n, 5)
        kk.decode_attn_quant(lay, c, q, out2, None, None, ws)
        kk.dequantize(lay, c, rows)
        kk.quantize(lay, rows, back)

    def results():
        torch.cuda.synchronize()
        return [T.bits(x).clone() for x in (out, out2, *(getattr(c, f) for f in c.FIELDS), *(getattr(back, f) for f in back.FIELDS),
                                            *(getattr(rows, f) for f in rows.FIELDS))]

    body()
    want = results()
    graph = torch.cuda.CUDAGraph()
    restore()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        body()
    for _ in range(4):
        restore()
        out.normal_()
        out2.zero_()
        torch.cuda.synchronize()
        graph.replay()
        for a, b in zip(results(), want):
            assert torch.equal(a, b)
    stream = torch.cuda.Stream()
    restore()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        body()
    for a, b in zip(results(), want):
        assert torch.equal(a, b)


def test_two_caches_on_two_streams_with_workspaces_of_their_own():
    kk = U.kk()
    g = gen(22)
    lay = T.layout(1, 8, 4, 128, "bf16")
    cs = [T.state(g, lay, 900, 800) for _ in range(2)]
    twins = [copy_of(kk, lay, c) for c in cs]
    ws = [kk.new_workspace(lay, 900, 900) for _ in range(2)]
    q = T.rows(g, (1, 32, 128), "bf16")
    k_t, v_t = T.rows(g, (1, 8, 128), "bf16"), T.rows(g, (1, 8, 128), "bf16")
    outs = [torch.zeros_like(q) for _ in range(4)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(30):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                kk.decode_step_quant(lay, cs[i], q, k_t, v_t, outs[i], None, ALPHA, None, ws[i])
    torch.cuda.synchronize()
    for i in range(2):
        for _ in range(30):
            kk.decode_step_quant(lay, twins[i], q, k_t, v_t, outs[2 + i], None, ALPHA, None, ws[0])
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(T.bits(outs[i]), T.bits(outs[2 + i]))
        for f in cs[i].FIELDS:
            assert torch.equal(T.bits(getattr(cs[i], f)), T.bits(getattr(twins[i], f))), f


def test_offsets_beyond_32_bits():
    """40 heads of 2^20 slots: the last head's codes begin at 5.1e9 bytes, the rows of its bf16 image at 1e10."""
    kk = U.kk()
    g = gen(31)
    H, cap, D = 40, 1 << 20, 128
    lay = T.layout(1, H, 1, D, "bf16")
    small = T.layout(1, 1, 1, D, "bf16")
    c = kk.QuantCache(lay, cap)
    one = T.state(g, small, 100, 70)
    for f in c.FIELDS:
        src = getattr(one, f)[0, 0]
        dst = getattr(c, f)[0, H - 1]
        (dst[:len(src)] if src.dim() else dst).copy_(src)
    c.votes[0, H - 2] = 1                                   # the head before: full but for one slot, zero codes
    c.log_s[0, H - 2] = 0.0
    c.len[0, H - 2] = cap - 1
    ws = kk.new_workspace(lay, cap, cap)
    q = T.rows(g, (1, H, D), "bf16")
    k_t, v_t = T.rows(g, (1, H, D), "bf16"), T.rows(g, (1, H, D), "bf16")
    out = torch.zeros_like(q)
    kk.decode_step_quant(lay, c, q, k_t, v_t, out, None, ALPHA, None, ws)
    kk.append_quant(lay, c, k_t, v_t)
    rows = kk.Cache(lay, cap)
    kk.dequantize(lay, c, rows)
    kk.append_quant(small, one, k_t[:, H - 1:].contiguous(), v_t[:, H - 1:].contiguous())
    o1 = torch.zeros(1, 1, D, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    n = 71
    assert int(c.len[0, H - 1]) == 72 and int(c.len[0, H - 2]) == cap
    for f in ("k", "v", "k_scale", "v_scale", "votes"):
        m = n if f in ("k", "v", "votes") else 3
        assert torch.equal(T.bits(getattr(c, f)[0, H - 1, :m]), T.bits(getattr(one, f)[0, 0, :m])), f
    (o, _, _), (eo, _, _) = T.attention(one, small, q[:, H - 1:], 0, 0)
    assert (np.abs(U.to_host(out)[0, H - 1:] - o) <= eo).all()
    (kc, ks), _ = T.head(c, 0, H - 1)
    np.testing.assert_array_equal(U.to_host(rows.k[0, H - 1, :72]), Q.values(kc, ks))
    want = Q.quantize(U.to_host(k_t)[0, H - 2:H - 1])
    last = Q.append(np.zeros((31, D), np.uint8), np.array([2.0 ** 0]), U.to_host(k_t)[0, H - 2:H - 1])   # (the scale there was 1)
    T.same_values(T.codes(c.k[0, H - 2, -1:]), last[0][31:])
    assert float(c.k_scale[0, H - 2, -1]) == max(1.0, want[1][0])
    np.testing.assert_array_equal(U.to_host(rows.k[0, H - 2, -1]), Q.values(*last)[31])
    back = kk.QuantCache(lay, cap)
    kk.quantize(lay, rows, back)
    torch.cuda.synchronize()
    assert torch.equal(back.len, c.len)
    got = [Q.VALUES[T.codes(x.k[0, h, :72])] * np.repeat(x.k_scale[0, h, :3].cpu().numpy(), 32)[:72, None] for x in (c, back) for h in (H - 1,)]
    np.testing.assert_array_equal(*got)


def test_dump_and_reload(tmp_path):
    kk = U.kk()
    lay = T.layout(1, 2, 2, 64, "bf16")
    c = T.state(gen(41), lay, 77, [[77, 30]])
    c.save(str(tmp_path / "c.pt"))
    o = kk.QuantCache(lay, 77)
    o.load(str(tmp_path / "c.pt"))
    for f in c.FIELDS:
        assert torch.equal(T.bits(getattr(c, f)), T.bits(getattr(o, f))), f
    with pytest.raises(ValueError):
        kk.QuantCache(lay, 78).load(str(tmp_path / "c.pt"))


def test_refused_on_device_buffers():
    """Nothing is launched and nothing touched."""
    kk = U.kk()
    lay = T.layout(1, 2, 2, 64, "bf16")
    c = T.state(gen(51), lay, 1000, 900)
    before = T.raw(c)
    q = T.rows(gen(1), (1, 4, 64), "bf16")
    kt = T.rows(gen(2), (1, 2, 64), "bf16")
    out = torch.full_like(q, 7.0)
    c.plan_slots_per_split = 64
    with pytest.raises(kk.KeepKVError) as e:                # needs partial results, has no room
        kk.decode_step_quant(lay, c, q, kt, kt, out, None, ALPHA, None, torch.zeros(1024, dtype=torch.uint8, device="cuda"))
    assert e.value.status == kk.ERR_WORKSPACE
    c.plan_slots_per_split = 0
    rows = kk.Cache(lay, 999)
    with pytest.raises(kk.KeepKVError) as e:
        kk.dequantize(lay, c, rows)
    assert e.value.status == kk.ERR_INVALID_ARG
    for call in (kk.match, kk.merge_inplace):
        with pytest.raises((TypeError, AttributeError)):
            call(lay, c, 10, None, None, None, 0.5, None, None, None) if call is kk.match else call(lay, c, None, 10, None, None, None, None, 0.9, None)
    torch.cuda.synchronize()
    assert (out == 7.0).all()
    for f, x in T.raw(c).items():
        assert torch.equal(x, before[f]), f
    assert C.sizeof(kk._QuantCache) == C.sizeof(kk._Cache) + 16
