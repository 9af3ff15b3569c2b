"""Plumbing of the tests of caches held in 8 bits: random states, the oracle's view of them, bounds on what a kernel may be off."""
import numpy as np
import torch

from oracle import keepkv_oracle as O
from oracle import quant_oracle as Q
from tests import gpu_util as U

NAN_CODE = 127


def layout(B, H, G, D, dtype):
    kk = U.kk()
    return kk.Layout(B, H * G, H, D, kk.BF16 if dtype == "bf16" else kk.F32, D ** -0.5)


def rows(gen, shape, dtype, spread=1.0):
    """Rows of the storage type with magnitudes that differ from row to row, on the GPU."""
    x = torch.randn(shape, generator=gen, device="cuda")
    if spread != 1.0:
        x *= spread ** torch.randn((*shape[:-1], 1), generator=gen, device="cuda")
    return x.bfloat16() if dtype == "bf16" else x


def bits(t):
    return t.contiguous().view(torch.uint8)


def raw(cache):
    """Every array of a cache as bytes."""
    torch.cuda.synchronize()
    return {f: bits(getattr(cache, f)).clone() for f in cache.FIELDS}


def codes(t):
    return t.view(torch.uint8).cpu().numpy()


def same_values(got, want):
    """Code arrays that stand for the same values (any NaN for any NaN, either zero)."""
    np.testing.assert_array_equal(Q.VALUES[got], Q.VALUES[want])


def state(gen, lay, cap, lens, spread=1.0):
    """A QuantCache with `lens` live slots per head ([B, H] list or array), written by the oracle, everything dead poisoned."""
    kk = U.kk()
    c = kk.QuantCache(lay, cap)
    B, H, D = lay.batch, lay.n_kv_heads, lay.head_dim
    lens = np.broadcast_to(np.asarray(lens, np.int32), (B, H)).copy()
    k, v = np.full((B, H, cap, D), NAN_CODE, np.uint8), np.full((B, H, cap, D), NAN_CODE, np.uint8)
    nb = -(-cap // Q.BLOCK)
    ks, vs = np.full((B, H, nb), np.nan, np.float32), np.full((B, H, nb), np.nan, np.float32)
    for x, s in ((k, ks), (v, vs)):
        r = rows(gen, (B, H, cap, D), "f32", spread).cpu().numpy()
        for b in range(B):
            for h in range(H):
                n = lens[b, h]
                x[b, h, :n], sc = Q.quantize(r[b, h, :n])
                s[b, h, :len(sc)] = sc
    dead = torch.arange(cap, device="cuda") >= torch.from_numpy(lens).cuda().unsqueeze(-1)
    c.k.view(torch.uint8).copy_(torch.from_numpy(k))
    c.v.view(torch.uint8).copy_(torch.from_numpy(v))
    c.k_scale.copy_(torch.from_numpy(ks))
    c.v_scale.copy_(torch.from_numpy(vs))
    c.votes.random_(1, 9, generator=gen)
    c.log_s.normal_(generator=gen)
    c.votes[dead] = -7
    c.log_s[dead] = float("nan")
    c.born.random_(0, 5, generator=gen)
    c.t_obs.fill_(9)
    c.len.copy_(torch.from_numpy(lens))
    return c


def head(c, b, h):
    """Codes and scales of one head's live slots, as the oracle holds them."""
    n = int(c.len[b, h])
    nb = -(-n // Q.BLOCK)
    return tuple((codes(x[b, h, :n]), s[b, h, :nb].cpu().numpy().astype(np.float64)) for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)))


EPS32 = 2.0 ** -24            # half a step of f32


def attention(c, lay, q, b, h):
    """Oracle attention of one head and how far a kernel that sums in f32 may be from it:
    (out [G, D], lse [G], mean logit [n]), (bounds on the same).

    With A = scale * sum_d |q_d k_d| at most over slots and heads, a logit is a sum of D exact products (D half steps of A), times
    the scales (3 more); so a weight and the sum of weights are each off by a factor within e^+-d, d = (D + 4) A EPS32 + |z| EPS32 for
    adding ln p and subtracting the maximum (|z| <= A + ln p), and the hardware's exp2 and log2 (2^-22 and, of ln p, 2^-22 of it).
    P is held in bf16 terms, two (2^-16) or, f32 layouts, three (2^-24), sums over n slots in f32 add n half steps: in all an output is off
    by at most w = 2 d + 2^-16 (2^-24) + 2^-21 + (n + 16) EPS32 times sum_i w_i |v_i|, before it is rounded to its type.

    Beside that, where all weights but one are below 2^-100: the 16 rows of the matrix product hold each head 16 / G times, a slot's
    weight in one of them and the smallest normal number, not zero, in the others, in each of the terms; a tile's sum is scaled by
    at most 1 and divided by a sum of weights of at least 1.  So (16 / G - 1) * 2 (3) * 2^-126 * sum_i |v_i| at most is added."""
    G, D = lay.n_q_heads // lay.n_kv_heads, lay.head_dim
    (kc, ks), (vc, vs) = head(c, b, h)
    n = len(kc)
    K, V = (Q.values(kc, ks), Q.values(vc, vs)) if n else (np.zeros((0, D)), np.zeros((0, D)))
    qh = U.to_host(q)[b, h * G:(h + 1) * G].astype(np.float64)
    votes = c.votes[b, h, :n].cpu().numpy()
    scale = U.f32(lay.scale)
    out, lse, mean = O.decode_attn(qh, K, V, votes, n, scale)
    if n == 0:
        return (out, lse, mean), (np.zeros((G, D)), np.zeros(G), np.zeros(0))
    A = scale * (np.abs(qh)[:, None, :] * np.abs(K)[None]).sum(-1).max()
    lp = np.log(votes.max())
    d = (D + 4) * A * EPS32 + 4 * (A + lp) * EPS32 + lp * 2.0 ** -22
    w = 2 * d + 2.0 ** (-16 if lay.dtype == U.kk().BF16 else -24) + 2.0 ** -21 + (n + 16) * EPS32
    z = scale * qh @ K.T + np.log(votes)
    p = np.exp(z - lse[:, None])
    half = 2.0 ** -8 if lay.dtype == U.kk().BF16 else EPS32
    e_out = half * np.abs(out) * (1 + w) + w * (p @ np.abs(V)) + (16 // G - 1) * (2 if lay.dtype == U.kk().BF16 else 3) * 2.0 ** -126 * (1 + half) * np.abs(V).sum(0) + 1e-38
    return (out, lse, mean), (e_out, d + (n + 16) * EPS32 + 2.0 ** -22 + np.abs(lse) * 4 * EPS32, np.full(n, (D + 6) * A * EPS32))


def ema(old, x, alpha):
    """ln(alpha e^old + (1 - alpha) e^x) and a bound: f32 operands and a hardware logarithm and exponential (2^-21 together)."""
    with np.errstate(divide="ignore"):
        r = np.logaddexp((np.log(alpha) if alpha > 0 else -np.inf) + old, np.log1p(-alpha) + x)
    size = np.maximum(np.abs(x), np.where(np.isfinite(old), np.abs(old), 0)) + 3
    return r, 4 * size * EPS32 + 2.0 ** -20
