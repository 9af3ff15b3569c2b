"""Host side of the caches held in 8 bits: refusals before anything is launched, plans, workspace sizes, what takes which cache."""
import ctypes as C

import pytest

from tests import gpu_util as U

P = C.c_void_p(16)
HEAD = 64 * 1024 + 256


def structs(kk, capacity=884, k=16, scale=16, **over):
    c = kk._Cache(k, 16, 16, 16, 16, 16, 16, capacity, 0, 0, 0)       # non-null dummies; never dereferenced on these paths
    for f, v in over.items():
        setattr(c, f, v)
    return c, kk._QuantCache(c, scale, 16)


def lay(kk, B=8, Hq=32, Hkv=8, D=128, dtype=1):
    return C.byref(kk.Layout(B, Hq, Hkv, D, dtype, 0.1).c())


def calls(kk, L, rows, codes, kt=P, q=P, out=P, ws_bytes=1 << 40, tokens=1, alpha=0.9):
    lib = kk._lib
    R, K = (None if x is None else C.byref(x) for x in (rows, codes))
    return {"quantize": lib.keepkv_quantize(L, R, K, None), "dequantize": lib.keepkv_dequantize(L, K, R, None),
            "append": lib.keepkv_append_quant(L, K, kt, kt, tokens, None, None, None),
            "attn": lib.keepkv_decode_attn_quant(L, K, q, out, None, None, P, ws_bytes, None),
            "step": lib.keepkv_decode_step_quant(L, K, q, kt, kt, out, None, C.c_float(alpha), None, P, ws_bytes, None)}


def test_refused_before_any_launch():
    kk = U.kk()
    rows, codes = structs(kk)
    bad = kk.ERR_INVALID_ARG
    assert set(calls(kk, None, rows, codes).values()) == {bad}
    assert set(calls(kk, lay(kk), None, None).values()) == {bad}
    assert set(calls(kk, lay(kk, Hq=30), rows, codes).values()) == {bad}
    for field in ("k", "v", "votes", "log_s", "born", "t_obs", "len"):
        assert set(calls(kk, lay(kk), *structs(kk, **{field: None})).values()) == {bad}, field
    assert set(calls(kk, lay(kk), rows, structs(kk, scale=None)[1]).values()) == {bad}
    assert set(calls(kk, lay(kk), *structs(kk, capacity=0)).values()) == {bad}
    assert set(calls(kk, lay(kk), *structs(kk, capacity=(1 << 20) + 1)).values()) == {bad}
    assert set(calls(kk, lay(kk), rows, structs(kk, k=24)[1]).values()) == {bad}                    # not aligned to 16 bytes
    r = calls(kk, lay(kk, Hq=24), rows, structs(kk, k=32, v=32)[1])                                 # groups of three
    assert set(r.values()) == {kk.ERR_UNSUPPORTED}
    r = calls(kk, lay(kk, D=96), rows, structs(kk, k=32, v=32)[1])
    assert set(r.values()) == {kk.ERR_UNSUPPORTED}
    r = calls(kk, lay(kk, B=4097, Hq=16, Hkv=4), rows, structs(kk, k=32, v=32)[1])                  # 16388 heads
    assert set(r.values()) == {kk.ERR_UNSUPPORTED}
    r = calls(kk, lay(kk), rows, codes)                                                             # codes and rows in one place
    assert r["quantize"] == r["dequantize"] == bad


def test_refused_per_call():
    kk = U.kk()
    bad = kk.ERR_INVALID_ARG
    rows, codes = structs(kk)[0], structs(kk, k=32, v=32)[1]
    small_rows, small_codes = structs(kk, capacity=883)[0], structs(kk, capacity=883, k=32, v=32)[1]
    L = lay(kk)
    assert kk._lib.keepkv_quantize(L, C.byref(rows), C.byref(small_codes), None) == bad
    assert kk._lib.keepkv_dequantize(L, C.byref(codes), C.byref(small_rows), None) == bad
    for kt in (None, C.c_void_p(24)):
        r = calls(kk, L, small_rows, small_codes, kt=kt, ws_bytes=0)
        assert r["append"] == r["step"] == bad
    lib, K = kk._lib, C.byref(codes)
    assert lib.keepkv_append_quant(L, K, P, P, 0, None, None, None) == bad
    for a in (-0.1, 1.0, float("nan")):
        assert lib.keepkv_decode_step_quant(L, K, P, P, P, P, None, C.c_float(a), None, P, 1 << 40, None) == bad
    for q, out in ((None, P), (P, None), (C.c_void_p(20), P), (P, C.c_void_p(20))):
        assert lib.keepkv_decode_attn_quant(L, K, q, out, None, None, P, 1 << 40, None) == bad
    for plan in ({"plan_wavefronts": -1}, {"plan_wavefronts": 5}, {"plan_slots_per_split": -64}, {"plan_slots_per_split": 32}):
        assert lib.keepkv_decode_attn_quant(L, C.byref(structs(kk, k=32, v=32, **plan)[1]), P, P, None, None, P, 1 << 40, None) == bad
    for ws, n in ((None, 0), (P, 1000), (C.c_void_p(24), 1 << 40)):                                # splits need room
        assert lib.keepkv_decode_attn_quant(L, C.byref(structs(kk, k=32, v=32, plan_slots_per_split=128)[1]), P, P, None, None, ws, n,
                                            None) == kk.ERR_WORKSPACE


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 8])
@pytest.mark.parametrize("units", [1, 8, 40, 64, 256, 513, 1000])
def test_plans_and_workspace(units, G, D, dtype):
    """Well-formed for every shape, and covered by the workspace of any larger cache."""
    kk = U.kk()
    layout = kk.Layout(units, G, 1, D, dtype, 0.1)
    for cap in (1, 31, 64, 65, 500, 884, 4100, 32768, 1 << 20):
        ns, per, waves = kk.decode_plan_quant(layout, cap)
        assert per % 32 == 0 and per >= 64 and waves in (4, 8)
        assert ns == -(-cap // per) and (ns == 1 or ns * units <= 512)
    for largest in (100, 600, 900, 5000, 32768):
        have = kk.workspace_bytes(layout, largest, max(1, largest // 10))
        for cap in range(1, largest + 1, max(1, largest // 61)):
            ns = kk.decode_plan_quant(layout, cap)[0]
            assert ns == 1 or HEAD + units * G * ns * (D + 2) * 4 <= have, (largest, cap)
    with pytest.raises(kk.KeepKVError):
        kk.decode_plan_quant(layout, 0)
    with pytest.raises(kk.KeepKVError):
        kk.decode_plan_quant(kk.Layout(units, G, 1, 96, dtype, 0.1), 100)


def test_which_call_takes_which_cache():
    """Calls that read no rows take both kinds; a QuantCache is refused where rows are read, a Cache where codes are."""
    kk = U.kk()
    layout = kk.Layout(1, 2, 2, 64, kk.BF16, 0.1)
    codes, rows = kk.QuantCache(layout, 40, device="cpu"), kk.Cache(layout, 40, device="cpu")
    assert codes.k_scale.shape == (1, 2, 2) and codes.k.shape == (1, 2, 40, 64) and codes.k.element_size() == 1
    assert kk._state(codes).capacity == kk._state(rows).capacity == 40 and kk._state(codes).k == codes.k.data_ptr()
    q = codes.quant_c()
    assert (q.c.len, q.k_scale, q.v_scale) == (codes.len.data_ptr(), codes.k_scale.data_ptr(), codes.v_scale.data_ptr())
    for f in (lambda: kk.decode_attn(layout, codes, None, None, None, None, None),
              lambda: kk.decode_step(layout, codes, None, None, None, None, None, 0.9, None, None),
              lambda: kk.match(layout, codes, 4, None, None, None, 0.5, None, None, None),
              lambda: kk.append(layout, codes, None, None), lambda: kk.score_window(layout, codes, None, 1, 0.9),
              lambda: kk.merge(layout, codes, rows, 4, None, None, None, None, 0.9, None, None),
              lambda: kk.merge(layout, rows, codes, 4, None, None, None, None, 0.9, None, None),
              lambda: kk.merge_inplace(layout, codes, None, 4, None, None, None, None, 0.9, None),
              lambda: kk.prefill_match(layout, codes, 0.5, None, None, None),
              lambda: kk.prefill_merge(layout, codes, rows, None, 0.9, None),
              lambda: kk.quantize(layout, codes, codes), lambda: kk.quantize(layout, rows, rows),
              lambda: kk.dequantize(layout, rows, rows), lambda: kk.dequantize(layout, codes, codes),
              lambda: kk.append_quant(layout, rows, None, None), lambda: kk.decode_attn_quant(layout, rows, None, None, None, None, None),
              lambda: kk.decode_step_quant(layout, rows, None, None, None, None, None, 0.9, None, None)):
        with pytest.raises(TypeError):
            f()
