"""The extension's functions for caches held in 8 bits fill the same C structs as ctypes does and raise what ctypes raises."""
import ctypes as C

import pytest

from tests import gpu_util as U
from tests.test_pycall import P, _Raising, _Tensor, _cache


def _codes(kk, cls=None):
    c = _cache(kk, cls or kk.QuantCache)
    c.k_scale, c.v_scale = _Tensor(1 << 41), _Tensor(1 << 42)
    return c


def _recorders(kk, log):
    """C functions that note their arguments, in the order of kk._HOT_QUANT."""
    codes, rows = C.sizeof(kk._QuantCache), C.sizeof(kk._Cache)

    def noting(sizes, *types):
        def f(lay, *rest):
            log.append((C.string_at(lay, C.sizeof(kk._Layout)), *(C.string_at(x, n) for x, n in zip(rest, sizes)), *rest[len(sizes):]))
            return len(log)
        return C.CFUNCTYPE(C.c_int, P, *([P] * len(sizes)), *types)(f)
    return [noting([codes], P, P, P, P, P, C.c_float, P, P, C.c_size_t, P), noting([codes], P, P, P, P, P, C.c_size_t, P),
            noting([codes], P, P, C.c_int32, P, P, P), noting([rows, codes], P), noting([codes, rows], P)]


def _bind(kk, functions):
    from paper_2504_09936_amd import _pycall
    return dict(zip(kk._HOT_QUANT, _pycall.bind_quant(lambda device: 77 + device, lambda: 2, C.ArgumentError,
                                                      *(C.cast(f, P).value for f in functions))))


def _arguments(kk):
    t = [_Tensor(4096 * (i + 1), 100) for i in range(7)]
    lay = kk.Layout(3, 32, 8, 128, kk.BF16, 0.0883883)
    rows, codes = _cache(kk), _codes(kk)
    return {"decode_step_quant": [lay, codes, t[0], t[1], t[2], t[3], None, 0.9, t[4], t[5]],
            "decode_attn_quant": [lay, codes, t[0], t[1], None, t[2], None], "append_quant": [lay, codes, t[0], t[1], 9, t[2], None],
            "quantize": [lay, rows, codes], "dequantize": [lay, codes, rows]}


def _slow(kk, monkeypatch, functions):
    monkeypatch.setattr(kk, "_stream", lambda: 79)
    for name, f in zip(kk._HOT_QUANT, functions):
        monkeypatch.setattr(kk._lib, "keepkv_" + name, f)


def test_same_structs_and_arguments_as_ctypes(monkeypatch):
    kk = U.kk()
    a, b = [], []
    fast = _bind(kk, keep := _recorders(kk, a))
    _slow(kk, monkeypatch, _recorders(kk, b))
    monkeypatch.setattr(kk, "_check", lambda st, where: None)
    monkeypatch.setattr(kk, "_fast_quant", dict.fromkeys(kk._HOT_QUANT))
    for i, (name, args) in enumerate(_arguments(kk).items()):
        assert fast[name](*args) == i + 1
        getattr(kk, name)(*args)
    assert a == b and len(a) == 5 and keep


def test_calls_go_through_the_extension(monkeypatch):
    kk = U.kk()
    log = []
    functions = _recorders(kk, log)
    monkeypatch.setattr(kk, "_fast_quant", _bind(kk, functions))
    monkeypatch.setattr(kk, "_check", lambda st, where: None)
    for name, args in _arguments(kk).items():
        getattr(kk, name)(*args)
    assert len(log) == 5 and all(x[-1] == 79 for x in log)


@pytest.mark.parametrize("call,what,value", [
    ("decode_step_quant", 2, object()), ("decode_step_quant", 7, "0.9"), ("decode_step_quant", 9, _Raising()), ("append_quant", 4, 2.0),
    ("append_quant", 4, None), ("append_quant", 5, object()), ("decode_attn_quant", 3, _Tensor(1.5)), ("quantize", 1, None),
    ("decode_step_quant", "k_scale", object()), ("dequantize", "v_scale", None), ("append_quant", "capacity", 884.0)])
def test_wrong_arguments_raise_what_ctypes_raises(monkeypatch, call, what, value):
    kk = U.kk()
    log = []
    functions = _recorders(kk, log)

    def raised(fast):
        monkeypatch.setattr(kk, "_fast_quant", fast)
        args = _arguments(kk)[call]
        if isinstance(what, str):
            setattr(args[1], what, value)
        else:
            args[what] = value
        with pytest.raises(Exception) as e:
            getattr(kk, call)(*args)
        return e.type

    monkeypatch.setattr(kk, "_stream", lambda: 79)
    assert raised(_bind(kk, functions)) is raised(dict.fromkeys(kk._HOT_QUANT)) and not log


def test_other_classes_go_through_ctypes(monkeypatch):
    kk = U.kk()

    class Window(kk.QuantCache):
        def quant_c(self):
            s = super().quant_c()
            s.c.capacity = 7
            return s

    log = []
    functions = _recorders(kk, log)
    _slow(kk, monkeypatch, functions)
    monkeypatch.setattr(kk, "_check", lambda st, where: None)
    monkeypatch.setattr(kk, "_fast_quant", _bind(kk, functions))
    args = _arguments(kk)["append_quant"]
    args[1] = _codes(kk, Window)
    kk.append_quant(*args)
    assert kk._QuantCache.from_buffer_copy(log[-1][1]).c.capacity == 7
