"""An extension built before the calls on 8-bit caches: those go through ctypes, the others through the extension."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_an_extension_without_the_calls_on_codes():
    code = ("import sys, types\n"
            "from paper_2504_09936_amd import _pycall\n"
            "old = types.ModuleType('paper_2504_09936_amd._pycall')\n"
            "old.bind = _pycall.bind\n"
            "sys.modules['paper_2504_09936_amd._pycall'] = old\n"
            "import paper_2504_09936_amd as package\n"
            "package._pycall = old\n"
            "from paper_2504_09936_amd import binding as kk\n"
            "assert all(kk._fast.values()) and not any(kk._fast_quant.values()) and kk._pycall is old\n"
            "kk._stream = lambda: None\n"
            "lay = kk.Layout(1, 2, 2, 64, kk.BF16, 0.1)\n"
            "try:\n"
            "    kk.append_quant(lay, kk.QuantCache(lay, 40, device='cpu'), None, None)\n"
            "except kk.KeepKVError as e:\n"
            "    assert e.status == kk.ERR_INVALID_ARG\n"
            "else:\n"
            "    raise AssertionError('not refused')\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
