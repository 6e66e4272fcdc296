"""Which kernels the rotation of heads takes for calls beyond the last cache, without a GPU (see tests/recorder)."""

import ctypes as C
import json
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

AT = 1 << 40                                             # an aligned address that nothing touches


def _launches(calls):
    """[[tokens, fp32, backward], ..]: the kernels of each call, 40 normed heads of 128 and 8 of values."""
    from tests import recorder
    out = subprocess.run([sys.executable, os.path.abspath(__file__), recorder._runtime(), recorder.LIB],
                         input=json.dumps(calls), capture_output=True, text=True, timeout=120)
    assert out.returncode == 0, out.stderr
    return json.loads(out.stdout)


def _main():
    rt = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)          # before the library: its names win
    lib = C.CDLL(sys.argv[2])
    ptr, i64, i32, f32 = C.c_void_p, C.c_int64, C.c_int32, C.c_float

    class Rope(C.Structure):
        _fields_ = [("head_dim", i32), ("rot_dim", i32), ("adjacent", i32), ("n_axes", i32), ("inv_freq", ptr), ("axis", ptr)]

    class Heads(C.Structure):
        _fields_ = [("data", ptr), ("token_stride", i64), ("head_stride", i64)]

    freq = (C.c_double * 64)(*[1.0] * 64)
    rope = Rope(128, 128, 0, 1, C.addressof(freq), None)
    heads = [C.byref(Heads(AT, n * 128, 128)) for n in (32, 8, 8)]
    out = []
    for tokens, fp32, backward in json.load(sys.stdin):
        a = [None, None, f32(1e-6), ptr(AT), C.byref(rope), i32(fp32), i64(tokens), i32(32), i32(8), *heads]
        if backward:
            rc = lib.spkv_qk_norm_rope_backward(*heads, *heads[:2], *a, None, None, None, C.c_size_t(0), None)
        else:
            rc = lib.spkv_qk_norm_rope(*heads, *a, None)
        assert rc == 0
        buf, got = C.create_string_buffer(1024), []
        while rt.rec_take(buf, 1024) >= 0:
            got.append(buf.value.decode().rsplit(" ", 3)[0])
        out.append(got)
    json.dump(out, sys.stdout)


@pytest.mark.parametrize("backward", [0, 1])
def test_loads_and_stores_without_retention(backward):
    """bf16 calls past the last cache alone: fp32 ones are slower that way at every size."""
    tokens = [1000, 16384, 40000]
    modes = [int(k[0][k[0].index("EEv") - 1]) for k in _launches([[t, 0, backward] for t in tokens])]
    assert modes == [0, 1, 2]
    modes = [int(k[0][k[0].index("EEv") - 1]) for k in _launches([[t, 1, backward] for t in tokens])]
    assert modes == [0, 0, 0]


if __name__ == "__main__":
    _main()
