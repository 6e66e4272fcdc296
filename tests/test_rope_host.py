"""What spkv_qk_norm_rope and its backward pass refuse, before any GPU call (no GPU)."""

import ctypes as C
import math

import pytest
import torch

import paper_2605_14037_amd as spkv
from paper_2605_14037_amd import binding as B

E_INVAL = -1
PTR = 1 << 20          # a 16-byte aligned address that is never followed


class Heads(C.Structure):
    """spkv_heads_t"""
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


def _call(rope=None, backward=False, **kw):
    a = dict(q=(PTR, 4 * 128, 128), k=(PTR, 2 * 128, 128), v=None, q_weight=None, k_weight=None, eps=1e-6,
             positions=PTR, dtype=B.BF16, n=5, hq=4, hk=2, q_out=(PTR, 4 * 128, 128), k_out=(PTR, 2 * 128, 128),
             v_out=None, x=((PTR, 512, 128), (PTR, 256, 128)), dqw=None, dkw=None, ws=None, ws_bytes=0)
    a.update(kw)
    r = spkv.Rope(128) if rope is None else rope
    s = r.struct if isinstance(r, spkv.Rope) else r

    def heads(t):
        return None if t is None else C.byref(Heads(*t))

    lib = spkv.load_library()
    io = [heads(a["q"]), heads(a["k"]), heads(a["v"])]
    out = [heads(a["q_out"]), heads(a["k_out"]), heads(a["v_out"])]
    shared = [a["q_weight"], a["k_weight"], a["eps"], a["positions"], s, a["dtype"], a["n"], a["hq"], a["hk"]]
    if not backward:
        return lib.spkv_qk_norm_rope(*io, *shared, *out, None)
    return lib.spkv_qk_norm_rope_backward(*io, heads(a["x"][0]), heads(a["x"][1]), *shared, *out, a["dqw"], a["dkw"],
                                          a["ws"], a["ws_bytes"], None)


def test_no_tokens_is_no_work():
    assert _call(n=0) == 0 and _call(n=0, backward=True) == 0


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("bad", [
    dict(q=None), dict(k=None), dict(q_out=None), dict(k_out=None), dict(v=(PTR, 256, 128)), dict(v_out=(PTR, 256, 128)),
    dict(q=(0, 512, 128)), dict(q=(PTR + 2, 512, 128)), dict(q_out=(PTR + 8, 512, 128)),
    dict(q=(PTR, 513, 128)), dict(q=(PTR, 512, 132)), dict(k=(PTR, -256, 128)),
    dict(q_out=(PTR, 512, 64)), dict(q_out=(PTR, 0, 128)), dict(k_out=(PTR, 128, 128)), dict(k_out=(PTR, 120, 1024)),
    dict(q_weight=PTR + 4), dict(k_weight=PTR + 8), dict(eps=float("nan")), dict(eps=float("inf")),
    dict(positions=None), dict(positions=PTR + 2), dict(dtype=2), dict(dtype=-1), dict(n=-1), dict(n=1 << 28),
    dict(hq=0), dict(hk=0)])
def test_arguments_out_of_the_rules(backward, bad):
    assert _call(backward=backward, **bad) == E_INVAL


def _struct(**kw):
    r = spkv.Rope(128, sections=[32, 32])
    for name, value in kw.items():
        setattr(r.struct, name, value)
    r.struct.keep = r
    return r.struct


@pytest.mark.parametrize("bad", [dict(head_dim=96), dict(head_dim=256), dict(rot_dim=-2), dict(rot_dim=130), dict(rot_dim=24),
                                 dict(rot_dim=7, adjacent=1), dict(n_axes=0), dict(n_axes=5), dict(n_axes=1),
                                 dict(inv_freq=None)])
def test_rotations_out_of_the_rules(bad):
    assert _call(rope=_struct(**bad)) == E_INVAL
    assert _call(rope=None, backward=True, n=0) == 0


def test_frequencies_have_to_be_finite():
    for f in (math.nan, math.inf):
        assert _call(rope=spkv.Rope(128, inv_freq=[1.0] * 63 + [f])) == E_INVAL


@pytest.mark.parametrize("bad", [
    dict(x=(None, (PTR, 256, 128))), dict(x=((PTR, 512, 128), None)), dict(dqw=PTR, ws=None, ws_bytes=1 << 30),
    dict(dqw=PTR, ws=PTR, ws_bytes=1023), dict(dkw=PTR, ws=PTR + 4, ws_bytes=1 << 30), dict(dqw=PTR + 4, ws=PTR, ws_bytes=1 << 30),
    dict(dqw=PTR, ws=PTR, ws_bytes=1 << 30, eps=-1.0)])
def test_backward_pass_refuses(bad):
    assert _call(backward=True, **bad) == E_INVAL


def test_workspace_is_enough_for_any_number_of_tokens():
    lib = spkv.load_library()
    size = lib.spkv_qk_norm_rope_backward_workspace_bytes
    assert size(1, 1, 1, 128) == size(1 << 20, 32, 8, 128) == 1024 * 2 * 128 * 4
    assert size(10, 32, 8, 96) == 0 and size(-1, 32, 8, 64) == 0 and size(1, 0, 8, 64) == 0


def test_rope_descriptions():
    r = spkv.Rope(128, sections=[16, 24, 24], theta=1e6)
    assert r.n_axes == 3 and list(r._axis) == [0] * 16 + [1] * 24 + [2] * 24
    assert r._freq[0] == 1.0 and r._freq[63] == pytest.approx(1e6 ** (-126 / 128))
    with pytest.raises(ValueError):
        spkv.Rope(128, sections=[16, 24])
    with pytest.raises(ValueError):
        spkv.Rope(128, sections=[64], axis=[0] * 64)
    with pytest.raises(ValueError):
        spkv.Rope(64, inv_freq=[1.0] * 31)
    assert spkv.Rope(64, rot_dim=0).struct.rot_dim == 0


def test_python_calls_refuse_host_tensors():
    rope, q = spkv.Rope(64), torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    pos = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="q: need a cuda"):
        spkv.qk_norm_rope(q, q[:, :2], pos, rope)
    with pytest.raises(ValueError, match="bf16 or fp32"):
        spkv.qk_norm_rope(q.half(), q[:, :2].half(), pos, rope)
    with pytest.raises(ValueError, match="heads of 64 elements"):
        spkv.qk_norm_rope(q, q[:, :2], pos, spkv.Rope(128))
