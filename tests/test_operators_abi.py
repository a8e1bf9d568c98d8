"""The operators around the attention reject bad arguments with the documented
status codes before touching the GPU (no compute call is made here)."""
import ctypes

import pytest

from paper_2511_00576_amd import _lib


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


FAKE = ctypes.c_void_p(0x10000)  # aligned, never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x10008)
INVALID, UNSUPPORTED, CAPACITY = _lib.EVA_ERR_INVALID, _lib.EVA_ERR_UNSUPPORTED, _lib.EVA_ERR_CAPACITY


# ---- head norms with rotation ------------------------------------------------
ROPE = dict(x=FAKE, sb=0, sl=512, gq=FAKE, gk=FAKE, turns=FAKE, rot=64, inter=0, start=None, offsets=None, eps=1e-6,
            Q=FAKE, K=FAKE, V=FAKE, dx=FAKE, dgq=FAKE, dgk=FAKE, ws=FAKE, ws_bytes=1 << 30, B=1, H=4, H_kv=2, L=64, d=64,
            dtype=_lib.EVA_BF16)


def rope(lib, **kw):
    a = dict(ROPE, **kw)
    return lib.eva_qk_norm_rope(a["x"], a["sb"], a["sl"], a["gq"], a["gk"], a["turns"], a["rot"], a["inter"], a["start"],
                                a["offsets"], a["eps"], a["Q"], a["K"], a["V"], a["B"], a["H"], a["H_kv"], a["L"],
                                a["d"], a["dtype"], None)


def rope_backward(lib, **kw):
    a = dict(ROPE, **kw)
    return lib.eva_qk_norm_rope_backward(a["x"], a["sb"], a["sl"], a["gq"], a["gk"], a["turns"], a["rot"], a["inter"],
                                         a["start"], a["offsets"], a["eps"], a["Q"], a["K"], a["V"], a["dx"], a["dgq"],
                                         a["dgk"], a["ws"], a["ws_bytes"], a["B"], a["H"], a["H_kv"], a["L"], a["d"],
                                         a["dtype"], None)


@pytest.mark.parametrize("call", [rope, rope_backward])
@pytest.mark.parametrize("kw,code", [
    (dict(B=0), INVALID), (dict(L=0), INVALID), (dict(H=0), INVALID), (dict(H_kv=-1), INVALID),
    (dict(x=None), INVALID), (dict(x=ODD), INVALID), (dict(gq=ODD), INVALID), (dict(Q=None), INVALID),
    (dict(V=ODD), INVALID), (dict(sl=516), INVALID), (dict(sb=-8), INVALID), (dict(sb=4), INVALID),
    (dict(rot=24), INVALID), (dict(rot=80), INVALID), (dict(rot=-16), INVALID), (dict(turns=None), INVALID),
    (dict(turns=ctypes.c_void_p(0x10004)), INVALID), (dict(inter=2), INVALID),
    (dict(eps=-1e-6), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(d=96), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(L=2 ** 30 + 1), UNSUPPORTED),
    (dict(B=4, L=2 ** 30), UNSUPPORTED), (dict(H=65000, H_kv=300), UNSUPPORTED),
])
def test_norm_rope_rejects(lib, call, kw, code):
    assert call(lib, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(dx=None), INVALID), (dict(dgq=None), INVALID), (dict(dgk=None), INVALID), (dict(ws=None), INVALID),
    (dict(ws=ODD), INVALID), (dict(ws_bytes=16 * 2 * 64 * 4 - 1), CAPACITY),
])
def test_norm_rope_backward_rejects(lib, kw, code):
    assert rope_backward(lib, **kw) == code
    assert lib.eva_qk_norm_rope_backward_workspace_bytes(1, 64, 64) == 16 * 2 * 64 * 4
    assert lib.eva_qk_norm_rope_backward_workspace_bytes(0, 64, 64) == 0
    assert lib.eva_qk_norm_rope_backward_workspace_bytes(4, 2 ** 30, 64) == 0
