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
    (dict(B=4, L=2 ** 30), UNSUPPORTED), (dict(B=1, L=2 ** 26 - 63), UNSUPPORTED), (dict(H=65000, H_kv=300), UNSUPPORTED),
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


# ---- drafted trees, accepted paths, 8-bit cache ----------------------------------
def make_rcache(**kw):
    a = dict(B=2, H=4, H_kv=2, d=64, W=8, C=4, dtype=_lib.EVA_BF16, window=0, R=32, S_max=32, max_tok=100,
             n_tok=0x50000, arrive=0x60000, k_ring=0x10000, vt_ring=0x20000, k_sum=0x30000, vt_sum=0x40000)
    a.update(kw)
    return _lib.EvaRCacheStruct(**a)


def make_qcache(**kw):
    a = dict(B=2, H=4, H_kv=2, d=64, W=8, C=4, window=0, R=64, S_max=64, max_tok=100, n_tok=0x50000, arrive=0x60000,
             k_ring=0x10000, vt_ring=0x20000, k_sum=0x30000, vt_sum=0x40000, k_ring_exp=0x70000, v_ring_exp=0x80000,
             k_sum_exp=0x90000, v_sum_exp=0xa0000)
    a.update(kw)
    return _lib.EvaQCacheStruct(**a)


BAD_QCACHES = [
    (dict(B=0), INVALID), (dict(H=5), INVALID), (dict(W=0), INVALID), (dict(C=0), INVALID), (dict(C=8193), INVALID),
    (dict(d=96), UNSUPPORTED), (dict(R=32), INVALID), (dict(R=96), INVALID), (dict(S_max=96), INVALID),
    (dict(W=62), CAPACITY), (dict(max_tok=260), CAPACITY), (dict(max_tok=0), INVALID), (dict(max_tok=2 ** 30 + 1), UNSUPPORTED),
    (dict(n_tok=0), INVALID), (dict(arrive=0), INVALID), (dict(k_ring=0), INVALID), (dict(vt_sum=0x40008), INVALID),
    (dict(k_ring_exp=0), INVALID), (dict(v_sum_exp=0xa0004), INVALID), (dict(window=3), INVALID), (dict(window=-1), INVALID),
    (dict(B=40000), UNSUPPORTED),
]


@pytest.mark.parametrize("kw,code", BAD_QCACHES)
def test_qcache_validation(lib, kw, code):
    c = ctypes.byref(make_qcache(**kw))
    assert lib.eva_qcache_fill(c, FAKE, FAKE, FAKE, FAKE, 8, FAKE, None) == code
    assert lib.eva_qcache_append(c, FAKE, FAKE, None, None) == code
    assert lib.eva_qappend_path(c, FAKE, FAKE, None, None, 2, None, None) == code
    assert lib.eva_qcache_read(c, ctypes.byref(make_rcache()), None) == code
    assert lib.eva_qdecode_step(c, FAKE, FAKE, None, None, 0, None) == code
    assert lib.eva_qappend_decode(c, FAKE, FAKE, FAKE, FAKE, None, None, 0, None) == code
    assert lib.eva_qtree_attention(c, FAKE, FAKE, FAKE, FAKE, None, FAKE, 2, None, None, 0, None) == code
    assert lib.eva_qdecode_workspace_bytes(c) == 0
    assert lib.eva_qtree_workspace_bytes(c, 2) == 0


def test_qcache_calls_reject(lib):
    c = ctypes.byref(make_qcache())
    assert lib.eva_qcache_fill(c, FAKE, FAKE, FAKE, FAKE, 8, None, None) == INVALID
    assert lib.eva_qcache_fill(c, ODD, FAKE, FAKE, FAKE, 8, FAKE, None) == INVALID
    assert lib.eva_qcache_fill(c, FAKE, FAKE, None, FAKE, 8, FAKE, None) == INVALID
    assert lib.eva_qcache_fill(c, FAKE, FAKE, FAKE, FAKE, 0, FAKE, None) == INVALID
    assert lib.eva_qcache_fill(c, FAKE, FAKE, FAKE, FAKE, 2 ** 30 + 1, FAKE, None) == UNSUPPORTED
    assert lib.eva_qcache_append(c, None, FAKE, None, None) == INVALID
    assert lib.eva_qcache_append(c, FAKE, ODD, None, None) == INVALID
    assert lib.eva_qdecode_step(c, None, FAKE, None, None, 0, None) == INVALID
    assert lib.eva_qdecode_step(c, FAKE, ODD, None, None, 0, None) == INVALID
    assert lib.eva_qappend_decode(c, FAKE, FAKE, FAKE, None, None, None, 0, None) == INVALID
    assert lib.eva_qappend_decode(c, FAKE, FAKE, None, FAKE, None, None, 0, None) == INVALID
    assert lib.eva_qcache_read(c, None, None) == INVALID
    assert lib.eva_qcache_read(c, ctypes.byref(make_rcache(max_tok=99)), None) == CAPACITY
    assert lib.eva_qcache_read(c, ctypes.byref(make_rcache(dtype=_lib.EVA_F32)), None) == UNSUPPORTED
    for kw in (dict(B=1), dict(H=8), dict(H_kv=4, H=4), dict(d=128), dict(W=9), dict(C=5), dict(window=1),
               dict(rf=1, rf_lambda=0.1)):
        assert lib.eva_qcache_read(c, ctypes.byref(make_rcache(**kw)), None) == INVALID, kw


@pytest.mark.parametrize("kind", ["r", "q"])
def test_trees_and_paths_reject(lib, kind):
    make = make_rcache if kind == "r" else make_qcache
    tree, path = getattr(lib, f"eva_{kind}tree_attention"), getattr(lib, f"eva_{kind}append_path")
    size = getattr(lib, f"eva_{kind}tree_workspace_bytes")

    def call(cache=None, **kw):
        a = dict(q=FAKE, k=FAKE, v=FAKE, parents=FAKE, o=FAKE, T=4)
        a.update(kw)
        return tree(ctypes.byref(cache or make()), a["q"], a["k"], a["v"], a["parents"], None, a["o"], a["T"], None, None, 0,
                    None)

    for name in ("q", "k", "v", "o", "parents"):
        assert call(**{name: None}) == INVALID
    for name in ("q", "k", "v", "o"):
        assert call(**{name: ODD}) == INVALID
    assert call(T=0) == INVALID
    assert call(T=9) == INVALID                             # deeper than the window
    big = dict(W=100, R=128, max_tok=100)
    assert call(make(**big), T=65) == UNSUPPORTED
    assert call(make(window=2), T=2) == UNSUPPORTED         # blocked window
    assert call(make(window=3)) == INVALID
    assert path(ctypes.byref(make()), None, FAKE, None, None, 2, None, None) == INVALID
    assert path(ctypes.byref(make()), FAKE, ODD, None, None, 2, None, None) == INVALID
    assert path(ctypes.byref(make()), FAKE, FAKE, None, None, 0, None, None) == INVALID
    assert path(ctypes.byref(make()), FAKE, FAKE, None, None, 9, None, None) == INVALID
    assert path(ctypes.byref(make(**big)), FAKE, FAKE, None, None, 65, None, None) == UNSUPPORTED
    for T in (-1, 0, 9, 65):
        assert size(ctypes.byref(make()), T) == 0
    assert call(make(H=2 ** 30, H_kv=2)) == UNSUPPORTED     # more columns than a grid
