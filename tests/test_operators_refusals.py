"""Calls around the attention that are refused before any work: caches that are
not on the GPU, and what the C entries answer before anything is enqueued.  No
compute call is made here."""
import ctypes

import pytest
import torch

from paper_2511_00576_amd import _lib, eva

B, H, HKV, D, T = 1, 2, 1, 64, 3


def rows(n, t=None):
    return torch.zeros((B, n, D) if t is None else (B, n, t, D), dtype=torch.bfloat16)


def caches():
    return (eva.QuantCache(B, H, HKV, D, 16, 4, 60, device="cpu"), eva.RaggedCache(B, H, HKV, D, 16, 4, 60, device="cpu"))


@pytest.mark.parametrize("name", ["fill", "append", "read", "decode", "append_decode", "tree", "path"])
def test_caches_in_host_memory_are_refused(name):
    # with operands in host memory too: their addresses must not reach a kernel
    quant, ragged = caches()
    k, kt = rows(HKV), rows(HKV, T)
    calls = {
        "fill": lambda c: eva.qcache_fill(c, kt, kt, rows(HKV, 0), rows(HKV, 0), torch.ones(B, dtype=torch.int32)),
        "append": lambda c: eva.qcache_append(c, k, k),
        "read": lambda c: eva.qcache_read(c, ragged),
        "decode": lambda c: eva.qdecode_step(c, rows(H)),
        "append_decode": lambda c: eva.qappend_decode(c, rows(H), k, k),
        "tree": lambda c: eva.tree_attention(c, rows(H, T), kt, kt, torch.full((B, T), -1, dtype=torch.int32)),
        "path": lambda c: eva.append_path(c, kt, kt),
    }
    for cache in (quant, ragged) if name in ("tree", "path") else (quant,):
        with pytest.raises(RuntimeError, match="ROCm device"):
            calls[name](cache)


# ---- the C entries: addresses that are never dereferenced -------------------------
FAKE = ctypes.c_void_p(0x10000)
INVALID, UNSUPPORTED = _lib.EVA_ERR_INVALID, _lib.EVA_ERR_UNSUPPORTED


def quant_struct(**kw):
    a = dict(B=2, H=4, H_kv=2, d=64, W=8, C=4, window=0, R=64, S_max=64, max_tok=100, n_tok=0x50000, arrive=0x60000,
             k_ring=0x10000, vt_ring=0x20000, k_sum=0x30000, vt_sum=0x40000, k_ring_exp=0x70000, v_ring_exp=0x80000,
             k_sum_exp=0x90000, v_sum_exp=0xa0000)
    a.update(kw)
    return _lib.EvaQCacheStruct(**a)


@pytest.mark.parametrize("kw", [
    dict(H=2 ** 30, H_kv=2),             # more columns than a launch has
    dict(B=30000, H=2 ** 17, H_kv=2),    # more workgroups
])
def test_append_and_decode_is_refused_before_the_append(kw):
    # (an append that is enqueued answers EVA_ERR_HIP where there is no GPU)
    lib, c = _lib.load(), ctypes.byref(quant_struct(**kw))
    assert lib.eva_qdecode_step(c, FAKE, FAKE, None, None, 0, None) == UNSUPPORTED
    assert lib.eva_qappend_decode(c, FAKE, FAKE, FAKE, FAKE, None, None, 0, None) == UNSUPPORTED


OFF4 = ctypes.c_void_p(0x10002)  # not on four bytes


@pytest.mark.parametrize("kind", ["r", "q"])
def test_misaligned_parents_are_refused(kind):
    lib = _lib.load()
    if kind == "q":
        c = quant_struct()
    else:
        c = _lib.EvaRCacheStruct(B=2, H=4, H_kv=2, d=64, W=8, C=4, dtype=_lib.EVA_BF16, window=0, R=32, S_max=32, max_tok=100,
                                 n_tok=0x50000, arrive=0x60000, k_ring=0x10000, vt_ring=0x20000, k_sum=0x30000, vt_sum=0x40000)
    tree = getattr(lib, f"eva_{kind}tree_attention")
    assert tree(ctypes.byref(c), FAKE, FAKE, FAKE, OFF4, None, FAKE, 4, None, None, 0, None) == INVALID


@pytest.mark.parametrize("start,offsets,dgq,dgk", [(OFF4, None, FAKE, FAKE), (None, OFF4, FAKE, FAKE), (None, None, OFF4, FAKE),
                                                   (None, None, FAKE, OFF4)])
def test_misaligned_operands_of_head_norms_are_refused(start, offsets, dgq, dgk):
    lib = _lib.load()
    head = (FAKE, 0, 512, FAKE, FAKE, FAKE, 64, 0, start, offsets, 1e-6)
    size = (1, 4, 2, 64, 64, _lib.EVA_BF16)
    if start or offsets:
        assert lib.eva_qk_norm_rope(*head, FAKE, FAKE, FAKE, *size, None) == INVALID
    assert lib.eva_qk_norm_rope_backward(*head, FAKE, FAKE, FAKE, FAKE, dgq, dgk, FAKE, 1 << 30, *size, None) == INVALID
