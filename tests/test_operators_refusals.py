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
