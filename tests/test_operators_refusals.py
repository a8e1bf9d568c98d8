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
