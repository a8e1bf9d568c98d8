"""Rows that are split over workgroups: what the join makes of shares in which
every key is NaN (they have no maximum, and a sum that is NaN)."""
import math

import pytest
import torch

from paper_2511_00576_amd import eva, inputs

pytestmark = pytest.mark.gpu

B, H, HKV, D, W, C, N = 1, 4, 2, 64, 700, 4, 8700


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    eva._lib.load()


def prompt(dtype, chunk=32):
    """A prompt whose first summaries' keys are NaN in kv head 0: all that the
    first eight shares hold, four chunks of `chunk` keys each."""
    _, k, v = inputs.qkv(B, H, HKV, N, D, dtype, seed=3)
    k, v = k.cuda(), v.cuda()
    Ks, Vs = eva.build_summaries(k, v, C)
    Ks[:, 0, :8 * 4 * chunk] = math.nan
    return k, v, Ks, Vs


def check(o, one, what):
    """o [B, H, ...]: the rows of kv head 0 are NaN, the others as without splits."""
    assert torch.isnan(o[:, :H // HKV]).all(), f"{what}: NaN keys were lost"
    assert torch.isfinite(o[:, H // HKV:]).all(), what
    assert torch.isnan(one[:, :H // HKV]).all() and torch.isfinite(one[:, H // HKV:]).all(), f"{what}, not split"


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "f32"])
def test_trees(kind):
    dtype = torch.float32 if kind == "f32" else torch.bfloat16
    rows = prompt(dtype, 64 if kind == "e4m3" else 32)
    lens = torch.tensor([N], dtype=torch.int32, device="cuda")
    if kind == "e4m3":
        cache = eva.QuantCache(B, H, HKV, D, W, C, max_tokens=N + 8, fill=0.0)
        eva.qcache_fill(cache, *rows, lens)
        size = eva._lib.load().eva_qtree_workspace_bytes
    else:
        cache = eva.RaggedCache(B, H, HKV, D, W, C, max_tokens=N + 8, dtype=dtype, fill=0.0)
        eva.rcache_fill(cache, *rows, lens)
        size = eva._lib.load().eva_rtree_workspace_bytes
    q, k, v = (inputs.normal((B, h, 2, D), 5 + h, dtype).cuda() for h in (H, HKV, HKV))
    parents = torch.tensor([[-1, 0]], dtype=torch.int32, device="cuda")
    splits = size(eva.ctypes.byref(cache.struct), 2) // (4 * B * HKV * (H // HKV * 2) * (D + 2))
    assert splits > 8, "the shape must split its rows more than eight times"
    check(eva.tree_attention(cache, q, k, v, parents), eva.tree_attention(cache, q, k, v, parents, use_workspace=False), kind)
    if kind == "e4m3":
        q = q[:, :, 0].contiguous()
        check(eva.qdecode_step(cache, q), eva.qdecode_step(cache, q, use_workspace=False), "decode")


def test_ragged_and_uniform_decode():
    rows = prompt(torch.bfloat16)
    q = inputs.normal((B, H, D), 9, torch.bfloat16).cuda()
    cache = eva.RaggedCache(B, H, HKV, D, W, C, max_tokens=N + 8, fill=0.0)
    eva.rcache_fill(cache, *rows, torch.tensor([N], dtype=torch.int32, device="cuda"))
    assert cache.ws.numel() // (B * HKV * 16 * (D + 2)) > 8, "the shape must split its rows more than eight times"
    check(eva.rdecode_step(cache, q), eva.rdecode_step(cache, q, use_workspace=False), "ragged")
    cache = eva.Cache(B, H, HKV, D, W, C, max_tokens=N + 8, fill=0.0)
    eva.cache_fill(cache, *rows)
    check(eva.decode_step(cache, q), eva.decode_step(cache, q, use_workspace=False), "uniform")
