"""Head norms with rotation of more key and value heads than query heads, which
the projection's layout allows: every head of every kind is written, forward
and backward.  Tolerances as in test_gpu_norm_rope.py."""
import math

import pytest
import torch

from paper_2511_00576_amd import eva
from test_gpu_norm_rope import Reference, U, half_step, make, split, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    eva._lib.load()


@pytest.mark.parametrize("B,L,H,Hkv,d,dtype,inter", [
    (3, 41, 1, 2, 64, torch.bfloat16, False),
    (2, 65, 4, 8, 128, torch.bfloat16, False),
    (2, 33, 8, 12, 64, torch.float32, True),
    (1, 1, 1, 3, 128, torch.float32, False),
    (2, 1500, 2, 7, 64, torch.bfloat16, True),
    (1, 130, 1, 32, 128, torch.bfloat16, False),
    (4, 9, 16, 17, 64, torch.float32, False),
])
def test_more_key_heads_than_query_heads(B, L, H, Hkv, d, dtype, inter):
    x, w, _, _, pos, freq, grads = make(B, L, H, Hkv, d, d, dtype, 7 * L + Hkv)
    ref = Reference(freq, pos, 1e-6, inter, d)
    how = dict(turns=eva.rope_turns(d), q_weight=w[0].cuda(), k_weight=w[1].cuda(), interleaved=inter)
    # what is not written stays NaN
    out = [torch.full((B, n, L, d), math.nan, dtype=dtype, device="cuda") for n in (H, Hkv, Hkv)]
    eva.qk_norm_rope(x.cuda(), H, Hkv, out=out, **how)
    left = torch.full(x.shape, math.nan, dtype=dtype, device="cuda")
    del left  # (the gradient's memory, most likely)
    got = eva.qk_norm_rope_backward(x.cuda(), *(t.cuda() for t in grads), **how)
    rows, dx = split(x.double(), H, Hkv), split(got[0], H, Hkv)
    round_ = 0 if dtype == torch.float32 else half_step(x)
    for i, name in enumerate("QK"):
        y, mag = ref.forward(rows[i], w[i].double())
        within(out[i], y, round_ * y.abs() + 24 * U * mag, name)
        d64, dmag, dg, dgmag = ref.backward(rows[i], w[i].double(), grads[i].double())
        within(dx[i], d64, round_ * d64.abs() + 64 * U * dmag, "d" + name)
        within(got[1 + i], dg, (64 + 1024) * U * dgmag, f"weight {name}")
    assert torch.equal(out[2].cpu(), split(x, H, Hkv)[2]), "V"
    assert torch.equal(dx[2].cpu(), grads[2]), "dV"
