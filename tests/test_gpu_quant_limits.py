"""The limits that eva.h states for the rows of the 8-bit cache: how far an
entry may be off, and what becomes of entries near the ends of bf16's range."""
import math

import pytest
import torch

from paper_2511_00576_amd import eva

pytestmark = pytest.mark.gpu

D = 64


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    eva._lib.load()


def held(rows):
    """bf16 rows [n, D] as an 8-bit cache holds them as keys and as values:
    (values in 64 bits, exponent bytes)."""
    n = len(rows)
    x = rows.reshape(1, 1, n, D).cuda()
    cache = eva.QuantCache(1, 1, 1, D, n, n, max_tokens=n, fill=0.0)
    none = torch.zeros(1, 1, 1, D, dtype=torch.bfloat16, device="cuda")
    eva.qcache_fill(cache, x, x, none, none, torch.tensor([n], dtype=torch.int32, device="cuda"))
    k = cache.k_ring[0, 0, :n].cpu().double()
    v = cache.vt_ring[0, 0].cpu().double().permute(0, 2, 1).reshape(-1, D)[:n]
    ke, ve = (t[0, 0, :n].cpu() for t in (cache.k_ring_exp, cache.v_ring_exp))
    assert torch.equal(ke, ve) and torch.equal(k.nan_to_num(nan=1e9), v.nan_to_num(nan=1e9))
    return k * torch.pow(2.0, ke.double() - 127).unsqueeze(-1), ke


def test_entries_are_off_by_half_a_step_at_most():
    g = torch.Generator().manual_seed(3)
    n = 512
    # entries from the row's largest down to 2^-24 of it, rows of every size
    x = torch.randn(n, D, generator=g).double() * torch.pow(2.0, -24 * torch.rand(n, D, generator=g).double())
    x *= torch.pow(2.0, torch.randint(-130, 124, (n, 1), generator=g).double())
    x[0], x[0, :2] = 0, torch.tensor([448.0, 7.5 * 2.0 ** -9])   # subnormal codes: off by more than 2^-4 of themselves
    x[1], x[1, :2] = 0, torch.tensor([225.0, 4.5 * 2.0 ** -9])
    x = x.bfloat16()
    y, e = held(x)
    x = x.double()
    err, top = (y - x).abs(), x.abs().amax(-1, keepdim=True)
    step = torch.pow(2.0, e.double() - 127).unsqueeze(-1)
    assert (err <= torch.maximum(2.0 ** -4 * x.abs(), 2.0 ** -10 * step)).all()
    usual = (top >= 2.0 ** -118).squeeze(-1)
    assert usual.any() and not usual.all()
    x, err, top = x[usual], err[usual], top[usual]
    big = x.abs() >= 2.0 ** -13 * top
    assert (err[big] <= 2.0 ** -4 * x.abs()[big]).all()
    assert (err <= torch.maximum(2.0 ** -4 * x.abs(), 2.0 ** -17 * top)).all()


def test_entries_near_the_largest_of_bf16():
    # steps of 2^120 there: 448 2^119 is 224 of them, the last code's border, a tie
    # that goes to it, 232
    x = torch.zeros(5, D, dtype=torch.float64)
    x[:, 0] = torch.tensor([224.0, 231.0, 232.0, 233.0, -255.0]).double() * 2.0 ** 120
    x[:, 1] = 2.0 ** 119
    y, e = held(x.bfloat16())
    assert e.tolist() == [246] * 5
    assert (y[:3, 0] == 448 * 2.0 ** 119).all() and torch.isnan(y[3:, 0]).all()
    assert (y[:, 1] == 2.0 ** 119).all() and (y[:, 2:] == 0).all()
