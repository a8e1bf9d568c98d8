"""The paged cache where numbers and tables are at their limits: infinite values under the
smallest weights, scores of any magnitude, pages that the pool does not have."""
import math

import pytest
import torch

from paper_2511_00576_amd import eva
from paged_reference import mean_bound, tiles
from test_gpu_paged import BF16, F32, INF, build, ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    eva._lib.load()


def place(cache, b, pos):
    """Page and place of a position."""
    P = cache.struct.P
    return int(cache.table.table[b, pos // P]), pos % P


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("use_workspace", [True, False])
@pytest.mark.parametrize("n", [20, 4000])
@pytest.mark.parametrize("below", [60, 66, 70, 74, 78, 82, 86, 87])
def test_an_infinite_value_under_a_small_weight_is_infinite(below, n, use_workspace, dtype):
    """All scores are 0 but one, `below` under them: its weight, e^-below of the others' and 2^-126 or more
    (87 / ln 2 = 125.5), is not 0, and times an infinite value that is infinite."""
    P, d, pos = 32, 64, n - 7
    cache, ks, vs = build(1, 2, 1, d, P, [n], dtype, seed=5)
    cache.k[cache.table.table[0, :-(-n // P)].long()] = 0.0
    page, off = place(cache, 0, pos)
    cache.k[page, 0, off, 0] = -float(below)          # q . k / sqrt(64) = -below
    cache.vt[page, 0, off // 8, :16, off % 8] = INF
    cache.vt[page, 0, off // 8, 16:32, off % 8] = -INF
    q = torch.zeros(1, 2, d, dtype=dtype)
    q[:, :, 0] = 8.0
    o = eva.paged_decode(cache, q.cuda(), use_workspace=use_workspace)[0].cpu().double()
    assert (o[:, :16] == INF).all() and (o[:, 16:32] == -INF).all()
    # the other features: the mean of the other rows, by weights of 1 exactly, of which n are summed one by one
    # at worst, and divided; the row's own part is e^-60 or less.  bf16's output is rounded, half a step
    rest = [p for p in range(n) if p != pos]
    v = vs[0][rest, 0, 32:].double()
    bound = (2 * n + 4) * 2.0 ** -24 * v.abs().mean(0) + math.exp(-60) * float(vs[0].abs().max())
    if dtype == BF16:
        # (a weight of 1 is off by 2^-30, what is left of it)
        bound = bound + 2.0 ** -8 * v.mean(0).abs() + 2.0 ** -29 * v.abs().mean(0)
    assert ((o[:, 32:] - v.mean(0)).abs() <= bound).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("use_workspace", [True, False])
@pytest.mark.parametrize("n", [20, 3000])
@pytest.mark.parametrize("power", [3, 13, 14, 16, 20, 40])
def test_scores_of_any_magnitude(power, n, use_workspace, dtype):
    """Queries and keys of small whole numbers times 2^power: products and their sums (64 times 64 at most) are exact
    in fp32, and from 2^13 on two different scores differ by 2^26 / 8 or more, so that a row is the mean of the values
    of its highest scores: of t of them, t additions and a division, u each.  2^3: by 8 or more, all weights count."""
    P, d, G = 32, 64, 2
    cache, ks, vs = build(2, G, 1, d, P, [n, n // 2 + 1], dtype, seed=power)
    g = torch.Generator().manual_seed(power)
    q = torch.randint(-8, 9, (2, G, d), generator=g)
    q[:, :, 0] += (q == 0).all(-1)
    small = torch.randint(-8, 9, cache.k.shape, generator=g)
    cache.k.copy_(torch.ldexp(small.double(), torch.tensor(power)).to(dtype))
    table = cache.table.table.cpu().long()
    o = eva.paged_decode(cache, torch.ldexp(q.double(), torch.tensor(power)).to(dtype).cuda(),
                         use_workspace=use_workspace).cpu().double()
    for b, m in enumerate((n, n // 2 + 1)):
        k = small[table[b], 0].reshape(-1, d)[:m]
        score = torch.ldexp((q[b] @ k.T).double() / 8, torch.tensor(2 * power))
        p = torch.softmax(score, -1)
        v = vs[b][:, 0].double()
        want, size = p @ v, p @ v.abs()
        ties = int((p > 0).sum(-1).max())
        bound = (2 * ties + 8) * 2.0 ** -24 * size
        if power == 3:   # logits of up to 2^6 2^9 / 8 = 4096: 4 u of that in a weight of the numerator and of the denominator
            bound = bound + 8 * 4096 * 2.0 ** -24 * (size + want.abs())
        if dtype == BF16:
            bound = bound + 2.0 ** -8 * want.abs() + 2.0 ** -15 * size
        assert torch.isfinite(o[b]).all()
        assert ((o[b] - want).abs() <= bound).all()


@pytest.mark.parametrize("T", [3, 40])
@pytest.mark.parametrize("P", [16, 64])
def test_a_page_that_the_pool_does_not_have_has_no_slots(P, T):
    """Entries so far outside that page times P passes 2^32 and would lie inside: neither the page that a sequence
    has, nor one from the stack of free pages, gives a slot; what comes after them is written."""
    N, far = 9, 2 ** 32 // P
    t = eva.PageTable(4, P, N, 8 * P)
    n = [P + 2, P - 1, 0, 5]
    t.n_tok.copy_(ints(n))
    t.table[0, :2] = ints([0, far + 1])      # its second page, which is being filled
    t.table[1, 0] = 1
    t.table[3, 0] = -7
    rows = [[0, far + 1], [1], [], [-7]]
    stack = [2, 3, 4, -1, far + 4, 5, 6, 7]
    t.free_pages[:8] = ints(stack)
    t.n_free.fill_(8)
    counts = [T, T, 0, 2]
    slots, start, granted = eva.page_extend(t, T, ints(counts))
    assert granted.tolist() == counts and start.tolist() == n
    want = []
    for b, c in enumerate(counts):
        while len(rows[b]) * P < n[b] + c:
            rows[b].append(stack.pop())
        places = [(rows[b][p // P], p % P) for p in range(n[b], n[b] + c)]
        want.append([(page if 0 <= page < N else -1) * P + off for page, off in places] + [-1] * (T - c))
        assert t.table[b].tolist() == rows[b] + [-1] * (8 - len(rows[b]))
    assert slots.tolist() == want
    # rows in the pages that there are, whatever comes before them, and the means of those that are completed
    cache = eva.PagedCache(t, 2, 1, 64, F32, fill=0.0)
    k, v = (torch.randn(4, 1, T, 64, generator=torch.Generator().manual_seed(P + T + i)) for i in range(2))
    eva.paged_append(cache, k.cuda(), v.cuda(), slots)
    ref_k, ref_v, done = torch.zeros(N, 1, P, 64), torch.zeros(N, 1, P, 64), []
    for b, row in enumerate(want):
        for i, s in enumerate(row):
            if s >= 0:
                ref_k[s // P, 0, s % P], ref_v[s // P, 0, s % P] = k[b, 0, i], v[b, 0, i]
                done += [s // P] if s % P == P - 1 else []
    assert torch.equal(cache.k.cpu(), ref_k) and torch.equal(cache.vt.cpu(), tiles(ref_v))
    assert (1 in done) and (P > 16 or T < 40 or 7 in done)
    for page in range(N):
        err = (cache.k_mean[page, 0].cpu().double() - ref_k[page, 0].double().mean(0)).abs()
        assert (err <= mean_bound(ref_k[page, 0])).all() if page in done else (cache.k_mean[page] == 0).all()
    # rows that meet a page that there is not are NaN
    o = eva.paged_decode(cache, torch.ones(4, 2, 64, device="cuda"))
    assert o[0].isnan().all() and (o[2] == 0).all() and o[3].isnan().all()
    assert o[1].isnan().all() == any(not 0 <= page < N for page in rows[1])
