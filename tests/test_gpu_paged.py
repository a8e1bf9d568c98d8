"""The paged cache: its table, the append, the decode over all of a sequence's pages or
over chosen ones, and the choice, against plain models (paged_reference.py) and 64-bit rows
with derived bounds."""
import math

import pytest
import torch

from paper_2511_00576_amd import eva, inputs
from paged_reference import Table, attend, choice, keys_of, mean_bound, random_pages, tiles

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
NAN, INF = math.nan, math.inf


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    eva._lib.load()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---- table --------------------------------------------------------------------
def extend_both(t, m, T, counts):
    slots, start, granted = eva.page_extend(t, T, None if counts is None else ints(counts))
    want = m.extend(T, counts)
    for got, ref, what in zip((slots, start, granted), want, ("slots", "start", "granted")):
        assert got.tolist() == ref, what
    m.check(t)
    return want


# B, P, pages of the pool, tokens that a sequence may hold, T
TABLES = [(1, 16, 1, 16, 1), (1, 256, 9, 2000, 700), (3, 16, 40, 300, 5), (70, 32, 300, 400, 16), (70, 32, 300, 400, 17),
          (5, 64, 200, 5000, 1025), (1030, 16, 2500, 64, 3), (2100, 16, 5000, 100, 20), (64, 128, 70, 1000, 1)]


@pytest.mark.parametrize("B,P,N,most,T", TABLES)
def test_table_follows_its_definition(B, P, N, most, T):
    g = torch.Generator().manual_seed(B + T)
    t, m = eva.PageTable(B, P, N, most), Table(B, P, N, -(-most // P))
    m.check(t)
    extend_both(t, m, T, None)
    short = 0
    for step in range(6):
        counts = (torch.randint(-2, T + 3, (B,), generator=g) * (torch.rand(B, generator=g) < 0.8)).tolist()
        _, _, granted = extend_both(t, m, T, counts)
        short += sum(0 < min(max(c, 0), T) != k for c, k in zip(counts, granted))
        if step % 2:
            # some leave, some take tokens back, most stay
            lens = [(-3 if i % 7 == 0 else n - (i % 5) if i % 2 else 2 ** 31 - 1) for i, n in enumerate(m.n)]
            eva.page_truncate(t, ints(lens))
            m.truncate(lens)
            m.check(t)
    eva.page_truncate(t, ints([0] * B))
    m.truncate([0] * B)
    m.check(t)
    assert sorted(t.free_pages.tolist()) == list(range(N))


def test_a_short_stack_serves_in_order():
    t, m = eva.PageTable(5, 16, 4, 200), Table(5, 16, 4, 13)
    # two pages, three (one too many), one (held up by the one before), none, none
    _, _, granted = extend_both(t, m, 40, [32, 40, 1, 0, 0])
    assert granted == [32, 0, 0, 0, 0]
    # three pages of two that are left: what comes after it waits, although it would fit
    _, _, granted = extend_both(t, m, 40, [0, 40, 16, 1, 0])
    assert granted == [0, 0, 0, 0, 0]
    _, _, granted = extend_both(t, m, 40, [8, 17, 0, 0, 0])   # a third page, then two
    assert granted == [8, 0, 0, 0, 0]
    _, _, granted = extend_both(t, m, 40, [8, 17, 0, 0, 16])  # within its page; two do not fit; one behind it
    assert granted == [8, 0, 0, 0, 0]
    _, _, granted = extend_both(t, m, 40, [0, 16, 0, 0, 0])
    assert granted == [0, 16, 0, 0, 0] and m.stack == []


@pytest.mark.parametrize("T", [1, 9, 300])
def test_taking_back_restores_table_and_stack(T):
    t = eva.PageTable(20, 16, 500, 1000)
    eva.page_extend(t, 333, ints([(i * 29) % 334 for i in range(20)]))
    before = [x.clone() for x in (t.n_tok, t.table, t.free_pages[:t.n_free.item()], t.n_free)]
    eva.page_extend(t, T, ints([(i * 7) % (T + 1) for i in range(20)]))
    eva.page_truncate(t, before[0])
    after = [t.n_tok, t.table, t.free_pages[:t.n_free.item()], t.n_free]
    assert all(torch.equal(a, b) for a, b in zip(before, after))


# ---- append -------------------------------------------------------------------
def pools_of(cache):
    return [cache.k.clone(), cache.vt.clone(), cache.k_mean.clone()]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("P,d,Hkv", [(16, 64, 3), (32, 128, 1), (64, 128, 2), (128, 64, 2), (256, 128, 1)])
def test_append_writes_rows_tiles_and_means(dtype, P, d, Hkv):
    g = torch.Generator().manual_seed(P + d)
    B, most = 4, 3 * P + 40
    N = B * -(-most // P) + 2
    t = eva.PageTable(B, P, N, most)
    caches = [eva.PagedCache(t, 2 * Hkv, Hkv, d, dtype, fill=7.0) for _ in range(2)]
    ref_k = torch.full((N, Hkv, P, d), 7.0, dtype=dtype)
    ref_v = ref_k.clone()
    written, mean = [[] for _ in range(B)], {}
    for T in (1, 2 * P - 3, 5, 1, 37, P):
        counts = [max(0, T - (b * 5) % (T + 1)) for b in range(B)]
        slots, start, granted = eva.page_extend(t, T, ints(counts))
        k, v = (torch.randn(B, Hkv, T, d, generator=g).to(dtype) for _ in range(2))
        eva.paged_append(caches[0], k.cuda(), v.cuda(), slots)
        # the other cache: the same tokens one by one
        for i in range(T):
            eva.paged_append(caches[1], k[:, :, i].contiguous().cuda(), v[:, :, i].contiguous().cuda(),
                             slots[:, i:i + 1].contiguous())
        for b, row_ in enumerate(slots.tolist()):
            for i, s in enumerate(row_):
                if s < 0:
                    continue
                ref_k[s // P, :, s % P], ref_v[s // P, :, s % P] = k[b, :, i], v[b, :, i]
                if s % P == P - 1:
                    mean[s // P] = ref_k[s // P].clone()
    assert len(mean) >= 4
    for a, b in zip(pools_of(caches[0]), pools_of(caches[1])):
        assert torch.equal(a, b), "token by token gives other bits"
    assert torch.equal(caches[0].k.cpu(), ref_k)
    assert torch.equal(caches[0].vt.cpu(), tiles(ref_v))
    got = caches[0].k_mean.cpu().double()
    for page in range(N):
        for h in range(Hkv):
            if page in mean:
                ref = mean[page][h].double()
                assert ((got[page, h] - ref.mean(0)).abs() <= mean_bound(ref)).all()
            else:
                assert (got[page, h] == 7.0).all(), "the mean of a page that is not complete was written"


def test_append_skips_slots_outside_the_pool():
    t = eva.PageTable(2, 16, 3, 64)
    cache = eva.PagedCache(t, 2, 2, 64, fill=0.0)
    k = torch.ones(2, 2, 4, 64, dtype=BF16, device="cuda")
    eva.paged_append(cache, k, k, ints([[46, 47, 48, 49], [-1, -5, 2 ** 31 - 1, -2 ** 31]]))
    assert cache.k.sum() == 2 * 2 * 64 and cache.vt.sum() == 2 * 2 * 64  # places 14 and 15 of page 2
    cache = eva.PagedCache(t, 2, 2, 64, fill=0.0, means=False)  # no means kept
    eva.paged_append(cache, k, k, ints([[14, 15, -1, -1], [-1, -1, -1, -1]]))
    assert cache.k.sum() == 2 * 2 * 64


# ---- decode -------------------------------------------------------------------
def build(B, H, Hkv, d, P, lens, dtype=BF16, seed=1, garbage=NAN, most=None, spare=3):
    """A cache of sequences of these lengths in random pages, garbage everywhere else: (cache, k, v) with
    k, v [B][n, Hkv, d] on the CPU."""
    g = torch.Generator().manual_seed(seed)
    max_pages = max(1, -(-(most or max(lens)) // P))
    N = sum(-(-n // P) for n in lens) + spare
    table, free, n_free = random_pages(B, P, lens, N, max_pages, g)
    t = eva.PageTable(B, P, N, max_pages * P,
                      storage=(ints(lens), table.cuda(), torch.nn.functional.pad(free, (0, N - n_free)).cuda(), ints([n_free])))
    kp, vp = (torch.full((N, Hkv, P, d), garbage, dtype=dtype) for _ in range(2))
    mean = torch.full((N, Hkv, d), garbage)
    ks, vs = [], []
    for b, n in enumerate(lens):
        k, v = (torch.randn(n, Hkv, d, generator=g).to(dtype) for _ in range(2))
        for j in range(-(-n // P)):
            rows = slice(j * P, min(n, j * P + P))
            page = int(table[b, j])
            kp[page, :, :rows.stop - rows.start] = k[rows].transpose(0, 1)
            vp[page, :, :rows.stop - rows.start] = v[rows].transpose(0, 1)
            if rows.stop - rows.start == P:
                mean[page] = k[rows].float().mean(0)
        ks.append(k)
        vs.append(v)
    cache = eva.PagedCache(t, H, Hkv, d, dtype, storage=(kp.cuda(), tiles(vp).cuda(), mean.cuda()))
    return cache, ks, vs


def query(B, H, d, dtype, seed=1):
    return torch.randn(B, H, d, generator=torch.Generator().manual_seed(seed + 99)).to(dtype)


def check_rows(o, q, ks, vs, P, dtype, pages=None, skip=()):
    B, H, d = q.shape
    o = o.cpu().double()
    for b in range(B):
        if b in skip:
            continue
        n, Hkv = ks[b].shape[:2]
        G = H // Hkv
        for h in range(Hkv):
            at = list(range(n)) if pages is None else keys_of(pages[b][h], P, n)
            got = o[b, h * G:(h + 1) * G]
            if not at:
                assert (got == 0).all(), f"b{b} kv{h}: a row without keys is not zeros"
                continue
            kk, vv = ks[b][at, h].double(), vs[b][at, h].double()
            ref, bound = attend(q[b, h * G:(h + 1) * G], kk, vv, dtype)
            assert torch.isfinite(got).all(), f"b{b} kv{h}: not finite"
            over = ((got - ref).abs() - bound).max()
            assert over <= 0, f"b{b} kv{h}: {float(over):.3e} over the bound"


# B, H, Hkv, d, P, lens
DECODES = [
    (1, 1, 1, 64, 16, [1]),
    (3, 2, 1, 128, 16, [0, 1, 16]),
    (5, 12, 4, 64, 16, [17, 31, 32, 33, 47]),
    (4, 4, 4, 128, 32, [1, 32, 33, 200]),
    (2, 32, 8, 128, 64, [777, 1000]),
    (3, 16, 1, 128, 128, [127, 129, 500]),           # 16 heads a kv head
    (2, 40, 2, 64, 64, [333, 65]),                   # 20: two groups
    (2, 48, 1, 128, 256, [700, 255]),                # 48: three
    (9, 6, 2, 64, 32, [3000, 0, 5, 1, 64, 2, 0, 900, 31]),
    (1, 8, 8, 128, 16, [2500]),                      # shared by many workgroups
    (80, 2, 2, 64, 16, [(37 * i) % 150 for i in range(80)]),   # more sequences than lanes
    (200, 1, 1, 128, 32, [(91 * i) % 400 for i in range(200)]),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("use_workspace", [True, False])
@pytest.mark.parametrize("B,H,Hkv,d,P,lens", DECODES)
def test_decode(B, H, Hkv, d, P, lens, use_workspace, dtype):
    print(f"decode B{B} H{H}/{Hkv} d{d} P{P} {dtype} ws={use_workspace}", flush=True)
    cache, ks, vs = build(B, H, Hkv, d, P, lens, dtype)
    q = query(B, H, d, dtype)
    o = eva.paged_decode(cache, q.cuda(), use_workspace=use_workspace)
    check_rows(o, q, ks, vs, P, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("P", [16, 64])
def test_decode_shares_long_rows(P, dtype):
    # rows of very different lengths over all workgroups, and a table that has room for many more
    lens = [9000, 3, 700, 0, 12001, 64]
    cache, ks, vs = build(6, 8, 2, 128, P, lens, dtype, seed=3, most=40000)
    lib, c = eva._lib.load(), cache
    assert lib.eva_paged_decode_workspace_bytes(c.ref, c.table.ref, 0) > 0
    q = query(6, 8, 128, dtype, seed=3)
    o = eva.paged_decode(cache, q.cuda())
    check_rows(o, q, ks, vs, P, dtype)
    assert torch.equal(o, eva.paged_decode(cache, q.cuda())), "the same call gives other bits"


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,H,Hkv", [(90, 8, 8), (270, 40, 2), (1100, 1, 1)])
def test_more_rows_than_workgroups(B, H, Hkv, dtype):
    # a workgroup's part begins and ends inside rows and holds several; a row of many workgroups among them
    lens = [4000 if i == B // 2 else 330 if i % 3 else (i * 37) % 300 for i in range(B)]
    cache, ks, vs = build(B, H, Hkv, 64, 32, lens, dtype, seed=B)
    q = query(B, H, 64, dtype, seed=B)
    active = [int(i % 7 != 2) for i in range(B)]
    out = torch.full((B, H, 64), 3.0, dtype=dtype, device="cuda")
    o = eva.paged_decode(cache, q.cuda(), active=ints(active), out=out)
    skip = [b for b in range(B) if not active[b]]
    check_rows(o, q, ks, vs, 32, dtype, skip=skip)
    assert (o[skip] == 3).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,H,Hkv,longest,most", [
    (6, 6, 3, 32, 5000),       # rows so short that a wave takes each
    (150, 16, 8, 120, 5000),   # many rows, of up to eight chunks
    (150, 16, 8, 60, 64),      # many, in a table with room for no more
    (70, 40, 2, 100, 5000),    # 20 heads a kv head
    (300, 4, 4, 31, 31),       # 1200 rows of one chunk
])
def test_short_rows(B, H, Hkv, longest, most, dtype):
    lens = [(i * 53) % (longest + 1) for i in range(B)]
    cache, ks, vs = build(B, H, Hkv, 64, 16, lens, dtype, seed=longest, most=most)
    q = query(B, H, 64, dtype)
    active = [int(i % 9 != 4) for i in range(B)]
    for ws in (True, False):
        out = torch.full((B, H, 64), 3.0, dtype=dtype, device="cuda")
        o = eva.paged_decode(cache, q.cuda(), active=ints(active), out=out, use_workspace=ws)
        check_rows(o, q, ks, vs, 16, dtype, skip=[b for b in range(B) if not active[b]])
        assert (o[ints(active) == 0] == 3).all()
        lists = [[[(b + h) % 3, 7, -1, 0] for h in range(Hkv)] for b in range(B)]
        o = eva.paged_decode(cache, q.cuda(), pages=ints(lists), use_workspace=ws)
        check_rows(o, q, ks, vs, 16, dtype, lists)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_inactive_and_empty_rows(dtype):
    lens = [40, 500, 0, 33, 0]
    cache, ks, vs = build(5, 4, 2, 64, 16, lens, dtype)
    q = query(5, 4, 64, dtype)
    for ws in (True, False):
        out = torch.full((5, 4, 64), 3.0, dtype=dtype, device="cuda")
        o = eva.paged_decode(cache, q.cuda(), active=ints([1, 0, 1, 2, 0]), out=out, use_workspace=ws)
        assert o is out
        check_rows(o, q, ks, vs, 16, dtype, skip=(1, 4))
        assert (o[1] == 3).all() and (o[4] == 3).all()
        o = eva.paged_decode(cache, q.cuda(), active=ints([0] * 5), out=out.fill_(3), use_workspace=ws)
        assert (o == 3).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("use_workspace", [True, False])
@pytest.mark.parametrize("P", [16, 32, 128])
def test_decode_of_listed_pages(P, use_workspace, dtype):
    lens = [P * 9 + 5, 3 * P, 0, 7, 70 * P]
    cache, ks, vs = build(5, 6, 2, 64, P, lens, dtype, seed=P)
    q = query(5, 6, 64, dtype)
    # any order, the same page twice, entries that are none of the sequence's, an odd number of pages
    lists = [[[9, 0, 4], [3, 3, -1]], [[2, 1, 0], [7, -1, 2 ** 31 - 1]], [[0, 1, 2], [-1, -1, -1]], [[0, 0, 0], [1, 0, 0]],
             [[69, 5, 0], [-2 ** 31, 12, 13]]]
    o = eva.paged_decode(cache, q.cuda(), pages=ints(lists), use_workspace=use_workspace)
    check_rows(o, q, ks, vs, P, dtype, lists)
    # longer lists than any sequence has pages, rows over several workgroups
    S = 100
    g = torch.Generator().manual_seed(P)
    lists = [[torch.randint(0, 71, (S,), generator=g).tolist() for _ in range(2)] for _ in range(5)]
    o = eva.paged_decode(cache, q.cuda(), pages=ints(lists), use_workspace=use_workspace)
    check_rows(o, q, ks, vs, P, dtype, lists)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("use_workspace", [True, False])
@pytest.mark.parametrize("n", [20, 4000])
def test_values_that_are_not_finite(n, use_workspace, dtype):
    # what a row sees decides, what lies behind its end or in other pages does not (build() puts NaN there)
    P, d = 32, 64
    cache, ks, vs = build(6, 2, 1, d, P, [n] * 6, dtype, seed=4)
    table = cache.table.table.cpu()

    def put(pool, b, pos, x, tile=False):
        page, off = int(table[b, pos // P]), pos % P
        if tile:
            pool[page, 0, off // 8, :, off % 8] = x
        else:
            pool[page, 0, off] = x

    pos = n - 3
    big = torch.finfo(dtype).max
    put(cache.k, 1, pos, NAN)                     # a key of NaN: the row is NaN
    put(cache.vt, 2, pos, INF, tile=True)         # an infinite value: infinite
    for p in range(n):
        put(cache.k, 3, p, -big)                  # scores of -inf alone: the formula has no value
    put(cache.k, 4, pos, big)                     # a score of +inf
    for p in range(0, n, 2):
        put(cache.k, 5, p, -big)                  # every second weight is 0
    q = torch.ones(6, 2, d, dtype=dtype)
    q[0] = query(1, 2, d, dtype)[0]
    o = eva.paged_decode(cache, q.cuda(), use_workspace=use_workspace).cpu().double()
    check_rows(o, q, ks, vs, P, dtype, skip=(1, 2, 3, 4, 5))
    assert o[1].isnan().all() and (o[2] == INF).all() and o[3].isnan().all() and o[4].isnan().all()
    odd = list(range(1, n, 2))
    ref, bound = attend(q[5], ks[5][odd, 0].double(), vs[5][odd, 0].double(), dtype)
    # (weights of 0 add nothing, exactly)
    assert ((o[5] - ref).abs() <= bound).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("P", [16, 64])
def test_whole_shares_without_weight(P, dtype):
    # the first half of a long row scores -inf: shares that hold nothing else have no maximum
    n, d = 6000, 64
    cache, ks, vs = build(1, 2, 2, d, P, [n], dtype, seed=8)
    cache.k[cache.table.table[0, :3008 // P].long()] = -torch.finfo(dtype).max
    q = torch.ones(1, 2, d, dtype=dtype)
    first = 3008 // P * P
    o = eva.paged_decode(cache, q.cuda())
    check_rows(o, q, [k[first:] for k in ks], [v[first:] for v in vs], P, dtype)
    # and NaN keys there make the row NaN
    cache.k[cache.table.table[0, 3].long()] = NAN
    assert eva.paged_decode(cache, q.cuda()).isnan().all()


@pytest.mark.parametrize("use_workspace", [True, False])
@pytest.mark.parametrize("P", [16, 64])
def test_pages_outside_the_pool_make_the_row_nan(P, use_workspace):
    lens = [500, 500, 500, 500]
    cache, ks, vs = build(4, 4, 2, 64, P, lens, seed=6)
    N = cache.table.struct.n_pages
    t = cache.table.table
    t[0, 3], t[1, -(-500 // P) - 1], t[2, 0] = N, -1, 2 ** 31 - 1
    q = query(4, 4, 64, BF16)
    o = eva.paged_decode(cache, q.cuda(), use_workspace=use_workspace)
    assert o[:3].isnan().all()
    check_rows(o, q, ks, vs, P, BF16, skip=(0, 1, 2))
    # counts outside the row's room are read as the nearest inside; the entries there are -1
    cache.table.n_tok.copy_(ints([-5, 0, 0, 2 ** 31 - 1]))
    o = eva.paged_decode(cache, q.cuda(), use_workspace=use_workspace)
    assert (o[:3] == 0).all()


def test_offsets_beyond_32_bits():
    # pools of 4.3 GB each: pages at their very end
    N, P, Hkv, d = 8200, 256, 8, 128
    t = eva.PageTable(2, P, N, 4 * P)
    cache = eva.PagedCache(t, 8, Hkv, d)
    t.free_pages.copy_(torch.arange(N, dtype=torch.int32))  # the last pages on top
    slots, *_ = eva.page_extend(t, 2 * P + 9, ints([2 * P + 9, P]))
    assert int(slots.max()) == N * P - 1 and (N - 4) * P * Hkv * d > 2 ** 31
    k, v = (torch.randn(2, Hkv, 2 * P + 9, d, generator=torch.Generator().manual_seed(i)).bfloat16() for i in (1, 2))
    eva.paged_append(cache, k.cuda(), v.cuda(), slots)
    q = query(2, 8, d, BF16)
    o = eva.paged_decode(cache, q.cuda())
    ks, vs = ([x[b, :, :n].transpose(0, 1) for b, n in enumerate((2 * P + 9, P))] for x in (k, v))
    check_rows(o, q, ks, vs, P, BF16)
    pages = eva.paged_select(cache, q.cuda(), 2)
    assert pages[1].tolist() == [[0, -1]] * 8 and pages[0].tolist() == [[0, 2]] * 8


# ---- choice -------------------------------------------------------------------
def check_choice(cache, q, lens, S, first, last):
    B, H, d = q.shape
    Hkv, P = cache.struct.H_kv, cache.struct.P
    pages = eva.paged_select(cache, q.cuda(), S, first, last).tolist()
    table, mean = cache.table.table.cpu().long(), cache.k_mean.cpu()
    for b, n in enumerate(lens):
        held = -(-n // P)
        for h in range(Hkv):
            want = choice(q[b].reshape(Hkv, -1, d)[h], mean[table[b, :held], h], held, S, first, last)
            assert pages[b][h] == want, f"b{b} kv{h}"
    return pages


# B, H, Hkv, d, P, lens, S, first, last
CHOICES = [
    (1, 1, 1, 64, 16, [1], 1, 0, 1),
    (3, 4, 2, 128, 16, [0, 16, 17], 2, 1, 1),
    (4, 12, 4, 64, 16, [2999, 300, 320, 337], 21, 1, 1),
    (2, 8, 8, 128, 64, [5000, 1100], 17, 0, 2),
    (2, 40, 2, 64, 32, [3333, 700], 9, 2, 3),       # 20 heads a kv head
    (2, 3, 1, 128, 32, [2000, 65], 4, 2, 2),        # nothing to rank: first and last alone
    (1, 4, 1, 64, 16, [80000], 300, 1, 1),          # 5000 pages: more scores than LDS holds
    (70, 2, 1, 64, 16, [(97 * i) % 700 for i in range(70)], 5, 1, 1),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,H,Hkv,d,P,lens,S,first,last", CHOICES)
def test_choice(B, H, Hkv, d, P, lens, S, first, last, dtype):
    cache, ks, vs = build(B, H, Hkv, d, P, lens, dtype, seed=S)
    q = query(B, H, d, dtype, seed=S)
    pages = check_choice(cache, q, lens, S, first, last)
    o = eva.paged_decode(cache, q.cuda(), pages=ints(pages))
    check_rows(o, q, ks, vs, P, dtype, pages)


@pytest.mark.parametrize("B,pages,Hkv", [(1, 120, 2), (2, 700, 3), (1, 4500, 1), (64, 300, 4)])
def test_choice_by_every_route(B, pages, Hkv):
    # scored by the choosing workgroup (few pages, or rows that fill the chip) or before it, kept in LDS or not
    lens = [16 * pages - 3 * (i % 5) for i in range(B)]
    lib = eva._lib.load()
    g = torch.Generator().manual_seed(pages)
    N = B * pages
    t = eva.PageTable(B, 16, N, 16 * pages)
    t.n_tok.copy_(ints(lens))
    t.table.copy_(torch.randperm(N, generator=g).int().view(B, pages))
    mean = torch.randn(N, Hkv, 64, generator=g)
    empty = torch.empty(N, Hkv, 16, 64, dtype=BF16, device="cuda")
    cache = eva.PagedCache(t, 2 * Hkv, Hkv, 64, storage=(empty, empty.view(N, Hkv, 2, 64, 8), mean.cuda()))
    alone = lib.eva_paged_select_workspace_bytes(cache.ref, t.ref, 40) == 0
    assert alone == (pages == 120 or B == 64)
    q = query(B, 2 * Hkv, 64, BF16, seed=pages)
    check_choice(cache, q, lens, 40, 2, 3)
    # one score far above all others, and more that tie than are ranked one against the other
    at = t.table.long()
    mean[:] = mean[0]
    mean[at[:, 5].cpu()] = 1e4 * q[:, ::2].float()
    mean[at[:, 7].cpu()] = -1e4 * q[:, ::2].float()
    mean[at[:, 20:60].cpu().flatten()] = mean[0] * 1.5
    cache.k_mean.copy_(mean)
    for S in (6, 30, 60, 100):
        check_choice(cache, q, lens, S, 1, 1)
    mean[at[:, 10:].cpu().flatten()] = NAN
    mean[at[:, 12].cpu()] = INF
    cache.k_mean.copy_(mean)
    for S in (3, 40, pages - 1):
        check_choice(cache, q, lens, S, 1, 1)


def test_equal_scores_take_the_lower_page():
    lens = [100 * 16]
    cache, *_ = build(1, 2, 1, 64, 16, lens, F32)
    mean = cache.k_mean
    at = cache.table.table[0].long()
    q = query(1, 2, 64, F32)
    mean[at] = mean[at[0]].clone()                  # all tie
    check_choice(cache, q, lens, 10, 1, 1)
    mean[at[50:]] *= 2                              # two groups that tie, of 50
    mean[at[60]] = 0.0                              # scores of 0 and -0
    mean[at[61]] = -0.0
    for S in (10, 49, 51, 60, 99):
        check_choice(cache, q, lens, S, 1, 1)
    mean[at] = 0.0
    mean[at[::2]] = -0.0
    assert check_choice(cache, q, lens, 7, 1, 1)[0][0] == [0, 1, 2, 3, 4, 5, 99]


def test_scores_that_are_not_finite_and_lost_pages():
    lens = [64 * 16] * 2
    cache, *_ = build(2, 4, 2, 64, 16, lens, F32)
    at = cache.table.table.long()
    cache.k_mean[at[0, 20], 0, 3] = NAN
    cache.k_mean[at[0, 30], 0, 3] = INF             # +inf for queries that are positive there
    cache.k_mean[at[0, 40], 1] = -INF               # NaN or -inf
    q = query(2, 4, 64, F32)
    q[0, :, 3] = 1.0
    pages = check_choice(cache, q, lens, 6, 1, 1)
    assert 20 in pages[0][0] and 30 in pages[0][0]
    # an entry outside the pool ranks first and makes the row NaN
    cache.table.table[1, 33] = cache.table.struct.n_pages
    pages = eva.paged_select(cache, q.cuda(), 6)
    assert (pages[1] == 33).any(-1).all()
    o = eva.paged_decode(cache, q.cuda(), pages=pages)
    assert o[1].isnan().all()


# ---- together -------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_prompt_generation_and_rollback(dtype):
    """A ragged batch: prompts (whose own attention is the prefill's, with a window of all tokens), generated
    tokens, a sequence that leaves and another that takes its place, rejected tokens, chosen pages."""
    B, H, Hkv, d, P, L, steps = 3, 6, 2, 64, 16, 90, 40
    g = torch.Generator().manual_seed(12)
    t = eva.PageTable(B, P, 40, 400)
    cache = eva.PagedCache(t, H, Hkv, d, dtype, fill=NAN)
    ks, vs = [torch.zeros(0, Hkv, d, dtype=dtype) for _ in range(B)], [torch.zeros(0, Hkv, d, dtype=dtype) for _ in range(B)]

    def add(T, counts):
        k, v = (torch.randn(B, Hkv, T, d, generator=g).to(dtype) for _ in range(2))
        slots, start, granted = eva.page_extend(t, T, ints(counts))
        assert start.tolist() == [len(x) for x in ks] and granted.tolist() == counts
        eva.paged_append(cache, k.cuda(), v.cuda(), slots)
        for b, c in enumerate(counts):
            ks[b] = torch.cat([ks[b], k[b, :, :c].transpose(0, 1)])
            vs[b] = torch.cat([vs[b], v[b, :, :c].transpose(0, 1)])
        return k, v

    def back(lens):
        eva.page_truncate(t, ints(lens))
        for b, n in enumerate(lens):
            ks[b], vs[b] = ks[b][:n], vs[b][:n]

    lens = [90, 31, 64]
    k, v = add(L, lens)
    q = torch.randn(B, H, L, d, generator=g).to(dtype)
    whole = eva.prefill(q.cuda(), k.cuda(), v.cuda(), W=L, C=16)
    last = torch.stack([q[b, :, n - 1] for b, n in enumerate(lens)])
    o = eva.paged_decode(cache, last.cuda())
    check_rows(o, last, ks, vs, P, dtype)
    # apart by each side's output rounding and by the prefill's rounded weights: 2^-8 of the largest value
    # each, and 2^-15 for the decode's weights
    same = torch.stack([whole[b, :, n - 1] for b, n in enumerate(lens)])
    assert (same.double() - o.double()).abs().max() <= (3 * 2.0 ** -8 + 2.0 ** -14) * float(v.abs().max())
    for s in range(steps):
        if s == 10:
            back([0, len(ks[1]), len(ks[2])])
            add(50, [50, 0, 0])
        if s % 7 == 3:                      # drafted tokens, of which some are taken back
            had = [len(x) for x in ks]
            add(8, [8, 5, 0])
            back([n + 1 for n in had])
        add(1, [1, 1, 1])
        q = query(B, H, d, dtype, seed=s)
        check_rows(eva.paged_decode(cache, q.cuda()), q, ks, vs, P, dtype)
        pages = check_choice(cache, q, [len(x) for x in ks], 5, 1, 1)
        check_rows(eva.paged_decode(cache, q.cuda(), pages=ints(pages)), q, ks, vs, P, dtype, pages)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_step_in_a_captured_graph(dtype):
    """A whole step replayed: counts, pages and slots advance on the device; each replay is compared with the
    same step made eagerly on a twin."""
    B, H, Hkv, d, P = 4, 8, 2, 64, 16
    lens = [1500, 40, 0, 15]
    g = torch.Generator().manual_seed(5)
    twins = [build(B, H, Hkv, d, P, lens, dtype, seed=2, most=4000, spare=60, garbage=0.0)[0] for _ in range(2)]
    q, k, v = (torch.empty(B, h, d, dtype=dtype, device="cuda") for h in (H, Hkv, Hkv))

    def step(cache):
        slots, start, granted = eva.page_extend(cache.table)
        eva.paged_append(cache, k, v, slots)
        pages = eva.paged_select(cache, q, 6)
        return eva.paged_decode(cache, q), eva.paged_decode(cache, q, pages=pages), pages, slots

    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    for x in (q, k, v):
        x.copy_(torch.randn(x.shape, generator=g))
    step(twins[0])
    step(twins[1])
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        out = step(twins[0])
    for i in range(20):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=g))
        graph.replay()
        want = step(twins[1])
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b), f"replay {i}"
        assert torch.equal(twins[0].k_mean, twins[1].k_mean) and torch.equal(twins[0].table.table, twins[1].table.table)


def test_two_streams_and_two_graphs_at_once():
    # calls that overlap have workspaces of their own
    caches = [build(2, 8, 2, 128, 32, [5000 + 300 * i, 77], seed=i) for i in range(2)]
    qs = [query(2, 8, 128, BF16, seed=i).cuda() for i in range(2)]
    want = [eva.paged_decode(c[0], q) for c, q in zip(caches, qs)]
    torch.cuda.synchronize()
    streams, graphs, outs = [torch.cuda.Stream() for _ in range(2)], [], []
    for c, q, s in zip(caches, qs, streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            pages = eva.paged_select(c[0], q, 9)
            outs.append((eva.paged_decode(c[0], q), eva.paged_decode(c[0], q, pages=pages)))
        graphs.append(graph)
    for _ in range(5):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for o, w, c, q in zip(outs, want, caches, qs):
            assert torch.equal(o[0], w)
            assert torch.equal(o[1], eva.paged_decode(c[0], q, pages=eva.paged_select(c[0], q, 9)))


def test_layers_share_a_table_with_head_norms_between():
    """Two layers of different heads on one table, queries and keys from qk_norm_rope at page_extend's positions."""
    B, d, P = 3, 64, 32
    t = eva.PageTable(B, P, 30, 300)
    shapes = ((4, 2), (8, 8))
    layers = [eva.PagedCache(t, H, Hkv, d) for H, Hkv in shapes]
    turns = eva.rope_turns(32)
    rows = [[[], []] for _ in shapes]
    g = torch.Generator().manual_seed(3)
    had = [0] * B
    for T, counts in ((70, [70, 33, 1]), (1, [1, 1, 1]), (1, [1, 0, 1])):
        slots, start, _ = eva.page_extend(t, T, ints(counts))
        for layer, (H, Hkv), r in zip(layers, shapes, rows):
            x = torch.randn(B, T, (H + 2 * Hkv) * d, generator=g).bfloat16().cuda()
            q, k, v = eva.qk_norm_rope(x, H, Hkv, turns=turns, start=start)
            eva.paged_append(layer, k, v, slots)
            for b, c in enumerate(counts):
                for store, y in zip(r, (k, v)):
                    new = y[b, :, :c].transpose(0, 1).cpu()
                    if len(store) <= b:
                        store.append(new)
                    else:
                        store[b] = torch.cat([store[b], new])
            last = torch.stack([q[b, :, max(c - 1, 0)] for b, c in enumerate(counts)]).contiguous()
            o = eva.paged_decode(layer, last)
            check_rows(o, last.cpu(), r[0], r[1], P, BF16)
        had = [h + c for h, c in zip(had, counts)]
    assert t.n_tok.tolist() == had
