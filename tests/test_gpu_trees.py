"""Attention of drafted trees over ragged caches (bf16, fp32, 8-bit) and the
append of accepted paths, against plain 64-bit models (rows_reference.py)."""
import math

import pytest
import torch

from paper_2511_00576_amd import _lib, eva, inputs
from rows_reference import ALIGNED, BLOCKED, SLIDING, Model, line_of, plain, quantised, random_tree, row

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    eva._lib.load()


def start(kind, B, H, Hkv, d, W, C, lens, window, seed, fill=math.nan, room=128, R=None):
    """A cache filled with prompts of the given lengths, and its models."""
    dtype = F32 if kind == "f32" else BF16
    L = max(max(lens), 1)
    _, k, v = inputs.qkv(B, H, Hkv, L, d, dtype, seed=seed)
    if kind == "e4m3":
        cache = eva.QuantCache(B, H, Hkv, d, W, C, max_tokens=L + room, fill=fill, window=window, R=R)
    else:
        cache = eva.RaggedCache(B, H, Hkv, d, W, C, max_tokens=L + room, dtype=dtype, fill=fill, window=window, R=R)
    Ks, Vs = eva.build_summaries(k.cuda(), v.cuda(), C)
    fill_ = eva.qcache_fill if kind == "e4m3" else eva.rcache_fill
    fill_(cache, k.cuda(), v.cuda(), Ks, Vs, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    held = quantised if kind == "e4m3" else plain
    Ks, Vs = Ks.cpu(), Vs.cpu()
    models = [[Model(k[b, g, :n], v[b, g, :n], Ks[b, g, :n // C], Vs[b, g, :n // C], W, C, window, held) for g in range(Hkv)]
              for b, n in enumerate(lens)]
    return cache, models, dtype


def draft(B, H, Hkv, T, d, dtype, seed):
    g = torch.Generator().manual_seed(seed + 77)
    return [torch.randn(B, h, T, d, generator=g).to(dtype) for h in (H, Hkv, Hkv)]


def check(o, q, k, v, parents, models, dtype, nodes=None, active=None, left=None):
    B, H, T, d = q.shape
    G = H // k.shape[1]
    o = o.cpu().double()
    for b in range(B):
        for t in range(T):
            if (nodes is not None and t >= nodes[b]) or (active is not None and not active[b]):
                if left is not None:
                    assert (o[b, :, t] == left).all(), f"row {b}, {t} was written"
                continue
            line = line_of(parents[b].tolist(), t)
            for g, m in enumerate(models[b]):
                p = len(m.k) + len(line) - 1
                kk, vv, bias = m.keys(p, [(k[b, g, i].double(), v[b, g, i].double()) for i in line])
                ref, bound = row(q[b, g * G:(g + 1) * G, t], kk, vv, bias, dtype)
                got = o[b, g * G:(g + 1) * G, t]
                assert torch.isfinite(got).all(), f"b{b} g{g} node {t}: not finite"
                over = ((got - ref).abs() - bound).max()
                assert over <= 0, f"b{b} g{g} node {t}: {float(over):.3e} over the bound"


def run(kind, B, H, Hkv, d, W, C, lens, T, window=SLIDING, seed=1, use_workspace=True, parents=None):
    print(f"tree {kind} B{B} H{H}/{Hkv} d{d} W{W} C{C} T{T} lens={lens} window={window} ws={use_workspace}", flush=True)
    cache, models, dtype = start(kind, B, H, Hkv, d, W, C, lens, window, seed)
    q, k, v = draft(B, H, Hkv, T, d, dtype, seed)
    if parents is None:
        parents = random_tree(B, T, torch.Generator().manual_seed(seed))
    o = eva.tree_attention(cache, q.cuda(), k.cuda(), v.cuda(), parents.cuda(), use_workspace=use_workspace)
    check(o, q, k, v, parents, models, dtype)
    return cache, models, (q, k, v), o


# B, H, Hkv, d, W, C, lens, T, window
SHAPES = [
    (1, 1, 1, 64, 1, 1, [0], 1, SLIDING),              # an empty sequence: the node alone
    (2, 2, 1, 128, 16, 4, [0, 1], 3, SLIDING),
    (1, 32, 8, 128, 256, 64, [777], 8, SLIDING),       # 32 columns
    (3, 4, 4, 64, 33, 7, [40, 500, 31], 33, SLIDING),  # T = W, odd everything
    (2, 8, 1, 128, 64, 16, [1000, 64], 64, SLIDING),   # 512 columns, the largest tree
    (2, 12, 4, 64, 200, 24, [611, 199], 13, ALIGNED),
    (2, 5, 1, 128, 100, 33, [340, 99], 11, ALIGNED),   # 55 columns
    (3, 16, 2, 128, 128, 8, [300, 127, 128], 1, BLOCKED),
    (4, 8, 8, 128, 64, 64, [63, 64, 65, 191], 5, SLIDING),
    (1, 24, 1, 64, 512, 256, [2000], 4, SLIDING),      # 96 columns of one kv head
    (2, 40, 2, 64, 96, 32, [333, 95], 1, SLIDING),     # 20 columns
]


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_tree(kind, shape):
    B, H, Hkv, d, W, C, lens, T, window = shape
    run(kind, B, H, Hkv, d, W, C, lens, T, window, seed=T + W)


# more than 512 workgroups of 16 columns: the shapes that bf16 and 8-bit caches
# take through LDS, 64 columns a workgroup or 128
WIDE = [
    (66, 8, 2, 128, 64, 16, 13, SLIDING),   # 52 columns
    (129, 4, 2, 64, 20, 5, 20, ALIGNED),    # 40, T = W
    (18, 16, 2, 64, 100, 33, 63, SLIDING),  # 504
    (17, 8, 1, 128, 64, 8, 64, SLIDING),    # 512, the largest tree
    (40, 24, 2, 128, 33, 7, 12, ALIGNED),   # 144
]


def wide_lens(B):
    return [(37 * i) % 200 if i % 5 else 300 + i for i in range(B)]


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "f32"])
@pytest.mark.parametrize("shape", WIDE)
def test_many_columns(kind, shape):
    B, H, Hkv, d, W, C, T, window = shape
    assert B * Hkv * -(-H // Hkv * T // 16) > 512
    run(kind, B, H, Hkv, d, W, C, wide_lens(B), T, window, seed=T + W)


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "f32"])
@pytest.mark.parametrize("T", [2, 20])
def test_long_rows_are_split_and_joined(kind, T):
    # 2000 summaries and a long window of one sequence: rows go over several
    # workgroups with a workspace, and over one without
    for ws in (True, False):
        cache, *_ = run(kind, 1, 4, 2, 64, 700, 4, [8700], T, seed=5, use_workspace=ws)
    n = eva._lib.load()
    size = n.eva_qtree_workspace_bytes if kind == "e4m3" else n.eva_rtree_workspace_bytes
    assert size(eva.ctypes.byref(cache.struct), T) > 0, "the shape must split its rows"


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "f32"])
def test_many_units(kind):
    # 300 units of 16 columns: no splits, four waves each
    run(kind, 75, 4, 4, 64, 40, 8, [(37 * i) % 200 for i in range(75)], 5, seed=9)


@pytest.mark.parametrize("B,H,T", [(2, 4, 5), (130, 8, 10)])  # 16 and 64 columns a workgroup
def test_stale_exponent_bytes(B, H, T):
    """Bytes that no row has, where there is no row: of scales that are infinite."""
    lens = [30 + 3 * (b % 7) for b in range(B)]
    cache, models, dtype = start("e4m3", B, H, 2, 128, 100, 16, lens, SLIDING, 6)
    q, k, v = draft(B, H, 2, T, 128, dtype, 6)
    parents = random_tree(B, T, torch.Generator().manual_seed(6))
    for b, n in enumerate(lens):
        for ring, held in ((cache.k_ring_exp, n), (cache.v_ring_exp, n), (cache.k_sum_exp, n // 16), (cache.v_sum_exp, n // 16)):
            ring[b, :, held:] = 255
    o = eva.tree_attention(cache, q.cuda(), k.cuda(), v.cuda(), parents.cuda())
    check(o, q, k, v, parents, models, dtype)


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "f32"])
@pytest.mark.parametrize("d,T", [(64, 5), (128, 1)])
def test_units_that_nearly_fill_the_chip(kind, d, T):
    # 150 workgroups with a window of several chunks: not split, 12 waves each
    run(kind, 50, 6, 3, d, 200, 16, wide_lens(50), T, SLIDING, seed=d + T)


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "f32"])
@pytest.mark.parametrize("times", [1, 12])  # 12: shapes of many columns
def test_sizes_activity_and_rows_left_as_they_were(kind, times):
    B, H, Hkv, d, W, C, T = 5 * times, 8, 2, 128, 64, 16, 20
    cache, models, dtype = start(kind, B, H, Hkv, d, W, C, [100, 3, 0, 64, 200] * times, SLIDING, 3)
    q, k, v = draft(B, H, Hkv, T, d, dtype, 3)
    parents = random_tree(B, T, torch.Generator().manual_seed(4))
    nodes, active = [20, 7, 1, 0, 13] * times, [1, 1, 1, 1, 0] * times
    # absent nodes hold what a padded batch may hold
    for b in range(B):
        parents[b, nodes[b]:] = 10 ** 9
        for x in (q, k, v):
            x[b, :, nodes[b]:] = math.nan
    out = torch.full((B, H, T, d), 7.0, dtype=dtype, device="cuda")
    before = {n: t.clone() for n, t in vars(cache).items() if torch.is_tensor(t)}
    o = eva.tree_attention(cache, q.cuda(), k.cuda(), v.cuda(), parents.cuda(),
                           n_nodes=torch.tensor(nodes, dtype=torch.int32, device="cuda"),
                           active=torch.tensor(active, dtype=torch.int32, device="cuda"), out=out)
    assert o is out
    check(o, q, k, v, parents, models, dtype, nodes, active, left=7.0)
    for n, t in before.items():
        assert torch.equal(t.view(torch.uint8), getattr(cache, n).view(torch.uint8)), f"{n} was written"
    # sizes out of range are clamped
    o = eva.tree_attention(cache, q[:, :, :5].contiguous().cuda(), k[:, :, :5].contiguous().cuda(),
                           v[:, :, :5].contiguous().cuda(), parents[:, :5].contiguous().cuda(),
                           n_nodes=torch.tensor([9, 5, -3, 0, 5] * times, dtype=torch.int32, device="cuda"),
                           out=torch.full((B, H, 5, d), 7.0, dtype=dtype, device="cuda"))
    check(o[:2], q[:2, :, :5], k[:2, :, :5], v[:2, :, :5], parents[:2], models[:2], dtype)
    assert (o[2:4] == 7).all()


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "f32"])
def test_parents_that_name_no_earlier_node_make_roots(kind):
    parents = torch.tensor([[-1, 1, 0, 70, -9, 4, 2 ** 31 - 1, 6]], dtype=torch.int32)
    clean = torch.tensor([[-1, -1, 0, -1, -1, 4, -1, 6]], dtype=torch.int32)
    cache, models, dtype = start(kind, 1, 4, 2, 64, 32, 8, [77], SLIDING, 6)
    q, k, v = draft(1, 4, 2, 8, 64, dtype, 6)
    o = eva.tree_attention(cache, q.cuda(), k.cuda(), v.cuda(), parents.cuda())
    check(o, q, k, v, clean, models, dtype)


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("B,H", [(1, 4), (172, 4), (90, 8)])  # 16, 64 and 128 columns a workgroup
def test_values_that_are_not_finite_reach_only_the_rows_that_see_them(kind, bad, B, H):
    """A drafted sibling, a position that only shallow nodes still see, and the
    newest summary that only deep ones see."""
    Hkv, d, W, C, T, n = 1, 64, 32, 8, 12, 103
    dtype = F32 if kind == "f32" else BF16
    parents = torch.tensor([[-1, 0, 1, 2, 3, 4, 5, 6, 7, 0, 9, -1]] * B, dtype=torch.int32)
    depth = [len(line_of(parents[0].tolist(), t)) - 1 for t in range(T)]
    q, k, v = (x.repeat(B, 1, 1, 1) for x in draft(1, H, Hkv, T, d, dtype, 8))
    _, K, V = (x.repeat(B, 1, 1, 1) for x in inputs.qkv(1, H, Hkv, n, d, dtype, seed=8))
    Ks, Vs = (t.cpu() for t in eva.build_summaries(K.cuda(), V.cuda(), C))
    lo = [first for first in (n + dd - W + 1 for dd in depth)]
    place = n - W + 3          # seen up to depth 2
    chunk = max(lo) // C - 1   # seen by the deepest alone
    for what in ("draft", "ring", "summary"):
        k2, v2, V2, Vs2 = k.clone(), v.clone(), V.clone(), Vs.clone()
        if what == "draft":
            v2[:, 0, 9, 5] = bad   # node 9: seen by 9 and 10
            sees = [9 in line_of(parents[0].tolist(), t) for t in range(T)]
        elif what == "ring":
            V2[:, 0, place, 5] = bad
            sees = [x <= place for x in lo]
        else:
            Vs2[:, 0, chunk, 5] = bad
            sees = [x // C > chunk for x in lo]
        assert any(sees) and not all(sees)
        if kind == "e4m3":
            cache = eva.QuantCache(B, H, Hkv, d, W, C, max_tokens=n + 64, fill=math.nan)
            eva.qcache_fill(cache, K.cuda(), V2.cuda(), Ks.cuda(), Vs2.cuda(), torch.tensor([n] * B, dtype=torch.int32, device="cuda"))
        else:
            cache = eva.RaggedCache(B, H, Hkv, d, W, C, max_tokens=n + 64, dtype=dtype, fill=math.nan)
            eva.rcache_fill(cache, K.cuda(), V2.cuda(), Ks.cuda(), Vs2.cuda(), torch.tensor([n] * B, dtype=torch.int32, device="cuda"))
        o = eva.tree_attention(cache, q.cuda(), k2.cuda(), v2.cuda(), parents.cuda()).cpu().float()
        assert torch.equal(o.isnan(), o[:1].expand_as(o).isnan()) and torch.equal(o.nan_to_num(), o[:1].expand_as(o).nan_to_num())
        # an 8-bit row holds NaN for what is not finite
        want = math.nan if kind == "e4m3" and what != "draft" else bad
        for t in range(T):
            x = o[0, :, t]
            assert torch.isfinite(x[:, :5]).all() and torch.isfinite(x[:, 6:]).all(), (what, t)
            if not sees[t]:
                assert torch.isfinite(x[:, 5]).all(), (what, t)
            elif math.isnan(want):
                assert torch.isnan(x[:, 5]).all(), (what, t)
            else:
                assert (x[:, 5] == want).all(), (what, t)


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "f32"])
def test_extreme_logits(kind):
    # logits of several thousand, one key far above all others, and keys of the
    # type's lowest value: the softmax takes its maximum first
    cache, models, dtype = start(kind, 1, 2, 1, 64, 16, 4, [50], SLIDING, 2)
    q, k, v = draft(1, 2, 1, 6, 64, dtype, 2)
    q *= 300
    k[0, 0, 2] *= 100
    parents = torch.tensor([[-1, 0, 1, 2, -1, 4]], dtype=torch.int32)
    o = eva.tree_attention(cache, q.cuda(), k.cuda(), v.cuda(), parents.cuda())
    check(o, q, k, v, parents, models, dtype)
    q = torch.full_like(q, 1e-3)
    k[0, 0, 4] = torch.finfo(dtype).min
    o = eva.tree_attention(cache, q.cuda(), k.cuda(), v.cuda(), parents.cuda()).cpu().float()
    assert torch.isfinite(o).all()


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "f32"])
@pytest.mark.parametrize("W,C,n,T", [(64, 16, 250, 40), (8, 1, 30, 8), (33, 7, 20, 33), (64, 96, 500, 64)])
def test_path_is_the_same_as_tokens_one_by_one(kind, W, C, n, T):
    # several chunks complete inside a path, a ring wraps inside it
    B, H, Hkv, d = 3, 4, 2, 64
    lens = [n, n - 3, 0]
    a, _, dtype = start(kind, B, H, Hkv, d, W, C, lens, SLIDING, 5, fill=0.0)
    b, _, _ = start(kind, B, H, Hkv, d, W, C, lens, SLIDING, 5, fill=0.0)
    _, k, v = draft(B, H, Hkv, T, d, dtype, 5)
    gen = torch.Generator().manual_seed(1)
    path = torch.stack([torch.randperm(T, generator=gen) for _ in range(B)]).int()
    path[1, 1] = path[1, 0]                      # the same token twice
    counts = torch.tensor([T, T // 2, T - 1], dtype=torch.int32)
    eva.append_path(a, k.cuda(), v.cuda(), path.cuda(), counts.cuda())
    one = eva.qcache_append if kind == "e4m3" else eva.rcache_append
    for i in range(T):
        at = path[:, i].long()
        rows = [x[torch.arange(B), :, at].contiguous().cuda() for x in (k, v)]
        one(b, *rows, active=(i < counts).int().cuda())
    torch.cuda.synchronize()
    assert a.n_tok.tolist() == [x + c for x, c in zip(lens, counts.tolist())]
    for name, t in vars(a).items():
        if torch.is_tensor(t):
            assert torch.equal(t.view(torch.uint8), getattr(b, name).view(torch.uint8)), name


@pytest.mark.parametrize("rf", [0.1])
def test_path_of_a_cache_with_stochastic_summaries(rf):
    B, H, Hkv, d, W, C, T = 2, 4, 2, 64, 32, 8, 20
    caches = [eva.RaggedCache(B, H, Hkv, d, W, C, 100, fill=0.0, rf_lambda=rf, rf_seed=9) for _ in range(2)]
    _, k, v = draft(B, H, Hkv, T, d, BF16, 1)
    eva.append_path(caches[0], k.cuda(), v.cuda())
    for i in range(T):
        eva.rcache_append(caches[1], k[:, :, i].contiguous().cuda(), v[:, :, i].contiguous().cuda())
    assert caches[0].n_tok.tolist() == [T, T]
    for name in ("k_ring", "vt_ring", "k_sum", "vt_sum", "arrive"):
        assert torch.equal(getattr(caches[0], name), getattr(caches[1], name)), name


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "f32"])
def test_paths_that_end_early(kind):
    B, H, Hkv, d, W, C, T = 5, 2, 1, 64, 32, 8, 6
    cache, _, dtype = start(kind, B, H, Hkv, d, W, C, [20, 20, 20, 20, 20], SLIDING, 4, fill=0.0, room=4)
    _, k, v = draft(B, H, Hkv, T, d, dtype, 4)
    path = torch.arange(T).repeat(B, 1).int()
    path[0, 2] = T           # no such token: two are taken
    path[1, 0] = -1          # none
    counts = torch.tensor([5, 5, 99, -4, 3], dtype=torch.int32)  # the third is full after 4
    active = torch.tensor([1, 1, 1, 1, 0], dtype=torch.int32)
    eva.append_path(cache, k.cuda(), v.cuda(), path.cuda(), counts.cuda(), active.cuda())
    assert cache.n_tok.tolist() == [22, 20, 24, 20, 20] and cache.arrive.tolist() == [0] * B


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "f32"])
def test_drafted_generation(kind):
    """Norms and rotation of drafted tokens, the tree's rows, the accepted path
    into the cache, three times over, against the model throughout."""
    B, H, Hkv, d, W, C, T = 3, 8, 2, 64, 48, 8, 12
    lens = [60, 7, 131]
    cache, models, dtype = start(kind, B, H, Hkv, d, W, C, lens, SLIDING, 21)
    gen = torch.Generator().manual_seed(2)
    turns = eva.rope_turns(d)
    w = (1 + 0.1 * torch.randn(d, generator=gen)).to(dtype).cuda()
    for step in range(3):
        x = torch.randn(B, T, (H + 2 * Hkv) * d, generator=gen).to(dtype).cuda()
        parents = random_tree(B, T, gen)
        depth = torch.tensor([[len(line_of(parents[b].tolist(), t)) - 1 for t in range(T)] for b in range(B)],
                             dtype=torch.int32)
        q, k, v = eva.qk_norm_rope(x, H, Hkv, turns=turns, q_weight=w, k_weight=w, start=cache.n_tok, offsets=depth.cuda())
        o = eva.tree_attention(cache, q, k, v, parents.cuda())
        q, k, v = q.cpu(), k.cpu(), v.cpu()
        check(o, q, k, v, parents, models, dtype)
        path, counts = torch.zeros(B, T, dtype=torch.int32), torch.zeros(B, dtype=torch.int32)
        for b in range(B):
            line = line_of(parents[b].tolist(), int(torch.randint(0, T, (1,), generator=gen)))
            path[b, :len(line)] = torch.tensor(line, dtype=torch.int32)
            counts[b] = len(line)
            for g, m in enumerate(models[b]):
                for t in line:
                    m.append(k[b, g, t], v[b, g, t])
        eva.append_path(cache, k.cuda(), v.cuda(), path.cuda(), counts.cuda())
        assert cache.n_tok.tolist() == [len(m[0].k) for m in models]
        # the models go on with the summaries as the cache holds them
        to = eva.qcache_read(cache, eva.RaggedCache(B, H, Hkv, d, W, C, cache.struct.max_tok)) if kind == "e4m3" else cache
        ks, vt = to.k_sum.cpu().double(), to.vt_sum.cpu().double()
        vs = vt.permute(0, 1, 2, 4, 3).reshape(ks.shape)
        step_ = {"bf16": 2.0 ** -8, "e4m3": 2.0 ** -4, "f32": 0.0}[kind]
        for b in range(B):
            for g, m in enumerate(models[b]):
                for i in range(len(m.ks)):
                    for ref, got in ((m.ks, ks), (m.vs, vs)):
                        x = got[b, g, i]
                        # half a step of the cache's type, or of its smallest
                        # entries (2^-10 of a power of two that 448 of them
                        # hold the row's largest), and sums of C rows in fp32
                        top = ref[i].abs().max()
                        low = 2.0 ** -10 * 2 * top / 224 if kind == "e4m3" else 0.0
                        assert ((x - ref[i]).abs() <= step_ * ref[i].abs() + low + 4 * (C + d) * 2.0 ** -24 * (1 + top) * 4).all()
                        ref[i] = x


def test_another_stream_and_replayed_capture():
    """Two captured graphs and eager calls take turns on one cache: workspaces
    belong to a call."""
    B, H, Hkv, d, W, C, T = 1, 4, 1, 64, 600, 4, 6
    for kind in ("bf16", "e4m3"):
        cache, models, dtype = start(kind, B, H, Hkv, d, W, C, [3000], SLIDING, 13)
        sets = [[t.cuda() for t in draft(B, H, Hkv, T, d, dtype, s)] for s in (1, 2)]
        parents = random_tree(B, T, torch.Generator().manual_seed(3)).cuda()
        eager = [eva.tree_attention(cache, *x, parents) for x in sets]
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            eva.tree_attention(cache, *sets[0], parents)
        torch.cuda.synchronize()
        graphs, held = [], []
        for x in sets:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                held.append(eva.tree_attention(cache, *x, parents))
            graphs.append(g)
        for i in range(4):
            for g in graphs:
                g.replay()
            again = [eva.tree_attention(cache, *x, parents) for x in sets]
            torch.cuda.synchronize()
            for a, b, c in zip(held, again, eager):
                assert torch.equal(a, c) and torch.equal(b, c), f"replay {i}"
            for h in held:
                h.zero_()


def test_captured_generation_step():
    # tree attention and path append in one graph: the counts advance on the device
    B, H, Hkv, d, W, C, T = 2, 4, 2, 64, 64, 8, 4
    for kind in ("bf16", "e4m3"):
        (a, _, dtype), (b, _, _) = (start(kind, B, H, Hkv, d, W, C, [50, 9], SLIDING, 17, fill=0.0) for _ in range(2))
        q, k, v = (t.cuda() for t in draft(B, H, Hkv, T, d, dtype, 17))
        parents = torch.tensor([[-1, 0, 1, 0]] * B, dtype=torch.int32, device="cuda")
        path = torch.tensor([[0, 3, 0, 0]] * B, dtype=torch.int32, device="cuda")
        counts = torch.tensor([2, 1], dtype=torch.int32, device="cuda")

        def step(c):
            o = eva.tree_attention(c, q, k, v, parents)
            eva.append_path(c, k, v, path, counts)
            return o

        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            step(a)
        torch.cuda.synchronize()
        step(b)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            held = step(a)
        for i in range(5):
            g.replay()
            o = step(b)
            torch.cuda.synchronize()
            assert torch.equal(held, o) and torch.equal(a.n_tok, b.n_tok), f"replay {i}"
        assert a.n_tok.tolist() == [50 + 12, 9 + 6]


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "f32"])
def test_refusals(kind):
    B, H, Hkv, d, W, C, T = 2, 4, 2, 64, 16, 4, 3
    cache, _, dtype = start(kind, B, H, Hkv, d, W, C, [20, 5], SLIDING, 1, fill=0.0)
    q, k, v = (t.cuda() for t in draft(B, H, Hkv, T, d, dtype, 1))
    p = torch.full((B, T), -1, dtype=torch.int32, device="cuda")
    other = F32 if dtype == BF16 else BF16
    for bad, error in [
        ((q.to(other), k, v, p), ValueError), ((q, k.to(other), v, p), ValueError), ((q, k, v[:1], p), ValueError),
        ((q, k, v, p.long()), ValueError), ((q, k, v, p[:1]), ValueError), ((q[0], k, v, p), ValueError),
        ((q.cpu(), k, v, p), RuntimeError), ((q, k, v, p.cpu()), RuntimeError),
        ((q.transpose(2, 3).contiguous().transpose(2, 3), k, v, p), ValueError),
    ]:
        with pytest.raises(error):
            eva.tree_attention(cache, *bad)
    with pytest.raises(ValueError):
        eva.tree_attention(cache, q, k, v, p, n_nodes=torch.zeros(B, device="cuda"))
    with pytest.raises(ValueError):
        eva.tree_attention(cache, q, k, v, p, out=torch.empty(B, H, d, T, dtype=dtype, device="cuda"))
    q, k, v = (t.cuda() for t in draft(B, H, Hkv, W + 1, d, dtype, 1))  # deeper than the window
    p = torch.full((B, W + 1), -1, dtype=torch.int32, device="cuda")
    with pytest.raises(_lib.EvaError):
        eva.tree_attention(cache, q, k, v, p)
    with pytest.raises(_lib.EvaError):
        eva.append_path(cache, k, v)
    with pytest.raises(ValueError):
        eva.append_path(cache, k, v[:, :, :3])
    with pytest.raises(ValueError):
        eva.append_path(cache, k, v, path=p[:, :3])
    cache, _, _ = start(kind, B, H, Hkv, d, 70, C, [20, 5], BLOCKED, 1, fill=0.0)
    q, k, v = (t.cuda() for t in draft(B, H, Hkv, 2, d, dtype, 1))
    with pytest.raises(_lib.EvaError):
        eva.tree_attention(cache, q, k, v, torch.full((B, 2), -1, dtype=torch.int32, device="cuda"))
    q, k, v = (t.cuda() for t in draft(B, H, Hkv, 65, d, dtype, 1))
    with pytest.raises(_lib.EvaError):
        eva.append_path(cache, k, v)
