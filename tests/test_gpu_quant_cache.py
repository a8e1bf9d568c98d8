"""The 8-bit decode cache: codes and exponents of every write against torch's
own e4m3 conversion, rows read back, decode rows against the 64-bit model of
the same codes (rows_reference.py)."""
import math

import pytest
import torch

from paper_2511_00576_amd import _lib, eva, inputs
from rows_reference import ALIGNED, BLOCKED, SLIDING, Model, quantise, quantised, row, value

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    eva._lib.load()


def untile(vt):
    """[B, Hkv, n / 16, d, 16] -> [B, Hkv, n, d]."""
    B, Hkv, n, d, _ = vt.shape
    return vt.permute(0, 1, 2, 4, 3).reshape(B, Hkv, n * 16, d)


def arrays(c):
    """Codes (as bytes) and exponents of keys and values, ring and summaries."""
    u8 = lambda t: t.view(torch.uint8).cpu()  # noqa: E731
    return {"kr": (u8(c.k_ring), c.k_ring_exp.cpu()), "vr": (untile(u8(c.vt_ring)), c.v_ring_exp.cpu()),
            "ks": (u8(c.k_sum), c.k_sum_exp.cpu()), "vs": (untile(u8(c.vt_sum)), c.v_sum_exp.cpu())}


def same_rows(got, at, rows, what):
    """The held rows got[..., at, :] are the quantised `rows` [n, d]."""
    codes, exp = quantise(rows)
    have, hexp = got[0][at], got[1][at]
    assert torch.equal(hexp, exp), f"{what}: exponents"
    nan = torch.isnan(codes.float())
    assert torch.equal(torch.where(nan, 0, have & (255 - 0)), torch.where(nan, 0, codes.view(torch.uint8))), f"{what}: codes"
    assert ((have[nan] & 0x7f) == 0x7f).all(), f"{what}: NaN"


def prompts(B, Hkv, L, d, seed, scale=True):
    g = torch.Generator().manual_seed(seed)
    k, v = (torch.randn(B, Hkv, L, d, generator=g) for _ in range(2))
    if scale:  # rows of very different size
        k *= torch.pow(2.0, torch.randint(-30, 30, (B, Hkv, L, 1), generator=g).float())
        v *= torch.pow(2.0, torch.randint(-6, 6, (B, Hkv, L, 1), generator=g).float())
    return k.bfloat16(), v.bfloat16()


def special_rows(k):
    """Rows at the format's edges: zeros, one entry, 448 and just above, ties,
    bf16's smallest and largest, infinities and NaN."""
    d = k.shape[-1]
    rows = torch.zeros(12, d)
    rows[1, 3] = -5.0
    rows[2] = torch.linspace(1, 448, d)
    rows[3] = torch.linspace(1, 450, d)
    rows[4] = 17 + 2 * torch.arange(d) % 64          # halfway between codes
    rows[5, :3] = torch.tensor([3e38, -3.3e38, 1.0])
    rows[6, :3] = torch.tensor([1e-38, 1e-40, -9.2e-41])
    rows[7] = torch.randn(d, generator=torch.Generator().manual_seed(1))
    rows[7, 5] = math.nan
    rows[8, 5], rows[8, 6], rows[8, 7] = math.inf, 2.0, -0.5
    rows[9] = -math.inf
    rows[10] = -0.0
    rows[11] = 448 * 2.0 ** -20
    n = min(k.shape[2], len(rows))
    k[:, :, :n] = rows[:n].bfloat16()


@pytest.mark.parametrize("B,Hkv,d,W,C,lens,R", [
    (1, 1, 64, 1, 1, [1], None),
    (2, 3, 128, 100, 7, [0, 333], None),
    (3, 2, 64, 64, 64, [63, 64, 127], None),
    (4, 1, 128, 200, 24, [700, 1, 263, 512], 320),
    (2, 2, 64, 16, 4, [15, 900], 192),
])
def test_fill_and_read_back(B, Hkv, d, W, C, lens, R):
    L = max(lens)
    k, v = prompts(B, Hkv, L, d, 1)
    special_rows(k)
    special_rows(v)
    Ks, Vs = prompts(B, Hkv, L // C, d, 2)
    cache = eva.QuantCache(B, Hkv, Hkv, d, W, C, max_tokens=L, fill=math.nan, R=R)
    marked = {n: t.clone() for n, t in arrays(cache).items() for t in [t[0]]}
    eva.qcache_fill(cache, k.cuda(), v.cuda(), Ks.cuda(), Vs.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    assert cache.n_tok.tolist() == lens
    got = arrays(cache)
    R = cache.R
    to = eva.RaggedCache(B, Hkv, Hkv, d, W, C, max_tokens=L + 5, fill=7.0)
    assert eva.qcache_read(cache, to) is to
    assert to.n_tok.tolist() == lens and to.arrive.tolist() == [0] * B
    tk, tv = to.k_ring.cpu().double(), to.vt_ring.cpu().double().permute(0, 1, 2, 4, 3).reshape(to.k_ring.shape)
    tks, tvs = to.k_sum.cpu().double(), to.vt_sum.cpu().double().permute(0, 1, 2, 4, 3).reshape(to.k_sum.shape)

    def as_bf16(rows):  # below 2^-126 bf16 is subnormal
        return value(*quantise(rows)).to(torch.bfloat16).double()

    for b, n in enumerate(lens):
        pos = torch.arange(max(0, n - R), n)
        near = pos[-min(R, to.R):] if n else pos
        for g in range(Hkv):
            same_rows((got["kr"][0][b, g], got["kr"][1][b, g]), pos % R, k[b, g, pos], "keys")
            same_rows((got["vr"][0][b, g], got["vr"][1][b, g]), pos % R, v[b, g, pos], "values")
            s = torch.arange(n // C)
            same_rows((got["ks"][0][b, g], got["ks"][1][b, g]), s, Ks[b, g, s], "summary keys")
            same_rows((got["vs"][0][b, g], got["vs"][1][b, g]), s, Vs[b, g, s], "summary values")
            # nothing else was written
            free = torch.ones(R, dtype=torch.bool)
            free[pos % R] = False
            assert torch.equal(got["kr"][0][b, g, free], marked["kr"][b, g, free])
            assert torch.equal(got["vr"][0][b, g, free], marked["vr"][b, g, free])
            assert torch.equal(got["ks"][0][b, g, n // C:], marked["ks"][b, g, n // C:])
            assert torch.equal(got["vs"][0][b, g, n // C:], marked["vs"][b, g, n // C:])
            for t, rows, at in ((tk, k[b, g, near], near % to.R), (tv, v[b, g, near], near % to.R),
                                (tks, Ks[b, g, s], s), (tvs, Vs[b, g, s], s)):
                assert torch.equal(torch.nan_to_num(t[b, g, at], nan=1e30), torch.nan_to_num(as_bf16(rows), nan=1e30))
                rest = torch.ones(t.shape[2], dtype=torch.bool)
                rest[at] = False
                assert (t[b, g, rest] == 7).all()


def test_fill_takes_no_padding_and_clamps_lengths():
    B, Hkv, d, W, C, L = 3, 1, 64, 32, 8, 90
    k, v = prompts(B, Hkv, L, d, 5)
    Ks, Vs = prompts(B, Hkv, L // C, d, 6)
    cache = eva.QuantCache(B, Hkv, Hkv, d, W, C, max_tokens=70, fill=0.0)
    eva.qcache_fill(cache, k.cuda(), v.cuda(), Ks.cuda(), Vs.cuda(), torch.tensor([-5, 1000, 8], dtype=torch.int32, device="cuda"))
    assert cache.n_tok.tolist() == [0, 70, 8]
    got = arrays(cache)
    assert (got["kr"][0][0] == 0).all() and (got["ks"][0][2, :, 1:] == 0).all() and (got["kr"][0][2, :, 8:] == 0).all()
    pos = torch.arange(70 - cache.R, 70)
    same_rows((got["kr"][0][1, 0], got["kr"][1][1, 0]), pos % cache.R, k[1, 0, pos], "keys")


def test_append_and_its_summaries():
    B, Hkv, d, W, C = 2, 2, 128, 20, 5
    cache = eva.QuantCache(B, Hkv, Hkv, d, W, C, max_tokens=40, fill=math.nan)
    k, v = prompts(B, Hkv, 40, d, 7, scale=False)
    for i in range(40):
        eva.qcache_append(cache, k[:, :, i].contiguous().cuda(), v[:, :, i].contiguous().cuda())
    assert cache.n_tok.tolist() == [40, 40]
    eva.qcache_append(cache, k[:, :, 0].contiguous().cuda(), v[:, :, 0].contiguous().cuda())  # full: nothing
    assert cache.n_tok.tolist() == [40, 40] and cache.arrive.tolist() == [0, 0]
    got = arrays(cache)
    pos = torch.arange(0, 40)[-cache.R:]
    for b in range(B):
        for g in range(Hkv):
            same_rows((got["kr"][0][b, g], got["kr"][1][b, g]), pos % cache.R, k[b, g, pos], "keys")
            same_rows((got["vr"][0][b, g], got["vr"][1][b, g]), pos % cache.R, v[b, g, pos], "values")
            m = Model(k[b, g, :0], v[b, g, :0], k[b, g, :0], v[b, g, :0], W, C, SLIDING, quantised)
            for i in range(40):
                m.append(k[b, g, i], v[b, g, i])
            for name, ref in (("ks", torch.stack(m.ks)), ("vs", torch.stack(m.vs))):
                held = value(got[name][0][b, g, :8].view(torch.float8_e4m3fn), got[name][1][b, g, :8])
                # half a step, or half of the smallest (2^-10 of the row's power
                # of two, at most top / 224), and fp32 sums of C rows
                top = ref.abs().amax(-1, keepdim=True)
                bound = 2.0 ** -4 * ref.abs() + 2.0 ** -10 * top / 224 + 16 * (C + d) * 2.0 ** -24 * (1 + top)
                assert ((held - ref).abs() <= bound).all(), name


DECODE = [
    # B, H, Hkv, d, W, C, lens, window
    (1, 1, 1, 64, 1, 1, [1], SLIDING),
    (3, 4, 2, 64, 33, 7, [40, 500, 31], SLIDING),
    (2, 32, 8, 128, 512, 128, [2500, 511], SLIDING),
    (2, 20, 1, 128, 100, 33, [340, 99], ALIGNED),     # 20 heads a kv head
    (4, 8, 8, 128, 64, 16, [63, 64, 65, 191], BLOCKED),
    (3, 16, 2, 64, 96, 32, [333, 1, 96], BLOCKED),
    (70, 4, 4, 64, 40, 8, [(37 * i) % 200 + 1 for i in range(70)], SLIDING),
    (1, 4, 2, 64, 700, 4, [8700], SLIDING),           # rows split over workgroups
    (1, 8, 1, 128, 2000, 16, [9000], ALIGNED),
]


def filled(B, H, Hkv, d, W, C, lens, window, seed, room=16):
    L = max(lens)
    _, k, v = inputs.qkv(B, H, Hkv, L, d, torch.bfloat16, seed=seed)
    Ks, Vs = eva.build_summaries(k.cuda(), v.cuda(), C)
    cache = eva.QuantCache(B, H, Hkv, d, W, C, max_tokens=L + room, fill=math.nan, window=window)
    for t in (cache.k_ring_exp, cache.v_ring_exp, cache.k_sum_exp, cache.v_sum_exp):
        t.fill_(255)  # bytes that no row has
    eva.qcache_fill(cache, k.cuda(), v.cuda(), Ks, Vs, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    Ks, Vs = Ks.cpu(), Vs.cpu()
    models = [[Model(k[b, g, :n], v[b, g, :n], Ks[b, g, :n // C], Vs[b, g, :n // C], W, C, window, quantised)
               for g in range(Hkv)] for b, n in enumerate(lens)]
    return cache, models


def check_rows(o, q, models, only=None):
    B, H, d = q.shape
    G = H // len(models[0])
    o = o.cpu().double()
    for b in range(B):
        if only is not None and not only[b]:
            continue
        for g, m in enumerate(models[b]):
            ref, bound = row(q[b, g * G:(g + 1) * G], *m.keys(len(m.k) - 1), torch.bfloat16)
            over = ((o[b, g * G:(g + 1) * G] - ref).abs() - bound).max()
            assert over <= 0, f"b{b} g{g}: {float(over):.3e} over the bound"


@pytest.mark.parametrize("B,H,Hkv,d,W,C,lens,window", DECODE)
def test_decode(B, H, Hkv, d, W, C, lens, window):
    cache, models = filled(B, H, Hkv, d, W, C, lens, window, 3)
    q = inputs.normal((B, H, d), 5, torch.bfloat16)
    for ws in (True, False):
        check_rows(eva.qdecode_step(cache, q.cuda(), use_workspace=ws), q, models)
    # the fused step: append, then decode
    k, v = (inputs.normal((B, Hkv, d), s, torch.bfloat16) for s in (6, 7))
    o = eva.qappend_decode(cache, q.cuda(), k.cuda(), v.cuda())
    assert cache.n_tok.tolist() == [n + 1 for n in lens]
    for b in range(B):
        for g, m in enumerate(models[b]):
            m.append(k[b, g], v[b, g])
    check_rows(o, q, models)


def test_decode_of_inactive_empty_and_full_sequences():
    B, H, Hkv, d, W, C = 4, 4, 2, 64, 32, 8
    cache, models = filled(B, H, Hkv, d, W, C, [50, 1, 40, 50], SLIDING, 4, room=0)
    cache.n_tok[1] = 0
    q = inputs.normal((B, H, d), 5, torch.bfloat16)
    active = torch.tensor([1, 1, 0, 1], dtype=torch.int32, device="cuda")
    out = torch.full((B, H, d), 7.0, dtype=torch.bfloat16, device="cuda")
    assert eva.qdecode_step(cache, q.cuda(), active=active, out=out) is out
    assert (out[1] == 0).all() and (out[2] == 7).all()
    check_rows(out, q, models, [1, 0, 0, 1])
    k, v = (inputs.normal((B, Hkv, d), s, torch.bfloat16) for s in (6, 7))
    out = eva.qappend_decode(cache, q.cuda(), k.cuda(), v.cuda(), active=active)
    assert cache.n_tok.tolist() == [50, 1, 40, 50]  # sequences 0 and 3 are full
    check_rows(out, q, models, [1, 0, 0, 1])
    # sequence 1: its own token alone, whatever the query
    want = quantised(v[1]).repeat_interleave(H // Hkv, 0)
    assert torch.equal(out[1].cpu().double(), want.to(torch.bfloat16).double())


def test_read_back_cache_goes_on():
    # decode over the copy and over the 8-bit cache agree within bf16's roundings,
    # and the copy takes appends
    B, H, Hkv, d, W, C = 2, 8, 2, 128, 100, 16
    cache, models = filled(B, H, Hkv, d, W, C, [300, 77], SLIDING, 9)
    to = eva.qcache_read(cache, eva.RaggedCache(B, H, Hkv, d, W, C, 400, fill=math.nan, R=128))
    q = inputs.normal((B, H, d), 5, torch.bfloat16)
    check_rows(eva.rdecode_step(to, q.cuda()), q, models)
    k, v = (inputs.normal((B, Hkv, d), s, torch.bfloat16) for s in (6, 7))
    o = eva.rappend_decode(to, q.cuda(), k.cuda(), v.cuda())
    for b in range(B):
        for g, m in enumerate(models[b]):
            m.held = lambda x: x.double()
            m.append(k[b, g], v[b, g])
    check_rows(o, q, models)


def test_replayed_capture():
    B, H, Hkv, d, W, C = 2, 8, 2, 64, 64, 8
    a, _ = filled(B, H, Hkv, d, W, C, [100, 30], SLIDING, 9)
    b, _ = filled(B, H, Hkv, d, W, C, [100, 30], SLIDING, 9)
    q, k, v = (inputs.normal((B, h, d), 5, torch.bfloat16).cuda() for h in (H, Hkv, Hkv))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        eva.qappend_decode(a, q, k, v)
    torch.cuda.synchronize()
    eva.qappend_decode(b, q, k, v)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        held = eva.qappend_decode(a, q, k, v)
    for i in range(10):
        k.copy_(inputs.normal((B, Hkv, d), i, torch.bfloat16))
        graph.replay()
        o = eva.qappend_decode(b, q, k, v)
        torch.cuda.synchronize()
        assert torch.equal(held, o) and torch.equal(a.n_tok, b.n_tok), f"replay {i}"
    for name, (codes, exp) in arrays(a).items():
        other = arrays(b)[name]
        assert torch.equal(codes, other[0]) and torch.equal(exp, other[1]), name


def test_refusals():
    B, H, Hkv, d, W, C = 2, 4, 2, 64, 16, 4
    cache = eva.QuantCache(B, H, Hkv, d, W, C, 60, fill=0.0)
    q, k = torch.zeros(B, H, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, Hkv, d, dtype=torch.bfloat16, device="cuda")
    for call, error in [
        (lambda: eva.qdecode_step(cache, q.float()), ValueError),
        (lambda: eva.qdecode_step(cache, q[:1]), ValueError),
        (lambda: eva.qdecode_step(cache, q.cpu()), RuntimeError),
        (lambda: eva.qdecode_step(cache, q, active=torch.ones(B, device="cuda")), ValueError),
        (lambda: eva.qdecode_step(cache, q, out=torch.empty(B, H, d, device="cuda")), ValueError),
        (lambda: eva.qcache_append(cache, k, k.float()), ValueError),
        (lambda: eva.qappend_decode(cache, q, k, k[:, :1]), ValueError),
        (lambda: eva.qcache_read(cache, eva.RaggedCache(B, H, Hkv, d, W, C, 59)), _lib.EvaError),
        (lambda: eva.qcache_read(cache, eva.RaggedCache(B, H, Hkv, d, W + 1, C, 60)), _lib.EvaError),
        (lambda: eva.qcache_read(cache, eva.RaggedCache(B, H, Hkv, d, W, C, 60, dtype=torch.float32)), _lib.EvaError),
        (lambda: eva.qcache_read(cache, eva.RaggedCache(B, H, Hkv, d, W, C, 60, rf_lambda=0.1)), _lib.EvaError),
    ]:
        with pytest.raises(error):
            call()
    K = torch.zeros(B, Hkv, 8, d, dtype=torch.bfloat16, device="cuda")
    S = torch.zeros(B, Hkv, 2, d, dtype=torch.bfloat16, device="cuda")
    lens = torch.tensor([8, 8], dtype=torch.int32, device="cuda")
    for args, error in [((K.float(), K, S, S, lens), ValueError), ((K, K, S, S, lens.long()), ValueError),
                        ((K, K, S[:, :, :1], S, lens), ValueError), ((K, K, S, S, lens.cpu()), RuntimeError)]:
        with pytest.raises(error):
            eva.qcache_fill(cache, *args)
    assert cache.n_tok.tolist() == [0, 0]
    with pytest.raises(_lib.EvaError):  # a ring shorter than window and chunk
        eva.qcache_append(eva.QuantCache(B, H, Hkv, d, 100, C, 60, R=64), k, k)
