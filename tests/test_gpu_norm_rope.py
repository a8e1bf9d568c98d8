"""Head norms with rotation and their backward against the formula in 64 bits.

Tolerances count roundings of half a step, u = 2^-24 in fp32 and 2^-8 for the
one of a bf16 output.  Forward: the root mean square of d terms (each lane adds
16 squares, then log2(d / 16) additions; all terms positive) is off by at most
(16 + 3) u relative, its reciprocal root by half of that and 2 u, two products
2 u; the angle in half turns is rounded once (2^-25, so 2 pi u / 4 radians)
and each of sine and cosine is off by 4 u at most; the turn adds 2 u: 24 u of
|a| + |b| covers it, the pair before its turn.  Backward: the turn back the
same, then products and a mean of d terms of either sign: 64 u of the terms'
magnitudes.
"""
import math

import pytest
import torch

from paper_2511_00576_amd import eva

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    eva._lib.load()


def half_step(t):
    return torch.finfo(t.dtype).eps / 2


def split(t, H, Hkv):
    """[B, L, (H + 2 Hkv) d] -> three of [B, heads, L, d]."""
    B, L, n = t.shape
    d = n // (H + 2 * Hkv)
    return [p.reshape(B, L, -1, d).transpose(1, 2) for p in torch.split(t, [H * d, Hkv * d, Hkv * d], -1)]


class Reference:
    """The formula on 64-bit CPU tensors.  freq in radians per position, pos [B, L]."""

    def __init__(self, freq, pos, eps, interleaved, d):
        self.eps, self.d = eps, d
        r = 2 * len(freq)
        ang = pos.double().unsqueeze(-1) * freq
        self.cos, self.sin = torch.cos(ang).unsqueeze(1), torch.sin(ang).unsqueeze(1)
        i = torch.arange(r // 2)
        self.a, self.b = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)

    def turn(self, y, sign=1):
        out = y.clone()
        a, b = y[..., self.a], y[..., self.b]
        out[..., self.a] = a * self.cos - sign * b * self.sin
        out[..., self.b] = sign * a * self.sin + b * self.cos
        return out

    def pair(self, y):
        """|a| + |b| of each feature's pair (its own magnitude where it is not turned)."""
        m = y.abs().clone()
        s = m[..., self.a] + m[..., self.b]
        m[..., self.a] = s
        m[..., self.b] = s
        return m

    def rstd(self, x):
        return torch.rsqrt(x.square().mean(-1, keepdim=True) + self.eps)

    def forward(self, x, g):
        n = x if g is None else x * self.rstd(x) * g
        return self.turn(n), self.pair(n)

    def backward(self, x, g, dy):
        dn, mag = self.turn(dy, -1), self.pair(dy)
        if g is None:
            return dn, mag, None, None
        r = self.rstd(x)
        xh = x * r
        t = dn * g
        dx = r * (t - xh * (t * xh).mean(-1, keepdim=True))
        m = mag * g.abs()
        return (dx, r * (m + xh.abs() * (m * xh.abs()).mean(-1, keepdim=True)), (dn * xh).sum((0, 1, 2)),
                (mag * xh.abs()).sum((0, 1, 2)))


def make(B, L, H, Hkv, d, rot, dtype, seed, norm=(True, True), far=0, tree=False, inv_freq=None):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(B, L, (H + 2 * Hkv) * d, generator=g) * 1.5).to(dtype)
    w = [(1 + 0.3 * torch.randn(d, generator=g)).to(dtype) if n else None for n in norm]
    start = torch.randint(0, far, (B,), generator=g).int() if far else None
    offsets = torch.randint(0, 7, (B, L), generator=g).int() if tree else None
    pos = torch.arange(L).expand(B, L) if offsets is None else offsets
    if start is not None:
        pos = pos + start.unsqueeze(1)
    freq = torch.tensor([10000.0 ** (-2 * i / rot) for i in range(rot // 2)] if inv_freq is None else inv_freq,
                        dtype=torch.float64)
    grads = [torch.randn(B, n, L, d, generator=g).to(dtype) for n in (H, Hkv, Hkv)]
    return x, w, start, offsets, pos, freq, grads


def cuda(t):
    return None if t is None else t.cuda()


def within(got, ref, bound, what):
    got = got.cpu().double()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = (got - ref).abs() - bound
    assert over.max() <= 0, f"{what}: {float(over.max()):.3e} over the bound"


CASES = [
    # B, L, H, Hkv, d, rot, dtype, interleaved, norms, far, tree
    (1, 1, 1, 1, 64, 64, torch.bfloat16, False, (True, True), 0, False),
    (1, 1, 32, 8, 128, 128, torch.bfloat16, False, (True, True), 5000, False),
    (64, 1, 32, 8, 128, 128, torch.bfloat16, True, (True, True), 8192, False),
    (3, 129, 12, 4, 64, 32, torch.float32, True, (True, True), 100_000_000, False),
    (2, 257, 7, 7, 128, 16, torch.float32, False, (True, False), 2 ** 30, False),
    (2, 65, 10, 1, 128, 48, torch.bfloat16, False, (False, True), 77, False),
    (1, 1000, 24, 3, 64, 48, torch.bfloat16, True, (True, True), 0, False),
    (5, 13, 16, 2, 128, 128, torch.bfloat16, False, (True, True), 4096, True),
    (2, 31, 5, 5, 64, 0, torch.float32, False, (True, True), 0, False),
    (2, 31, 4, 2, 64, 64, torch.bfloat16, False, (False, False), 9, False),
    (1, 4099, 17, 17, 128, 128, torch.float32, False, (True, True), 3, False),
    # few heads: several tokens a wave, the last wave's part of the lanes idle
    (3, 171, 1, 1, 128, 128, torch.bfloat16, True, (True, True), 50, True),
    (5, 41, 2, 1, 64, 48, torch.float32, False, (True, True), 2 ** 20, False),
    (2, 1, 3, 3, 64, 64, torch.bfloat16, False, (True, False), 0, False),
    (7, 3000, 1, 1, 64, 32, torch.bfloat16, False, (True, True), 0, False),
    (1, 17, 3, 1, 128, 16, torch.float32, True, (False, True), 9, False),
    (2, 333, 8, 8, 64, 64, torch.bfloat16, True, (True, True), 0, False),
]


@pytest.mark.parametrize("B,L,H,Hkv,d,rot,dtype,inter,norm,far,tree", CASES)
def test_forward_and_backward(B, L, H, Hkv, d, rot, dtype, inter, norm, far, tree):
    x, w, start, offsets, pos, freq, grads = make(B, L, H, Hkv, d, rot, dtype, 11 * L + H, norm, far, tree)
    ref = Reference(freq, pos, 1e-6, inter, d)
    how = dict(turns=eva.rope_turns(rot) if rot else None, q_weight=cuda(w[0]), k_weight=cuda(w[1]), eps=1e-6,
               start=cuda(start), offsets=cuda(offsets), interleaved=inter)
    out = eva.qk_norm_rope(x.cuda(), H, Hkv, **how)
    got = eva.qk_norm_rope_backward(x.cuda(), *(t.cuda() for t in grads), **how)
    again = eva.qk_norm_rope_backward(x.cuda(), *(t.cuda() for t in grads), **how)
    assert all(a is b or torch.equal(a, b) for a, b in zip(got, again)), "the backward's bits vary"
    rows = split(x.double(), H, Hkv)
    dx = split(got[0], H, Hkv)
    round_ = 0 if dtype == torch.float32 else half_step(x)
    for i, name in enumerate("QK"):
        g = None if w[i] is None else w[i].double()
        y, mag = ref.forward(rows[i], g)
        within(out[i], y, round_ * y.abs() + 24 * U * mag, name)
        d64, dmag, dg, dgmag = ref.backward(rows[i], g, grads[i].double())
        within(dx[i], d64, round_ * d64.abs() + 64 * U * dmag, "d" + name)
        if g is None:
            assert got[1 + i] is None
        else:
            # a lane adds its tokens' sweeps one by one, then waves and
            # workgroups: under 1024 additions in a row
            within(got[1 + i], dg, (64 + 1024) * U * dgmag, f"weight {name}")
    assert torch.equal(out[2].cpu(), split(x, H, Hkv)[2]), "V"
    assert torch.equal(dx[2].cpu(), grads[2]), "dV"


def test_far_positions_are_exact():
    # at 2^30 and a frequency of one radian the angle in fp32 would be off by
    # tens of radians; negative starts are turns back
    for p in (2 ** 30, -5, 2 ** 31 - 1):
        x, _, _, _, _, freq, _ = make(1, 4, 2, 1, 64, 64, torch.float32, 5)
        start = torch.tensor([p], dtype=torch.int32)
        offsets = torch.tensor([[0, 1, 2 ** 30, 7]], dtype=torch.int32)
        pos = start.long().unsqueeze(1) + offsets.long()  # past 32 bits: added in 64
        ref = Reference(freq, pos, 0.0, False, 64)
        out = eva.qk_norm_rope(x.cuda(), 2, 1, turns=eva.rope_turns(64), start=start.cuda(), offsets=offsets.cuda())
        y, mag = ref.forward(split(x.double(), 2, 1)[0], None)
        # the reference's own angle, a product in 64 bits, is off by 2^-53 of it
        # and turns' frequency (53 bits) by as much
        within(out[0], y, (24 * U + 2 * 2.0 ** -53 * pos.abs().max()) * mag, f"position {p}")


def test_turns_from_given_frequencies():
    f = [0.5, 0.25, 3.0, 1e-9, 0.0, 0.1, 0.2, 0.3]
    x, w, _, _, pos, freq, _ = make(2, 50, 3, 1, 64, 16, torch.float32, 8, inv_freq=f)
    out = eva.qk_norm_rope(x.cuda(), 3, 1, turns=eva.rope_turns(16, inv_freq=f), q_weight=w[0].cuda())
    y, mag = Reference(freq, pos, 1e-6, False, 64).forward(split(x.double(), 3, 1)[0], w[0].double())
    within(out[0], y, 24 * U * mag, "Q")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strided_rows(dtype):
    # the projection's output inside a wider buffer, batches and tokens strided,
    # and one row for all sequences (stride 0)
    B, L, H, Hkv, d = 3, 17, 4, 2, 64
    n = (H + 2 * Hkv) * d
    wide = torch.randn(B, L + 2, n + 32, device="cuda").to(dtype)
    view = wide[:, 1:L + 1, 16:16 + n]
    t = eva.rope_turns(64)
    for v in (view, view[:1].expand(B, L, n), view.transpose(0, 1)[:L].transpose(0, 1)):
        a = eva.qk_norm_rope(v, H, Hkv, turns=t)
        b = eva.qk_norm_rope(v.contiguous(), H, Hkv, turns=t)
        assert all(torch.equal(p, q) for p, q in zip(a, b))
        g = [torch.randn_like(p) for p in a]
        w = torch.ones(d, dtype=dtype, device="cuda")
        a = eva.qk_norm_rope_backward(v, *g, turns=t, q_weight=w, k_weight=w)
        b = eva.qk_norm_rope_backward(v.contiguous(), *g, turns=t, q_weight=w, k_weight=w)
        assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_rows_of_zeros_and_not_finite_stay_in_their_rows():
    B, L, H, Hkv, d = 1, 6, 2, 1, 64
    x = torch.randn(B, L, (H + 2 * Hkv) * d)
    x[0, 1] = 0
    x[0, 2, 5] = math.nan
    x[0, 3, d + 1] = math.inf
    w = torch.ones(d).cuda()
    t = eva.rope_turns(d)
    q, k, v = eva.qk_norm_rope(x.cuda(), H, Hkv, turns=t, q_weight=w, k_weight=w)
    assert (q[0, :, 1] == 0).all() and (k[0, :, 1] == 0).all()
    bad = ~torch.isfinite(q[0]).all(-1).cpu()
    assert bad.tolist() == [[False, False, True, False, False, False], [False, False, False, True, False, False]]
    assert torch.isfinite(k).all() and torch.isfinite(v).all()


def test_gradient_against_differences():
    B, L, H, Hkv, d = 2, 9, 3, 1, 64
    x, w, start, _, pos, freq, grads = make(B, L, H, Hkv, d, 64, torch.float32, 3, far=1000)
    ref = Reference(freq, pos, 1e-6, True, d)
    x64, w64 = x.double(), [t.double() for t in w]

    def loss(xx, ww):
        r = split(xx, H, Hkv)
        out = [ref.forward(r[0], ww[0])[0], ref.forward(r[1], ww[1])[0], r[2]]
        return sum((o * g.double()).sum() for o, g in zip(out, grads))

    got = eva.qk_norm_rope_backward(x.cuda(), *(t.cuda() for t in grads), turns=eva.rope_turns(64),
                                    q_weight=w[0].cuda(), k_weight=w[1].cuda(), start=start.cuda(), interleaved=True)
    gen = torch.Generator().manual_seed(1)
    h = 1e-5
    for _ in range(4):
        v = torch.randn(x.shape, generator=gen).double()
        u = [torch.randn(d, generator=gen).double() for _ in range(2)]
        diff = (loss(x64 + h * v, [a + h * b for a, b in zip(w64, u)]) -
                loss(x64 - h * v, [a - h * b for a, b in zip(w64, u)])) / (2 * h)
        dot = (got[0].cpu().double() * v).sum() + sum((g.cpu().double() * b).sum() for g, b in zip(got[1:], u))
        # h^2 times third derivatives, and 64 u of some 4000 terms of order one:
        # far below 1e-3 of a sum of order 60
        assert abs(float(diff - dot)) <= 1e-3 * (1 + abs(float(diff)))


def test_no_tokens():
    x = torch.empty(2, 0, 4 * 64, device="cuda")
    q, k, v = eva.qk_norm_rope(x, 2, 1)
    assert q.shape == (2, 2, 0, 64) and k.shape == v.shape == (2, 1, 0, 64)
    w = torch.ones(64, device="cuda")
    dx, dq, dk = eva.qk_norm_rope_backward(x, q, k, v, q_weight=w)
    assert dx.shape == x.shape and (dq == 0).all() and dk is None


def test_another_stream_and_replayed_capture():
    B, L, H, Hkv, d = 2, 40, 8, 2, 128
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    t = eva.rope_turns(d)
    x = torch.randn(B, L, (H + 2 * Hkv) * d, device="cuda").bfloat16()

    def step():
        out = eva.qk_norm_rope(x, H, Hkv, turns=t, q_weight=w, k_weight=w)
        return [*out, *eva.qk_norm_rope_backward(x, *out, turns=t, q_weight=w, k_weight=w)]

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        held = step()
    for i in range(4):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(i)).bfloat16())
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, step())), f"replay {i}"


def test_refusals():
    x = torch.randn(2, 5, 4 * 64, device="cuda")
    t = eva.rope_turns(64)
    w = torch.ones(64, device="cuda")
    with pytest.raises(RuntimeError):
        eva.qk_norm_rope(x.cpu(), 2, 1)
    with pytest.raises(ValueError):
        eva.qk_norm_rope(x, 3, 1)
    with pytest.raises(TypeError):
        eva.qk_norm_rope(x.half(), 2, 1)
    with pytest.raises(ValueError):
        eva.qk_norm_rope(x, 2, 1, q_weight=w.bfloat16())
    with pytest.raises(ValueError):
        eva.qk_norm_rope(x, 2, 1, turns=t.int())
    with pytest.raises(RuntimeError):
        eva.qk_norm_rope(x, 2, 1, turns=t.cpu())
    with pytest.raises(ValueError):
        eva.qk_norm_rope(x, 2, 1, start=torch.zeros(3, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        eva.qk_norm_rope(x.transpose(1, 2).contiguous().transpose(1, 2), 2, 1)
    with pytest.raises(eva._lib.EvaError):
        eva.qk_norm_rope(x, 2, 1, turns=t[:20].clone())  # 40 turned features: not a multiple of 16
    with pytest.raises(eva._lib.EvaError):
        eva.qk_norm_rope(x, 2, 1, q_weight=w, eps=-1.0)
    with pytest.raises(eva._lib.EvaError):
        eva.qk_norm_rope(torch.randn(2, 5, 4 * 64 + 1, device="cuda")[..., 1:], 2, 1)  # rows off 16 bytes
    with pytest.raises(eva._lib.EvaError):
        eva.qk_norm_rope(torch.randn(2, 5, 4 * 32, device="cuda"), 2, 1)  # d = 32
    q, k, v = eva.qk_norm_rope(x, 2, 1)
    with pytest.raises(ValueError):
        eva.qk_norm_rope_backward(x, q, k, v[:, :, :4])
    with pytest.raises(ValueError):
        eva.qk_norm_rope(x, 2, 1, out=(q[:1], k, v))
