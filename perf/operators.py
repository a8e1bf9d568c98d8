"""Operators around the attention step, as cases that can be timed and checked.

Each case's "kind" says which operator one pass goes through:

  rope        eva.qk_norm_rope: the projection's output [B, L, (H + 2 Hkv) d] becomes
              normalised, rotated queries and keys and the values, head-major
  rope_train  the same, then eva.qk_norm_rope_backward
  fill        eva.qcache_fill: a prompt's window and summaries quantised into an 8-bit
              cache, then eva.qcache_read: the cache read back as a bf16 one
  append      eva.append_path: the accepted path of a drafted tree goes into the cache,
              chunks it completes are summarised; an 8-bit cache is then read back
  decode      eva.qdecode_step: one query a sequence over an 8-bit cache
  tree        eva.tree_attention: drafted tokens over a bf16, fp32 or 8-bit cache

`own` false computes them from elementary torch operations in 32 bits (angles in 64).
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
BASE = 10000.0


def _rope(name, kind, B, L, H, Hkv, d, rot, dtype="bf16", norm=True, interleaved=False, far=0):
    return dict(name=name, kind=kind, B=B, L=L, H=H, Hkv=Hkv, d=d, rot=rot, dtype=dtype, norm=norm,
                interleaved=interleaved, far=far)


def _cache(name, kind, B, H, Hkv, d, W, C, L, cache="e4m3", T=0, window="sliding"):
    return dict(name=name, kind=kind, B=B, H=H, Hkv=Hkv, d=d, W=W, C=C, L=L, cache=cache, T=T, window=window)


def listed():
    return [
        # one generated token for each of 64 sequences at positions of their own
        _rope("rope_token", "rope", 64, 1, 32, 8, 128, 128, far=8192),
        # a batch of 8k prompts of a grouped-query model
        _rope("rope_prompt", "rope", 4, 8192, 32, 8, 128, 128),
        # fp32, an odd length, half of a small head rotated in adjacent pairs, far positions
        _rope("rope_odd_f32", "rope", 3, 1499, 12, 4, 64, 32, dtype="f32", interleaved=True, far=100_000_000),
        # one layer's training step at 4k
        _rope("rope_train", "rope_train", 4, 4096, 32, 8, 128, 128),
        # prompts of different lengths (up to 4k) of 32 sequences go into an 8-bit cache
        _cache("fill_batch", "fill", 32, 32, 8, 128, 256, 16, 4096),
        # a batch accepts up to 8 drafted tokens a sequence into 8-bit caches
        _cache("append_quant", "append", 64, 32, 8, 128, 256, 64, 2048, T=8),
        # 8-bit decode: one user (latency), and a full batch at 8k context
        _cache("decode_single", "decode", 1, 32, 8, 128, 512, 128, 8000),
        _cache("decode_batch", "decode", 64, 32, 8, 128, 512, 128, 8192),
        # 8 drafted tokens of one user's conversation over a bf16 cache (latency)
        _cache("tree_chat", "tree", 1, 32, 8, 128, 256, 64, 777, cache="bf16", T=8),
        # 12 drafted tokens of every sequence of a batch over 8-bit caches
        _cache("tree_quant", "tree", 64, 32, 8, 128, 512, 128, 8192, T=12),
        # wide trees of 64 tokens, the largest there are
        _cache("tree_wide", "tree", 32, 32, 8, 128, 512, 128, 8192, cache="bf16", T=64),
        # fp32, three heads a kv head, odd chunks, the chunk-aligned window
        _cache("tree_odd_f32", "tree", 5, 12, 4, 64, 200, 24, 2999, cache="f32", T=13, window="chunk_aligned"),
    ]


def _cost(c):
    w = work(c)
    return w["bytes"] / 4e12 + w["flops"] / (1e14 if c.get("cache") == "f32" else 8e14)


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["rope", "rope_train", "fill", "append", "decode", "tree", "tree"])
        Hkv = rng.choice([1, 2, 4, 8, 8, 12, 16, 32])
        H = Hkv * rng.choice([1, 1, 2, 3, 4, 4, 8])
        d = rng.choice([64, 128, 128])
        if H > 64:
            continue
        if kind.startswith("rope"):
            rot = rng.choice([d, d, d // 2, 16, 48])
            c = _rope("", kind, log(1, 64), log(1, 8192), H, Hkv, d, rot, rng.choice(["bf16", "bf16", "f32"]),
                      rng.random() < 0.8, rng.random() < 0.3, rng.choice([0, log(1, 1 << 28)]))
            size = c["B"] * c["L"] * (H + 2 * Hkv) * d
        else:
            W = rng.choice([128, 256, 512, 1024, log(64, 1024)])
            C = rng.choice([16, 32, 64, 128, 256, log(8, 256)])
            cache = "e4m3" if kind in ("fill", "decode") else rng.choice(["bf16", "e4m3", "e4m3", "f32"])
            window = rng.choice(["sliding", "sliding", "chunk_aligned"])
            c = _cache("", kind, log(1, 64), H, Hkv, d, W, C, log(1, 16384), cache,
                       log(1, 64) if kind in ("append", "tree") else 0, window)
            size = c["B"] * Hkv * d * (c["L"] if kind == "fill" else W + C)
        if _cost(c) <= most and size <= 1 << 28:
            del c["name"]
            return c


# ---- sizes ----------------------------------------------------------------
def _lens(c):
    """Tokens of each sequence: spread over the upper two thirds of [1, L], the longest first."""
    B, L = c["B"], c["L"]
    return [max(1, L - (2 * L // 3) * i // max(1, B - 1) - (i * 7) % 13 * (i > 0)) for i in range(B)]


def _ring(c):
    return -(-(c["W"] + c["C"] - 1) // 64) * 64


def _tokens(c):
    return c["L"] + 128


def _first(c, p):
    """First exact position of the row at position p."""
    lo = max(0, p - c["W"] + 1)
    return lo // c["C"] * c["C"] if c["window"] == "chunk_aligned" else lo


def work(c):
    B, H, Hkv, d, L = (c[k] for k in ("B", "H", "Hkv", "d", "L"))
    if c["kind"].startswith("rope"):
        e = 4 if c["dtype"] == "f32" else 2
        n = B * L * (H + 2 * Hkv) * d
        # read x, write Q, K, V; backward: x again, their gradients, dx
        return {"bytes": n * e * (5 if c["kind"] == "rope_train" else 2), "flops": n * (30 if c["kind"] == "rope_train" else 10)}
    row = {"e4m3": 2 * d + 2, "bf16": 4 * d, "f32": 8 * d}[c["cache"]]  # a key and a value as the cache holds them
    e = 8 * d if c["cache"] == "f32" else 4 * d                          # a key and a value outside
    lens, T = _lens(c), c["T"]
    kept = sum(min(n, _ring(c)) + n // c["C"] for n in lens) * Hkv
    if c["kind"] == "fill":
        return {"bytes": kept * (e + 2 * row + 4 * d), "flops": kept * d * 8}
    if c["kind"] == "append":
        new = B * Hkv * T * (1 + 1 / c["C"])
        n = new * (e + row) + (kept * (row + 4 * d) if c["cache"] == "e4m3" else 0)
        return {"bytes": int(n), "flops": int(new * d * 8)}
    t = T or 1
    rows = sum(n - _first(c, n) + _first(c, n) // c["C"] for n in lens)
    if c["kind"] == "tree":
        b = rows * Hkv * row + B * T * (Hkv + H) * e
        return {"bytes": b, "flops": (rows + B * (T + 1) // 2) * t * H * d * 4}
    return {"bytes": rows * Hkv * row + B * H * e, "flops": rows * H * d * 4}


# ---- quantisation (the 8-bit cache's definition) ---------------------------
def _pow2(e):
    """2^e of whole numbers, exactly."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _quant(x):
    """[..., d] -> (codes in e4m3, exponents [...]): the smallest power of two that brings the row within 448."""
    x = x.float()
    m, e = torch.frexp(x.abs().amax(-1))          # amax = m 2^e, 1/2 <= m < 1 (0 for a row of zeros)
    e = torch.where(m > 0, e - 9 + (m > 0.875).to(e.dtype), torch.zeros_like(e)).clamp(-126, 119)
    return (x * _pow2(-e).unsqueeze(-1)).to(torch.float8_e4m3fn), e


def _value(q, e):
    return q.float() * _pow2(e).unsqueeze(-1)


# ---- inputs ---------------------------------------------------------------
def _inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape, dtype=torch.bfloat16, scale=1.0):
        return (torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(dtype)

    B, H, Hkv, d, L = (c[k] for k in ("B", "H", "Hkv", "d", "L"))
    if c["kind"].startswith("rope"):
        dt = DTYPES[c["dtype"]]
        x = {"x": normal(B, L, (H + 2 * Hkv) * d, dtype=dt, scale=1.7), "gq": None, "gk": None}
        if c["norm"]:
            x["gq"], x["gk"] = ((1 + 0.2 * normal(d, dtype=torch.float32)).to(dt) for _ in range(2))
        x["start"] = torch.randint(0, max(1, c["far"]), (B,), generator=g, device="cuda").int() if c["far"] else None
        x["freq"] = BASE ** (-torch.arange(c["rot"] // 2, device="cuda", dtype=torch.float64) * 2 / c["rot"])
        if c["kind"] == "rope_train":
            x["dQ"] = normal(B, H, L, d, dtype=dt)
            x["dK"], x["dV"] = normal(B, Hkv, L, d, dtype=dt), normal(B, Hkv, L, d, dtype=dt)
        return x
    dt = DTYPES.get(c["cache"], torch.bfloat16)
    lens = _lens(c)
    x = {"lens": torch.tensor(lens, dtype=torch.int32, device="cuda")}
    nc, R, T = L // c["C"], _ring(c), c["T"]
    # a chunk's summary is an average of C rows
    x["Ks"], x["Vs"] = (normal(B, Hkv, nc, d, dtype=dt, scale=c["C"] ** -0.5) for _ in range(2))
    if c["kind"] == "fill":
        x["K"], x["V"] = (normal(B, Hkv, L, d, dtype=dt) for _ in range(2))
        return x
    # the exact rows that the cache still has, by their slot (position mod R)
    x["Kr"], x["Vr"] = (normal(B, Hkv, R, d, dtype=dt) for _ in range(2))
    if c["kind"] == "decode":
        x["q"] = normal(B, H, d, dtype=dt)
        return x
    x["k"], x["v"] = (normal(B, Hkv, T, d, dtype=dt) for _ in range(2))
    if c["kind"] == "tree":
        x["q"] = normal(B, H, T, d, dtype=dt)
    # a drafter's tree: every second token or so continues its forerunner, the others any earlier one
    cg = torch.Generator().manual_seed(int(seed))
    t = torch.arange(T)
    parent = (torch.rand(B, T, generator=cg) * (t + 1)).long() - 1
    parent = torch.minimum(torch.where(torch.rand(B, T, generator=cg) < 0.5, t - 1, parent), t - 1)
    if c["kind"] == "tree":
        x["parents"] = parent.int().cuda()
        return x
    # what a verifier accepted: the tokens from the root to some node
    path, count = torch.zeros(B, T, dtype=torch.int32), torch.zeros(B, dtype=torch.int32)
    for b in range(B):
        nodes, m = [], int(torch.randint(0, T, (1,), generator=cg))
        while m >= 0:
            nodes.append(m)
            m = int(parent[b, m])
        path[b, :len(nodes)] = torch.tensor(nodes[::-1], dtype=torch.int32)
        count[b] = len(nodes)
    x["path"], x["count"] = path.cuda(), count.cuda()
    return x


def _slot_pos(c, lens):
    """Position that each slot of the ring holds, below lens: [B, R] (negative: none)."""
    j = torch.arange(_ring(c), device=lens.device)
    last = lens.long().unsqueeze(1) - 1
    return last - (last - j) % _ring(c)


def _capacity(c):
    return max(32, -(-(_tokens(c) // c["C"] + 1) // 32) * 32)


def prepare(c, seed):
    x = _inputs(c, seed)
    s = {"case": c, **x}
    if c["kind"].startswith("rope"):
        # the frequencies in turns per position times 2^64
        s["turns"] = (x["freq"] / (2 * math.pi) * 2.0 ** 64).round().long()
        return s
    B, H, Hkv, d, R, S = c["B"], c["H"], c["Hkv"], c["d"], _ring(c), _capacity(c)
    if own:
        from paper_2511_00576_amd import _lib, eva

        window = {"sliding": _lib.EVA_WINDOW_SLIDING, "chunk_aligned": _lib.EVA_WINDOW_CHUNK_ALIGNED}[c["window"]]
        a = (B, H, Hkv, d, c["W"], c["C"], _tokens(c))
        if c["cache"] == "e4m3":
            s["cache"] = eva.QuantCache(*a, R=R, fill=0.0, window=window)
        else:
            s["cache"] = eva.RaggedCache(*a, dtype=DTYPES[c["cache"]], R=R, fill=0.0, window=window)
        if c["kind"] in ("fill", "append") and c["cache"] == "e4m3":
            s["to"] = eva.RaggedCache(*a, R=R, fill=0.0, window=window)
        if c["kind"] != "fill":
            # the prompt's history, in the cache before the call
            pos = _slot_pos(c, x["lens"])
            at = pos.clamp(min=0)[:, None, :, None].expand(-1, Hkv, -1, d)
            K, V = (torch.zeros(B, Hkv, c["L"], d, dtype=t.dtype, device="cuda").scatter_add_(
                2, at, torch.where((pos >= 0)[:, None, :, None], t, 0)) for t in (x["Kr"], x["Vr"]))
            (eva.qcache_fill if c["cache"] == "e4m3" else eva.rcache_fill)(s["cache"], K, V, x["Ks"], x["Vs"], x["lens"])
            del s["Kr"], s["Vr"], s["Ks"], s["Vs"]
        return s
    if c["kind"] != "fill":
        # the same cache as a program without the framework's would keep it: rows by slot and by chunk
        pad = torch.zeros(B, Hkv, S - x["Ks"].shape[2], d, dtype=x["Ks"].dtype, device="cuda")
        rows = {"kr": x["Kr"], "vr": x["Vr"], "ks": torch.cat([x["Ks"], pad], 2), "vs": torch.cat([x["Vs"], pad], 2)}
        valid = (_slot_pos(c, x["lens"]) >= 0)[:, None, :, None]
        chunk = (torch.arange(S, device="cuda") < (x["lens"] // c["C"]).unsqueeze(1))[:, None, :, None]
        s["rows"] = {k: torch.where(valid if k.endswith("r") else chunk, t, 0) for k, t in rows.items()}
        if c["cache"] == "e4m3":
            s["rows"] = {k: _quant(t) for k, t in s["rows"].items()}
        del s["Kr"], s["Vr"], s["Ks"], s["Vs"]
    return s


# ---- the plain forms --------------------------------------------------------
def _angles(s, B, L):
    pos = torch.arange(L, device="cuda", dtype=torch.float64).unsqueeze(0)
    if s["start"] is not None:
        pos = pos + s["start"].double().unsqueeze(1)
    a = pos.unsqueeze(-1) * s["freq"]
    return torch.cos(a).float().unsqueeze(2), torch.sin(a).float().unsqueeze(2)  # [B or 1, L, 1, rot / 2]


def _pairs(y, rot, interleaved):
    return (y[..., 0:rot:2], y[..., 1:rot:2]) if interleaved else (y[..., :rot // 2], y[..., rot // 2:rot])


def _turn(y, cos, sin, rot, interleaved):
    """Rotates the pairs of the first rot features of [B, L, heads, d]."""
    a, b = _pairs(y, rot, interleaved)
    a, b = a * cos - b * sin, a * sin + b * cos
    r = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([r, y[..., rot:]], -1)


def _rope_plain(s):
    c = s["case"]
    B, L, H, Hkv, d = (c[k] for k in ("B", "L", "H", "Hkv", "d"))
    dt = s["x"].dtype
    cos, sin = _angles(s, B, L)

    def forward(x, g):
        x = x.reshape(B, L, -1, d).float()
        inv = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        y = x if g is None else x * inv * g.float()
        return x, inv, _turn(y, cos, sin, c["rot"], c["interleaved"]).to(dt).transpose(1, 2).contiguous()

    xq, xk, xv = torch.split(s["x"], [H * d, Hkv * d, Hkv * d], -1)
    fq, fk = forward(xq, s["gq"]), forward(xk, s["gk"])
    out = [fq[2], fk[2], xv.reshape(B, L, Hkv, d).transpose(1, 2).contiguous()]
    if c["kind"] == "rope":
        return out

    def backward(f, dy, g):
        x, inv, _ = f
        dn = _turn(dy.transpose(1, 2).float(), cos, -sin, c["rot"], c["interleaved"])
        if g is None:
            return dn, None
        xh = x * inv
        dg = (dn * xh).sum((0, 1, 2))
        dn = dn * g.float()
        return inv * (dn - xh * (dn * xh).mean(-1, keepdim=True)), dg

    dq, dgq = backward(fq, s["dQ"], s["gq"])
    dk, dgk = backward(fk, s["dK"], s["gk"])
    dx = torch.cat([t.reshape(B, L, -1) for t in (dq, dk, s["dV"].transpose(1, 2).float())], -1).to(dt)
    return [*out, dx, dgq, dgk]


def _tiled(v):
    """[B, Hkv, n, d] -> [B, Hkv, n / 8, d, 8]: values as the bf16 and fp32 caches hold them."""
    B, Hkv, n, d = v.shape
    return v.reshape(B, Hkv, n // 8, 8, d).transpose(-1, -2).contiguous()


def _fill_plain(s):
    c = s["case"]
    lens, Hkv, d = s["lens"].long(), c["Hkv"], c["d"]
    pos = _slot_pos(c, s["lens"])
    valid = (pos >= 0)[:, None, :, None]
    at = pos.clamp(min=0)[:, None, :, None].expand(-1, Hkv, -1, d)
    S, n = _capacity(c), s["Ks"].shape[2]
    chunk = (torch.arange(S, device="cuda") < (lens // c["C"]).unsqueeze(1))[:, None, :, None]

    def through(rows, keep):
        return torch.where(keep, _value(*_quant(rows)), 0).bfloat16()

    kr, vr = (through(s[k].gather(2, at), valid) for k in ("K", "V"))
    ks, vs = (through(torch.nn.functional.pad(s[k], (0, 0, 0, S - n)), chunk) for k in ("Ks", "Vs"))
    return [s["lens"], kr, _tiled(vr), ks, _tiled(vs)]


def _append_plain(s):
    c = s["case"]
    B, Hkv, d, C, T, R = c["B"], c["Hkv"], c["d"], c["C"], c["T"], _ring(c)
    n, count = s["lens"].long(), s["count"].long()
    quant = c["cache"] == "e4m3"
    # the accepted tokens, in their slots
    i = torch.arange(T, device="cuda")
    p = n.unsqueeze(1) + i
    new = (i < count.unsqueeze(1))[:, None, :, None]
    slot = (p % R)[:, None, :, None].expand(-1, Hkv, -1, d)
    take = s["path"].long()[:, None, :, None].expand(-1, Hkv, -1, d)

    def held(name):
        return _value(*s["rows"][name]) if quant else s["rows"][name].float()

    def stored(x):  # as the cache holds a row
        return _value(*_quant(x)) if quant else x.to(s["k"].dtype).float()

    def write(name, rows):
        old = held(name)
        return old.scatter(2, slot, torch.where(new, stored(rows.gather(2, take)), old.gather(2, slot)))

    kr, vr = write("kr", s["k"]), write("vr", s["v"])
    # the chunks that they complete
    first = n // C
    ch = first.unsqueeze(1) + torch.arange((T + C - 1) // C, device="cuda")
    done = ((ch + 1) * C <= (n + count).unsqueeze(1))[:, None, :, None]
    rows = ((ch * C).unsqueeze(-1) + torch.arange(C, device="cuda")) % R
    at = rows.reshape(B, 1, -1, 1).expand(-1, Hkv, -1, d)
    k, v = (t.gather(2, at).reshape(B, Hkv, -1, C, d) for t in (kr, vr))
    kh = k.mean(-2)
    a = torch.softmax((k * kh.unsqueeze(-2)).sum(-1) / math.sqrt(d), -1)
    vh = (a.unsqueeze(-1) * v).sum(-2)
    cat = ch[:, None, :, None].expand(-1, Hkv, -1, d)

    def put(name, x):
        old = held(name)
        return old.scatter(2, cat, torch.where(done, stored(x), old.gather(2, cat)))

    ks, vs = put("ks", kh), put("vs", vh)
    dt = s["k"].dtype
    kr, vr, ks, vs = (t.to(dt) for t in (kr, vr, ks, vs))
    return [(n + count).int(), kr, _tiled(vr), ks, _tiled(vs)]


def _attend_plain(s):
    """Queries over the cache: of the last position (decode), or of a drafted tree."""
    c = s["case"]
    B, H, Hkv, d, C = (c[k] for k in ("B", "H", "Hkv", "d", "C"))
    quant, T = c["cache"] == "e4m3", max(1, c["T"])
    n = s["lens"].long()
    kr, vr, ks, vs = (_value(*s["rows"][k]) if quant else s["rows"][k].float() for k in ("kr", "vr", "ks", "vs"))
    if c["kind"] == "tree":
        # line[b, t, u]: u is t or a forerunner of t
        par = s["parents"].long()
        eye = torch.eye(T, device="cuda")
        step = eye + torch.nn.functional.one_hot(par + 1, T + 1)[..., 1:].float()
        step = (step @ step > 0).float()
        step = (step @ step > 0).float()
        step = (step @ step > 0).float()
        step = (step @ step > 0).float()
        step = (step @ step > 0).float()
        line = step @ step > 0
        p = n.unsqueeze(1) + line.sum(-1) - 1
        kk, vv = [s["k"].float()], [s["v"].float()]
    else:
        line = torch.zeros(B, 1, 0, dtype=torch.bool, device="cuda")
        p = n.unsqueeze(1) - 1
        kk, vv = [], []
    lo = (p - c["W"] + 1).clamp(min=0)
    if c["window"] == "chunk_aligned":
        lo = lo // C * C
    pos = _slot_pos(c, s["lens"]).unsqueeze(1)
    in_window = (pos >= lo.unsqueeze(-1))
    seen = torch.arange(ks.shape[2], device="cuda") < (lo // C).unsqueeze(-1)
    ok = torch.cat([seen, in_window, line], -1)                                    # [B, T, keys]
    kk, vv = torch.cat([ks, kr, *kk], 2), torch.cat([vs, vr, *vv], 2)
    q = s["q"].reshape(B, Hkv, H // Hkv * T, d).float()
    x = (q @ kk.transpose(2, 3).contiguous() / math.sqrt(d)).reshape(B, H, T, -1)
    x[..., :ks.shape[2]] += math.log(C)
    x = x.masked_fill(~ok.unsqueeze(1), -math.inf)
    w = torch.exp(x - x.amax(-1, keepdim=True))
    w = (w / w.sum(-1, keepdim=True)).reshape(B, Hkv, H // Hkv * T, -1)
    return [(w @ vv).reshape(s["q"].shape).to(s["q"].dtype)]


# ---- one pass -------------------------------------------------------------
def run(s):
    c = s["case"]
    if not own:
        return {"rope": _rope_plain, "rope_train": _rope_plain, "fill": _fill_plain, "append": _append_plain,
                "decode": _attend_plain, "tree": _attend_plain}[c["kind"]](s)
    from paper_2511_00576_amd import eva

    if c["kind"].startswith("rope"):
        how = dict(turns=s["turns"], q_weight=s["gq"], k_weight=s["gk"], eps=EPS, start=s["start"],
                   interleaved=c["interleaved"])
        out = list(eva.qk_norm_rope(s["x"], c["H"], c["Hkv"], **how))
        if c["kind"] == "rope_train":
            out += eva.qk_norm_rope_backward(s["x"], s["dQ"], s["dK"], s["dV"], **how)
        return out
    if c["kind"] == "fill":
        eva.qcache_fill(s["cache"], s["K"], s["V"], s["Ks"], s["Vs"], s["lens"])
    elif c["kind"] == "append":
        # the tokens are rolled back before each pass (as a server rolls back
        # rejected ones), so that every pass appends at the same positions
        s["cache"].n_tok.copy_(s["lens"])
        eva.append_path(s["cache"], s["k"], s["v"], s["path"], s["count"])
    elif c["kind"] == "decode":
        return [eva.qdecode_step(s["cache"], s["q"])]
    else:
        return [eva.tree_attention(s["cache"], s["q"], s["k"], s["v"], s["parents"])]
    out = s["cache"]
    if c["cache"] == "e4m3":
        out = eva.qcache_read(s["cache"], s["to"])
    return [s["cache"].n_tok, out.k_ring, out.vt_ring, out.k_sum, out.vt_sum]


# ---- the same in 64 bits --------------------------------------------------
def _e4m3(x):
    """Nearest e4m3 value of each entry of a 64-bit tensor within 448, ties to even: steps of 2^(e-3), 2^-9 at least."""
    _, e = torch.frexp(x.abs().clamp(min=2.0 ** -6))
    step = ((e.long() - 4 + 1023) << 52).view(torch.float64)
    return torch.round(x / step) * step


def _stored64(x):
    """Rows as an 8-bit cache holds them."""
    top = x.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top / 448)
    e = torch.where(top > 0, e - (m == 0.5).to(e.dtype), torch.zeros_like(e))
    step = ((e.long() + 1023) << 52).view(torch.float64)
    return _e4m3(x / step) * step


def _rope64(c, x):
    H, Hkv, d, rot = c["H"], c["Hkv"], c["d"], c["rot"]
    pos = torch.arange(c["L"], device="cuda", dtype=torch.float64)
    res, dg = [], []
    for b in range(c["B"]):
        a = (pos + (0 if x["start"] is None else float(x["start"][b]))).unsqueeze(-1) * x["freq"]
        e = torch.polar(torch.ones_like(a), a).unsqueeze(1)  # unit complex numbers [L, 1, rot / 2]
        xb = x["x"][b].double().requires_grad_()
        gs = [None if g is None else g.double().requires_grad_() for g in (x["gq"], x["gk"])]

        def head(lo, n, g):
            y = xb[:, lo * d:(lo + n) * d].reshape(-1, n, d)
            if g is not None:
                y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / d + EPS) * g
            r = y[..., :rot]
            z = torch.complex(r[..., 0::2], r[..., 1::2]) if c["interleaved"] else torch.complex(r[..., :rot // 2], r[..., rot // 2:])
            z = z * e
            z = torch.view_as_real(z).flatten(-2) if c["interleaved"] else torch.cat([z.real, z.imag], -1)
            return torch.cat([z, y[..., rot:]], -1).transpose(0, 1)

        out = [head(0, H, gs[0]), head(H, Hkv, gs[1]), xb[:, (H + Hkv) * d:].reshape(-1, Hkv, d).transpose(0, 1)]
        if c["kind"] == "rope_train":
            torch.autograd.backward(out, [x[k][b].double() for k in ("dQ", "dK", "dV")])
            dg.append([None if g is None else g.grad for g in gs])
            out.append(xb.grad)
        res.append([t.detach() for t in out])
    res = [torch.stack(t).cpu() for t in zip(*res)]
    if c["kind"] == "rope_train":
        res += [None if t[0] is None else torch.stack(t).sum(0).cpu() for t in zip(*dg)]
    return res


def _tree64(c, x, b, n, stored):
    """Output rows [H, T, d] of sequence b: each node's own list of keys."""
    H, Hkv, d, C, R = c["H"], c["Hkv"], c["d"], c["C"], _ring(c)
    T = max(1, c["T"])
    Kr, Vr, Ks, Vs = (stored(x[k][b].double()) for k in ("Kr", "Vr", "Ks", "Vs"))
    q = x["q"][b].double().reshape(H, T, d)
    out = torch.empty_like(q)
    parents = x["parents"][b].tolist() if c["kind"] == "tree" else None
    for t in range(T):
        line, m = [], t
        while parents is not None and m >= 0:
            line.append(m)
            m = parents[m]
        p = n - 1 + len(line)
        lo = _first(c, p)
        s = lo // C
        slots = torch.arange(lo, n, device="cuda") % R
        kk, vv = [Ks[:, :s], Kr[:, slots]], [Vs[:, :s], Vr[:, slots]]
        if line:
            kk.append(x["k"][b][:, line].double())
            vv.append(x["v"][b][:, line].double())
        kk, vv = torch.cat(kk, 1), torch.cat(vv, 1)
        z = torch.matmul(kk, q[:, t].reshape(Hkv, H // Hkv, d).transpose(1, 2).contiguous()) / math.sqrt(d)
        z[:, :s] += math.log(C)
        out[:, t] = torch.matmul(torch.softmax(z, 1).transpose(1, 2).contiguous(), vv).reshape(H, d)
    return out.reshape(x["q"][b].shape)


def exact(c, seed):
    x = _inputs(c, seed)
    if c["kind"].startswith("rope"):
        return _rope64(c, x)
    lens, C, R, S = _lens(c), c["C"], _ring(c), _capacity(c)
    stored = _stored64 if c["cache"] == "e4m3" else (lambda t: t)
    if c["kind"] in ("decode", "tree"):
        return [torch.stack([_tree64(c, x, b, n, stored) for b, n in enumerate(lens)]).cpu()]
    res = []
    for b, n in enumerate(lens):
        Hkv, d = c["Hkv"], c["d"]
        kr, vr = torch.zeros(2, Hkv, R, d, dtype=torch.float64, device="cuda")
        ks, vs = torch.zeros(2, Hkv, S, d, dtype=torch.float64, device="cuda")
        ks[:, :n // C], vs[:, :n // C] = (stored(x[k][b, :, :n // C].double()) for k in ("Ks", "Vs"))
        at = torch.arange(max(0, n - R), n, device="cuda")
        if c["kind"] == "fill":
            kr[:, at % R], vr[:, at % R] = (stored(x[k][b, :, at].double()) for k in ("K", "V"))
        else:
            kr[:, at % R], vr[:, at % R] = (stored(x[k][b, :, at % R].double()) for k in ("Kr", "Vr"))
            for i in range(int(x["count"][b])):
                node, p = int(x["path"][b, i]), n + i
                kr[:, p % R], vr[:, p % R] = (stored(x[k][b, :, node].double()) for k in ("k", "v"))
                if (p + 1) % C == 0:
                    rows = torch.arange(p + 1 - C, p + 1, device="cuda") % R
                    kh = kr[:, rows].sum(1) / C
                    w = torch.softmax((kr[:, rows] * kh.unsqueeze(1)).sum(-1) / math.sqrt(d), 1)
                    ks[:, p // C], vs[:, p // C] = stored(kh), stored((w.unsqueeze(-1) * vr[:, rows]).sum(1))
        tile = [t.reshape(Hkv, -1, 8, d).permute(0, 1, 3, 2) for t in (vr, vs)]
        res.append([kr, tile[0], ks, tile[1]])
    return [None] + [torch.stack(t).cpu() for t in zip(*res)]
