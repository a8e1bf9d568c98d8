"""Operators of a paged cache, as cases that can be timed and checked.

The layers of a hybrid model that keep full softmax attention hold every key and value of
every sequence, in pages of P tokens that a table, shared by the layers, gives to sequences.
Each case's "kind" says which operator one pass goes through:

  plan    eva.page_truncate and eva.page_extend: rejected tokens are taken back, pages and
          slots for new tokens handed out
  append  eva.paged_append: new tokens' rows go to their slots, pages that they complete
          get their mean key
  decode  eva.paged_decode: one query a sequence over all its tokens
  sparse  eva.paged_select, then eva.paged_decode over the pages that each kv head's
          queries choose by the pages' mean keys
  step    all of them, as one layer of a generation step goes through them

`own` false computes them from elementary torch operations in 32 bits (pages' scores in 64:
what is chosen must not depend on the order of a sum).
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(name, kind, B, L, P, H=32, Hkv=8, d=128, T=0, S=0, lens="spread", dtype="bf16", short=False):
    """B sequences of up to L tokens (lens: how they spread), pages of P tokens, T new tokens at
    most, S pages chosen; short: the free pages do not suffice for all new tokens."""
    return dict(name=name, kind=kind, B=B, L=L, P=P, H=H, Hkv=Hkv, d=d, T=T, S=S, lens=lens, dtype=dtype, short=short)


def listed():
    return [
        # one token for each of 64 running requests (latency)
        _case("plan_step", "plan", 64, 8192, 64, T=1),
        # 256 places of a server, a third of them new requests with prompts of up to 4k
        _case("plan_prompts", "plan", 256, 4096, 64, T=4096, lens="new"),
        # one generated token of 64 sequences goes into its pages (latency)
        _case("append_token", "append", 64, 8192, 64, T=1),
        # prompts of up to 4k tokens go into pages
        _case("append_prompts", "append", 8, 4096, 64, T=4096, lens="new"),
        # one user's conversation (latency)
        _case("decode_single", "decode", 1, 8000, 64),
        # a full batch at 8k context
        _case("decode_batch", "decode", 64, 8192, 64),
        # one document of 128k tokens beside fifteen short chats
        _case("decode_ragged", "decode", 16, 131072, 32, lens="one_long"),
        # fp32, three heads a kv head, small pages, odd lengths
        _case("decode_odd_f32", "decode", 5, 2999, 16, H=12, Hkv=4, d=64, dtype="f32"),
        # one user's 128k context, of which 64 pages are attended
        _case("sparse_single", "sparse", 1, 131072, 64, S=64),
        # a batch at 32k context
        _case("sparse_batch", "sparse", 32, 32768, 64, S=48),
        # fp32, small pages, few of them
        _case("sparse_odd_f32", "sparse", 3, 2999, 16, H=12, Hkv=4, d=64, S=21, dtype="f32"),
        # one layer's step of generation: rollback, slots, append, choice, attention
        _case("layer_step", "step", 32, 8192, 64, T=1, S=32),
    ]


def _cost(c):
    w = work(c)
    return w["bytes"] / 4e12 + w["flops"] / (1e14 if c["dtype"] == "f32" else 8e14)


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["plan", "append", "decode", "decode", "sparse", "sparse", "step"])
        Hkv = rng.choice([1, 2, 4, 8, 8, 12, 16, 32])
        H = Hkv * rng.choice([1, 1, 2, 3, 4, 4, 8, 16, 20])
        if H > 64:
            continue
        c = _case("", kind, log(1, 512 if kind == "plan" else 64), log(1, 131072), rng.choice([16, 32, 64, 64, 128, 256]), H, Hkv,
                  rng.choice([64, 128, 128]), 0, 0, rng.choice(["spread", "spread", "even", "one_long"]),
                  rng.choice(["bf16", "bf16", "bf16", "f32"]))
        if kind in ("plan", "append"):
            c["T"] = rng.choice([1, log(1, 16), log(1, c["L"])])
            c["lens"] = rng.choice(["spread", "new", "one_long"])
            c["short"] = kind == "plan" and rng.random() < 0.3
        if kind == "step":
            c["T"] = 1
        if kind in ("sparse", "step"):
            c["S"] = log(4, 256)
        # the plain form pads every sequence to the longest
        pad = c["B"] * c["L"] * (1 if kind == "plan" else Hkv * c["d"])
        if _cost(c) <= most and pad <= 1 << (28 if kind == "plan" else 31) and _pool(c) * c["P"] * Hkv * c["d"] <= 1 << (40 if kind == "plan" else 30):
            del c["name"]
            return c


# ---- sizes ----------------------------------------------------------------
def _lens(c):
    """Tokens of each sequence before the call."""
    B, L = c["B"], c["L"]
    if c["lens"] == "even":
        return [L] * B
    if c["lens"] == "one_long":
        return [L if i == B // 3 else max(1, L // 100 + (i * 37) % 101) if L > 200 else max(1, L // 2) for i in range(B)]
    n = [max(1, L - (2 * L // 3) * i // max(1, B - 1) - (i * 7) % 13 * (i > 0)) for i in range(B)]
    # every third place holds a new request, which has no tokens yet
    return [0 if c["lens"] == "new" and i % 3 == 0 else v for i, v in enumerate(n)]


def _counts(c):
    """Tokens that each sequence asks for."""
    B, T = c["B"], c["T"]
    if c["kind"] == "step":
        return [1] * B
    if T == 1:
        return [0 if i % 8 == 5 else 1 for i in range(B)]
    if c["lens"] == "new":  # prompts for the new ones, a token for the others
        return [max(1, T - T // 2 * i // max(1, B - 1) - (i * 5) % 7) if i % 3 == 0 else 1 for i in range(B)]
    return [(T - i * 11) % (T + 1) for i in range(B)]


def _extra(c):
    """Drafted tokens that were rejected since, still in the table."""
    return [(i * 5 + 3) % 9 if c["kind"] in ("plan", "step") and n else 0 for i, n in enumerate(_lens(c))]


def _pages(n, P):
    return -(-n // P)


def _row_pages(c):
    """Pages that a row of the table has room for."""
    return _pages(c["L"] + max(c["T"], 1) + 16, c["P"])


def _pool(c):
    """Pages of the pool."""
    P = c["P"]
    held = sum(_pages(n + x, P) for n, x in zip(_lens(c), _extra(c)))
    new = sum(_pages(n + t, P) - _pages(n, P) for n, t in zip(_lens(c), _counts(c))) if c["T"] else 0
    return held + (new * 3 // 4 if c["short"] else new) + c["B"] // 8 + 1


def _kept(c, n):
    """Tokens that the query of a sequence of n tokens attends."""
    P, S = c["P"], c["S"]
    held = _pages(n, P)
    return n if not S or held <= S else (S - 1) * P + n - (held - 1) * P


def work(c):
    B, H, Hkv, d, P, T = (c[k] for k in ("B", "H", "Hkv", "d", "P", "T"))
    e = 4 if c["dtype"] == "f32" else 2
    lens, counts = _lens(c), _counts(c) if T else [0] * B
    w = {"bytes": 0, "flops": 0}
    if c["kind"] in ("plan", "step"):
        new = sum(_pages(n + t, P) - _pages(n, P) for n, t in zip(lens, counts))
        w["bytes"] += 4 * (B * T + 6 * B + 2 * new)
        w["flops"] += 4 * B * T
    if c["kind"] in ("append", "step"):
        done = sum((n + t) // P - n // P for n, t in zip(lens, counts))
        w["bytes"] += sum(counts) * Hkv * d * 4 * e + 4 * B * T + done * Hkv * d * 4
        w["flops"] += done * P * Hkv * d
    if c["kind"] in ("decode", "sparse", "step"):
        lens = [n + t for n, t in zip(lens, counts)] if c["kind"] == "step" else lens
        kept = sum(_kept(c, n) for n in lens)
        w["bytes"] += kept * Hkv * d * 2 * e + 2 * B * H * d * e
        w["flops"] += kept * H * d * 4
        if c["S"]:
            scored = sum(_pages(n, P) for n in lens if _pages(n, P) > c["S"])
            w["bytes"] += scored * Hkv * d * 4
            w["flops"] += scored * H * d * 2
    return w


# ---- inputs ---------------------------------------------------------------
def _inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    B, H, Hkv, d, P, T, N, M = (*(c[k] for k in ("B", "H", "Hkv", "d", "P", "T")), _pool(c), _row_pages(c))
    dt = DTYPES[c["dtype"]]

    def normal(*shape, scale=1.0, dtype=dt):
        return (torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(dtype)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    lens, extra = _lens(c), _extra(c)
    x = {"lens": ints(lens)}
    # pages lie in any order, as after hours of requests coming and going
    order = torch.randperm(N, generator=g, device="cuda").int()
    held = ints([_pages(n + r, P) for n, r in zip(lens, extra)]).long()
    j = torch.arange(M, device="cuda")
    has = j < held.unsqueeze(1)
    rank = (held.cumsum(0) - held).unsqueeze(1) + j
    x["table"] = torch.where(has, order[rank.clamp(max=N - 1)], -1).int()
    total = sum(_pages(n + r, P) for n, r in zip(lens, extra))
    x["n_tok"] = ints([n + r for n, r in zip(lens, extra)])
    x["free"] = torch.cat([order[total:], order[:total]]).contiguous()
    x["n_free"] = ints([N - total])
    if T:
        x["counts"] = ints(_counts(c))
    if c["kind"] == "plan":
        # what varies with the seed besides the pages: which sequences ask
        cut = torch.rand(B, generator=g, device="cuda")
        x["counts"] = torch.where(cut < 0.1, x["counts"] // 2, x["counts"]).int()
        return x
    # keys of a page have a part in common, which its mean shows
    x["k"] = (normal(N, Hkv, P, d, dtype=torch.float32) + normal(N, Hkv, 1, d, scale=0.5, dtype=torch.float32)).to(dt)
    x["vt"] = normal(N, Hkv, P // 8, d, 8)  # values: slot s, feature f of a page at [s / 8][f][s % 8]
    x["mean"] = x["k"].float().mean(2)
    if T:
        x["k_new"], x["v_new"] = normal(B, Hkv, T, d), normal(B, Hkv, T, d)
    if c["kind"] == "append":
        # the table as it stands once the new tokens have their pages
        need = _pages(x["lens"].long() + x["counts"].long(), P)
        rank = total + (need - held).cumsum(0).unsqueeze(1) - (need - held).unsqueeze(1) + j - held.unsqueeze(1)
        x["table"] = torch.where((j >= held.unsqueeze(1)) & (j < need.unsqueeze(1)), order[rank.clamp(0, N - 1)], x["table"]).int()
        x["slots"] = _slots(x["table"], x["lens"], x["counts"], T, P)
    else:
        x["q"] = normal(B, H, d)
    return x


def _slots(table, start, counts, T, P):
    """Slot of each new token: page times P plus its place in the page, -1 where there is none."""
    t = torch.arange(T, device=table.device)
    pos = start.long().unsqueeze(1) + t
    page = table.long().gather(1, (pos // P).clamp(max=table.shape[1] - 1))
    return torch.where(t < counts.long().unsqueeze(1), page * P + pos % P, -1).int()


def prepare(c, seed):
    s = {"case": c, **_inputs(c, seed)}
    if own:
        # the handles that a program keeps, over the same memory
        from paper_2511_00576_amd import eva

        s["pages"] = eva.PageTable(c["B"], c["P"], _pool(c), _row_pages(c) * c["P"],
                                   storage=(s["n_tok"], s["table"], s["free"], s["n_free"]))
        if c["kind"] != "plan":
            s["cache"] = eva.PagedCache(s["pages"], c["H"], c["Hkv"], c["d"], dtype=DTYPES[c["dtype"]],
                                        storage=(s["k"], s["vt"], s["mean"]))
    return s


# ---- the plain forms --------------------------------------------------------
def _held(n, P):
    return (n + P - 1) // P


def _truncate_plain(s):
    """Sequences keep at most lens tokens; the pages that they leave go back on the stack of free ones."""
    P, M, N = s["case"]["P"], s["table"].shape[1], s["free"].numel()
    n, lens = s["n_tok"].long(), s["lens"].long()
    keep = torch.minimum(n, lens.clamp(min=0))
    j = torch.arange(M, device="cuda")
    drop = (j >= _held(keep, P).unsqueeze(1)) & (j < _held(n, P).unsqueeze(1))
    rank = drop.flatten().cumsum(0)
    dropped = rank[-1]
    at = torch.where(drop.flatten(), s["n_free"].long() + dropped - rank, N)
    free = torch.cat([s["free"], s["free"][:1]]).scatter_(0, at, s["table"].flatten())
    s["free"].copy_(free[:N])
    s["table"].copy_(torch.where(drop, -1, s["table"]))
    s["n_free"].add_(dropped.int())
    s["n_tok"].copy_(keep)


def _extend_plain(s):
    """Pages and slots for new tokens: (slots, start, granted)."""
    P, T, M, N = s["case"]["P"], s["case"]["T"], s["table"].shape[1], s["free"].numel()
    n, count = s["n_tok"].long(), s["counts"].long().clamp(0, T)
    count = torch.where(n + count > M * P, 0, count)
    held = _held(n, P)
    need = _held(n + count, P) - held
    upto = need.cumsum(0)
    granted = torch.where((need == 0) | (upto <= s["n_free"]), count, 0)
    need = _held(n + granted, P) - held
    j = torch.arange(M, device="cuda")
    new = (j >= held.unsqueeze(1)) & (j < (held + need).unsqueeze(1))
    at = s["n_free"].long() - 1 - ((need.cumsum(0) - need - held).unsqueeze(1) + j)
    s["table"].copy_(torch.where(new, s["free"][at.clamp(0, N - 1)], s["table"]))
    s["n_free"].sub_(need.sum().int())
    s["n_tok"].copy_(n + granted)
    return _slots(s["table"], n, granted, T, P), n.int(), granted.int()


def _append_plain(s, slots):
    c = s["case"]
    P, N = c["P"], s["k"].shape[0]
    B, Hkv, T, d = s["k_new"].shape
    # rows without a slot are written over the first one that has one
    at = slots.flatten().long()
    first = torch.argmax((at >= 0).int())
    at = torch.where(at >= 0, at, at[first])
    src = torch.where(slots.flatten() >= 0, torch.arange(B * T, device="cuda"), first)
    k, v = (s[n].transpose(1, 2).reshape(B * T, Hkv, d)[src] for n in ("k_new", "v_new"))
    page, off = at // P, at % P
    s["k"][page, :, off] = k
    s["vt"][page, :, off // 8, :, off % 8] = v
    # pages that the tokens complete: of P neighbours, which lie at successive places, one at most does
    full = (slots >= 0) & (slots % P == P - 1)
    page = torch.nn.functional.pad(torch.where(full, slots // P, -1), (0, -T % P), value=-1).reshape(-1, P).amax(-1).long()
    some = page.clamp(min=0)
    mean = s["k"][some].float().mean(2)
    out = torch.cat([s["mean"], s["mean"][:1]])
    out[torch.where(page >= 0, page, N)] = mean
    s["mean"].copy_(out[:N])


def _choose_plain(s):
    """Pages that the queries of each kv head choose: [B, Hkv, S], -1 where there are fewer."""
    c = s["case"]
    B, H, Hkv, d, P, S = (c[k] for k in ("B", "H", "Hkv", "d", "P", "S"))
    M = s["table"].shape[1]
    held = _held(s["n_tok"].long(), P).reshape(B, 1, 1)
    mean = s["mean"][s["table"].long().clamp(min=0)].double().transpose(1, 2).contiguous()  # [B, Hkv, M, d]
    q = s["q"].double().reshape(B, Hkv, H // Hkv, d).transpose(2, 3).contiguous()
    score = (mean @ q).amax(-1)
    j = torch.arange(M, device="cuda")
    score = torch.where((j == 0) | (j == held - 1), math.inf, torch.where(j < held, score, -math.inf))
    at = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :S]
    at = torch.where(at < held, at, M).sort(-1).values
    at = torch.nn.functional.pad(at, (0, max(0, S - M)), value=M)
    return torch.where(at < M, at, -1).int()


def _attend_plain(s, pages=None):
    c = s["case"]
    B, H, Hkv, d, P = (c[k] for k in ("B", "H", "Hkv", "d", "P"))
    M = s["table"].shape[1]
    n = s["n_tok"].long().reshape(B, 1, 1)
    if pages is None:
        j = torch.arange(M, device="cuda").expand(B, 1, M)
    else:
        j = pages.long()
    page = s["table"].long().unsqueeze(1).expand(B, j.shape[1], M).gather(2, j.clamp(min=0)).clamp(min=0)
    head = torch.arange(Hkv, device="cuda").reshape(1, Hkv, 1)
    k = s["k"][page, head].float().reshape(B, Hkv, -1, d)
    v = s["vt"][page, head].transpose(-1, -2).float().reshape(B, Hkv, -1, d)
    pos = (j.unsqueeze(-1) * P + torch.arange(P, device="cuda")).flatten(2)
    seen = (pos >= 0) & (pos < n)
    q = s["q"].float().reshape(B, Hkv, H // Hkv, d)
    x = (k @ q.transpose(2, 3).contiguous()).transpose(2, 3) / math.sqrt(d)
    x = x.masked_fill(~seen.unsqueeze(2), -math.inf)
    w = torch.exp(x - x.amax(-1, keepdim=True))
    w = (w / w.sum(-1, keepdim=True)).contiguous()
    return (w @ v).reshape(B, H, d).to(s["q"].dtype)


# ---- one pass -------------------------------------------------------------
def run(s):
    c = s["case"]
    kind = c["kind"]
    if own:
        from paper_2511_00576_amd import eva

        if kind in ("plan", "step"):
            # tokens are rolled back before each pass (as a server rolls back rejected
            # ones), so that every pass hands out the same places
            eva.page_truncate(s["pages"], s["lens"])
            slots, start, granted = eva.page_extend(s["pages"], c["T"], s["counts"])
        if kind in ("append", "step"):
            eva.paged_append(s["cache"], s["k_new"], s["v_new"], slots if kind == "step" else s["slots"])
        if kind in ("sparse", "step"):
            pages = eva.paged_select(s["cache"], s["q"], c["S"])
            o = eva.paged_decode(s["cache"], s["q"], pages=pages)
        if kind == "decode":
            o = eva.paged_decode(s["cache"], s["q"])
    else:
        if kind in ("plan", "step"):
            _truncate_plain(s)
            slots, start, granted = _extend_plain(s)
        if kind in ("append", "step"):
            _append_plain(s, slots if kind == "step" else s["slots"])
        if kind in ("sparse", "step"):
            pages = _choose_plain(s)
            o = _attend_plain(s, pages)
        if kind == "decode":
            o = _attend_plain(s)
    if kind == "plan":
        return [slots, start, granted, s["table"], s["n_tok"], s["free"], s["n_free"]]
    if kind == "append":
        return [s["k"], s["vt"], s["mean"]]
    if kind == "sparse":
        return [o, pages]
    if kind == "step":
        return [o, pages, slots, s["k"], s["vt"], s["mean"]]
    return [o]


# ---- the same in 64 bits --------------------------------------------------
def _row64(c, x, b, pages, tail=None):
    """Output rows [H, d] of sequence b over the tokens of its pages (pages[g]: those of kv head g);
    tail: (position, key, value) of a token that the pool does not hold yet."""
    H, Hkv, d, P = c["H"], c["Hkv"], c["d"], c["P"]
    n = int(x["lens"][b]) + (tail is not None)
    table, rows = x["table"][b], []
    for g in range(Hkv):
        lp = torch.tensor(pages[g], device="cuda")
        pos = (lp.unsqueeze(1) * P + torch.arange(P, device="cuda")).flatten()
        pp = table[lp].long().clamp(min=0)
        K = x["k"][pp, g].double().reshape(-1, d)
        V = x["vt"][pp, g].double().permute(0, 1, 3, 2).reshape(-1, d)
        if tail is not None:
            K[pos == n - 1], V[pos == n - 1] = tail[0][g].double(), tail[1][g].double()
        K, V = K[pos < n], V[pos < n]
        q = x["q"][b].double().reshape(Hkv, H // Hkv, d)[g]
        rows.append(torch.softmax(torch.matmul(q, K.t().contiguous()) / math.sqrt(d), 1) @ V)
    return torch.cat(rows)


def _choice64(c, x, b, n):
    """Pages of each kv head of sequence b, of n tokens, in their order."""
    Hkv, P, S = c["Hkv"], c["P"], c["S"]
    held = _pages(n, P)
    if not S or held <= S:
        return [list(range(held))] * Hkv
    q = x["q"][b].double().reshape(Hkv, -1, c["d"])
    inner = x["table"][b][1:held - 1].long()
    res = []
    for g in range(Hkv):
        score = (x["mean"][inner, g].double().unsqueeze(1) * q[g]).sum(-1).max(-1).values.tolist()
        best = sorted(range(len(score)), key=lambda i: (-score[i], i))[:S - 2]
        res.append([0] + sorted(i + 1 for i in best) + [held - 1])
    return res


def _places(c, x):
    """Slots [B, T] of a step's new tokens, by lists."""
    P, T = c["P"], c["T"]
    stack, table = x["free"].tolist()[:int(x["n_free"])], [[p for p in row if p >= 0] for row in x["table"].tolist()]
    for row, n in reversed(list(zip(table, _lens(c)))):
        while len(row) > _pages(n, P):
            stack.append(row.pop())
    slots = []
    for row, n, t in zip(table, _lens(c), x["counts"].tolist()):
        while len(row) < _pages(n + t, P):
            row.append(stack.pop())
        slots.append([row[i // P] * P + i % P for i in range(n, n + t)] + [-1] * (T - t))
    return torch.tensor(slots, device="cuda")


def exact(c, seed):
    if c["kind"] == "plan":
        return None  # whole numbers alone
    x = _inputs(c, seed)
    B, P, T = c["B"], c["P"], c["T"]
    if c["kind"] in ("decode", "sparse"):
        o = torch.stack([_row64(c, x, b, _choice64(c, x, b, n)) for b, n in enumerate(_lens(c))])
        return [o] if c["kind"] == "decode" else [o, None]
    slots, o = x.get("slots"), None
    if c["kind"] == "step":
        # a new page, where a sequence needs one, is filled by its first token: no earlier one is read
        o = torch.stack([_row64(c, x, b, _choice64(c, x, b, n + 1), (x["k_new"][b, :, 0], x["v_new"][b, :, 0]))
                         for b, n in enumerate(_lens(c))])
        slots = _places(c, x)
    k, vt, mean = x["k"], x["vt"], x["mean"].double()
    v = vt.permute(0, 1, 2, 4, 3).reshape(k.shape)  # a copy, by slot
    for b in range(B):
        to = slots[b][slots[b] >= 0].long()
        m = to.numel()
        k[to // P, :, to % P] = x["k_new"][b, :, :m].transpose(0, 1)
        v[to // P, :, to % P] = x["v_new"][b, :, :m].transpose(0, 1)
        full = to[to % P == P - 1] // P
        mean[full] = k[full].double().sum(2) / P
    vt = v.reshape(*k.shape[:2], P // 8, 8, c["d"]).permute(0, 1, 2, 4, 3).contiguous()
    return [k, vt, mean] if o is None else [o, None, None, k, vt, mean]
