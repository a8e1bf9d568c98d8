"""Ways of the paged decode and choice that the other tests do not take: parts within rows for more
sequences than lanes, sequences that share pages; and the prompt's rows, by type."""
import pytest
import torch

from paper_2511_00576_amd import eva
from paged_reference import attend
from test_gpu_paged import BF16, F32, build, check_choice, check_rows, ints, query

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    eva._lib.load()


def parts_within_rows(lens, active, unit, most, tokens):
    """The decode's sharing rule: (chunks of a part, parts of every sequence) where parts end with their rows, as
    they do if the 512 workgroups suffice for that; else None."""
    chunks = [max(1, -(-n // tokens)) if on else 0 for n, on in zip(lens, active)]
    wgs = min(512, len(lens) * unit * -(--(-most // tokens) // 4))
    part = max(-(-sum(chunks) * unit // wgs), 4)
    parts = [-(-c // part) for c in chunks]
    return (part, parts) if part <= 64 and sum(parts) * unit <= wgs else None


# long rows among short ones by sequence; the first window of 64 sequences, the second, and the third
WITHIN = [
    (100, 1, 1, 64, 60, {10: 1500, 70: 3000, 99: 4000}),
    (100, 6, 2, 64, 60, {0: 2011, 63: 3999, 64: 1777, 65: 100}),
    (66, 1, 1, 128, 16, {5: 10780, 20: 10784, 33: 10770, 63: 10780, 64: 10781, 65: 10769}),    # parts of five and nine chunks
    (150, 40, 1, 64, 50, {3: 900, 128: 3100, 149: 700}),                                       # two groups of heads
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("B,H,Hkv,d,short,long", WITHIN)
def test_parts_within_rows_of_more_sequences_than_lanes(B, H, Hkv, d, short, long, masked, dtype):
    P = 32
    lens = [long.get(i, (i * 37) % (short + 1)) for i in range(B)]
    active = [int(not masked or i in long or i % 20 != 13) for i in range(B)]
    if masked and B != 66:
        active[min(long)] = 0
    tokens = 16 if dtype == F32 and d == 128 else 32
    unit = Hkv * (-(-(H // Hkv) // 32) if H // Hkv > 16 else 1)
    part, parts = parts_within_rows(lens, active, unit, -(-max(lens) // P) * P, tokens)
    split = [b for b in range(B) if parts[b] > 1]
    assert any(b >= 64 for b in split) and (B == 66) == (part > 4)
    cache, ks, vs = build(B, H, Hkv, d, P, lens, dtype, seed=B + H)
    q = query(B, H, d, dtype, seed=B)
    out = torch.full((B, H, d), 3.0, dtype=dtype, device="cuda")
    o = eva.paged_decode(cache, q.cuda(), active=ints(active), out=out)
    off = [b for b in range(B) if not active[b]]
    check_rows(o, q, ks, vs, P, dtype, skip=off)
    assert (o[off] == 3).all()
    # lists of pages whose rows are split as well
    S = 60
    g = torch.Generator().manual_seed(B)
    lists = [[torch.randperm(S, generator=g).tolist() for _ in range(Hkv)] for _ in range(B)]
    o = eva.paged_decode(cache, q.cuda(), pages=ints(lists), active=ints(active), out=out)
    check_rows(o, q, ks, vs, P, dtype, lists, skip=off)
    assert (o[off] == 3).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("use_workspace", [True, False])
@pytest.mark.parametrize("prompt,most", [(64, 0), (3200, 0), (3200, 9000)])
def test_sequences_that_share_a_prompt(prompt, most, use_workspace, dtype):
    """Sequences whose first pages are one's: each attends the common rows and then its own."""
    P, d, H, Hkv = 32, 64, 4, 2
    own = [40, 1, 0, 333, 32]
    lens = [prompt + n for n in own]
    cache, ks, vs = build(5, H, Hkv, d, P, lens, dtype, seed=prompt, most=most or None)
    table = cache.table.table
    table[1:, :prompt // P] = table[0, :prompt // P].clone()
    for b in range(1, 5):
        ks[b][:prompt], vs[b][:prompt] = ks[0][:prompt], vs[0][:prompt]
    q = query(5, H, d, dtype, seed=prompt)
    o = eva.paged_decode(cache, q.cuda(), use_workspace=use_workspace)
    check_rows(o, q, ks, vs, P, dtype)
    pages = check_choice(cache, q, lens, 4, 1, 1)
    o = eva.paged_decode(cache, q.cuda(), pages=ints(pages), use_workspace=use_workspace)
    check_rows(o, q, ks, vs, P, dtype, pages)


@pytest.mark.parametrize("P,d", [(16, 64), (64, 128)])
def test_the_prompts_last_row_in_fp32(P, d):
    """A prompt's last row from the prefill, with a window of all tokens, and from the paged cache: both are the
    64-bit row within fp32's bound, so they differ by twice that at most."""
    H, Hkv, lens = 6, 2, [90, 31, 64, 1, 200]
    B, L = len(lens), max(lens)
    g = torch.Generator().manual_seed(d)
    t = eva.PageTable(B, P, 60, 400)
    cache = eva.PagedCache(t, H, Hkv, d, F32)
    q, k, v = (torch.randn(B, h, L, d, generator=g) for h in (H, Hkv, Hkv))
    slots, *_ = eva.page_extend(t, L, ints(lens))
    eva.paged_append(cache, k.cuda(), v.cuda(), slots)
    whole = eva.prefill(q.cuda(), k.cuda(), v.cuda(), W=L, C=16).cpu().double()
    last = torch.stack([q[b, :, n - 1] for b, n in enumerate(lens)])
    o = eva.paged_decode(cache, last.cuda()).cpu().double()
    for b, n in enumerate(lens):
        for h in range(H):
            ref, bound = attend(last[b, h:h + 1], k[b, h * Hkv // H, :n].double(), v[b, h * Hkv // H, :n].double(), F32)
            assert ((o[b, h] - ref[0]).abs() <= bound[0]).all()
            assert ((whole[b, h, n - 1] - ref[0]).abs() <= bound[0]).all()
            assert float(bound.max()) < 1e-3
