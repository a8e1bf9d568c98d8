"""The paged cache's calls reject bad arguments with the documented status codes and
errors before touching the GPU (no compute call is made here)."""
import ctypes

import pytest
import torch

from paper_2511_00576_amd import _lib, eva
from paged_reference import Table

INVALID, UNSUPPORTED, CAPACITY = _lib.EVA_ERR_INVALID, _lib.EVA_ERR_UNSUPPORTED, _lib.EVA_ERR_CAPACITY
FAKE = ctypes.c_void_p(0x10000)  # aligned, never dereferenced: validation fails first
OFF2 = ctypes.c_void_p(0x10002)
OFF8 = ctypes.c_void_p(0x10008)


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def table(**kw):
    a = dict(B=2, P=64, n_pages=100, max_pages=40, n_tok=0x50000, table=0x60000, free_pages=0x70000, n_free=0x80000)
    a.update(kw)
    return _lib.EvaPageTableStruct(**a)


def pool(**kw):
    a = dict(H=4, H_kv=2, d=64, dtype=_lib.EVA_BF16, P=64, n_pages=100, k=0x10000, vt=0x20000, k_mean=0x30000)
    a.update(kw)
    return _lib.EvaPCacheStruct(**a)


def ref(x):
    return None if x is None else ctypes.byref(x)


def extend(lib, t=None, counts=FAKE, T=3, slots=FAKE, start=FAKE, granted=FAKE):
    return lib.eva_page_extend(ref(t or table()), counts, T, slots, start, granted, None)


def truncate(lib, t=None, lens=FAKE):
    return lib.eva_page_truncate(ref(t or table()), lens, None)


def append(lib, c=None, k=FAKE, v=FAKE, slots=FAKE, B=2, T=3):
    return lib.eva_paged_append(ref(c or pool()), k, v, slots, B, T, None)


def decode(lib, c=None, t=None, q=FAKE, o=FAKE, pages=None, S=0, active=None, ws=None, n=0):
    return lib.eva_paged_decode(ref(c or pool()), ref(t or table()), q, o, pages, S, active, ws, n, None)


def select(lib, c=None, t=None, q=FAKE, S=5, first=1, last=1, pages=FAKE, ws=FAKE, n=1 << 30):
    return lib.eva_paged_select(ref(c or pool()), ref(t or table()), q, S, first, last, pages, ws, n, None)


LONG = table(max_pages=2000)  # more pages a sequence than one workgroup scores and ranks
TABLES = [(dict(B=0), INVALID), (dict(P=0), INVALID), (dict(P=8), INVALID), (dict(P=48), INVALID), (dict(P=512), INVALID),
          (dict(n_pages=0), INVALID), (dict(max_pages=0), INVALID), (dict(n_tok=None), INVALID), (dict(table=0x60002), INVALID),
          (dict(free_pages=None), INVALID), (dict(n_free=0x80001), INVALID), (dict(n_pages=2 ** 24 + 1), UNSUPPORTED),
          (dict(max_pages=2 ** 24 + 1), UNSUPPORTED), (dict(B=65536), UNSUPPORTED), (dict(B=60000, max_pages=20000), UNSUPPORTED)]
POOLS = [(dict(H=0), INVALID), (dict(H_kv=0), INVALID), (dict(H=5), INVALID), (dict(k=None), INVALID), (dict(vt=0x20008), INVALID),
         (dict(k_mean=0x30004), INVALID), (dict(P=24), INVALID), (dict(n_pages=0), INVALID), (dict(d=96), UNSUPPORTED),
         (dict(dtype=2), UNSUPPORTED), (dict(n_pages=2 ** 24 + 1), UNSUPPORTED)]


@pytest.mark.parametrize("kw,code", TABLES)
def test_tables_are_checked(lib, kw, code):
    t = table(**kw)
    assert extend(lib, t) == code and truncate(lib, t) == code
    c = pool(P=t.P, n_pages=t.n_pages) if t.P in (16, 32, 64, 128, 256) and 0 < t.n_pages <= 2 ** 24 else pool()
    assert decode(lib, c, t) == code and select(lib, c, t) == code
    assert lib.eva_paged_decode_workspace_bytes(ref(c), ref(t), 0) == 0
    assert lib.eva_paged_select_workspace_bytes(ref(c), ref(t), 5) == 0


@pytest.mark.parametrize("kw,code", POOLS)
def test_pools_are_checked(lib, kw, code):
    c = pool(**kw)
    assert append(lib, c) == code and decode(lib, c) == code and select(lib, c) == code


def test_null_structs(lib):
    assert lib.eva_page_extend(None, FAKE, 1, FAKE, FAKE, FAKE, None) == INVALID
    assert lib.eva_page_truncate(None, FAKE, None) == INVALID
    assert lib.eva_paged_append(None, FAKE, FAKE, FAKE, 1, 1, None) == INVALID
    assert lib.eva_paged_decode(None, ref(table()), FAKE, FAKE, None, 0, None, None, 0, None) == INVALID
    assert lib.eva_paged_decode(ref(pool()), None, FAKE, FAKE, None, 0, None, None, 0, None) == INVALID
    assert lib.eva_paged_select(ref(pool()), None, FAKE, 5, 1, 1, FAKE, FAKE, 1 << 30, None) == INVALID
    assert lib.eva_paged_decode_workspace_bytes(None, None, 0) == 0


@pytest.mark.parametrize("call,kw,code", [
    (extend, dict(T=0), INVALID), (extend, dict(slots=None), INVALID), (extend, dict(start=None), INVALID),
    (extend, dict(granted=None), INVALID), (extend, dict(counts=OFF2), INVALID), (extend, dict(slots=OFF2), INVALID),
    (extend, dict(T=2 ** 30 + 1), UNSUPPORTED), (extend, dict(t=table(B=65535), T=300000), UNSUPPORTED), (truncate, dict(lens=None), INVALID), (truncate, dict(lens=OFF2), INVALID),
    (append, dict(B=0), INVALID), (append, dict(T=0), INVALID), (append, dict(k=None), INVALID), (append, dict(v=OFF8), INVALID),
    (append, dict(slots=None), INVALID), (append, dict(slots=OFF2), INVALID), (append, dict(B=65536), UNSUPPORTED),
    (append, dict(T=2 ** 30 + 1), UNSUPPORTED), (append, dict(B=60000, T=60000), UNSUPPORTED),
    (decode, dict(q=None), INVALID), (decode, dict(o=OFF8), INVALID), (decode, dict(S=3), INVALID),
    (decode, dict(pages=FAKE), INVALID), (decode, dict(pages=FAKE, S=-1), INVALID), (decode, dict(pages=OFF2, S=3), INVALID),
    (decode, dict(active=OFF2), INVALID), (decode, dict(t=table(P=32)), INVALID), (decode, dict(t=table(n_pages=99)), INVALID),
    (decode, dict(c=pool(H=80000, H_kv=40000)), UNSUPPORTED),
    (decode, dict(c=pool(H=2 ** 30)), UNSUPPORTED),                        # rows
    (decode, dict(c=pool(H=60000, H_kv=30000), t=table(max_pages=2 ** 24)), UNSUPPORTED),  # chunks of all rows
    (select, dict(S=0), INVALID), (select, dict(first=-1), INVALID), (select, dict(last=0), INVALID),
    (select, dict(first=4, last=2), INVALID), (select, dict(q=None), INVALID), (select, dict(pages=OFF2), INVALID),
    (select, dict(c=pool(k_mean=None)), INVALID), (select, dict(t=table(P=32)), INVALID),
    (select, dict(t=LONG, ws=None), INVALID), (select, dict(t=LONG, ws=OFF8), INVALID),
    (select, dict(t=LONG, n=2 * 2 * 2000 * 8 - 1), CAPACITY),
])
def test_calls_are_checked(lib, call, kw, code):
    assert call(lib, **kw) == code


def test_workspaces(lib):
    c, t = pool(), table()
    assert lib.eva_paged_select_workspace_bytes(ref(c), ref(LONG), 5) == 2 * 2 * 2000 * 8
    assert lib.eva_paged_select_workspace_bytes(ref(c), ref(t), 5) == 0
    assert lib.eva_paged_decode_workspace_bytes(ref(c), ref(t), 0) > 0
    # rows of 12 blocks of 16 KB of keys and values, and of one more: 768 tokens of 64 features
    assert lib.eva_paged_decode_workspace_bytes(ref(c), ref(t), 12) == 0
    assert lib.eva_paged_decode_workspace_bytes(ref(c), ref(t), 13) > 0
    assert lib.eva_paged_decode_workspace_bytes(ref(c), ref(table(B=100)), 24) == 0   # twice that from 192 rows on
    assert lib.eva_paged_decode_workspace_bytes(ref(c), ref(table(B=100)), 25) > 0
    assert lib.eva_paged_decode_workspace_bytes(ref(c), ref(t), -1) == 0


# ---- the binding ----------------------------------------------------------------
def host(means=True):
    t = eva.PageTable(2, 16, 10, 100, device="cpu")
    return t, eva.PagedCache(t, 4, 2, 64, means=means)


def test_host_memory_is_refused():
    t, c = host()
    q, k = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    n = torch.ones(2, dtype=torch.int32)
    for call in (lambda: eva.page_extend(t), lambda: eva.page_extend(t, 3, n), lambda: eva.page_truncate(t, n),
                 lambda: eva.paged_append(c, k, k, n.reshape(2, 1)), lambda: eva.paged_decode(c, q),
                 lambda: eva.paged_select(c, q, 3), lambda: eva.paged_decode(c, q, pages=torch.zeros(2, 2, 3, dtype=torch.int32))):
        with pytest.raises(RuntimeError, match="ROCm device"):
            call()


def test_shapes_and_types_are_refused():
    t, c = host()
    q, k = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 1, 64, dtype=torch.bfloat16)
    n, slots = torch.ones(2, dtype=torch.int32), torch.zeros(2, 1, dtype=torch.int32)
    pages = torch.zeros(2, 2, 3, dtype=torch.int32)
    for call in (lambda: eva.page_extend(t, 0), lambda: eva.page_extend(t, 1, n.long()), lambda: eva.page_extend(t, 1, n[:1]),
                 lambda: eva.page_truncate(t, n.float()), lambda: eva.paged_append(c, k.float(), k, slots),
                 lambda: eva.paged_append(c, k, k[:, :1], slots), lambda: eva.paged_append(c, k, k, n),
                 lambda: eva.paged_append(c, k, k, slots.long()),
                 lambda: eva.paged_append(c, k.expand(2, 2, 3, 64), k.expand(2, 2, 3, 64), slots.expand(2, 3)),
                 lambda: eva.paged_decode(c, q[:1]), lambda: eva.paged_decode(c, q.float()),
                 lambda: eva.paged_decode(c, q, pages=pages[0]), lambda: eva.paged_decode(c, q, pages=pages[:, :1]),
                 lambda: eva.paged_decode(c, q, pages=pages[..., :0]), lambda: eva.paged_decode(c, q, pages=pages.long()),
                 lambda: eva.paged_decode(c, q, active=n.bool()), lambda: eva.paged_decode(c, q, out=q.float()),
                 lambda: eva.paged_select(c, q, 0), lambda: eva.paged_select(c, q[:, :2], 3),
                 lambda: eva.PageTable(2, 48, 10, 100, device="cpu"),
                 lambda: eva.PageTable(2, 16, 10, 100, device="cpu", storage=(n, n, n, n)),
                 lambda: eva.PagedCache(t, 4, 2, 64, storage=(c.k, c.k, c.k_mean))):
        with pytest.raises(ValueError):
            call()


def test_no_tokens_are_no_call():
    t, c = host()
    eva.paged_append(c, torch.zeros(2, 2, 0, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 0, 64, dtype=torch.bfloat16),
                     torch.zeros(2, 0, dtype=torch.int32))


def test_arrays_that_there_are_already():
    t, c = host()
    t2 = eva.PageTable(2, 16, 10, 100, device="cpu", storage=(t.n_tok, t.table, t.free_pages, t.n_free))
    c2 = eva.PagedCache(t2, 4, 2, 64, storage=(c.k, c.vt, None))
    assert c2.k is c.k and c2.struct.k == c.k.data_ptr() and not c2.struct.k_mean
    assert t2.struct.table == t.table.data_ptr() and t2.struct.max_pages == 7


# ---- the tests' own model of the table ----------------------------------------------
def test_model_gives_and_takes_back():
    m = Table(2, 16, 5, 4)
    slots, start, granted = m.extend(20, [17, 3])
    assert granted == [17, 3] and slots[0][:2] == [0, 1] and slots[0][16] == 16 and slots[1][:3] == [32, 33, 34]
    before = (list(m.n), [list(r) for r in m.rows], list(m.stack))
    m.extend(20, [20, 0])
    m.truncate([17, 3])
    assert before == (m.n, m.rows, m.stack)
    # 17 + 50 tokens are more than four pages hold, so the first needs nothing; the other's 3 + 40 need the two that are left
    assert m.extend(50, [50, 40])[2] == [0, 40] and m.stack == []
