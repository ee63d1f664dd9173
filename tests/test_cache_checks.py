"""Refusals of the 4-bit cache's calls, each told by its own text or status."""
import ctypes

import pytest
import torch

from paper_2604_00754_b200 import binding as sa
from paper_2604_00754_b200.cache import KVCache
from test_cache_host import FAKE, ODD, OTHER, ST, append, attend, cache


def test_append_checks_the_holders_it_is_given():
    assert append(cache(refs=FAKE + 2)) == 1
    c = cache(refs=FAKE + 2, lens=None)                  # a read looks at no holders
    st = (ctypes.c_int64 * 3)(1024, 128, 60)             # and stops at its strides
    assert sa.load_library().sa_cache_read(ctypes.byref(c), 0, 1, 1, FAKE, 2 * FAKE, sa.BF16, st, None, None, None, None) == 1


# ---- the head dimension: a pool of 16 tokens of 64 dimensions a page is also one of 32 of 32 and of 64 of 16

OTHER_DIMENSIONS = [16, 32]
TOKENS = "the pool's pages do not hold that many tokens of this head dimension"


def books():
    return (torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))


def rows(d, dtype=torch.bfloat16):
    return torch.zeros(2, 2, 1, d, dtype=dtype)


@pytest.mark.parametrize("d", OTHER_DIMENSIONS + [128])
@pytest.mark.parametrize("said", ["by the pool", "by the call"])
def test_tensors_of_another_head_dimension_are_refused(d, said):
    pool, kw = sa.sa_cache_pool(1, 4, 2, 16, 64, device="cpu"), {}
    if said == "by the call":
        pool, kw = pool.clone(), dict(page=16)
    table, lens = books()
    x, q = rows(d), torch.zeros(2, 4, 1, d, dtype=torch.bfloat16)
    for call in (lambda: sa.sa_cache_append(pool, table, lens, x, x.clone(), **kw),
                 lambda: sa.sa_cache_read(pool, table, x, x.clone(), **kw),
                 lambda: sa.sa_cache_attend(pool, table, lens, q, **kw)):
        with pytest.raises(ValueError, match=TOKENS):
            call()


@pytest.mark.parametrize("d", OTHER_DIMENSIONS)
def test_a_cache_refuses_tensors_of_another_head_dimension(d):
    c = KVCache(1, 2, 64, 2, 40, page=16, device="cpu")
    x = rows(d)
    for call in (lambda: c.append(0, x, x.clone()), lambda: c.read(0, x, x.clone()), lambda: c.attend(0, x)):
        with pytest.raises(ValueError, match=TOKENS):
            call()
    c.pool = c.pool.clone()                                  # says nothing; the cache still knows
    with pytest.raises(ValueError, match=TOKENS):
        c.append(0, x, x.clone())


def test_a_page_that_is_not_the_pools_is_refused():
    pool, (table, lens) = sa.sa_cache_pool(1, 4, 2, 16, 64, device="cpu"), books()
    refs = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="made for 16 tokens per page, not 32"):
        sa.sa_cache_append(pool, table, lens, rows(32), rows(32), page=32)
    with pytest.raises(ValueError, match="made for 16 tokens per page, not 32"):
        sa.sa_cache_reserve(pool, table, lens, refs, lens.clone(), page=32)


@pytest.mark.parametrize("kw", [{}, dict(page=16)])
def test_the_right_head_dimension_gets_as_far_as_the_device(kw):
    pool, (table, lens) = sa.sa_cache_pool(1, 4, 2, 16, 64, device="cpu"), books()
    for p in (pool, pool.clone()):
        with pytest.raises(ValueError, match="must be on a CUDA device"):
            sa.sa_cache_append(p, table, lens, rows(64), rows(64), **kw)
        with pytest.raises(ValueError, match="must be on a CUDA device"):
            sa.sa_cache_read(p, table, rows(64), rows(64), **kw)
        with pytest.raises(ValueError, match="must be on a CUDA device"):
            sa.sa_cache_attend(p, table, lens, rows(64), **kw)


# ---- numbers that the C calls take in 32 bits

@pytest.mark.parametrize("kw", [dict(layer=1 << 32), dict(layer=-(1 << 32)), dict(w=(1 << 32) + 5), dict(flags=1 << 33),
                                dict(layer=1 << 70), dict(page=(1 << 32) + 16)])
def test_numbers_past_32_bits_are_refused(kw):
    pool, (table, lens) = sa.sa_cache_pool(1, 4, 2, 16, 64, device="cpu").clone(), books()
    with pytest.raises(ValueError, match="numbers of 32 bits"):
        sa.sa_cache_attend(pool, table, lens, rows(64), **kw)
    if not {"w", "flags"} & set(kw):
        with pytest.raises(ValueError, match="numbers of 32 bits"):
            sa.sa_cache_append(pool, table, lens, rows(64), rows(64), **kw)
        with pytest.raises(ValueError, match="numbers of 32 bits"):
            sa.sa_cache_read(pool, table, rows(64), rows(64), **kw)
    if "page" in kw:
        refs = torch.zeros(4, dtype=torch.int32)
        with pytest.raises(ValueError, match="numbers of 32 bits"):
            sa.sa_cache_reserve(pool, table, lens, refs, lens.clone(), **kw)
        with pytest.raises(ValueError, match="numbers of 32 bits"):
            sa.sa_cache_fork(table, lens, refs, lens[:1], lens[1:], **kw)


def test_batches_past_32_bits_are_refused():
    pool, (table, lens) = sa.sa_cache_pool(1, 4, 2, 16, 64, device="cpu"), books()
    many = rows(64)[:1].expand((1 << 32) + 1, 2, 1, 64)
    for call in (lambda: sa.sa_cache_append(pool, table, lens, many, many), lambda: sa.sa_cache_attend(pool, table, lens, many)):
        with pytest.raises(ValueError, match="a dimension of 2.31 or more"):
            call()


# ---- outputs whose rows share memory: which row stays would be chance

@pytest.mark.parametrize("B,strides", [(2, (0, 128, 64)), (1, (1024, 0, 64)), (2, (0, 0, 64))])
def test_outputs_that_share_memory_are_refused(B, strides):
    st = (ctypes.c_int64 * 3)(*strides)
    assert attend(cache(), B=B, ys=st) == 1
    assert sa.load_library().sa_cache_read(ctypes.byref(cache()), 0, B, 1, FAKE, OTHER, sa.BF16, st, None, None, None, None) == 1


def test_inputs_may_share_memory():
    st = (ctypes.c_int64 * 3)(0, 0, 64)
    assert attend(cache(), B=2, qs=st, ws_bytes=64) == 3            # as far as its workspace


# ---- what each Python call says of tensors that do not fit; a call without a fault gets as far as the device

@pytest.fixture
def t():
    table, lens = books()
    return dict(pool=sa.sa_cache_pool(1, 4, 2, 16, 64, device="cpu"), table=table, lens=lens,
                refs=torch.zeros(4, dtype=torch.int32), x=rows(64), q=torch.zeros(2, 4, 1, 64, dtype=torch.bfloat16),
                list=torch.zeros(2, dtype=torch.int32))


POOL = r"pool must be contiguous uint8 \[layers, pages, Hkv, 2, page \* \(d/2 \+ d/16\)\]"
TABLE, LENS = r"table must be contiguous int32 \[slots, row\]", r"lens must be contiguous int32 \[slots\]"
LISTS = "counts must be contiguous int32"
DEVICE = "must be on a CUDA device"


def attend_of(t, **kw):
    return sa.sa_cache_attend(t["pool"], t["table"], t["lens"], t["q"], **kw)


def append_of(t, **kw):
    return sa.sa_cache_append(t["pool"], t["table"], t["lens"], t["x"], t.get("v", t["x"]), **kw)


def read_of(t, **kw):
    return sa.sa_cache_read(t["pool"], t["table"], t["x"], t.get("v", t["x"]), **kw)


def half(x):
    return torch.cat((x, x), 1)[:, ::2]


@pytest.mark.parametrize("name,change,text", [
    ("pool", lambda x: x.int(), POOL), ("pool", lambda x: x[0], POOL), ("pool", half, POOL),
    ("pool", lambda x: x[:, :, :, :1].contiguous(), POOL), ("table", lambda x: x.long(), TABLE),
    ("table", half, TABLE), ("table", lambda x: x[0], TABLE)])
def test_caches_that_do_not_fit_say_so(t, name, change, text):
    t[name] = change(t[name])
    for call in (attend_of, append_of, read_of):
        with pytest.raises(ValueError, match=text):
            call(t)


@pytest.mark.parametrize("change", [lambda x: x.long(), lambda x: x[:1], lambda x: torch.stack((x, x), 1)[:, 0]])
def test_lists_that_do_not_fit_say_so(t, change):
    good, bad = t["list"], change(t["list"])
    for call, names in ((attend_of, ("slots", "counts")), (append_of, ("slots", "counts")),
                        (read_of, ("slots", "starts", "counts"))):
        for name in names:
            with pytest.raises(ValueError, match=LISTS):
                call(t, **{name: bad})
            with pytest.raises(ValueError, match=DEVICE):
                call(t, **{name: good})
    t["lens"] = bad
    for call in (attend_of, append_of):
        with pytest.raises(ValueError, match=LENS):
            call(t)
    with pytest.raises(ValueError, match=DEVICE):
        read_of(t)                                           # looks at no lengths


@pytest.mark.parametrize("x,v,text", [
    (lambda x: x[0], lambda x: x[0], r"k and v must be \[B,Hkv,T,d\]"), (lambda x: x, lambda x: x[:1], r"k and v must be \[B,Hkv,T,d\]"),
    (lambda x: x, lambda x: x.float(), r"k and v must be \[B,Hkv,T,d\]"),
    (lambda x: half(x.transpose(1, 3)).transpose(1, 3), lambda x: half(x.transpose(1, 3)).transpose(1, 3), "head dimension must be contiguous"),
    (lambda x: x, lambda x: torch.cat((x, x), 1)[:, :2], "k and v must share their strides"),
    (lambda x: x[:, :1].contiguous(), lambda x: x[:, :1].contiguous(), "k and v must have the pool's heads")])
def test_keys_and_values_that_do_not_fit_say_so(t, x, v, text):
    t["x"], t["v"] = x(t["x"]), v(t["x"])
    for call in (append_of, read_of):
        with pytest.raises(ValueError, match=text):
            call(t)


def test_read_into_rows_that_share_memory_says_so(t):
    t["x"] = t["v"] = t["x"][:1].expand(2, 2, 1, 64)
    with pytest.raises(ValueError, match="an output shares memory between its rows"):
        read_of(t)
    with pytest.raises(ValueError, match=DEVICE):
        append_of(t)                                         # broadcast inputs are fine


@pytest.mark.parametrize("kw,text", [
    (dict(y=torch.zeros(2, 4, 1, 64)), "y must have the shape and type of q"),
    (dict(y=torch.zeros(2, 4, 2, 64, dtype=torch.bfloat16)), "y must have the shape and type of q"),
    (dict(y=torch.zeros(2, 1, 1, 64, dtype=torch.bfloat16).expand(2, 4, 1, 64)), "an output shares memory between its rows"),
    (dict(lse=torch.zeros(2, 4)), "lse must be contiguous float32"), (dict(lse=torch.zeros(2, 4, 1).double()), "lse must be contiguous float32"),
    (dict(lse=torch.zeros(2, 4, 2)[..., :1]), "lse must be contiguous float32")])
def test_outputs_of_attend_that_do_not_fit_say_so(t, kw, text):
    with pytest.raises(ValueError, match=text):
        attend_of(t, **kw)


def test_queries_that_do_not_fit_say_so(t):
    q = t["q"]
    for bad, kind, text in ((q[0], ValueError, r"q must be \[B,Hq,T,d\]"), (q.half(), TypeError, "float32 or bfloat16"),
                            (half(q.transpose(1, 3)).transpose(1, 3), ValueError, "head dimension must be contiguous"),
                            (q[:, :3].contiguous(), sa.SaError, "sa_cache_attend")):
        t["q"] = bad
        with pytest.raises(kind, match=text):
            attend_of(t)
    t["q"] = q
    with pytest.raises(ValueError, match=DEVICE):
        attend_of(t)


def test_books_that_do_not_fit_say_so(t):
    table, lens, refs, two = t["table"], t["lens"], t["refs"], t["list"]
    reserve = lambda **kw: sa.sa_cache_reserve(*((t | kw)[n] for n in ("pool", "table", "lens", "refs", "add")), 16, kw.get("got"))  # noqa: E731
    t["add"] = two
    REFS = r"refs must be contiguous int32 \[pages\]"
    for kw, text in ((dict(refs=refs[:3]), REFS), (dict(refs=refs.long()), REFS), (dict(lens=lens[:1]), LENS), (dict(table=table.long()), TABLE),
                     (dict(add=two[:1]), r"add must be contiguous int32 \[slots\]"), (dict(add=two.long()), r"add must be contiguous int32 \[slots\]"),
                     (dict(got=two[:1]), r"got must be contiguous int32 \[slots\]"), (dict(got=two.float()), r"got must be contiguous int32 \[slots\]"),
                     ({}, DEVICE)):
        with pytest.raises(ValueError, match=text):
            reserve(**kw)
    for refs_, live, text in ((refs[:3], None, REFS), (refs, two, r"live must be int32 \[1\]"), (refs, None, DEVICE)):
        with pytest.raises(ValueError, match=text):
            sa.sa_cache_compact(t["pool"], table, refs_, live)
    for a, b, text in ((two, two[:1], "parents and children must have one length"), (two.long(), two, "slot lists must be contiguous int32"),
                       (two, two, DEVICE)):
        with pytest.raises(ValueError, match=text):
            sa.sa_cache_fork(table, lens, refs, a, b, page=16)
    for slots, text in ((two.long(), "slot lists must be contiguous int32"), (two, DEVICE)):
        with pytest.raises(ValueError, match=text):
            sa.sa_cache_free(table, lens, refs, slots)
    with pytest.raises(ValueError, match=r"refs must be contiguous int32 \[pages\]"):
        append_of(t, refs=refs[:3])
    with pytest.raises(ValueError, match=DEVICE):
        append_of(t, refs=refs)


# ---- reads of the C library, k and v in two places

@pytest.mark.parametrize("kw,expect", [
    (dict(k=None), 1), (dict(v=None), 1), (dict(k=ODD), 1), (dict(v=ODD), 1), (dict(dt=5), 1), (dict(layer=7), 1),
    (dict(layer=-1), 1), (dict(B=0), 1), (dict(T=0), 1), (dict(st=None), 1), (dict(st=(ctypes.c_int64 * 3)(1024, 100, 64)), 1),
    (dict(st=(ctypes.c_int64 * 3)(-8, 128, 64)), 1), (dict(T=2, st=(ctypes.c_int64 * 3)(1024, 128, 56)), 1), (dict(B=1 << 17), 2),
    (dict(T=1 << 30), 2), (dict(slots=0x1001), 1), (dict(starts=0x1002), 1), (dict(counts=0x1003), 1), (dict(v=FAKE), 1)])
def test_read_refusals(kw, expect):
    a = dict(layer=0, B=1, T=1, k=FAKE, v=OTHER, dt=sa.BF16, st=ST, slots=None, starts=None, counts=None) | kw
    assert sa.load_library().sa_cache_read(ctypes.byref(cache(lens=None)), *a.values(), None) == expect


@pytest.mark.parametrize("kw,expect", [(dict(pool=None), 1), (dict(pool=ODD), 1), (dict(table=None), 1), (dict(k_scale=0.3), 1),
                                       (dict(v_scale=0.0), 1), (dict(page=24), 1), (dict(d=40), 2)])
def test_reads_of_bad_caches_are_refused(kw, expect):
    assert sa.load_library().sa_cache_read(ctypes.byref(cache(**kw)), 0, 1, 1, FAKE, OTHER, sa.BF16, ST, None, None, None, None) == expect
