"""Host-side checks of the 4-bit cache that need no GPU: sizes and refusals before any launch, and the
float64 statement that the GPU tests compare with."""
import ctypes

import numpy as np
import pytest
import torch

import cache_ref as ref
from paper_2604_00754_b200 import binding as sa

FAKE, ODD, OTHER = 0x1000, 0x1004, 0x2000          # never dereferenced: every case fails before a launch
ST = (ctypes.c_int64 * 3)(1024, 128, 64)


def cache(**kw):
    base = dict(pool=FAKE, table=FAKE, lens=FAKE, refs=FAKE, layers=2, pages=8, Hkv=2, d=64, page=32, slots=3,
                row=4, k_scale=0.5, v_scale=1.0)
    return sa.SaCache(**(base | kw))


def attend(c, layer=0, B=1, T=1, Hq=4, q=FAKE, dt=sa.BF16, qs=ST, slots=None, counts=None, w=0, flags=1, scale=0.0,
           y=OTHER, ys=ST, lse=None, ws=FAKE, ws_bytes=1 << 40):
    return sa.load_library().sa_cache_attend(ctypes.byref(c), layer, B, T, Hq, q, dt, qs, slots, counts, w, flags,
                                             scale, y, ys, lse, ws, ws_bytes, None)


def append(c, layer=0, B=1, T=1, k=FAKE, v=FAKE, dt=sa.BF16, st=ST, slots=None, counts=None):
    return sa.load_library().sa_cache_append(ctypes.byref(c), layer, B, T, k, v, dt, st, slots, counts, None)


GEOMETRY = [(dict(layers=0), 1), (dict(pages=0), 1), (dict(Hkv=0), 1), (dict(page=24), 1), (dict(page=256), 1),
            (dict(slots=0), 1), (dict(row=0), 1), (dict(d=40), 2), (dict(d=272), 2), (dict(row=1 << 26), 2), (dict(slots=1 << 20, row=1 << 12), 2),
            (dict(table=None), 1), (dict(table=FAKE + 2), 1)]


@pytest.mark.parametrize("kw,expect", GEOMETRY + [
    (dict(pool=None), 1), (dict(pool=ODD), 1), (dict(lens=None), 1), (dict(k_scale=0.3), 1), (dict(v_scale=0.0), 1),
    (dict(k_scale=-1.0), 1), (dict(v_scale=float("inf")), 1), (dict(v_scale=float("nan")), 1),
    (dict(k_scale=2.0 ** 40), 1)])
def test_bad_caches_are_refused(kw, expect):
    assert attend(cache(**kw)) == expect
    assert append(cache(**kw)) == expect


@pytest.mark.parametrize("kw,expect", [
    (dict(layer=2), 1), (dict(layer=-1), 1), (dict(B=0), 1), (dict(T=0), 1), (dict(Hq=3), 1), (dict(Hq=0), 1),
    (dict(q=None), 1), (dict(q=ODD), 1), (dict(y=None), 1), (dict(y=ODD), 1), (dict(y=FAKE), 1), (dict(dt=2), 1), (dict(w=-1), 1),
    (dict(flags=2), 1), (dict(flags=5), 1), (dict(scale=-1.0), 1), (dict(scale=float("nan")), 1),
    (dict(scale=float("inf")), 1), (dict(lse=0x1002), 1), (dict(slots=0x1001), 1), (dict(counts=0x1001), 1),
    (dict(qs=None), 1), (dict(qs=(ctypes.c_int64 * 3)(1024, 128, 60)), 1), (dict(T=2, qs=(ctypes.c_int64 * 3)(0, 0, 56)), 1),
    (dict(ys=(ctypes.c_int64 * 3)(-8, 0, 64)), 1), (dict(ws=None), 1), (dict(ws=ODD), 1), (dict(ws_bytes=64), 3),
    (dict(B=70000), 2), (dict(B=65535, T=1 << 24), 2)])
def test_attend_refusals(kw, expect):
    assert attend(cache(), **kw) == expect


@pytest.mark.parametrize("kw,expect", [
    (dict(k=None), 1), (dict(v=ODD), 1), (dict(dt=5), 1), (dict(layer=7), 1), (dict(T=0), 1), (dict(st=None), 1),
    (dict(st=(ctypes.c_int64 * 3)(1024, 100, 64)), 1), (dict(B=1 << 17), 2), (dict(T=1 << 30), 2)])
def test_append_and_read_refusals(kw, expect):
    assert append(cache(), **kw) == expect
    a = dict(layer=0, B=1, T=1, k=FAKE, v=FAKE, dt=sa.BF16, st=ST) | kw
    assert sa.load_library().sa_cache_read(ctypes.byref(cache(lens=None)), *a.values(), None, None, None, None) == expect


def test_one_tensor_for_both_outputs_is_refused():
    a = dict(layer=0, B=1, T=1, k=FAKE, v=FAKE, dt=sa.BF16, st=ST)
    assert sa.load_library().sa_cache_read(ctypes.byref(cache()), *a.values(), None, None, None, None) == 1


def test_books_refusals():
    lib, c = sa.load_library(), cache()
    r = ctypes.byref
    for kw, expect in GEOMETRY + [(dict(refs=None), 1), (dict(lens=None), 1)]:
        bad = cache(**kw)
        assert lib.sa_cache_free(r(bad), 1, FAKE, None) == expect
        assert lib.sa_cache_fork(r(bad), 1, FAKE, FAKE, None) == expect
        assert lib.sa_cache_reserve(r(bad), FAKE, OTHER, FAKE, 1 << 30, None) == expect
        if "lens" not in kw:
            assert lib.sa_cache_compact(r(bad), FAKE, FAKE, 1 << 30, None) == expect
    assert lib.sa_cache_free(None, 1, FAKE, None) == 1
    assert lib.sa_cache_free(r(c), -1, FAKE, None) == 1
    assert lib.sa_cache_free(r(c), 1, None, None) == 1
    assert lib.sa_cache_free(r(c), 0, None, None) == 0          # nothing to do, nothing launched
    assert lib.sa_cache_fork(r(c), 1, FAKE, None, None) == 1
    assert lib.sa_cache_fork(r(c), 0, None, None, None) == 0
    assert lib.sa_cache_reserve(r(c), None, FAKE, FAKE, 1 << 30, None) == 1
    assert lib.sa_cache_reserve(r(c), FAKE, None, FAKE, 1 << 30, None) == 1
    assert lib.sa_cache_reserve(r(c), FAKE, OTHER, None, 1 << 30, None) == 1
    assert lib.sa_cache_reserve(r(c), FAKE, FAKE, FAKE, 1 << 30, None) == 1      # add and got are one
    assert lib.sa_cache_reserve(r(c), FAKE, OTHER, FAKE, 16, None) == 3
    assert lib.sa_cache_reserve(r(cache(pool=ODD)), FAKE, OTHER, FAKE, 1 << 30, None) == 1
    assert lib.sa_cache_compact(r(c), FAKE, FAKE, 16, None) == 3
    assert lib.sa_cache_compact(r(c), 0x1002, FAKE, 1 << 30, None) == 1


def test_sizes():
    lib, c = sa.load_library(), cache()
    assert lib.sa_cache_page_bytes(ctypes.byref(c)) == 2 * 2 * 32 * (32 + 4)
    assert lib.sa_cache_page_bytes(ctypes.byref(cache(d=20))) == 0
    wrong = ctypes.c_size_t(-1).value
    assert lib.sa_cache_ws_bytes(ctypes.byref(c)) >= 4 * (3 * 3 + 8)
    assert lib.sa_cache_ws_bytes(ctypes.byref(cache(page=1))) == wrong
    assert 0 < lib.sa_cache_attend_ws_bytes(ctypes.byref(c), 1, 1, 4, sa.BF16) < wrong
    assert lib.sa_cache_attend_ws_bytes(ctypes.byref(c), 1, 1, 5, sa.BF16) == wrong
    assert "cache" in sa.status_string(8)


def tensors(d=64, P=16):
    return dict(pool=sa.sa_cache_pool(1, 4, 2, P, d, device="cpu"), table=torch.zeros(2, 3, dtype=torch.int32),
                lens=torch.zeros(2, dtype=torch.int32), refs=torch.zeros(4, dtype=torch.int32))


def test_python_calls_check_their_tensors():
    t = tensors()
    q = torch.zeros(2, 4, 1, 64, dtype=torch.bfloat16)
    k = torch.zeros(2, 2, 1, 64, dtype=torch.bfloat16)
    call = lambda **kw: sa.sa_cache_attend(t["pool"], t["table"], t["lens"], kw.pop("q", q), **kw)  # noqa: E731
    for kw in (dict(q=q[0]), dict(y=torch.zeros(2, 4, 1, 64)), dict(lse=torch.zeros(2, 4)), dict(slots=torch.zeros(2)),
               dict(counts=torch.zeros(3, dtype=torch.int32)), dict(q=torch.zeros(2, 4, 1, 80, dtype=torch.bfloat16)),
               dict(q=torch.zeros(2, 4, 2, 128, dtype=torch.bfloat16)[..., ::2]),
               dict(q=torch.zeros(2, 4, 3, 64), y=torch.zeros(2, 4, 1, 64).expand(2, 4, 3, 64))):
        with pytest.raises(ValueError):
            call(**kw)
    with pytest.raises(TypeError):
        call(q=q.half())
    with pytest.raises(sa.SaError):
        call(q=torch.zeros(2, 3, 1, 64, dtype=torch.bfloat16))
    for bad in (dict(pool=t["pool"][:, ::2]), dict(pool=t["pool"].int()), dict(table=t["table"].long()),
                dict(lens=torch.zeros(3, dtype=torch.int32)), dict(table=t["table"][:, :2])):
        a = t | bad
        with pytest.raises(ValueError):
            sa.sa_cache_append(a["pool"], a["table"], a["lens"], k, k)
    for x, y in ((k, k[:1]), (k, k.float()), (k.expand(2, 2, 1, 64), torch.zeros(2, 1, 2, 64).bfloat16().transpose(1, 2)[:, :, :1].expand(2, 2, 5, 64)),
                 (torch.zeros(2, 3, 1, 64), torch.zeros(2, 3, 1, 64))):
        with pytest.raises(ValueError):
            sa.sa_cache_append(t["pool"], t["table"], t["lens"], x, y)
    with pytest.raises(ValueError):
        sa.sa_cache_read(t["pool"], t["table"], k[:1].expand(2, 2, 1, 64), k)
    with pytest.raises(ValueError):
        sa.sa_cache_fork(t["table"], t["lens"], t["refs"], t["lens"], t["lens"][:1], page=16)
    with pytest.raises(ValueError):
        sa.sa_cache_reserve(t["pool"], t["table"], t["lens"], t["refs"], t["refs"], page=16)
    with pytest.raises(ValueError):
        sa.sa_cache_reserve(t["pool"], t["table"], t["lens"], t["refs"], t["lens"], page=48)
    with pytest.raises(ValueError):
        sa.sa_cache_compact(t["pool"], t["table"], t["refs"][:2])


# The statement itself: what the formats are, and that rounding is to the nearest.
def test_reference_formats():
    assert list(ref.E4M3[:2]) == [0, 2.0 ** -9] and ref.E4M3[8] == 2.0 ** -6 and ref.E4M3[126] == 448
    assert list(ref.nearest(np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 9.0]), ref.E2M1)) == [0, 2, 2, 4, 4, 6, 6, 7]
    x = np.linspace(-40, 40, 1600).reshape(2, 5, 160)
    y = ref.rounded(x, 0.25)
    top = np.abs(x).reshape(2, 5, 10, 16).max(-1)
    # half a step of a code is at most 1/6 of the largest, and the scale itself is off by at most 1/16
    assert (np.abs(x - y).reshape(2, 5, 10, 16).max(-1) <= top * (1 / 6) * (1 + 1 / 8)).all()
    x[0, 0, 3] = np.nan
    assert np.isnan(ref.rounded(x, 0.25)[0, 0, :16]).all() and np.isfinite(ref.rounded(x, 0.25)[0, 0, 16:]).all()


def test_reference_books():
    b = ref.Books([[3, 1, -1], [-1] * 3, [-1] * 3], [20, 0, 0], [0, 1, 0, 1, 0], 16)
    b.fork([0, 0], [1, 2])
    assert b.refs == [0, 3, 0, 3, 0] and b.table[2] == [3, 1, -1]
    assert b.reserve([1, 1, 13]) == [1, 1, 0]       # three free pages: the last slot needs two more
    assert b.table == [[3, 0, -1], [3, 2, -1], [3, 1, -1]] and b.pool == [1, 1, 1, 3, 4]
    b.free([0])
    assert b.compact() == 3 and b.refs == [2, 1, 1, 0, 0] and b.table[1] == [0, 2, -1]
