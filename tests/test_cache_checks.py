"""Refusals of the 4-bit cache's calls, each told by its own text or status."""
import ctypes

import pytest
import torch

from paper_2604_00754_b200 import binding as sa
from paper_2604_00754_b200.cache import KVCache
from test_cache_host import FAKE, OTHER, append, attend, cache


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
