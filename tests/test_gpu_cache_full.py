"""Steps of the 4-bit cache while the pool is full: who has no room stays as it was, and nobody else changes."""
import numpy as np
import pytest
import torch

import cache_ref as ref
from paper_2604_00754_b200 import binding as sa
from paper_2604_00754_b200.cache import KVCache

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("d,dt", [(64, torch.bfloat16), (80, torch.float32)])
def test_append_leaves_pages_that_others_hold(d, dt):
    """One free page for three holders of a part-full one: without their counts the two others write nothing."""
    c = KVCache(2, 2, d, 4, 48, pages=4, page=16)
    k, v = (torch.randn(4, 2, 20, d, device="cuda").to(dt) for _ in range(2))
    assert c.reserve(ints([20, 0, 0, 5])).tolist() == [1, 1, 1, 1]
    for layer in range(2):
        c.append(layer, k, v, counts=ints([20, 0, 0, 5]))
    c.advance(ints([20, 0, 0, 5]))
    c.fork(ints([0, 0]), ints([1, 2]))
    assert c.reserve(ints([1, 1, 1, 1])).tolist() == [1, 0, 0, 1]
    pool, table = c.pool.clone(), c.table.clone()
    c.append(1, k[:, :, :1], v[:, :, :1])
    assert sa.sa_read_status() == 8 and sa.sa_read_status() == 0
    shared = int(table[1, 1])
    assert int(table[2, 1]) == shared and int(c.refs[shared]) == 2
    assert torch.equal(c.pool[:, shared], pool[:, shared]) and torch.equal(c.pool[0], pool[0])
    for s in (0, 3):                                        # those that have room did write
        page = int(table[s, int(c.lens[s]) // 16])
        assert not torch.equal(c.pool[1, page], pool[1, page])
    # what the books do not name is what a caller without them may write
    sa.sa_cache_append(c.pool, c.table, c.lens, k[:1, :, :1], v[:1, :, :1], slots=ints([1]))
    assert sa.sa_read_status() == 0 and not torch.equal(c.pool[0, shared], pool[0, shared])


@pytest.mark.parametrize("chunk,pages", [(1, 7), (3, 9)])
def test_a_captured_step_goes_on_through_a_full_pool(chunk, pages):
    """Beams in one graph until the pool is full, and on after one left; tokens, books and y against lists."""
    d, Hq, Hkv, S, P = 64, 4, 2, 5, 16
    c = KVCache(1, Hkv, d, S, 112, pages=pages, page=P)
    c.pool.fill_(0)
    k, v, q = (torch.zeros(S, h, chunk, d, dtype=torch.bfloat16, device="cuda") for h in (Hkv, Hkv, Hq))
    slots, add = ints([3, 0, 4, 1, 2]), ints([0] * S)
    y, got = torch.zeros_like(q), ints([0] * S)

    def step():
        room = c.reserve(add)
        new = add * room
        counts = new[slots]
        c.append(0, k, v, slots, counts)
        c.attend(0, q, slots, counts, y=y)
        c.advance(new)
        got.copy_(room)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                              # warm-up: nobody adds anything
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    books = ref.Books([[-1] * 7 for _ in range(S)], [0] * S, [0] * pages, P)
    kept = {s: (np.zeros((Hkv, 0, d)), np.zeros((Hkv, 0, d))) for s in range(S)}
    refused = 0
    for i in range(40):
        if i == 10:
            c.fork(ints([0, 1]), ints([2, 3]))
            books.fork([0, 1], [2, 3])
            kept[2], kept[3] = kept[0], kept[1]
        if i == 32:
            c.free(ints([1, 2]))
            books.free([1, 2])
            kept[1] = kept[2] = (np.zeros((Hkv, 0, d)),) * 2
        live = [0, 1] if i < 10 else [0, 1, 2, 3] if i < 32 else [0, 3, 4]
        want = [chunk if s in live else 0 for s in range(S)]
        add.copy_(ints(want))
        for t in (k, v, q):
            t.normal_()
        y.fill_(7.0)
        g.replay()
        room = books.reserve(want)
        refused += room.count(0)
        lens = list(books.lens)
        books.lens = [n + w * r for n, w, r in zip(lens, want, room)]
        assert got.tolist() == room and c.lens.tolist() == books.lens
        assert c.table.tolist() == books.table and c.refs.tolist() == books.refs
        for b, s in enumerate(slots.tolist()):
            if not (want[s] and room[s]):
                assert (y[b] == 7).all()
                continue
            new = (np.concatenate([o, ref.rounded(x[b].double().cpu().numpy(), 2.0 ** -4)], 1) for o, x in zip(kept[s], (k, v)))
            kept[s] = tuple(new)
            out, _ = ref.attend(q[b].double().cpu().numpy(), *kept[s], lens[s], d ** -0.5, True, 0)
            tol = 2.0 ** -8 * np.abs(out) + 2.0 ** -10 * np.abs(kept[s][1]).max()
            assert (np.abs(y[b].double().cpu().numpy() - out) <= tol).all()
    assert refused > 5
    most = max(books.lens)
    ko, vo = (torch.zeros(S, Hkv, most, d, device="cuda") for _ in range(2))
    c.read(0, ko, vo, counts=c.lens)
    for s in range(S):
        for o, x in ((ko, kept[s][0]), (vo, kept[s][1])):
            assert np.array_equal(o[s, :, :books.lens[s]].double().cpu().numpy(), x)
    assert sa.sa_read_status() == 0


# ---- who stands in whose way

def test_a_row_that_is_too_short_takes_no_pages_and_stops_nobody():
    """Pages running out stops the slots behind; a short row, a bad number and a bad entry do not, and take none."""
    short, out = (sa.sa_cache_pool(1, 8, 1, 16, 16) for _ in range(2))
    table = ints([[0, -1], [1, 99], [2, -1], [3, -1], [4, -1]])
    refs, lens = ints([1, 1, 1, 1, 1, 0, 0, 0]), ints([16] * 5)
    got = sa.sa_cache_reserve(short, table, lens, refs, ints([17, 1, -1, 1, 16]), page=16)
    assert sa.sa_read_status() == 8 and got.tolist() == [0, 0, 0, 1, 1]
    assert table.tolist() == [[0, -1], [1, 99], [2, -1], [3, 5], [4, 6]] and refs.tolist() == [1] * 7 + [0]
    table, refs = ints([[0, -1, -1], [1, -1, -1], [2, -1, -1]]), ints([1] * 7 + [0])
    got = sa.sa_cache_reserve(out, table, ints([16] * 3), refs, ints([17, 1, 0]), page=16)
    assert sa.sa_read_status() == 0 and got.tolist() == [0, 0, 1] and refs.tolist() == [1] * 7 + [0]
