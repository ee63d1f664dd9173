"""The 4-bit cache on the GPU against float64: quantising, reading, attention, the books, and a run of all.

Tolerances.  Stored values are compared for equality: every rounding decision is exact.  Attention: y is
rounded once to its type (bf16 2^-8, fp32 2^-24 of the value), and the probabilities' products are summed
with errors relative to sum p |v|, at most the largest |v| of the head: fp32 sums, scores off by 2^-21 of
their size each way and, in bf16 calls, p rounded to 11 bits (2^-11).  So bf16: 2^-8 |y| + 2^-10 max|v|; fp32: the
score's error e changes p by a factor 1 + e: 2^-20 (1 + max|score|) max|v|.  lse: 2^-20 (1 + max|score|) + 2^-20."""
import numpy as np
import pytest
import torch

import cache_ref as ref
from paper_2604_00754_b200 import binding as sa

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def f64(t):
    return t.detach().double().cpu().numpy()


def filled(rng, B, Hkv, d, P, held, layers=1, garbage=0xff, spare=2, row=None):
    """A cache whose slot b holds held[b] pages, every byte of the pool `garbage` (0xff: NaN scales)."""
    need = [int(n) for n in held]
    row = max(max(need), 1) if row is None else row
    pages = sum(need) + spare
    ids = rng.permutation(pages)
    table = np.full((B, row), -1)
    for b, n in enumerate(need):
        table[b, :n], ids = ids[:n], ids[n:]
    refs = np.zeros(pages)
    refs[table[table >= 0]] = 1
    pool = torch.full((layers, pages, Hkv, 2, P * (d // 2 + d // 16)), garbage, dtype=torch.uint8, device="cuda")
    return pool, ints(table), ints(refs)


def attend_case(rng, dt, B, T, Hq, Hkv, d, P, lens, causal=True, w=0, counts=None, slots=None, k_scale=2.0 ** -4,
                v_scale=2.0 ** -3, scale=0.0, bnhd=False, spread=1.0, extra=0):
    """Packs random K, V in numpy, runs the kernel, compares with the float64 statement."""
    lens = np.asarray(lens)
    S = len(lens)
    slot_of = np.arange(B) if slots is None else np.asarray(slots)
    end = lens + (T if causal else 0)
    pool, table, _ = filled(rng, S, Hkv, d, P, -(-end // P) + extra)
    host, tab = pool.cpu().numpy(), table.cpu().numpy()
    kv = []
    for s in range(S):
        sides = []
        for side, t in ((0, k_scale), (1, v_scale)):
            x = rng.standard_normal((Hkv, end[s], d)) * (spread if side == 0 else 1.0)
            c, f = ref.quantise(x, t)
            for i in range(end[s]):
                for h in range(Hkv):
                    ref.pack(host[0], tab[s, i // P], h, side, i % P, c[h, i].astype(np.uint8), f[h, i].astype(np.uint8), P)
            sides.append(ref.values(c, f, t))
        kv.append(sides)
    pool.copy_(torch.from_numpy(host))
    q = torch.from_numpy(rng.standard_normal((B, T, Hq, d) if bnhd else (B, Hq, T, d))).to(DT[dt]).cuda()
    q = q.transpose(1, 2) if bnhd else q
    y = torch.full((B, Hq, T, d), 7.0, dtype=DT[dt], device="cuda")
    lse = torch.full((B, Hq, T), 7.0, device="cuda")
    sa.sa_cache_attend(pool, table, ints(lens), q, w=w, flags=sa.CAUSAL if causal else 0, scale=scale, y=y, lse=lse,
                       slots=None if slots is None else ints(slots), counts=None if counts is None else ints(counts),
                       k_scale=k_scale, v_scale=v_scale)
    assert sa.sa_read_status() == 0
    y, lse = f64(y), f64(lse)
    for b in range(B):
        n = T if counts is None else counts[b]
        k, v = kv[slot_of[b]]
        sc = scale or d ** -0.5
        wy, wl = ref.attend(f64(q[b])[:, :n], k, v, lens[slot_of[b]], sc, causal, w)
        size = np.abs(f64(q[b])).sum(-1).max(initial=0) * np.abs(k).max(initial=0) * sc
        top = np.abs(v).max(initial=0)
        tol = 2.0 ** -8 * np.abs(wy) + 2.0 ** -10 * top if dt == "bf16" else 2.0 ** -20 * (1 + min(size, 64)) * top
        assert (np.abs(y[b, :, :n] - wy) <= tol).all(), (b, np.abs(y[b, :, :n] - wy).max())
        seen = np.isfinite(wl)
        assert np.array_equal(np.isneginf(lse[b, :, :n]), ~seen) and (y[b, :, :n][~seen] == 0).all()
        assert (np.abs(lse[b, :, :n][seen] - wl[seen]) <= 2.0 ** -20 * (2 + min(size, 64))).all()
        assert (y[b, :, n:] == 7).all() and (lse[b, :, n:] == 7).all()       # rows behind the counts
    return y


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [16, 48, 64, 80, 128, 192, 256])
def test_attend_head_dimensions(dt, d):
    rng = np.random.default_rng(d)
    attend_case(rng, dt, 2, 1, 4, 2, d, 16, [0, 130])
    attend_case(rng, dt, 2, 3, 6, 2, d, 32, [65, 7])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
def test_attend_lengths_and_pages(dt, P):
    # zero, one, and both sides of units, steps and pages; every page's rest holds NaN
    lens = [0, 1, 14, 15, 16, 17, 31, 62, 63, 64, 65, 126, 127, 128, 129, 300]
    attend_case(np.random.default_rng(P), dt, len(lens), 1, 8, 2, 64, P, lens)
    attend_case(np.random.default_rng(P + 1), dt, len(lens), 2, 2, 2, 64, P, lens, causal=False)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,T", [(1, 1, 1), (5, 1, 1), (16, 2, 1), (8, 1, 2), (9, 3, 5), (32, 2, 1), (24, 8, 3),
                                      (4, 4, 17), (40, 1, 3), (2, 2, 70)])
def test_attend_head_layouts_and_rows(dt, Hq, Hkv, T):
    rng = np.random.default_rng(Hq * 100 + T)
    attend_case(rng, dt, 2, T, Hq, Hkv, 128, 64, [90, 2], bnhd=True)
    attend_case(rng, dt, 2, T, Hq, Hkv, 64, 16, [50, 0], causal=False, scale=0.3)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("w", [1, 2, 15, 16, 17, 64, 100, 1 << 30])
@pytest.mark.parametrize("causal", [True, False])
def test_attend_windows(dt, w, causal):
    # without the new tokens' keys a narrow window leaves the later rows empty
    attend_case(np.random.default_rng(w % 1000), dt, 3, 9, 4, 2, 64, 16, [200, 0, 37], causal=causal, w=w)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 80])
def test_attend_slots_counts_and_row_stride(dt, d):
    rng = np.random.default_rng(5)
    attend_case(rng, dt, 3, 4, 4, 2, d, 32, [70, 5, 0, 33, 128], slots=[4, 0, 2], counts=[4, 0, 1], extra=1)
    attend_case(rng, dt, 4, 3, 4, 1, d, 32, [70, 5], slots=[1, 1, 0, 1], counts=[3, 2, 1, 0])   # one slot, read twice


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("B,lens", [(1, [9000]), (3, [5000, 0, 4000]), (150, None)])
def test_attend_long_and_many(dt, B, lens):
    """Segments cut over many shares, and many segments in one; each also against a batch of its own."""
    rng = np.random.default_rng(B)
    lens = rng.integers(0, 90, B) if lens is None else lens
    attend_case(rng, dt, B, 1, 4, 2, 64, 64, lens, spread=3.0)


@pytest.mark.parametrize("d", [64, 128, 256, 48])
def test_attend_same_bits_again_and_from_other_memory(d):
    """Two calls, a captured and replayed one, and one on another stream with its own workspace: one result."""
    rng = np.random.default_rng(1)
    pool, table, _ = filled(rng, 5, 2, d, 32, [40, 3, 1, 20, 33])
    lens = ints([1270, 70, 5, 600, 1040])
    k, v = (torch.randn(5, 2, 1270, d, device="cuda").bfloat16() for _ in range(2))
    sa.sa_cache_append(pool, table, ints([0] * 5), k, v, counts=lens)
    q = torch.randn(5, 8, 2, d, device="cuda").bfloat16()
    args = (pool, table, lens, q)
    want = sa.sa_cache_attend(*args, flags=0, want_lse=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = sa.sa_cache_attend(*args, flags=0, want_lse=True)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = sa.sa_cache_attend(*args, flags=0, want_lse=True)
    got[0].fill_(3)
    g.replay()
    g.replay()
    again = sa.sa_cache_attend(*args, flags=0, want_lse=True)
    for x in (other, got, again):
        assert torch.equal(x[0], want[0]) and torch.equal(x[1], want[1])
    # lengths are read at replay, not at capture
    lens.copy_(ints([3, 70, 0, 599, 900]))
    g.replay()
    now = sa.sa_cache_attend(*args, flags=0, want_lse=True)
    assert torch.equal(got[0], now[0]) and torch.equal(got[1], now[1])
    assert sa.sa_read_status() == 0


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 80, 128, 256])
def test_attend_values_that_are_not_finite(d, dt):
    """A NaN or an infinity reaches the rows that see it and no others."""
    rng = np.random.default_rng(2)
    pool, table, _ = filled(rng, 2, 2, d, 16, [8, 8])
    zero = ints([0, 0])
    k, v = (torch.randn(2, 2, 128, d, device="cuda") for _ in range(2))
    q = torch.randn(2, 4, 40, d, device="cuda").to(DT[dt])
    sa.sa_cache_append(pool, table, zero, k, v)
    lens = ints([60, 60])
    clean = sa.sa_cache_attend(pool, table, lens, q)
    v[0, 0, 70, 3] = float("nan")
    v[1, 1, 90, 3] = float("inf")
    k[1, 0, 80, 5] = float("-inf")
    sa.sa_cache_append(pool, table, zero, k, v)
    y = sa.sa_cache_attend(pool, table, lens, q)
    for b, heads, first in ((0, (0, 1), 10), (1, (2, 3), 30), (1, (0, 1), 20)):
        for h in heads:
            part = y[b, h, first:]
            block = part[:, :16] if (b, h // 2) != (1, 0) else part
            assert block.isnan().all()
            assert torch.equal(y[b, h, :first], clean[b, h, :first])
    assert torch.equal(y[0, 2:], clean[0, 2:])
    q[0, 1, 4] = float("inf")
    y = sa.sa_cache_attend(pool, table, lens, q)
    assert y[0, 1, 4].isnan().all() and torch.equal(y[0, 1, :4], clean[0, 1, :4]) and torch.equal(y[0, 2:], clean[0, 2:])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("size", [1e-30, 1e-4, 1.0, 300.0, 1e20])
def test_attend_sizes_of_queries(dt, size):
    """Queries of any size: the scores stay the same where the scale takes it back."""
    rng = np.random.default_rng(3)
    for d in (64, 80):
        pool, table, _ = filled(rng, 1, 1, d, 16, [10])
        k, v = (torch.randn(1, 1, 150, d, device="cuda") for _ in range(2))
        sa.sa_cache_append(pool, table, ints([0]), k, v)
        q = torch.randn(1, 4, 1, d, device="cuda").to(DT[dt])
        e = float(2.0 ** np.round(np.log2(size)))        # powers of two: exact in both types
        one = sa.sa_cache_attend(pool, table, ints([150]), q, flags=0, scale=0.2, want_lse=True)
        two = sa.sa_cache_attend(pool, table, ints([150]), (q.float() * e).to(DT[dt]), flags=0, scale=0.2 / e, want_lse=True)
        # the scale itself may round once more: 2^-23 of the scores
        assert (one[1] - two[1]).abs().max() < 2.0 ** -20 * (1 + one[1].abs().max())
        assert (one[0].float() - two[0].float()).abs().max() <= 2.0 ** (-7 if dt == "bf16" else -18) * v.abs().max()


@pytest.mark.parametrize("d", [64, 128, 80])
def test_attend_fp32_sums_over_many_keys(d):
    """fp32 over 6000 keys, by so many sequences (of the same pages) that one CTA goes through all keys of a head.

    Errors of keys are independent: 2^-22 |score| of the score (|score| < 8) and 2^-22 of the exponential, below 2^-19
    of each term p v, and the running sum is rounded, not cut off: relative to the sum, whose terms have both signs as
    the errors have, 2^-19 too."""
    n, B, Hkv = 6000, 120, 4
    pool, table, _ = filled(np.random.default_rng(3), 1, Hkv, d, 128, [-(-n // 128)])
    k, v = torch.randn(1, Hkv, n, d, device="cuda") * 0.5, torch.randn(1, Hkv, n, d, device="cuda")
    sa.sa_cache_append(pool, table, ints([0]), k, v)
    sa.sa_cache_read(pool, table, k, v)
    q = torch.randn(B, 2 * Hkv, 1, d, device="cuda")
    y = sa.sa_cache_attend(pool, table.expand(B, -1).contiguous(), ints([n] * B), q, flags=0).double()
    s = (q.double().view(B, Hkv, 2, d) @ k.double().transpose(2, 3)) / d ** 0.5
    want = (s.softmax(-1) @ v.double()).view(B, 2 * Hkv, 1, d)
    assert (y - want).norm() <= 2.0 ** -19 * want.norm()


def test_attend_on_two_streams_at_once():
    """Calls that overlap, each with a workspace of its own, do not touch each other."""
    rng = np.random.default_rng(8)
    jobs, streams = [], [torch.cuda.Stream() for _ in range(2)]
    for d, dt in ((128, "bf16"), (64, "f32")):
        pool, table, _ = filled(rng, 7, 2, d, 64, [30, 1, 2, 17, 40, 5, 8])
        lens = ints([1900, 3, 100, 1024, 2500, 300, 512])
        k, v = (torch.randn(7, 2, 2500, d, device="cuda").to(DT[dt]) for _ in range(2))
        sa.sa_cache_append(pool, table, ints([0] * 7), k, v, counts=lens)
        q = torch.randn(7, 8, 3, d, device="cuda").to(DT[dt])
        jobs.append((pool, table, lens, q, sa.sa_cache_attend(pool, table, lens, q, flags=0)))
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(sa.sa_cache_attend(*jobs[i][:4], flags=0))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(y, jobs[i][4]) for y in got[i])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_attend_views(dt):
    """q and y as parts of wider tensors: rows 16 bytes apart from others' values, which stay."""
    rng = np.random.default_rng(9)
    pool, table, _ = filled(rng, 3, 2, 64, 16, [3, 1, 5])
    k, v = (torch.randn(3, 2, 70, 64, device="cuda").to(DT[dt]) for _ in range(2))
    lens = ints([40, 9, 70])
    sa.sa_cache_append(pool, table, ints([0, 0, 0]), k, v, counts=lens)
    wide = torch.randn(3, 2, 12 * 64 + 8, device="cuda").to(DT[dt])          # a fused projection's output
    q = wide[:, :, 8:8 + 8 * 64].view(3, 2, 8, 64).transpose(1, 2)
    out = torch.full((3, 2, 8, 72), 7.0, dtype=DT[dt], device="cuda")
    y = out[..., :64].transpose(1, 2)
    sa.sa_cache_attend(pool, table, lens, q, flags=0, y=y)
    assert torch.equal(y, sa.sa_cache_attend(pool, table, lens, q.contiguous(), flags=0)) and (out[..., 64:] == 7).all()
    one = sa.sa_cache_attend(pool, table, lens, q[:, :, :1], flags=0)        # one token: any token stride
    assert torch.equal(one, y[:, :, :1])
    assert sa.sa_read_status() == 0


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 80, 128, 256])
def test_attend_scores_of_any_size(d, dt):
    """Scores up to 1e36, all of one sign: the largest takes everything, whatever its sign."""
    rng = np.random.default_rng(10)
    pool, table, _ = filled(rng, 1, 1, d, 16, [19])
    k, v = torch.randn(1, 1, 300, d, device="cuda").abs(), torch.randn(1, 1, 300, d, device="cuda")
    q = (torch.randn(1, 4, 2, d, device="cuda").abs() * 1e34).to(DT[dt])
    for sign in (1, -1):
        sa.sa_cache_append(pool, table, ints([0]), sign * k, v)
        ks, vs = torch.empty_like(k), torch.empty_like(v)
        sa.sa_cache_read(pool, table, ks, vs)
        s = f64(q)[0] @ f64(ks)[0, 0].T * d ** -0.5
        y, lse = sa.sa_cache_attend(pool, table, ints([300]), q, flags=0, want_lse=True)
        assert np.array_equal(f64(y)[0], f64(vs.to(DT[dt]))[0, 0][s.argmax(-1)])
        assert (np.abs(f64(lse)[0] - s.max(-1)) <= 2.0 ** -20 * np.abs(s).max(-1)).all()


# ---- append and read

def hard_values(rng, shape, dt):
    """Values on and next to every border, tiny, large, zero and signed ones."""
    x = rng.standard_normal(shape)
    flat = x.reshape(-1, 16)
    for i in range(0, len(flat), 3):
        s = ref.E4M3[rng.integers(1, 127)] / 16
        flat[i, 0] = 6 * s
        flat[i, 1:8] = np.array([.25, .75, 1.25, 1.75, 2.5, 3.5, 5]) * s * rng.choice([-1, 1], 7)
    for i in range(1, len(flat), 7):
        flat[i] *= 2.0 ** rng.integers(-40, 30)
    flat[2] = 0
    if len(flat) > 12:
        m = (ref.E4M3[20:36] + ref.E4M3[21:37]) / 2 * 6 / 16       # on the border between two scales
        flat[5], flat[6] = 0, 0
        flat[5, 3], flat[6, 9] = m[0], -m[1]
    t = torch.from_numpy(x).to(DT[dt])
    if dt == "f32":                                                # and the neighbours of borders
        bits = t.view(torch.int32)
        near = torch.from_numpy(rng.integers(-1, 2, shape).astype(np.int32))
        t = torch.where(t == 0, t, (bits + near).view(torch.float32))
    return t.cuda()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("Hkv,d,P,T,bnhd", [(1, 16, 16, 1, False), (2, 64, 32, 77, True), (3, 80, 128, 130, False),
                                            (8, 128, 64, 200, True), (1, 256, 16, 33, False), (2, 48, 64, 9, True)])
@pytest.mark.parametrize("scales", [(2.0 ** -4, 2.0 ** -6), (1.0, 2.0 ** 3)])
def test_append_and_read_are_exact(dt, Hkv, d, P, T, bnhd, scales):
    rng = np.random.default_rng(d + T)
    B, S, layers = 3, 5, 2
    lens = np.array([0, 3, P - 1, 2 * P, 11])
    counts = [T, 0, max(1, T // 2)]
    slots = [2, 0, 4]
    pool, table, _ = filled(rng, S, Hkv, d, P, -(-(lens + T) // P), layers=layers, garbage=0xA5)
    before = pool.clone()
    shape = (B, T, Hkv, d) if bnhd else (B, Hkv, T, d)
    k, v = (hard_values(rng, shape, dt) for _ in range(2))
    if bnhd:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    kw = dict(slots=ints(slots), counts=ints(counts), k_scale=scales[0], v_scale=scales[1], layer=1)
    sa.sa_cache_append(pool, table, ints(lens), k, v, **kw)
    want, tab = before.cpu().numpy(), table.cpu().numpy()
    for b, s in enumerate(slots):
        for side, x, t in ((0, k, scales[0]), (1, v, scales[1])):
            c, f = ref.quantise(f64(x[b])[:, :counts[b]], t)
            for i in range(counts[b]):
                pos = lens[s] + i
                for h in range(Hkv):
                    ref.pack(want[1], tab[s, pos // P], h, side, pos % P, c[h, i].astype(np.uint8), f[h, i].astype(np.uint8), P)
    # every byte, those of other tokens, slots and the other layer among them (the sign of a zero aside)
    got = pool.cpu().numpy()
    assert np.array_equal(got[0], want[0])
    at = P * d // 2
    zero = lambda x: np.where(x & 7, x, 0)  # noqa: E731
    for half in (got[1][..., :at] & 15, want[1][..., :at] & 15), (got[1][..., :at] >> 4, want[1][..., :at] >> 4):
        assert np.array_equal(zero(half[0]), zero(half[1]))
    assert np.array_equal(got[1][..., at:], want[1][..., at:])
    ko, vo = (torch.full_like(x, 7.0) for x in (k, v))
    sa.sa_cache_read(pool, table, ko, vo, starts=ints(lens[slots]), **kw)
    for b in range(B):
        for x, o, t in ((k, ko, scales[0]), (v, vo, scales[1])):
            assert np.array_equal(f64(o[b])[:, :counts[b]], ref.rounded(f64(x[b])[:, :counts[b]], t))
            assert (o[b][:, counts[b]:] == 7).all()
    assert sa.sa_read_status() == 0


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_append_of_values_that_are_not_finite_or_too_large(dt):
    pool, table, _ = filled(np.random.default_rng(0), 1, 1, 64, 16, [1])
    k = torch.ones(1, 1, 4, 64, dtype=DT[dt], device="cuda")
    k[0, 0, 0, 5], k[0, 0, 1, 20], k[0, 0, 2, 40] = float("nan"), float("-inf"), -3e38
    sa.sa_cache_append(pool, table, ints([0]), k, k, k_scale=1.0, v_scale=2.0 ** -4)
    ko, vo = torch.empty_like(k), torch.empty_like(k)
    sa.sa_cache_read(pool, table, ko, vo, k_scale=1.0, v_scale=2.0 ** -4)
    for o, t in ((ko, 1.0), (vo, 2.0 ** -4)):
        assert np.array_equal(f64(o), ref.rounded(f64(k), t), equal_nan=True)
        assert o[0, 0, 0, :16].isnan().all() and o[0, 0, 1, 16:32].isnan().all() and o[0, 0, 2, 40] == -2688 * t


# ---- what only the device can see

def test_bad_books_are_recorded_and_skipped():
    rng = np.random.default_rng(4)
    for d in (64, 80):
        pool, table, refs = filled(rng, 2, 1, d, 16, [3, 2], garbage=0)
        k = torch.randn(2, 1, 4, d, device="cuda")
        q = torch.randn(2, 2, 1, d, device="cuda")
        good = table.clone()
        sa.sa_cache_append(pool, good, ints([0, 0]), torch.randn(2, 1, 30, d, device="cuda"), torch.randn(2, 1, 30, d, device="cuda"))
        before = pool.clone()
        y0 = sa.sa_cache_attend(pool, good, ints([16, 16]), q, flags=0)

        def recorded():
            assert sa.sa_read_status() == 8 and sa.sa_read_status() == 0

        table[0, 1] = 99
        for t, lens, kw in ((good, [0, 0], dict(slots=ints([5, -1]))), (good, [0, 0], dict(counts=ints([-1, 5]))),
                            (good, [-1, 1 << 30], {}), (good, [48, 46], dict(counts=ints([1, 4])))):
            sa.sa_cache_append(pool, t, ints(lens), k, k, **kw)
            recorded()
        # slot 1 holds two pages of three: tokens 32 and on have none
        assert torch.equal(pool, before)
        for lens, kw in (([0, 0], dict(slots=ints([2, 1 << 20]))), ([0, 0], dict(counts=ints([2, -7]))),
                         ([-5, 49], {}), ([48, 48], {})):
            y = torch.full_like(q, 7.0)
            sa.sa_cache_attend(pool, good, ints(lens), q, y=y, **kw)
            recorded()
            if lens != [48, 48]:
                assert (y == 7).all()
        # keys without a page are hidden: the first page alone counts
        y = sa.sa_cache_attend(pool, table, ints([30, 30]), q, flags=0)
        recorded()
        assert torch.equal(y[0], y0[0])
        out = torch.full_like(k, 7.0)
        sa.sa_cache_read(pool, good, out, out.clone(), starts=ints([-3, 47]))
        recorded()
        assert (out == 7).all()


def test_bad_fork_free_reserve_are_recorded():
    rng = np.random.default_rng(6)

    def state():
        pool, table, refs = filled(rng, 6, 1, 16, 16, [2, 1, 0, 0, 0, 0], row=3, spare=3)
        return pool, table, ints([20, 16, 0, 0, 0, 0]), refs

    for parents, children, done in (([0, 0], [2, 2], [2]), ([0, 1], [2, 1], [2]), ([0], [0], []), ([0, 9], [6, 3], []),
                                    ([0, 1], [1, 2], [2]), ([0, 2], [2, 3], [3]), ([-1], [3], [])):
        pool, table, lens, refs = state()
        t0, l0, r0 = table.clone(), lens.clone(), refs.clone()
        sa.sa_cache_fork(table, lens, refs, ints(parents), ints(children), page=16)
        assert sa.sa_read_status() == 8
        for s in range(6):
            if s not in done:
                assert torch.equal(table[s], t0[s]) and lens[s] == l0[s]
        forked = [parents[children.index(s)] for s in done]
        for a, s in zip(forked, done):
            assert lens[s] == l0[a]
        assert int(refs.sum()) == int(r0.sum()) + sum(int((t0[a] >= 0).sum()) for a in forked)
    pool, table, lens, refs = state()
    lens[0] = 40                                               # three pages' length, two pages
    sa.sa_cache_fork(table, lens, refs, ints([0]), ints([2]), page=16)
    assert sa.sa_read_status() == 8 and lens[2] == 0 and (table[2] == -1).all()
    pool, table, lens, refs = state()
    sa.sa_cache_free(table, lens, refs, ints([0, 0, 7, -1]))
    assert sa.sa_read_status() == 8 and int(refs.sum()) == 1 and (table[0] == -1).all() and int(refs.min()) == 0
    pool, table, lens, refs = state()
    table[0, 1] = 77
    got = sa.sa_cache_reserve(pool, table, lens, refs, ints([1, 1, -2, 0, 16, 0]), page=16)
    assert sa.sa_read_status() == 8 and got.tolist() == [0, 1, 0, 1, 1, 1]
    pool, table, lens, refs = state()
    got = sa.sa_cache_reserve(pool, table, lens, refs, ints([29, 1, 0, 0, 0, 33]), page=16)   # rows too short: no error
    assert sa.sa_read_status() == 0 and got.tolist() == [0, 1, 1, 1, 1, 0]      # three are free: one and three do not fit


# ---- the books against lists

@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("layers,Hkv,d,P,S,row,pages", [(3, 2, 32, 16, 12, 6, 60), (1, 1, 16, 64, 40, 9, 300),
                                                        (2, 3, 128, 128, 5, 40, 130), (1, 1, 16, 16, 1500, 4, 5000),
                                                        (1, 2, 16, 16, 70, 90, 4000)])
def test_books_follow_the_lists(seed, layers, Hkv, d, P, S, row, pages):
    rng = np.random.default_rng(seed)
    pool = torch.randint(0, 256, (layers, pages, Hkv, 2, P * (d // 2 + d // 16)), dtype=torch.uint8, device="cuda")
    first = pool.clone()
    table, lens, refs = ints(np.full((S, row), -1)), ints([0] * S), ints([0] * pages)
    b = ref.Books(table.tolist(), lens.tolist(), refs.tolist(), P)

    def same():
        assert table.tolist() == b.table and refs.tolist() == b.refs and lens.tolist() == b.lens
        used = torch.tensor([p for p, r in enumerate(b.refs) if r > 0], dtype=torch.long, device="cuda")
        label = torch.tensor(b.pool, dtype=torch.long, device="cuda")
        assert torch.equal(pool[:, used], first[:, label[used]])

    for _ in range(8):
        add = rng.integers(0, row * P // 2, S) * (rng.random(S) < 0.6)
        got = sa.sa_cache_reserve(pool, table, lens, refs, ints(add), page=P)
        assert got.tolist() == b.reserve(add.tolist())
        same()
        grown = np.where(got.cpu().numpy() == 1, add * (rng.random(S) < 0.8), 0)     # some room stays unused
        lens += ints(grown)
        b.lens = lens.tolist()
        empty = [s for s in range(S) if b.lens[s] == 0 and b.table[s][0] < 0]
        others = [s for s in range(S) if s not in set(empty)]
        if empty and others:
            kids = list(rng.permutation(empty)[:4])
            dads = [int(x) for x in rng.choice(others, len(kids))]
            sa.sa_cache_fork(table, lens, refs, ints(dads), ints(kids), page=P)
            b.fork(dads, [int(x) for x in kids])
            same()
        gone = [int(x) for x in rng.permutation(S)[:rng.integers(0, S // 3 + 1)]]
        sa.sa_cache_free(table, lens, refs, ints(gone))
        b.free(gone)
        if rng.random() < 0.5:
            some = int(rng.integers(0, S))                       # a length taken back: pages behind it stay
            lens[some] = b.lens[some] = b.lens[some] // 2
        same()
        live = sa.sa_cache_compact(pool, table, refs)
        assert live.tolist() == [b.compact()]
        same()
    assert sa.sa_read_status() == 0


def test_reserve_without_pages_and_empty_lists():
    pool, table, refs = filled(np.random.default_rng(0), 3, 1, 16, 16, [1, 1, 0], row=4, spare=1)
    lens = ints([16, 16, 0])
    got = sa.sa_cache_reserve(pool, table, lens, refs, ints([1, 17, 1]), page=16)
    assert got.tolist() == [1, 0, 0] and int((refs == 0).sum()) == 0        # the second did not fit, so none behind it
    got = sa.sa_cache_reserve(pool, table, lens, refs, ints([0, 0, 0]), page=16)
    assert got.tolist() == [1, 1, 1]
    sa.sa_cache_free(table, lens, refs, ints([]))
    sa.sa_cache_fork(table, lens, refs, ints([]), ints([]), page=16)
    assert sa.sa_cache_compact(pool, table, refs).item() == 3 and sa.sa_read_status() == 0


# ---- far offsets

@pytest.mark.parametrize("d", [128, 96])
def test_pages_past_32_bits(d):
    """Pages whose bytes lie beyond 2^32 of the pool: append, read, attend and compact find them."""
    P, Hkv = 128, 8
    each = Hkv * 2 * P * (d // 2 + d // 16)
    pages = (9 << 29) // each + 4
    pool = torch.zeros(1, pages, Hkv, 2, each // (2 * Hkv), dtype=torch.uint8, device="cuda")
    assert pool.numel() > 1 << 32
    table, refs, lens = ints([[pages - 1, 0, pages - 3]]), torch.zeros(pages, dtype=torch.int32, device="cuda"), ints([300])
    refs[[pages - 1, 0, pages - 3]] = 1
    k, v = (torch.randn(1, Hkv, 300, d, device="cuda").bfloat16() for _ in range(2))
    sa.sa_cache_append(pool, table, ints([0]), k, v)
    q = torch.randn(1, 8, 1, d, device="cuda").bfloat16()
    y = sa.sa_cache_attend(pool, table, lens, q, flags=0)
    near = torch.zeros(1, 3, Hkv, 2, each // (2 * Hkv), dtype=torch.uint8, device="cuda")
    sa.sa_cache_append(near, ints([[0, 1, 2]]), ints([0]), k, v)
    assert torch.equal(y, sa.sa_cache_attend(near, ints([[0, 1, 2]]), lens, q, flags=0))
    assert torch.equal(pool[0, [pages - 1, 0, pages - 3]].sum((1, 2, 3)), near[0].sum((1, 2, 3)))
    assert sa.sa_cache_compact(pool, table, refs).item() == 3
    assert table.tolist() == [[2, 0, 1]] and torch.equal(pool[0, [2, 0, 1]], near[0])
    assert torch.equal(y, sa.sa_cache_attend(pool, table, lens, q, flags=0)) and sa.sa_read_status() == 0
