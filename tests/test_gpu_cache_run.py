"""The cache's calls as a program uses them, together: prefill, decode steps, branches, packing, a captured step.

Tolerances as in test_gpu_cache: y in bf16 is off by at most 2^-8 of its value and 2^-10 of the largest |v|.  What is
rotated is rounded to bf16 before it is stored, and the reference starts from those rounded values."""
import numpy as np
import pytest
import torch

import cache_ref as ref
from paper_2604_00754_b200 import binding as sa
from paper_2604_00754_b200.cache import KVCache

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def f64(t):
    return t.detach().double().cpu().numpy()


def rotate(x, positions, table):
    """x [B,H,T,d] by positions [B,T]: token-major, as one sequence of B*T tokens."""
    B, H, T, d = x.shape
    flat = x.permute(0, 2, 1, 3).reshape(1, B * T, H, d).transpose(1, 2)
    cs, sn = (t[positions.flatten().long()].contiguous() for t in table)
    out = sa.sa_rope_apply(flat, flat, cs, sn, kv=True)
    return out.transpose(1, 2).reshape(B, T, H, d).transpose(1, 2)


class Model:
    """Two layers of attention; what stands in the cache as float64, per layer and sequence, beside it."""

    def __init__(self, d=64, Hq=8, Hkv=2, slots=6, page=32, layers=2, seed=0, pages=None):
        self.cache = KVCache(layers, Hkv, d, slots, 700, page=page, pages=pages)
        self.cache.pool.fill_(0xff)
        self.Hq, self.Hkv, self.d, self.layers, self.slots = Hq, Hkv, d, layers, slots
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.table = sa.sa_rope_table(1000, d)
        self.kv = {}

    def draw(self, B, H, T):
        # token-major, as a projection leaves them
        return torch.randn(B, T, H, self.d, generator=self.gen, device="cuda").bfloat16().transpose(1, 2)

    def step(self, slots, T, counts=None):
        """T new tokens of each listed slot through all layers; every y is checked."""
        c, B = self.cache, len(slots)
        counts = [T] * B if counts is None else counts
        ids, cnt = ints(slots), ints(counts)
        add = torch.zeros(self.slots, dtype=torch.int32, device="cuda")
        add[ids.long()] = cnt
        assert c.reserve(add).bool().all()
        positions = c.lens[ids.long()].unsqueeze(1) + torch.arange(T, device="cuda")
        for layer in range(self.layers):
            q = rotate(self.draw(B, self.Hq, T), positions, self.table)
            k = rotate(self.draw(B, self.Hkv, T), positions, self.table)
            v = self.draw(B, self.Hkv, T)
            c.append(layer, k, v, ids, cnt)
            y = f64(c.attend(layer, q, ids, cnt))
            lens = c.lens.tolist()
            for i, s in enumerate(slots):
                n = counts[i]
                old = self.kv.get((layer, s), (np.zeros((self.Hkv, 0, self.d)),) * 2)
                new = [np.concatenate([o, ref.rounded(f64(x[i])[:, :n], 2.0 ** -4)], 1) for o, x in zip(old, (k, v))]
                self.kv[layer, s] = tuple(new)
                want, _ = ref.attend(f64(q[i])[:, :n], *new, lens[s], self.d ** -0.5, True, 0)
                tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * np.abs(new[1]).max(initial=0)
                assert (np.abs(y[i, :, :n] - want) <= tol).all(), (layer, s)
        c.advance(add)

    def fork(self, parents, children):
        self.cache.fork(ints(parents), ints(children))
        for layer in range(self.layers):
            for a, b in zip(parents, children):
                self.kv[layer, b] = self.kv[layer, a]

    def free(self, slots):
        self.cache.free(ints(slots))
        for layer in range(self.layers):
            for s in slots:
                self.kv.pop((layer, s), None)


@pytest.mark.parametrize("d,page", [(64, 32), (128, 64), (80, 16), (256, 128)])
def test_prompts_steps_branches_and_packing(d, page):
    m = Model(d=d, page=page)
    m.step([0, 1, 2], 130, [130, 77, 0])        # prompts, one of them not yet there
    m.step([0, 1], 1)
    m.step([2, 0], 40, [40, 3])
    m.fork([0, 0, 1], [3, 4, 5])                # samples of one prompt
    m.step([3, 0, 4, 5, 1], 1)                  # all of them write: each on a page of its own
    m.step([4], 5)
    m.free([0, 1])
    live = m.cache.compact().item()
    assert live == int((m.cache.refs > 0).sum()) and int(m.cache.table.max()) < live
    m.step([3, 4, 5], 2)                        # on packed pages
    m.step([0], 20)                             # a new sequence in a slot that was used
    assert sa.sa_read_status() == 0


def test_prefill_fills_the_cache_and_goes_on():
    """SA prefill of a prompt, its K and V appended, single tokens after it."""
    n, d, Hq, Hkv, w = 300, 128, 8, 2, 64
    m = Model(d=d, Hq=Hq, Hkv=Hkv, slots=2, page=64, layers=1)
    q, k, v = m.draw(2, Hq, n), m.draw(2, Hkv, n), m.draw(2, Hkv, n)
    perm, inv = sa.sa_make_perm(3, 0, 2, n)
    y = sa.sa_forward_rope(q, k, v, perm, inv, *(t[:n] for t in m.table), w)
    kr = sa.sa_rope_apply(k, k, *(t[:n] for t in m.table), kv=True)
    add = ints([n, n])
    m.cache.reserve(add)
    m.cache.append(0, kr, v)
    m.cache.advance(add)
    m.kv = {(0, s): (ref.rounded(f64(kr[s]), 2.0 ** -4), ref.rounded(f64(v[s]), 2.0 ** -4)) for s in range(2)}
    for _ in range(3):
        m.step([0, 1], 1)
    # the prefix comes back for a prefill that goes on from it
    ko, vo = torch.empty_like(kr), torch.empty_like(v)
    m.cache.read(0, ko, vo)
    assert np.array_equal(f64(ko), np.stack([m.kv[0, s][0][:, :n] for s in range(2)]))
    assert torch.isfinite(y.float()).all() and sa.sa_read_status() == 0


@pytest.mark.parametrize("d", [64, 128])
def test_prefix_joined_with_the_chunks_own_attention(d):
    """The cached prefix by flags 0, the chunk's own keys by sliding-window attention, joined through lse."""
    n, T, Hq, Hkv = 210, 40, 4, 2
    m = Model(d=d, Hq=Hq, Hkv=Hkv, slots=1, page=16, layers=1)
    m.step([0], n)
    q, k, v = (m.draw(1, h, T) for h in (Hq, Hkv, Hkv))
    y0, l0 = m.cache.attend(0, q, flags=0, want_lse=True)
    y1, l1 = sa.sa_swa_forward(q, k, v, T + 1, want_lse=True)
    top = torch.maximum(l0, l1)
    a, b = ((x - top).exp().unsqueeze(-1) for x in (l0, l1))
    y = (a * y0.float() + b * y1.float()) / (a + b)
    kp, vp = m.kv[0, 0]
    want, _ = ref.attend(f64(q[0]), np.concatenate([kp, f64(k[0])], 1), np.concatenate([vp, f64(v[0])], 1), n, d ** -0.5,
                         True, 0)
    # each branch was rounded to bf16, the sliding-window one with bf16 probabilities: 2^-8 of the largest |v| each
    assert np.abs(f64(y[0]) - want).max() <= 2.0 ** -7 * max(np.abs(vp).max(), float(v.abs().max()))


def test_a_captured_step_replays_with_the_lengths_of_the_moment():
    """reserve, append, attend and advance in one graph, replayed while the sequences grow over page borders."""
    d, Hq, Hkv, S, steps = 64, 4, 2, 3, 40
    a, b = (Model(d=d, Hq=Hq, Hkv=Hkv, slots=S, page=16, layers=1, seed=1) for _ in range(2))
    for m in (a, b):
        m.cache.pool.fill_(0)
    k, v, q = (torch.zeros(S, h, 1, d, dtype=torch.bfloat16, device="cuda") for h in (Hkv, Hkv, Hq))
    add = ints([1, 1, 1])

    def step(c):
        got = c.reserve(add)
        c.append(0, k, v)
        y = c.attend(0, q)
        c.advance(add)
        return got, y

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(a.cache)                                       # warm-up; taken back
    torch.cuda.current_stream().wait_stream(side)
    a.free(range(S))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got, y = step(a.cache)
    for i in range(steps):
        for t, h in ((k, Hkv), (v, Hkv), (q, Hq)):
            t.copy_(a.draw(S, h, 1))
        g.replay()
        want_got, want = step(b.cache)
        assert torch.equal(y, want) and torch.equal(got, want_got)
    assert a.cache.lens.tolist() == [steps] * S and torch.equal(a.cache.table, b.cache.table)
    assert torch.equal(a.cache.refs, b.cache.refs) and sa.sa_read_status() == 0


def test_cache_on_another_stream_than_the_default():
    m = Model(slots=2, layers=1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m.step([0, 1], 50)
        m.step([1], 1)
        assert sa.sa_read_status() == 0
