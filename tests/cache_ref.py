"""Float64 statements of the 4-bit cache for the tests: formats, rounding, attention, books.

Written from the definitions in sa.h on the CPU with numpy; nothing of the library is used."""
import numpy as np

E2M1 = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])
E4M3 = np.array([(m / 8 if e == 0 else 1 + m / 8) * 2.0 ** ((-6 if e == 0 else e - 7))
                 for e in range(16) for m in range(8)][:127])


def nearest(x, grid):
    """Index into an ascending grid of what is nearest to x >= 0; ties to the even index; saturating."""
    at = np.clip(np.searchsorted(grid, x), 1, len(grid) - 1)
    up, down = grid[at] - x, x - grid[at - 1]
    return np.where((up < down) | ((up == down) & (at % 2 == 0)), at, at - 1)


def quantise(x, t):
    """x [..., d] float64 -> codes [..., d] (0..15) and scale bytes [..., d/16]."""
    y = (x / t).reshape(*x.shape[:-1], x.shape[-1] // 16, 16)
    bad = ~np.isfinite(y).all(-1)
    y = np.where(bad[..., None], 0, y)
    s = nearest(np.abs(y).max(-1) / 6, E4M3)
    f = E4M3[s][..., None]
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.where(f > 0, np.abs(y) / f, 0)
    c = nearest(q, E2M1) + 8 * ((y < 0) & (f > 0))
    return np.where(bad[..., None], 0, c).reshape(x.shape), np.where(bad, 0x7f, s)


def values(codes, scales, t):
    s = np.append(E4M3, np.nan)[scales & 127] * t
    return E2M1[codes & 7] * np.where(codes & 8, -1, 1) * np.repeat(s, 16, -1)


def rounded(x, t):
    return values(*quantise(x, t), t)


def pack(pool, page, h, side, i, codes, scales, P):
    """Writes one token's codes and scales into pool [pages, Hkv, 2, bytes] (uint8)."""
    d = codes.shape[-1]
    buf = pool[page, h, side]
    buf[i * d // 2:(i + 1) * d // 2] = codes[::2] | codes[1::2] << 4
    at = P * d // 2 + i * d // 16
    buf[at:at + d // 16] = scales


def attend(q, k, v, length, scale, causal, w, counts=None):
    """q [Hq,T,d], k and v [Hkv,n,d] (n keys have pages); returns y, lse (natural)."""
    Hq, T, d = q.shape
    Hkv, n, _ = k.shape
    pos = length + np.arange(T)[:, None]
    j = np.arange(n)
    seen = (j <= pos) if causal else np.broadcast_to(j < length, (T, n))
    if w > 0:
        seen = seen & (pos - j < w)
    y, lse = np.zeros(q.shape), np.full((Hq, T), -np.inf)
    for h in range(Hq):
        for t in range(T):
            at = np.flatnonzero(seen[t])
            if len(at):
                s = (q[h, t] @ k[h * Hkv // Hq, at].T) * scale
                m = s.max()
                p = np.exp(s - m)
                lse[h, t] = m + np.log(p.sum())
                y[h, t] = p @ v[h * Hkv // Hq, at] / p.sum()
    return y, lse


class Books:
    """The books as lists; pages hold labels in place of contents."""

    def __init__(self, table, lens, refs, P, pool=None):
        self.table, self.lens, self.refs, self.P = [list(r) for r in table], list(lens), list(refs), P
        self.pool = list(range(len(refs))) if pool is None else list(pool)

    def free(self, slots):
        for s in slots:
            for p in self.table[s]:
                if p >= 0:
                    self.refs[p] -= 1
            self.table[s], self.lens[s] = [-1] * len(self.table[s]), 0

    def fork(self, parents, children):
        for a, b in zip(parents, children):
            n = -(-self.lens[a] // self.P)
            self.table[b] = self.table[a][:n] + [-1] * (len(self.table[a]) - n)
            self.lens[b] = self.lens[a]
            for p in self.table[a][:n]:
                self.refs[p] += 1

    def reserve(self, add):
        before, free, used, got = list(self.refs), [p for p, r in enumerate(self.refs) if r == 0], 0, []
        for s, n in enumerate(add):
            row, length = self.table[s], self.lens[s]
            last = -(-(length + n) // self.P) if n else 0
            if last > len(row):
                got.append(0)
                continue
            want = [j for j in range(length // self.P, last) if row[j] < 0 or before[row[j]] > 1]
            used += len(want)
            ok = not want or used <= len(free)
            got.append(int(ok))
            for k, j in enumerate(want if ok else []):
                new, old = free[used - len(want) + k], row[j]
                if old >= 0:
                    self.refs[old] -= 1
                    if j * self.P < length:
                        self.pool[new] = self.pool[old]
                self.refs[new], row[j] = 1, new
        return got

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        holes = [p for p in range(live) if self.refs[p] == 0]
        to = dict(zip([p for p in range(live, len(self.refs)) if self.refs[p] > 0], holes))
        for old, new in to.items():
            self.pool[new], self.refs[new], self.refs[old] = self.pool[old], self.refs[old], 0
        self.table = [[to.get(p, p) for p in r] for r in self.table]
        return live
