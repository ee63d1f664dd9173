"""Score sums of fp32 calls over the 4-bit cache: added with roundings, not cut off.

All scores are of one sign and their softmax is nearly one key's, so that lse shows a score's own error.  Roundings of a
score, in units of 2^-24 of it: 16 additions to the running sum of 256 dimensions, which grows evenly (8.5 at most, to
either side); q as two terms of 11 bits (4, to either side); a matrix instruction's own cut over 16 dimensions, two terms
(2, towards 0); the constants 1/sqrt(d), log2(e), their product and ln(2) (4, the same in every row); the products by the last
two (2, to either side).  Together 20.5 in any row.  Over 512 rows with 300 keys what goes to either side cancels: the mean's
bound is 6, and 2 for what is left of 512 draws (measured: at most 1.3).  Sums in one accumulator were off by 8 to 9 at
d = 192 and 256."""
import pytest
import torch

from paper_2604_00754_b200 import binding as sa

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("d", [128, 192, 256])
@pytest.mark.parametrize("size", [64.0, 1e34])       # below and above what the copy for full tiles takes
@pytest.mark.parametrize("sign", [1, -1])
def test_fp32_scores_are_rounded_not_cut_off(d, size, sign):
    gen = torch.Generator(device="cuda").manual_seed(d)
    k, v = (torch.randn(1, 1, 300, d, device="cuda", generator=gen) for _ in range(2))
    q = torch.randn(1, 32, 16, d, device="cuda", generator=gen).abs() * size
    pool, table = sa.sa_cache_pool(1, 19, 1, 16, d), ints([list(range(19))])
    sa.sa_cache_append(pool, table, ints([0]), sign * k.abs(), v)
    ks, vs = torch.empty_like(k), torch.empty_like(v)
    sa.sa_cache_read(pool, table, ks, vs)
    s = q[0].double() @ ks[0, 0].double().T * d ** -0.5
    _, lse = sa.sa_cache_attend(pool, table, ints([300]), q, flags=0, want_lse=True)
    want = s.logsumexp(-1)
    error = (lse[0].double() - want) / want.abs() * 2 ** 24
    assert float(error.abs().max()) <= 20.5
    assert abs(float(error.mean())) <= 8
    assert sa.sa_read_status() == 0
