"""Attention where scores, weights or values are at the ends of what float32 holds, over the paged cache (pcg_cache_attend) and of
packed prompts (pcg_prompt_attend).  Run with ``-m gpu`` on an MI355X."""
import pytest
import torch

import attention as ref
import paper_2511_13732_amd as pcg
from test_gpu_attend import DTYPES, gen

pytestmark = pytest.mark.gpu


def ints(*x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def over_cache(q, k, v, window=0, scale=None, page_size=16):
    """The last q.shape[0] tokens of one request of k.shape[0]."""
    n, G, D = k.shape
    m, blocks = q.shape[0], -(-n // page_size)
    pad = lambda x: torch.cat([x, x.new_zeros((blocks * page_size - n, G, D))]).view(blocks, page_size, G, D).cuda()  # noqa: E731
    table = torch.arange(blocks, dtype=torch.int32).view(1, -1).cuda()
    return pcg.cache_attend(pcg.KvCache(pad(k), pad(v)), q.cuda(), table, ints(n - m), ints(0, m), longest=m, window=window, scale=scale).cpu()


def as_prompt(q, k, v, window=0, scale=None, longest=None):
    n = q.shape[0]
    return pcg.prompt_attend(q.cuda(), k.cuda(), v.cuda(), ints(0, n), longest=longest or n, window=window, scale=scale).cpu()


# ------------------------------------------------------------------------------------------------ scores

# A score of 2^24 in powers of two is rounded by one; these are 2^16, 2^23 and more, up to 2^60.
LARGE = [16, 23, 25, 31, 37, 60]


def rounding(dtype):
    """Relative to sum w |v|: a weight is w = 2^x of an exact x within [-2, 2] where keys are alike, the same for all; its rounding to
    bf16, and of the output, half a step each; in float32 a sum of n products and one of n weights, a reciprocal and a product, within
    (2 n + 8) steps of 2^-23."""
    return (lambda n: (2 * n + 8) * 2.0 ** -23) if dtype == torch.float32 else (lambda n: 2.0 ** -8 * 2.02 + (2 * n + 8) * 2.0 ** -23)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("power", LARGE)
@pytest.mark.parametrize("sign", [1, -1])
def test_keys_alike_count_alike_however_large_their_scores(dtype, D, power, sign):
    """All keys the same: every row is the mean of the values that it sees, whatever the score."""
    dt, n, H, G = DTYPES[dtype], 150, 4, 2
    scale = 0.3
    q = torch.randn((n, H, D), generator=gen(power)).abs() + 0.1
    # q . k is D times 2^power or so, in powers of two
    q = (q * 2.0 ** (power / 2)).to(dt)
    k = (sign * (torch.randn((1, G, D), generator=gen(2)).abs() + 0.1) * 2.0 ** (power / 2)).to(dt).expand(n, G, D).contiguous()
    v = torch.randn((n, G, D), generator=gen(3)).to(dt)
    for window in (0, 1, 40):
        lo = [max(0, t - window + 1) if window else 0 for t in range(n)]
        mean = torch.stack([v[lo[t]:t + 1].double().mean(0) for t in range(n)]).repeat_interleave(H // G, 1)
        mag = torch.stack([v[lo[t]:t + 1].double().abs().mean(0) for t in range(n)]).repeat_interleave(H // G, 1)
        tol = rounding(dt)(n) * mag
        for m in (1, 9, 70):
            got = over_cache(q[n - m:], k, v, window, scale).double()
            assert ((got - mean[n - m:]).abs() <= tol[n - m:]).all(), (window, m)
        for longest in (1, n):
            got = as_prompt(q, k, v, window, scale, longest).double()
            assert ((got - mean).abs() <= tol).all(), (window, longest)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("best", [0, 63, 64, 100, 190])
@pytest.mark.parametrize("long", [200, 9000])
def test_the_largest_of_large_scores_has_all_the_weight(dtype, best, long):
    """One key's score is 2^35 or more above all others: its value is the output."""
    dt, H, G, D, m = DTYPES[dtype], 6, 3, 64, 5
    n = long
    q = ((torch.randn((m, H, D), generator=gen(best)).abs() + 0.1) * 2.0 ** 16).to(dt)
    k = ((torch.randn((n, G, D), generator=gen(1)).abs() + 0.1) * 2.0 ** 16).to(dt)
    k[best] = (k[best] * 0 + 2.0 ** 24).to(dt)
    v = torch.randn((n, G, D), generator=gen(4)).to(dt)
    want = v[best].double().repeat_interleave(H // G, 0)
    got = over_cache(q, k, v).double()
    assert ((got - want).abs() <= rounding(dt)(1) * want.abs()).all()
    if n <= 200:
        rows = torch.cat([q] * (n // m))
        for longest in (1, n):
            got = as_prompt(rows, k, v, longest=longest).double()[best:]
            assert ((got - want).abs() <= rounding(dt)(1) * want.abs()).all()


def test_a_far_row_does_not_move_the_others():
    """Rows of the same block with ordinary scores keep their bits beside one whose scores are far out."""
    dt, n, H, G, D = torch.float32, 96, 4, 1, 64
    q, k, v = (torch.randn((n, h, D), generator=gen(s)).to(dt) for s, h in ((1, H), (2, G), (3, G)))
    clean = as_prompt(q, k, v)
    near = q.clone()
    near[40, 2] *= 2.0 ** 30
    far = as_prompt(near, k, v)
    others = torch.ones((n, H), dtype=torch.bool)
    others[40, 2] = False
    # the references of a block may follow earlier beside it: the same sums from another reference, off by 2 n + 64 steps each way
    off = (far - clean).abs()[others]
    assert (off <= 2 * (2 * n + 64) * 2.0 ** -23 * v.abs().max()).all()
    assert torch.isfinite(far).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("n,m", [(40, 2), (40, 30), (300, 100), (7000, 1)])
def test_rows_without_a_score_above_minus_infinity_are_zeros_whatever_the_values(dtype, bad, n, m):
    """Every score -infinity, in one tile, several and in parts that are joined."""
    dt, H, G, D = DTYPES[dtype], 3, 1, 64
    q, k = torch.ones((m, H, D), dtype=dt), torch.full((n, G, D), -float("inf"), dtype=dt)
    v = torch.randn((n, G, D), generator=gen(n)).to(dt)
    v[::3, 0, 5] = bad
    v[n // 2] = bad
    for window in (0, 17):
        assert (over_cache(q, k, v, window) == 0).all()
        if m > 1:
            for longest in (1, m):
                assert (as_prompt(q, k[:m], v[:m], window, longest=longest) == 0).all()


# ------------------------------------------------------------------------------------------------ values

def odd_rows(kind, n, G, D, dt, places, seed):
    """Keys and values of which those at `places` are not finite: +infinity in column 3, -infinity in column 5, in column 7 first one and
    then the other, NaN in column D - 1 of the last place.  "low": their weights are e^-500 or so beside the others'; "rising": so are those of the
    first half of all keys."""
    k, v = (torch.randn((n, G, D), generator=gen(s)) for s in (seed, seed + 1))
    k *= 0.1
    if kind == "low":
        k[list(places)] = -8.0
    if kind == "rising":
        k[:n // 2] -= 8.0
    k, v = k.to(dt), v.to(dt)
    for i, j in enumerate(places):
        v[j, 0, 3], v[j, 0, 5] = float("inf"), -float("inf")
        v[j, 0, 7] = float("inf") if i % 2 == 0 else -float("inf")
    v[places[-1], G - 1, D - 1] = float("nan")
    return k, v


def check_odd(got, q, k, v, first, window, dt):
    """Rows of q at positions first, first + 1, ..: where a row sees values that are not finite their sum, and the definition elsewhere."""
    m, H, D = q.shape
    G = k.shape[1]
    odd = torch.where(torch.isfinite(v), torch.zeros_like(v), v)
    finite = torch.where(torch.isfinite(v), v, torch.zeros_like(v))
    want = ref.attend_rows(q, k, finite, first, 1.0, window)
    sums = torch.zeros((m, H, D), dtype=torch.float64)
    for t in range(m):
        p = first + t
        lo = max(0, p - window + 1) if window else 0
        sums[t] = odd[lo:p + 1].double().sum(0).repeat_interleave(H // G, 0)
    plain = sums == 0
    ref.check(torch.where(plain, got.double(), 0.0), tuple(torch.where(plain, x, 0.0) for x in want), dt)
    bad = ~plain
    same = (got.double() == sums) | (torch.isnan(got) & torch.isnan(sums))
    assert same[bad].all(), (bad & ~same).nonzero()[0].tolist()


KINDS = ["plain", "low", "rising"]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("places", [(0,), (5, 40), (63, 64, 200), (130, 299), (20, 21, 22, 90, 150)])
def test_an_infinity_counts_whatever_its_weight_and_wherever_it_lies_in_a_prompt(dtype, D, kind, places):
    dt, n, H, G = DTYPES[dtype], 300, 4, 2
    k, v = odd_rows(kind, n, G, D, dt, places, D)
    q = (torch.ones((n, H, D)) + 0.01 * torch.randn((n, H, D), generator=gen(9))).to(dt)
    for window in (0, 90):
        for longest in (1, n):
            check_odd(as_prompt(q, k, v, window, 1.0, longest), q, k, v, 0, window, dt)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,page_size", [(64, 16), (128, 16), (96, 5)])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,places", [(300, (0,)), (300, (70, 150)), (300, (31, 64, 299)), (9000, (10, 4000)), (9000, (2500, 8999))])
def test_an_infinity_counts_whatever_its_weight_and_wherever_it_lies_in_a_cache(dtype, D, page_size, kind, n, places):
    dt, H, G = DTYPES[dtype], 6, 2
    k, v = odd_rows(kind, n, G, D, dt, places, D)
    for m in (1, 9, 20, 70):
        q = (torch.ones((m, H, D)) + 0.01 * torch.randn((m, H, D), generator=gen(m))).to(dt)
        for window in (0, 120):
            check_odd(over_cache(q, k, v, window, 1.0, page_size), q, k, v, n - m, window, dt)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_everything_not_finite(dtype):
    """All values NaN, or all infinite: every element is, in as much time as one tile takes."""
    dt, n, H, G, D = DTYPES[dtype], 2000, 4, 2, 128
    k = torch.randn((n, G, D), generator=gen(1)).to(dt)
    q = torch.randn((n, H, D), generator=gen(2)).to(dt)
    for x in (float("nan"), float("inf")):
        v = torch.full_like(k, x)
        for got in (over_cache(q[:50], k, v), as_prompt(q[:300], k[:300], v[:300])):
            assert (torch.isnan(got) if x != x else got == x).all()
