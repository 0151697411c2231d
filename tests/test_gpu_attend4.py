"""Attention of new tokens over a paged cache of 4-bit codes (pcg_cache4_attend) against the definition in double, element by
element.  Run with ``-m gpu`` on an MI355X.

Tolerances are those of tests/attention.py, whose terms are counted per product: with float32 rows every product of a query or weight
with a code is three, of 8 bits each, so that sums have three times the terms."""
import math

import pytest
import torch

import attention
import cache4 as ref
import paper_2511_13732_amd as pcg

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def gen(seed):
    return torch.Generator().manual_seed(seed)


def starts_of(new):
    s = [0]
    for m in new:
        s.append(s[-1] + m)
    return s


def make_cache(lens, page_size, G, D, layout, seed, spare=3, sizes=(-2, 2)):
    """A cache whose pages are dealt at random, with codes of any kind and scales of NaN wherever no request has a token, the table with entries
    outside the cache behind every request's pages, and each request's keys and values in double."""
    g = gen(seed)
    held = [-(-n // page_size) for n in lens]
    total = sum(held) + spare
    order = torch.randperm(total, generator=g).tolist()
    width = max(held + [1]) + 2
    table = torch.full((len(lens), width), -5, dtype=torch.int32)
    table[:, -1] = total + 7
    row = -(-D // 32) * 16
    k, v = (torch.randint(0, 256, (total, page_size, G, row), generator=g).to(torch.uint8) for _ in range(2))
    s = torch.full((total, page_size, G, 2), math.nan, dtype=torch.bfloat16)
    rows = []
    for b, n in enumerate(lens):
        pages = [order.pop() for _ in range(held[b])]
        table[b, :held[b]] = torch.tensor(pages, dtype=torch.int32)
        at = torch.tensor(pages, dtype=torch.long)
        j = torch.arange(n)
        page, slot = (at[j // page_size] if n else j), j % page_size
        s[page, slot] = (0.3 * 2.0 ** (sizes[0] + (sizes[1] - sizes[0]) * torch.rand((n, G, 2), generator=g))).to(torch.bfloat16)
        rows.append(tuple(ref.values(ref.unpacked(x[page, slot], D), s[page, slot][..., i]) for i, x in enumerate((k, v))))
    if layout == "heads":
        k, v, s = (x.transpose(1, 2).contiguous().cuda().transpose(1, 2) for x in (k, v, s))
    elif layout == "mixed":            # a head's codes and scales in one row
        x = torch.zeros((total, page_size, G, 2 * row + 16), dtype=torch.uint8)
        x[..., :row], x[..., row:2 * row], x[..., 2 * row:2 * row + 4] = k, v, s.view(torch.uint8)
        x = x.cuda()
        k, v, s = x[..., :row], x[..., row:2 * row], x[..., 2 * row:2 * row + 4].view(torch.bfloat16)
    else:
        k, v, s = k.cuda(), v.cuda(), s.cuda()
    return pcg.KvCache4(k, v, s, D), table.cuda(), rows


def check(got, want, dtype, what=""):
    out, mag, err = want
    attention.check(got, (out, mag, err * (3 if dtype == torch.float32 else 1)), dtype, what)


def run(ctx, new, H, G, D, dtype, page_size=16, layout="heads", window=0, seed=0, pad=3, longest=None, sigma=1.5, scale=None, sizes=(-2, 2)):
    dt = DTYPES[dtype]
    cache, table, rows = make_cache([c + n for c, n in zip(ctx, new)], page_size, G, D, layout, seed, sizes=sizes)
    st = starts_of(new)
    q = (sigma * torch.randn((st[-1] + pad, H + 2, D), generator=gen(seed + 1))).to(dt).cuda()[:, 1:H + 1]
    out = torch.full((st[-1] + pad, H, D), 77.0, dtype=dt, device="cuda")
    scale = D ** -0.5 if scale is None else scale
    pcg.cache4_attend(cache, q, table, torch.tensor(ctx, dtype=torch.int32).cuda(), torch.tensor(st, dtype=torch.int32).cuda(),
                      longest=max(new + [0]) if longest is None else longest, scale=scale, window=window, out=out)
    assert (out[st[-1]:] == 77.0).all()
    for b in range(len(ctx)):
        want = attention.attend_rows(q[st[b]:st[b + 1]], *rows[b], ctx[b], scale, window)
        check(out[st[b]:st[b + 1]], want, dt, (b, ctx[b], new[b]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [8, 40, 64, 72, 96, 128])
@pytest.mark.parametrize("H,G", [(1, 1), (8, 2), (15, 5), (7, 1)])
def test_chunks_of_a_step(dtype, D, H, G):
    run([0, 1, 37, 64, 200, 15], [5, 1, 4, 9, 3, 2], H, G, D, dtype, seed=D + H)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page_size,layout", [(1, "slots"), (7, "heads"), (16, "mixed"), (64, "slots"), (100, "mixed"), (300, "heads")])
def test_pages_that_end_inside_a_tile(dtype, page_size, layout):
    run([3, 130, 257, 99], [1, 3, 2, 1], 8, 2, 64, dtype, page_size=page_size, layout=layout, seed=page_size)
    run([130, 31], [70, 33], 4, 2, 128, dtype, page_size=page_size, layout=layout, seed=page_size + 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_single_tokens(dtype):
    run([0, 1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 500], [1] * 13, 8, 2, 128, dtype, seed=3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page_size,D,window", [(16, 128, 0), (24, 40, 0), (32, 72, 50), (5, 96, 70)])
@pytest.mark.parametrize("chunk", [8, 9, 16, 17, 32, 33])
def test_rows_on_both_sides_of_a_block(dtype, page_size, D, window, chunk):
    """Four query heads a shared head: 32, 36, 64, 68, 128 and 132 rows at most, each with its own cut of the work."""
    run([210, 0, 77], [chunk, 1, chunk - 3], 8, 2, D, dtype, page_size=page_size, window=window, seed=chunk)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("longest", [1, 16, 400])
def test_long_and_short_chunks_together(dtype, longest):
    """Whatever bound on the chunks is named, the rows are the same."""
    run([300, 7, 0, 40, 90], [1, 150, 67, 0, 33], 4, 1, 64, dtype, longest=longest, seed=longest)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window", [1, 5, 64, 100, 1000])
def test_sliding_windows(dtype, window):
    run([0, 70, 333, 130], [9, 5, 3, 80], 6, 2, 64, dtype, window=window, page_size=24, seed=window)
    run([700, 1500], [40, 3], 4, 1, 128, dtype, window=window, seed=window + 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sigma,sizes", [(0.0, (-2, 2)), (30.0, (-2, 2)), (1.5, (-12, 6)), (1.0, (-30, -25))])
def test_flat_and_sharp_rows_and_scales_of_all_sizes(dtype, sigma, sizes):
    run([120, 700], [4, 3], 4, 2, 64, dtype, sigma=sigma, sizes=sizes, seed=11)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_caches_in_many_parts(dtype):
    """Runs end inside units, parts of a unit are many; offsets of pages pass what a page takes."""
    run([20011], [2], 8, 1, 128, dtype, seed=21, page_size=64)
    run([9000, 40, 3000], [1, 9, 17], 8, 2, 64, dtype, seed=22, page_size=7, layout="slots")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_rows_at_all_and_requests_without_any(dtype):
    run([5, 9], [0, 0], 4, 2, 64, dtype)
    run([0, 5, 0, 9, 0], [0, 2, 0, 1, 0], 4, 2, 64, dtype)
    cache, table, _ = make_cache([4], 16, 2, 64, "heads", 0)
    e = torch.empty((0, 4, 64), device="cuda")
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert pcg.cache4_attend(cache, e, table, one, torch.zeros(2, dtype=torch.int32, device="cuda")).shape == (0, 4, 64)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window", [0, 30])
@pytest.mark.parametrize("n,longest", [(3, 3), (17, 17), (40, 40), (170, 1)])
def test_what_a_row_does_not_see_has_no_effect(dtype, window, n, longest):
    """Keys and values that are NaN reach exactly the rows that see them, and all of their head there."""
    dt, H, G, D, ctx = DTYPES[dtype], 4, 2, 64, 145
    cache, table, rows = make_cache([ctx + n], 16, G, D, "heads", n)
    (k, v), = rows
    bad_key, bad_value = ctx + n - 1 - n // 3, ctx + n - 1
    for j, i in ((bad_key, 0), (bad_value, 1), (20, 1)):
        if j == 20 and not window:
            continue                   # without a window every row sees it
        cache.scales[int(table[0, j // 16]), j % 16, 1, i] = math.inf if j == 20 else math.nan
        (k, v)[i][j, 1] = math.nan
    q = torch.randn((n, H, D), generator=gen(1)).to(dt).cuda()
    out = pcg.cache4_attend(cache, q, table, torch.tensor([ctx], dtype=torch.int32).cuda(), torch.tensor([0, n], dtype=torch.int32).cuda(),
                            longest=longest, window=window)
    pos = ctx + torch.arange(n)
    first = (pos - window + 1).clamp(min=0) if window else torch.zeros_like(pos)
    struck = sum(((first <= j) & (j <= pos)).long() for j in (bad_key, bad_value) + ((20,) if window else ())) > 0
    got = out.cpu().float()
    assert torch.isfinite(got[:, :2]).all() and torch.equal(torch.isnan(got[:, 2:]).all(dim=2), struck[:, None].expand(n, 2))
    assert torch.isfinite(got[~struck]).all()
    for h, rows_ in ((0, slice(None)), (1, ~struck)):
        want = attention.attend_rows(q[:, 2 * h:2 * h + 2], k[:, h:h + 1].nan_to_num(0), v[:, h:h + 1].nan_to_num(0), ctx, D ** -0.5, window)
        check(out[:, 2 * h:2 * h + 2].cpu()[rows_], tuple(x[rows_] for x in want), dt)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page_size", [16, 5])
def test_pages_outside_the_cache_read_as_zeros(dtype, page_size):
    dt, H, G, D, ctx, n = DTYPES[dtype], 4, 2, 72, 77, 2
    cache, table, rows = make_cache([ctx + n], page_size, G, D, "slots", 4)
    (k, v), = rows
    for block, page in ((1, -1), (2, cache.num_pages), (3, 1 << 30)):
        table[0, block] = page
        k[block * page_size:(block + 1) * page_size] = 0
        v[block * page_size:(block + 1) * page_size] = 0
    short = table[:, :60 // page_size].contiguous()            # keys past the table's last block
    q = torch.randn((n, H, D), generator=gen(1)).to(dt).cuda()
    for t in (table, short):
        lens = min(ctx, t.shape[1] * page_size - (0 if t is short else 1))
        kk, vv = k.clone(), v.clone()
        kk[t.shape[1] * page_size:], vv[t.shape[1] * page_size:] = 0, 0
        out = pcg.cache4_attend(cache, q, t, torch.tensor([ctx], dtype=torch.int32).cuda(), torch.tensor([0, n], dtype=torch.int32).cuda())
        # a length is at most what the table has room for
        check(out, attention.attend_rows(q, kk, vv, lens if t is short else ctx, D ** -0.5), dt)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_without_a_score(dtype):
    """Scores of -infinity everywhere: zeros, also beside a value that is NaN."""
    dt, D = DTYPES[dtype], 32
    cache = pcg.KvCache4.empty(2, 16, 1, D, "cuda")
    cache.k.fill_(0x22)                # ones
    cache.v.fill_(0x22)
    cache.scales.fill_(1.0)
    cache.scales[0, 3, 0, 1] = math.nan
    q = torch.zeros((2, 1, D), dtype=dt, device="cuda")
    q[0, 0, 4] = -math.inf
    table = torch.tensor([[0, 1]], dtype=torch.int32).cuda()
    out = pcg.cache4_attend(cache, q, table, torch.tensor([18], dtype=torch.int32).cuda(), torch.tensor([0, 2], dtype=torch.int32).cuda())
    assert (out[0] == 0).all() and torch.isnan(out[1]).all()
    cache.scales[0, 3, 0, 1] = 1.0
    out = pcg.cache4_attend(cache, q, table, torch.tensor([18], dtype=torch.int32).cuda(), torch.tensor([0, 2], dtype=torch.int32).cuda())
    assert (out[0] == 0).all() and (out[1] == 1).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_scores_and_values(dtype):
    """Scores far beyond 2^24, whose differences are whole steps; scales near the ends of the range."""
    dt, D, n = DTYPES[dtype], 64, 90
    cache, table, rows = make_cache([n], 16, 1, D, "heads", 3)
    q = torch.full((1, 1, D), 2.0, dtype=dt, device="cuda")
    cache.k.fill_(0)
    cache.k[..., 0] = 7                # one element of 6
    sizes = torch.arange(n).double()
    page, slot = table[0].cpu().long()[torch.arange(n) // 16], torch.arange(n) % 16
    big = (2.0 ** 60 * (1 + (sizes % 7) / 128)).to(torch.bfloat16)
    cache.scales[page, slot, 0, 0] = big.cuda()
    _, v = rows[0]
    out = pcg.cache4_attend(cache, q, table, torch.tensor([n - 1], dtype=torch.int32).cuda(), torch.tensor([0, 1], dtype=torch.int32).cuda(), scale=1.0)
    top = big == big.max()
    want = v[top].mean(dim=0)
    tol = 2.0 ** -7 * v[top].abs().mean(dim=0) if dtype == "bf16" else 2.0 ** -20 * v[top].abs().mean(dim=0)
    assert ((out[0, 0].double().cpu() - want[0]).abs() <= tol[0] + 1e-30).all()
    # values of 1e36 in a sum of 90, weights up to 2^8: within float32
    cache.scales[page, slot, 0, 0] = 1.0
    cache.scales[page, slot, 0, 1] = 1e33
    cache.k.zero_()
    out = pcg.cache4_attend(cache, q, table, torch.tensor([n - 1], dtype=torch.int32).cuda(), torch.tensor([0, 1], dtype=torch.int32).cuda())
    unit = float(torch.tensor(1e33).to(torch.bfloat16))
    codes = ref.values(ref.unpacked(cache.v.cpu()[page, slot], D), torch.ones((n, 1), dtype=torch.bfloat16)) * unit
    want = attention.attend_rows(q.cpu(), torch.zeros((n, 1, D), dtype=torch.float64), codes, n - 1, D ** -0.5)
    check(out, want, dt)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("longest", [3, 12, 40])
def test_the_same_bits_from_any_workspace(dtype, longest):
    dt, H, G, D = DTYPES[dtype], 8, 2, 128
    ctx, new = [900, 3, 2100], [3, 1, 2]
    cache, table, _ = make_cache([c + n for c, n in zip(ctx, new)], 16, G, D, "heads", 8)
    st = starts_of(new)
    q = torch.randn((st[-1], H, D), generator=gen(1)).to(dt).cuda()
    lens, starts = (torch.tensor(x, dtype=torch.int32).cuda() for x in (ctx, st))
    n = pcg.cache4_attend_workspace_bytes(3, st[-1], H, G, D, longest)
    outs = []
    for fill in (0, 255, 127):
        ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
        outs.append(pcg.cache4_attend(cache, q, table, lens, starts, longest=longest, workspace=ws))
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
