"""Attention of new tokens over the paged cache (pcg_cache_attend) and of packed prompts (pcg_prompt_attend) against the
definition in double, element by element.  Run with ``-m gpu`` on an MI355X."""
import math

import pytest
import torch

import attention as ref
import paper_2511_13732_amd as pcg

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def gen(seed):
    return torch.Generator().manual_seed(seed)


def make_cache(lens, page_size, G, D, dtype, layout, seed, spare=3, fill=math.nan):
    """A cache whose pages are dealt at random, with `fill` wherever no request has a token, the table with entries outside the
    cache behind every request's pages, and each request's keys and values."""
    g = gen(seed)
    held = [-(-n // page_size) for n in lens]
    total = sum(held) + spare
    order = torch.randperm(total, generator=g).tolist()
    width = max(held + [1]) + 2
    table = torch.full((len(lens), width), -5, dtype=torch.int32)
    table[:, -1] = total + 7
    shape = (total, page_size, G, D) if layout == "slots" else (total, G, page_size, D)
    k = torch.full(shape, fill, dtype=dtype)
    v = torch.full(shape, fill, dtype=dtype)
    kc, vc = (k, v) if layout == "slots" else (k.transpose(1, 2), v.transpose(1, 2))
    rows = []
    for b, n in enumerate(lens):
        pages = [order.pop() for _ in range(held[b])]
        table[b, :held[b]] = torch.tensor(pages, dtype=torch.int32)
        x = torch.randn((2, n, G, D), generator=g).to(dtype)
        for j in range(n):
            kc[pages[j // page_size], j % page_size] = x[0, j]
            vc[pages[j // page_size], j % page_size] = x[1, j]
        rows.append((x[0], x[1]))
    k, v = k.cuda(), v.cuda()
    if layout != "slots":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    return pcg.KvCache(k, v), table.cuda(), rows


def starts_of(new):
    s = [0]
    for m in new:
        s.append(s[-1] + m)
    return s


def run_cache(ctx, new, H, G, D, dtype, page_size=16, layout="slots", window=0, seed=0, pad=3, longest=None, sigma=1.5,
              scale=None):
    dt = DTYPES[dtype]
    cache, table, rows = make_cache([c + n for c, n in zip(ctx, new)], page_size, G, D, dt, layout, seed)
    st = starts_of(new)
    q = (sigma * torch.randn((st[-1] + pad, H + 2, D), generator=gen(seed + 1))).to(dt).cuda()[:, 1:H + 1]
    out = torch.full((st[-1] + pad, H, D), 77.0, dtype=dt, device="cuda")
    scale = D ** -0.5 if scale is None else scale
    pcg.cache_attend(cache, q, table, torch.tensor(ctx, dtype=torch.int32).cuda(), torch.tensor(st, dtype=torch.int32).cuda(),
                     longest=max(new + [0]) if longest is None else longest, scale=scale, window=window, out=out)
    assert (out[st[-1]:] == 77.0).all()
    for b in range(len(ctx)):
        want = ref.attend_rows(q[st[b]:st[b + 1]], *rows[b], ctx[b], scale, window)
        ref.check(out[st[b]:st[b + 1]], want, dt, (b, ctx[b], new[b]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [8, 64, 72, 128])
@pytest.mark.parametrize("H,G", [(1, 1), (8, 2), (15, 5), (7, 1)])
def test_chunks_of_a_step(dtype, D, H, G):
    run_cache([0, 1, 37, 64, 200, 15], [5, 1, 4, 9, 3, 2], H, G, D, dtype, seed=D + H)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page_size,layout", [(1, "slots"), (7, "heads"), (16, "heads"), (64, "slots"), (100, "slots"), (300, "heads")])
def test_pages_that_end_inside_a_tile(dtype, page_size, layout):
    run_cache([3, 130, 257, 99], [1, 3, 2, 1], 8, 2, 64, dtype, page_size=page_size, layout=layout, seed=page_size)
    run_cache([130, 31], [70, 33], 4, 2, 128, dtype, page_size=page_size, layout=layout, seed=page_size + 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_single_tokens(dtype):
    run_cache([0, 1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 500], [1] * 13, 8, 2, 128, dtype, seed=3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page_size,D,window", [(16, 128, 0), (24, 40, 0), (32, 72, 50), (5, 96, 70)])
@pytest.mark.parametrize("chunk", [8, 9, 16, 17, 32, 33])
def test_rows_on_both_sides_of_a_block(dtype, page_size, D, window, chunk):
    """Four query heads a shared head: 32, 36, 64, 68, 128 and 132 rows at most, each with its own cut of the work."""
    run_cache([210, 0, 77], [chunk, 1, chunk - 3], 8, 2, D, dtype, page_size=page_size, window=window, seed=chunk)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("longest", [1, 16, 400])
def test_long_and_short_chunks_together(dtype, longest):
    """Whatever bound on the chunks is named, the rows are the same."""
    run_cache([300, 7, 0, 40, 90], [1, 150, 67, 0, 33], 4, 1, 64, dtype, longest=longest, seed=longest)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window", [1, 5, 64, 100, 1000])
def test_sliding_windows(dtype, window):
    run_cache([0, 70, 333, 130], [9, 5, 3, 80], 6, 2, 64, dtype, window=window, page_size=24, seed=window)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sigma", [0.0, 30.0])
def test_flat_and_sharp_rows(dtype, sigma):
    run_cache([120, 700], [4, 3], 4, 2, 64, dtype, sigma=sigma, seed=11)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_rows_at_all_and_requests_without_any(dtype):
    run_cache([5, 9], [0, 0], 4, 2, 64, dtype)
    run_cache([0, 5, 0, 9, 0], [0, 2, 0, 1, 0], 4, 2, 64, dtype)
    cache, table, _ = make_cache([4], 16, 2, 64, torch.float32, "slots", 0)
    e = torch.empty((0, 4, 64), device="cuda")
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert pcg.cache_attend(cache, e, table, one, torch.zeros(2, dtype=torch.int32, device="cuda")).shape == (0, 4, 64)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [3, 40, 170])
def test_what_a_row_does_not_see_has_no_effect(dtype, n):
    """Keys and values of later tokens that are NaN or infinite reach exactly the rows that see them."""
    dt, H, G, D, ctx = DTYPES[dtype], 4, 2, 64, 45
    cache, table, rows = make_cache([ctx + n], 16, G, D, dt, "slots", n)
    k, v = rows[0]
    bad = ctx + n - 1 - n // 3
    for j, (kx, vx) in ((bad, (1.0, math.inf)), (ctx + n - 1, (math.nan, math.nan))):
        page, slot = int(table[0, j // 16]), j % 16
        k[j, 1] = k[j, 1] * kx
        v[j, 1, 3] = vx
        cache.k[page, slot] = k[j].cuda()
        cache.v[page, slot] = v[j].cuda()
    q = torch.randn((n, H, D), generator=gen(5)).to(dt).cuda()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    out = pcg.cache_attend(cache, q, table, i32(ctx), i32(0, n), longest=n)
    want = ref.attend_rows(q, k, v, ctx, D ** -0.5)
    seen = bad - ctx
    finite = lambda w, sl: tuple(x[sl] for x in w)  # noqa: E731
    ref.check(out[:seen], finite(want, slice(0, seen)), dt)                       # nobody ahead sees anything of it
    assert torch.isfinite(out[:, :2]).all()                                       # the other shared head
    assert torch.isfinite(out[:n - 1, 2:, :3]).all() and torch.isfinite(out[:n - 1, 2:, 4:]).all()
    assert (out[seen:n - 1, 2:, 3] == math.inf).all()
    assert torch.isnan(out[n - 1, 2:]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_see_nothing_give_zeros(dtype):
    """Every score -infinity."""
    dt = DTYPES[dtype]
    cache, table, rows = make_cache([40], 16, 1, 64, dt, "slots", 1)
    cache.k.fill_(-math.inf)
    q = torch.ones((2, 3, 64), dtype=dt, device="cuda")
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    out = pcg.cache_attend(cache, q, table, i32(38), i32(0, 2))
    assert (out == 0).all()


def test_pages_outside_the_cache_read_as_zeros():
    dt = torch.float32
    cache, table, rows = make_cache([64], 16, 2, 64, dt, "slots", 2)
    k, v = (x.clone() for x in rows[0])
    for block, entry in ((1, -1), (2, cache.num_pages)):
        table[0, block] = entry
        k[16 * block:16 * block + 16] = 0
        v[16 * block:16 * block + 16] = 0
    q = torch.randn((3, 4, 64), generator=gen(1)).cuda()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    out = pcg.cache_attend(cache, q, table, i32(61), i32(0, 3))
    ref.check(out, ref.attend_rows(q, k, v, 61, 0.125), dt)


@pytest.mark.parametrize("dtype,G,H,ctx", [("bf16", 8, 32, 9000), ("f32", 2, 6, 5001), ("bf16", 1, 8, 20000), ("bf16", 2, 2, 4096)])
def test_a_long_cache_is_split(dtype, G, H, ctx):
    run_cache([ctx, 17, ctx // 3], [3, 2, 1], H, G, 64, dtype, page_size=32, seed=ctx)
    run_cache([ctx], [1], H, G, 128, dtype, page_size=64, layout="heads", seed=ctx + 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_row_in_more_parts_than_a_wave_has_lanes(dtype):
    run_cache([21000], [1], 1, 1, 64, dtype, page_size=64, seed=21)
    run_cache([21000], [40], 1, 1, 64, dtype, page_size=16, seed=22)


def test_offsets_past_32_bits():
    """Pages so far apart that elements and bytes are counted past 2^32."""
    D, G, ps, dt = 64, 1, 16, torch.bfloat16
    far = 3 * (1 << 30)                                             # elements between two pages: 6 GB
    big = torch.empty(2 * far + ps * G * D, dtype=dt, device="cuda")
    view = lambda t: t.as_strided((3, ps, G, D), (far, G * D, D, 1))  # noqa: E731
    big2 = torch.empty_like(big)
    cache = pcg.KvCache(view(big), view(big2))
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32).cuda()
    k, v = (torch.randn((48, G, D), generator=gen(s)).to(dt) for s in (1, 2))
    slots = torch.tensor([int(table[0, j // ps]) * ps + j % ps for j in range(48)], dtype=torch.int32).cuda()
    pcg.cache_write(cache, k.cuda(), v.cuda(), slots)
    q = torch.randn((2, 4, D), generator=gen(3)).to(dt).cuda()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    out = pcg.cache_attend(cache, q, table, i32(46), i32(0, 2))
    ref.check(out, ref.attend_rows(q, k, v, 46, 0.125), dt)


# ---------------------------------------------------------------------------------------- prompts

def run_prompt(new, H, G, D, dtype, window=0, seed=0, pad=2, longest=None, order="together", sigma=1.5):
    dt = DTYPES[dtype]
    st = starts_of(new)
    T = st[-1] + pad
    x = torch.randn((T, H + 2 * G, D), generator=gen(seed))
    x[:, :H] *= sigma
    x[st[-1]:] = math.nan
    x = x.to(dt).cuda()
    if order == "heads":
        x = x.transpose(0, 1).contiguous().transpose(0, 1)
    q, k, v = x[:, :H], x[:, H:H + G], x[:, H + G:]
    out = torch.full((T, H, D), 77.0, dtype=dt, device="cuda")
    pcg.prompt_attend(q, k, v, torch.tensor(st, dtype=torch.int32).cuda(), longest=longest or max(new + [1]), window=window, out=out)
    assert (out[st[-1]:] == 77.0).all()
    for b in range(len(new)):
        s = slice(st[b], st[b + 1])
        ref.check(out[s], ref.attend_rows(q[s], k[s], v[s], 0, D ** -0.5, window), dt, (b, new[b]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [16, 64, 80, 128])
@pytest.mark.parametrize("H,G,order", [(1, 1, "together"), (8, 2, "heads"), (10, 2, "together")])
def test_packed_prompts(dtype, D, H, G, order):
    run_prompt([1, 0, 33, 2, 64, 150], H, G, D, dtype, seed=D + H, order=order)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window", [1, 17, 100])
def test_prompts_with_windows(dtype, window):
    run_prompt([5, 300, 129], 4, 2, 64, dtype, window=window, seed=window)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 31, 127, 128, 129, 257, 700])
def test_one_prompt(dtype, n):
    run_prompt([n], 2, 1, 128, dtype, seed=n, pad=0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,window", [(64, 0), (128, 0), (24, 0), (80, 40)])
def test_prompts_whose_waves_have_rows_of_their_own(dtype, D, window):
    """No prompt is named as long beside the chip's load: blocks of 128 rows."""
    run_prompt([1, 0, 33, 2, 64, 400], 8, 2, D, dtype, window=window, seed=D, longest=1)
    run_prompt([129] * 6, 12, 12, D, dtype, window=window, seed=D + 1, longest=1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("longest", [1, 300])
def test_values_that_are_not_finite_reach_only_the_rows_that_see_them(dtype, longest):
    dt, n, H, G, D = DTYPES[dtype], 300, 4, 2, 64
    q = torch.randn((n, H, D), generator=gen(1)).to(dt).cuda()
    k, v = (torch.randn((n, G, D), generator=gen(s)).to(dt).cuda() for s in (2, 3))
    clean = pcg.prompt_attend(q, k, v, torch.tensor([0, n], dtype=torch.int32).cuda(), longest=longest)
    v[200, 0, 5] = -math.inf
    v[250] = math.nan
    out = pcg.prompt_attend(q, k, v, torch.tensor([0, n], dtype=torch.int32).cuda(), longest=longest)
    want = ref.attend_rows(q[:200], k[:200], v[:200], 0, D ** -0.5)
    ref.check(out[:200], want, dt)
    assert torch.isnan(out[250:]).all()
    assert (out[200:250, :2, 5] == -math.inf).all()
    rest = torch.ones(D, dtype=torch.bool)
    rest[5] = False
    # the rows between see the infinity in one column of one shared head
    assert torch.isfinite(out[200:250, 2:]).all() and torch.isfinite(out[200:250, :2][:, :, rest.cuda()]).all()
    assert torch.equal(out[:128], clean[:128])
