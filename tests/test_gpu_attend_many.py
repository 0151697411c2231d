"""Attention of more requests than a wave of the run search takes at a time, of short ones and of ones with several blocks of rows, over the
paged cache and as prompts.  Run with ``-m gpu`` on an MI355X."""
import pytest
import torch

import attention as ref
import paper_2511_13732_amd as pcg
from test_gpu_attend import DTYPES, gen, starts_of

pytestmark = pytest.mark.gpu


def batch(B, lens, new, H, G, D, dt, page_size, seed):
    """Every request's pages dealt at random; (cache, table on the GPU, queries, keys and values on the host, table on the host)."""
    held = [-(-(n + m) // page_size) for n, m in zip(lens, new)]
    total = sum(held)
    order = torch.randperm(total, generator=gen(seed)).to(torch.int32)
    table = torch.full((B, max(held + [1])), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    k, v = (torch.randn((max(total, 1), page_size, G, D), generator=gen(seed + s)).to(dt) for s in (1, 2))
    q = torch.randn((sum(new), H, D), generator=gen(seed + 3)).to(dt)
    return pcg.KvCache(k.cuda(), v.cuda()), table.cuda(), q, k, v, table


def check_some(out, q, k, v, table, lens, new, page_size, which, dt, window=0):
    st, D = starts_of(new), q.shape[2]
    for b in which:
        j = torch.arange(lens[b] + new[b])
        page = table[b, j // page_size].long()
        s = slice(st[b], st[b + 1])
        ref.check(out[s], ref.attend_rows(q[s], k[page, j % page_size], v[page, j % page_size], lens[b], D ** -0.5, window), dt, (b, lens[b], new[b]))


def ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,longest", [(129, 3), (257, 3), (700, 3), (700, 20), (700, 40)])
def test_more_requests_than_lanes(dtype, D, B, longest):
    """Two query heads a shared head: blocks of 32 rows in float32 and 64 in bf16, of 64 and of 128."""
    dt, H, G, ps = DTYPES[dtype], 4, 2, 16
    r = torch.randint(0, 40, (B,), generator=gen(B))
    r[::50] = 900
    lens, new = r.tolist(), torch.randint(0, 4, (B,), generator=gen(D)).tolist()
    cache, table, q, k, v, host = batch(B, lens, new, H, G, D, dt, ps, B)
    out = pcg.cache_attend(cache, q.cuda(), table, ints(lens), ints(starts_of(new)), longest=longest)
    check_some(out, q, k, v, host, lens, new, ps, [*range(0, B, 9), *range(0, B, 50), B - 1], dt)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,longest", [(200, 100), (300, 100), (300, 5), (600, 100)])
@pytest.mark.parametrize("window", [0, 33])
def test_many_requests_with_several_blocks_of_rows(dtype, D, B, longest, window):
    """Every third request has more rows than a block, some empty ones between; with `longest` 5 in blocks of 32 or 64 rows."""
    dt, H, G, ps = DTYPES[dtype], 4, 1, 16
    new = torch.randint(0, 6, (B,), generator=gen(B))
    new[::3] = torch.randint(33, 101, (len(new[::3]),), generator=gen(1))
    new[7::40] = 0
    new = new.tolist()
    lens = torch.randint(0, 200, (B,), generator=gen(D + 1)).tolist()
    cache, table, q, k, v, host = batch(B, lens, new, H, G, D, dt, ps, B)
    out = pcg.cache_attend(cache, q.cuda(), table, ints(lens), ints(starts_of(new)), longest=longest, window=window)
    check_some(out, q, k, v, host, lens, new, ps, [0, 1, *range(3, B, 31), *range(63, B, 64), *range(66, B, 66), B - 2, B - 1], dt, window)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B", [65, 300, 3000])
def test_many_prompts(dtype, B):
    dt, H, G, D = DTYPES[dtype], 4, 1, 64
    new = torch.randint(0, 5, (B,), generator=gen(B))
    new[::9] = torch.randint(30, 90, (len(new[::9]),), generator=gen(2))
    new = new.tolist()
    st = starts_of(new)
    q, k, v = (torch.randn((st[-1], h, D), generator=gen(s)).to(dt) for s, h in ((1, H), (2, G), (3, G)))
    for longest in (1, 90):
        out = pcg.prompt_attend(q.cuda(), k.cuda(), v.cuda(), ints(st), longest=longest)
        for b in [0, 1, *range(9, B, 9 * max(1, B // 300)), *range(2, B, B // 16), B - 1]:
            s = slice(st[b], st[b + 1])
            ref.check(out[s], ref.attend_rows(q[s], k[s], v[s], 0, D ** -0.5), dt, (b, new[b]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_time_of_a_prompt_does_not_grow_with_their_number(dtype):
    """262 144 prompts of one token, some empty: each sees itself, and its output is its value (a weight of one at most a rounding off, a
    sum, a reciprocal and two products).  All of them in 100 ms, fifty times what they take; where every workgroup goes through all
    requests it is a second."""
    dt, B, D = DTYPES[dtype], 1 << 18, 8
    new = torch.ones(B, dtype=torch.int32)
    new[3::7] = 0
    st = torch.cat([torch.zeros(1, dtype=torch.int32), new.cumsum(0).to(torch.int32)]).cuda()
    T = int(st[-1])
    q, k, v = (torch.randn((T, 1, D), generator=gen(s)).to(dt).cuda() for s in (1, 2, 3))
    out = torch.empty_like(q)
    pcg.prompt_attend(q, k, v, st, longest=1, out=out)
    half = torch.finfo(dt).eps / 2
    assert ((out.double() - v.double()).abs() <= (half * 2.02 + 8 * 2.0 ** -23) * v.double().abs()).all()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    pcg.prompt_attend(q, k, v, st, longest=1, out=out)
    b.record()
    b.synchronize()
    assert a.elapsed_time(b) < 100
