"""Rotated rows into the cache, of 16 bits and of 4, and attention over it together, as a serving loop uses them.  Run with ``-m gpu`` on
an MI355X.

Attention is compared with its definition in double over what the definitions of rotation and of codes make of every token: both are exact
up to the last rounding (tests/cache4.py), so that tolerances are those of attention alone."""
import pytest
import torch

import attention
import cache4 as ref
import paper_2511_13732_amd as pcg
import workloads as W
from test_gpu_attend4 import check, make_cache, starts_of

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def gen(seed):
    return torch.Generator().manual_seed(seed)


class Layer:
    """One attention layer over a vocabulary: every token has fixed queries, keys and values, which know nothing of its position."""

    def __init__(self, V, H, G, D, dtype, rotation, four, seed):
        self.H, self.G, self.D, self.dtype, self.rotation, self.four = H, G, D, dtype, rotation, four
        self.token = torch.randn((V, H + 2 * G, D), generator=gen(seed)).to(dtype).cuda()
        self.head = torch.randn((H * D, V), generator=gen(seed + 1)).cuda() * 3.0 / (H * D) ** 0.5

    def qkv(self, tokens):
        x = self.token[tokens.long()]
        return x[:, :self.H], x[:, self.H:self.H + self.G], x[:, self.H + self.G:]

    def logits(self, out):
        return (out.float().reshape(out.shape[0], -1) @ self.head).to(self.dtype)

    def held(self, tokens):
        """Queries of a request's tokens as attention gets them, and keys and values as the cache holds them, from the definitions."""
        turn = self.rotation.table.cpu()[:len(tokens)]
        q, k, v = (x.cpu() for x in self.qkv(tokens))
        q, k = (ref.rotate(x, turn, self.rotation.interleaved) for x in (q, k))
        if self.four:
            k, v = (ref.values(*ref.quantise(x.float())) for x in (k, v))
        else:
            k = k.to(self.dtype)
        return q.to(self.dtype), k, v

    def new_cache(self, pages, page_size):
        if self.four:
            c = pcg.KvCache4.empty(pages, page_size, self.G, self.D, "cuda")
            c.scales.fill_(float("nan"))
            return c
        return pcg.KvCache(*(torch.full((pages, page_size, self.G, self.D), float("nan"), dtype=self.dtype, device="cuda") for _ in range(2)))

    def bring(self, cache, tokens, step):
        q, k, v = self.qkv(tokens)
        call = pcg.cache4_append if self.four else pcg.cache_append
        return call(cache, k, v, step.slots, rotation=self.rotation, positions=step.positions, q=q)

    def attend(self, cache, q, pages, step, longest):
        call = pcg.cache4_attend if self.four else pcg.cache_attend
        return call(cache, q, pages.block_table, pages.lens, step.q_start, longest=longest)


@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("dtype,page_size,H,G,D,dim,interleaved", [("bf16", 16, 8, 2, 64, 64, False), ("f32", 7, 6, 3, 72, 40, True),
                                                                  ("bf16", 32, 12, 1, 128, 128, True)])
def test_a_serving_loop(four, dtype, page_size, H, G, D, dim, interleaved):
    dt, V, B, K = DTYPES[dtype], 1500, 5, 4
    rp, mem = W.random_groups(V, 900, 3, 20, seed=3, cover=False)
    groups = pcg.Groups.from_csr(V, rp, mem, "cuda", reverse=True)
    layer = Layer(V, H, G, D, dt, pcg.Rotation.of(400, dim, "cuda", interleaved=interleaved), four, seed=D)
    g = gen(9)
    pages = pcg.Pages.empty(B, 60, page_size, 40, "cuda")
    cache = layer.new_cache(60, page_size)
    kept = [[] for _ in range(B)]                  # tokens in the cache for good

    def compare(b, chunk, out):
        n = len(kept[b])
        if not chunk:
            return
        q, k, v = layer.held(torch.tensor(kept[b] + chunk).cuda())
        want = attention.attend_rows(q[n:], k, v, n, D ** -0.5)
        (check if four else attention.check)(out, want, dt, (b, n))

    # prompts, one place empty
    prompts = [torch.randint(0, V, (n,), generator=g).tolist() for n in (40, 1, 33, 0, 70)]
    step = pcg.pages_step(pages, torch.tensor([len(p) for p in prompts], dtype=torch.int32).cuda(), max_tokens=150)
    out = layer.attend(cache, layer.bring(cache, torch.tensor([t for p in prompts for t in p] + [0] * 6).cuda(), step), pages, step, 70)
    st = step.q_start.tolist()
    for b in range(B):
        compare(b, prompts[b], out[st[b]:st[b + 1]])
        kept[b] += prompts[b]
    last = torch.randint(0, V, (B,), generator=g).cuda()
    commit, ended = None, [False, False, False, True, False]
    for it in range(4):
        add, fresh = [K + 1] * B, {}
        if it == 2:                                # one ends, a prompt comes into the empty place
            ended[1], add[1] = True, -1
            fresh[3] = torch.randint(0, V, (21,), generator=g).tolist()
            add[3], ended[3] = 21, False
        add = [0 if ended[b] and a > 0 else a for b, a in enumerate(add)]
        want = [max(a, 0) for a in add]
        step = pcg.pages_step(pages, torch.tensor(add, dtype=torch.int32).cuda(), commit=commit, commit_extra=1, max_tokens=sum(want) + 3)
        if it == 2:
            kept[1] = []
        assert step.refused.item() == 0 and pages.lens.tolist() == [len(x) for x in kept]
        draft = torch.randn((B, K, V), generator=g).to(dt).cuda() * 2
        ptok, pgrp = pcg.propose(groups, draft, seed=1, offset=it)
        chunks = [fresh.get(b) or ([int(last[b])] + ptok[b].tolist() if want[b] else []) for b in range(B)]
        q = layer.bring(cache, torch.tensor([t for c in chunks for t in c] + [0] * 3).cuda(), step)
        out = layer.attend(cache, q, pages, step, K + 1)
        st = step.q_start.tolist()
        for b in range(B):
            compare(b, chunks[b], out[st[b]:st[b + 1]])
        target = torch.randn((B, K + 1, V), generator=g).to(dt).cuda()
        steps = [b for b in range(B) if want[b] == K + 1 and b not in fresh]
        for b in steps:
            target[b] = layer.logits(out[st[b]:st[b + 1]])
        res = pcg.verify(groups, target, draft, ptok, pgrp, seed=5, offset=it)
        commit, accepted = res.accept_len.clone(), res.accept_len.tolist()
        for b in range(B):
            if b in fresh:
                commit[b] = 1 << 20
                kept[b] += fresh[b]
                last[b] = 7
            elif b in steps:
                kept[b] += chunks[b][:accepted[b] + 1]
                last[b] = res.out_tokens[b, accepted[b]]


def state(B, H, G, D, dt, seed, page_size=16, ctx=300, chunk=5, layout="heads"):
    """Requests with some tokens each in a cache of 4 bits that was filled by the call itself, and rows for the next chunk."""
    g = gen(seed)
    blocks = -(-(ctx + 8 * chunk) // page_size)
    pages = pcg.Pages.empty(B, B * blocks, page_size, blocks, "cuda")
    cache = pcg.KvCache4.empty(B * blocks, page_size, G, D, "cuda")
    if layout == "slots":
        cache = pcg.KvCache4(cache.k.contiguous(), cache.v.contiguous(), cache.scales.contiguous(), D)
    lens = torch.randint(1, ctx, (B,), generator=g).to(torch.int32)
    step = pcg.pages_step(pages, lens.cuda(), max_tokens=int(lens.sum()))
    rotation = pcg.Rotation.of(ctx + 8 * chunk, D, "cuda")
    k, v = (torch.randn((int(lens.sum()), G, D), generator=g).to(dt).cuda() for _ in range(2))
    pcg.cache4_append(cache, k, v, step.slots, rotation=rotation, positions=step.positions)
    x = torch.randn((B * chunk, H + 2 * G, D), generator=g).to(dt).cuda()
    return pages, cache, rotation, x


def copied(cache):
    """The same cache in memory of its own, strides and all."""
    return pcg.KvCache4(cache.k.clone(), cache.v.clone(), cache.scales.clone(), cache.head_dim)


@pytest.mark.parametrize("dtype,H,G,D,chunk,layout", [("bf16", 8, 2, 128, 5, "slots"), ("f32", 4, 4, 64, 1, "heads"), ("bf16", 8, 1, 64, 40, "heads")])
def test_a_recorded_step_replays_to_the_eager_result(dtype, H, G, D, chunk, layout):
    """Page table, rows into the cache, attention, and the state that moves on with every replay; eager work and synchronisations between,
    in the same workspace."""
    dt, B = DTYPES[dtype], 6
    pages, cache, rotation, x = state(B, H, G, D, dt, 1, chunk=chunk, ctx=700, layout=layout)
    other = pcg.Pages(pages.block_table.clone(), pages.free_pages.clone(), pages.state.clone(), pages.page_size)
    cache2, rows = copied(cache), B * chunk
    accept = torch.zeros(B, dtype=torch.int32, device="cuda")
    ws = torch.empty(pcg.cache4_attend_workspace_bytes(B, rows, H, G, D, chunk), dtype=torch.uint8, device="cuda")

    def buffers():
        return (pcg.pages_step_outputs(B, rows, "cuda"), *(torch.zeros((rows, H, D), dtype=dt, device="cuda") for _ in range(2)))

    def step(pg, kv, o, turned, out):
        pcg.pages_step(pg, chunk, commit=accept, commit_extra=1, max_tokens=rows, out=o)
        pcg.cache4_append(kv, x[:, H:H + G], x[:, H + G:], o.slots, rotation=rotation, positions=o.positions, q=x[:, :H], q_out=turned)
        pcg.cache4_attend(kv, turned, pg.block_table, pg.lens, o.q_start, longest=chunk, out=out, workspace=ws)

    got, want = buffers(), buffers()
    side = torch.cuda.Stream()
    live = (pages.state, pages.block_table, pages.free_pages, cache.k, cache.v, cache.scales)
    saved = [t.clone() for t in live]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step(pages, cache, *got)                      # warm-up outside the capture
    side.synchronize()
    for t, s in zip(live, saved):
        t.copy_(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(pages, cache, *got)
    for it in range(5):
        x.copy_(torch.randn(x.shape, generator=gen(it)).to(dt))
        accept.copy_(torch.randint(0, chunk, (B,), generator=gen(it)).to(torch.int32))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        ws.fill_(255)                                 # eager work between the replays
        step(other, cache2, *want)
        torch.cuda.synchronize()
        assert torch.equal(pages.state, other.state) and torch.equal(got[0].slots, want[0].slots)
        for a, b in ((got[1], want[1]), (got[2], want[2]), (cache.k, cache2.k), (cache.v, cache2.v),
                     (cache.scales.view(torch.int16), cache2.scales.view(torch.int16))):
            assert torch.equal(a, b)
        assert (got[2] != 0).any()


def test_calls_on_two_streams_do_not_disturb_each_other():
    dt, H, G, D, chunk, B = torch.bfloat16, 8, 2, 128, 6, 12
    jobs = []
    for seed in (1, 2):
        pages, cache, rotation, x = state(B, H, G, D, dt, seed, ctx=2500, chunk=chunk, layout=("heads", "slots")[seed - 1])
        o = pcg.pages_step(pages, chunk, max_tokens=B * chunk)
        ws = torch.full((pcg.cache4_attend_workspace_bytes(B, B * chunk, H, G, D, chunk),), 255, dtype=torch.uint8, device="cuda")
        jobs.append((pages, cache, rotation, x, o, ws))
    torch.cuda.synchronize()

    def one(j, rounds):
        pages, cache, rotation, x, o, ws = jobs[j]
        res = []
        for _ in range(rounds):
            q = pcg.cache4_append(cache, x[:, H:H + G], x[:, H + G:], o.slots, rotation=rotation, positions=o.positions, q=x[:, :H])
            res.append(pcg.cache4_attend(cache, q, pages.block_table, pages.lens, o.q_start, longest=chunk, workspace=ws))
        return res

    alone = [one(j, 1)[0] for j in (0, 1)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    results = [[], []]
    for _ in range(10):
        for j, s in enumerate(streams):
            with torch.cuda.stream(s):
                results[j] += one(j, 2)
    torch.cuda.synchronize()
    for j in (0, 1):
        assert all(torch.equal(r, alone[j]) for r in results[j])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_two_recorded_calls_share_a_workspace(dtype):
    """One after the other, in either order, with other sizes."""
    dt, H, G, D = DTYPES[dtype], 8, 2, 64
    jobs, ws = [], torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    for seed, chunk, B in ((1, 3, 9), (2, 30, 4)):
        pages, cache, _, x = state(B, H, G, D, dt, seed, ctx=1200, chunk=chunk)
        o = pcg.pages_step(pages, chunk, max_tokens=B * chunk)
        q, out = x[:, :H], torch.zeros((B * chunk, H, D), dtype=dt, device="cuda")

        def call(out, pages=pages, cache=cache, q=q, o=o, chunk=chunk):
            pcg.cache4_attend(cache, q, pages.block_table, pages.lens, o.q_start, longest=chunk, out=out, workspace=ws)
        call(out)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(out)
        jobs.append((graph, out, out.clone(), call))       # a replay reads what the call was made with
    for order in ((0, 1), (1, 0), (0, 0), (1, 1)):
        for _, out, _, _ in jobs:
            out.zero_()
        for j in order:
            jobs[j][0].replay()
        torch.cuda.synchronize()
        for j in set(order):
            assert torch.equal(jobs[j][1], jobs[j][2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["heads", "slots"])
@pytest.mark.parametrize("longest_chunk", [1, 13, 26])
def test_many_requests(dtype, layout, longest_chunk):
    """More requests than lanes, with and without rows, some with none in the cache; heads in pairs where their slots lie next to each other."""
    dt, H, G, D = DTYPES[dtype], 8, 2, 128
    g = gen(longest_chunk)
    ctx = torch.randint(0, 90, (301,), generator=g).tolist()
    new = [0 if n % 5 == 0 else min(n, longest_chunk) for n in torch.randint(0, 30, (301,), generator=g).tolist()]
    ctx[0], ctx[300], new[300] = 0, 3001, 2
    cache, table, rows = make_cache([c + n for c, n in zip(ctx, new)], 16, G, D, layout, 5)
    st = starts_of(new)
    q = (1.5 * torch.randn((st[-1], H, D), generator=g)).to(dt).cuda()
    out = pcg.cache4_attend(cache, q, table, *(torch.tensor(x, dtype=torch.int32).cuda() for x in (ctx, st)), longest=longest_chunk)
    for b in list(range(0, 301, 7)) + [300]:
        if new[b]:
            check(out[st[b]:st[b + 1]], attention.attend_rows(q[st[b]:st[b + 1]], *rows[b], ctx[b], D ** -0.5), dt, b)
    assert (out == 0).all(dim=(1, 2)).sum() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,G,D,window", [(4, 4, 64, 0), (8, 2, 128, 0), (8, 2, 128, 333)])
def test_long_pieces(dtype, H, G, D, window):
    """Pieces of prompts of many row blocks a head, next to a request that decodes; outputs between other columns."""
    dt = DTYPES[dtype]
    ctx, new = [300, 40, 0], [257, 1, 500]
    cache, table, rows = make_cache([c + n for c, n in zip(ctx, new)], 32, G, D, "heads", 6)
    st = starts_of(new)
    q = (1.5 * torch.randn((st[-1], H, D), generator=gen(1))).to(dt).cuda()
    wide = torch.full((st[-1] + 2, H + 3, D + 8), 55.0, dtype=dt, device="cuda")
    out = wide[1:-1, 2:2 + H, :D]
    pcg.cache4_attend(cache, q, table, *(torch.tensor(x, dtype=torch.int32).cuda() for x in (ctx, st)), longest=500, window=window, out=out)
    for b in range(3):
        check(out[st[b]:st[b + 1]], attention.attend_rows(q[st[b]:st[b + 1]], *rows[b], ctx[b], D ** -0.5, window), dt, b)
    out.fill_(55.0)
    assert (wide == 55.0).all()


@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("page_size", [16, 12])
def test_pages_far_behind_each_other(four, page_size):
    """Offsets that do not fit 32 bits: pages a megabyte apart, in a cache of five gigabytes."""
    dt, H, G, D, n = torch.bfloat16, 8, 2, 128, 100
    apart, count = 1 << 20, 5000
    room = torch.empty((count, apart), dtype=torch.uint8, device="cuda")
    row = D // 2 if four else 2 * D

    def view(at, width):
        return room.as_strided((count, page_size, G, width), (apart, G * row, row, 1), at)
    if four:
        scales = room.view(torch.bfloat16).as_strided((count, page_size, G, 2), (apart // 2, G * 2, 2, 1), 40000)
        cache = pcg.KvCache4(view(0, row), view(1 << 18, row), scales, D)
    else:
        cache = pcg.KvCache(view(0, row).view(dt), view(1 << 18, row).view(dt))
    blocks = -(-n // page_size)
    pages = torch.randperm(1500, generator=gen(1))[:blocks] + 3500
    table = pages.to(torch.int32)[None].cuda()
    at = torch.arange(n)
    slots = (pages[at // page_size] * page_size + at % page_size).to(torch.int32).cuda()
    rotation = pcg.Rotation.of(n, D, "cuda")
    q, k, v = (torch.randn((n, h, D), generator=gen(h)).to(dt).cuda() for h in (H, G, G + 1))
    v = v[:, :G]
    q_out = (pcg.cache4_append if four else pcg.cache_append)(cache, k, v, slots, rotation=rotation, positions=at.to(torch.int32).cuda(), q=q)
    turn = rotation.table.cpu()
    kk, vv = ref.rotate(k, turn, False), v.cpu().float()
    if four:
        kk, vv = (ref.values(*ref.quantise(x)) for x in (kk, vv))
        for got, x in zip(pcg.cache4_read(cache, slots, dtype=torch.float32), (kk, vv)):
            assert torch.equal(got.cpu().double(), x)
    else:
        kk = kk.to(dt)
    lens, starts = (torch.tensor(x, dtype=torch.int32).cuda() for x in ([n - 3], [0, 3]))
    out = (pcg.cache4_attend if four else pcg.cache_attend)(cache, q_out[n - 3:], table, lens, starts, longest=3)
    (check if four else attention.check)(out, attention.attend_rows(q_out[n - 3:], kk, vv, n - 3, D ** -0.5), dt)


@pytest.mark.parametrize("apart", [1 << 27, (1 << 27) - 16])
def test_slots_far_behind_each_other(apart):
    """Slots of a page so far from each other that 16 of them do not fit 32 bits, and just fit."""
    dt, H, G, D, n, page_size = torch.bfloat16, 4, 2, 64, 40, 16
    row = D // 2
    room = torch.empty(3 * page_size * apart, dtype=torch.uint8, device="cuda")

    def view(x, at, width, unit):
        return x.as_strided((3, page_size, G, width), (page_size * apart // unit, apart // unit, row // unit, 1), at // unit)
    cache = pcg.KvCache4(view(room, 0, row, 1), view(room, 1024, row, 1), view(room.view(torch.bfloat16), 2048, 2, 2), D)
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32).cuda()
    at = torch.arange(n)
    slots = (table[0].cpu().long()[at // page_size] * page_size + at % page_size).to(torch.int32).cuda()
    rotation = pcg.Rotation.of(n, D, "cuda")
    q, k, v = (torch.randn((n, h, D), generator=gen(i)).to(dt).cuda() for i, h in enumerate((H, G, G)))
    q_out = pcg.cache4_append(cache, k, v, slots, rotation=rotation, positions=at.to(torch.int32).cuda(), q=q)
    kk, vv = (ref.values(*ref.quantise(x)) for x in (ref.rotate(k, rotation.table.cpu(), False), v.cpu().float()))
    for got, x in zip(pcg.cache4_read(cache, slots, dtype=torch.float32), (kk, vv)):
        assert torch.equal(got.cpu().double(), x)
    lens, starts = (torch.tensor(x, dtype=torch.int32).cuda() for x in ([n - 3], [0, 3]))
    out = pcg.cache4_attend(cache, q_out[n - 3:], table, lens, starts, longest=3)
    check(out, attention.attend_rows(q_out[n - 3:], kk, vv, n - 3, D ** -0.5), dt)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_windows_longer_than_any_request(dtype):
    """As far as numbers of 32 bits go: what every row sees is what it sees without one, to the bit."""
    dt, H, G, D = DTYPES[dtype], 8, 2, 64
    ctx, new = [0, 700, 90], [40, 3, 12]
    cache, table, _ = make_cache([c + n for c, n in zip(ctx, new)], 16, G, D, "heads", 9)
    st = starts_of(new)
    q = (1.5 * torch.randn((st[-1], H, D), generator=gen(1))).to(dt).cuda()
    lens, starts = (torch.tensor(x, dtype=torch.int32).cuda() for x in (ctx, st))
    want = pcg.cache4_attend(cache, q, table, lens, starts, longest=40)
    for window in (703, (1 << 31) - 1, (1 << 31) - 2, (1 << 31) - 64, 1 << 30):
        assert torch.equal(pcg.cache4_attend(cache, q, table, lens, starts, longest=40, window=window), want), window


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page_size,D,window", [(16, 128, 0), (7, 40, 0), (32, 64, 50), (5, 72, 70)])
@pytest.mark.parametrize("longest", [10, 30])
def test_many_shared_heads(dtype, page_size, D, window, longest):
    """Work for the whole chip out of few requests, 20 and 60 rows a shared head at most."""
    dt, H, G = DTYPES[dtype], 256, 128
    ctx, new = [90, 0, 41, 130], [longest, 1, 9, longest - 2]
    cache, table, rows = make_cache([c + n for c, n in zip(ctx, new)], page_size, G, D, "heads", D)
    st = starts_of(new)
    q = (1.5 * torch.randn((st[-1], H, D), generator=gen(2))).to(dt).cuda()
    lens, starts = (torch.tensor(x, dtype=torch.int32).cuda() for x in (ctx, st))

    def call():
        return pcg.cache4_attend(cache, q, table, lens, starts, longest=longest, window=window)
    out = call()
    for b in range(4):
        at = list(range(st[b], st[b + 1], 4)) + [st[b + 1] - 1]
        for t in at:
            check(out[t:t + 1], attention.attend_rows(q[t:t + 1], *rows[b], ctx[b] + t - st[b], D ** -0.5, window), dt, (b, t))
    # the last token's key or value of one shared head is NaN: its own row's heads there are, and nothing else changes
    for i, head in ((0, 5), (1, 127)):
        j = ctx[3] + new[3] - 1
        where = (int(table[3, j // page_size]), j % page_size, head, i)
        was = cache.scales[where].clone()
        cache.scales[where] = float("nan")
        got = call()
        struck = torch.zeros(got.shape, dtype=torch.bool, device="cuda")
        struck[-1, 2 * head:2 * head + 2] = True
        assert torch.isnan(got[struck]).all() and torch.equal(got[~struck], out[~struck])
        cache.scales[where] = was
