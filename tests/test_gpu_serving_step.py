"""The calls around a step's forward pass together, as a serving loop uses them: page table and slots, keys and values into the
cache, attention over it, verification, and what was accepted back into the page table.  Run with ``-m gpu`` on an MI355X."""
import numpy as np
import pytest
import torch

import attention as ref
import paper_2511_13732_amd as pcg
import workloads as W

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


class Layer:
    """One attention layer over a vocabulary: every token at every position has fixed queries, keys and values."""

    def __init__(self, V, H, G, D, dtype, seed):
        g = torch.Generator().manual_seed(seed)
        self.H, self.G, self.D, self.dtype, self.V = H, G, D, dtype, V
        self.token = torch.randn((V, (H + 2 * G) * D), generator=g).cuda()
        self.place = torch.randn((4096, (H + 2 * G) * D), generator=g).cuda()
        self.head = torch.randn((H * D, V), generator=g).cuda() * 3.0 / (H * D) ** 0.5

    def qkv(self, tokens, positions):
        x = (self.token[tokens.long()] + self.place[positions.long()]).to(self.dtype).view(-1, self.H + 2 * self.G, self.D)
        return x[:, :self.H], x[:, self.H:self.H + self.G], x[:, self.H + self.G:]

    def logits(self, out):
        return (out.float().reshape(out.shape[0], -1) @ self.head).to(self.dtype)


@pytest.mark.parametrize("dtype,page_size,H,G,D", [("bf16", 16, 8, 2, 64), ("f32", 7, 6, 3, 72), ("bf16", 32, 12, 1, 128)])
def test_a_serving_loop(dtype, page_size, H, G, D):
    dt, V, B, K = DTYPES[dtype], 1500, 5, 4
    rp, mem = W.random_groups(V, 900, 3, 20, seed=3, cover=False)
    groups = pcg.Groups.from_csr(V, rp, mem, "cuda", reverse=True)
    layer = Layer(V, H, G, D, dt, seed=D)
    gen = torch.Generator().manual_seed(9)
    pages = pcg.Pages.empty(B, 60, page_size, 40, "cuda")
    shape = (60, page_size, G, D)
    cache = pcg.KvCache(torch.full(shape, float("nan"), dtype=dt, device="cuda"), torch.full(shape, float("nan"), dtype=dt, device="cuda"))
    kept = [[] for _ in range(B)]                  # tokens in the cache for good

    def check(b, chunk, out):
        """Rows of request b's chunk against attention over its whole history in double."""
        n = len(kept[b])
        hist = torch.tensor(kept[b] + chunk).cuda()
        q, k, v = layer.qkv(hist, torch.arange(len(hist), device="cuda"))
        ref.check(out, ref.attend_rows(q[n:], k, v, n, D ** -0.5), dt, (b, n))

    # prompts, one place empty
    prompts = [torch.randint(0, V, (n,), generator=gen).tolist() for n in (40, 1, 33, 0, 70)]
    add = torch.tensor([len(p) for p in prompts], dtype=torch.int32).cuda()
    rows = int(add.sum()) + 6
    step = pcg.pages_step(pages, add, max_tokens=rows)
    tokens = torch.tensor([t for p in prompts for t in p] + [0] * 6).cuda()
    q, k, v = layer.qkv(tokens, step.positions)
    pcg.cache_write(cache, k, v, step.slots)
    out = pcg.prompt_attend(q, k, v, step.q_start, longest=70)
    st = step.q_start.tolist()
    for b in range(B):
        check(b, prompts[b], out[st[b]:st[b + 1]])
        kept[b] += prompts[b]
    last = torch.randint(0, V, (B,), generator=gen).cuda()
    commit, ended = None, [False, False, False, True, False]
    for it in range(5):
        add = [K + 1] * B
        fresh = {}
        if it == 2:
            ended[1], add[1] = True, -1
        if it == 3:                                # new prompts in the empty places, in the same pass as the others' chunks
            for b, n in ((1, 37), (3, 2)):
                fresh[b] = torch.randint(0, V, (n,), generator=gen).tolist()
                add[b], ended[b] = n, False
        for b in range(B):
            if ended[b] and add[b] > 0:
                add[b] = 0
        want = [max(a, 0) for a in add]
        step = pcg.pages_step(pages, torch.tensor(add, dtype=torch.int32).cuda(), commit=commit, commit_extra=1,
                              max_tokens=sum(want) + 3)
        assert step.refused.item() == 0
        for b in range(B):
            if add[b] < 0:
                kept[b] = []
        assert pages.lens.tolist() == [len(x) for x in kept] and pages.chunk.tolist() == want
        # the draft proposes on random rows
        draft = torch.randn((B, K, V), generator=gen).to(dt).cuda() * 2
        ptok, pgrp = pcg.propose(groups, draft, seed=1, offset=it)
        chunks = [fresh.get(b) or ([int(last[b])] + ptok[b].tolist() if want[b] else []) for b in range(B)]
        tokens = torch.tensor([t for c in chunks for t in c] + [0] * 3).cuda()
        q, k, v = layer.qkv(tokens, step.positions)
        pcg.cache_write(cache, k, v, step.slots)
        out = pcg.cache_attend(cache, q, pages.block_table, pages.lens, step.q_start, longest=K + 1)
        st = step.q_start.tolist()
        assert st[-1] == sum(want)
        for b in range(B):
            check(b, chunks[b], out[st[b]:st[b + 1]])
        # verification on the target's rows; requests without a step of their own get any
        target = torch.randn((B, K + 1, V), generator=gen).to(dt).cuda()
        steps = [b for b in range(B) if want[b] == K + 1 and b not in fresh]
        for b in steps:
            target[b] = layer.logits(out[st[b]:st[b + 1]])
        res = pcg.verify(groups, target, draft, ptok, pgrp, seed=5, offset=it)
        accepted = res.accept_len.tolist()
        commit = res.accept_len.clone()
        for b in range(B):
            if b in fresh:
                commit[b] = 1 << 20                # the whole prompt stays (no more than the chunk is kept)
                kept[b] += fresh[b]
                last[b] = 7
            elif b in steps:
                kept[b] += chunks[b][:accepted[b] + 1]
                last[b] = res.out_tokens[b, accepted[b]]
                assert res.out_tokens[b, :accepted[b]].tolist() == chunks[b][1:accepted[b] + 1]
    # everything goes back
    pcg.pages_step(pages, -1, max_tokens=0)
    assert pages.free_count.item() == 60 and sorted(pages.free_pages.tolist()) == list(range(60))


def serving_state(B, H, G, D, dt, seed, page_size=16, ctx=300, chunk=5):
    g = torch.Generator().manual_seed(seed)
    blocks = -(-(ctx + 8 * chunk) // page_size)
    pages = pcg.Pages.empty(B, B * blocks, page_size, blocks, "cuda")
    shape = (B * blocks, page_size, G, D)
    cache = pcg.KvCache(torch.randn(shape, generator=g).to(dt).cuda(), torch.randn(shape, generator=g).to(dt).cuda())
    lens = torch.randint(1, ctx, (B,), generator=g).to(torch.int32)
    pcg.pages_step(pages, lens.cuda(), max_tokens=int(lens.sum()))
    x = torch.randn((B * chunk, H + 2 * G, D), generator=g).to(dt).cuda()
    return pages, cache, x


@pytest.mark.parametrize("dtype,H,G,D,chunk", [("bf16", 8, 2, 128, 5), ("f32", 4, 4, 64, 1), ("bf16", 8, 1, 64, 40)])
def test_a_recorded_step_replays_to_the_eager_result(dtype, H, G, D, chunk):
    """Page table, write, attention and the state that moves on with every replay; eager work and synchronisations between."""
    dt, B = DTYPES[dtype], 6
    pages, cache, x = serving_state(B, H, G, D, dt, 1, chunk=chunk, ctx=700)
    other = pcg.Pages(pages.block_table.clone(), pages.free_pages.clone(), pages.state.clone(), pages.page_size)
    cache2 = pcg.KvCache(cache.k.clone(), cache.v.clone())
    rows = B * chunk
    accept = torch.zeros(B, dtype=torch.int32, device="cuda")
    ws = torch.empty(pcg.cache_attend_workspace_bytes(B, rows, H, G, D, chunk), dtype=torch.uint8, device="cuda")

    def buffers():
        return pcg.pages_step_outputs(B, rows, "cuda"), torch.zeros((rows, H, D), dtype=dt, device="cuda"), \
            torch.zeros((rows, H, D), dtype=dt, device="cuda")

    def step(pg, kv, bufs):
        o, out, prompt = bufs
        pcg.pages_step(pg, chunk, commit=accept, commit_extra=1, max_tokens=rows, out=o)
        pcg.cache_write(kv, x[:, H:H + G], x[:, H + G:], o.slots)
        pcg.cache_attend(kv, x[:, :H], pg.block_table, pg.lens, o.q_start, longest=chunk, out=out, workspace=ws)
        pcg.prompt_attend(x[:, :H], x[:, H:H + G], x[:, H + G:], o.q_start, longest=chunk, out=prompt)

    got, want = buffers(), buffers()
    side = torch.cuda.Stream()
    saved = pages.state.clone(), pages.block_table.clone(), pages.free_pages.clone(), cache.k.clone(), cache.v.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step(pages, cache, got)                       # warm-up outside the capture
    side.synchronize()
    for t, s in zip((pages.state, pages.block_table, pages.free_pages, cache.k, cache.v), saved):
        t.copy_(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(pages, cache, got)
    for it in range(5):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(it)).to(dt))
        accept.copy_(torch.randint(0, chunk, (B,), generator=torch.Generator().manual_seed(it)).to(torch.int32))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        ws.fill_(255)                                 # eager work between the replays
        step(other, cache2, want)
        torch.cuda.synchronize()
        assert torch.equal(pages.state, other.state)
        for a, b in ((got[0].q_start, want[0].q_start), (got[0].slots, want[0].slots), (got[0].positions, want[0].positions),
                     (got[1], want[1]), (got[2], want[2]), (cache.k, cache2.k), (cache.v, cache2.v)):
            assert torch.equal(a, b)
        for b in range(B):
            n = int(pages.held[b])
            assert torch.equal(pages.block_table[b, :n], other.block_table[b, :n])


def test_calls_on_two_streams_do_not_disturb_each_other():
    dt, H, G, D, chunk, B = torch.bfloat16, 8, 2, 128, 6, 12
    jobs = []
    for seed in (1, 2):
        pages, cache, x = serving_state(B, H, G, D, dt, seed, ctx=3000, chunk=chunk)
        o = pcg.pages_step(pages, chunk, max_tokens=B * chunk)
        pcg.cache_write(cache, x[:, H:H + G], x[:, H + G:], o.slots)
        ws = torch.full((pcg.cache_attend_workspace_bytes(B, B * chunk, H, G, D, chunk),), 255, dtype=torch.uint8, device="cuda")
        jobs.append((pages, cache, x, o, ws))
    torch.cuda.synchronize()

    def one(j, rounds):
        pages, cache, x, o, ws = jobs[j]
        res = []
        for _ in range(rounds):
            res.append(pcg.cache_attend(cache, x[:, :H], pages.block_table, pages.lens, o.q_start, longest=chunk, workspace=ws))
            res.append(pcg.prompt_attend(x[:, :H], x[:, H:H + G], x[:, H + G:], o.q_start, longest=chunk))
        return res

    want = [one(0, 1), one(1, 1)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [None, None]
    for j in (0, 1):
        with torch.cuda.stream(streams[j]):
            got[j] = one(j, 12)
    for s in streams:
        s.synchronize()
    for j in (0, 1):
        for i, t in enumerate(got[j]):
            assert torch.equal(t, want[j][i % 2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("chunk,ctx", [(1, 2000), (9, 5000), (60, 900)])
def test_the_same_call_gives_the_same_bits_whatever_is_in_the_workspace(dtype, chunk, ctx):
    dt, H, G, D, B = DTYPES[dtype], 8, 2, 64, 3
    pages, cache, x = serving_state(B, H, G, D, dt, chunk, ctx=ctx, chunk=chunk)
    o = pcg.pages_step(pages, chunk, max_tokens=B * chunk)
    outs = []
    for fill in (0, 255, 127):
        ws = torch.full((pcg.cache_attend_workspace_bytes(B, B * chunk, H, G, D, chunk),), fill, dtype=torch.uint8, device="cuda")
        outs.append(pcg.cache_attend(cache, x[:, :H], pages.block_table, pages.lens, o.q_start, longest=chunk, workspace=ws))
    outs.append(pcg.cache_attend(cache, x[:, :H], pages.block_table, pages.lens, o.q_start, longest=chunk))
    for t in outs[1:]:
        assert torch.equal(t, outs[0])


def test_many_requests():
    """More requests than a workgroup has threads, most of them short, some empty."""
    B, H, G, D, dt = 700, 2, 1, 64, torch.bfloat16
    g = torch.Generator().manual_seed(4)
    lens = torch.randint(0, 40, (B,), generator=g).to(torch.int32)
    lens[::50] = 900
    new = torch.randint(0, 4, (B,), generator=g).to(torch.int32)
    pages = pcg.Pages.empty(B, 5000, 16, 60, "cuda")
    cache = pcg.KvCache(*(torch.randn((5000, 16, G, D), generator=g).to(dt).cuda() for _ in range(2)))
    pcg.pages_step(pages, lens.cuda(), max_tokens=int(lens.sum()))
    o = pcg.pages_step(pages, new.cuda(), max_tokens=int(new.sum()))
    q = torch.randn((int(new.sum()), H, D), generator=g).to(dt).cuda()
    st, table = o.q_start.tolist(), pages.block_table.cpu()
    k, v = cache.k.cpu(), cache.v.cpu()
    for longest in (3, 40):                            # 32 rows a workgroup, 128 rows a workgroup
        out = pcg.cache_attend(cache, q, pages.block_table, pages.lens, o.q_start, longest=longest)
        for b in [*range(0, B, 23), *range(0, B, 50)]:
            n, m = int(lens[b]), int(new[b])
            j = torch.arange(n + m)
            page = table[b, j // 16].long()
            ref.check(out[st[b]:st[b + 1]], ref.attend_rows(q[st[b]:st[b + 1]], k[page, j % 16], v[page, j % 16], n, D ** -0.5), dt,
                      (b, n, m))
    # and as prompts of their own
    kv = torch.randn((int(new.sum()), 2 * G, D), generator=g).to(dt).cuda()
    out = pcg.prompt_attend(q, kv[:, :G], kv[:, G:], o.q_start, longest=3)
    for b in range(0, B, 11):
        s = slice(st[b], st[b + 1])
        ref.check(out[s], ref.attend_rows(q[s], kv[s, :G], kv[s, G:], 0, D ** -0.5), dt, b)
