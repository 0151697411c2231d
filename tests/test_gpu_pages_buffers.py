"""Buffers of a step that are kept from call to call with different limits, and batches whose slots a second launch fills
(pcg_pages_step).  Run with ``-m gpu`` on an MI355X."""
import random

import pytest
import torch

import attention as ref
import paper_2511_13732_amd as pcg
from test_gpu_pages import compare, tolists, whole

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [40, 5000])
def test_a_buffer_with_more_rows_than_the_step_may_have(rows):
    """Rows behind the limit are no request's, whatever an earlier step left there: written as a whole, the batch leaves the cache alone."""
    B, G, D, page_size = 4, 1, 8, 4
    pages = pcg.Pages.empty(B, 40, page_size, 10, "cuda")
    cache = pcg.KvCache(*(torch.zeros((40, page_size, G, D), device="cuda") for _ in range(2)))
    out = pcg.pages_step_outputs(B, rows, "cuda")
    out.slots.fill_(3)
    out.positions.fill_(12345)
    for limit, add in ((rows, 9), (20, 5), (7, 1), (0, 0)):
        step = pcg.pages_step(pages, add, max_tokens=limit, out=out)
        assert step is out
        n = int(step.q_start[-1])
        assert n == B * add
        assert (step.slots[:n] >= 0).all() and (step.slots[n:] == -1).all() and (step.positions[n:] == 0).all()
        before = cache.k.clone(), cache.v.clone()
        new = torch.full((rows, G, D), float(limit + 1), device="cuda")
        pcg.cache_write(cache, new, new, step.slots)
        for x, was in zip((cache.k, cache.v), before):
            changed = (x != was).flatten(0, 1).any(-1).any(-1).nonzero().flatten().tolist()
            assert sorted(changed) == sorted(step.slots[:n].tolist())


def test_a_recorded_step_fills_the_rows_behind_its_limit():
    B = 3
    pages = pcg.Pages.empty(B, 60, 4, 20, "cuda")
    out = pcg.pages_step_outputs(B, 50, "cuda")
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        pcg.pages_step(pages, 2, max_tokens=8, out=out)
    for it in range(4):
        out.slots.fill_(7)
        out.positions.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert (out.slots[:6] >= 0).all() and (out.slots[6:] == -1).all()
        assert out.positions.tolist() == [2 * it, 2 * it + 1] * 3 + [0] * 44


@pytest.mark.parametrize("B,page_size,num_pages,max_blocks,max_tokens,steps",
                         [(64, 16, 900, 40, 3000, 6), (1, 16, 400, 300, 2600, 6), (256, 2, 5000, 40, 4000, 4), (256, 16, 2000, 60, 4097, 4),
                          (65536, 4, 90000, 3, 70000, 2)])
def test_slots_that_a_second_launch_fills(B, page_size, num_pages, max_blocks, max_tokens, steps):
    rng = random.Random(B + max_tokens)
    pages = pcg.Pages.empty(B, num_pages, page_size, max_blocks, "cuda")
    for step in range(steps):
        state = pages.state.tolist()
        add = [rng.randint(0, 2 * max_tokens // B + 1) if rng.random() < 0.9 else -1 for _ in range(B)]
        commit = [rng.randint(0, max(c, 1)) for c in state[2 * B:3 * B]]
        want = ref.pages_step(*tolists(pages), page_size, commit, 1, add, max_tokens)
        out = pcg.pages_step(pages, torch.tensor(add, dtype=torch.int32).cuda(), max_tokens=max_tokens,
                             commit=torch.tensor(commit, dtype=torch.int32).cuda(), commit_extra=1)
        compare(pages, out, want, max_tokens)
        whole(pages)
