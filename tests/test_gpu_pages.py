"""Page table, slot map and cache rows (pcg_pages_step, pcg_cache_write) against the same in plain Python; every value has to be
equal.  Run with ``-m gpu`` on an MI355X."""
import random

import pytest
import torch

import attention as ref
import paper_2511_13732_amd as pcg

pytestmark = pytest.mark.gpu


def tolists(pages):
    return pages.block_table.tolist(), pages.free_pages.tolist(), pages.state.tolist()


def compare(pages, out, want, max_tokens):
    state, table, free, q_start, slots, positions, refused = want
    assert pages.state.tolist() == state
    B = pages.B
    for b in range(B):                      # what stands behind the pages held means nothing
        held = state[B + b]
        assert pages.block_table[b, :held].tolist() == table[b][:held], b
    count = state[3 * B]
    assert pages.free_pages[:count].tolist() == free[:count]
    assert out.q_start.tolist() == q_start
    assert out.slots[:max_tokens].tolist() == slots and out.positions[:max_tokens].tolist() == positions
    assert out.refused.item() == refused


def whole(pages):
    """Every page is held once or free once."""
    B, st = pages.B, pages.state.tolist()
    seen = pages.free_pages[:st[3 * B]].tolist()
    for b in range(B):
        seen += pages.block_table[b, :st[B + b]].tolist()
    assert sorted(seen) == list(range(pages.num_pages))


@pytest.mark.parametrize("B,page_size,num_pages,max_blocks,max_tokens,steps",
                         [(1, 16, 40, 30, 9, 12), (5, 4, 60, 20, 40, 20), (64, 16, 900, 40, 600, 8), (64, 1, 1200, 40, 300, 8),
                          (300, 8, 1500, 12, 5000, 6), (1024, 8, 4000, 9, 9000, 4), (1025, 8, 4000, 9, 9000, 4),
                          (2600, 3, 6000, 9, 4000, 4)])
def test_steps_of_a_pool(B, page_size, num_pages, max_blocks, max_tokens, steps):
    rng = random.Random(B + num_pages)
    pages = pcg.Pages.empty(B, num_pages, page_size, max_blocks, "cuda")
    for step in range(steps):
        state = pages.state.tolist()
        add = [rng.choice([0, 1, 4, 9, rng.randint(0, 3 * page_size * max_blocks // 2)]) if rng.random() < 0.9 else -rng.randint(1, 9)
               for _ in range(B)]
        commit = None if step % 3 == 2 else [rng.randint(-2, max(c, 1)) for c in state[2 * B:3 * B]]
        each = step % 4 != 3
        if not each:
            add = [3] * B
        want = ref.pages_step(*tolists(pages), page_size, commit, step % 2, add, max_tokens)
        out = pcg.pages_step(pages, torch.tensor(add, dtype=torch.int32).cuda() if each else 3, max_tokens=max_tokens,
                             commit=None if commit is None else torch.tensor(commit, dtype=torch.int32).cuda(),
                             commit_extra=step % 2)
        compare(pages, out, want, max_tokens)
        whole(pages)


def test_another_state_array_leaves_the_first_alone():
    pages = pcg.Pages.empty(3, 20, 4, 6, "cuda")
    pcg.pages_step(pages, 5, max_tokens=15)
    before = pages.state.clone()
    nxt = torch.full_like(before, -3)
    pcg.pages_step(pages, 2, max_tokens=15, state_out=nxt)
    assert torch.equal(pages.state, before)
    again = pcg.pages_step(pages, 2, max_tokens=15)
    assert torch.equal(pages.state, nxt) and again.q_start.tolist() == [0, 2, 4, 6]


def test_what_a_broken_state_says_stays_inside_the_arrays():
    """Lengths, page counts and a free count that cannot be: guards around the arrays stay as they are."""
    B, n, blocks = 4, 10, 5
    guard = lambda k: torch.full((k + 64,), 12345, dtype=torch.int32, device="cuda")  # noqa: E731
    tab, free = guard(B * blocks), guard(n)
    table, stack = tab[32:32 + B * blocks].view(B, blocks), free[32:32 + n]
    table.fill_(3)
    stack.copy_(torch.arange(n))
    state = torch.tensor([-5, 1 << 30, 7, 2, 99, -1, 1 << 30, 3, 1 << 30, 4, -9, 5, 1 << 30], dtype=torch.int32).cuda()
    pages = pcg.Pages(table, stack, state, 4)
    for add in (-1, 3, 1 << 30, 0):
        pcg.pages_step(pages, add, max_tokens=20)
    torch.cuda.synchronize()
    for g, k in ((tab, B * blocks), (free, n)):
        assert (g[:32] == 12345).all() and (g[32 + k:] == 12345).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,G,D,page_size,layout", [(1, 1, 8, 1, "slots"), (70, 3, 72, 5, "heads"), (700, 8, 128, 16, "slots"),
                                                    (333, 2, 64, 64, "heads")])
def test_rows_go_to_their_slots_and_nowhere_else(dtype, T, G, D, page_size, layout):
    g = torch.Generator().manual_seed(T)
    pages = -(-T // page_size) + 3
    shape = (pages, page_size, G, D) if layout == "slots" else (pages, G, page_size, D)
    base = [torch.randn(shape, generator=g).to(dtype).cuda() for _ in range(2)]
    k, v = (x if layout == "slots" else x.transpose(1, 2) for x in base)
    cache = pcg.KvCache(k, v)
    new = torch.randn((T, 2 * G + 1, D), generator=g).to(dtype).cuda()
    kn, vn = new[:, :G], new[:, G:2 * G]
    slots = torch.randperm(pages * page_size, generator=g)[:T].to(torch.int32)
    slots[::7] = -1 - slots[::7]
    slots[3::11] = pages * page_size + torch.arange(len(slots[3::11]), dtype=torch.int32)
    want = [x.clone() for x in (k, v)]
    for t in range(T):
        s = int(slots[t])
        if 0 <= s < pages * page_size:
            want[0][s // page_size, s % page_size] = kn[t]
            want[1][s // page_size, s % page_size] = vn[t]
    pcg.cache_write(cache, kn, vn, slots.cuda())
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])
