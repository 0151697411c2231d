"""The serving loop of README.md, run as it stands with the page table's plain form in place of the library: what it keeps of prompts
and of chunks.  No GPU needed."""
import os
import re
from types import SimpleNamespace

import torch

import attention as ref
from conftest import ROOT

B, K, PAGE, BLOCKS, POOL, ROWS, V = 4, 4, 4, 30, 100, 80, 11


class Pages:
    def __init__(self):
        self.table, self.free, self.state = [[0] * BLOCKS for _ in range(B)], list(range(POOL)), [0] * (3 * B) + [POOL]
        self.block_table = torch.zeros((B, BLOCKS), dtype=torch.int32)

    @property
    def lens(self):
        return torch.tensor(self.state[:B])


def library(accepted, log):
    """The calls that the loop makes; `accepted` gives every verification's accepted lengths."""
    def pages_step(pages, add, *, max_tokens, commit=None, commit_extra=0):
        if commit is not None:
            assert commit.dtype == torch.int32 and commit.shape == (B,)
        pages.state, pages.table, pages.free, q_start, slots, positions, refused = ref.pages_step(
            pages.table, pages.free, pages.state, PAGE, None if commit is None else commit.tolist(), commit_extra, add.tolist(), max_tokens)
        log.append((pages.state[:B], pages.state[2 * B:3 * B]))
        return SimpleNamespace(q_start=torch.tensor(q_start), slots=torch.tensor(slots))

    def verify(groups, target, draft, tokens, pgroups):
        assert target.shape == (B, K + 1, V)
        return SimpleNamespace(accept_len=torch.tensor(accepted.pop(0), dtype=torch.int32))

    return SimpleNamespace(Pages=SimpleNamespace(empty=lambda *a: Pages()), KvCache=lambda k, v: (k, v), pages_step=pages_step, verify=verify,
                           cache_write=lambda kv, k, v, slots: None,
                           cache_attend=lambda kv, q, table, lens, q_start, longest: torch.zeros((ROWS, 1, 8)))


class Serving:
    """True for so many steps; before each, what the caller's scheduler sets."""

    def __init__(self, steps, names):
        self.steps, self.names = list(steps), names

    def __bool__(self):
        if not self.steps:
            return False
        add, prompt = self.steps.pop(0)
        self.names["add"] = torch.tensor(add, dtype=torch.int32)
        self.names["brought_prompt"] = torch.tensor(prompt)
        return True


def test_the_loop_keeps_prompts_whole_and_of_chunks_what_was_accepted():
    text = open(os.path.join(ROOT, "README.md")).read()
    code, = [b for b in re.findall(r"```python\n(.*?)```", text, re.S) if "pages_step" in b]
    log, no = [], [False] * B
    steps = [([5, 5, 5, 0], no), ([5, -1, 5, 0], no), ([5, 23, 5, 9], [False, True, False, True]), ([5, 7, 5, 5], [False, True, False, False]),
             ([5, 5, 5, 5], no)]
    accepted = [[4, 0, 2, 1], [1, 3, 0, 0], [0, 1, 4, 0], [2, 0, 1, 3], [0, 0, 0, 0]]
    names = dict(torch=torch, B=B, K=K, num_pages=POOL, page_size=PAGE, max_blocks=BLOCKS, rows=ROWS, layers=[(0, 0)],
                 prompt_lens=torch.tensor([20, 1, 30, 0], dtype=torch.int32), k_new=None, v_new=None, q=None, groups=None, draft_logits=None,
                 prop_tokens=None, prop_groups=None, head=lambda x: torch.zeros((x.shape[0], V)))
    names.update(pcg=library(accepted, log), serving=Serving(steps, names))
    exec(code, names)
    assert log == [([0, 0, 0, 0], [20, 1, 30, 0]),
                   ([20, 1, 30, 0], [5, 5, 5, 0]),            # the prompts as they were
                   ([25, 0, 33, 0], [5, 0, 5, 0]),            # accepted 4, ended, accepted 2, an empty place
                   ([27, 0, 34, 0], [5, 23, 5, 9]),           # accepted 1 and 0; two prompts come in
                   ([28, 23, 39, 9], [5, 7, 5, 5]),           # the prompts whole beside accepted 0 and 4; a piece more of one
                   ([31, 30, 41, 13], [5, 5, 5, 5])]
