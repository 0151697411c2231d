"""Attention over 4 bits where some of a workgroup's waves have no keys: 64 keys of each 256 are a wave's, so that caches of up to 192 keys leave
waves without any, whose part of shared memory the others' rows go through at the end.  Entries of the page table behind a request's
pages are -1, which is NaN as float32.  Run with ``-m gpu`` on an MI355X."""
import pytest
import torch

import attention
import paper_2511_13732_amd as pcg
from test_gpu_attend4 import DTYPES, check, gen, make_cache, starts_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("chunk,page_size,window", [(12, 16, 0), (9, 16, 0), (9, 24, 0), (11, 32, 40), (8, 16, 0), (5, 7, 0), (1, 16, 0), (4, 5, 33)])
def test_caches_that_leave_waves_without_keys(dtype, D, chunk, page_size, window):
    """Four query heads a shared head: up to 48 rows in three, two and one blocks of 16, over 1 to 200 keys."""
    dt, H, G = DTYPES[dtype], 8, 2
    total = [1, 2, 15, 16, 17, 33, 48, 63, 64, 65, 66, 80, 127, 128, 129, 130, 145, 160, 176, 191, 192, 193, 194, 200]
    new = [min(chunk, n) for n in total]
    ctx = [n - m for n, m in zip(total, new)]
    cache, table, rows = make_cache(total, page_size, G, D, "heads", seed=chunk + D)
    used = (torch.tensor(total) + page_size - 1) // page_size
    table[torch.arange(table.shape[1])[None] >= used[:, None]] = -1
    st = starts_of(new)
    q = torch.randn((st[-1], H, D), generator=gen(chunk)).to(dt).cuda()
    out = pcg.cache4_attend(cache, q, table, torch.tensor(ctx, dtype=torch.int32).cuda(), torch.tensor(st, dtype=torch.int32).cuda(), longest=chunk,
                            window=window)
    for b, n in enumerate(total):
        check(out[st[b]:st[b + 1]], attention.attend_rows(q[st[b]:st[b + 1]], *rows[b], ctx[b], D ** -0.5, window), dt, (b, n))
