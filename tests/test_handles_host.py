"""Objects of the binding that keep addresses of tensors.  No GPU needed."""
import pytest
import torch

import paper_2511_13732_amd as pcg


def addresses(x):
    r = x._ref.contents
    return (r.k, r.v) if isinstance(x, pcg.KvCache) else (r.block_table, r.free_pages)


def test_a_cache_whose_tensors_are_replaced_names_the_new_ones():
    new = lambda *s: torch.zeros(s or (4, 16, 2, 64))  # noqa: E731
    cache = pcg.KvCache(new(), new())
    k, v = new(), new()
    cache.k = k
    cache.v = v
    assert addresses(cache) == (k.data_ptr(), v.data_ptr())
    for bad in (new(4, 16, 2, 32), new().double(), new(4, 2, 16, 64).transpose(1, 2)):
        with pytest.raises((ValueError, TypeError)):
            cache.k = bad
        assert cache.k is k and addresses(cache) == (k.data_ptr(), v.data_ptr()) and cache.head_dim == 64
        assert cache._ref.contents.head_dim == 64
    with pytest.raises(TypeError):
        pcg.KvCache(new().half(), new().half())


def test_a_pool_whose_tensors_are_replaced_names_the_new_ones():
    pages = pcg.Pages.empty(4, 10, 16, 3, "cpu")
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    table, free, state = i(4, 5), i(20), i(13)
    pages.block_table = table
    pages.free_pages = free
    pages.state = state
    pages.page_size = 8
    assert addresses(pages) == (table.data_ptr(), free.data_ptr()) and pages.state is state
    r = pages._ref.contents
    assert (r.max_blocks, r.table_stride, r.num_pages, r.page_size) == (5, 5, 20, 8) == (pages.max_blocks, 5, pages.num_pages, 8)
    for name, bad in (("block_table", i(3, 5)), ("block_table", i(4, 6)[:, ::2]), ("state", i(12)), ("state", i(13).float()),
                      ("free_pages", i(2, 5)), ("page_size", 0)):
        was = getattr(pages, name)
        with pytest.raises(ValueError):
            setattr(pages, name, bad)
        assert getattr(pages, name) is was and addresses(pages) == (table.data_ptr(), free.data_ptr())
    # two states in turn, as a caller does who keeps the last one
    pages.state, other = i(13), pages.state
    assert other is state


def test_sizes_that_the_library_would_take_for_others_are_refused():
    """Beyond 2^31, on a device that holds no memory."""
    far = (1 << 32) + 8
    new = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device="meta")  # noqa: E731
    i = lambda *s: new(*s, dtype=torch.int32)  # noqa: E731
    for shape in ((far, 1, 1, 8), (1, far, 1, 8), (1, 1, far, 8), (1, 1, 1, far)):
        with pytest.raises(ValueError):
            pcg.KvCache(new(*shape), new(*shape))
    for table, free in ((i(far, 1), i(4)), (i(1, far), i(4)), (i(1, 1), i(far))):
        with pytest.raises(ValueError):
            pcg.Pages(table, free, i(3 * table.shape[0] + 1), 1)
    cache = pcg.KvCache(new(4, 16, 1, 8), new(4, 16, 1, 8))
    ws = torch.empty(1 << 10, dtype=torch.uint8, device="meta")
    good = dict(q=new(3, 2, 8), block_table=i(2, 3), lens=i(2), q_start=i(3))
    for bad in (dict(q=new(1, far, 8)), dict(block_table=i(2, far)), dict(block_table=i(far, 3), lens=i(far), q_start=i(far + 1))):
        with pytest.raises(ValueError):
            pcg.cache_attend(cache, workspace=ws, **{**good, **bad})
    for q, k, b in ((new(1, far, 8), new(1, 1, 8), 2), (new(1, far, 8), new(1, far, 8), 2), (new(1, 1, far), new(1, 1, far), 2),
                    (new(1, 1, 8), new(1, 1, 8), far + 1)):
        with pytest.raises(ValueError):
            pcg.prompt_attend(q, k, k, i(b))
