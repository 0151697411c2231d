"""Refusals of the calls around a step's forward pass (no GPU needed: every call here returns before it touches a pointer),
and the plain forms that the GPU tests compare with, on cases worked by hand."""
import ctypes as C
import math

import pytest
import torch

import attention as ref
import paper_2511_13732_amd as pcg
from paper_2511_13732_amd.binding import _KvCacheStruct, _PagesStruct
from test_abi_host import BAD_DTYPE, BAD_SHAPE, BAD_STRIDE, MISALIGNED, NULL_ARG, OK, P, WS_SMALL

BAD_SCALE = -12


def cache_struct(**k):
    c = dict(k=P, v=P, dt=1, num_pages=10, page_size=16, kv_heads=2, head_dim=64, page_stride=16 * 128, slot_stride=128,
             head_stride=64)
    c.update(k)
    return _KvCacheStruct(*c.values())


def test_structures_match_the_header():
    assert C.sizeof(_KvCacheStruct) == 64 and C.sizeof(_PagesStruct) == 40
    assert pcg.strerror(BAD_SCALE) != "unknown status"


BAD_CACHES = [(dict(k=None), NULL_ARG), (dict(v=None), NULL_ARG), (dict(dt=2), BAD_DTYPE), (dict(num_pages=0), BAD_SHAPE),
              (dict(page_size=0), BAD_SHAPE), (dict(num_pages=1 << 20, page_size=1 << 11), BAD_SHAPE), (dict(kv_heads=0), BAD_SHAPE),
              (dict(head_dim=0), BAD_SHAPE), (dict(head_dim=68), BAD_SHAPE), (dict(head_dim=136), BAD_SHAPE),
              (dict(page_stride=0), BAD_STRIDE), (dict(slot_stride=-128), BAD_STRIDE), (dict(head_stride=60), BAD_STRIDE),
              (dict(dt=0, head_stride=66), BAD_STRIDE), (dict(k=P + 8), MISALIGNED), (dict(v=P + 2), MISALIGNED)]


def write(cache=None, k=P, v=P, T=4, kt=128, kh=64, vt=128, vh=64, slots=P, **c):
    return pcg.lib().pcg_cache_write(C.byref(cache or cache_struct(**c)), k, v, T, kt, kh, vt, vh, slots, None)


def attend(cache=None, q=P, qt=256, qh=64, heads=4, T=4, table=P, ts=8, blocks=8, lens=P, starts=P, B=2, longest=2, scale=1.0,
           window=0, out=P, ot=256, oh=64, ws=P, wsb=1 << 40, **c):
    return pcg.lib().pcg_cache_attend(C.byref(cache or cache_struct(**c)), q, qt, qh, heads, T, table, ts, blocks, lens, starts,
                                      B, longest, scale, window, out, ot, oh, ws, wsb, None)


def prompt(q=P, k=P, v=P, dt=1, T=4, heads=4, kv=2, D=64, qt=256, qh=64, kt=128, kh=64, vt=128, vh=64, starts=P, B=2, longest=2,
           scale=1.0, window=0, out=P, ot=256, oh=64):
    return pcg.lib().pcg_prompt_attend(q, k, v, dt, T, heads, kv, D, qt, qh, kt, kh, vt, vh, starts, B, longest, scale, window,
                                       out, ot, oh, None)


@pytest.mark.parametrize("bad,status", BAD_CACHES)
def test_caches_that_are_refused(bad, status):
    assert write(**bad) == status
    assert attend(**bad) == status


@pytest.mark.parametrize("bad,status", [(dict(T=-1), BAD_SHAPE), (dict(T=1 << 40), BAD_SHAPE), (dict(k=None), NULL_ARG),
                                        (dict(v=None), NULL_ARG), (dict(slots=None), NULL_ARG), (dict(kt=0), BAD_STRIDE),
                                        (dict(vt=130), BAD_STRIDE), (dict(kh=-64), BAD_STRIDE), (dict(vh=4), BAD_STRIDE),
                                        (dict(k=P + 4), MISALIGNED), (dict(v=P + 8), MISALIGNED), (dict(slots=P + 2), MISALIGNED)])
def test_rows_that_are_refused(bad, status):
    assert write(**bad) == status


QUERIES = [(dict(heads=3), BAD_SHAPE), (dict(heads=0), BAD_SHAPE), (dict(B=-1), BAD_SHAPE), (dict(T=-1), BAD_SHAPE),
           (dict(longest=-1), BAD_SHAPE), (dict(longest=1 << 31), BAD_SHAPE), (dict(window=-1), BAD_SHAPE), (dict(T=1 << 31), BAD_SHAPE), (dict(scale=0.0), BAD_SCALE),
           (dict(scale=math.nan), BAD_SCALE), (dict(scale=math.inf), BAD_SCALE), (dict(scale=-1.0), BAD_SCALE),
           (dict(q=None), NULL_ARG), (dict(out=None), NULL_ARG), (dict(starts=None), NULL_ARG), (dict(qt=0), BAD_STRIDE),
           (dict(qh=4), BAD_STRIDE), (dict(ot=-256), BAD_STRIDE), (dict(oh=65), BAD_STRIDE), (dict(q=P + 2), MISALIGNED),
           (dict(out=P + 8), MISALIGNED), (dict(starts=P + 1), MISALIGNED)]


@pytest.mark.parametrize("bad,status", QUERIES)
def test_queries_that_are_refused(bad, status):
    assert attend(**bad) == status
    assert prompt(**bad) == status


@pytest.mark.parametrize("bad,status", [(dict(blocks=0), BAD_SHAPE), (dict(blocks=1 << 28), BAD_SHAPE), (dict(blocks=(1 << 27) - 1, ts=1 << 27), BAD_SHAPE), (dict(ts=7), BAD_STRIDE),
                                        (dict(table=None), NULL_ARG), (dict(lens=None), NULL_ARG), (dict(ws=None), NULL_ARG),
                                        (dict(table=P + 2), MISALIGNED), (dict(lens=P + 2), MISALIGNED), (dict(ws=P + 16), MISALIGNED),
                                        (dict(wsb=0), WS_SMALL)])
def test_tables_that_are_refused(bad, status):
    assert attend(**bad) == status


def test_the_workspace_is_what_the_helper_says():
    need = pcg.cache_attend_workspace_bytes(2, 4, 4, 2, 64, 2)
    assert need > 0 and attend(wsb=need - 1) == WS_SMALL
    for bad in ((-1, 4, 4, 2, 64, 2), (2, -4, 4, 2, 64, 2), (2, 4, 3, 2, 64, 2), (2, 4, 4, 2, 60, 2), (2, 4, 4, 2, 64, -2), (2, 4, 4, 2, 64, 1 << 31)):
        assert pcg.cache_attend_workspace_bytes(*bad) == 0


@pytest.mark.parametrize("bad,status", [(dict(dt=7), BAD_DTYPE), (dict(kv=0), BAD_SHAPE), (dict(D=4), BAD_SHAPE), (dict(D=192), BAD_SHAPE),
                                        (dict(k=None), NULL_ARG), (dict(v=None), NULL_ARG), (dict(kt=0), BAD_STRIDE),
                                        (dict(kt=1 << 27), BAD_STRIDE), (dict(vt=1 << 30), BAD_STRIDE), (dict(vh=12), BAD_STRIDE),
                                        (dict(k=P + 8), MISALIGNED), (dict(v=P + 4), MISALIGNED)])
def test_prompts_that_are_refused(bad, status):
    assert prompt(**bad) == status


def test_nothing_to_do_is_not_an_error():
    assert write(T=0, k=None, v=None, slots=None) == OK
    for empty in (dict(T=0), dict(B=0)):
        assert attend(q=None, out=None, starts=None, lens=None, table=None, ws=None, wsb=0, **empty) == OK
        assert prompt(q=None, k=None, v=None, out=None, starts=None, **empty) == OK


def step(pages=True, B=4, num_pages=10, page_size=16, blocks=5, table=P, ts=5, free=P, si=P, so=P, commit=None, add=P, tokens=8,
         qs=P, slots=P, positions=P, refused=P):
    g = _PagesStruct(B, num_pages, page_size, blocks, table, ts, free)
    return pcg.lib().pcg_pages_step(C.byref(g) if pages else None, si, so, commit, 0, add, 0, tokens, qs, slots, positions, refused,
                                    None)


@pytest.mark.parametrize("bad,status", [(dict(pages=False), NULL_ARG), (dict(table=None), NULL_ARG), (dict(free=None), NULL_ARG),
                                        (dict(si=None), NULL_ARG), (dict(so=None), NULL_ARG), (dict(qs=None), NULL_ARG),
                                        (dict(slots=None), NULL_ARG), (dict(B=0), BAD_SHAPE), (dict(B=65537), BAD_SHAPE),
                                        (dict(num_pages=0), BAD_SHAPE), (dict(page_size=0), BAD_SHAPE), (dict(blocks=0), BAD_SHAPE),
                                        (dict(tokens=-1), BAD_SHAPE), (dict(tokens=1 << 31), BAD_SHAPE),
                                        (dict(num_pages=1 << 27), BAD_SHAPE), (dict(blocks=1 << 27), BAD_SHAPE),
                                        (dict(blocks=1 << 16, ts=1 << 16, B=1 << 15, page_size=1), BAD_SHAPE), (dict(ts=4), BAD_STRIDE),
                                        (dict(table=P + 1), MISALIGNED), (dict(commit=P + 2), MISALIGNED), (dict(so=P + 3), MISALIGNED)])
def test_pools_that_are_refused(bad, status):
    assert step(**bad) == status


def test_tensors_that_do_not_fit_are_refused():
    f = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype)  # noqa: E731
    i = lambda *s: f(*s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):
        pcg.KvCache(f(4, 16, 2, 64), f(4, 16, 2, 32))
    with pytest.raises(ValueError):
        pcg.KvCache(f(4, 16, 2, 64), f(4, 2, 16, 64).transpose(1, 2))
    with pytest.raises(ValueError):
        pcg.KvCache(f(4, 16, 64, 2).transpose(2, 3), f(4, 16, 64, 2).transpose(2, 3))
    with pytest.raises(TypeError):
        pcg.KvCache(f(4, 16, 2, 64).half(), f(4, 16, 2, 64).half())
    cache = pcg.KvCache(f(4, 16, 2, 64), f(4, 16, 2, 64))
    good = dict(q=f(3, 4, 64), block_table=i(2, 3), lens=i(2), q_start=i(3))
    for bad in (dict(q=f(3, 4, 32)), dict(q=f(3, 4, 64, dtype=torch.bfloat16)), dict(q=f(3, 4, 128)[:, :, ::2]),
                dict(block_table=i(3, 3)), dict(block_table=i(2, 6)[:, ::2]), dict(block_table=f(2, 3)), dict(lens=f(2)), dict(q_start=i(2)),
                dict(out=f(2, 4, 64)), dict(out=f(3, 2, 64))):
        with pytest.raises(ValueError):
            pcg.cache_attend(cache, **{**good, **bad})
    for bad in ((f(3, 2, 64), f(2, 2, 64), i(3)), (f(3, 2, 64), f(3, 2, 64), i(2)), (f(3, 1, 64), f(3, 2, 64), i(3)),
                (f(3, 2, 64), f(3, 2, 64), f(3))):
        with pytest.raises(ValueError):
            pcg.cache_write(cache, *bad)
    for bad in ((f(3, 4, 64), f(2, 2, 64), f(3, 2, 64), i(2)), (f(3, 4, 64), f(3, 2, 64), f(3, 2, 32), i(2)),
                (f(3, 4, 64), f(3, 2, 64), f(3, 2, 64), f(2))):
        with pytest.raises(ValueError):
            pcg.prompt_attend(*bad)
    with pytest.raises(ValueError):
        pcg.Pages(i(4, 3), i(10), i(12), 16)
    with pytest.raises(ValueError):
        pcg.Pages(i(4, 6)[:, ::2], i(10), i(13), 16)
    pages = pcg.Pages.empty(4, 10, 16, 3, "cpu")
    assert pages.free_count.item() == 10 and pages.lens.numel() == pages.held.numel() == pages.chunk.numel() == 4
    for bad in (dict(add=i(3)), dict(add=1, commit=f(4)), dict(add=1, state_out=i(12)),
                dict(add=1, out=pcg.pages_step_outputs(4, 7, "cpu")), dict(add=1, out=pcg.pages_step_outputs(5, 8, "cpu"))):
        with pytest.raises(ValueError):
            pcg.pages_step(pages, max_tokens=8, **bad)


def test_sizes_whose_grids_do_not_fit_are_refused():
    assert attend(T=1 << 26) == prompt(T=1 << 26) == BAD_SHAPE                    # 4 heads
    assert attend(B=1 << 21) == prompt(B=1 << 21) == BAD_SHAPE                    # 2 shared heads
    assert write(T=1 << 27) == BAD_SHAPE                                          # 16 parts a row
    assert attend(scale=3e38) == prompt(scale=3e38) == BAD_SCALE


def test_numbers_that_the_library_would_take_for_others_are_refused():
    f = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype)  # noqa: E731
    i = lambda *s: f(*s, dtype=torch.int32)  # noqa: E731
    cache = pcg.KvCache(f(4, 16, 2, 64), f(4, 16, 2, 64))
    good = dict(q=f(3, 4, 64), block_table=i(2, 3), lens=i(2), q_start=i(3), workspace=f(1 << 10, dtype=torch.uint8))
    for bad in (dict(window=1 << 32), dict(window=-1), dict(workspace=f(1, dtype=torch.uint8).expand(1 << 30)),
                dict(workspace=torch.zeros(1 << 10, dtype=torch.uint8, device="meta"))):
        with pytest.raises(ValueError):
            pcg.cache_attend(cache, **{**good, **bad})
    with pytest.raises(ValueError):
        pcg.prompt_attend(f(3, 4, 64), f(3, 2, 64), f(3, 2, 64), i(2), window=(1 << 32) + 5)
    for size in (0, -16, (1 << 32) + 16):
        with pytest.raises(ValueError):
            pcg.Pages(i(4, 3), i(10), i(13), size)
    pages = pcg.Pages.empty(4, 10, 16, 3, "cpu")
    for bad in (dict(add=1 << 32), dict(add=1, commit=i(4), commit_extra=1 << 32)):
        with pytest.raises(ValueError):
            pcg.pages_step(pages, max_tokens=8, **bad)
    for bad in ((i(5), i(8), i(8), i(2)), (i(5), f(8), i(8), i(1)), (i(5), i(16)[::2], i(8), i(1)),
                (i(5), i(8), torch.zeros(8, dtype=torch.int32, device="meta"), i(1))):
        with pytest.raises(ValueError):
            pcg.PagesStep(*bad)
    elsewhere = pcg.pages_step_outputs(4, 8, "meta")
    with pytest.raises(ValueError):
        pcg.pages_step(pages, 1, max_tokens=8, out=elsewhere)


# ------------------------------------------------------------------ the plain forms, by hand

def test_plain_pages_by_hand():
    # two pages of two slots each, one request of room for two pages
    state, table, free = [0, 0, 0, 0, 0, 0, 3], [[9, 9], [9, 9]], [0, 1, 2]
    s = ref.pages_step(table, free, state, 2, None, 0, [3, 1], 8)
    assert s == ([0, 0, 2, 1, 3, 1, 0], [[2, 1], [0, 9]], [0, 1, 2], [0, 3, 4], [4, 5, 2, 0, -1, -1, -1, -1], [0, 1, 2, 0, 0, 0, 0, 0], 0)
    # the first keeps one of three and wants one: one page comes back, which the second takes for two more
    s = ref.pages_step(s[1], s[2], s[0], 2, [0, 0], 1, [1, 2], 3)
    assert s == ([1, 1, 1, 2, 1, 2, 0], [[2, 1], [0, 1]], [1, 1, 2], [0, 1, 3], [5, 1, 2], [1, 1, 2], 0)
    # no page left: the first that needs one is refused; the second ends
    t = ref.pages_step(s[1], s[2], s[0], 2, None, 0, [2, 0], 3)
    assert t[0] == [2, 3, 1, 2, 0, 0, 0] and t[3] == [0, 0, 0] and t[6] == 1
    t = ref.pages_step(s[1], s[2], s[0], 2, None, 0, [2, -1], 3)
    assert t[0] == [2, 0, 2, 0, 2, 0, 1] and t[1][0] == [2, 1] and t[2][:2] == [0, 1] and t[4] == [2, 3, -1] and t[6] == 0
    # more rows than the batch has, and than the table has room for
    assert ref.pages_step(s[1], s[2], s[0], 2, None, 0, [0, 4], 3)[6] == 1
    s = ref.pages_step(table, free, state, 2, None, 0, [5, 1], 8)
    assert s[0] == [0, 0, 0, 1, 0, 1, 2] and s[3] == [0, 0, 1] and s[6] == 1


def test_plain_attention_by_hand():
    q = torch.tensor([[[1.0, 0.0]], [[0.0, 2.0]]])
    k = torch.tensor([[[math.log(3.0), 0.0]], [[0.0, 0.5]]])
    v = torch.tensor([[[1.0, -1.0]], [[5.0, 3.0]]])
    out, mag, err = ref.attend_rows(q, k, v, 0, 1.0)
    assert torch.allclose(out[0, 0], torch.tensor([1.0, -1.0], dtype=torch.float64))
    w = math.e / (1 + math.e)
    assert torch.allclose(out[1, 0], torch.tensor([1 - w + 5 * w, -1 + w + 3 * w], dtype=torch.float64), atol=1e-7)
    assert torch.allclose(mag[1, 0], torch.tensor([1 - w + 5 * w, 1 - w + 3 * w], dtype=torch.float64), atol=1e-7)
    assert (err > 0).all() and (err < 1e-4).all()
    # with a window of one every row sees itself
    assert torch.equal(ref.attend_rows(q, k, v, 0, 1.0, window=1)[0][:, 0], v[:, 0].double())
    # nothing to see
    assert (ref.attend_rows(q[:1, :, :1] + 1, k[:, :, :1] * 0 - math.inf, v[:, :, :1], 1, 1.0)[0] == 0).all()
    assert (ref.attend_rows(q, k[:0], v[:0], 0, 1.0)[0] == 0).all()
