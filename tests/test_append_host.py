"""Refusals of the calls that bring rows into a cache with their rotation, and of those over a cache of 4 bits (no GPU needed: every call
here returns before it touches a pointer); the plain forms that the GPU tests compare with, on cases worked by hand."""
import ctypes as C
import math

import pytest
import torch

import cache4 as ref
import paper_2511_13732_amd as pcg
from paper_2511_13732_amd.binding import _KvCache4Struct, _RotationStruct
from test_abi_host import BAD_DTYPE, BAD_SHAPE, BAD_STRIDE, MISALIGNED, NULL_ARG, OK, P, WS_SMALL
from test_cache_host import BAD_CACHES, BAD_SCALE, QUERIES, cache_struct


def cache4_struct(**k):
    c = dict(k=P, v=P, scales=P, num_pages=10, page_size=16, kv_heads=2, head_dim=64, page_stride=16 * 64, slot_stride=64, head_stride=32,
             scale_page_stride=32, scale_slot_stride=2, scale_head_stride=1)
    c.update(k)
    return _KvCache4Struct(*c.values())


def rotation(rotate=True, table=P, stride=64, places=100, dim=64, interleaved=0):
    return C.byref(_RotationStruct(table, stride, places, dim, interleaved)) if rotate else None


ROTATION = ("rotate", "table", "stride", "places", "dim")


def rows(positions=P, q=P, qt=256, qh=64, heads=4, qo=P, ot=256, oh=64, k=P, kt=128, kh=64, v=P, vt=128, vh=64, T=4, slots=P, **r):
    return rotation(**r), positions, q, qt, qh, heads, qo, ot, oh, k, kt, kh, v, vt, vh, T, slots, None


def split(kw, names):
    return {n: kw[n] for n in kw if n in names}, {n: kw[n] for n in kw if n not in names}


CACHE = ("num_pages", "page_size", "kv_heads", "head_dim", "page_stride", "slot_stride", "head_stride")
CACHE4 = CACHE + ("scales", "scale_page_stride", "scale_slot_stride", "scale_head_stride")


def append(cache=None, **kw):
    c, r = split(kw, CACHE)
    return pcg.lib().pcg_cache_append(C.byref(cache or cache_struct(**c)), *rows(**r))


def append4(cache=None, dt=1, **kw):
    c, r = split(kw, CACHE4)
    return pcg.lib().pcg_cache4_append(C.byref(cache or cache4_struct(**c)), dt, *rows(**r))


def read4(cache=None, dt=1, k=P, kt=128, kh=64, v=P, vt=128, vh=64, T=4, slots=P, **c):
    return pcg.lib().pcg_cache4_read(C.byref(cache or cache4_struct(**c)), dt, k, kt, kh, v, vt, vh, T, slots, None)


def attend4(cache=None, dt=1, q=P, qt=256, qh=64, heads=4, T=4, table=P, ts=8, blocks=8, lens=P, starts=P, B=2, longest=2, scale=1.0,
            window=0, out=P, ot=256, oh=64, ws=P, wsb=1 << 40, **c):
    return pcg.lib().pcg_cache4_attend(C.byref(cache or cache4_struct(**c)), dt, q, qt, qh, heads, T, table, ts, blocks, lens, starts,
                                       B, longest, scale, window, out, ot, oh, ws, wsb, None)


def test_structures_match_the_header():
    assert C.sizeof(_RotationStruct) == 32 and C.sizeof(_KvCache4Struct) == 88


@pytest.mark.parametrize("bad,status", BAD_CACHES)
def test_caches_that_are_refused(bad, status):
    assert append(cache=cache_struct(**bad)) == status


@pytest.mark.parametrize("bad,status", [(dict(k=None), NULL_ARG), (dict(v=None), NULL_ARG), (dict(scales=None), NULL_ARG),
                                        (dict(num_pages=0), BAD_SHAPE), (dict(page_size=0), BAD_SHAPE),
                                        (dict(num_pages=1 << 20, page_size=1 << 11), BAD_SHAPE), (dict(kv_heads=0), BAD_SHAPE),
                                        (dict(head_dim=0), BAD_SHAPE), (dict(head_dim=68), BAD_SHAPE), (dict(head_dim=136), BAD_SHAPE),
                                        (dict(page_stride=0), BAD_STRIDE), (dict(slot_stride=-64), BAD_STRIDE), (dict(head_stride=24), BAD_STRIDE),
                                        (dict(page_stride=1 << 33), BAD_STRIDE), (dict(scale_page_stride=0), BAD_STRIDE),
                                        (dict(scale_slot_stride=-1), BAD_STRIDE), (dict(scale_head_stride=1 << 33), BAD_STRIDE),
                                        (dict(k=P + 8), MISALIGNED), (dict(v=P + 4), MISALIGNED), (dict(scales=P + 2), MISALIGNED)])
def test_caches_of_4_bits_that_are_refused(bad, status):
    for call in (append4, read4, attend4):
        assert call(cache=cache4_struct(**bad)) == status


@pytest.mark.parametrize("bad,status", [(dict(T=-1), BAD_SHAPE), (dict(T=1 << 31), BAD_SHAPE), (dict(T=1 << 24), BAD_SHAPE), (dict(heads=0), BAD_SHAPE),
                                        (dict(heads=65537), BAD_SHAPE), (dict(dim=0), BAD_SHAPE), (dict(dim=66), BAD_SHAPE), (dict(dim=7), BAD_SHAPE),
                                        (dict(dim=-2), BAD_SHAPE), (dict(places=0), BAD_SHAPE), (dict(table=None), NULL_ARG),
                                        (dict(positions=None), NULL_ARG), (dict(stride=63), BAD_STRIDE), (dict(stride=1 << 33), BAD_STRIDE),
                                        (dict(table=P + 2), MISALIGNED), (dict(positions=P + 1), MISALIGNED), (dict(rotate=False), NULL_ARG),
                                        (dict(qo=None), NULL_ARG), (dict(k=None), NULL_ARG), (dict(v=None), NULL_ARG), (dict(slots=None), NULL_ARG),
                                        (dict(qt=0), BAD_STRIDE), (dict(qh=4), BAD_STRIDE), (dict(ot=-256), BAD_STRIDE), (dict(oh=65), BAD_STRIDE),
                                        (dict(kt=0), BAD_STRIDE), (dict(vt=130), BAD_STRIDE), (dict(kh=-64), BAD_STRIDE), (dict(vh=4), BAD_STRIDE),
                                        (dict(q=P + 2), MISALIGNED), (dict(qo=P + 8), MISALIGNED), (dict(k=P + 4), MISALIGNED),
                                        (dict(v=P + 8), MISALIGNED), (dict(slots=P + 2), MISALIGNED)])
def test_rows_that_are_refused(bad, status):
    assert append(**bad) == status
    assert append4(**bad) == status


@pytest.mark.parametrize("bad,status", [(dict(T=-1), BAD_SHAPE), (dict(T=1 << 31), BAD_SHAPE), (dict(T=1 << 23), BAD_SHAPE), (dict(k=None), NULL_ARG),
                                        (dict(v=None), NULL_ARG), (dict(slots=None), NULL_ARG), (dict(kt=0), BAD_STRIDE), (dict(vt=130), BAD_STRIDE),
                                        (dict(kh=-64), BAD_STRIDE), (dict(vh=4), BAD_STRIDE), (dict(k=P + 4), MISALIGNED),
                                        (dict(v=P + 8), MISALIGNED), (dict(slots=P + 2), MISALIGNED)])
def test_values_that_are_refused(bad, status):
    assert read4(**bad) == status


@pytest.mark.parametrize("bad,status", QUERIES)
def test_queries_that_are_refused(bad, status):
    assert attend4(**bad) == status


@pytest.mark.parametrize("bad,status", [(dict(blocks=0), BAD_SHAPE), (dict(blocks=1 << 28), BAD_SHAPE), (dict(blocks=(1 << 27) - 1, ts=1 << 27), BAD_SHAPE),
                                        (dict(ts=7), BAD_STRIDE), (dict(table=None), NULL_ARG), (dict(lens=None), NULL_ARG), (dict(ws=None), NULL_ARG),
                                        (dict(table=P + 2), MISALIGNED), (dict(lens=P + 2), MISALIGNED), (dict(ws=P + 16), MISALIGNED),
                                        (dict(wsb=0), WS_SMALL), (dict(T=1 << 26), BAD_SHAPE), (dict(B=1 << 21), BAD_SHAPE), (dict(scale=3e38), BAD_SCALE)])
def test_tables_that_are_refused(bad, status):
    assert attend4(**bad) == status


def test_types_that_are_refused():
    for call in (append4, read4, attend4):
        assert call(dt=2) == call(dt=-1) == BAD_DTYPE


def test_the_workspace_is_what_the_helper_says():
    for longest in (2, 10, 20):
        need = pcg.cache4_attend_workspace_bytes(2, 4, 4, 2, 64, longest)
        assert need > 0 and attend4(wsb=need - 1, longest=longest) == WS_SMALL
    # what is enough for one call is enough for smaller and larger ones
    assert len({pcg.cache4_attend_workspace_bytes(B, 999, 8 * G, G, 128, longest) for B in (1, 300) for G in (1, 8) for longest in (1, 6, 8, 400)}) == 1
    for bad in ((-1, 4, 4, 2, 64, 2), (2, -4, 4, 2, 64, 2), (2, 4, 3, 2, 64, 2), (2, 4, 4, 2, 60, 2), (2, 4, 4, 2, 64, -2), (2, 4, 4, 2, 64, 1 << 31)):
        assert pcg.cache4_attend_workspace_bytes(*bad) == 0


def test_nothing_to_do_is_not_an_error():
    for call in (append, append4):
        assert call(T=0, q=None, qo=None, k=None, v=None, slots=None, positions=None) == OK
        assert call(T=0, q=None, qo=None, k=None, v=None, slots=None, positions=None, rotate=False) == OK
    assert read4(T=0, k=None, v=None, slots=None) == OK
    for empty in (dict(T=0), dict(B=0)):
        assert attend4(q=None, out=None, starts=None, lens=None, table=None, ws=None, wsb=0, **empty) == OK


def test_tensors_that_do_not_fit_are_refused():
    f = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype)  # noqa: E731
    i = lambda *s: f(*s, dtype=torch.int32)  # noqa: E731
    u = lambda *s: f(*s, dtype=torch.uint8)  # noqa: E731
    h = lambda *s: f(*s, dtype=torch.bfloat16)  # noqa: E731
    good = dict(k=u(4, 16, 2, 48), v=u(4, 16, 2, 48), scales=h(4, 16, 2, 2), head_dim=72)
    pcg.KvCache4(**good)
    for bad in (dict(k=u(4, 16, 2, 32)), dict(k=u(4, 16, 2, 32), v=u(4, 16, 2, 32)), dict(v=u(4, 2, 16, 48).transpose(1, 2)), dict(head_dim=64),
                dict(head_dim=97), dict(scales=h(4, 16, 2)), dict(scales=f(4, 16, 2, 2)), dict(scales=h(4, 16, 2, 4)[..., ::2]),
                dict(scales=h(4, 16, 2, 3)[..., :2]), dict(v=f(4, 16, 2, 48)), dict(k=u(4, 16, 48, 2).transpose(2, 3), v=u(4, 16, 48, 2).transpose(2, 3)),
                dict(scales=h(4, 16, 2, 2).to("meta"))):
        with pytest.raises(ValueError):
            pcg.KvCache4(**{**good, **bad})
    for bad in (f(4), f(4, 7), f(4, 0), f(0, 8), h(4, 8), f(4, 16)[:, ::2]):
        with pytest.raises(ValueError):
            pcg.Rotation(bad)
    r, p = pcg.Rotation(f(9, 64)), i(3)
    dense = pcg.KvCache(f(4, 16, 2, 64), f(4, 16, 2, 64))
    four = pcg.KvCache4.empty(4, 16, 2, 64, "cpu")
    with pytest.raises(ValueError):    # a field that does not fit is refused, and the cache stays what it was
        four.k = u(4, 16, 2, 48)
    assert four.k.shape == (4, 16, 2, 32)
    rows = dict(k=f(3, 2, 64), v=f(3, 2, 64), slots=i(3), rotation=r, positions=p, q=f(3, 4, 64))
    for cache, call in ((dense, pcg.cache_append), (four, pcg.cache4_append)):
        for bad in (dict(k=f(2, 2, 64)), dict(v=h(3, 2, 64)), dict(v=f(3, 1, 64)), dict(slots=f(3)), dict(positions=i(4)), dict(positions=None),
                    dict(rotation=None), dict(rotation=None, q=None), dict(q=f(3, 4, 32)), dict(q=h(3, 4, 64)), dict(q_out=f(3, 2, 64)),
                    dict(q=None, q_out=f(3, 4, 64)), dict(q=f(3, 4, 128)[:, :, ::2]), dict(rotation=pcg.Rotation(f(9, 64).to("meta")))):
            with pytest.raises(ValueError):
                call(cache, **{**rows, **bad})
    with pytest.raises(ValueError):
        pcg.cache_append(dense, **{**rows, "k": h(3, 2, 64), "v": h(3, 2, 64)})
    with pytest.raises(TypeError):
        pcg.cache4_append(four, **{**rows, "k": f(3, 2, 64, dtype=torch.float16), "v": f(3, 2, 64, dtype=torch.float16)})
    for bad in (dict(out=(f(3, 2, 64), h(3, 2, 64))), dict(out=(f(2, 2, 64), f(2, 2, 64))), dict(slots=f(3))):
        with pytest.raises(ValueError):
            pcg.cache4_read(four, **{**dict(slots=i(3)), **bad})
    good = dict(q=f(3, 4, 64), block_table=i(2, 3), lens=i(2), q_start=i(3), workspace=f(1 << 10, dtype=torch.uint8))
    for bad in (dict(q=f(3, 4, 32)), dict(q=f(3, 4, 128)[:, :, ::2]), dict(block_table=i(3, 3)), dict(block_table=f(2, 3)), dict(lens=f(2)),
                dict(q_start=i(2)), dict(out=f(2, 4, 64)), dict(out=h(3, 4, 64)), dict(window=1 << 32), dict(window=-1),
                dict(workspace=torch.zeros(1 << 10, dtype=torch.uint8, device="meta"))):
        with pytest.raises(ValueError):
            pcg.cache4_attend(four, **{**good, **bad})


def test_tables_of_an_odd_number_of_elements_are_refused():
    """An odd dim would give the angles of one more element, and pairs of one less."""
    assert pcg.Rotation.of(3, 6, "cpu").dim == 6
    for dim in (1, 7, 0, -2):
        with pytest.raises(ValueError):
            pcg.Rotation.of(3, dim, "cpu")
    for positions in (0, -1):
        with pytest.raises(ValueError):
            pcg.Rotation.of(positions, 6, "cpu")


def test_objects_whose_fields_are_replaced_name_the_new_ones():
    new = lambda n, dtype=torch.uint8: torch.zeros((4, 16, 2, n), dtype=dtype)  # noqa: E731
    cache = pcg.KvCache4(new(32), new(32), new(2, torch.bfloat16), 64)
    k, v, s = new(32), new(32), new(2, torch.bfloat16)
    cache.k, cache.v, cache.scales = k, v, s
    r = cache._ref.contents
    assert (r.k, r.v, r.scales) == (k.data_ptr(), v.data_ptr(), s.data_ptr())
    cache.head_dim = 40
    assert cache._ref.contents.head_dim == 40
    turn, table = pcg.Rotation(torch.zeros(9, 64)), torch.zeros(5, 32)
    turn.table = table
    turn.interleaved = True
    r = turn._ref.contents
    assert (r.table, r.positions, r.dim, r.interleaved) == (table.data_ptr(), 5, 32, 1) and (turn.positions, turn.dim) == (5, 32)


def test_sizes_that_the_library_would_take_for_others_are_refused():
    """Beyond 2^31, on a device that holds no memory."""
    far = 1 << 32
    new = lambda *s, dtype=torch.uint8: torch.empty(s, dtype=dtype, device="meta")  # noqa: E731
    for shape in ((far, 1, 1), (1, far, 1), (1, 1, far)):
        with pytest.raises(ValueError):
            pcg.KvCache4(new(*shape, 32), new(*shape, 32), new(*shape, 2, dtype=torch.bfloat16), 64)
    with pytest.raises(ValueError):
        pcg.KvCache4(new(1, 1, 1, far // 2), new(1, 1, 1, far // 2), new(1, 1, 1, 2, dtype=torch.bfloat16), far)
    for shape in ((far, 2), (1, far)):
        with pytest.raises(ValueError):
            pcg.Rotation(new(*shape, dtype=torch.float32))


# ------------------------------------------------------------------ the plain forms, by hand

def test_plain_rotation_by_hand():
    x = torch.tensor([[[1.0, 2.0, 3.0, 4.0, 5.0]]])
    rows = torch.tensor([[0.0, 0.5, 1.0, -1.0]])                  # cosines 0, 1/2, sines 1, -1
    assert ref.rotate(x, rows, False).tolist() == [[[0 - 3.0, 1.0 + 4.0, 0 + 1.0, 2.0 - 2.0, 5.0]]]
    assert ref.rotate(x, rows, True).tolist() == [[[0 - 2.0, 0 + 1.0, 1.5 + 4.0, 2.0 - 3.0, 5.0]]]


def test_plain_codes_by_hand():
    x = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.25, -0.3, 0.0])
    codes, scale = ref.quantise(x)
    assert scale.item() == 1.0 and codes.tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 15, 9, 0]
    assert ref.values(codes, scale).tolist() == [6.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, -6.0, -0.5, 0.0]
    bits = ref.packed(codes)
    assert bits.shape == (16,) and bits[:2].tolist() == [0x07, 0x22] and torch.equal(ref.unpacked(bits, 11), codes)
    codes, scale = ref.quantise(torch.tensor([[1.0, math.inf], [0.0, 0.0], [-3.4e38, 0.0]]))
    assert math.isnan(scale[0]) and codes[0].tolist() == [0, 0] and codes[1].tolist() == [0, 0] and scale[1] == 0
    assert codes[2, 0] == 15 and math.isfinite(6 * float(scale[2]))
