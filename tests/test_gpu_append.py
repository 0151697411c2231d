"""New rows into a paged cache with the rotation on the way (pcg_cache_append), into a cache of 4-bit codes (pcg_cache4_append) and back
out of it (pcg_cache4_read), bit by bit against their definitions.  Run with ``-m gpu`` on an MI355X."""
import math

import pytest
import torch

import cache4 as ref
import paper_2511_13732_amd as pcg

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rows_of(T, H, G, D, dtype, seed, sigma=1.0):
    """Queries, keys and values as parts of a projection's row, with a gap between them."""
    x = (sigma * torch.randn((T, H + 2 * G + 1, D), generator=gen(seed))).to(dtype).cuda()
    return x[:, :H], x[:, H + 1:H + 1 + G], x[:, H + 1 + G:]


def slots_of(T, pages, page_size, seed, out=0.2):
    """Slots in any order, some rows left out: no slot, or one past the cache's last."""
    g = gen(seed)
    slots = torch.randperm(pages * page_size, generator=g)[:T].int()
    kind = torch.rand(T, generator=g)
    slots[kind < out / 2] = -1
    slots[(kind >= out / 2) & (kind < out)] = pages * page_size + 3
    return slots


def empty4(pages, page_size, G, D, layout):
    """A cache of 4 bits that holds what no call writes."""
    if layout == "heads":
        c = pcg.KvCache4.empty(pages, page_size, G, D, "cuda")
    else:                              # keys, values and scales beside each other
        row = -(-D // 32) * 16
        x = torch.zeros((pages, page_size, G, 2 * row + 16), dtype=torch.uint8, device="cuda")
        c = pcg.KvCache4(x[..., :row], x[..., row:2 * row], x[..., 2 * row + 4:2 * row + 8].view(torch.bfloat16), D)
    c.k.fill_(0xab)
    c.v.fill_(0xcd)
    c.scales.fill_(11.0)
    return c


def check(T, H, G, D, dtype, rot, interleaved, page_size, layout, four, seed, places=90, table=None, in_place=False, sigma=1.0, k=None, v=None):
    dt, pages = DTYPES[dtype], -(-T // page_size) + 2
    q, kr, vr = rows_of(T, H, G, D, dt, seed, sigma)
    k, v = kr if k is None else k, vr if v is None else v
    slots = slots_of(T, pages, page_size, seed + 1)
    positions = torch.randint(0, places, (T,), generator=gen(seed + 2)).int()
    away = torch.rand(T, generator=gen(seed + 3)) < 0.1
    positions[away] = torch.where(torch.rand(int(away.sum()), generator=gen(seed + 4)) < 0.5, -1, places).int()
    rotation = pcg.Rotation(torch.randn((places, rot), generator=gen(seed + 5)).cuda() if table is None else table, interleaved)
    there = (slots >= 0) & (slots < pages * page_size) & ~away
    at = there.nonzero()[:, 0]
    page, slot = slots[at].long() // page_size, slots[at].long() % page_size
    turn = rotation.table.cpu()[positions[at].long()]
    want_q = ref.rotate(q[at.cuda()], turn, interleaved).to(dt)
    want_k, want_v = ref.rotate(k[at.cuda()], turn, interleaved), v[at.cuda()].cpu()
    q_out = q if in_place else torch.full((T, H, D), 77.0, dtype=dt, device="cuda")
    before = q_out.clone()
    if four:
        cache = empty4(pages, page_size, G, D, layout)
        got = pcg.cache4_append(cache, k, v, slots.cuda(), rotation=rotation, positions=positions.cuda(), q=q, q_out=q_out)
    else:
        shape = (pages, G, page_size, D) if layout == "heads" else (pages, page_size, G, D)
        held = [torch.full(shape, 55.0, dtype=dt, device="cuda") for _ in range(2)]
        cache = pcg.KvCache(*(x.transpose(1, 2) if layout == "heads" else x for x in held))
        got = pcg.cache_append(cache, k, v, slots.cuda(), rotation=rotation, positions=positions.cuda(), q=q, q_out=q_out)
    assert got is q_out
    assert torch.equal(q_out.cpu()[at], want_q) and torch.equal(q_out[~there.cuda()], before[~there.cuda()])
    rest = torch.ones((pages, page_size), dtype=torch.bool)
    rest[page, slot] = False
    if not four:
        assert torch.equal(cache.k.cpu()[page, slot], want_k.to(dt)) and torch.equal(cache.v.cpu()[page, slot], want_v)
        assert (cache.k.cpu()[rest] == 55.0).all() and (cache.v.cpu()[rest] == 55.0).all()
        return
    again = min(T, 3)
    read = torch.cat([slots, slots[:again], torch.full((2,), -5, dtype=torch.int32)]).cuda()
    for of in DTYPES.values():
        out = tuple(torch.full((T + again + 2, G + 1, D), 33.0, dtype=of, device="cuda")[:, 1:] for _ in range(2))
        assert pcg.cache4_read(cache, read, out=out)[0] is out[0]
        for i, (x, bits, fill) in enumerate(((want_k, cache.k, 0xab), (want_v, cache.v, 0xcd))):
            codes, scale = ref.quantise(x.float())
            mine = bits.cpu()[page, slot]
            assert torch.equal(cache.scales.cpu()[page, slot][..., i].view(torch.int16), scale.view(torch.int16))
            # a zero may have either sign where the number was one
            assert torch.equal(mine, ref.packed(torch.where(codes % 8 == 0, ref.unpacked(mine, D) & 8, codes)))
            assert (bits.cpu()[rest] == fill).all() and (cache.scales.cpu()[rest] == 11.0).all()
            assert torch.equal(out[i][:T].cpu()[at], ref.values(codes, scale).to(of))
            inside = ((slots >= 0) & (slots < pages * page_size)).cuda()
            assert (out[i][:T][~inside] == 33.0).all() and (out[i][T + again:] == 33.0).all() and torch.equal(out[i][T:T + again], out[i][:again])


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,rot", [(128, 128), (128, 64), (64, 32), (64, 2), (72, 72), (80, 48), (96, 20), (8, 8), (8, 6), (120, 118)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_head_sizes_and_rotated_parts(four, dtype, D, rot, interleaved):
    check(37, 6, 2, D, dtype, rot, interleaved, 16, "heads", four, seed=D + rot)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 63, 1000])
@pytest.mark.parametrize("H,G,page_size,layout", [(1, 1, 1, "slots"), (15, 5, 7, "slots"), (32, 8, 64, "heads")])
def test_heads_and_pages(four, dtype, T, H, G, page_size, layout):
    check(T, H, G, 64, dtype, 64, False, page_size, layout, four, seed=T + H)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rot,interleaved", [(128, False), (96, True), (34, False)])
def test_rows_turned_in_place(four, dtype, rot, interleaved):
    check(50, 5, 1, 128, dtype, rot, interleaved, 16, "slots", four, seed=rot, in_place=True)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tables_of_any_alignment(four, dtype):
    wide = torch.randn((40, 71), generator=gen(3)).cuda()
    for table in (wide[:, 3:67], wide[:, 4:68], wide[::2, :64], wide[:1, :64]):
        check(21, 4, 2, 64, dtype, 64, False, 16, "heads", four, seed=5, places=table.shape[0], table=table)
        check(21, 4, 2, 64, dtype, 64, True, 16, "heads", four, seed=6, places=table.shape[0], table=table)


def test_far_positions():
    """The angles of a position of a million, formed in double: the table's error is its rounding to float32."""
    r = pcg.Rotation.of(1_000_001, 16, "cuda")
    i = torch.arange(8, dtype=torch.float64)
    angle = 1_000_000 * 10000.0 ** (-i / 8)
    # an angle is off by a few steps of double at its size, 2^20
    assert (r.table[-1].double().cpu() - torch.cat([angle.cos(), angle.sin()])).abs().max() <= 2.0 ** -25 + 4 * 2.0 ** (20 - 53)
    check(9, 2, 1, 16, "f32", 16, False, 16, "heads", False, seed=1, places=1_000_001, table=r.table)


@pytest.mark.parametrize("four", [False, True])
def test_without_rotation(four):
    T, G, D = 30, 3, 72
    _, k, v = rows_of(T, 1, G, D, torch.float32, 9)
    slots = torch.randperm(48, generator=gen(1))[:T].int().cuda()
    if not four:
        a, b = (pcg.KvCache(*(torch.zeros((3, 16, G, D), device="cuda") for _ in range(2))) for _ in range(2))
        assert pcg.cache_append(a, k, v, slots) is None
        pcg.cache_write(b, k, v, slots)
        assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v)
        return
    c = pcg.KvCache4.empty(3, 16, G, D, "cuda")
    assert pcg.cache4_append(c, k, v, slots) is None
    for got, x in zip(pcg.cache4_read(c, slots, dtype=torch.float32), (k, v)):
        assert torch.equal(got.double().cpu(), ref.values(*ref.quantise(x)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_numbers_on_borders_and_at_the_ends_of_the_range(dtype):
    """Ties, numbers a step beside them, zeros, the smallest and largest numbers, and what is not finite."""
    dt, D = DTYPES[dtype], 64
    eps = torch.finfo(dt).eps
    borders = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    line = [x * f for x in borders for f in (1, 1 - eps / 2, 1 + eps)] + [6.0, 0.0, -0.0]
    line += [-x for x in line]
    line = torch.tensor((line + [0.0] * D)[:D], dtype=torch.float64)
    some = []
    for unit in (1.0, 1.5, 1.9921875, 1.0078125):
        for e in (0, 10, -30, 120, -120):
            some.append(line * unit * 2.0 ** e)
    some += [line * 0, line * 2.0 ** -130, line * 2.0 ** -148, line / 6 * torch.finfo(dt).max, torch.full((D,), torch.finfo(dt).max, dtype=torch.float64)]
    x = torch.stack(some).to(dt)[:, None]
    assert torch.isfinite(x).all()
    odd = x[:3].clone()
    odd[0, 0, 5], odd[1, 0, 63], odd[2, 0, 0] = math.inf, math.nan, -math.inf
    x = torch.cat([x, odd, x[:1]]).expand(-1, 2, -1).contiguous()
    x[-1, 1] = math.nan                                   # one head's numbers do not touch another's
    T = x.shape[0]
    c, slots = pcg.KvCache4.empty(T, 1, 2, D, "cuda"), torch.arange(T, dtype=torch.int32).cuda()
    pcg.cache4_append(c, x.cuda(), -x.cuda(), slots)
    for i, (bits, y) in enumerate(((c.k, x), (c.v, -x))):
        codes, scale = ref.quantise(y.float())
        mine = ref.unpacked(bits[:, 0].cpu(), D)
        assert torch.equal(torch.isnan(scale), torch.isnan(c.scales[:, 0, :, i].cpu()))
        fine = torch.isfinite(scale)
        assert torch.equal(c.scales[:, 0, :, i].cpu()[fine], scale[fine])
        assert torch.equal(torch.where(codes % 8 == 0, mine & 7, mine), torch.where(codes % 8 == 0, 0, codes))
    got = pcg.cache4_read(c, slots, dtype=torch.float32)[0].cpu()
    assert torch.isfinite(got[:T - 4]).all() and torch.isnan(got[T - 4:T - 1]).all()
    assert torch.isfinite(got[-1, 0]).all() and torch.isnan(got[-1, 1]).all()


def test_no_rows():
    c4 = pcg.KvCache4.empty(2, 16, 2, 64, "cuda")
    c = pcg.KvCache(torch.zeros((2, 16, 2, 64), device="cuda"), torch.zeros((2, 16, 2, 64), device="cuda"))
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    e = torch.zeros((0, 2, 64), device="cuda")
    r = pcg.Rotation.of(4, 64, "cuda")
    assert pcg.cache_append(c, e, e, none, rotation=r, positions=none, q=e).shape == (0, 2, 64)
    assert pcg.cache4_append(c4, e, e, none, rotation=r, positions=none, q=e).shape == (0, 2, 64)
    assert pcg.cache4_read(c4, none)[0].shape == (0, 2, 64)


def test_another_stream_and_a_graph():
    """A captured call replayed with other rows in the same places, on a stream of its own."""
    T, H, G, D = 40, 8, 2, 128
    c, r = pcg.KvCache4.empty(4, 16, G, D, "cuda"), pcg.Rotation.of(100, D, "cuda")
    q, k, v = (torch.zeros((T, n, D), dtype=torch.bfloat16, device="cuda") for n in (H, G, G))
    slots, positions = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda")
    q_out = torch.zeros_like(q)
    back = [torch.zeros_like(k), torch.zeros_like(k)]
    stream = torch.cuda.Stream()

    def both():
        pcg.cache4_append(c, k, v, slots, rotation=r, positions=positions, q=q, q_out=q_out)
        pcg.cache4_read(c, slots, out=back)

    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        both()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            both()
    for it in range(3):
        g = gen(it)
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=g))
        slots.copy_(torch.randperm(64, generator=g)[:T])
        positions.copy_(torch.randint(0, 100, (T,), generator=g))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        turn = r.table.cpu()[positions.cpu().long()]
        assert torch.equal(q_out.cpu(), ref.rotate(q, turn, False).to(q.dtype))
        for got, x in zip(back, (ref.rotate(k, turn, False), v.cpu().float())):
            assert torch.equal(got.cpu(), ref.values(*ref.quantise(x)).to(torch.bfloat16))
