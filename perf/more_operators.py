"""More operators around one speculative step's forward pass, as cases that can be timed and compared: new keys and values into
the paged cache with the position rotation of keys and queries on the way (`append`), the same into a cache held in 4 bits and
back as the values that it then holds (`append4`), and the attention of new tokens over such a cache (`attend4`).

With `own` false every operator is computed in its plain form, by elementary tensor operations; with `own` true by the library's
calls.  Lengths are a function of the case alone (the seed deals them to the requests in another order), so that `work` knows them.

Rotation: a table row of a position holds the cosines of dim / 2 angles and then their sines.  Elements (a, b) of a head are a pair
(i and i + dim / 2, or 2 i and 2 i + 1 where `pairs` is "next") and become (a cos - b sin, b cos + a sin); elements behind dim stay.

4 bits: an element is scale * code, with one bfloat16 scale a token and shared head for its key and one for its value, and codes of one
sign, two exponent and one mantissa bit: 0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives.  The scale is the largest absolute value / 6 rounded to
bfloat16, the code the nearest one, ties to the even one; keys are rounded to float32 once they are rotated.

A case is a dict:
  call        "append" | "append4" | "attend4"
  B           requests
  ctx         the longest request's tokens in the cache; the others' spread down to `short` of it
  chunk       new tokens of a request: K + 1 in a step, 1 in plain decoding, more where a prompt goes in by pieces;
              `ragged`: from one to that many
  heads, kv_heads, head_dim, dtype, page_size, window (0: none)
  rotate      rotated elements of a head; pairs "half" or "next"
  layout      of the cache: "slots" ([page, slot, head, :]) or "heads" ([page, head, slot, :])
  padding     rows of the batch behind the last request's (a captured graph has a fixed number of rows)
"""
import math
import random

import torch

own = False

_MODEL = dict(heads=32, kv_heads=8, head_dim=128, dtype="bf16", rotate=128, pairs="half")
_BASE = dict(_MODEL, B=64, ctx=2000, short=0.25, chunk=9, ragged=False, page_size=16, window=0, layout="slots", padding=0)


def listed():
    return [
        # one interactive sequence's new tokens of one layer: latency is all there is
        dict(_BASE, name="append_b1_k3", call="append", B=1, chunk=4, ctx=700),
        # the serving batch's step of eight drafted tokens, one layer
        dict(_BASE, name="append_b64_k8", call="append", padding=24),
        # a batch of prompts, fp32, half of every head rotated in neighbouring pairs, pages by heads
        dict(_BASE, name="append_prompts_f32", call="append", B=16, ctx=0, chunk=2048, ragged=True, dtype="f32", head_dim=64, rotate=32,
             pairs="next", heads=16, layout="heads", page_size=64),
        # the serving batch's step into a cache of 4 bits
        dict(_BASE, name="append4_b64_k8", call="append4", padding=24, layout="heads"),
        # a batch of prompts that goes into it
        dict(_BASE, name="append4_prompts", call="append4", B=24, ctx=0, chunk=3000, ragged=True, page_size=64, layout="heads"),
        # plain decoding of one sequence, a token a pass
        dict(_BASE, name="attend4_b1_decode", call="attend4", B=1, chunk=1, ctx=1500, layout="heads"),
        # the target's pass over the full serving batch: nine new tokens a sequence
        dict(_BASE, name="attend4_b64_k8", call="attend4", padding=24, layout="heads"),
        # plain decoding of a large batch, which such a cache makes room for
        dict(_BASE, name="attend4_b128_decode", call="attend4", B=128, chunk=1, ctx=6000),
        # few long sequences: what is read is split over the whole chip
        dict(_BASE, name="attend4_b2_ctx120k", call="attend4", B=2, ctx=120000, short=0.9, page_size=64, layout="heads"),
        # prompts that go in by pieces next to sequences that decode
        dict(_BASE, name="attend4_b8_pieces", call="attend4", B=8, ctx=8000, chunk=1024, ragged=True, page_size=32, layout="heads"),
        # fp32 queries, a head size and a ratio of heads that fit nothing, a sliding window
        dict(_BASE, name="attend4_b12_f32_window", call="attend4", B=12, heads=15, kv_heads=5, head_dim=80, rotate=80, dtype="f32",
             chunk=7, ragged=True, window=1000, page_size=24, ctx=4001),
        # fp32 queries of a draft model whose heads share nothing
        dict(_BASE, name="attend4_b32_f32", call="attend4", B=32, heads=12, kv_heads=12, head_dim=64, rotate=64, dtype="f32", chunk=5,
             ctx=3500, layout="heads"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    c = dict(_BASE, call=rng.choice(["append"] * 2 + ["append4"] * 2 + ["attend4"] * 4))
    c["B"] = _log_uniform(rng, 1, 128)
    c["kv_heads"] = rng.choice([1, 2, 4, 5, 8, 8])
    c["heads"] = c["kv_heads"] * rng.choice([1, 3, 4, 4, 7, 8])
    c["head_dim"] = rng.choice([128, 128, 64, 64, 80, 96, 8 * rng.randint(1, 16)])
    c["rotate"] = rng.choice([c["head_dim"], c["head_dim"], 2 * rng.randint(1, c["head_dim"] // 2)])
    c["pairs"] = rng.choice(["half", "half", "next"])
    c["dtype"] = rng.choice(["bf16", "bf16", "f32"])
    c["page_size"] = rng.choice([16, 16, 32, 64, 128, rng.randint(1, 100)])
    c["layout"] = rng.choice(["slots", "heads"])
    c["window"] = rng.choice([0, 0, 0, _log_uniform(rng, 16, 4096)])
    c["short"] = rng.choice([0.02, 0.25, 1.0])
    c["ctx"] = _log_uniform(rng, 1, 60000)
    c["chunk"] = rng.choice([1, rng.randint(2, 9), rng.randint(2, 17), _log_uniform(rng, 16, 2000)])
    c["ragged"] = rng.random() < 0.5
    c["padding"] = rng.choice([0, rng.randint(1, 64)])
    # no more than the largest listed cases
    while c["B"] > 1 and _too_much(c):
        c["B"] -= max(1, c["B"] // 8)
    while _too_much(c):
        c["ctx"], c["chunk"] = c["ctx"] * 3 // 4, max(1, c["chunk"] * 3 // 4)
    return c


def _too_much(c):
    w = work(c)
    return (w["bytes"] > 0.45e9 or w["flops"] > (6e10 if c["dtype"] == "f32" else 2e11) or sum(m for _, m in _lengths(c)) > 24000 or
            _cache_elems(c) > 1.0e9)


# ------------------------------------------------------------------------------------ lengths

def _spread(n, key):
    """(i + 1/2) / n in an order that only n and key decide, the largest among them made 1."""
    u = [(i + 0.5) / n for i in range(n - 1)] + [1.0]
    random.Random(1000 * n + key).shuffle(u)
    return u


def _lengths(c):
    """[(tokens in the cache, new tokens)] of the requests."""
    B = c["B"]
    ctx = [round(c["ctx"] * (c["short"] + (1 - c["short"]) * u)) for u in _spread(B, 1)]
    new = [max(1, round(c["chunk"] * u * u)) if c["ragged"] else c["chunk"] for u in _spread(B, 2)]
    return list(zip(ctx, new))


def _dealt(c, seed):
    pairs = _lengths(c)
    random.Random(seed).shuffle(pairs)
    return pairs


def _pairs(c):
    """How many (row, key) pairs one head sees, and how many keys of the cache anybody sees."""
    seen = keys = 0
    for n, m in _lengths(c):
        w = c["window"] or n + m
        # row at position p sees min(p + 1, w) keys
        a, b = n + 1, n + m
        full = max(0, b - max(a, w) + 1)
        some = m - full
        seen += full * w + some * (a + a + some - 1) // 2
        keys += n + m - max(0, n + 1 - w)
    return seen, keys


def _blocks(c, n):
    return -(-n // c["page_size"])


def _cache_elems(c):
    pages = sum(_blocks(c, n + m) for n, m in _lengths(c))
    return 2 * pages * c["page_size"] * c["kv_heads"] * c["head_dim"]


def _row4(c):
    """Bytes of a token's key or value in 4 bits, all shared heads: codes and a scale each."""
    return c["kv_heads"] * (c["head_dim"] / 2 + 2)


def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    new = sum(m for _, m in _lengths(c))
    kv, q = c["kv_heads"] * c["head_dim"] * e, c["heads"] * c["head_dim"] * e
    if c["call"] == "attend4":
        seen, keys = _pairs(c)
        return {"bytes": 2 * keys * _row4(c) + 2 * new * q, "flops": 4.0 * c["head_dim"] * c["heads"] * seen}
    # a row of the rotation's table, a position and a slot a token; queries in and out, keys and values in
    row = 2 * q + 2 * kv + 4 * c["rotate"] + 8
    flops = 3.0 * (c["heads"] + c["kv_heads"]) * c["rotate"]
    if c["call"] == "append":
        return {"bytes": new * (row + 2 * kv), "flops": new * flops}
    # into the cache, and read back from it as values
    return {"bytes": new * (row + 4 * _row4(c) + 2 * kv), "flops": new * (flops + 4.0 * c["kv_heads"] * c["head_dim"])}


# ------------------------------------------------------------------------------------- inputs

def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _generator(seed, purpose):
    return torch.Generator(device="cuda").manual_seed(7_919 * (seed + 1) + purpose)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def _qkv(c, rows, seed):
    """Queries, keys and values of `rows` tokens as a projection leaves them: parts of one row."""
    H, G, D = c["heads"], c["kv_heads"], c["head_dim"]
    x = torch.randn((rows, H + 2 * G, D), device="cuda", generator=_generator(seed, 1))
    x[:, :H] *= 2.0          # logits with a standard deviation of two: some rows are sharp, most are not
    x = x.to(_dtype(c))
    return x[:, :H], x[:, H:H + G], x[:, H + G:]


def _new_cache(c, pages):
    """Keys and values, of the dtype or (call "append4", "attend4") as codes two a byte, with their scales."""
    P, G, D = c["page_size"], c["kv_heads"], c["head_dim"]

    def make(last, dtype):
        if c["layout"] == "heads":
            return torch.zeros((pages, G, P, last), dtype=dtype, device="cuda").transpose(1, 2)
        return torch.zeros((pages, P, G, last), dtype=dtype, device="cuda")

    if c["call"] == "append":
        return [make(D, _dtype(c)) for _ in range(2)]
    # codes in pieces of 16 bytes, two scales a token and head
    return [make(-(-D // 32) * 16, torch.uint8) for _ in range(2)] + [make(2, torch.bfloat16)]


def _fill_cache(c, cache, seed):
    """Keys and values of earlier tokens, normally distributed, each head of a size of its own."""
    g, G, D = _generator(seed, 2), c["kv_heads"], c["head_dim"]
    P = c["page_size"]
    size = torch.exp(0.3 * torch.randn((2, G, 1), device="cuda", generator=g))
    step = max(1, (1 << 26) // (P * G * D))
    for lo in range(0, cache[0].shape[0], step):
        hi = min(cache[0].shape[0], lo + step)
        for i in range(2):
            codes, scale = _quantise(torch.randn((hi - lo, P, G, D), device="cuda", generator=g) * size[i])
            cache[i][lo:hi] = _packed(codes, cache[i].shape[3])
            cache[2][lo:hi, :, :, i] = scale


def prepare(case, seed):
    c = case
    pairs = _dealt(c, seed)
    starts = [0]
    for _, m in pairs:
        starts.append(starts[-1] + m)
    rows = starts[-1] + c["padding"]
    q, k, v = _qkv(c, rows, seed)
    out = torch.zeros((rows, c["heads"], c["head_dim"]), dtype=q.dtype, device="cuda")
    s = dict(call=c["call"], case=c, pairs=pairs, starts=starts, q=q, out=out)
    held = [_blocks(c, n + m) for n, m in pairs]
    order = list(range(sum(held)))
    random.Random(seed).shuffle(order)
    table = torch.zeros((c["B"], max(held) + 1), dtype=torch.int32)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    s["cache"] = _new_cache(c, sum(held))
    if c["call"] == "attend4":
        _fill_cache(c, s["cache"], seed)
        s.update(table=table.cuda(), lens=_i32([n for n, _ in pairs]), q_start=_i32(starts), scale=1.0 / math.sqrt(c["head_dim"]),
                 longest=max(m for _, m in pairs))
    else:
        slots = torch.full((rows,), -1, dtype=torch.int32)
        positions = torch.zeros(rows, dtype=torch.int32)
        for b, (n, m) in enumerate(pairs):
            p = torch.arange(n, n + m)
            positions[starts[b]:starts[b + 1]] = p.int()
            slots[starts[b]:starts[b + 1]] = table[b, p // c["page_size"]] * c["page_size"] + (p % c["page_size"]).int()
        longest = max(n + m for n, m in pairs)
        half = c["rotate"] // 2
        angle = torch.arange(longest, device="cuda").double()[:, None] * 10000.0 ** (-torch.arange(half, device="cuda").double() / half)
        s.update(k=k, v=v, slots=slots.cuda(), positions=positions.cuda(),
                 table=torch.cat([angle.cos(), angle.sin()], dim=1).float())
    if c["call"] == "append4":
        s["back"] = [torch.zeros((rows, c["kv_heads"], c["head_dim"]), dtype=q.dtype, device="cuda") for _ in range(2)]
    if own:
        import paper_2511_13732_amd as pcg
        s["kv"] = pcg.KvCache(*s["cache"]) if c["call"] == "append" else pcg.KvCache4(*s["cache"], head_dim=c["head_dim"])
        if c["call"] == "attend4":
            n = pcg.cache4_attend_workspace_bytes(c["B"], rows, c["heads"], c["kv_heads"], c["head_dim"], s["longest"])
            s["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        else:
            s["rotation"] = pcg.Rotation(s["table"], interleaved=c["pairs"] == "next")
    return s


# -------------------------------------------------------------------------------- plain forms

_BORDERS = ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False))   # True: a tie goes up
_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _quantise(x):
    """(codes, scales) of float32 x [..., D]; a border times a scale is exact."""
    scale = (x.abs().amax(dim=-1) / 6.0).to(torch.bfloat16)
    size, unit = x.abs(), scale.float()[..., None]
    code = torch.zeros(x.shape, dtype=torch.uint8, device=x.device)
    for border, up in _BORDERS:
        code += (size >= border * unit) if up else (size > border * unit)
    code = torch.where(unit == 0, 0, code)
    return code + 8 * (x < 0).to(torch.uint8), scale


def _packed(codes, last):
    """Two codes a byte, the first in its low half."""
    pad = torch.zeros((*codes.shape[:-1], 2 * last), dtype=torch.uint8, device=codes.device)
    pad[..., :codes.shape[-1]] = codes
    return pad[..., 0::2] + 16 * pad[..., 1::2]


def _values(packed, scale, D):
    """float32 values of packed codes [..., bytes] with scales [...]."""
    codes = torch.stack([packed & 15, packed >> 4], dim=-1).flatten(-2)[..., :D].long()
    level = torch.tensor(_LEVELS + tuple(-x for x in _LEVELS), device=packed.device)
    return level[codes] * scale.float()[..., None]


def _rotated(c, x, table):
    """Rows x [m, heads, D] in double, each turned by its row [m, rotate] of the table."""
    x, table, half = x.double(), table.double()[:, None], c["rotate"] // 2
    cos, sin = table[..., :half], table[..., half:]
    if c["pairs"] == "next":
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([turned, x[..., 2 * half:]], dim=-1)


def _plain_append(s):
    c, cache, there = s["case"], s["cache"], torch.nonzero(s["slots"] >= 0)[:, 0]
    at, table = s["slots"][there].long(), s["table"][s["positions"][there].long()]
    page = torch.div(at, c["page_size"], rounding_mode="floor")
    slot = at - page * c["page_size"]
    s["out"][there] = _rotated(c, s["q"][there], table).to(s["out"].dtype)
    keys, values = _rotated(c, s["k"][there], table).float(), s["v"][there]
    if c["call"] == "append":
        cache[0][page, slot], cache[1][page, slot] = keys.to(values.dtype), values
        return [s["out"], *cache]
    for i, x in enumerate((keys, values.float())):
        codes, scale = _quantise(x)
        cache[i][page, slot] = _packed(codes, cache[i].shape[3])
        cache[2][page, slot, :, i] = scale
        s["back"][i][there] = _values(cache[i][page, slot], cache[2][page, slot, :, i], c["head_dim"]).to(values.dtype)
    return [s["out"], *s["back"]]


def _plain_rows(q, k, v, first, scale, window):
    """Rows q [m, H, D] at positions first, first + 1, .. of a sequence with keys k, values v [n, G, D]; float32."""
    m, H, D = q.shape
    n, G, _ = k.shape
    out = torch.empty((G, H // G, m, D), dtype=torch.float32, device=q.device)
    q = q.float().view(m, G, H // G, D).permute(1, 2, 0, 3).contiguous()
    k, v = k.permute(1, 2, 0).contiguous(), v.transpose(0, 1).contiguous()
    step = max(1, (1 << 28) // (n * (H // G)))           # scores of a gigabyte at most
    for lo in range(0, m, step):
        hi = min(m, lo + step)
        p = first + torch.arange(lo, hi, device=q.device)[:, None]
        j = torch.arange(n, device=q.device)[None]
        hidden = (j > p) | (j <= p - window) if window else j > p
        for g in range(G):
            x = torch.matmul(q[g, :, lo:hi], k[g]) * scale
            x = x.masked_fill(hidden, -math.inf)
            x = torch.exp(x - x.amax(dim=2, keepdim=True))
            out[g, :, lo:hi] = torch.matmul(x, v[g]) / x.sum(dim=2, keepdim=True)
    return out.permute(2, 0, 1, 3).reshape(m, H, D)


def _plain_attend(s):
    c, out = s["case"], s["out"]
    for b, (n, m) in enumerate(s["pairs"]):
        lo, hi = s["starts"][b], s["starts"][b + 1]
        pages = s["table"][b, :_blocks(c, n + m)].long()
        held = [x[pages].flatten(0, 1)[:n + m] for x in s["cache"]]
        k, v = (_values(held[i], held[2][..., i], c["head_dim"]) for i in range(2))
        out[lo:hi] = _plain_rows(s["q"][lo:hi], k, v, n, s["scale"], c["window"]).to(out.dtype)
    return out


def run(state):
    s = state
    if not own:
        return _plain_attend(s) if s["call"] == "attend4" else _plain_append(s)
    import paper_2511_13732_amd as pcg
    if s["call"] == "append":
        pcg.cache_append(s["kv"], s["k"], s["v"], s["slots"], rotation=s["rotation"], positions=s["positions"], q=s["q"], q_out=s["out"])
        return [s["out"], *s["cache"]]
    if s["call"] == "append4":
        pcg.cache4_append(s["kv"], s["k"], s["v"], s["slots"], rotation=s["rotation"], positions=s["positions"], q=s["q"], q_out=s["out"])
        pcg.cache4_read(s["kv"], s["slots"], out=s["back"])
        return [s["out"], *s["back"]]
    return pcg.cache4_attend(s["kv"], s["q"], s["table"], s["lens"], s["q_start"], longest=s["longest"], scale=s["scale"],
                             window=s["case"]["window"], out=s["out"], workspace=s["workspace"])


# ------------------------------------------------------------------------------------- 64 bits

def _turn(c, s, rows, x):
    """The rotation as a product of complex numbers."""
    half = c["rotate"] // 2
    t = s["table"][s["positions"][rows].long()].double()
    turn = torch.complex(t[:, :half], t[:, half:])[:, None]
    x = x.double()
    if c["pairs"] == "next":
        y = torch.view_as_real(torch.view_as_complex(x[..., :2 * half].reshape(*x.shape[:2], half, 2).contiguous()) * turn).reshape(*x.shape[:2], -1)
    else:
        y = torch.complex(x[..., :half].contiguous(), x[..., half:2 * half].contiguous()) * turn
        y = torch.cat([y.real, y.imag], dim=2)
    return torch.cat([y, x[..., 2 * half:]], dim=2)


def _nearest(x):
    """float32 x as the values that 4 bits hold of it, in double: the nearest level, ties to the one with an even number."""
    x = x.float().double()
    unit = (x.abs().amax(dim=2, keepdim=True) / 6.0).to(torch.bfloat16).double()
    level = torch.tensor(_LEVELS, dtype=torch.float64, device=x.device)
    off = (x.abs()[..., None] - level * unit[..., None]).abs()
    best = off.amin(dim=3, keepdim=True)
    even = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7], device=x.device)
    pick = even[(off == best)[..., even].to(torch.uint8).argmax(dim=3)]
    return level[pick] * unit * x.sign()


def exact(case, seed):
    """From the definitions, in double: rotated queries with the caches' new rows or the values held of them; attention."""
    c = case
    if work(c)["flops"] > 4e12:
        return None
    s = prepare(c, seed)
    if c["call"] != "attend4":
        rows = torch.nonzero(s["slots"] >= 0)[:, 0]
        out = s["out"].double()
        out[rows] = _turn(c, s, rows, s["q"][rows])
        keys, values = _turn(c, s, rows, s["k"][rows]), s["v"][rows].double()
        if c["call"] == "append":
            both = [x.double() for x in s["cache"]]
            at = s["slots"][rows].long()
            for x, new in zip(both, (keys, values)):
                x[at // c["page_size"], at % c["page_size"]] = new
            return [out, *both]
        back = [x.double() for x in s["back"]]
        for x, new in zip(back, (keys, values)):
            for some in rows.split(2048):
                at = torch.searchsorted(rows, some)
                x[some] = _nearest(new[at])
        return [out, *back]
    H, G, D = c["heads"], c["kv_heads"], c["head_dim"]
    level = torch.tensor(_LEVELS, dtype=torch.float64, device="cuda")
    out = torch.zeros((s["q"].shape[0], H, D), dtype=torch.float64, device="cuda")
    for b, (n, m) in enumerate(s["pairs"]):
        rows = s["starts"][b]
        pos = torch.arange(n + m, device="cuda")
        page, slot = s["table"][b].long()[pos // c["page_size"]], pos % c["page_size"]

        def held(i, g):
            x = s["cache"][i][page, slot, g][:, torch.arange(D, device="cuda") // 2].long() >> (4 * (torch.arange(D, device="cuda") % 2)) & 15
            return torch.where(x >= 8, -1.0, 1.0) * level[x % 8] * s["cache"][2][page, slot, g, i].double()[:, None]

        for g in range(G):
            keys, values = held(0, g), held(1, g)
            for lo in range(0, m, 512):
                hi = min(m, lo + 512)
                last = n + torch.arange(lo, hi, device="cuda")
                begin = max(0, n + lo - c["window"] + 1) if c["window"] else 0
                j = torch.arange(begin, n + hi, device="cuda")
                sees = j[None] <= last[:, None]
                if c["window"]:
                    sees &= j[None] > last[:, None] - c["window"]
                for h in range(g * (H // G), (g + 1) * (H // G)):
                    x = s["q"][rows + lo:rows + hi, h].double() @ keys[begin:n + hi].T
                    weight = torch.softmax(torch.where(sees, x * s["scale"], -math.inf), dim=1)
                    out[rows + lo:rows + hi, h] = weight @ values[begin:n + hi]
    return out
