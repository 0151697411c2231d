"""The operators around one speculative step's forward pass, as cases that can be timed and compared: the page table
and slot map of the step's new tokens (`pages`), their keys and values into the paged cache (`write`), their attention over it
(`attend`), and the attention of packed prompts before any step (`prompt`).

With `own` false every operator is computed in its plain form, by elementary tensor operations in 32 bits; with `own` true by the
library's calls.  Lengths are a function of the case alone (the seed deals them to the requests in another order), so that
`work` knows them.

A case is a dict:
  call        "pages" | "write" | "attend" | "prompt"
  B           requests
  ctx         the longest request's tokens in the cache (prompt: the longest prompt); the others' spread down to `short` of it
  chunk       new tokens of a request: K + 1 in a step, 1 in plain decoding, more where a prompt goes in by pieces;
              `ragged`: from one to that many
  heads, kv_heads, head_dim, dtype, page_size, window (0: none)
  layout      of the cache: "slots" ([page, slot, head, :]) or "heads" ([page, head, slot, :])
  ended       pages: a part of the requests that have ended, and as many that come with a prompt of up to `admit` tokens
  scarce      pages: the pool holds too few pages for everybody
  padding     rows of the batch behind the last request's (a captured graph has a fixed number of rows)
"""
import math
import random

import torch

own = False

_MODEL = dict(heads=32, kv_heads=8, head_dim=128, dtype="bf16")
_BASE = dict(_MODEL, B=64, ctx=2000, short=0.25, chunk=9, ragged=False, page_size=16, window=0, layout="slots",
             ended=0.0, admit=0, scarce=False, padding=0)


def listed():
    return [
        # bookkeeping of one interactive sequence: three drafted tokens, latency is all there is
        dict(_BASE, name="pages_b1_k3", call="pages", B=1, chunk=4, ctx=700),
        # bookkeeping of the full serving batch between two steps of eight drafted tokens
        dict(_BASE, name="pages_b64_k8", call="pages"),
        # a large pool where an eighth of the requests has ended and new prompts come in: tens of thousands of new tokens
        dict(_BASE, name="pages_b512_admit", call="pages", B=512, ended=0.125, admit=2048, page_size=32, padding=77),
        # the serving batch's new keys and values of one layer
        dict(_BASE, name="write_b64_k8", call="write", padding=24),
        # a batch of prompts' keys and values, fp32, pages by heads
        dict(_BASE, name="write_prompts_f32", call="write", B=16, ctx=0, chunk=2048, ragged=True, dtype="f32", head_dim=64,
             heads=16, layout="heads", page_size=64),
        # plain decoding of one sequence, a token a pass
        dict(_BASE, name="attend_b1_decode", call="attend", B=1, chunk=1, ctx=1500),
        # the target's pass over the full serving batch: nine new tokens a sequence
        dict(_BASE, name="attend_b64_k8", call="attend", padding=24),
        # few long sequences: what is read is split over the whole chip
        dict(_BASE, name="attend_b2_ctx120k", call="attend", B=2, ctx=120000, short=0.9, page_size=64, layout="heads"),
        # prompts that go in by pieces next to sequences that decode
        dict(_BASE, name="attend_b8_pieces", call="attend", B=8, ctx=8000, chunk=1024, ragged=True, page_size=32),
        # fp32, a head size and a ratio of heads that fit nothing, a sliding window
        dict(_BASE, name="attend_b12_f32_window", call="attend", B=12, heads=15, kv_heads=5, head_dim=80, dtype="f32",
             chunk=7, ragged=True, window=1000, page_size=24, ctx=4001),
        # a batch of prompts, packed
        dict(_BASE, name="prompt_b6_8k", call="prompt", B=6, ctx=8000, short=0.1, padding=13),
        # short fp32 prompts of a small draft model
        dict(_BASE, name="prompt_b9_f32", call="prompt", B=9, ctx=1111, heads=12, kv_heads=12, head_dim=64, dtype="f32"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    c = dict(_BASE, call=rng.choice(["pages", "write"] + ["attend"] * 3 + ["prompt"] * 2))
    c["B"] = _log_uniform(rng, 1, 512 if c["call"] == "pages" else 128)
    c["kv_heads"] = rng.choice([1, 2, 4, 5, 8, 8])
    c["heads"] = c["kv_heads"] * rng.choice([1, 3, 4, 4, 7, 8])
    c["head_dim"] = rng.choice([128, 128, 64, 64, 80, 96, 8 * rng.randint(1, 16)])
    c["dtype"] = rng.choice(["bf16", "bf16", "f32"])
    c["page_size"] = rng.choice([16, 16, 32, 64, 128, rng.randint(1, 100)])
    c["layout"] = rng.choice(["slots", "slots", "heads"])
    c["window"] = rng.choice([0, 0, 0, _log_uniform(rng, 16, 4096)])
    c["short"] = rng.choice([0.02, 0.25, 1.0])
    c["ctx"] = _log_uniform(rng, 1, 8000 if c["call"] == "prompt" else 60000)
    c["chunk"] = rng.choice([1, rng.randint(2, 9), rng.randint(2, 17), _log_uniform(rng, 16, 2000)])
    c["ragged"] = rng.random() < 0.5
    c["padding"] = rng.choice([0, rng.randint(1, 64)])
    if c["call"] == "pages":
        c["ended"] = rng.choice([0.0, 0.1, 0.5])
        c["admit"] = _log_uniform(rng, 1, 4000) if c["ended"] else 0
        c["scarce"] = rng.random() < 0.3
    # no more than the largest listed cases
    while c["B"] > 1 and _too_much(c):
        c["B"] -= max(1, c["B"] // 8)
    while _too_much(c):
        c["ctx"], c["chunk"] = c["ctx"] * 3 // 4, max(1, c["chunk"] * 3 // 4)
    return c


def _too_much(c):
    w = work(c)
    new, table = _places(c)
    return (w["bytes"] > 0.6e9 or w["flops"] > (1.2e11 if c["dtype"] == "f32" else 1.2e12) or new > 200000 or
            c["B"] * table > 2000000 or _cache_elems(c) * (4 if c["dtype"] == "f32" else 2) > 2.5e9)


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
    if c["call"] == "prompt":
        return [(0, max(1, n)) for n in ctx]
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


def _places(c):
    """(most new tokens of the batch, entries of a request's row of the table)"""
    new = sum(m for _, m in _lengths(c))
    if c["call"] == "pages":
        new += int(c["B"] * c["ended"]) * max(0, c["admit"])
    return new + c["padding"], _blocks(c, max(c["ctx"] + 2 * c["chunk"], c["admit"])) + 2


def _cache_elems(c):
    if c["call"] in ("pages", "prompt"):
        return 0
    pages = sum(_blocks(c, n + m) for n, m in _lengths(c))
    return 2 * pages * c["page_size"] * c["kv_heads"] * c["head_dim"]


def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    new = sum(m for _, m in _lengths(c))
    row = c["kv_heads"] * c["head_dim"] * e
    if c["call"] == "pages":
        # state read and written, kept and wanted tokens, chunk borders, a slot and a position a token
        return {"bytes": 4 * (2 * (3 * c["B"] + 1) + 3 * c["B"] + 1 + 2 * _places(c)[0]), "flops": 0}
    if c["call"] == "write":
        return {"bytes": new * (4 * row + 4), "flops": 0}
    seen, keys = _pairs(c)
    return {"bytes": 2 * keys * row + 2 * new * c["heads"] * c["head_dim"] * e, "flops": 4.0 * c["head_dim"] * c["heads"] * seen}


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


def _new_cache(c, pages, seed):
    shape = (pages, c["page_size"], c["kv_heads"], c["head_dim"])
    if c["layout"] == "heads":
        shape = (pages, c["kv_heads"], c["page_size"], c["head_dim"])
    g = _generator(seed, 2)
    both = [torch.randn(shape, device="cuda", generator=g, dtype=torch.float32).to(_dtype(c)) for _ in range(2)]
    return [x.transpose(1, 2) if c["layout"] == "heads" else x for x in both]


def _prepare_pages(c, seed):
    """A pool in the middle of serving: every request holds the pages of its tokens and of its last chunk."""
    rng = random.Random(seed)
    pairs = _dealt(c, seed)
    B, ps = c["B"], c["page_size"]
    rows, width = _places(c)
    lens, chunk = [n for n, _ in pairs], [m for _, m in pairs]
    held = [_blocks(c, n + m) for n, m in pairs]
    add = list(chunk)
    out = int(B * c["ended"])
    for b in rng.sample(range(B), out):
        add[b] = -1                                    # has ended: everything goes back
    fresh = rng.sample(range(B), out)
    for i, b in enumerate(fresh):                      # an empty place gets a new prompt
        lens[b] = chunk[b] = held[b] = 0
        add[b] = max(1, round(c["admit"] * (i + 1) / out))
    commit = [rng.randint(0, max(0, m - 1)) for m in chunk]
    # pages of the pool: what everybody held, and room for what comes (scarce: for little of it)
    coming = sum(_blocks(c, m) + 1 for _, m in pairs) + out * (_blocks(c, c["admit"]) + 1)
    total = sum(_blocks(c, n + m) for n, m in pairs) + (coming // 8 if c["scarce"] else coming)
    spare = total - sum(held)
    order = list(range(total))
    rng.shuffle(order)
    table = torch.zeros((B, width), dtype=torch.int32)
    at = 0
    for b in range(B):
        table[b, :held[b]] = torch.tensor(order[at:at + held[b]], dtype=torch.int32)
        at += held[b]
    free = order[at:] + [0] * at
    return dict(call="pages", B=B, page_size=ps, max_tokens=rows, table=table.cuda(), free=_i32(free),
                state=_i32(lens + held + chunk + [spare]), commit=_i32(commit), add=_i32(add))


def prepare(case, seed):
    c = case
    if c["call"] == "pages":
        s = _prepare_pages(c, seed)
        if own:
            import paper_2511_13732_amd as pcg
            s["pages"] = pcg.Pages(s["table"], s["free"], s["state"], c["page_size"])
            s["next"] = torch.empty_like(s["state"])
            s["out"] = pcg.pages_step_outputs(s["B"], s["max_tokens"], "cuda")
        return s
    pairs = _dealt(c, seed)
    starts = [0]
    for _, m in pairs:
        starts.append(starts[-1] + m)
    new = starts[-1]
    rows = new + c["padding"]
    q, k, v = _qkv(c, rows, seed)
    s = dict(call=c["call"], case=c, pairs=pairs, q=q, k=k, v=v, starts=starts, q_start=_i32(starts),
             scale=1.0 / math.sqrt(c["head_dim"]))
    if c["call"] == "prompt":
        s["out"] = torch.zeros((rows, c["heads"], c["head_dim"]), dtype=q.dtype, device="cuda")
        s["longest"] = max(m for _, m in pairs)
        return s
    rng = random.Random(seed)
    held = [_blocks(c, n + m) for n, m in pairs]
    total = sum(held)
    order = list(range(total))
    rng.shuffle(order)
    table = torch.zeros((c["B"], max(held) + 1), dtype=torch.int32)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    s["cache"] = _new_cache(c, total, seed)
    if c["call"] == "write":
        slots = torch.full((rows,), -1, dtype=torch.int32)
        for b, (n, m) in enumerate(pairs):
            p = torch.arange(n, n + m)
            slots[starts[b]:starts[b + 1]] = table[b, p // c["page_size"]] * c["page_size"] + (p % c["page_size"]).int()
        s["slots"] = slots.cuda()
    else:
        s["table"] = table.cuda()
        s["lens"] = _i32([n for n, _ in pairs])
        s["out"] = torch.zeros((rows, c["heads"], c["head_dim"]), dtype=q.dtype, device="cuda")
        s["longest"] = max(m for _, m in pairs)
    if own:
        import paper_2511_13732_amd as pcg
        s["kv"] = pcg.KvCache(*s["cache"])
        if c["call"] == "attend":
            n = pcg.cache_attend_workspace_bytes(c["B"], rows, c["heads"], c["kv_heads"], c["head_dim"], s["longest"])
            s["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return s


# -------------------------------------------------------------------------------- plain forms

def _ceil_div(a, b):
    return torch.div(a + (b - 1), b, rounding_mode="floor")


def _plain_pages(s):
    B, ps, room = s["B"], s["page_size"], s["table"].shape[1]
    lens, held, chunk = (s["state"][i * B:(i + 1) * B].long() for i in range(3))
    free = s["state"][3 * B].long()
    add, dev = s["add"].long(), s["add"].device
    kept = torch.minimum((s["commit"].long() + 1).clamp(min=0), chunk)
    lens = torch.where(add < 0, 0, lens + kept)
    want = add.clamp(min=0)
    need = _ceil_div(lens + want, ps)
    refused = need > room
    want = torch.where(refused, 0, want)
    refused = refused | ((want > 0) & (want.cumsum(0) > s["max_tokens"]))
    want = torch.where(refused, 0, want)
    need = torch.where(refused, held, need)
    back, take = (held - need).clamp(min=0), (need - held).clamp(min=0)
    top = free + back.sum()
    late = (take > 0) & (take.cumsum(0) > top)
    refused = refused | late
    need, want, take = torch.where(late, held, need), torch.where(late, 0, want), torch.where(late, 0, take)
    # given back, in order of request and block, onto the stack; taken from its top
    at = torch.arange(room, device=dev)
    gives = (at >= need[:, None]) & (at < held[:, None])
    pages = s["table"].long()[gives]
    stack = s["free"].long()
    stack[free + torch.arange(pages.numel(), device=dev)] = pages
    takes = (at >= held[:, None]) & (at < need[:, None])
    table = s["table"].long()
    table[takes] = stack[top - 1 - torch.arange(int(takes.sum()), device=dev)]
    q_start = torch.cat([torch.zeros(1, dtype=torch.long, device=dev), want.cumsum(0)])
    row = torch.arange(s["max_tokens"], device=dev)
    b = (row[:, None] >= q_start[None, 1:]).sum(1)
    there = b < B
    b = b.clamp(max=B - 1)
    position = torch.where(there, lens[b] + row - q_start[b], 0)
    block = torch.div(position, ps, rounding_mode="floor")
    slot = torch.where(there, table[b, block] * ps + position - block * ps, -1)
    state = torch.cat([lens, need, want, (top - take.sum())[None]])
    count = (refused & (add > 0)).sum()[None]
    return [x.to(torch.int32) for x in (state, table, stack, q_start, slot, position, count)]


def _plain_write(s):
    slots, (k, v) = s["slots"], s["cache"]
    there = slots >= 0
    at = slots[there].long()
    page = torch.div(at, k.shape[1], rounding_mode="floor")
    for cache, rows in ((k, s["k"]), (v, s["v"])):
        cache[page, at - page * k.shape[1]] = rows[there]
    return [k, v]


def _plain_rows(q, k, v, first, scale, window):
    """Rows q [m, H, D] at positions first, first + 1, .. of a sequence with keys k, values v [n, G, D]; float32."""
    m, H, D = q.shape
    n, G, _ = k.shape
    out = torch.empty((G, H // G, m, D), dtype=torch.float32, device=q.device)
    q = q.float().view(m, G, H // G, D).permute(1, 2, 0, 3).contiguous()
    k, v = k.float().permute(1, 2, 0).contiguous(), v.float().transpose(0, 1).contiguous()
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
        if c["call"] == "prompt":
            k, v = s["k"][lo:hi], s["v"][lo:hi]
        else:
            pages = s["table"][b, :_blocks(c, n + m)].long()
            k, v = (x[pages].reshape(-1, c["kv_heads"], c["head_dim"])[:n + m] for x in s["cache"])
        out[lo:hi] = _plain_rows(s["q"][lo:hi], k, v, n, s["scale"], c["window"]).to(out.dtype)
    return out


def run(state):
    s = state
    if not own:
        return {"pages": _plain_pages, "write": _plain_write, "attend": _plain_attend, "prompt": _plain_attend}[s["call"]](s)
    import paper_2511_13732_amd as pcg
    if s["call"] == "pages":
        o = pcg.pages_step(s["pages"], s["add"], commit=s["commit"], commit_extra=1, max_tokens=s["max_tokens"],
                           state_out=s["next"], out=s["out"])
        return [s["next"], s["table"], s["free"], o.q_start, o.slots, o.positions, o.refused]
    if s["call"] == "write":
        pcg.cache_write(s["kv"], s["k"], s["v"], s["slots"])
        return s["cache"]
    if s["call"] == "prompt":
        return pcg.prompt_attend(s["q"], s["k"], s["v"], s["q_start"], longest=s["longest"], scale=s["scale"],
                                 window=s["case"]["window"], out=s["out"])
    return pcg.cache_attend(s["kv"], s["q"], s["table"], s["lens"], s["q_start"], longest=s["longest"], scale=s["scale"],
                            window=s["case"]["window"], out=s["out"], workspace=s["workspace"])


# ------------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    """The attention calls from the definition, in double, the caches with their new rows; page tables are whole numbers."""
    c = case
    if c["call"] == "pages" or work(c)["flops"] > 4e12:
        return None
    s = prepare(c, seed)
    if c["call"] == "write":
        both = [x.double() for x in s["cache"]]
        row = torch.nonzero(s["slots"] >= 0)[:, 0]
        for x, new in zip(both, (s["k"], s["v"])):
            x[s["slots"][row].long() // c["page_size"], s["slots"][row].long() % c["page_size"]] = new[row].double()
        return both
    H, G, D = c["heads"], c["kv_heads"], c["head_dim"]
    out = torch.zeros((s["q"].shape[0], H, D), dtype=torch.float64, device="cuda")
    for b, (n, m) in enumerate(s["pairs"]):
        rows = s["q_start"][b].item()
        if c["call"] == "prompt":
            keys, values = s["k"][rows:rows + m].double(), s["v"][rows:rows + m].double()
        else:
            pos = torch.arange(n + m, device="cuda")
            page, slot = s["table"][b].long()[pos // c["page_size"]], pos % c["page_size"]
            keys, values = s["cache"][0][page, slot].double(), s["cache"][1][page, slot].double()
        for lo in range(0, m, 512):
            hi = min(m, lo + 512)
            last = n + torch.arange(lo, hi, device="cuda")
            begin = max(0, n + lo - c["window"] + 1) if c["window"] else 0
            j = torch.arange(begin, n + hi, device="cuda")
            sees = j[None] <= last[:, None]
            if c["window"]:
                sees &= j[None] > last[:, None] - c["window"]
            for h in range(H):
                x = s["q"][rows + lo:rows + hi, h].double() @ keys[begin:n + hi, h // (H // G)].T
                weight = torch.softmax(torch.where(sees, x * s["scale"], -math.inf), dim=1)
                out[rows + lo:rows + hi, h] = weight @ values[begin:n + hi, h // (H // G)]
    return out
