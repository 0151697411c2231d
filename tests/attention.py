"""Attention and page bookkeeping from their definitions, in double and in plain Python, for the tests of the calls
around a step's forward pass."""
import math

import torch


def attend_rows(q, k, v, first, scale, window=0):
    """Rows q [m, H, D] at positions first, first + 1, .. over keys and values [n, G, D] of positions 0 .. n - 1: the outputs in
    double and, for each, how far a computation in float32 may be from them (see ``allowed``).

    With u = 2^-23 (a rounding of an fp32 operation, truncating or not): a score is a sum of D products, off by at most
    (D + 4) u scale sum |q_i k_i| with its scaling, the argument of the exponential by another u of its size, and the exponential by a
    few u; a weight is therefore off by e = 2 (D + 8) u M + 8 u relative to the others at most, M the row's largest scale sum |q_i k_i|
    (at least 1).  Sums over n keys in any order add n u.  Numerator and denominator: twice that, times sum w_j |v_j|.  The numerator and
    denominator of parts that are joined carry a few roundings more, inside the 64 u."""
    m, H, D = q.shape
    n, G, _ = k.shape
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    out = torch.zeros((m, H, D), dtype=torch.float64)
    mag = torch.zeros((m, H, D), dtype=torch.float64)
    err = torch.zeros((m, H, D), dtype=torch.float64)
    u = 2.0 ** -23
    for t in range(m):
        p = first + t
        lo = max(0, p - window + 1) if window else 0
        hi = min(p + 1, n)
        if hi <= lo:
            continue
        for g in range(G):
            hs = slice(g * (H // G), (g + 1) * (H // G))
            s = scale * (q[t, hs] @ k[lo:hi, g].T)
            top = s.amax(dim=1, keepdim=True)
            w = torch.where(torch.isneginf(top), 0.0, torch.exp(s - top))
            total = w.sum(dim=1, keepdim=True)
            w = torch.where(total == 0, 0.0, w / total)
            out[t, hs] = w @ v[lo:hi, g]
            mag[t, hs] = w @ v[lo:hi, g].abs()
            M = (scale * (q[t, hs].abs() @ k[lo:hi, g].abs().T)).amax(dim=1, keepdim=True).clamp(min=1.0)
            err[t, hs] = 2 * (2 * (D + 8) * u * M + (hi - lo + 64) * u) * mag[t, hs]
    return out, mag, err


def allowed(out, mag, err, dtype):
    """With bfloat16 every weight is rounded once (half a step: 2^-8 of it) and the output once."""
    if dtype == torch.bfloat16:
        half = torch.finfo(dtype).eps / 2
        return err + half * mag + half * (out.abs() + err + half * mag) + 1e-30
    return err + torch.finfo(dtype).eps / 2 * out.abs() + 1e-30


def check(got, ref, dtype, what=""):
    out, mag, err = ref
    got = got.double().cpu()
    off = (got - out).abs()
    tol = allowed(out, mag, err, dtype)
    bad = ~(off <= tol) & ~(torch.isnan(got) & torch.isnan(out)) & ~(got == out)
    assert not bad.any(), (what, int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist(), float(got[bad][0]), float(out[bad][0]),
                           float(tol[bad][0]))


def pages_step(table, free, state, page_size, commit, extra, add, max_tokens):
    """The bookkeeping of one step in plain Python, on lists; returns (state, table, free, q_start, slots, positions, refused)."""
    B, room = len(table), len(table[0])
    lens, held, chunk, count = state[:B], state[B:2 * B], state[2 * B:3 * B], state[3 * B]
    table, free = [list(r) for r in table], list(free)
    want, need, out = [0] * B, [0] * B, [False] * B
    lens = [0 if add[b] < 0 else lens[b] + (chunk[b] if commit is None else min(max(commit[b] + extra, 0), chunk[b]))
            for b in range(B)]
    running = 0
    for b in range(B):
        want[b] = max(add[b], 0)
        need[b] = math.ceil((lens[b] + want[b]) / page_size)
        if need[b] > room:
            out[b] = True
            continue
        running += want[b]
        out[b] = want[b] > 0 and running > max_tokens
    for b in range(B):
        if not out[b]:
            for j in range(need[b], held[b]):
                free[count] = table[b][j]
                count += 1
    top, running, taken = count, 0, 0
    for b in range(B):
        if not out[b] and need[b] > held[b]:
            running += need[b] - held[b]
            if running > top:
                out[b] = True
                continue
            for j in range(held[b], need[b]):
                taken += 1
                table[b][j] = free[top - taken]
    got = [0 if out[b] else want[b] for b in range(B)]
    q_start = [0]
    slots, positions = [], []
    for b in range(B):
        q_start.append(q_start[-1] + got[b])
        for j in range(got[b]):
            p = lens[b] + j
            positions.append(p)
            slots.append(table[b][p // page_size] * page_size + p % page_size)
    slots += [-1] * (max_tokens - len(slots))
    positions += [0] * (max_tokens - len(positions))
    state = lens + [held[b] if out[b] else need[b] for b in range(B)] + got + [top - taken]
    return state, table, free, q_start, slots, positions, sum(out[b] and add[b] > 0 for b in range(B))
