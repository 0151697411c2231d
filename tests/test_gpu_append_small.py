"""Codes and scales of the smallest numbers (pcg_cache4_append), whose scales have no full eight bits: against whole-number arithmetic on
multiples of 2^-149, the step of the smallest float32.  Run with ``-m gpu`` on an MI355X."""
import random

import pytest
import torch

import paper_2511_13732_amd as pcg
from cache4 import unpacked

HALVES = (0, 1, 2, 3, 4, 6, 8, 12)             # the levels, in halves
STEP = 1 << 16                                 # of a scale below 2^-125, in steps of float32


def scale_of(m):
    """The nearest multiple of STEP to m / 6, ties to the even one, for m / 6 < 2^24; in units of STEP."""
    n, rest = divmod(m, 6 * STEP)
    return n + (2 * rest > 6 * STEP or (2 * rest == 6 * STEP and n % 2))


def code_of(x, unit):
    """The nearest level to |x| / (unit STEP), ties to the even code."""
    off = [abs(2 * abs(x) - h * unit * STEP) for h in HALVES]
    best = [c for c in range(8) if off[c] == min(off)]
    return 0 if unit == 0 else min(best, key=lambda c: c % 2) + (8 if x < 0 else 0)


def float_of(m):
    """m 2^-149, exact, as float32."""
    x = torch.tensor(float(m) * 2.0 ** -149, dtype=torch.float64)
    assert x.float().double() == x
    return float(x)


def maxima():
    """Six times what lies in the middle of two scales, and numbers beside it, across the subnormal scales and the first normal ones."""
    out = []
    for k in list(range(0, 40)) + [63, 64, 100, 126, 127, 128, 129, 191, 200, 254]:
        middle = 6 * (STEP // 2) * (2 * k + 1)
        step = 1 << max(0, middle.bit_length() - 24)
        out += [middle + d * step for d in (-2, -1, 0, 1, 2) if (middle + d * step).bit_length() <= 24 or (middle + d * step) % step == 0]
    return out + [1, 2, 3, 5, 6, 7, STEP - 1, STEP, 3 * STEP - 1, 3 * STEP, 3 * STEP + 1, 6 * STEP, (1 << 23) - 1, 1 << 23, (1 << 23) + 1]


def test_the_whole_number_arithmetic_by_hand():
    assert [scale_of(m) for m in (0, 3 * STEP - 1, 3 * STEP, 3 * STEP + 1, 6 * STEP, 9 * STEP - 1, 9 * STEP, 9 * STEP + 1)] == [0, 0, 0, 1, 1, 1, 2, 2]
    assert scale_of(589823) == 1 and scale_of(196609) == 1 and scale_of(983041) == 3
    # a quarter and three quarters of a scale of 4 steps, 5 of it, a step beside them, and more than six of it
    assert [code_of(x * STEP, 4) for x in (1, 3, -3, 20, 30)] == [0, 2, 10, 6, 7] and code_of(STEP + 1, 4) == 1 and code_of(20 * STEP + 1, 4) == 7
    assert len(maxima()) > 200


@pytest.mark.gpu
def test_scales_below_the_normal_numbers():
    g, D, rows = random.Random(5), 32, []
    for m in maxima():
        unit = scale_of(m)
        step = 1 << max(0, m.bit_length() - 24)
        # borders of codes of that scale and numbers beside them, where they are not above the maximum
        some = [h * unit * STEP // 4 + d for h in (1, 3, 5, 7, 10, 14, 20) for d in (-step, 0, step)] + [g.randrange(m + 1) for _ in range(9)]
        row = [m] + [x // step * step for x in some if 0 <= x <= m]
        rows.append([x if g.random() < 0.5 else -x for x in row] + [0] * (D - len(row)))
    x = torch.tensor([[float_of(v) for v in row] for row in rows])[:, None]
    T = x.shape[0]
    c, slots = pcg.KvCache4.empty(T, 1, 1, D, "cuda"), torch.arange(T, dtype=torch.int32).cuda()
    pcg.cache4_append(c, x.cuda(), -x.cuda(), slots)
    scales = torch.tensor([scale_of(abs(row[0])) * 2.0 ** -133 for row in rows], dtype=torch.float64)
    for i, (bits, sign) in enumerate(((c.k, 1), (c.v, -1))):
        assert torch.equal(c.scales[:, 0, 0, i].double().cpu(), scales)
        mine = unpacked(bits[:, 0, 0].cpu(), D)
        want = torch.tensor([[code_of(sign * v, scale_of(abs(row[0]))) for v in row] for row in rows], dtype=torch.uint8)
        # a zero may have either sign
        assert torch.equal(torch.where(want % 8 == 0, mine & 7, mine), torch.where(want % 8 == 0, 0, want))
    level = torch.tensor([h / 2 for h in HALVES] + [-h / 2 for h in HALVES], dtype=torch.float64)
    back = pcg.cache4_read(c, slots, dtype=torch.float32)[0][:, 0].double().cpu()
    assert torch.equal(back, level[unpacked(c.k[:, 0, 0].cpu(), D).long()] * scales[:, None])
