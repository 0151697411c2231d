"""Attention over 4 bits where weights times values' scales are so small that bfloat16 has fewer than eight bits of them, or none of a part of
them: what is multiplied are multiples of 2^-133, the step of the smallest bfloat16.  Run with ``-m gpu`` on an MI355X."""
import pytest
import torch

import attention
import paper_2511_13732_amd as pcg
from test_gpu_attend4 import DTYPES, gen, make_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("exponent", [-100, -112, -118, -124, -129])
def test_values_near_the_smallest_numbers(dtype, exponent):
    """A weight times a scale is cut off (float32 rows) or rounded (bfloat16) to a multiple of 2^-133, which is off by a step at most and meets
    a code of 6 at most; weights are those by the row's largest score or larger, and so is their sum.  The sum of products is rounded to float32, and the
    output to its type, whose steps are no finer than the smallest numbers'."""
    dt, H, G, D, n = DTYPES[dtype], 4, 2, 64, 150
    cache, table, rows = make_cache([n], 16, G, D, "heads", seed=5)
    (k, v), = rows
    at = torch.arange(n)
    page, slot = table[0].cpu().long()[at // 16], at % 16
    scales = cache.scales.cpu()
    was = scales[page, slot, :, 1].double()
    small = (2.0 ** exponent * (1 + torch.rand((n, G), generator=gen(1)))).to(torch.bfloat16)
    scales[page, slot, :, 1] = small
    cache.scales.copy_(scales)
    v = v / was[..., None] * small.double()[..., None]                  # codes times the new scales
    q = torch.randn((1, H, D), generator=gen(2)).to(dt).cuda()
    out = pcg.cache4_attend(cache, q, table, torch.tensor([n - 1], dtype=torch.int32).cuda(), torch.tensor([0, 1], dtype=torch.int32).cuda())
    # the definition with scales of ordinary size: it is 2^exponent times this
    want, mag, err = (x * 2.0 ** exponent for x in attention.attend_rows(q.cpu(), k, v * 2.0 ** -exponent, n - 1, D ** -0.5))
    score = torch.einsum("hd,nhd->hn", q[0].double().cpu(), k.repeat_interleave(H // G, dim=1)) * D ** -0.5
    total = torch.exp(score - score.amax(dim=1, keepdim=True)).sum(dim=1)[:, None]
    half = torch.finfo(dt).eps / 2
    tol = err * 3 if dtype == "f32" else err + half * mag
    tol = tol + 6 * n * 2.0 ** -133 * (1 + err / mag) / total + 6 * n * 2.0 ** -149     # weights times scales; scalings of sums
    tol = tol + half * (want.abs() + tol) + (2.0 ** -134 if dtype == "bf16" else 2.0 ** -150)
    off = (out.double().cpu() - want).abs()
    assert (off <= tol).all(), (float(off.max()), float(tol.max()))
