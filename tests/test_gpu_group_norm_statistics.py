"""Group normalisation's statistics where they are easily lost: infinities and NaN."""
import math

import pytest
import torch

from paper_2511_11446_b200 import binding as B

pytestmark = pytest.mark.gpu
EPS = 1e-5


def _ws(n, rows, C, G):
    return torch.full((B.dp_group_norm_workspace(n, rows, C, G),), 0xFF, dtype=torch.uint8, device="cuda")


def _affine(C, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return ((1 + 0.3 * torch.randn(C, generator=gen, device="cuda")).to(torch.bfloat16),
            (0.3 * torch.randn(C, generator=gen, device="cuda")).to(torch.bfloat16), gen)


@pytest.mark.parametrize("act", [B.DP_ACT_NONE, B.DP_ACT_SILU])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("n,rows,C,G", [(2, 64, 1280, 32), (3, 2000, 320, 32)])
def test_groups_with_infinities_are_not_numbers(n, rows, C, G, value, act):
    """The variance of a group that holds an infinity or a NaN is not a number, nor is any of its outputs; other groups and samples
    keep their bits."""
    gamma, beta, gen = _affine(C, 3)
    x = torch.randn(n * rows, C, generator=gen, device="cuda").to(torch.bfloat16)
    per = C // G
    y0, y1 = (torch.zeros(n * rows, C, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    call = lambda x, y: B.dp_group_norm(x, n, rows, C, C, G, gamma, beta, EPS, act, y, C, _ws(n, rows, C, G))  # noqa: E731
    call(x, y0)
    for row, ch in ((rows - 1, per + 1), (0, 0), (rows, 5 * per), (rows + rows // 2, 7 * per - 1)):
        bad = x.clone()
        bad[row, ch] = value
        call(bad, y1)
        hit = torch.zeros(n, rows, G, per, dtype=torch.bool, device="cuda")
        hit[row // rows, :, ch // per] = True
        hit = hit.view(n * rows, C)
        assert y1[hit].isnan().all()
        assert torch.equal(y1[~hit].view(torch.int16), y0[~hit].view(torch.int16))
        q = torch.zeros(n * rows, C, dtype=torch.int8, device="cuda")
        s_a = torch.zeros(n, rows, device="cuda")
        B.dp_group_norm_daq(bad, n, rows, C, C, G, gamma, beta, EPS, act, q, C, s_a, _ws(n, rows, C, G))
        ok = torch.ones(n, dtype=torch.bool)
        ok[row // rows] = False
        assert s_a[row // rows].isnan().all() and s_a[ok.cuda()].isfinite().all()
