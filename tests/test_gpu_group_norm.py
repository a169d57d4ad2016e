"""dp_group_norm and dp_group_norm_daq against their definition in 64 bits."""
import pytest
import torch

import attention_ref as R
from paper_2511_11446_b200 import binding as B

pytestmark = pytest.mark.gpu
EPS = 1e-5
SHAPES = [(2, 64, 1280, 32), (1, 1, 8, 1), (3, 1, 64, 8), (1, 7, 64, 32), (2, 255, 320, 32), (1, 1023, 640, 32), (5, 100, 72, 9),
          (1, 33, 2560, 32), (2, 17, 4608, 36), (1, 2049, 384, 2), (9, 37, 960, 30), (40, 16, 128, 128), (1, 300, 1024, 1024),
          (300, 3, 64, 4), (1, 20000, 24, 3), (1, 129, 2304, 16), (2, 1000, 1152, 32)]


def _inputs(n, rows, C, seed, level=1.0, ldx=None):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    ldx = ldx or C
    x = torch.full((n * rows, ldx), float("nan"), dtype=torch.bfloat16, device="cuda")
    x[:, :C] = (torch.randn(n * rows, C, generator=gen, device="cuda") +
                level * torch.randn(C, generator=gen, device="cuda")).to(torch.bfloat16)
    gamma = (1 + 0.3 * torch.randn(C, generator=gen, device="cuda")).to(torch.bfloat16)
    beta = (0.3 * torch.randn(C, generator=gen, device="cuda")).to(torch.bfloat16)
    return x, gamma, beta


def _ws(n, rows, C, G):
    return torch.full((B.dp_group_norm_workspace(n, rows, C, G),), 0xFF, dtype=torch.uint8, device="cuda")  # (NaN as floats)


def _check_y(y, x, C, n, rows, G, gamma, beta, act):
    want, tol = R.group_norm(x[:, :C], n, rows, G, gamma, beta, EPS, act == B.DP_ACT_SILU)
    off = (y[:, :C].double() - want).abs() - (tol + R.BF16 * (want.abs() + tol))
    assert (off <= 0).all(), (float(off.max()), (off > 0).nonzero()[:4].tolist())


def _check_codes(q, s_a, x, C, n, rows, G, gamma, beta, act):
    want, tol = R.group_norm(x[:, :C], n, rows, G, gamma, beta, EPS, act == B.DP_ACT_SILU)
    amax, at = want.abs().amax(1), tol.amax(1)
    s = s_a.double().view(-1)
    live = amax > 1e-25
    assert ((s - amax / 127).abs() <= at / 127 + 2.0 ** -23 * amax / 127)[live].all()
    assert (s[~live] == 0).all() and not q[:, :C][~live].any()
    # the code of a value that is off by tol, its scale by at / 127: at most half a step and that much from the real quotient
    real = want[live] / (amax[live] / 127).view(-1, 1)
    slack = 0.5 + (tol[live] + real.abs() / 127 * at[live].view(-1, 1)) / (amax[live] / 127).view(-1, 1) * 1.01 + 127 * 2.0 ** -22
    assert ((q[:, :C][live].double() - real).abs() <= slack).all()
    assert int(q.abs().max()) <= 127


@pytest.mark.parametrize("affine", [True, False])
@pytest.mark.parametrize("act", [B.DP_ACT_NONE, B.DP_ACT_SILU])
@pytest.mark.parametrize("n,rows,C,G", SHAPES)
def test_bf16(n, rows, C, G, act, affine):
    x, gamma, beta = _inputs(n, rows, C, C + rows)
    if not affine:
        gamma = beta = None
    y = torch.zeros(n * rows, C, dtype=torch.bfloat16, device="cuda")
    B.dp_group_norm(x, n, rows, C, C, G, gamma, beta, EPS, act, y, C, _ws(n, rows, C, G))
    _check_y(y, x, C, n, rows, G, gamma, beta, act)


@pytest.mark.parametrize("act", [B.DP_ACT_NONE, B.DP_ACT_SILU])
@pytest.mark.parametrize("n,rows,C,G", [s for s in SHAPES if s[2] % 16 == 0])
def test_codes(n, rows, C, G, act):
    x, gamma, beta = _inputs(n, rows, C, C + rows + 1)
    q = torch.full((n * rows, C), 99, dtype=torch.int8, device="cuda")
    s_a = torch.full((n * rows,), -1.0, device="cuda")
    B.dp_group_norm_daq(x, n, rows, C, C, G, gamma, beta, EPS, act, q, C, s_a, _ws(n, rows, C, G))
    _check_codes(q, s_a, x, C, n, rows, G, gamma, beta, act)


@pytest.mark.parametrize("n,rows,C,G", [(3, 1301, 320, 32), (200, 600, 192, 8), (1, 5000, 1280, 32), (3, 700, 1296, 9), (2, 601, 1920, 32)])
def test_codes_of_maps_beyond_shared_memory(n, rows, C, G):
    """The second kernel's CTAs are cut unlike the first's up to 1280 channels, and like them beyond."""
    test_codes(n, rows, C, G, B.DP_ACT_SILU)


@pytest.mark.parametrize("n,rows,C,G", [(2, 70, 320, 32), (1, 2000, 64, 4), (2, 9, 2560, 32)])
def test_pitches(n, rows, C, G):
    x, gamma, beta = _inputs(n, rows, C, 3, ldx=C + 40)
    y = torch.full((n * rows, C + 8), 5.0, dtype=torch.bfloat16, device="cuda")
    B.dp_group_norm(x, n, rows, C, C + 40, G, gamma, beta, EPS, B.DP_ACT_SILU, y, C + 8, _ws(n, rows, C, G))
    _check_y(y, x, C, n, rows, G, gamma, beta, B.DP_ACT_SILU)
    assert (y[:, C:] == 5.0).all()
    q = torch.full((n * rows, C + 16), 99, dtype=torch.int8, device="cuda")
    s_a = torch.empty(n * rows, device="cuda")
    B.dp_group_norm_daq(x, n, rows, C, C + 40, G, gamma, beta, EPS, B.DP_ACT_NONE, q, C + 16, s_a, _ws(n, rows, C, G))
    _check_codes(q[:, :C], s_a, x, C, n, rows, G, gamma, beta, B.DP_ACT_NONE)
    assert (q[:, C:] == 99).all()


@pytest.mark.parametrize("rows", [1, 300, 5000])
def test_constant_maps_and_levels_far_above_the_spread(rows):
    """A constant group has variance 0 and gives beta; a level of 200 with steps of 1 keeps its digits."""
    n, C, G = 2, 320, 32
    x, gamma, beta = _inputs(n, rows, C, 9)
    x[:, :100] = 1000.0
    x[:, 100:200] = 200.0 + torch.randint(0, 2, (n * rows, 100), device="cuda").to(torch.bfloat16)
    y = torch.zeros(n * rows, C, dtype=torch.bfloat16, device="cuda")
    B.dp_group_norm(x, n, rows, C, C, G, gamma, beta, EPS, B.DP_ACT_NONE, y, C, _ws(n, rows, C, G))
    assert torch.equal(y[:, :100], beta[:100].expand(n * rows, 100))
    _check_y(y, x, C, n, rows, G, gamma, beta, B.DP_ACT_NONE)
    x.zero_()
    q = torch.full((n * rows, C), 99, dtype=torch.int8, device="cuda")
    s_a = torch.full((n * rows,), -1.0, device="cuda")
    B.dp_group_norm_daq(x, n, rows, C, C, G, None, None, EPS, B.DP_ACT_SILU, q, C, s_a, _ws(n, rows, C, G))
    assert not q.any() and not s_a.any()


def test_large_map_in_parts():
    """A batch beyond the L2, and one sample of many rows."""
    for n, rows, C, G in ((20, 16384, 320, 32), (1, 300_001, 64, 32)):
        x, gamma, beta = _inputs(n, rows, C, 11)
        y = torch.zeros(n * rows, C, dtype=torch.bfloat16, device="cuda")
        B.dp_group_norm(x, n, rows, C, C, G, gamma, beta, EPS, B.DP_ACT_SILU, y, C, _ws(n, rows, C, G))
        for b in {0, n // 2, n - 1}:  # (a sample at a time: 64 bits of all of them take memory)
            at = slice(b * rows, (b + 1) * rows)
            _check_y(y[at], x[at], C, 1, rows, G, gamma, beta, B.DP_ACT_SILU)


def test_same_bits_on_streams_and_in_graphs():
    n, rows, C, G = 3, 500, 640, 32
    x, gamma, beta = _inputs(n, rows, C, 12)
    ys = [torch.zeros(n * rows, C, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    ws = [_ws(n, rows, C, G) for _ in range(3)]
    call = lambda i: B.dp_group_norm(x, n, rows, C, C, G, gamma, beta, EPS, B.DP_ACT_SILU, ys[i], C, ws[i])  # noqa: E731
    call(0)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        call(1)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(2)
    for _ in range(3):
        ys[2].zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(ys[0], ys[2])
    assert torch.equal(ys[0], ys[1])
    for _ in range(5):  # one workspace, call behind call
        call(0)
    torch.cuda.synchronize()
    assert torch.equal(ys[0], ys[2])
