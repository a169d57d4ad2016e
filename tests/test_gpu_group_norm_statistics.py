"""Group normalisation's statistics where they are easily lost: an untypical first value, levels far above the spread, maps whose
parts are unlike each other, infinities and NaN; outputs beside the inputs, offsets beyond 32 bits."""
import math

import pytest
import torch

from paper_2511_11446_b200 import binding as B

pytestmark = pytest.mark.gpu
EPS = 1e-5
U = 2.0 ** -24  # half a step of an fp32 value, relative to it


def _ws(n, rows, C, G):
    return torch.full((B.dp_group_norm_workspace(n, rows, C, G),), 0xFF, dtype=torch.uint8, device="cuda")


def _want(x, n, rows, C, G, gamma, beta, silu):
    """One sample of n, [rows, C], in 64 bits: act(h) and the bound of its error before the output's rounding.

    Runs of F = 24 rows of a channel are summed about one of their own values, p. With q = sum (x - p)^2 <= (F + 1) M2 (p is one of
    the values, so (p - mean)^2 <= M2), a run's M2 is off by (3 F + 12) U q at most and its mean by (F + 3) U sqrt(q / F), 5 (F + 3) U
    standard deviations. Each of a thread's K runs rounds the mean once more. Then L lanes are joined in blocks of 16, P channels (up
    to 48, else about their mean) and T parts of the rows, each about the first of them, whose weight is 1 / k of the whole, k = 16, P, T:
    that costs M2 k times the roundings of a chain of c, (c + 4) U, c = 16, P, T / 8 + 4; and the mean c sqrt(k) U standard
    deviations. Means are held about the group's first value p0: 8 roundings of |mean - p0|. So, in units of the standard deviation,
      e = U (5 (F + 3 + K) + L^1.5 + P^1.5 + T^1.5 + 8 m + 16),   m = |mean - p0| / std,
    is the mean off by, v = U ((3 F + 12) (F + 1) + 16 (16 + 4) + P' (P' + 4) + T (T / 8 + 8)) + 2 e the variance of itself, P' = min(P, 48), and
    h = gamma z + beta by |gamma| (e + |z| v / 2 + 4 U |z|) + 2 U |beta| and what rounding the mean to fp32 costs, 2 U |mean| / std. The
    activation multiplies that by 1.1 at most and adds 2^-21 (2 + |h|) of its value."""
    d = x.double().view(rows, G, C // G)
    var, mean = torch.var_mean(d, dim=(0, 2), correction=0, keepdim=True)
    std = torch.sqrt(var + EPS)
    z = ((d - mean) / std).reshape(rows, C)
    F, L, P, T = 24, max(1, 640 // (C // 8)), C // G, max(8, min(148 // n, rows // 16 + 1))
    K, P1 = rows // (T * L * F) + 1, min(P, 48)
    spread = lambda t: t.expand_as(d).reshape(rows, C)  # noqa: E731
    m = spread((mean - d[:1, :, :1]).abs() / std)
    e = U * (5 * (F + 3 + K) + L ** 1.5 + P ** 1.5 + T ** 1.5 + 8 * m + 16)
    v = U * ((3 * F + 12) * (F + 1) + 16 * 20 + P1 * (P1 + 4) + T * (T / 8 + 8)) + 2 * e
    g, b = gamma.double(), beta.double()
    h = z * g + b
    tol = g.abs() * (e + z.abs() * v / 2 + 4 * U * z.abs() + 2 * U * spread(mean.abs() / std)) + 2 * U * b.abs()
    if silu:
        y = h * torch.sigmoid(h)
        return y, 1.1 * tol + 2.0 ** -21 * (2 + h.abs()) * y.abs()
    return h, tol


def _affine(C, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return ((1 + 0.3 * torch.randn(C, generator=gen, device="cuda")).to(torch.bfloat16),
            (0.3 * torch.randn(C, generator=gen, device="cuda")).to(torch.bfloat16), gen)


def _check(x, n, rows, C, G, gamma, beta, act, samples):
    y = torch.zeros(n * rows, C, dtype=torch.bfloat16, device="cuda")
    B.dp_group_norm(x, n, rows, C, C, G, gamma, beta, EPS, act, y, C, _ws(n, rows, C, G))
    for s in samples:
        at = slice(s * rows, (s + 1) * rows)
        want, tol = _want(x[at], n, rows, C, G, gamma, beta, act == B.DP_ACT_SILU)
        off = (y[at].double() - want).abs() - (tol + 2.0 ** -8 * (want.abs() + tol))
        assert (off <= 0).all(), (s, float(off.max()), int((off > 0).sum()))


SHAPES = [(2, 64, 1280, 32), (1, 2000, 64, 8), (8, 1023, 640, 32), (16, 16384, 320, 32), (150, 8192, 320, 32), (1, 300_001, 64, 32)]


@pytest.mark.parametrize("act", [B.DP_ACT_NONE, B.DP_ACT_SILU])
@pytest.mark.parametrize("level,spread,first", [(100.0, 0.5, 0.0), (0.0, 1.0, 1000.0), (0.0, 1.0, -100.0)])
@pytest.mark.parametrize("n,rows,C,G", SHAPES)
def test_untypical_first_values(n, rows, C, G, level, spread, first, act):
    """A sample's first row is far from all others (a padded corner, an outlier)."""
    gamma, beta, gen = _affine(C, rows)
    x = torch.empty(n * rows, C, dtype=torch.bfloat16, device="cuda")
    for s in range(n):
        x[s * rows:(s + 1) * rows] = level + spread * torch.randn(rows, C, generator=gen, device="cuda")
    x[::rows] = first
    _check(x, n, rows, C, G, gamma, beta, act, {0, n // 2, n - 1})


@pytest.mark.parametrize("n,rows,C,G", SHAPES)
def test_maps_whose_parts_are_unlike(n, rows, C, G):
    """Level and spread change along the rows: leaving out or taking twice a part of them moves mean and variance."""
    gamma, beta, gen = _affine(C, rows + 1)
    t = torch.linspace(0, 1, rows, device="cuda").view(rows, 1)
    x = torch.empty(n * rows, C, dtype=torch.bfloat16, device="cuda")
    for s in range(n):
        x[s * rows:(s + 1) * rows] = 10 * t * t - 3 + (0.3 + 4 * t) * torch.randn(rows, C, generator=gen, device="cuda")
    _check(x, n, rows, C, G, gamma, beta, B.DP_ACT_NONE, {0, n // 2, n - 1})


@pytest.mark.parametrize("every", [1, 7])
def test_outliers_in_many_rows(every):
    """Every few rows a channel is far out, the rows that threads begin with among them."""
    n, rows, C, G = 4, 8000, 320, 32
    gamma, beta, gen = _affine(C, every)
    x = torch.randn(n * rows, C, generator=gen, device="cuda")
    x[::every, ::5] += 300.0
    _check(x.to(torch.bfloat16), n, rows, C, G, gamma, beta, B.DP_ACT_SILU, range(n))


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


def test_silu_far_below_zero():
    """h / (1 + e^-h) to its last bits down to h = -43, and to |h| 2^-62 below."""
    rows, C, G = 64, 64, 1
    x = torch.zeros(rows, C, device="cuda")
    x[:, :32], x[:, 32:] = -1.0, 1.0  # mean 0, variance 1
    x = x.to(torch.bfloat16)
    beta = torch.zeros(C, device="cuda")
    beta[:32] = torch.linspace(-1, -88, 32, device="cuda")
    beta[32::2] = torch.linspace(-40, -80, 16, device="cuda")  # pairs of a small and a large one
    gamma, beta = torch.ones(C, dtype=torch.bfloat16, device="cuda"), beta.to(torch.bfloat16)
    y = torch.zeros(rows, C, dtype=torch.bfloat16, device="cuda")
    B.dp_group_norm(x, 1, rows, C, C, G, gamma, beta, 0.0, B.DP_ACT_SILU, y, C, _ws(1, rows, C, G))
    h = x.double() + beta.double()
    want = h * torch.sigmoid(h)
    # h is off by 2^-20 at most (its size below 128, four roundings); then as for any other value
    tol = want.abs() * (2.0 ** -8 + 2.0 ** -20 + 2.0 ** -21 * (2 + h.abs())) + torch.where(h < -42.9, h.abs() * 2.0 ** -62, 0.0)
    assert ((y.double() - want).abs() <= tol).all(), ((y.double() - want).abs() - tol).max()


def test_outputs_beside_the_inputs():
    """y, or codes, in columns of x's own rows: nothing overlaps."""
    n, rows, C, G = 2, 300, 320, 32
    gamma, beta, gen = _affine(C, 4)
    buf = torch.randn(n * rows, 2 * C, generator=gen, device="cuda").to(torch.bfloat16)
    x0 = buf[:, :C].clone()
    y = torch.zeros(n * rows, C, dtype=torch.bfloat16, device="cuda")
    B.dp_group_norm(x0, n, rows, C, C, G, gamma, beta, EPS, B.DP_ACT_SILU, y, C, _ws(n, rows, C, G))
    q, s0, s1 = torch.zeros(n * rows, C, dtype=torch.int8, device="cuda"), *(torch.zeros(n * rows, device="cuda") for _ in range(2))
    B.dp_group_norm_daq(x0, n, rows, C, C, G, gamma, beta, EPS, B.DP_ACT_SILU, q, C, s0, _ws(n, rows, C, G))
    B.dp_group_norm(buf, n, rows, C, 2 * C, G, gamma, beta, EPS, B.DP_ACT_SILU, buf[:, C:], 2 * C, _ws(n, rows, C, G))
    assert torch.equal(buf[:, C:], y) and torch.equal(buf[:, :C], x0)
    codes = buf.view(torch.int8)  # rows of 4 C bytes, x in the first 2 C
    B.dp_group_norm_daq(buf, n, rows, C, 2 * C, G, gamma, beta, EPS, B.DP_ACT_SILU, codes[:, 2 * C:], 4 * C, s1, _ws(n, rows, C, G))
    assert torch.equal(codes[:, 2 * C:3 * C], q) and torch.equal(s0, s1) and torch.equal(buf[:, :C], x0)


def test_every_operand_beyond_32_bit_offsets():
    """Rows 2^20 elements apart: the last of x, y and the codes lie behind element 2^32."""
    n, rows, C, G, ld = 3, 1400, 64, 8, 1 << 20
    M = n * rows
    assert (M - 1) * ld > 1 << 32
    gamma, beta, gen = _affine(C, 5)
    x0 = torch.randn(M, C, generator=gen, device="cuda").to(torch.bfloat16)
    y0 = torch.zeros(M, C, dtype=torch.bfloat16, device="cuda")
    q0, s0, s1 = torch.zeros(M, C, dtype=torch.int8, device="cuda"), *(torch.zeros(M, device="cuda") for _ in range(2))
    B.dp_group_norm(x0, n, rows, C, C, G, gamma, beta, EPS, B.DP_ACT_SILU, y0, C, _ws(n, rows, C, G))
    B.dp_group_norm_daq(x0, n, rows, C, C, G, gamma, beta, EPS, B.DP_ACT_SILU, q0, C, s0, _ws(n, rows, C, G))
    x, y = (torch.empty(M, ld, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    x[:, :C] = x0
    B.dp_group_norm(x, n, rows, C, ld, G, gamma, beta, EPS, B.DP_ACT_SILU, y, ld, _ws(n, rows, C, G))
    assert torch.equal(y[:, :C], y0)
    q = y.view(torch.int8)[:, :ld]  # (rows 2 ld bytes apart)
    B.dp_group_norm_daq(x, n, rows, C, ld, G, gamma, beta, EPS, B.DP_ACT_SILU, q, 2 * ld, s1, _ws(n, rows, C, G))
    assert torch.equal(q[:, :C], q0) and torch.equal(s0, s1)


@pytest.mark.parametrize("size", [1.0, 1e12, 1e-8])
@pytest.mark.parametrize("n,rows,C,G", [(1, 5000, 8, 1), (2, 3000, 24, 3), (1, 900, 1024, 1024), (3, 700, 4608, 4), (2, 1, 64, 4), (1, 13, 64, 8),
                                        (400, 40, 72, 9), (7, 401, 2304, 1)])
def test_untypical_values_at_odd_shapes(n, rows, C, G, size):
    """One lane or 640 of them, one group or as many as channels, fewer rows than lanes, CTAs without rows; large and small numbers."""
    gamma, beta, gen = _affine(C, rows + C)
    x = torch.randn(n * rows, C, generator=gen, device="cuda") + 30
    x[::rows] = -200.0
    x[n * rows // 2, C // 2] = 900.0
    x = (x * size).to(torch.bfloat16)
    _check(x, n, rows, C, G, gamma, beta, B.DP_ACT_NONE, range(min(n, 5)))
