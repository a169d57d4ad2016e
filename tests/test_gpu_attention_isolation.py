"""What dp_attention's results may depend on: the bits of a sequence's rows are the same whatever finite values stand in other
sequences' rows, in rows of no sequence and in keys that the mask hides; and rows whose offsets pass 32 bits."""
import math

import pytest
import torch

import attention_ref as R
from paper_2511_11446_b200 import binding as B

pytestmark = pytest.mark.gpu
FORMS = [0, B.DP_FLAG_FORCE_SIMT, B.DP_FLAG_FORCE_MMA]


def _starts(lens):
    return torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")


def _bits(H, D, lq, lk, q, k, v, causal, cap, slopes, flags):
    y = torch.zeros(q.shape[0], H * D, dtype=torch.bfloat16, device="cuda")
    at = B.make_attn(H, H, D, len(lq), max(lq), max(lk), 1 / math.sqrt(D), q_start=_starts(lq), k_start=_starts(lk),
                     mask=B.DP_MASK_CAUSAL if causal else B.DP_MASK_NONE, cap=cap, slopes=slopes)
    B.dp_attention(at, q, H * D, q.shape[0], k, H * D, v, H * D, k.shape[0], y, H * D, None, flags)
    return y.view(torch.int16)


def _inputs(H, D, Mq, Mk, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda n: torch.randn(n, H * D, generator=gen, device="cuda")  # noqa: E731
    return [(1.5 * rnd(Mq)).to(torch.bfloat16), rnd(Mk).to(torch.bfloat16), rnd(Mk).to(torch.bfloat16)], rnd


@pytest.mark.parametrize("flags", FORMS)
@pytest.mark.parametrize("causal,biased", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("cap", [0.0, 8.0])
@pytest.mark.parametrize("D", [64, 72, 128])
def test_bits_do_not_depend_on_other_sequences(D, cap, causal, biased, flags):
    """The first sequence's rows stay as they are when the second one's, and the rows behind it, go from zero to scores whose
    maxima rise from tile to tile and leave the range of the tanh's polynomial."""
    H = 4
    slopes = torch.linspace(0.1, 0.003, H, device="cuda") if biased else None
    for lq, lk in (([600, 90], [600, 90]), ([100, 40], [1000, 40]), ([260, 1], [77, 1])):
        (q, k, v), rnd = _inputs(H, D, sum(lq) + 70, sum(lk) + 70, 31 + D)
        out = []
        for size in (0.0, 12.0):
            for t, n in ((q, lq[0]), (k, lk[0]), (v, lk[0])):
                t[n:] = (size * rnd(t.shape[0] - n)).to(torch.bfloat16)
            out.append(_bits(H, D, lq, lk, q, k, v, causal, cap, slopes, flags)[:lq[0]])
        assert torch.equal(out[0], out[1]), int((out[0] != out[1]).sum())


@pytest.mark.parametrize("flags", FORMS)
@pytest.mark.parametrize("cap", [0.0, 8.0])
def test_bits_do_not_depend_on_hidden_keys(cap, flags):
    """Causal mask: keys behind a query go from zero to large ones."""
    H, D, n, seen = 4, 64, 400, 250
    (q, k, v), rnd = _inputs(H, D, n, n, 5)
    out = []
    for size in (0.0, 12.0):
        k[seen:] = (size * rnd(n - seen)).to(torch.bfloat16)
        out.append(_bits(H, D, [n], [n], q, k, v, True, cap, None, flags)[:seen])
    assert torch.equal(out[0], out[1]), int((out[0] != out[1]).sum())


@pytest.mark.parametrize("flags", FORMS)
@pytest.mark.parametrize("cap", [0.0, 8.0])
def test_bits_do_not_depend_on_other_queries(cap, flags):
    """A query's row is the same whatever the other queries of its sequence are."""
    H, D, n = 4, 64, 300
    (q, k, v), rnd = _inputs(H, D, n, n, 6)
    out = []
    for size in (0.0, 12.0):
        q[1::2] = (size * rnd(n // 2)).to(torch.bfloat16)
        out.append(_bits(H, D, [n], [n], q, k, v, False, cap, None, flags)[::2])
    assert torch.equal(out[0], out[1]), int((out[0] != out[1]).sum())


def test_every_operand_beyond_32_bit_offsets():
    """Queries, keys, values and outputs in columns of one buffer of 9 GB whose last sequence starts behind element 2^32."""
    H, D, ld, M, first = 2, 64, 1 << 20, 4400, 4150
    assert first * ld > 1 << 32
    n, W = M - first, H * D
    buf = torch.empty(M, ld, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(10)
    buf[first:, :3 * W] = torch.randn(n, 3 * W, generator=gen, device="cuda").to(torch.bfloat16)
    q, k, v, y = (buf[:, i * W:] for i in range(4))
    for nq, flags in ((1, 0), (n, 0), (n, B.DP_FLAG_FORCE_SIMT)):
        buf[first:, 3 * W:4 * W] = 7.0
        starts = (torch.tensor([a, M], dtype=torch.int32, device="cuda") for a in (M - nq, first))
        at = B.make_attn(H, H, D, 1, nq, n, 0.125, q_start=next(starts), k_start=next(starts))
        B.dp_attention(at, q, ld, M, k, ld, v, ld, M, y, ld, None, flags)
        a = first + n - nq
        rows = lambda t, at: t[at:, :W].reshape(M - at, H, D)  # noqa: E731
        want, tol = R.attention(rows(q, a), rows(k, first), rows(v, first), [nq], [n], rows(y, a), 0.125)
        assert ((rows(y, a).double() - want).abs() <= tol).all()
        assert (y[first:a, :W] == 7.0).all()


@pytest.mark.parametrize("flags", FORMS)
@pytest.mark.parametrize("cap", [0.0, 8.0])
@pytest.mark.parametrize("n", [20, 300])
def test_infinite_scores(n, cap, flags):
    """A row whose visible scores are all -inf has no weight to give and is zero, like one that sees no key; a score of +inf or NaN makes
    its row NaN (a cap takes infinite scores to its own size); keys at -inf count for nothing."""
    H, D = 2, 64
    gen = torch.Generator(device="cuda").manual_seed(12)
    v = torch.randn(n, H * D, generator=gen, device="cuda").to(torch.bfloat16)
    q, k = (torch.zeros(n, H * D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q3, k3 = q.view(n, H, D), k.view(n, H, D)
    k3[:, :, 0], k3[:, :, 1], k3[:n // 2, :, 1] = -1.0, -1.0, 1.0
    k3[n // 3, :, 2], k3[:, :, 3] = 2.0, -1.0
    q3[1, :, 0] = math.inf   # every score -inf
    q3[2, :, 0] = -math.inf  # every score +inf
    q3[3, :, 1] = math.inf   # the first half +inf, the second -inf
    q3[4, 0, 3] = math.nan   # head 0 only
    y = _bits(H, D, [n], [n], q, k, v, False, cap, None, flags).view(torch.bfloat16).view(n, H, D)
    mean = v.double().view(n, H, D).mean(0)
    tol = 2.0 ** -6 * v.double().abs().view(n, H, D).mean(0) + 1e-3
    if cap:
        for row in (1, 2):
            assert ((y[row].double() - mean).abs() <= tol).all()
    else:
        assert (y[1] == 0).all() and y[2].isnan().all() and y[3].isnan().all()
    assert y[4, 0].isnan().all()
    rest = torch.ones(n, H, dtype=torch.bool, device="cuda")
    rest[1:4], rest[4, 0] = False, False
    assert ((y.double() - mean).abs() <= tol)[rest].all()


@pytest.mark.parametrize("flags", FORMS)
@pytest.mark.parametrize("order", ["rows", "heads"])
@pytest.mark.parametrize("KV", [4, 1])
def test_operands_that_alternate_in_one_buffer(KV, order, flags):
    """q, k, v and y of a head side by side, [row][head][4][D] or [head][row][4][D]: only y's vectors change."""
    H, D, n = 4, 72, 210
    gen = torch.Generator(device="cuda").manual_seed(14)
    buf = torch.randn(n * H * 4 * D, generator=gen, device="cuda").to(torch.bfloat16)
    t = buf.view(n, H, 4, D) if order == "rows" else buf.view(H, n, 4, D).transpose(0, 1)
    before = t.clone()
    ld, hs = t.stride(0), t.stride(1)
    at = B.make_attn(H, KV, D, 1, n, n, 0.1, q_head_stride=hs, k_head_stride=hs, v_head_stride=hs, y_head_stride=hs)
    B.dp_attention(at, t[:, :, 0], ld, n, t[:, :, 1], ld, t[:, :, 2], ld, n, t[:, :, 3], ld, None, flags)
    want, tol = R.attention(before[:, :, 0], before[:, :KV, 1], before[:, :KV, 2], [n], [n], before[:, :, 3], 0.1)
    assert ((t[:, :, 3].double() - want).abs() <= tol).all()
    assert torch.equal(t[:, :, :3], before[:, :, :3])
