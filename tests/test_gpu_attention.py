"""dp_attention against its definition in 64 bits: layouts, lengths, masks, caps, biases, and what must not be touched."""
import math

import pytest
import torch

import attention_ref as R
from paper_2511_11446_b200 import binding as B

pytestmark = pytest.mark.gpu
FORMS = [0, B.DP_FLAG_FORCE_SIMT, B.DP_FLAG_FORCE_MMA]


def _starts(lens, at=0):
    out = [at]
    for n in lens:
        out.append(out[-1] + n)
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def _run(H, KV, D, lq, lk, *, causal=False, prefix=None, cap=0.0, slopes=None, fixed=False, pad=0, layout="qkv", flags=0,
         seed=0, spread=1.5):
    """One call on sequences of lengths lq, lk; the buffers' unused rows hold NaN."""
    gen = torch.Generator(device="cuda").manual_seed(1000 + seed)
    Mq, Mk = sum(lq) + pad, sum(lk) + pad
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    if layout == "qkv":  # one buffer, heads of q, k, v one behind the other (needs equal lengths)
        assert lq == lk
        buf = rnd(Mq, (H + 2 * KV) * D).to(torch.bfloat16)
        buf[:, :H * D] *= spread
        q, k, v = buf.split((H * D, KV * D, KV * D), 1)
        hs = {}
        q3, k3, v3 = q.reshape(Mq, H, D), k.reshape(Mk, KV, D), v.reshape(Mk, KV, D)
        y = rnd(Mq, H * D).to(torch.bfloat16)
        y3 = y.view(Mq, H, D)
        ld = (q.stride(0), k.stride(0), v.stride(0), y.stride(0))
    elif layout == "rows":  # buffers of their own, rows wider than the heads
        q, k, v, y = (rnd(M, n * D + 24).to(torch.bfloat16) for M, n in ((Mq, H), (Mk, KV), (Mk, KV), (Mq, H)))
        hs = {}
        q3, k3, v3, y3 = (t[:, :n * D].unflatten(1, (n, D)) for t, n in ((q, H), (k, KV), (v, KV), (y, H)))
        ld = tuple(t.stride(0) for t in (q, k, v, y))
        q = q * spread
        q3 = q[:, :H * D].unflatten(1, (H, D))
    else:  # head by head: [heads][rows][D + 8]
        q, k, v, y = (rnd(n, M, D + 8).to(torch.bfloat16) for M, n in ((Mq, H), (Mk, KV), (Mk, KV), (Mq, H)))
        hs = dict(q_head_stride=q.stride(0), k_head_stride=k.stride(0), v_head_stride=v.stride(0), y_head_stride=y.stride(0))
        q3, k3, v3, y3 = (t[:, :, :D].transpose(0, 1) for t in (q, k, v, y))
        ld = tuple(t.stride(1) for t in (q, k, v, y))
    if pad:  # rows behind the last sequence
        for t, M in ((q3, Mq), (k3, Mk), (v3, Mk)):
            t[M - pad:] = math.nan
        if layout == "qkv":
            buf[Mq - pad:] = math.nan
    y0 = y.clone()
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    qs, ks = (None, None) if fixed else (_starts(lq), _starts(lk))
    pf = None if prefix is None else torch.tensor(prefix, dtype=torch.int32, device="cuda")
    at = B.make_attn(H, KV, D, len(lq), max(lq), max(lk), 1 / math.sqrt(D), q_start=qs, k_start=ks,
                     mask=B.DP_MASK_CAUSAL if causal else B.DP_MASK_NONE, prefix=pf, cap=cap, slopes=slopes, **hs)
    B.dp_attention(at, q, ld[0], Mq, k, ld[1], v, ld[2], Mk, y, ld[3], st, flags)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    y03 = y0.view(y.shape)
    y03 = y03.view(Mq, H, D) if layout == "qkv" else (y03[:, :H * D].unflatten(1, (H, D)) if layout == "rows" else
                                                      y03[:, :, :D].transpose(0, 1))
    want, tol = R.attention(q3, k3, v3, lq, lk, y03, 1 / math.sqrt(D), cap, slopes, causal, prefix)
    got = y3.double()
    stays = tol < 0
    assert torch.equal(got[stays], want[stays]), "rows of no sequence have changed"
    bad = (~((got - want).abs() <= tol)) & ~stays
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), want[bad][:4].tolist(),
                           tol[bad][:4].tolist())
    if layout == "rows":
        assert torch.equal(y[:, H * D:].view(torch.int16), y0[:, H * D:].view(torch.int16))
    if layout == "heads":
        assert torch.equal(y[:, :, D:].view(torch.int16), y0[:, :, D:].view(torch.int16))
    return y


@pytest.mark.parametrize("flags", FORMS)
@pytest.mark.parametrize("D", [8, 40, 64, 72, 80, 88, 96, 128])
def test_head_dims(D, flags):
    _run(3, 3, D, [200, 131], [200, 131], flags=flags, seed=D)


@pytest.mark.parametrize("flags", FORMS)
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 385, 600])
def test_lengths_around_the_tiles(n, flags):
    _run(2, 1, 64, [n], [n], fixed=True, flags=flags, seed=n)
    _run(2, 2, 72, [n, n], [n, n], causal=True, flags=flags, seed=n + 1)


@pytest.mark.parametrize("flags", FORMS)
@pytest.mark.parametrize("layout", ["qkv", "rows", "heads"])
def test_layouts(layout, flags):
    _run(6, 2, 64, [100, 1, 333], [100, 1, 333], layout=layout, pad=9, flags=flags, causal=layout == "rows")


@pytest.mark.parametrize("flags", FORMS)
def test_packed_documents_and_garbage_behind_them(flags):
    lens = [77, 1, 256, 0, 130, 3, 513, 0]
    _run(4, 4, 72, lens, lens, pad=70, flags=flags)
    _run(4, 2, 128, lens, lens, pad=1, causal=True, flags=flags)


@pytest.mark.parametrize("flags", FORMS)
@pytest.mark.parametrize("causal", [False, True])
def test_cross_lengths_and_empty_sequences(causal, flags):
    """More queries than keys leaves rows without a key under the causal mask; no keys leaves all of them so: zeros."""
    lq, lk = [130, 40, 7, 300, 0, 5, 257], [70, 0, 900, 299, 12, 1, 1]
    y = _run(4, 2, 64, lq, lk, layout="rows", causal=causal, flags=flags)
    assert not y[130:170, :4 * 64].any()
    if causal:
        assert not y[:60, :4 * 64].any()  # 60 queries stand in front of the first key


@pytest.mark.parametrize("flags", FORMS)
@pytest.mark.parametrize("prefix", [[0, 0, 0], [1, 64, 300], [500, 129, 7], [-5, 128, 4000]])
def test_prefix(prefix, flags):
    _run(2, 2, 64, [300, 258, 301], [300, 258, 301], causal=True, prefix=prefix, flags=flags, seed=prefix[1])
    _run(2, 1, 96, [40, 500, 3], [300, 258, 301], causal=True, prefix=prefix, flags=flags, layout="rows", seed=prefix[1])


@pytest.mark.parametrize("flags", FORMS)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("cap,bias", [(2.0, False), (30.0, False), (50.0, True), (0.0, True)])
def test_cap_and_bias(cap, bias, causal, flags):
    H = 4
    slopes = torch.tensor([0.5, 0.0, 0.01, -0.003], device="cuda") if bias else None
    _run(H, 2, 64, [290, 129], [290, 129], cap=cap, slopes=slopes, causal=causal, flags=flags, spread=6.0)
    _run(H, 4, 72, [33, 140], [400, 129], cap=cap, slopes=slopes, causal=causal, flags=flags, spread=6.0, layout="rows",
         prefix=[100, 3] if causal else None)


@pytest.mark.parametrize("flags", [0, B.DP_FLAG_FORCE_SIMT])
@pytest.mark.parametrize("H,KV,D", [(16, 16, 72), (16, 4, 128), (12, 1, 64), (32, 1, 64), (6, 3, 40)])
def test_few_queries_over_long_contexts(H, KV, D, flags):
    _run(H, KV, D, [1, 1, 1], [5000, 64, 1], layout="rows", flags=flags)
    _run(H, KV, D, [1, 3, 16, 2], [3001, 777, 129, 0], layout="rows", causal=True, flags=flags, seed=5)
    _run(H, KV, D, [1], [20011], layout="heads", fixed=True, flags=flags, seed=6)


@pytest.mark.parametrize("flags", FORMS)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("H,KV,D", [(6, 2, 72), (16, 1, 128), (4, 4, 64), (5, 1, 40), (7, 1, 96), (40, 1, 8)])
def test_blocks_of_rows_over_long_contexts(H, KV, D, causal, flags):
    """More (query, head) rows than a block of 32, a query's heads in two blocks, keys cut over CTAs; sequences that end within
    a block, one without queries."""
    lq, lk = [20, 3, 0, 1, 17], [1500, 900, 640, 1, 33]
    _run(H, KV, D, lq, lk, causal=causal, layout="rows", pad=3, flags=flags, seed=H)
    _run(H, KV, D, lq, lk, causal=True, prefix=[0, 700, 5, 1, 40], cap=20.0, layout="heads", flags=flags, seed=D,
         slopes=torch.linspace(0.5, 0.004, H, device="cuda"))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D", [64, 72, 96, 128])
def test_keys_shared_by_two_warpgroups(D, causal):
    """Items of up to 128 queries of more keys than 384, several to a CTA: odd and even numbers of key tiles, one tile, none; the
    larger half's scores first or last."""
    lk = [400, 97, 1, 0, 385, 193, 96, 289, 640, 80] * 5
    lq = [128, 5, 1, 3, 100, 64, 96, 0, 17, 128] * 5
    _run(4, 2, D, lq, lk, causal=causal, layout="rows", pad=2, flags=B.DP_FLAG_FORCE_MMA, seed=D)
    _run(8, 8, D, [100] * 24, [500] * 24, fixed=True, causal=causal, layout="heads", flags=B.DP_FLAG_FORCE_MMA, seed=D + 1, spread=6.0,
         slopes=torch.linspace(1.0, -0.02, 8, device="cuda"))


@pytest.mark.parametrize("flags", FORMS)
def test_scores_of_large_spread(flags):
    """One key takes all the weight, and the running maximum jumps from tile to tile."""
    _run(2, 2, 64, [300], [300], flags=flags, spread=40.0)
    _run(2, 2, 64, [257], [700], flags=flags, spread=40.0, layout="rows", causal=True)


@pytest.mark.parametrize("flags", FORMS)
def test_scores_that_rise_along_the_keys(flags):
    """The maximum moves in every tile: each needs the sums so far taken to the new one."""
    H, D, n = 2, 64, 900
    q = torch.full((n, H * D), 1.0, device="cuda", dtype=torch.bfloat16)
    k = (torch.arange(n, device="cuda").view(n, 1) * 0.05).expand(n, H * D).to(torch.bfloat16).contiguous()
    gen = torch.Generator(device="cuda").manual_seed(3)
    v = torch.randn(n, H * D, generator=gen, device="cuda").to(torch.bfloat16)
    y = torch.zeros(n, H * D, device="cuda", dtype=torch.bfloat16)
    for sign in (1.0, -1.0):
        at = B.make_attn(H, H, D, 1, n, n, 1 / 8)
        B.dp_attention(at, (q * sign).contiguous(), H * D, n, k, H * D, v, H * D, n, y, H * D, None, flags)
        want, tol = R.attention((q * sign).view(n, H, D), k.view(n, H, D), v.view(n, H, D), [n], [n], y.view(n, H, D), 1 / 8)
        assert ((y.view(n, H, D).double() - want).abs() <= tol).all()


@pytest.mark.parametrize("flags", FORMS)
def test_hidden_keys_may_hold_anything(flags):
    """Keys that no query of the tile may see hold inf and NaN; values there are finite."""
    H, D, n = 2, 64, 300
    gen = torch.Generator(device="cuda").manual_seed(4)
    q, k, v = (torch.randn(n, H * D, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(3))
    q[-1] = 0  # (the last query sees every key: zeros, compared below without it)
    kk = k.clone()
    kk[-1] = math.inf
    kk[-2, ::2] = math.nan
    out = []
    for t in (k, kk):
        y = torch.zeros(n, H * D, device="cuda", dtype=torch.bfloat16)
        B.dp_attention(B.make_attn(H, H, D, 1, n, n, 0.125, mask=B.DP_MASK_CAUSAL), q, H * D, n, t, H * D, v, H * D, n, y,
                       H * D, None, flags)
        out.append(y[:n - 2])
    assert torch.equal(out[0], out[1]) and torch.isfinite(out[1]).all()


@pytest.mark.parametrize("flags", FORMS)
def test_offsets_that_leave_the_buffers_are_cut(flags):
    """Wrong offsets give wrong rows, never an access outside: the sequences that are right keep their results."""
    H, D, n = 2, 64, 200
    gen = torch.Generator(device="cuda").manual_seed(5)
    q, k, v = (torch.randn(n, H * D, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(3))
    y = torch.zeros(n, H * D, device="cuda", dtype=torch.bfloat16)
    qs = torch.tensor([0, 50, 50, 2000, 100, -7], dtype=torch.int32, device="cuda")
    ks = torch.tensor([0, 50, 40, 1 << 30, -(1 << 30), 90], dtype=torch.int32, device="cuda")
    at = B.make_attn(H, H, D, 5, 130, 130, 0.125, q_start=qs, k_start=ks)
    B.dp_attention(at, q, H * D, n, k, H * D, v, H * D, n, y, H * D, None, flags)
    torch.cuda.synchronize()
    want, tol = R.attention(q[:50].view(50, H, D), k[:50].view(50, H, D), v[:50].view(50, H, D), [50], [50],
                            y[:50].view(50, H, D), 0.125)
    assert ((y[:50].view(50, H, D).double() - want).abs() <= tol).all()


def test_queries_beyond_max_q_are_left_out():
    H, D = 2, 64
    q, k, v = (torch.randn(300, H * D, device="cuda").to(torch.bfloat16) for _ in range(3))
    y = torch.full((300, H * D), 7.0, device="cuda", dtype=torch.bfloat16)
    st = _starts([300])
    for flags in FORMS:
        y.fill_(7.0)
        B.dp_attention(B.make_attn(H, H, D, 1, 150, 300, 0.125, q_start=st, k_start=st), q, H * D, 300, k, H * D, v, H * D, 300,
                       y, H * D, None, flags)
        want, tol = R.attention(q.view(300, H, D), k.view(300, H, D), v.view(300, H, D), [300], [300], y.view(300, H, D), 0.125)
        assert ((y[:150].view(150, H, D).double() - want[:150]).abs() <= tol[:150]).all()
        assert (y[150:] == 7.0).all()


@pytest.mark.parametrize("flags", FORMS)
def test_same_bits_every_time_streams_and_graphs(flags):
    """No result depends on the order in which blocks run: eager, on another stream, captured and replayed."""
    H, KV, D, lens = 8, 4, 72, [300, 77, 512, 1]
    n = sum(lens)
    gen = torch.Generator(device="cuda").manual_seed(8)
    qkv = torch.randn(n, (H + 2 * KV) * D, generator=gen, device="cuda").to(torch.bfloat16)
    q, k, v = qkv.split((H * D, KV * D, KV * D), 1)
    st = _starts(lens)
    at = B.make_attn(H, KV, D, 4, 512, 512, 0.1, q_start=st, k_start=st, mask=B.DP_MASK_CAUSAL)
    outs = [torch.zeros(n, H * D, device="cuda", dtype=torch.bfloat16) for _ in range(3)]
    ld = qkv.stride(0)
    call = lambda y: B.dp_attention(at, q, ld, n, k, ld, v, ld, n, y, H * D, None, flags)  # noqa: E731
    call(outs[0])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        call(outs[1])
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(outs[2])
    for _ in range(3):
        outs[2].zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[2])
    assert torch.equal(outs[0], outs[1])


def test_two_calls_at_once_on_two_streams():
    H, D, n = 8, 64, 700
    gen = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn(n, 3 * H * D, generator=gen, device="cuda").to(torch.bfloat16)
    q, k, v = x.split(H * D, 1)
    at = B.make_attn(H, H, D, 1, n, n, 0.125)
    few = B.make_attn(H, H, D, 1, 3, n, 0.125)
    ref, ref1 = (torch.zeros(m, H * D, device="cuda", dtype=torch.bfloat16) for m in (n, 3))
    B.dp_attention(at, q, x.stride(0), n, k, x.stride(0), v, x.stride(0), n, ref, H * D)
    B.dp_attention(few, q, x.stride(0), 3, k, x.stride(0), v, x.stride(0), n, ref1, H * D)
    torch.cuda.synchronize()
    s = [torch.cuda.Stream() for _ in range(2)]
    ys = [torch.zeros(n, H * D, device="cuda", dtype=torch.bfloat16) for _ in range(4)]
    zs = [torch.zeros(3, H * D, device="cuda", dtype=torch.bfloat16) for _ in range(4)]
    torch.cuda.synchronize()
    for i in range(4):
        B.dp_attention(at, q, x.stride(0), n, k, x.stride(0), v, x.stride(0), n, ys[i], H * D, stream=s[i % 2])
        B.dp_attention(few, q, x.stride(0), 3, k, x.stride(0), v, x.stride(0), n, zs[i], H * D, stream=s[1 - i % 2])
    torch.cuda.synchronize()
    assert all(torch.equal(ref, y) for y in ys) and all(torch.equal(ref1, z) for z in zs)


def test_rows_beyond_32_bit_offsets():
    """Keys whose element offsets pass 2^31 and byte offsets 2^32: the last rows of a buffer of 5 GB."""
    H, D = 2, 64
    ld, Mk = 1 << 15, 80_000
    buf = torch.zeros(Mk * ld // 2 + ld, dtype=torch.bfloat16, device="cuda")  # rows of k and v overlap in the buffer: ld / 2 apart
    ld //= 2
    k = buf[:Mk * ld].view(Mk, ld)
    gen = torch.Generator(device="cuda").manual_seed(10)
    first = Mk - 200
    k[first:, :2 * H * D] = torch.randn(200, 2 * H * D, generator=gen, device="cuda").to(torch.bfloat16)
    assert (Mk - 1) * ld * 2 > 1 << 31
    for nq, flags in ((1, 0), (200, 0), (200, B.DP_FLAG_FORCE_SIMT)):
        q = torch.randn(nq, H * D, generator=gen, device="cuda").to(torch.bfloat16)
        y = torch.zeros(nq, H * D, dtype=torch.bfloat16, device="cuda")
        qs = torch.tensor([0, nq], dtype=torch.int32, device="cuda")
        ks = torch.tensor([first, Mk], dtype=torch.int32, device="cuda")
        at = B.make_attn(H, H, D, 1, nq, 200, 0.125, q_start=qs, k_start=ks)
        B.dp_attention(at, q, H * D, nq, k, ld, k[:, H * D:], ld, Mk, y, H * D, None, flags)
        kk, vv = k[first:, :H * D].reshape(200, H, D), k[first:, H * D:2 * H * D].reshape(200, H, D)
        want, tol = R.attention(q.view(nq, H, D), kk, vv, [nq], [200], y.view(nq, H, D), 0.125)
        assert ((y.view(nq, H, D).double() - want).abs() <= tol).all()


@pytest.mark.parametrize("flags", FORMS)
def test_output_in_columns_of_the_inputs_buffer(flags):
    """y beside q, k and v in the rows of one buffer: nothing overlaps, and only y's columns change."""
    H, D, n = 4, 64, 150
    W = H * D
    gen = torch.Generator(device="cuda").manual_seed(11)
    buf = torch.randn(n, 4 * W, generator=gen, device="cuda").to(torch.bfloat16)
    before = buf.clone()
    q, k, v, y = buf.split(W, 1)
    B.dp_attention(B.make_attn(H, H, D, 1, n, n, 0.125), q, 4 * W, n, k, 4 * W, v, 4 * W, n, y, 4 * W, None, flags)
    want, tol = R.attention(*(t.reshape(n, H, D) for t in (q, k, v)), [n], [n], y.reshape(n, H, D), 0.125)
    assert ((y.reshape(n, H, D).double() - want).abs() <= tol).all()
    assert torch.equal(buf[:, :3 * W], before[:, :3 * W])


@pytest.mark.parametrize("flags", [0, B.DP_FLAG_FORCE_MMA])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n_seq", [63, 64, 65, 150])
def test_many_sequences_of_unlike_lengths(n_seq, causal, flags):
    """More work items than SMs, sequences sorted by length up to 64 of them, empty ones among them."""
    gen = torch.Generator().manual_seed(n_seq)
    lens = torch.randint(0, 300, (n_seq,), generator=gen).tolist()
    lens[n_seq // 2], lens[-1], lens[0] = 0, 700, 1
    _run(4, 2, 40, lens, lens, causal=causal, flags=flags, pad=3, seed=n_seq)


@pytest.mark.parametrize("causal", [False, True])
def test_max_q_far_above_the_sequences(causal):
    """max_q and max_k of a longest sequence that is not in this batch: nearly all tiles of queries are not there."""
    n_seq, H, D = 2000, 4, 64
    gen = torch.Generator(device="cuda").manual_seed(5)
    lens = [(7 * i) % 4 for i in range(n_seq)]
    lens[3], lens[1500] = 700, 0
    M = sum(lens)
    q, k, v, y = (torch.randn(M, H * D, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(4))
    starts, st = _starts(lens), torch.zeros(1, dtype=torch.int32, device="cuda")
    at = B.make_attn(H, H, D, n_seq, 1 << 25, 1 << 25, 0.125, q_start=starts, k_start=starts, mask=int(causal))
    B.dp_attention(at, q, H * D, M, k, H * D, v, H * D, M, y, H * D, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    want, tol = R.attention(*(t.view(M, H, D) for t in (q, k, v)), lens, lens, y.view(M, H, D), 0.125, 0.0, None, causal)
    assert ((y.view(M, H, D).double() - want).abs() <= tol).all()


@pytest.mark.parametrize("D", [64, 72, 128])
def test_many_rounds_of_equal_items(D):
    _run(8, 8, D, [300] * 40, [300] * 40, fixed=True, seed=D)
    _run(8, 4, D, [520] * 12, [520] * 12, fixed=True, causal=True, prefix=[0, 5, 130, 600] * 3, seed=D)


def test_long_sequence():
    """Tiles far behind each other, and one query among them."""
    _run(1, 1, 64, [6000], [6000], fixed=True, causal=True, seed=1)
    _run(2, 1, 128, [130], [30011], layout="rows", seed=2)
