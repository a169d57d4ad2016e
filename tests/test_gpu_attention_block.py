"""The operators between a block's quantized linears, run together with them as a model's forward pass does: LayerNorm +
modulation + quantization, qkv, attention on the columns of its output, projection with its gated residual; and group norm to
codes, a projection, attention. Linears against the oracle on what really went in, the operators against 64 bits."""
import math

import numpy as np
import pytest
import torch

import attention_ref as R
import oracle
from paper_2511_11446_b200 import binding as B, synth
from gpu_util import DevLayer, bf16_to_np, to_dev_bf16
from helpers import bf16_ulp_dist

pytestmark = pytest.mark.gpu
SEED = synth.BASE_SEED + 1300


def _layer(layer, N, K, bits):
    w, s_w = synth.weights(SEED, layer, N, K, bits)
    return w, s_w, synth.bias(SEED, layer, N), DevLayer(w, s_w, synth.bias(SEED, layer, N), bits)


def _close(got, want, tol):
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist())


@pytest.mark.parametrize("H,D,lens", [(16, 72, [256, 256]), (6, 64, [100, 1, 300, 64])])
def test_transformer_block_from_tokens_to_the_residual_stream(H, D, lens):
    W, M = H * D, sum(lens)
    per = max(lens) if len(set(lens)) == 1 else M  # tokens that share a modulation vector
    x = synth.activations(SEED, 0, 0, M, W, 1.0, n_out=W // 100)
    rng = np.random.default_rng(SEED)
    n_mod = -(-M // per)
    shift, scale, gate = (synth.f32_to_bf16_bits(rng.normal(0, 0.3, (n_mod, W)).astype(np.float32)) for _ in range(3))
    qw, qs, qb, qkv = _layer(1, 3 * W, W, 4)
    pw, ps, pb, proj = _layer(2, W, W, 8)
    xd, shd, scd, gd = (to_dev_bf16(t) for t in (x, shift, scale, gate))
    codes = torch.empty(M, W, dtype=torch.int8, device="cuda")
    s_a = torch.empty(M, device="cuda")
    y_qkv = torch.empty(M, 3 * W, dtype=torch.bfloat16, device="cuda")
    att, out = (torch.empty(M, W, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    starts = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    at = B.make_attn(H, H, D, len(lens), max(lens), max(lens), 1 / math.sqrt(D), q_start=starts, k_start=starts)
    mma = B.DP_FLAG_FORCE_MMA | B.DP_FLAG_UNPACK_FIRST
    ws = torch.empty(max(B.dp_wq_linear_workspace(M, 3 * W, W, 4, mma), B.dp_wq_linear_workspace(M, W, W, 8, mma)),
                     dtype=torch.uint8, device="cuda")
    q, k, v = y_qkv.split(W, 1)

    def forward():
        B.dp_ln_modulate_daq(xd, M, W, W, shd, scd, per, 1e-6, codes, W, s_a)
        B.dp_wq_linear(qkv.w, codes, W, s_a, M, y_qkv, 3 * W, ws, None, st, B.DP_FLAG_FORCE_MMA)
        B.dp_attention(at, q, 3 * W, M, k, 3 * W, v, 3 * W, M, att, W, st)
        B.dp_wq_linear_residual(proj.w, att, W, M, xd, W, gd, per, out, W, ws, ws.numel(), st)

    def check():
        torch.cuda.synchronize()
        assert int(st.item()) == 0
        xin = bf16_to_np(xd)
        qo, so = oracle.ln_modulate_daq(xin, shift, scale, per, 1e-6)
        assert np.array_equal(bf16_to_np(y_qkv), oracle.epilogue(oracle.gemm_i32(qo, qw), so, qs, qb))
        want, tol = R.attention(*(t.reshape(M, H, D) for t in (q, k, v)), lens, lens, att.view(M, H, D), 1 / math.sqrt(D))
        _close(att.view(M, H, D), want, tol)
        ref = oracle.wq_linear_residual(bf16_to_np(att), oracle.pack(pw, 8), ps, pb, 8, xin, gate, per)
        assert bf16_ulp_dist(bf16_to_np(out), ref).max() <= 1

    forward()
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        forward()
    xd.copy_(to_dev_bf16(synth.activations(SEED, 7, 3, M, W, 2.0, n_out=W // 100)))
    for t in (codes, s_a, y_qkv, att, out):
        t.zero_()
    graph.replay()
    check()


def test_unet_block_from_a_map_to_attention():
    """A channels-last map through group norm to codes, the 8-bit qkv projection on them, attention over its pixels."""
    n, rows, H, D = 2, 144, 10, 64
    C = H * D
    gen = torch.Generator(device="cuda").manual_seed(21)
    x = torch.randn(n * rows, C, generator=gen, device="cuda").to(torch.bfloat16)
    gamma = (1 + 0.2 * torch.randn(C, generator=gen, device="cuda")).to(torch.bfloat16)
    beta = (0.2 * torch.randn(C, generator=gen, device="cuda")).to(torch.bfloat16)
    w, s_w, b, layer = _layer(3, 3 * C, C, 8)
    codes = torch.empty(n * rows, C, dtype=torch.int8, device="cuda")
    s_a = torch.empty(n * rows, device="cuda")
    y_qkv = torch.empty(n * rows, 3 * C, dtype=torch.bfloat16, device="cuda")
    att = torch.empty(n * rows, C, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(B.dp_group_norm_workspace(n, rows, C, 32), dtype=torch.uint8, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    q, k, v = y_qkv.split(C, 1)
    B.dp_group_norm_daq(x, n, rows, C, C, 32, gamma, beta, 1e-5, B.DP_ACT_NONE, codes, C, s_a, ws)
    B.dp_wq_linear(layer.w, codes, C, s_a, n * rows, y_qkv, 3 * C, None, None, st)
    B.dp_attention(B.make_attn(H, H, D, n, rows, rows, 0.125), q, 3 * C, n * rows, k, 3 * C, v, 3 * C, n * rows, att, C, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    h, tol = R.group_norm(x, n, rows, 32, gamma, beta, 1e-5, False)
    amax = h.abs().amax(1)
    real = h / (amax / 127).view(-1, 1)
    slack = 0.5 + (tol + real.abs() / 127 * tol.amax(1, keepdim=True)) / (amax / 127).view(-1, 1) * 1.01 + 127 * 2.0 ** -22
    assert ((codes.double() - real).abs() <= slack).all()
    y = oracle.epilogue(oracle.gemm_i32(codes.cpu().numpy(), w), s_a.cpu().numpy(), s_w, b)
    assert np.array_equal(bf16_to_np(y_qkv), y)
    want, tol = R.attention(*(t.reshape(-1, H, D) for t in (q, k, v)), [rows] * n, [rows] * n, att.view(-1, H, D), 0.125)
    _close(att.view(-1, H, D), want, tol)
