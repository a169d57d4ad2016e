"""The waits of dp_attention's tcgen05 kernel, made to run out (no fault, no hang: a tile of K or V that nothing loads). The kernel
returns by itself with DP_ERR_TIMEOUT in the caller's status word and leaves the context usable."""
import pytest
import torch

import attention_ref as R
from paper_2511_11446_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("skip", [0, 1, 3])
@pytest.mark.parametrize("D,nq,nk,causal", [(64, 300, 300, False), (72, 600, 600, True), (128, 100, 500, False)])
def test_a_tile_that_never_comes_ends_with_timeout_status_and_the_next_call_is_right(D, nq, nk, causal, skip):
    """(two tiles of queries to an item; causal ones of unlike lengths; keys shared by two warpgroups)"""
    H = 3
    gen = torch.Generator(device="cuda").manual_seed(D + skip)
    q, k, v = (torch.randn(n, H * D, generator=gen, device="cuda").to(torch.bfloat16) for n in (nq, nk, nk))
    y = torch.zeros(nq, H * D, dtype=torch.bfloat16, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    at = B.make_attn(H, H, D, 1, nq, nk, 0.125, mask=int(causal))

    def call():
        st.zero_()
        B.dp_attention(at, q, H * D, nq, k, H * D, v, H * D, nk, y, H * D, st, B.DP_FLAG_FORCE_MMA)
        return int(st.item())

    B.dp_debug_skip_stage_load(skip)
    assert call() == B.DP_ERR_TIMEOUT
    assert call() == B.DP_OK
    want, tol = R.attention(q.view(nq, H, D), k.view(nk, H, D), v.view(nk, H, D), [nq], [nk], y.view(nq, H, D), 0.125, causal=causal)
    assert ((y.view(nq, H, D).double() - want).abs() <= tol).all()
