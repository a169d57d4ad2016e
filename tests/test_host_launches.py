"""The library's host side on devices that are not there: its objects linked with a runtime that records calls (fake_cudart.c)
instead of CUDA's. What is launched, with which grids and attributes, on which of several devices; no kernel runs."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2511_11446_b200 import binding as B
from paper_2511_11446_b200 import build

HERE = os.path.dirname(os.path.abspath(__file__))
A = 1 << 40  # an aligned address that nobody dereferences
UNUSED = """cudaEventCreate cudaEventCreateWithFlags cudaEventDestroy cudaEventElapsedTime cudaEventRecord cudaEventSynchronize cudaFree
cudaGetSymbolAddress cudaGraphDestroy cudaGraphExecDestroy cudaGraphInstantiate cudaGraphLaunch cudaLaunchKernel cudaMalloc
cudaMemcpy2DAsync cudaMemcpyAsync cudaMemset cudaStreamBeginCapture cudaStreamCreateWithFlags cudaStreamDestroy cudaStreamEndCapture
cudaStreamWaitEvent""".split()


@pytest.fixture(scope="module")
def fake_path(tmp_path_factory):
    build.build()
    d = tmp_path_factory.mktemp("fake")
    obj, so = str(d / "fake.o"), str(d / "libfake.so")
    include = os.path.join(os.path.dirname(os.path.dirname(build.NVCC)), "include")
    subprocess.check_call([build.CC, "-O1", "-Wall", "-fPIC", "-I" + include, "-c", os.path.join(HERE, "fake_cudart.c"), "-o", obj])
    objs = [os.path.join(build.OBJ, s + ".o") for s in build.SOURCES]
    subprocess.check_call(["g++", "-shared", "-o", so, obj, *objs, "-Wl,-Bsymbolic", "-lpthread",
                           *("-Wl,--defsym=%s=fake_unused" % n for n in UNUSED)])
    return so


@pytest.fixture
def fake(fake_path, tmp_path):
    """A library that has not been used yet."""
    so = str(tmp_path / "lib.so")
    with open(fake_path, "rb") as f, open(so, "wb") as g:
        g.write(f.read())
    L = C.CDLL(so)
    os.remove(so)  # (mapped; a copy for every test takes room)
    for name in ("dp_attention", "dp_group_norm", "dp_group_norm_daq", "dp_daq_quantize", "dp_group_norm_workspace"):
        getattr(L, name).argtypes = getattr(B.lib(), name).argtypes
    L.dp_group_norm_workspace.restype = C.c_size_t
    return L


def _launches(L):
    out = []
    for i in range(L.fake_launches()):
        name, v = C.create_string_buffer(160), (C.c_longlong * 6)()
        assert L.fake_launch(i, name, 160, v) == 0
        out.append((name.value.decode(), *v))
    L.fake_clear_launches()
    return out


def _attention(L, n_seq=1, heads=4, kv_heads=4, dim=64, max_q=1, max_k=8192, packed=False, Mq=None, Mk=None, flags=0):
    a = B.dp_attn(heads, kv_heads, dim, n_seq, max_q, max_k, 0, 0, 0, 0, A if packed else None, A if packed else None, None, None,
                  0.125, 0.0, 0, 0)
    Mq, Mk = Mq or n_seq * max_q, Mk or n_seq * max_k
    ld, ldk, k = heads * dim, kv_heads * dim, 1 << 44
    return L.dp_attention(C.byref(a), k, ld, Mq, 2 * k, ldk, 3 * k, ldk, Mk, 4 * k, ld, None, flags, None)


def test_the_fake_takes_ordinary_calls(fake):
    assert _attention(fake) == B.DP_OK
    assert _attention(fake, max_q=512, max_k=512, n_seq=40) == B.DP_OK
    (few, *f), (tc, *t) = _launches(fake)
    assert "attn_few_kernel" in few and "attn_tc_kernel" in tc and t[0] == 148
    assert f[3] <= f[4] and t[3] <= t[4]  # dynamic shared memory within what the kernel was allowed


@pytest.mark.parametrize("flags", [0, B.DP_FLAG_FORCE_SIMT, B.DP_FLAG_FORCE_MMA])
@pytest.mark.parametrize("kw", [
    dict(n_seq=(1 << 31) - 1, heads=1 << 30, kv_heads=1 << 30, max_q=1 << 30, max_k=1 << 30),
    dict(n_seq=1 << 30, heads=1 << 30, kv_heads=1 << 29, max_q=(1 << 31) - 1024, max_k=800),
    dict(n_seq=1 << 30, heads=1 << 30, kv_heads=1, max_q=1 << 30, max_k=60),
    dict(n_seq=1 << 30, heads=1 << 6, kv_heads=1 << 6, max_q=1 << 28, max_k=100_000),   # 2^64 pairs and queries
    dict(n_seq=1 << 20, heads=1 << 12, kv_heads=1 << 12, max_q=1, max_k=1),             # 2^32 pairs of a sequence and a head
])
def test_more_tiles_than_a_grid_are_refused(fake, kw, flags):
    """(also where their number does not fit 64 bits)"""
    assert _attention(fake, dim=8, packed=True, Mq=1, Mk=1, flags=flags, **kw) == B.DP_ERR_SHAPE
    assert _launches(fake) == []


def test_each_device_has_its_own_room_for_clusters(fake):
    """What another device holds at once, asked when that one is first used, does not change a device's grids (and with them the order
    in which keys are summed)."""
    fake.fake_set_fit(1, 20)
    grids = []
    for device in (0, 1, 0, 1):
        fake.fake_set_device(device)
        assert _attention(fake, n_seq=4, max_k=8192) == B.DP_OK
        (name, grid, _, cluster, *_), = _launches(fake)
        assert "attn_few_kernel" in name
        grids.append((grid, cluster))
    assert grids[0] == grids[2] and grids[1] == grids[3]
    assert grids[0][1] > grids[1][1]


def _group_norm(L, codes):
    n = (1, 4096, 320, 320, 32, None, None, 1e-5, 0, 2 * A, 320)
    return L.dp_group_norm_daq(A, *n, 3 * A, 4 * A, 1 << 20, None) if codes else L.dp_group_norm(A, *n, 4 * A, 1 << 20, None)


def test_operators_prepare_their_kernels_on_their_own_first_call(fake):
    """Linears and their quantization do not wait for attention and group normalisation; each is prepared on every device that it is
    called on, once."""
    prepared = lambda d: [fake.fake_prepared(d, part) for part in (b"attn_", b"gn_")]  # noqa: E731
    for device in (0, 2):
        fake.fake_set_device(device)
        assert fake.dp_daq_quantize(A, 64, 1152, 1152, 2 * A, 1152, 3 * A, None, None) == B.DP_OK
        assert prepared(device) == [0, 0]
        assert _group_norm(fake, False) == B.DP_OK and _group_norm(fake, True) == B.DP_OK
        assert prepared(device)[0] == 0 and prepared(device)[1] > 0
        assert _attention(fake) == B.DP_OK and _attention(fake, n_seq=9, max_q=300, max_k=300) == B.DP_OK
        assert min(prepared(device)) > 0
        for name, _, _, _, smem, allowed, at in _launches(fake):
            assert at == device and (smem <= 48 << 10 or smem <= allowed), name
