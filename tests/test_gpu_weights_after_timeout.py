"""Attention weights after a call whose waits gave up: such a call may leave parts of units counted that never met, and
the later calls, of the same build or captured, give what they should."""
import ctypes
import os
import subprocess

import pytest
import torch

from test_gpu_weights import Weights

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def ctx(salt_lib):
    c = salt_lib.salt_ctx_create([64], [64], 1, 1, 1, 1, 1)
    yield c
    salt_lib.salt_ctx_destroy(c)


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    """Reaches into a plan's tables: no wait of the library runs out by itself."""
    so = tmp_path_factory.mktemp("probe") / "track_probe.so"
    root = os.path.dirname(HERE)
    subprocess.run(["nvcc", "-gencode", "arch=compute_103a,code=sm_103a", "-std=c++17", "-shared", "-Xcompiler", "-fPIC",
                    "-I", os.path.join(root, "include"), "-I", os.path.join(root, "paper_2608_03579_gb300", "csrc"),
                    "-o", str(so), os.path.join(HERE, "track_probe.cu")], check=True)
    lib = ctypes.CDLL(str(so))
    lib.track_after_timeout.argtypes = lib.track_split.argtypes = [ctypes.c_void_p]
    return lib


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("own", [0, 70])
def test_parts_that_never_met(salt_lib, ctx, probe, dim, own):
    """One tile of a chunk's rows, split in parts (and few rows' lists beside it)."""
    w = Weights(salt_lib, ctx, [700, 1], [700, own], heads=4, kv_heads=1, dim=dim, page=64)
    w.build()
    assert probe.track_split(w.plan.handle) == 1
    before = w.check()
    x = w.w.cuda()
    other = w.lse + 1.0   # (parts that were left behind are not by chance those of the later calls)
    q, lse = w.q.cuda(), other.cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        salt_lib.salt_attn_weights(w.plan, 0, q, lse, w.scale, x, 1.0)
    assert probe.track_after_timeout(w.plan.handle) == 0
    for _ in range(2):
        after = w.check(lse=other)
        x.copy_(w.w)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(x.cpu(), after)
    w.build()
    assert torch.equal(w.check(), before)
    assert salt_lib.salt_get_device_error(ctx) == 0
