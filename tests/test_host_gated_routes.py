"""Which kernels the gated block's and the 4-bit calls launch, with all their template arguments: tiles, whole
cache lines, loads past the caches, row tiles and waves, at both sides of each rule (from the library's own host
code on a machine without a GPU, see host_hip.py)."""
import ctypes as C
from types import SimpleNamespace

import pytest

import host_hip

X, DH, WG, WU, H, DX, DWG, DWU = (0x1000000000 * (i + 1) for i in range(8))


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    return host_hip.Host(host_hip.build(str(tmp_path_factory.mktemp("host"))))


def name(kernel):
    """kernel<arguments> with the truth values as 0 and 1"""
    return kernel.replace("true", "1").replace("false", "0").replace(" ", "")


def launches(host, T, m, f, type=1, **kw):
    """The forward call's kernel and the backward call's kernels of bf16 (1) or fp32 (0) gradients."""
    a = SimpleNamespace(x=X, ldx=m, Wg=WG, Wu=WU, dx=DX, dWg=DWG, dWu=DWU)
    a.__dict__.update(kw)
    h = C.c_void_p()
    assert host.lib.countdown_gated_create(m, f, T, 1 if type else 3, C.byref(h)) == 0
    try:
        host.launches()
        assert host.lib.countdown_gated_forward(h, a.x, a.ldx, T, a.Wg, a.Wu, type, H, f, None) == 0
        forward = [name(k) for k, _ in host.launches()]
        assert host.lib.countdown_gated_backward(h, a.x, a.ldx, DH, f, T, a.Wg, a.Wu, type, a.dx, m,
                                                 a.dWg, a.dWu, None) == 0
        return forward, [name(k) for k, _ in host.launches()]
    finally:
        assert host.lib.countdown_gated_destroy(h) == 0


@pytest.mark.parametrize("T,m,f,type,past", [
    (4, 4096, 14336, 1, 1), (64, 4096, 14336, 1, 1),   # one term: each weight is read once
    (4, 4096, 4096, 1, 0),                             # 64 MB
    (4, 4096, 4104, 1, 1),
    (65, 4096, 14336, 1, 0),                           # two tiles of tokens
    (4, 4096, 14336, 0, 0), (64, 8192, 28672, 0, 0),   # three terms: three times
    (1, 8192, 4096, 1, 0),                             # two
    (1, 8192, 4104, 1, 1),
])
def test_dx_reads_weights_past_the_caches_once(host, T, m, f, type, past):
    _, kernels = launches(host, T, m, f, type, dWg=None, dWu=None)
    assert kernels[1] == f"k_gt_product<2,64,128,64,2,2,1,3,{past},0>"
