"""Which kernels the gated block's and the 4-bit calls launch, with all their template arguments: tiles, whole
cache lines, loads past the caches, row tiles and waves, at both sides of each rule (from the library's own host
code on a machine without a GPU, see host_hip.py)."""
import ctypes as C
import re
import subprocess
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


def compiled(host, kernel):
    """The instantiations of a kernel that the library holds."""
    out = subprocess.run(["nm", "-C", host.lib._name], check=True, capture_output=True, text=True).stdout
    found = re.findall(rf"\(anonymous namespace\)::__device_stub__({kernel}<[^>]*>)", out)
    assert found
    return {name(k) for k in found}


# tokens, rows, cols of a project call; its row tiles, room for tokens, waves, and whether past the caches
Q4_PROJECT = [
    (1, 72, 264, 1, 4, 8, 0), (4, 6144, 264, 1, 4, 8, 0), (3, 4088, 33000, 1, 4, 8, 1),
    (5, 6136, 264, 1, 8, 8, 0), (8, 4088, 520, 1, 8, 8, 0), (7, 4088, 33000, 1, 8, 8, 1),
    (5, 6144, 264, 2, 8, 8, 0), (8, 8200, 264, 2, 8, 8, 0), (6, 8200, 17000, 2, 8, 8, 1),
    (9, 4096, 264, 1, 16, 8, 0), (16, 4088, 33000, 1, 16, 8, 1),
    (13, 4104, 1000, 1, 16, 4, 0), (16, 6136, 712, 1, 16, 4, 0), (13, 5000, 28680, 1, 16, 4, 1),
    (9, 6144, 264, 2, 16, 8, 0), (16, 8192, 264, 2, 16, 8, 0), (9, 8184, 17000, 2, 16, 8, 1),
    (9, 8200, 1000, 2, 16, 4, 0), (16, 8200, 17000, 2, 16, 4, 1),
]
# the same of a gated call, which has a tile of either matrix
Q4_GATED = [
    (1, 72, 264, 4, 8, 0), (4, 4104, 264, 4, 8, 0), (2, 4088, 16408, 4, 8, 1),
    (5, 4104, 264, 8, 8, 0), (8, 72, 264, 8, 8, 0), (8, 4088, 16408, 8, 8, 1),
    (9, 4096, 264, 16, 8, 0), (16, 4088, 16408, 16, 8, 1),
    (13, 4104, 1000, 16, 4, 0), (11, 5000, 13096, 16, 4, 1),
]


@pytest.mark.parametrize("group", [32, 64, 128])
def test_kernels_of_the_4_bit_calls(host, group):
    seen = set()
    for T, rows, cols, *want in Q4_PROJECT:
        host.launches()
        assert host.lib.countdown_q4_project(X, cols, T, WG, cols, rows, group, 0, None, 0, H, rows, None) == 0
        (kernel, _), = host.launches()
        tiles, room, waves, past = want
        assert name(kernel) == f"k_q4<{tiles},{group},{room},{waves},0,{past}>", (T, rows, cols)
        seen.add(name(kernel))
    for T, rows, cols, room, waves, past in Q4_GATED:
        host.launches()
        assert host.lib.countdown_q4_gated(X, cols, T, WG, WU, cols, rows, group, 1, H, rows, None) == 0
        (kernel, _), = host.launches()
        assert name(kernel) == f"k_q4<2,{group},{room},{waves},1,{past}>", (T, rows, cols)
        seen.add(name(kernel))
    assert seen == {k for k in compiled(host, "k_q4") if k.split(",")[1] == str(group)}


# tokens, d_model, d_ff, elements before x in its rows (which are 64 longer then); the tile of both projections: rows,
# columns, k, waves of each, stages, past the caches, whole cache lines (large: halves of 128 rows)
PROJECTIONS = [
    (1, 256, 688, 0, "16,16,256,1,1,4,3,0,0"), (16, 264, 688, 8, "16,16,256,1,1,4,3,0,0"),
    (16, 2120, 8192, 0, "16,16,256,1,1,4,3,1,0"),
    (17, 256, 2048, 0, "32,32,128,1,2,2,4,0,0"), (17, 264, 2048, 0, "32,32,128,1,2,2,5,0,1"),
    (17, 256, 2048, 8, "32,32,128,1,2,2,5,0,1"), (17, 256, 2048, 64, "32,32,128,1,2,2,4,0,0"),
    (20, 2112, 8192, 0, "32,32,128,1,2,2,4,1,0"), (20, 2120, 8192, 0, "32,32,128,1,2,2,5,1,1"),
    (128, 256, 4096, 0, "64,32,128,2,2,1,4,0,0"), (128, 264, 4096, 0, "64,32,128,2,2,1,5,0,1"),
    (48, 2112, 8192, 0, "64,32,128,2,2,1,4,1,0"), (48, 2120, 8192, 0, "64,32,128,2,2,1,5,1,1"),
    (200, 128, 3000, 0, "64,64,128,2,4,1,3,0,0"), (200, 128, 3000, 24, "64,64,64,2,4,1,6,0,1"),
    (64, 2048, 8200, 0, "64,64,128,2,4,1,3,1,0"), (64, 2056, 8200, 0, "64,64,64,2,4,1,6,1,1"),
    (500, 64, 3000, 0, "128,64,64,2,4,1,3,0,0"), (500, 72, 3000, 0, "128,64,64,2,4,1,4,0,1"),
    (700, 64, 3520, 0, "192,64,64,4,2,1,3,0,0"), (700, 64, 3520, 40, "192,64,64,4,2,1,4,0,1"),
    (900, 64, 4000, 0, "large1"), (900, 72, 4000, 0, "large1"), (2000, 264, 4104, 0, "large2"),
]
# tokens, d_model, d_ff, type (1 bf16, 0 fp32); the kernels behind the projections of a backward call
BEHIND = [
    (37, 256, 688, 1, "k_gt_back"), (300, 256, 1024, 0, "k_gt_product<2,64,128,64,2,2,1,3,0,0>",
                                     "k_gt_product<3,64,64,64,2,2,1,3,0,0>"),
    (4, 4096, 4104, 1, "k_gt_product<2,64,128,64,2,2,1,3,1,0>", "k_gt_product<3,128,128,64,2,2,1,2,0,0>"),
    (1300, 1544, 2056, 1, "k_gt_large<2,2>", "k_gt_product<3,128,128,64,2,2,1,2,0,0>"),
    (520, 2048, 2816, 0, "k_gt_large<2,2>", "k_gt_large<3,2>"),
]


def projection(kind, tile):
    return f"k_gt_large<{kind},{tile[5:]}>" if tile.startswith("large") else f"k_gt_product<{kind},{tile}>"


def test_kernels_of_the_gated_block(host):
    seen = set()
    for T, m, f, at, tile in PROJECTIONS:
        forward, backward = launches(host, T, m, f, x=X + 2 * at, ldx=m + (64 if at else 0))
        assert forward == [projection(0, tile)] and backward[0] == projection(1, tile), (T, m, f, at)
        seen.update(forward + backward)
    for T, m, f, type, *want in BEHIND:
        _, kernels = launches(host, T, m, f, type)
        assert [k for k in kernels[1:] if not k.startswith("k_gt_sum")] == want, (T, m, f, type)
        seen.update(kernels)
    for kernel in ("k_gt_product", "k_gt_large"):
        assert {k for k in seen if k.startswith(kernel)} == compiled(host, kernel)


def test_what_begins_inside_a_cache_line(host):
    """x's first row, its row length, the weights' row length or W_gate's first row."""
    for kw, lines in (({}, 0), ({"x": X + 16}, 1), ({"x": X + 128, "ldx": 320}, 0), ({"ldx": 264}, 1),
                      ({"Wg": WG + 64}, 1), ({"Wg": WG + 256}, 0)):
        forward, backward = launches(host, 200, 256, 3000, **kw)
        tile = "64,64,64,2,4,1,6,0,1" if lines else "64,64,128,2,4,1,3,0,0"
        assert forward == [projection(0, tile)] and backward[0] == projection(1, tile), kw
