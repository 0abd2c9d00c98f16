"""Refusals, workspaces and launches of the adapter and clipping calls at their limits, from the
library's own host code on a machine without a GPU (see host_hip.py)."""
import ctypes as C
import math
import os

import pytest

import host_hip

G, O, NORM = 0x100000000, 0x200000000, 0x300000000
F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    return host_hip.Host(host_hip.build(str(tmp_path_factory.mktemp("host"))))


@pytest.fixture
def clip(host):
    c = C.c_void_p()
    assert host.lib.countdown_clip_create(1000, C.byref(c)) == 0
    yield c
    assert host.lib.countdown_clip_destroy(c) == 0


def clip_call(host, c, grads, top, norm=NORM):
    words = [w for g in grads for w in g]
    return host.lib.countdown_clip_grads(c, (C.c_uint64 * max(1, len(words)))(*words), len(grads),
                                         top, norm, None)


@pytest.mark.parametrize("grads", [
    [(G, G, 10, F32), (G, O, 10, F32)], [(G, O, 10, F32), (G, G, 10, F32)],
    [(G, G, 10, F32), (G, O, 20, BF16)],  # the same bytes as another type
    [(G, G, 1 << 20, F32), (G, O, 1 << 20, F32)],
])
def test_a_gradient_scaled_in_place_and_read_by_another(host, clip, grads):
    """One tensor's output is another tensor's gradient, whose bytes are those of its own."""
    host.launches()
    assert clip_call(host, clip, grads, 1.0) == host.cd.CD_EINVAL
    assert host.launches() == []


def test_one_gradient_into_two_outputs(host, clip):
    for top in (1.0, math.inf):
        assert clip_call(host, clip, [(G, O, 10, F32), (G, O + 64, 10, F32)], top) == 0
    # with no limit the gradient in place is not written
    assert clip_call(host, clip, [(G, G, 10, F32), (G, O, 10, F32)], math.inf) == 0


# host_hip.cpp with the number of sums that each scaling launch adds up (k_clip_scale's third
# argument) behind its launch
STUB = """
#define hipLaunchKernel record_launch
#include "%s"
#undef hipLaunchKernel
namespace { std::string parts; }
extern "C" const char *host_hip_parts(void) { return parts.c_str(); }
extern "C" hipError_t hipLaunchKernel(const void *f, dim3 grid, dim3 block, void **args, size_t lds,
                                      hipStream_t s)
{
    if (names()[f] == "k_clip_scale")
        parts += std::to_string(grid.x) + " " + std::to_string(*(unsigned *)args[2]) + "\\n";
    return record_launch(f, grid, block, args, lds, s);
}
"""


@pytest.fixture(scope="module")
def counting(tmp_path_factory):
    root = tmp_path_factory.mktemp("counting")
    (root / "tests").mkdir()
    (root / "include").symlink_to(os.path.join(host_hip.ROOT, "include"))
    (root / "tests" / "host_hip.cpp").write_text(
        STUB % os.path.join(host_hip.ROOT, "tests", "host_hip.cpp"))
    with pytest.MonkeyPatch.context() as m:
        m.setattr(host_hip, "ROOT", str(root))
        lib = host_hip.build(str(root))
    h = host_hip.Host(lib)
    h.lib.host_hip_parts.restype = C.c_char_p
    return h


@pytest.mark.parametrize("n", [1, 96, 97, 1000, 20000])
def test_scaling_many_tensors_takes_work_in_proportion(counting, n):
    """n tensors of one chunk each. The first launch's workgroups, at most 96, add the n sums; the
    others must not do so again (n^2 sums in all)."""
    c = C.c_void_p()
    assert counting.lib.countdown_clip_create(n, C.byref(c)) == 0
    before = len(counting.lib.host_hip_parts())
    grads = [(G + 65536 * i, G + 65536 * i, 8191 if n > 1 else 1 << 20, F32) for i in range(n)]
    assert clip_call(counting, c, grads, 1.0) == 0
    rows = [tuple(map(int, line.split()))
            for line in counting.lib.host_hip_parts()[before:].decode().splitlines()]
    assert len(rows) == -(-n // 96)
    sums = n if n > 1 else (1 << 20) // 8192
    assert rows[0][1] == sums
    assert sum(grid * parts for grid, parts in rows) <= rows[0][0] * sums + n
    assert counting.lib.countdown_clip_destroy(c) == 0


# ------------------------------------------------------------------ adapters

PTR = {n: 0x100000000 * (i + 4) for i, n in enumerate(("x", "dy", "ids", "A", "B", "dx", "dA", "dB"))}


@pytest.mark.parametrize("out", ["dA", "dB"])
def test_an_empty_call_has_no_ids(host, out):
    """With T = 0 ids stands for no element, wherever it points."""
    h = C.c_void_p()
    assert host.lib.countdown_adapters_create(264, 520, 24, 3, 64, 1, C.byref(h)) == 0

    def call(T):
        return host.lib.countdown_adapters_backward(
            h, PTR["x"], 264, PTR["dy"], 520, T, PTR[out] + 64, PTR["A"], PTR["B"], None, 1, None, 0,
            PTR["dx"], 264, PTR["dA"], PTR["dB"], None)

    assert call(0) == 0 and call(1) == host.cd.CD_EINVAL
    assert host.lib.countdown_adapters_destroy(h) == 0


@pytest.mark.parametrize("sizes", [  # d_in, d_out, rank, adapters, tokens
    (4096, 4096, 16, 64, 8), (256, 688, 8, 3, 37), (264, 520, 24, 1024, 16), (64, 64, 256, 5, 1),
    (512, 256, 40, 7, 100000),
])
@pytest.mark.parametrize("train", [0, 1])
def test_the_workspace_takes_what_the_header_says(host, sizes, train):
    _, d_out, rank, n, tokens = sizes
    places = -(-tokens // 32) * 32 + 32 * (n + 1)
    size = places * (4 * rank + 4)
    if train:
        size = places * (8 * rank + 12 * (-(-rank // 16) * 16) + 4) + 2 * n * rank * d_out + (16 << 20)
    h = C.c_void_p()
    try:
        host.limit(size + tokens + 40 * n + 3 * 1024)
        assert host.lib.countdown_adapters_create(*sizes, train, C.byref(h)) == 0
        assert host.lib.countdown_adapters_destroy(h) == 0
        host.limit(size)
        assert host.lib.countdown_adapters_create(*sizes, train, C.byref(h)) == host.cd.CD_ENOMEM
    finally:
        host.limit()
