"""Refusals, workspaces and launches of the adapter and clipping calls at their limits, from the
library's own host code on a machine without a GPU (see host_hip.py)."""
import ctypes as C
import math

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
