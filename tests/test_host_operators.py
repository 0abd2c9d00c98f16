"""What the adapter and clipping calls refuse, allocate and launch, from the library's own
host code on a machine without a GPU (see host_hip.py)."""
import ctypes as C
import math

import pytest

import host_hip

D_IN, D_OUT, RANK, N, T = 264, 520, 24, 3, 64
P = {n: 0x100000000 * (i + 1) for i, n in enumerate(
    ("x", "dy", "W", "ids", "A", "B", "scale", "base", "y", "dA", "dB", "norm", "g0", "g1", "o0",
     "o1"))}


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    return host_hip.Host(host_hip.build(str(tmp_path_factory.mktemp("host"))))


def create(host, *args):
    h = C.c_void_p()
    return host.lib.countdown_adapters_create(*args, C.byref(h)), h


@pytest.fixture
def pool(host):
    st, h = create(host, D_IN, D_OUT, RANK, N, T, 1)
    assert st == host.cd.CD_OK
    yield h
    assert host.lib.countdown_adapters_destroy(h) == host.cd.CD_OK


def add(host, h, **kw):
    a = dict(x=P["x"], ldx=D_IN, T=T, ids=P["ids"], A=P["A"], B=P["B"], scale=P["scale"], type=0,
             base=P["base"], ldb=D_OUT, y=P["y"], ldy=D_OUT)
    a.update(kw)
    return host.lib.countdown_adapters_add(h, *a.values(), None)


def project(host, h, **kw):
    a = dict(x=P["x"], ldx=D_IN, T=16, W=P["W"], ids=P["ids"], A=P["A"], B=P["B"],
             scale=P["scale"], type=0, y=P["y"], ldy=D_OUT)
    a.update(kw)
    return host.lib.countdown_adapters_project(h, *a.values(), None)


def backward(host, h, **kw):
    a = dict(x=P["x"], ldx=D_IN, dy=P["dy"], lddy=D_OUT, T=T, ids=P["ids"], A=P["A"], B=P["B"],
             scale=P["scale"], type=1, base=P["base"], ldb=D_IN, dx=P["y"], lddx=D_IN, dA=P["dA"],
             dB=P["dB"])
    a.update(kw)
    return host.lib.countdown_adapters_backward(h, *a.values(), None)


@pytest.mark.parametrize("args,status", [
    ((8, 8, 8, 1, 1, 0), 0), ((65536, 65536, 256, 1024, 1, 1), 0),
    ((0, 8, 8, 1, 1, 0), -1), ((12, 8, 8, 1, 1, 0), -1), ((8, 12, 8, 1, 1, 0), -1),
    ((8, 8, 0, 1, 1, 0), -1), ((8, 8, 12, 1, 1, 0), -1), ((8, 8, 8, 0, 1, 0), -1),
    ((8, 8, 8, 1, 0, 0), -1), ((8, 8, 8, 1, 1, 2), -1), ((65544, 8, 8, 1, 1, 0), -2),
    ((8, 65544, 8, 1, 1, 0), -2), ((8, 8, 264, 1, 1, 0), -2), ((8, 8, 8, 1025, 1, 0), -2),
    ((8, 8, 8, 1, (1 << 20) + 1, 0), -2),
])
def test_pool_sizes(host, args, status):
    st, h = create(host, *args)
    assert st == status and bool(h) == (status == 0)
    assert host.lib.countdown_adapters_destroy(h) == 0


def test_a_failed_allocation_leaves_nothing(host):
    live = host.lib.host_hip_live_allocations()
    host.limit(64)
    try:
        st, h = create(host, D_IN, D_OUT, RANK, N, T, 1)
        assert st == host.cd.CD_ENOMEM and not h
        c = C.c_void_p()
        assert host.lib.countdown_clip_create(4, C.byref(c)) == host.cd.CD_ENOMEM and not c
    finally:
        host.limit()
    assert host.lib.host_hip_live_allocations() == live


def test_launches_by_the_work(host):
    """One launch for little work, two by token, three with the tokens grouped."""
    def kernels(call, sizes, **kw):
        st, h = create(host, *sizes, 1)
        assert st == 0
        host.launches()
        assert call(host, h, ldx=sizes[0], **kw) == 0
        out = [k.split("<")[0] for k, _ in host.launches()]
        assert host.lib.countdown_adapters_destroy(h) == 0
        return out

    by_token, grouped = ["k_ad_lat", "k_ad_up"], ["k_ad_group", "k_ad_shrink", "k_ad_expand"]
    for sizes, T, want in [((4096, 4096, 16, 16), 8, ["k_ad_token"]),
                           ((4096, 4096, 16, 16), 128, ["k_ad_token"]),
                           ((4096, 4096, 16, 16), 383, by_token),
                           ((4096, 4096, 16, 16), 384, grouped),
                           ((4096, 4096, 16, 16), 1024, grouped),
                           ((4096, 4096, 64, 16), 1, by_token),
                           ((512, 1024, 128, 4), 1, by_token),
                           ((4096, 14336, 64, 8), 57, grouped),
                           ((8, 8, 8, 1), 200000, ["k_ad_token"])]:
        assert kernels(add, (*sizes, T), T=T, ldb=sizes[1], ldy=sizes[1]) == want, (sizes, T)
    for sizes, T, want in [((4096, 4096, 16, 8), 1, ["k_ad_project"]),
                           ((4096, 4096, 16, 8), 8, ["k_ad_lat", "k_ad_project"]),
                           ((1000, 8192, 16, 8), 2, ["k_ad_project"]),
                           ((1000, 8200, 16, 8), 2, ["k_ad_lat", "k_ad_project"]),
                           ((1000, 1024, 40, 8), 1, ["k_ad_lat", "k_ad_project"])]:
        assert kernels(project, (*sizes, T), T=T, ldy=sizes[1]) == want
    back = ["k_ad_group", "k_ad_shrink", "k_ad_back"]
    for sizes, T, want in [((256, 688, 8, 3), 37, back), ((4096, 4096, 16, 4), 4096, back),
                           ((520, 1080, 40, 1), 4877, back + ["k_ad_sum"]),
                           ((4096, 4096, 16, 4), 16, ["k_ad_few_latents", "k_ad_few_back"]),
                           ((4096, 4096, 16, 1), 8, ["k_ad_few_latents", "k_ad_few_back"]),
                           ((4096, 4096, 16, 1), 9, back), ((256, 688, 40, 4), 1, back),
                           ((4096, 4096, 16, 4), 17, back), ((1024, 3000, 64, 4), 8, back)]:
        kw = dict(T=T, lddy=sizes[1], ldb=sizes[0], lddx=sizes[0])
        assert kernels(backward, (*sizes, T), **kw) == want


def test_calls_allocate_nothing(host, pool):
    live = host.lib.host_hip_live_allocations()
    assert add(host, pool) == 0 and project(host, pool) == 0 and backward(host, pool) == 0
    assert host.lib.host_hip_live_allocations() == live


BAD = [  # for every call
    dict(T=-1), dict(T=T + 1), dict(x=None), dict(x=P["x"] + 8), dict(ldx=D_IN - 8),
    dict(ldx=D_IN + 4), dict(ids=None), dict(ids=P["ids"] + 2), dict(A=None), dict(A=P["A"] + 2),
    dict(B=None), dict(B=P["B"] + 8), dict(scale=P["scale"] + 1), dict(type=2), dict(type=-1),
]
BAD_ADD = BAD + [
    dict(y=None), dict(y=P["y"] + 4), dict(ldy=D_OUT - 8), dict(ldy=D_OUT + 2),
    dict(base=P["base"] + 8), dict(ldb=0), dict(y=P["x"]), dict(y=P["A"]), dict(y=P["B"] + 64),
    dict(y=P["ids"]), dict(y=P["scale"]), dict(y=P["base"] + 16),
    dict(y=P["base"], ldy=D_OUT + 8),              # in place, but another stride
    dict(y=P["base"] + D_OUT * 4),                 # one row further
    dict(base=P["y"], ldb=1024, ldy=1024, y=P["y"] + 512 * 4),  # column slices that overlap
]


@pytest.mark.parametrize("kw", BAD_ADD, ids=str)
def test_add_refuses(host, pool, kw):
    host.launches()
    assert add(host, pool, **kw) == host.cd.CD_EINVAL
    assert host.launches() == []


def test_add_accepts(host, pool):
    for kw in (dict(base=None, ldb=0), dict(scale=None), dict(base=P["y"]), dict(type=1),
               dict(base=P["y"], ldb=2048, ldy=2048, y=P["y"] + 1024 * 4), dict(T=1), dict(ldx=272),
               dict(T=0), dict(T=0, x=None, ids=None, y=None, base=None)):
        assert add(host, pool, **kw) == 0, kw
    assert host.lib.countdown_adapters_add(None, P["x"], D_IN, T, P["ids"], P["A"], P["B"], None, 0,
                                           None, 0, P["y"], D_OUT, None) == host.cd.CD_EINVAL


@pytest.mark.parametrize("kw", BAD + [
    dict(W=None), dict(W=P["W"] + 8), dict(y=None), dict(y=P["W"]), dict(y=P["x"]), dict(ldy=8),
], ids=str)
def test_project_refuses(host, pool, kw):
    host.launches()
    assert project(host, pool, **kw) == host.cd.CD_EINVAL
    assert project(host, pool, T=17) == host.cd.CD_EUNSUPPORTED
    assert host.launches() == []
    assert project(host, pool, T=0, x=None, ids=None, y=None) == 0


@pytest.mark.parametrize("kw", BAD + [
    dict(dy=None), dict(dy=P["dy"] + 4), dict(lddy=D_OUT - 8), dict(dx=P["y"] + 2), dict(lddx=8),
    dict(dA=P["dA"] + 4), dict(dB=P["dB"] + 4), dict(dx=P["dy"]), dict(dx=P["x"]), dict(dA=P["A"]),
    dict(dB=P["B"]), dict(dA=P["dB"]), dict(dx=P["dA"]), dict(dA=P["x"]), dict(dB=P["dy"]),
    dict(dA=P["base"]), dict(ldb=D_IN + 8, base=P["y"]),
], ids=str)
def test_backward_refuses(host, pool, kw):
    host.launches()
    assert backward(host, pool, **kw) == host.cd.CD_EINVAL
    assert host.launches() == []


def test_backward_accepts(host, pool):
    for kw in (dict(base=None), dict(dx=None, base=None, lddx=0), dict(dA=None), dict(dB=None),
               dict(dx=None, dA=None, dB=None), dict(base=P["y"]), dict(type=0), dict(T=1),
               dict(T=0, x=None, dy=None, ids=None, dx=None)):
        assert backward(host, pool, **kw) == 0, kw
    st, h = create(host, D_IN, D_OUT, RANK, N, T, 0)
    assert st == 0
    assert backward(host, h) == host.cd.CD_EINVAL  # not a training pool
    assert host.lib.countdown_adapters_destroy(h) == 0


# ------------------------------------------------------------------ clipping

def clip_call(host, c, grads, top, norm=P["norm"]):
    words = [w for g in grads for w in g]
    return host.lib.countdown_clip_grads(c, (C.c_uint64 * max(1, len(words)))(*words), len(grads),
                                         top, norm, None)


@pytest.fixture
def clip(host):
    c = C.c_void_p()
    assert host.lib.countdown_clip_create(200, C.byref(c)) == 0
    yield c
    assert host.lib.countdown_clip_destroy(c) == 0


def test_clip_sizes(host):
    c = C.c_void_p()
    assert host.lib.countdown_clip_create(0, C.byref(c)) == host.cd.CD_EINVAL
    assert host.lib.countdown_clip_create(65537, C.byref(c)) == host.cd.CD_EUNSUPPORTED
    assert host.lib.countdown_clip_create(1, None) == host.cd.CD_EINVAL
    assert not c and host.lib.countdown_clip_destroy(None) == 0


G0, G1, O0, O1 = P["g0"], P["g1"], P["o0"], P["o1"]


@pytest.mark.parametrize("grads,top,kw", [
    ([(G0, O0, 10, 2)], 1.0, {}), ([(0, O0, 10, 0)], 1.0, {}), ([(G0, 0, 10, 0)], 1.0, {}),
    ([(G0 + 2, O0, 10, 0)], 1.0, {}), ([(G0 + 1, O0, 10, 1)], 1.0, {}),
    ([(G0, O0 + 2, 10, 0)], 1.0, {}), ([(G0, O0, 10, 0)], -0.5, {}),
    ([(G0, O0, 10, 0)], math.nan, {}), ([(G0, O0, 10, 0)], 1.0, dict(norm=P["norm"] + 4)),
    ([(G0, P["norm"], 10, 0)], 1.0, {}), ([(P["norm"], O0, 10, 0)], 1.0, {}),
    ([(G0, O0, 10, 0), (G1, O0 + 36, 10, 0)], 1.0, {}), ([(G0, G0, 10, 0)] * 2, 1.0, {}),
    ([(G0, G0 + 4, 10, 0)], 1.0, {}), ([(G0, G1, 10, 0), (G1, O1, 10, 0)], 1.0, {}),
    ([(G0, G1, 10, 0), (G1, G0, 10, 0)], 1.0, {}), ([(G0, O0, 1, 0)] * 201, 1.0, {}),
    ([(G0, G0, 10, 0), (G0, O0, 10, 0)], math.inf, dict(norm=G0)),
    ([(G0, G0, 40, 1), (G0 + 64, O0, 4, 1)], 1.0, {}),
])
def test_clip_refuses(host, clip, grads, top, kw):
    host.launches()
    assert clip_call(host, clip, grads, top, **kw) == host.cd.CD_EINVAL
    assert host.launches() == []


def test_clip_launches(host, clip):
    def kernels(*a, **kw):
        host.launches()
        assert clip_call(host, clip, *a, **kw) == 0
        return [k for k, _ in host.launches()]

    both, norm = ["k_clip_norm", "k_clip_scale"], ["k_clip_norm", "k_clip_total"]
    one, big = ["k_clip_one"], 1 << 20
    assert kernels([(G0, G0, big, 0), (G1, G1, 5, 1)], 1.0) == both
    assert kernels([(G0, G0, big, 0)], math.inf) == norm
    assert kernels([(G0, O0, big, 0)], math.inf) == both
    assert kernels([(G0, 0, big, 0)] * 2, math.inf) == norm  # the norm may count one twice
    assert kernels([], 1.0) == kernels([(0, 0, 0, 0)] * 200, 1.0) == ["k_clip_total"]
    many = [(G0 + 4096 * i, G0 + 4096 * i, 1024, 0) for i in range(200)]
    assert kernels(many, 1.0) == ["k_clip_norm"] * 3 + ["k_clip_scale"] * 3
    assert kernels(many[:33], 1.0) == both and kernels(many[:32], 1.0) == one
    assert kernels([(G0, 0, 8, 0)], math.inf) == one
    assert kernels([(G0, O0, big, 0)], 1.0, norm=None) == both
    assert kernels([(G0, O0, 8, 0)], 1.0, norm=None) == one
    assert clip_call(host, clip, [(G0, O0, (1 << 38) + 1, 0)], 1.0) == host.cd.CD_EUNSUPPORTED
    assert host.lib.countdown_clip_grads(clip, None, 1, 1.0, None, None) == host.cd.CD_EINVAL
    assert host.lib.countdown_clip_grads(None, None, 0, 1.0, None, None) == host.cd.CD_EINVAL
