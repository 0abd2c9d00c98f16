"""What the gated block's and the 4-bit calls refuse, allocate and launch, from the library's own
host code on a machine without a GPU (see host_hip.py)."""
import ctypes as C

import pytest

import host_hip

M, F, T = 264, 520, 64
F64 = -(-F // 64) * 64
P = {n: 0x100000000 * (i + 1) for i, n in enumerate(
    ("x", "dh", "Wg", "Wu", "h", "dx", "dWg", "dWu", "W", "base", "y", "codes", "scale", "packed"))}


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    return host_hip.Host(host_hip.build(str(tmp_path_factory.mktemp("host"))))


def create(host, *args):
    h = C.c_void_p()
    return host.lib.countdown_gated_create(*args, C.byref(h)), h


@pytest.fixture
def gated(host):
    st, h = create(host, M, F, T, 3)
    assert st == host.cd.CD_OK
    yield h
    assert host.lib.countdown_gated_destroy(h) == host.cd.CD_OK


def forward(host, gated, **kw):
    a = dict(x=P["x"], ldx=M, T=T, Wg=P["Wg"], Wu=P["Wu"], type=1, h=P["h"], ldh=F)
    a.update(kw)
    return host.lib.countdown_gated_forward(gated, *a.values(), None)


def backward(host, gated, **kw):
    a = dict(x=P["x"], ldx=M, dh=P["dh"], lddh=F, T=T, Wg=P["Wg"], Wu=P["Wu"], type=0, dx=P["dx"],
             lddx=M, dWg=P["dWg"], dWu=P["dWu"])
    a.update(kw)
    return host.lib.countdown_gated_backward(gated, *a.values(), None)


def project(host, **kw):
    a = dict(x=P["x"], ldx=M, T=16, W=P["W"], d_in=M, d_out=F, group=64, type=0, base=P["base"], ldb=F,
             y=P["y"], ldy=F)
    a.update(kw)
    return host.lib.countdown_q4_project(*a.values(), None)


def q4_gated(host, **kw):
    a = dict(x=P["x"], ldx=M, T=16, Wg=P["Wg"], Wu=P["Wu"], m=M, f=F, group=64, type=1, h=P["h"], ldh=F)
    a.update(kw)
    return host.lib.countdown_q4_gated(*a.values(), None)


@pytest.mark.parametrize("args,status", [
    ((8, 8, 1, 0), 0), ((65536, 65536, 1, 3), 0), ((8, 8, 1 << 20, 1), 0),
    ((0, 8, 1, 0), -1), ((12, 8, 1, 0), -1), ((8, 12, 1, 0), -1), ((8, 0, 1, 0), -1), ((8, 8, 0, 0), -1),
    ((8, 8, 1, 4), -1), ((8, 8, 1, 2), -1), ((65544, 8, 1, 0), -2), ((8, 65544, 1, 0), -2),
    ((8, 8, (1 << 20) + 1, 0), -2),
])
def test_sizes(host, args, status):
    st, h = create(host, *args)
    assert st == status and bool(h) == (status == 0)
    assert host.lib.countdown_gated_destroy(h) == 0


def test_a_failed_allocation_leaves_nothing(host):
    live = host.lib.host_hip_live_allocations()
    host.limit(1 << 20)
    try:
        st, h = create(host, M, F, T, 1)
        assert st == host.cd.CD_ENOMEM and not h
        st, h = create(host, M, F, T, 0)  # no workspace
        assert st == 0 and forward(host, h) == 0
        assert host.lib.countdown_gated_destroy(h) == 0
    finally:
        host.limit()
    assert host.lib.host_hip_live_allocations() == live


@pytest.mark.parametrize("flags,size", [(1, 4 * T * F64 + (128 << 10)), (3, 12 * T * F64)])
def test_the_workspace_takes_what_the_header_says(host, flags, size):
    most = size + (64 << 20)
    for limit, status in ((most + 256, 0), (most - 1, host.cd.CD_ENOMEM)):
        host.limit(limit)
        try:
            st, h = create(host, M, F, T, flags)
        finally:
            host.limit()
        assert st == status
        assert host.lib.countdown_gated_destroy(h) == 0


def test_calls_allocate_nothing(host, gated):
    live = host.lib.host_hip_live_allocations()
    assert forward(host, gated) == 0 and backward(host, gated) == 0
    assert project(host) == 0 and q4_gated(host) == 0
    assert host.lib.host_hip_live_allocations() == live


BAD = [
    dict(T=-1), dict(T=T + 1), dict(x=None), dict(x=P["x"] + 8), dict(ldx=M - 8), dict(ldx=M + 4),
    dict(Wg=None), dict(Wg=P["Wg"] + 2), dict(Wu=None), dict(Wu=P["Wu"] + 8), dict(type=2), dict(type=-1),
]
BAD_FORWARD = BAD + [
    dict(h=None), dict(h=P["h"] + 4), dict(ldh=F - 8), dict(ldh=F + 2), dict(h=P["x"]), dict(h=P["Wg"]),
    dict(h=P["Wu"] + 64), dict(h=P["x"] + 16, ldh=2 * F),
]
BAD_BACKWARD = BAD + [
    dict(dh=None), dict(dh=P["dh"] + 2), dict(lddh=F - 8), dict(lddh=F + 1), dict(dx=P["dx"] + 8),
    dict(lddx=M - 8), dict(lddx=M + 4), dict(dWg=P["dWg"] + 4), dict(dWu=P["dWu"] + 8), dict(dx=P["x"]),
    dict(dx=P["dh"]), dict(dx=P["Wg"]), dict(dWg=P["Wg"]), dict(dWu=P["x"] + 256), dict(dWg=P["dWu"]),
    dict(dWu=P["dWg"] + F * M * 4 - 16), dict(dx=P["dWg"] + 1024),
]


@pytest.mark.parametrize("kw", BAD_FORWARD, ids=str)
def test_forward_refuses(host, gated, kw):
    host.launches()
    assert forward(host, gated, **kw) == host.cd.CD_EINVAL
    assert host.launches() == []


@pytest.mark.parametrize("kw", BAD_BACKWARD, ids=str)
def test_backward_refuses(host, gated, kw):
    host.launches()
    assert backward(host, gated, **kw) == host.cd.CD_EINVAL
    assert host.launches() == []


FWD = ["k_gt_product<%d,16,16,", "k_gt_product<%d,32,32,", "k_gt_product<%d,64,32,", "k_gt_product<%d,64,64,",
       "k_gt_product<%d,128,64,", "k_gt_product<%d,192,64,", "k_gt_large<%d,1>", "k_gt_large<%d,2>"]


@pytest.mark.parametrize("shape,proj,dx,dw", [  # T, d_model, d_ff; the kernels by what they start with
    ((1, 256, 688), 0, "k_gt_back", None),
    ((1, 256, 1400), 0, "k_gt_product<2,64,128,", "k_gt_product<3,64,64,"),  # dg in two terms
    ((6, 256, 688), 0, "k_gt_back", None),
    ((1, 1032, 4104), 0, "k_gt_product<2,64,128,", "k_gt_product<3,128,128,"),
    ((257, 2056, 2056), 3, "k_gt_product<2,64,128,", "k_gt_large<3,2>"),
    ((300, 2104, 2600), 3, "k_gt_product<2,64,128,", "k_gt_large<3,2>"),
    ((16, 4096, 14336), 0, "k_gt_product<2,64,128,", "k_gt_product<3,128,128,"),
    ((17, 256, 688), 1, "k_gt_back", None),
    ((4000, 128, 512), 4, "k_gt_product<2,64,128,", "k_gt_product<3,64,64,"),  # tokens shared
    ((2048, 128, 512), 3, "k_gt_back", None),
    ((655, 1336, 6976), 7, "k_gt_product<2,64,128,", "k_gt_product<3,128,128,"),
    ((17, 256, 2056), 1, "k_gt_product<2,64,128,", "k_gt_product<3,64,64,"),
    ((100, 200, 2200), 2, "k_gt_product<2,64,128,", "k_gt_product<3,64,64,"),
    ((200, 136, 3000), 3, "k_gt_product<2,64,128,", "k_gt_product<3,64,64,"),
    ((500, 72, 3000), 4, "k_gt_product<2,64,128,", "k_gt_product<3,64,64,"),
    ((700, 72, 3504), 5, "k_gt_product<2,64,128,", "k_gt_product<3,64,64,"),
    ((900, 72, 4000), 6, "k_gt_product<2,64,128,", "k_gt_product<3,64,64,"),
    ((48, 1032, 16640), 3, "k_gt_product<2,64,128,", "k_gt_product<3,128,128,"),  # more than 256 tiles
    ((384, 72, 16640), 6, "k_gt_product<2,64,128,", "k_gt_product<3,128,128,"),
    ((2000, 264, 4104), 7, "k_gt_product<2,64,128,", "k_gt_product<3,128,128,"),
    ((1300, 1544, 2056), 5, "k_gt_large<2,2>", "k_gt_product<3,128,128,"),
    ((70, 1032, 4104), 3, "k_gt_product<2,64,128,", "k_gt_product<3,128,128,"),
    ((8192, 4096, 14336), 7, "k_gt_large<2,2>", "k_gt_large<3,2>"),
], ids=str)
def test_kernels_by_the_sizes(host, shape, proj, dx, dw):
    T, m, f = shape
    st, h = create(host, m, f, T, 1)
    assert st == 0
    host.launches()
    far = dict(ldx=m, T=T, Wg=P["Wg"], Wu=P["Wu"])
    assert forward(host, h, ldh=f, **far) == 0
    assert [k.startswith(FWD[proj] % 0) for k, _ in host.launches()] == [True]
    assert backward(host, h, lddh=f, lddx=m, type=1, **far) == 0
    got = [k for k, _ in host.launches() if not k.startswith("k_gt_sum")]
    assert host.lib.countdown_gated_destroy(h) == 0
    assert [k.startswith(w) for k, w in zip(got, (FWD[proj] % 1, dx, dw) if dw else (FWD[proj] % 1, dx))] == \
        [True] * (3 if dw else 2), got


def test_strides_past_what_the_kernels_reach(host, gated):
    big = (1 << 20) + 8
    host.launches()
    assert forward(host, gated, ldx=big) == host.cd.CD_EUNSUPPORTED
    assert backward(host, gated, ldx=big) == host.cd.CD_EUNSUPPORTED
    assert backward(host, gated, lddh=big) == host.cd.CD_EUNSUPPORTED
    assert host.launches() == []
    assert forward(host, gated, ldx=big - 8, ldh=1 << 22) == 0


def test_what_a_handle_was_made_for(host):
    for flags, kinds in ((0, ()), (1, (1,)), (3, (0, 1))):
        st, h = create(host, M, F, T, flags)
        assert st == 0 and forward(host, h) == 0 and forward(host, h, type=0) == 0
        for kind in (0, 1):
            assert backward(host, h, type=kind) == (0 if kind in kinds else host.cd.CD_EINVAL)
        assert host.lib.countdown_gated_destroy(h) == 0
    assert forward(host, None) == host.cd.CD_EINVAL and backward(host, None) == host.cd.CD_EINVAL


def test_empty_calls(host, gated):
    host.launches()
    none = dict(T=0, x=None, ldx=0)
    assert forward(host, gated, h=None, ldh=0, **none) == 0
    assert project(host, base=None, y=None, **none) == 0 and q4_gated(host, h=None, **none) == 0
    assert host.launches() == []
    assert backward(host, gated, dh=None, dx=None, **none) == 0
    assert [k for k, _ in host.launches()] == ["k_gt_zero", "k_gt_zero"]
    assert backward(host, gated, dx=None, dWg=None, dWu=None) == 0
    assert host.launches() == []


@pytest.mark.parametrize("shape,status", [
    ((8, 8, 32), 0), ((65536, 65536, 128), 0), ((0, 8, 32), -1), ((8, 0, 32), -1), ((12, 8, 32), -1),
    ((8, 12, 32), -1), ((8, 8, 0), -1), ((8, 8, 16), -1), ((8, 8, 256), -1), ((65544, 8, 64), -2),
    ((8, 65544, 64), -2),
])
def test_q4_sizes(host, shape, status):
    rows, cols, group = shape
    lib, packed = host.lib, P["packed"]
    n = lib.countdown_q4_bytes(*shape)
    assert n == (0 if status else -(-rows // 16) * -(-cols // 128) * (1024 + 4096 // group))
    host.launches()
    assert lib.countdown_q4_quantize(P["W"], cols, *shape, packed, None) == status
    assert lib.countdown_q4_pack(P["codes"], P["scale"], *shape, packed, None) == status
    assert lib.countdown_q4_unpack(packed, *shape, P["W"], cols, None) == status
    assert project(host, d_out=rows, d_in=cols, group=group, ldx=cols, ldb=rows, ldy=rows) == status
    assert q4_gated(host, f=rows, m=cols, group=group, ldx=cols, ldh=rows) == status
    assert (len(host.launches()) == 5) == (status == 0)


BAD_Q4 = [dict(T=-1), dict(x=None), dict(x=P["x"] + 2), dict(ldx=M - 8), dict(ldx=M + 4), dict(type=2),
          dict(group=48)]


@pytest.mark.parametrize("kw", BAD_Q4 + [
    dict(W=None), dict(W=P["W"] + 8), dict(y=None), dict(y=P["y"] + 8), dict(ldy=F - 8), dict(ldy=F + 4),
    dict(base=P["base"] + 4), dict(ldb=F - 8), dict(y=P["x"]), dict(y=P["W"] + 1024), dict(y=P["base"] + 32),
    dict(y=P["base"], ldy=F + 8),
], ids=str)
def test_q4_project_refuses(host, kw):
    host.launches()
    assert project(host, **kw) == host.cd.CD_EINVAL
    assert host.launches() == []


@pytest.mark.parametrize("kw", BAD_Q4 + [
    dict(Wg=None), dict(Wu=None), dict(Wg=P["Wg"] + 8), dict(Wu=P["Wu"] + 8), dict(h=None), dict(h=P["h"] + 8),
    dict(ldh=F - 8), dict(h=P["x"]), dict(h=P["Wg"]), dict(h=P["Wu"] + 64),
], ids=str)
def test_q4_gated_refuses(host, kw):
    host.launches()
    assert q4_gated(host, **kw) == host.cd.CD_EINVAL
    assert host.launches() == []


def test_q4_more_tokens(host):
    assert project(host, T=17) == host.cd.CD_EUNSUPPORTED and q4_gated(host, T=17) == host.cd.CD_EUNSUPPORTED
    assert project(host, y=P["base"]) == 0  # in place


def test_q4_weights_refuse(host):
    lib, shape, bad = host.lib, (F, M, 64), host.cd.CD_EINVAL
    host.launches()
    for W, ldw, packed in ((None, M, P["packed"]), (P["W"] + 2, M, P["packed"]), (P["W"], M - 8, P["packed"]),
                           (P["W"], M + 4, P["packed"]), (P["W"], M, None), (P["W"], M, P["packed"] + 8),
                           (P["W"], M, P["W"] + 1024)):
        assert lib.countdown_q4_quantize(W, ldw, *shape, packed, None) == bad
        assert lib.countdown_q4_unpack(packed, *shape, W, ldw, None) == bad
    for codes, scale, packed in ((None, P["scale"], P["packed"]), (P["codes"], None, P["packed"]),
                                 (P["codes"] + 8, P["scale"], P["packed"]), (P["codes"], P["scale"] + 2, P["packed"]),
                                 (P["codes"], P["scale"], None), (P["codes"], P["scale"], P["scale"]),
                                 (P["codes"], P["scale"], P["codes"] + 4096)):
        assert lib.countdown_q4_pack(codes, scale, *shape, packed, None) == bad
    assert host.launches() == []
