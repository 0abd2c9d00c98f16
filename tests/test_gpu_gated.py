"""The gated block and its backward pass against the definition in 64 bits.

Tolerances. A sum of n products accumulated in fp32 in any order is off by at most n * u times the
sum of the terms' magnitudes, u = 2^-23 (each addition by at most one unit in the last place); eight
more for the roundings beside it. With eg and eu so bounded for g and u:
  |SiLU'| <= 1.1, |SiLU''| <= 0.5, so h is off by 1.1 eg |u| + (|SiLU(g)| + 1.1 eg) eu, and by
  sixteen u of itself for exp, the division and the products (exp's relative error includes that of
  its argument's rounding, none here: the argument is g itself);
  du = dh SiLU(g) by |dh| 1.1 eg and sixteen u |du|;
  dg = dh u SiLU'(g) by |dh| (1.1 eu + 0.5 |u| eg) and 16 u |dh u| (1 + |g|) s (s (1 + g (1 - s)) is a
  difference of its two terms where g < 0).
What an operand is off enters a product times the other operand's magnitude. dg and du rounded to
bf16 (bf16 gradients) are off by half a step, 2^-8 of themselves, more; held in two bf16 terms (T d_ff <= 4096),
the first cut and the second rounded, by 2^-7 2^-8 / 2 = 2^-16. A result is rounded once to its type."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -23
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def cd():
    from paper_2505_17701_amd import binding

    return binding


class Case:
    def __init__(self, T, m, f, seed=1, sigma=None):
        g = torch.Generator(device="cuda").manual_seed(seed)
        sigma = sigma or 1.3 / m ** 0.5

        def rand(*shape, s=1.0):
            return (torch.randn(shape, generator=g, device="cuda") * s).to(BF16)

        self.T, self.m, self.f = T, m, f
        self.x, self.Wg, self.Wu = rand(T, m), rand(f, m, s=sigma), rand(f, m, s=sigma)
        self.dh = rand(T, f, s=0.1)

    def parts(self):
        x, Wg, Wu = self.x.double(), self.Wg.double(), self.Wu.double()
        g, u = x @ Wg.t(), x @ Wu.t()
        e = (self.m + 8) * U
        return g, u, e * (x.abs() @ Wg.abs().t()), e * (x.abs() @ Wu.abs().t())

    def h(self):
        """(h, bound of its error before the last rounding)"""
        g, u, eg, eu = self.parts()
        silu = g * torch.sigmoid(g)
        h = silu * u
        return h, 1.1 * eg * u.abs() + (silu.abs() + 1.1 * eg) * eu + 16 * U * h.abs()

    def grads(self, dtype):
        """{name: (value, bound)} of gradients of this type"""
        step = 0.0 if dtype is F32 else 2.0 ** -16 if self.T * self.f <= 4096 else 2.0 ** -8
        g, u, eg, eu = self.parts()
        x, Wg, Wu, dh = self.x.double(), self.Wg.double(), self.Wu.double(), self.dh.double()
        s = torch.sigmoid(g)
        slope = s * (1 + g * (1 - s))
        dg, du = dh * u * slope, dh * g * s
        tg = dh.abs() * (1.1 * eu + 0.5 * (u.abs() + eu) * eg + 16 * U * u.abs() * (1 + g.abs()) * s)
        tu = dh.abs() * 1.1 * eg + 16 * U * du.abs()
        tg = tg + step * (dg.abs() + tg)
        tu = tu + step * (du.abs() + tu)
        ag, au = dg.abs() + tg, du.abs() + tu
        n = 3  # products of a pair of elements, at most
        ex, ew = (2 * n * self.f + 64 + 8) * U, (n * self.T + 8) * U
        return {
            "dx": (dg @ Wg + du @ Wu,
                   tg @ Wg.abs() + tu @ Wu.abs() + ex * (ag @ Wg.abs() + au @ Wu.abs())),
            "dW_gate": (dg.t() @ x, tg.t() @ x.abs() + ew * (ag.t() @ x.abs())),
            "dW_up": (du.t() @ x, tu.t() @ x.abs() + ew * (au.t() @ x.abs())),
        }


def check(got, ref, bound, name=""):
    tol = bound + torch.finfo(got.dtype).eps / 2 * (ref.abs() + bound) + 1e-37
    over = (got.double() - ref).abs() - tol
    assert not bool(torch.isnan(over).any()), name
    assert float(over.max()) <= 0, \
        f"{name}: {int((over > 0).sum())} of {over.numel()} off, worst by {float(over.max()):.3e}"


SHAPES = [  # T, d_model, d_ff: every tile, its edges, one element of a tile, whole tiles
    (1, 8, 8), (1, 64, 64), (3, 264, 1360), (1, 256, 688), (2, 1000, 72), (7, 264, 8), (16, 4096, 520), (17, 72, 1000), (31, 520, 264),
    (32, 256, 512), (33, 136, 200), (64, 512, 256), (65, 1032, 136), (129, 64, 328), (256, 200, 64),
    (257, 328, 712), (300, 1000, 264), (512, 256, 512), (777, 264, 1032), (1025, 520, 136),
    (1300, 1544, 2056), (2048, 512, 1024), (4100, 72, 136),
    # tiles of the projections by how many workgroups they make (test_host_gated_q4.py names them)
    (100, 200, 2200), (200, 136, 3000), (500, 72, 3000), (700, 72, 3504), (900, 72, 4000), (2000, 264, 4104),
    (384, 72, 16640), (20, 72, 16400), (48, 1032, 16640),
    # dx in one part; the gradients of the weights in 256 x 256 tiles, of few and of many tokens
    (4100, 2104, 72), (70, 1032, 4104), (300, 2104, 2600), (257, 2056, 2056), (1, 1032, 4104),
    (4392, 168, 72), (1024, 256, 256), (1100, 8, 8), (655, 1336, 2000), (17, 264, 2056), (17, 264, 1032), (4000, 128, 512), (65, 520, 1000),  # launches of their own; one for dx and the weights' gradients
]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(cd, shape, dtype):
    c = Case(*shape)
    h = torch.empty((c.T, c.f), dtype=dtype, device="cuda")
    with cd.Gated(c.m, c.f, max_tokens=c.T) as p:
        assert cd.countdown_gated_forward(p, c.x, c.Wg, c.Wu, h=h) is h
    check(h, *c.h(), "h")


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_backward(cd, shape, dtype):
    c = Case(*shape)
    with cd.Gated(c.m, c.f, max_tokens=c.T + 3, train=True, fp32_grads=dtype is F32) as p:
        got = cd.countdown_gated_backward(p, c.x, c.dh, c.Wg, c.Wu)
    for g, (name, (ref, bound)) in zip(got, c.grads(dtype).items()):
        assert g.dtype is dtype
        check(g, ref, bound, name)


def test_gradients_against_differences(cd):
    """<dh, h> of inputs moved by t in a random direction, in 64 bits."""
    c = Case(40, 72, 136, seed=3)
    g = torch.Generator(device="cuda").manual_seed(9)
    with cd.Gated(c.m, c.f, c.T, train=True, fp32_grads=True) as p:
        got = cd.countdown_gated_backward(p, c.x, c.dh, c.Wg, c.Wu)
    args = [c.x.double(), c.Wg.double(), c.Wu.double()]

    def loss(x, Wg, Wu):
        a = x @ Wg.t()
        return (c.dh.double() * a * torch.sigmoid(a) * (x @ Wu.t())).sum()

    for i in range(3):
        way = torch.randn(args[i].shape, generator=g, device="cuda", dtype=torch.float64)
        t = 1e-5
        lo, hi = list(args), list(args)
        lo[i], hi[i] = args[i] - t * way, args[i] + t * way
        slope = (loss(*hi) - loss(*lo)) / (2 * t)  # off by t^2 times a third derivative, and 1e-16 |loss| / t
        mag = (got[i].double() * way).abs().sum()
        assert abs(float((got[i].double() * way).sum() - slope)) <= 1e-6 * float(mag)


@pytest.mark.parametrize("need", [(True, False, False), (False, True, False), (False, False, True),
                                  (False, True, True), (True, False, True), (False, False, False)], ids=str)
@pytest.mark.parametrize("shape", [(5, 264, 136), (300, 264, 712), (1024, 512, 1032)], ids=str)
def test_a_gradient_alone_has_the_same_bits(cd, shape, need):
    c = Case(*shape)
    with cd.Gated(c.m, c.f, c.T, train=True, fp32_grads=True) as p:
        for dtype in (BF16, F32):
            whole = cd.countdown_gated_backward(p, c.x, c.dh, c.Wg, c.Wu, dtype=dtype)
            some = cd.countdown_gated_backward(p, c.x, c.dh, c.Wg, c.Wu, dtype=dtype, need=need)
            for n, a, b in zip(need, whole, some):
                assert torch.equal(a, b) if n else b is None


def sliced(t, extra=16, fill=7.0):
    """t as a column slice of a wider tensor"""
    wide = torch.full((t.shape[0] + 2, t.shape[1] + 2 * extra), fill, dtype=t.dtype, device="cuda")
    view = wide[1:-1, extra:-extra]
    view.copy_(t)
    return wide, view


@pytest.mark.parametrize("shape", [(3, 264, 136), (20, 72, 264), (200, 136, 72), (700, 264, 520)], ids=str)
def test_strides_leave_the_rest(cd, shape):
    c = Case(*shape)
    for dtype in (BF16, F32):
        with cd.Gated(c.m, c.f, c.T, train=True, fp32_grads=True) as p:
            h = torch.empty((c.T, c.f), dtype=dtype, device="cuda")
            cd.countdown_gated_forward(p, c.x, c.Wg, c.Wu, h=h)
            want = cd.countdown_gated_backward(p, c.x, c.dh, c.Wg, c.Wu, dtype=dtype)
            _, x = sliced(c.x, fill=float("nan"))
            _, dh = sliced(c.dh, 24, float("nan"))
            hw, hv = sliced(torch.zeros_like(h))
            dxw, dxv = sliced(torch.zeros_like(want[0]), 8)
            cd.countdown_gated_forward(p, x, c.Wg, c.Wu, h=hv)
            got = cd.countdown_gated_backward(p, x, dh, c.Wg, c.Wu, dx=dxv)
        assert torch.equal(hv, h)
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        for wide, view, e in ((hw, hv, 16), (dxw, dxv, 8)):
            view.fill_(7.0)
            assert bool((wide == 7.0).all())


@pytest.mark.parametrize("T", [4, 40, 300])
def test_bad_numbers_stay_with_their_token_and_neuron(cd, T):
    c = Case(T, 264, 200)
    with cd.Gated(c.m, c.f, T, train=True, fp32_grads=True) as p:
        h = cd.countdown_gated_forward(p, c.x, c.Wg, c.Wu)
        dx, dWg, dWu = cd.countdown_gated_backward(p, c.x, c.dh, c.Wg, c.Wu)
        for bad in (float("nan"), float("inf"), -float("inf")):
            x, Wg = c.x.clone(), c.Wg.clone()
            x[T // 2, 5] = bad
            Wg[77, 3] = bad
            h2 = cd.countdown_gated_forward(p, x, Wg, c.Wu)
            hit = torch.zeros_like(h2, dtype=torch.bool)
            hit[T // 2], hit[:, 77] = True, True
            assert torch.equal(h2[~hit], h[~hit])
            assert not bool(torch.isfinite(h2[hit].float()).any())
            dh = c.dh.clone()
            dh[T // 2, 9] = bad
            got = cd.countdown_gated_backward(p, c.x, dh, c.Wg, c.Wu)
            assert not bool(torch.isfinite(got[0][T // 2]).any())
            rest = torch.arange(T, device="cuda") != T // 2
            assert torch.equal(got[0][rest], dx[rest])
            rows = torch.arange(c.f, device="cuda") != 9
            assert torch.equal(got[1][rows], dWg[rows]) and torch.equal(got[2][rows], dWu[rows])
            assert not bool(torch.isfinite(got[1][9]).any()) and not bool(torch.isfinite(got[2][9]).any())


def test_large_gates(cd):
    """SiLU and its slope where exp overflows or vanishes: h = g u or 0, no NaN."""
    m, f = 64, 64
    x = torch.zeros((8, m), device="cuda")
    x[:, 0] = torch.tensor([-1e30, -200.0, -95.0, -50.0, 50.0, 95.0, 200.0, 1e30])
    x[:, 1] = 2.0
    W = torch.zeros((f, m), device="cuda")
    V = torch.zeros((f, m), device="cuda")
    W[:, 0], V[:, 1] = 1.0, 0.5
    x, W, V = x.to(BF16), W.to(BF16), V.to(BF16)
    dh = torch.ones((8, f), device="cuda", dtype=BF16)
    with cd.Gated(m, f, 8, train=True, fp32_grads=True) as p:
        h = cd.countdown_gated_forward(p, x, W, V, h=torch.empty((8, f), device="cuda"))
        dx, _, _ = cd.countdown_gated_backward(p, x, dh, W, V)
    g = x[:, 0].double()
    s = torch.sigmoid(g)
    assert torch.allclose(h.double(), (g * s)[:, None].expand(8, f), rtol=1e-5, atol=1e-30)
    want = f * torch.where(s == 0, 0.0, s * (1 + g * (1 - s)))  # u = 1
    assert torch.allclose(dx[:, 0].double(), want, rtol=1e-5, atol=1e-30)


def test_gates_next_to_the_largest_number(cd):
    """h = g u or 0 and the slope 1 or 0 where g times a constant would overflow."""
    x = torch.zeros((4, 64), device="cuda")
    x[:, 0] = torch.tensor([3.3e38, -3.3e38, 1e38, -1e38])
    x[:, 1] = 2.0 ** -100
    W, V = torch.zeros((8, 64), device="cuda"), torch.zeros((8, 64), device="cuda")
    W[:, 0], V[:, 1] = 1.0, 1.0
    x, W, V = x.to(BF16), W.to(BF16), V.to(BF16)
    dh = torch.ones((4, 8), device="cuda", dtype=BF16)
    with cd.Gated(64, 8, 4, train=True, fp32_grads=True) as p:
        h = cd.countdown_gated_forward(p, x, W, V, h=torch.empty((4, 8), device="cuda"))
        dx, _, _ = cd.countdown_gated_backward(p, x, dh, W, V)
    open_ = (x[:, 0] > 0).double()
    want = open_ * x[:, 0].double() * 2.0 ** -100
    assert bool(((h.double() - want[:, None]).abs() <= 2.0 ** -21 * want[:, None]).all())
    assert bool(((dx[:, 0].double() - 8 * open_ * 2.0 ** -100).abs() <= 2.0 ** -20 * 2.0 ** -100).all())


def test_empty_call(cd):
    with cd.Gated(64, 136, 4, train=True) as p:
        x = torch.empty((0, 64), dtype=BF16, device="cuda")
        dh = torch.empty((0, 136), dtype=BF16, device="cuda")
        W = torch.ones((136, 64), dtype=BF16, device="cuda")
        V = torch.ones((136, 64), dtype=BF16, device="cuda")
        assert cd.countdown_gated_forward(p, x, W, V).shape == (0, 136)
        dx, dWg, dWu = cd.countdown_gated_backward(
            p, x, dh, W, V, dW_gate=torch.ones_like(W), dW_up=torch.ones_like(W))
        assert dx.shape == (0, 64) and not bool(dWg.any()) and not bool(dWu.any())


@pytest.mark.parametrize("T,m,f", [(3, 264, 520), (40, 256, 688), (600, 264, 520)])
def test_graph_replays_with_other_values(cd, T, m, f):
    c = [Case(T, m, f, seed=s) for s in (1, 2, 3)]
    x, dh, Wg, Wu = (t.clone() for t in (c[0].x, c[0].dh, c[0].Wg, c[0].Wu))
    with cd.Gated(m, f, T, train=True, fp32_grads=True) as p, cd.Gated(m, f, T, train=True, fp32_grads=True) as q:
        h = torch.empty((T, f), dtype=BF16, device="cuda")
        grads = [torch.empty(s, device="cuda") for s in ((T, m), (f, m), (f, m))]
        cd.countdown_gated_backward(p, x, dh, Wg, Wu, *grads)  # warm
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cd.countdown_gated_forward(p, x, Wg, Wu, h=h)
            cd.countdown_gated_backward(p, x, dh, Wg, Wu, *grads)
        for k in c + c[:1]:
            for a, b in zip((x, dh, Wg, Wu), (k.x, k.dh, k.Wg, k.Wu)):
                a.copy_(b)
            for t in grads + [h]:
                t.fill_(float("nan"))
            graph.replay()
            # another handle's eager call between the replays
            want = cd.countdown_gated_backward(q, k.x, k.dh, k.Wg, k.Wu)
            torch.cuda.synchronize()
            assert torch.equal(h, cd.countdown_gated_forward(q, k.x, k.Wg, k.Wu))
            for a, b in zip(grads, want):
                assert torch.equal(a, b)


def test_two_handles_on_two_streams(cd):
    c = [Case(500, 520, 712, seed=s) for s in (1, 2)]
    with cd.Gated(520, 712, 500, train=True) as p, cd.Gated(520, 712, 500, train=True) as q:
        want = [cd.countdown_gated_backward(p, k.x, k.dh, k.Wg, k.Wu) for k in c]
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in c]
        got = [[], []]
        for _ in range(8):
            for i, (s, h) in enumerate(zip(streams, (p, q))):
                with torch.cuda.stream(s):
                    got[i].append(cd.countdown_gated_backward(h, c[i].x, c[i].dh, c[i].Wg, c[i].Wu))
        torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(g, want[i]))


def test_a_stream_of_the_caller(cd):
    c = Case(100, 264, 520)
    with cd.Gated(264, 520, 100) as p:
        want = cd.countdown_gated_forward(p, c.x, c.Wg, c.Wu)
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        h = torch.empty_like(want)
        cd.countdown_gated_forward(p, c.x, c.Wg, c.Wu, h=h, stream=s)
        s.synchronize()
        assert torch.equal(h, want)


def test_rows_past_32_bits(cd):
    """Tokens whose rows lie past 2^32 bytes from the first (a wide row stride)."""
    T, m, f, ld = 2100, 64, 72, 1 << 20
    c = Case(T, m, f)
    wide = torch.empty((T, ld), dtype=BF16, device="cuda")  # 4.4 GB
    x = wide[:, 8:8 + m]
    x.copy_(c.x)
    with cd.Gated(m, f, T, train=True) as p:
        assert torch.equal(cd.countdown_gated_forward(p, x, c.Wg, c.Wu),
                           cd.countdown_gated_forward(p, c.x, c.Wg, c.Wu))
        for a, b in zip(cd.countdown_gated_backward(p, x, c.dh, c.Wg, c.Wu),
                        cd.countdown_gated_backward(p, c.x, c.dh, c.Wg, c.Wu)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("m", [8, 56, 64, 72, 80, 96, 144, 200, 1000])
@pytest.mark.parametrize("T,f,at", [(200, 5504, 0), (200, 5504, 24), (40, 2056, 0), (60, 4104, 8), (333, 8008, 0), (333, 8008, 40)])
def test_rows_that_begin_inside_a_cache_line(cd, m, T, f, at):
    c = Case(T, m, f)
    wide = torch.full((T, m + 64), float("nan"), dtype=BF16, device="cuda")
    x = wide[:, at:at + m]
    x.copy_(c.x)
    with cd.Gated(m, f, T, train=True) as p:
        h = cd.countdown_gated_forward(p, x, c.Wg, c.Wu, h=torch.empty((T, f), device="cuda"))
        check(h, *c.h(), "h")
        for g, (name, (ref, bound)) in zip(cd.countdown_gated_backward(p, x, c.dh, c.Wg, c.Wu), c.grads(BF16).items()):
            check(g, ref, bound, name)


def test_weights_that_begin_inside_a_cache_line(cd):
    c = Case(333, 192, 8008)
    flat = torch.full((2 * 192 * 8008 + 64,), float("nan"), dtype=BF16, device="cuda")
    n = 192 * 8008
    Wg, Wu = flat[8:8 + n].view(8008, 192), flat[n + 32:2 * n + 32].view(8008, 192)  # by 16 and by 64 bytes
    Wg.copy_(c.Wg), Wu.copy_(c.Wu)
    with cd.Gated(192, 8008, 333) as p:
        check(cd.countdown_gated_forward(p, c.x, Wg, Wu, h=torch.empty((333, 8008), device="cuda")), *c.h(), "h")


def test_tokens_past_32_bits(cd):
    """h, dg and du of more than 2^32 bytes, against the last tokens alone."""
    T, m, f, n = 131080, 64, 8200, 300  # T 2 f > 2^31 elements
    last = Case(n, m, f)
    x = torch.randn((T, m), device="cuda").to(BF16)
    dh = torch.zeros((T, f), dtype=BF16, device="cuda")
    x[-n:], dh[-n:] = last.x, last.dh
    with cd.Gated(m, f, T, train=True) as p:
        h = cd.countdown_gated_forward(p, x, last.Wg, last.Wu, h=torch.empty((T, f), device="cuda"))
        check(h[-n:], *last.h(), "h")
        del h
        dx, dWg, dWu = cd.countdown_gated_backward(p, x, dh, last.Wg, last.Wu)
    assert not bool(dx[:-n].any())
    # the other tokens add zeros to the weights' gradients: the sum of n tokens, in whatever order
    for got, (name, (ref, bound)) in zip((dx[-n:], dWg, dWu), last.grads(BF16).items()):
        check(got, ref, bound, name)


def test_largest_matrices(cd):
    """65536 x 65536: 2^33 bytes a matrix; the last neurons, whose dh alone is not zero."""
    T, m, n = 3, 65536, 64
    f = m
    last = Case(T, m, n)
    Wg = torch.randn((f, m), dtype=BF16, device="cuda").mul_(0.005)
    Wu = torch.randn((f, m), dtype=BF16, device="cuda").mul_(0.005)
    Wg[-n:], Wu[-n:] = last.Wg, last.Wu
    dh = torch.zeros((T, f), dtype=BF16, device="cuda")
    dh[:, -n:] = last.dh
    with cd.Gated(m, f, T, train=True) as p:
        h = cd.countdown_gated_forward(p, last.x, Wg, Wu, h=torch.empty((T, f), device="cuda"))
        check(h[:, -n:], *last.h(), "h")
        dx, dWg, dWu = cd.countdown_gated_backward(p, last.x, dh, Wg, Wu)
    assert not bool(dWg[:-n].any()) and not bool(dWu[:-n].any())
    last.f = f  # (T d_ff > 4096: one bf16 term; and as many products for dx)
    for got, (name, (ref, bound)) in zip((dx, dWg[-n:], dWu[-n:]), last.grads(BF16).items()):
        check(got, ref, bound, name)


def test_binding_refusals(cd):
    c = Case(4, 64, 72)
    with cd.Gated(64, 72, 4) as p, cd.Gated(64, 72, 4, train=True) as q:
        def forward(**kw):
            return cd.countdown_gated_forward(**{**dict(gated=p, x=c.x, W_gate=c.Wg, W_up=c.Wu), **kw})

        def backward(**kw):
            return cd.countdown_gated_backward(
                **{**dict(gated=q, x=c.x, dh=c.dh, W_gate=c.Wg, W_up=c.Wu), **kw})

        forward(), backward()
        f32 = torch.zeros((4, 72), device="cuda")
        for bad, error in [
            (dict(x=c.x.float()), TypeError), (dict(x=c.x[:, :56]), ValueError), (dict(x=c.x.cpu()), ValueError),
            (dict(W_gate=c.Wg.float()), TypeError), (dict(W_up=c.Wu[:64]), ValueError),
            (dict(W_up=c.Wu.t().contiguous().t()), ValueError), (dict(h=f32.double()), TypeError),
            (dict(h=f32[:3]), ValueError), (dict(x=c.x.repeat(2, 1)), cd.CountdownError),
        ]:
            with pytest.raises(error):
                forward(**bad)
        for bad, error in [
            (dict(gated=p), cd.CountdownError),  # made without train
            (dict(dh=f32), TypeError), (dict(dh=c.dh[:, :64]), ValueError),
            (dict(dtype=F32), cd.CountdownError),  # made without fp32_grads
            (dict(dtype=torch.float16), TypeError),
            (dict(dx=torch.empty((4, 64), dtype=BF16, device="cuda"), dtype=F32), TypeError),
            (dict(dW_gate=torch.empty((72, 64), dtype=BF16, device="cuda"),
                  dW_up=torch.empty((72, 64), device="cuda")), TypeError),
            (dict(dW_gate=c.Wg), cd.CountdownError), (dict(dx=c.x), cd.CountdownError),
            (dict(dW_gate=torch.empty((64, 72), dtype=BF16, device="cuda")), ValueError),
        ]:
            with pytest.raises(error):
                backward(**bad)
        closed = cd.Gated(64, 72, 4)
        closed.close()
        with pytest.raises(ValueError):
            forward(gated=closed)
