"""4-bit weights with group scales against the definition in 64 bits.

Tolerances, u = 2^-23. A code enters as 24 + c, the group's sum starts from -24 times the sum of its
x: over a group of G columns 2 G additions over magnitudes up to (24 + 8 + 24) |x| sum(scale), then one product
and one addition a group. So y is off by (2 G + 8) u * 56 * S + (groups + 8 + 8) u * Y with
S = sum |scale| |x| and Y = sum |scale| |code| |x| (the waves' eight parts, the base). h as in the
gated block: 1.1 eg |u| + (|SiLU(g)| + 1.1 eg) eu + 16 u |h|. A result is rounded once to its type."""
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


def wide(scale, group, cols):
    return scale.repeat_interleave(group, dim=1)[:, :cols]


class Matrix:
    def __init__(self, g, rows, cols, group):
        self.group = group
        self.codes = torch.randint(-8, 8, (rows, cols), generator=g, device="cuda", dtype=torch.int8)
        self.scale = ((torch.rand((rows, -(-cols // group)), generator=g, device="cuda") - 0.3) * 0.1).to(BF16)

    def dense(self):
        return self.codes.double() * wide(self.scale.double(), self.group, self.codes.shape[1])

    def pack(self, cd):
        return cd.countdown_q4_pack(self.codes, self.scale, self.group)

    def product(self, x):
        """(x W^T, bound of its error)"""
        x, w = x.double(), self.dense()
        s = x.abs() @ wide(self.scale.double().abs(), self.group, x.shape[1]).t()
        e = (2 * self.group + 8) * U * 56 * s + (self.scale.shape[1] + 16) * U * (x.abs() @ w.abs().t())
        return x @ w.t(), e


def check(got, ref, bound, name=""):
    tol = bound + torch.finfo(got.dtype).eps / 2 * (ref.abs() + bound) + 1e-37
    over = (got.double() - ref).abs() - tol
    assert not bool(torch.isnan(over).any()), name
    assert float(over.max()) <= 0, \
        f"{name}: {int((over > 0).sum())} of {over.numel()} off, worst by {float(over.max()):.3e}"


def rng(seed=1):
    return torch.Generator(device="cuda").manual_seed(seed)


def tokens(g, T, cols):
    return torch.randn((T, cols), generator=g, device="cuda").to(BF16)


SHAPES = [  # tokens, rows, cols: padded rows and columns, one block, several columns' chunks in LDS
    (1, 8, 8), (1, 16, 128), (2, 24, 136), (3, 256, 688), (16, 688, 256), (5, 40, 1000), (13, 1000, 3000),
    (1, 72, 4096), (16, 136, 4104), (7, 520, 11008), (16, 64, 14336), (1, 32, 33000), (2, 64, 65536),
    (16, 48, 28672), (11, 4096, 72),
]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_project(cd, shape, group):
    T, rows, cols = shape
    g = rng()
    W, x = Matrix(g, rows, cols, group), tokens(g, T, cols)
    q = W.pack(cd)
    ref, bound = W.product(x)
    check(cd.countdown_q4_project(x, q), ref, bound, "fp32")
    check(cd.countdown_q4_project(x, q, y=torch.empty((T, rows), dtype=BF16, device="cuda")), ref, bound, "bf16")
    for dtype in (F32, BF16):
        base = torch.randn((T, rows), generator=g, device="cuda").to(dtype)
        want = ref + base.double(), bound + U * (ref.abs() + base.double().abs())
        check(cd.countdown_q4_project(x, q, base=base), *want, "base")
        y = base.clone()
        assert cd.countdown_q4_project(x, q, base=y, y=y) is y  # in place
        check(y, *want, "in place")


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_gated(cd, shape, group):
    T, rows, cols = shape
    g = rng(2)
    Wg, Wu, x = Matrix(g, rows, cols, group), Matrix(g, rows, cols, group), tokens(g, T, cols)
    (a, ea), (u, eu) = Wg.product(x), Wu.product(x)
    silu = a * torch.sigmoid(a)
    bound = 1.1 * ea * u.abs() + (silu.abs() + 1.1 * ea) * eu + 16 * U * (silu * u).abs()
    for dtype in (F32, BF16):
        h = torch.empty((T, rows), dtype=dtype, device="cuda")
        cd.countdown_q4_gated(x, Wg.pack(cd), Wu.pack(cd), h=h)
        check(h, silu * u, bound, "h")


@pytest.mark.parametrize("T,rows", [(5, 6152), (9, 8008)])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_two_row_tiles_of_an_odd_number(cd, T, rows, group):
    g = rng(3)
    W, x = Matrix(g, rows, 712, group), tokens(g, T, 712)
    check(cd.countdown_q4_project(x, W.pack(cd)), *W.product(x), "y")


def test_largest_matrices(cd):
    """65536 x 65536: the last rows, past 2^31 bytes of the packed matrix."""
    n, rows, cols, group = 48, 65536, 65536, 128
    g = rng(4)
    last, x = Matrix(g, n, cols, group), tokens(g, 16, cols)
    W = Matrix(g, rows, cols, group)
    W.codes[-n:], W.scale[-n:] = last.codes, last.scale
    q = W.pack(cd)
    assert q.data.numel() > 2 ** 31
    ref, bound = last.product(x)
    for T in (1, 16):
        check(cd.countdown_q4_project(x[:T], q)[:, -n:], ref[:T], bound[:T], "y")
        h = cd.countdown_q4_gated(x[:T], q, q, h=torch.empty((T, rows), device="cuda"))
        a, e = ref[:T], bound[:T]
        silu = a * torch.sigmoid(a)
        check(h[:, -n:], silu * a, 1.1 * e * a.abs() + (silu.abs() + 1.1 * e) * e + 16 * U * (silu * a).abs(), "h")
    dense = cd.countdown_q4_unpack(q)
    check(dense[-n:], last.dense(), torch.zeros_like(last.dense()), "unpacked")
    again = cd.countdown_q4_quantize(dense, group)
    assert torch.equal(cd.countdown_q4_unpack(again)[-n:],
                       cd.countdown_q4_unpack(cd.countdown_q4_quantize(dense[-n:], group)))


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,cols", [(8, 8), (16, 128), (40, 1000), (256, 688), (24, 33000)])
def test_unpack_gives_back_what_was_packed(cd, rows, cols, group):
    W = Matrix(rng(3), rows, cols, group)
    q = W.pack(cd)
    assert q.data.numel() == cd.countdown_q4_bytes(rows, cols, group)
    want = W.dense().to(BF16)
    assert torch.equal(cd.countdown_q4_unpack(q), want)
    wider = torch.full((rows, cols + 16), 7.0, dtype=BF16, device="cuda")
    cd.countdown_q4_unpack(q, W=wider[:, 8:-8])
    assert torch.equal(wider[:, 8:-8], want)
    wider[:, 8:-8] = 7.0
    assert bool((wider == 7.0).all())


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,cols", [(8, 8), (40, 1000), (256, 688)])
def test_quantize(cd, rows, cols, group):
    """The same scales and codes as the definition in elementary fp32 operations, bit by bit."""
    g = rng(4)
    W = torch.randn((rows, cols + 8), generator=g, device="cuda").to(BF16)[:, :cols]
    W[0] = 0.0                          # a group of zeros
    W[1] = torch.where(W[1] > 0, 1.0, -1.0)  # ties of the largest magnitude
    W[2] = W[2] * 1e-38                 # below fp32's normal numbers, some
    W[3] = 3e38
    n = -(-cols // group)
    padded = torch.zeros((rows, n * group), device="cuda")
    padded[:, :cols] = W.float()
    top = padded.reshape(rows, n, group).abs().amax(dim=2)
    scale = (top / 7).to(BF16)
    each = wide(scale.float(), group, cols)
    codes = torch.where(each > 0, W.float() / each, 0.0).round().clamp(-8, 7).to(torch.int8)
    q = cd.countdown_q4_quantize(W, group)
    p = cd.countdown_q4_pack(codes, scale, group)
    assert torch.equal(q.data, p.data)
    back = cd.countdown_q4_unpack(q).double()  # off by half a step, and by the roundings of the scale
    off = (back - W.double()).abs()
    assert bool((off <= (0.5 + 8 * 2.0 ** -8) * each.double() + 1e-40).all())


def test_quantize_marks_groups_that_are_not_finite(cd):
    W = torch.randn((16, 256), generator=rng(), device="cuda").to(BF16)
    W[3, 5], W[7, 130], W[9, 200] = float("nan"), float("inf"), -float("inf")
    back = cd.countdown_q4_unpack(cd.countdown_q4_quantize(W, 64)).reshape(16, 4, 64)
    bad = torch.zeros((16, 4), dtype=torch.bool, device="cuda")
    bad[3, 0], bad[7, 2], bad[9, 3] = True, True, True
    assert bool(torch.isnan(back[bad]).all()) and bool(torch.isfinite(back[~bad].float()).all())


def test_codes_keep_their_low_bits(cd):
    codes = torch.arange(-128, 128, device="cuda", dtype=torch.int16).to(torch.int8).repeat(8, 1)
    scale = torch.ones((8, 2), dtype=BF16, device="cuda")
    want = (codes.int() & 15)
    want = torch.where(want > 7, want - 16, want)
    # the stored number is (code + 8) & 15: a code outside -8..7 counts modulo 16
    assert torch.equal(cd.countdown_q4_unpack(cd.countdown_q4_pack(codes, scale, 128)).int(), want)


@pytest.mark.parametrize("T", [1, 6, 16])
def test_strides_leave_the_rest(cd, T):
    g = rng(5)
    W, V, x = Matrix(g, 200, 520, 64), Matrix(g, 200, 520, 64), tokens(g, T, 520)
    q, r = W.pack(cd), V.pack(cd)
    wx = torch.full((T + 2, 600), float("nan"), dtype=BF16, device="cuda")
    xv = wx[1:-1, 40:560]
    xv.copy_(x)
    for dtype in (F32, BF16):
        wy = torch.full((T + 2, 232), 7.0, dtype=dtype, device="cuda")
        yv = wy[1:-1, 16:216]
        base = torch.randn((T, 240), generator=g, device="cuda").to(dtype)[:, 8:208]
        want = cd.countdown_q4_project(x, q, base=base.contiguous())
        assert torch.equal(cd.countdown_q4_project(xv, q, base=base, y=yv), want)
        h = cd.countdown_q4_gated(x, q, r, h=torch.empty((T, 200), dtype=dtype, device="cuda"))
        assert torch.equal(cd.countdown_q4_gated(xv, q, r, h=yv), h)
        yv.fill_(7.0)
        assert bool((wy == 7.0).all())


def test_bad_numbers_stay_with_their_token_and_row(cd):
    g = rng(6)
    W, x = Matrix(g, 72, 520, 32), tokens(g, 5, 520)
    want = cd.countdown_q4_project(x, W.pack(cd))
    for bad in (float("nan"), float("inf"), -float("inf")):
        y, V = x.clone(), Matrix(rng(6), 72, 520, 32)
        y[2, 300] = bad
        V.scale[40, 3] = bad
        got = cd.countdown_q4_project(y, V.pack(cd))
        hit = torch.zeros((5, 72), dtype=torch.bool, device="cuda")
        hit[2], hit[:, 40] = True, True
        assert torch.equal(got[~hit], want[~hit]) and not bool(torch.isfinite(got[hit]).any())


def test_empty_call(cd):
    W = Matrix(rng(), 72, 64, 32).pack(cd)
    x = torch.empty((0, 64), dtype=BF16, device="cuda")
    assert cd.countdown_q4_project(x, W).shape == (0, 72)
    assert cd.countdown_q4_gated(x, W, W).shape == (0, 72)


def test_graph_replays_with_other_values(cd):
    g = rng(7)
    W, V = Matrix(g, 520, 1032, 64), Matrix(g, 264, 520, 32)
    q, u, d = W.pack(cd), Matrix(g, 520, 1032, 64).pack(cd), V.pack(cd)
    x = tokens(g, 4, 1032)
    base = torch.randn((4, 264), generator=g, device="cuda")
    h = torch.empty((4, 520), dtype=BF16, device="cuda")
    y = torch.empty((4, 264), device="cuda")
    graph = torch.cuda.CUDAGraph()
    cd.countdown_q4_gated(x, q, u, h=h)
    with torch.cuda.graph(graph):
        cd.countdown_q4_gated(x, q, u, h=h)
        cd.countdown_q4_project(h, d, base=base, y=y)
    for seed in (1, 2, 3):
        x.copy_(tokens(rng(seed), 4, 1032))
        y.fill_(float("nan"))
        graph.replay()
        want = cd.countdown_q4_project(cd.countdown_q4_gated(x, q, u), d, base=base)
        torch.cuda.synchronize()
        assert torch.equal(y, want)


def test_one_matrix_on_two_streams(cd):
    g = rng(8)
    W = Matrix(g, 1032, 2056, 128).pack(cd)
    x = [tokens(g, 8, 2056), tokens(g, 3, 2056)]
    want = [cd.countdown_q4_project(v, W) for v in x]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in x], []
    for _ in range(10):
        for v, s in zip(x, streams):
            y = torch.empty((v.shape[0], 1032), device="cuda")
            s.wait_stream(torch.cuda.current_stream())
            cd.countdown_q4_project(v, W, y=y, stream=s)
            got.append(y)
    torch.cuda.synchronize()
    for i, y in enumerate(got):
        assert torch.equal(y, want[i % 2])


def test_binding_refusals(cd):
    g = rng(9)
    M = Matrix(g, 72, 64, 32)
    W, V, x = M.pack(cd), Matrix(g, 72, 64, 64).pack(cd), tokens(g, 4, 64)
    out = torch.empty((4, 72), device="cuda")
    for call, error in [
        (lambda: cd.countdown_q4_pack(M.codes, M.scale, 48), cd.CountdownError),
        (lambda: cd.countdown_q4_pack(M.codes, M.scale, 64), ValueError),
        (lambda: cd.countdown_q4_pack(M.codes.int(), M.scale, 32), TypeError),
        (lambda: cd.countdown_q4_pack(M.codes[:, :60].contiguous(), M.scale, 32), cd.CountdownError),
        (lambda: cd.countdown_q4_pack(M.codes.cpu(), M.scale, 32), ValueError),
        (lambda: cd.countdown_q4_quantize(M.codes, 32), TypeError),
        (lambda: cd.countdown_q4_quantize(x.t(), 32), ValueError),
        (lambda: cd.Q4(72, 64, 32, W.data[:-16]), ValueError),
        (lambda: cd.Q4(72, 64, 40, W.data), cd.CountdownError),
        (lambda: cd.countdown_q4_project(x.float(), W), TypeError),
        (lambda: cd.countdown_q4_project(x[:, :56], W), ValueError),
        (lambda: cd.countdown_q4_project(x.repeat(5, 1), W), cd.CountdownError),  # 20 tokens
        (lambda: cd.countdown_q4_project(x, W, y=out.double()), TypeError),
        (lambda: cd.countdown_q4_project(x, W, base=out.to(BF16), y=out), TypeError),
        (lambda: cd.countdown_q4_gated(x, W, V), ValueError),
        (lambda: cd.countdown_q4_unpack(W, W=out), TypeError),
    ]:
        with pytest.raises(error):
            call()


def test_a_layer_in_four_bits(cd):
    """The whole FFN of a decode step in 4 bits, and of the same tokens as a prompt: unpacked weights
    through the gated block."""
    g = rng(10)
    m, f, T = 256, 688, 9
    Wg, Wu = (torch.randn((f, m), generator=g, device="cuda").mul_(0.08).to(BF16) for _ in range(2))
    Wd = torch.randn((m, f), generator=g, device="cuda").mul_(0.08).to(BF16)
    qg, qu, qd = (cd.countdown_q4_quantize(w, 64) for w in (Wg, Wu, Wd))
    x = tokens(g, T, m)
    h = cd.countdown_q4_gated(x, qg, qu)
    y = cd.countdown_q4_project(h, qd)
    dg, du, dd = (cd.countdown_q4_unpack(q) for q in (qg, qu, qd))
    with cd.Gated(m, f, T) as p:
        hp = cd.countdown_gated_forward(p, x, dg, du)
    # what unpack rounds: half a bf16 step of each weight, and of h
    x64, a, b = x.double(), dg.double(), du.double()
    step = 2.0 ** -8 + 1e-5
    eg, eu = step * (x64.abs() @ a.abs().t()), step * (x64.abs() @ b.abs().t())
    gate, up = x64 @ a.t(), x64 @ b.t()
    silu = gate * torch.sigmoid(gate)
    eh = 1.1 * eg * up.abs() + (silu.abs() + 1.1 * eg) * eu
    eh = eh + 2 * step * ((silu * up).abs() + eh)
    assert bool(((h.double() - hp.double()).abs() <= eh + 1e-30).all())
    yp = hp.double() @ dd.double().t()
    ey = eh @ dd.double().abs().t() + step * ((hp.double().abs() + eh) @ dd.double().abs().t())
    assert bool(((y.double() - yp).abs() <= ey + 1e-30).all())
