"""The adapters on inputs whose results are exact in fp32, compared bit by bit.

Every x (or dy) is an odd number of 8 bits, and a row of the first factor has three entries,
65536, 256 and 1: a latent is a whole number of 24 bits, each of its three bytes odd and at least 129. Partial
sums in any order are whole numbers below 2^24, so nothing is rounded. The other factor
picks one latent for each result, times 1 or -1, and scales are powers of two. A latent that loses
its last byte, one of its bf16 terms, or any order in which these lie, changes results."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def cd():
    from paper_2505_17701_amd import binding

    return binding


def digits(g, T, width):
    """Odd numbers from 129 to 255, one sign a token."""
    sign = torch.randint(0, 2, (T, 1), generator=g) * 2 - 1
    return ((torch.randint(0, 64, (T, width), generator=g) * 2 + 129) * sign).double()


def weights(g, n, rank, width):
    """[n, rank, width]: 65536, 256 and 1 at three places of each row."""
    w = torch.zeros(n, rank, width).double()
    for a in range(n):
        for k in range(rank):
            at = torch.randperm(width, generator=g)[:3]
            w[a, k, at] = torch.tensor([65536.0, 256.0, 1.0]).double()
    return w


def pick(n, rank, width):
    """[n, rank, width]: one entry, 1 or -1, in each column."""
    w = torch.zeros(n, rank, width).double()
    at = torch.arange(width)
    for a in range(n):
        w[a, (at + 97 * a) % rank, at] = (1 - 2 * (at // rank % 2)).double()
    return w


def pick_tokens(ids, n, T, width):
    """[T, width]: in each column one entry, 1 or -1, among the tokens of each adapter."""
    w = torch.zeros(T, width).double()
    at = torch.arange(width)
    for a in range(n):
        rows = torch.nonzero(ids == a).flatten()
        if len(rows):
            w[rows[(at * 7 + a) % len(rows)], at] = (1 - 2 * (at % 2)).double()
    return w


def token_ids(g, T, n):
    """Runs of tokens; the last adapter has none where there are three or more."""
    ids = torch.empty(T, dtype=torch.int32)
    t = 0
    while t < T:
        m = int(torch.randint(1, max(2, T // 5 + 1), (1,), generator=g))
        ids[t:t + m] = int(torch.randint(-1 if n > 1 else 0, n - (n > 2), (1,), generator=g))
        t += m
    return ids


def latents(ids, v, w, scale):
    """scale_a w_a v_t [T, rank], zeros without an adapter."""
    out = torch.zeros(len(ids), w.shape[1]).double()
    for a in range(len(w)):
        rows = torch.nonzero(ids == a).flatten()
        out[rows] = scale[a] * (v[rows] @ w[a].t())
    used = out[(ids >= 0)] / scale[ids[ids >= 0].long()][:, None]
    for shift in (1, 256, 65536):  # all three bytes matter
        assert bool(((used.abs() / shift).floor() % 256 >= 129).all())
    return out


def dev(t):
    assert torch.equal(t.to(BF16).double(), t)
    return t.to(BF16).cuda()


FEW = [  # T, d_in, d_out, rank, adapters
    (1, 264, 520, 16, 1), (5, 264, 520, 24, 3), (16, 2056, 256, 8, 4), (13, 520, 1032, 32, 2),
]
BY_TOKEN = [(40, 264, 72, 40, 3), (64, 520, 1032, 128, 2), (3, 4096, 1064, 72, 2), (9, 72, 40, 256, 2)]
GROUPED = [
    (9000, 264, 680, 8, 3), (4300, 264, 712, 16, 1), (3000, 520, 424, 24, 5), (2200, 648, 328, 32, 4),
    (2600, 520, 136, 40, 3), (2100, 264, 248, 64, 6), (1100, 264, 520, 80, 5), (600, 264, 184, 256, 3),
    (8200, 72, 64, 72, 3), (8300, 136, 64, 136, 2), (8200, 64, 72, 256, 3),
]


@pytest.mark.parametrize("shape", FEW + BY_TOKEN + GROUPED)
def test_outputs(cd, shape):
    """y = B lat: lat's three bytes arrive in every output."""
    T, di, do, r, n = shape
    g = torch.Generator().manual_seed(1)
    ids, x, A = token_ids(g, T, n), digits(g, T, di), weights(g, n, r, di)
    scale = torch.tensor([1.0, -0.5, 4.0, -1.0, 0.125, 2.0])[:n].double()
    B = pick(n, r, do).transpose(1, 2).contiguous()
    lat = latents(ids, x, A, scale)
    want = torch.zeros(T, do).double()
    for a in range(n):
        rows = torch.nonzero(ids == a).flatten()
        want[rows] = lat[rows] @ B[a].t()
    args = (ids.cuda(), dev(A), dev(B), scale.float().cuda())
    with cd.Adapters(di, do, r, n, max_tokens=max(T, 16)) as pool:
        y = cd.countdown_adapters_add(pool, dev(x), *args)
        assert torch.equal(y.cpu().double(), want)
        if T <= 16:
            W = torch.zeros(do, di, dtype=BF16, device="cuda")
            y = cd.countdown_adapters_project(pool, dev(x), W, *args)
            assert torch.equal(y.cpu().double(), want)


@pytest.mark.parametrize("shape", FEW + BY_TOKEN + GROUPED)
def test_gradients_of_x_and_A(cd, shape):
    """dx = A^T glat and dA = glat x^T: glat's three bytes arrive in both."""
    T, di, do, r, n = shape
    g = torch.Generator().manual_seed(2)
    ids, dy, Bt = token_ids(g, T, n), digits(g, T, do), weights(g, n, r, do)
    scale = torch.tensor([-2.0, 1.0, 0.25, 8.0, -0.5, 1.0])[:n].double()
    A, x = pick(n, r, di), pick_tokens(ids, n, T, di)
    glat = latents(ids, dy, Bt, scale)
    dx, dA = torch.zeros(T, di).double(), torch.zeros(n, r, di).double()
    for a in range(n):
        rows = torch.nonzero(ids == a).flatten()
        dx[rows] = glat[rows] @ A[a]
        dA[a] = glat[rows].t() @ x[rows]
    args = (dev(x), dev(dy), ids.cuda(), dev(A), dev(Bt.transpose(1, 2).contiguous()),
            scale.float().cuda())
    with cd.Adapters(di, do, r, n, max_tokens=T, train=True) as pool:
        out = torch.empty(T, di, device="cuda")
        got = cd.countdown_adapters_backward(pool, *args, dx=out)
        assert torch.equal(got[0].cpu().double(), dx) and torch.equal(got[1].cpu().double(), dA)


@pytest.mark.parametrize("shape", FEW + BY_TOKEN + GROUPED)
def test_gradient_of_B(cd, shape):
    """dB = dy (scale lat)^T: lat's three bytes arrive in it."""
    T, di, do, r, n = shape
    g = torch.Generator().manual_seed(3)
    ids, x, A = token_ids(g, T, n), digits(g, T, di), weights(g, n, r, di)
    scale = torch.tensor([0.5, 1.0, -4.0, 1.0, -0.25, 16.0])[:n].double()
    dy = pick_tokens(ids, n, T, do)
    lat = latents(ids, x, A, scale)
    dB = torch.zeros(n, do, r).double()
    for a in range(n):
        rows = torch.nonzero(ids == a).flatten()
        dB[a] = dy[rows].t() @ lat[rows]
    B = pick(n, r, do).transpose(1, 2).contiguous()
    args = (dev(x), dev(dy), ids.cuda(), dev(A), dev(B), scale.float().cuda())
    with cd.Adapters(di, do, r, n, max_tokens=T, train=True) as pool:
        for need in ((True, True, True), (False, False, True)):
            got = cd.countdown_adapters_backward(pool, *args, need=need)
            assert torch.equal(got[2].cpu().double(), dB)
