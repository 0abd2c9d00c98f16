"""Every kernel of the 4-bit calls, at the calls of test_host_gated_routes.py, with the cases and bounds of
test_gpu_q4.py: four waves a workgroup, two row tiles, weights past the caches; row tiles of an odd number, last groups
of blocks that are not whole."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_q4 import BF16, F32, U, Matrix, check, rng, tokens  # noqa: E402
from test_host_gated_routes import Q4_GATED, Q4_PROJECT  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def cd():
    from paper_2505_17701_amd import binding

    return binding


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("call", [c[:3] for c in Q4_PROJECT], ids=str)
def test_project(cd, call, group):
    T, rows, cols = call
    g = rng(11)
    W, x = Matrix(g, rows, cols, group), tokens(g, T, cols)
    q = W.pack(cd)
    ref, bound = W.product(x)
    check(cd.countdown_q4_project(x, q), ref, bound, "y")
    base = torch.randn((T, rows), generator=g, device="cuda").to(BF16)
    y = base.clone()
    cd.countdown_q4_project(x, q, base=y, y=y)
    check(y, ref + base.double(), bound + U * (ref.abs() + base.double().abs()), "in place")


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("call", [c[:3] for c in Q4_GATED], ids=str)
def test_gated(cd, call, group):
    T, rows, cols = call
    g = rng(12)
    Wg, Wu, x = Matrix(g, rows, cols, group), Matrix(g, rows, cols, group), tokens(g, T, cols)
    (a, ea), (u, eu) = Wg.product(x), Wu.product(x)
    silu = a * torch.sigmoid(a)
    bound = 1.1 * ea * u.abs() + (silu.abs() + 1.1 * ea) * eu + 16 * U * (silu * u).abs()
    for dtype in (F32, BF16):
        h = torch.empty((T, rows), dtype=dtype, device="cuda")
        check(cd.countdown_q4_gated(x, Wg.pack(cd), Wu.pack(cd), h=h), silu * u, bound, "h")


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("most", [1, 0])
@pytest.mark.parametrize("T,rows,cols", [(1, 520, 4096), (7, 6152, 1000), (16, 4104, 1032)])
def test_small_codes(cd, T, rows, cols, group, most):
    """Codes of -1..1, or 0 alone, beside scales that are not: a code enters as 24 + c, so the bound (by 56 times the
    sum of |scale x|) is that of any codes, and codes of 0 need not give 0."""
    g = rng(13)
    W, V, x = Matrix(g, rows, cols, group), Matrix(g, rows, cols, group), tokens(g, T, cols)
    x[:, cols // 2] = 1000.0  # one column above the others
    for M in (W, V):
        M.codes.clamp_(-most, most)
    ref, bound = W.product(x)
    check(cd.countdown_q4_project(x, W.pack(cd)), ref, bound, "y")
    u, eu = V.product(x)
    silu = ref * torch.sigmoid(ref)
    check(cd.countdown_q4_gated(x, W.pack(cd), V.pack(cd), h=torch.empty((T, rows), device="cuda")), silu * u,
          1.1 * bound * u.abs() + (silu.abs() + 1.1 * bound) * eu + 16 * U * (silu * u).abs(), "h")


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("T,rows,cols", [(1, 520, 4096), (13, 4104, 4096)])
def test_errors_of_codes_by_their_size(cd, T, rows, cols, group):
    """The 2-norm of the error, which grows as the codes get smaller. A group's sum starts from -24 times the group's x
    and comes back by 24 + c. Let a product of 32 columns round once every 8 of them or less often; the partial sum
    of k columns is about 24 k^1/2 rms(scale x), and a rounding off by at most 2^-24 of it, independently. Their squares
    over both ways add up to 2 * 24^2 * 8 (1 + 2 + .. + group / 8) = 24^2 group^2 / 8 and more for few, against group c^2
    of the result: 8.5 group^1/2 / rms(c), 9 with the last step's; and (groups)^1/2 for adding up the groups."""
    g = rng(14)
    x = tokens(g, T, cols)
    for most in (8, 1):
        W = Matrix(g, rows, cols, group)
        W.codes.clamp_(-most, most)
        ref, _ = W.product(x)
        rms = float(W.codes.double().square().mean().sqrt())
        y = cd.countdown_q4_project(x, W.pack(cd)).double()
        limit = (9 * (group + 8) ** 0.5 / rms + (cols / group) ** 0.5) * 2.0 ** -24
        assert float((y - ref).norm() / ref.norm()) <= limit
