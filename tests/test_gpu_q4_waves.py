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
