"""The gated block's kernels that the sizes of test_gpu_gated.py do not reach, with its cases and bounds: tiles of
rows that begin on cache lines, weights past the caches, several terms of few tokens."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_gated import BF16, F32, Case, check  # noqa: E402
from test_host_gated_routes import PROJECTIONS  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def cd():
    from paper_2505_17701_amd import binding

    return binding


def forward_and_backward(cd, shape, dtype, at=0):
    c = Case(*shape)
    if at:  # rows of x at `at` of longer ones
        wide = torch.full((c.T, c.m + 64), float("nan"), dtype=BF16, device="cuda")
        wide[:, at:at + c.m] = c.x
        c.x = wide[:, at:at + c.m]
    with cd.Gated(c.m, c.f, c.T, train=True, fp32_grads=dtype is F32) as p:
        h = cd.countdown_gated_forward(p, c.x, c.Wg, c.Wu, h=torch.empty((c.T, c.f), dtype=dtype, device="cuda"))
        got = cd.countdown_gated_backward(p, c.x, c.dh, c.Wg, c.Wu)
    check(h, *c.h(), "h")
    for g, (name, (ref, bound)) in zip(got, c.grads(dtype).items()):
        check(g, ref, bound, name)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("call", [c[:4] for c in PROJECTIONS], ids=str)
def test_every_tile_of_the_projections(cd, call, dtype):
    forward_and_backward(cd, call[:3], dtype, call[3])


# more than 64 MB of weights: dx of fp32 gradients (three terms), of two terms, of one
@pytest.mark.parametrize("shape,dtype", [((4, 4096, 4104), F32), ((64, 2048, 8200), F32), ((1, 8192, 4096), BF16),
                                         ((4, 4096, 4104), BF16)], ids=str)
def test_weights_of_several_terms(cd, shape, dtype):
    forward_and_backward(cd, shape, dtype)


def test_gradients_whose_factors_alone_overflow(cd):
    """dg = dh u SiLU'(g) where dh u is past the largest number and the slope brings it back, or is 0.

    u = 2^125, dh = 2^14, both exact. dg is off by 16 (1 + |g|) s u 2^-23 as in test_gpu_gated.py, of which the slope is
    a part of (|g| - 1) / (|g| + 1) and more, 17 units; dx sums eight equal terms of three parts each, all of one
    sign or below 2^-7 of it: 24 additions, each off by 2^-24. (W_up's factors meet du in another column.)"""
    x = torch.zeros((4, 64), device="cuda")
    x[:, 0] = torch.tensor([-200.0, -60.0, -40.0, 2.0 ** -60])
    x[:, 1] = 2.0 ** 62
    W, V = torch.zeros((8, 64), device="cuda"), torch.zeros((8, 64), device="cuda")
    W[:, 0], V[:, 1] = 1.0, 2.0 ** 63
    x, W, V = x.to(BF16), W.to(BF16), V.to(BF16)
    dh = torch.full((4, 8), 2.0 ** 14, device="cuda", dtype=BF16)
    dh[3] = 2.0 ** -14
    with cd.Gated(64, 8, 4, train=True, fp32_grads=True) as p:
        dx, _, _ = cd.countdown_gated_backward(p, x, dh, W, V, need=(True, False, False))
    g = x[:, 0].double()
    s = torch.sigmoid(g)
    want = 8 * dh[:, 0].double() * 2.0 ** 125 * torch.where(g == -200.0, 0.0, s * (1 + g * (1 - s)))
    assert bool(torch.isfinite(dx).all())
    assert bool(((dx[:, 0].double() - want).abs() <= 32 * 2.0 ** -23 * want.abs()).all())


def test_forward_calls_of_one_handle_at_once(cd):
    """The forward call uses no workspace."""
    cases = [Case(300, 520, 2056, seed=s) for s in (1, 2)]
    with cd.Gated(520, 2056, 300) as p:
        want = [cd.countdown_gated_forward(p, c.x, c.Wg, c.Wu) for c in cases]
        torch.cuda.synchronize()
        streams, got = [torch.cuda.Stream() for _ in cases], []
        for _ in range(8):
            for c, s in zip(cases, streams):
                with torch.cuda.stream(s):
                    got.append(cd.countdown_gated_forward(p, c.x, c.Wg, c.Wu))
        torch.cuda.synchronize()
    for i, h in enumerate(got):
        assert torch.equal(h, want[i % 2])


@pytest.mark.parametrize("T", [5, 300])
def test_one_matrix_for_both_projections(cd, T):
    """Inputs may be one and the same."""
    c = Case(T, 264, 712)
    c.Wu = c.Wg
    with cd.Gated(c.m, c.f, T, train=True, fp32_grads=True) as p:
        h = cd.countdown_gated_forward(p, c.x, c.Wg, c.Wg, h=torch.empty((T, c.f), device="cuda"))
        got = cd.countdown_gated_backward(p, c.x, c.dh, c.Wg, c.Wg)
    check(h, *c.h(), "h")
    for g, (name, (ref, bound)) in zip(got, c.grads(F32).items()):
        check(g, ref, bound, name)
