"""The gated block's kernels that the sizes of test_gpu_gated.py do not reach, with its cases and bounds: tiles of
rows that begin on cache lines, weights past the caches, several terms of few tokens."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_gated import BF16, F32, Case, check  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def cd():
    from paper_2505_17701_amd import binding

    return binding


def forward_and_backward(cd, shape, dtype):
    c = Case(*shape)
    with cd.Gated(c.m, c.f, c.T, train=True, fp32_grads=dtype is F32) as p:
        h = cd.countdown_gated_forward(p, c.x, c.Wg, c.Wu, h=torch.empty((c.T, c.f), dtype=dtype, device="cuda"))
        got = cd.countdown_gated_backward(p, c.x, c.dh, c.Wg, c.Wu)
    check(h, *c.h(), "h")
    for g, (name, (ref, bound)) in zip(got, c.grads(dtype).items()):
        check(g, ref, bound, name)


# more than 64 MB of weights: dx of fp32 gradients (three terms), of two terms, of one
@pytest.mark.parametrize("shape,dtype", [((4, 4096, 4104), F32), ((64, 2048, 8200), F32), ((1, 8192, 4096), BF16),
                                         ((4, 4096, 4104), BF16)], ids=str)
def test_weights_of_several_terms(cd, shape, dtype):
    forward_and_backward(cd, shape, dtype)
