"""Adapters of more than 64 ranks over 8192 tokens and more, where tiles have 32 tokens: against the
definition in 64 bits, in both output types (tolerances: test_gpu_adapters.py)."""
import pytest

from test_gpu_adapters import Case, check

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def cd():
    from paper_2505_17701_amd import binding

    return binding


SHAPES = [  # T, d_in, d_out, rank, adapters, ids
    (8192, 136, 72, 72, 3, "runs"), (8200, 72, 264, 136, 5, "mixed"), (9001, 64, 136, 256, 2, "runs"),
    (8300, 264, 64, 200, 40, "mixed"), (8193, 64, 64, 64, 1, "one"), (8192, 72, 136, 104, 3, "none"),
]


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", SHAPES)
def test_long_batches_of_many_ranks(cd, shape, kind):
    c = Case(11, *shape)
    delta, mag = c.delta()
    want = c.grads()
    base, dbase = c.base.to(kind), c.dbase.to(kind)
    d = c.dev()
    with cd.Adapters(c.di, c.do, c.r, c.n, max_tokens=c.T, train=True) as pool:
        args = (d.ids, d.A, d.B, d.scale)
        y = cd.countdown_adapters_add(pool, d.x, *args, base=base.cuda())
        check(y, delta + base.double(), mag + base.double().abs(), c.di + c.r, "y")
        place = base.cuda()
        cd.countdown_adapters_add(pool, d.x, *args, base=place, y=place)
        assert torch.equal(place, y)
        dx, dA, dB = cd.countdown_adapters_backward(pool, d.x, d.dy, *args, base=dbase.cuda())
        v, m, adds = want["dx"]
        check(dx, v + dbase.double(), m + dbase.double().abs(), adds, "dx")
        check(dA, *want["dA"], "dA")
        check(dB, *want["dB"], "dB")
