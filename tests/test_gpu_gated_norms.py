"""fp32 results by the 2-norm of their error, close enough that a lost bf16 term of dg and du is seen.

A rounding to nearest is off by a number spread evenly over a step: in rms 2^-24 / 3^1/2 of the power of two
below the value, and over values spread evenly within a power of two 0.735 of that, E = 0.735 2^-24 / 3^1/2. Let an MFMA of
32 products round once every 8 of them or less often, independently, over partial sums that grow as a random walk: their
squares add up to n / 8 (1 / 2) of the result's, so n products are off by S(n) = (n / 16)^1/2 E of it.

g and u are off by e = S(d_model) of their rms; g's is at most 1.3 in these cases. SiLU(g) has an rms of at least half of
g's (s^2 + (1 - s)^2 >= 1/2 for g and -g together) and a slope of at most 1.1; the slope has an rms of at least 1/2
(SiLU'(g) + SiLU'(-g) = 1) and a slope of at most 1/2. So h is off by e + 2.2 e, du by 2.2 e, dg by e + 1.3 e, and all by 8 E
for the sigmoid and the products beside it. A gradient's sum adds S of its products, three for each pair of elements.

4 bits: 9 (group + 8)^1/2 / rms(c) + (groups)^1/2 roundings as in test_gpu_q4_waves.py."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from perf import more_operators as operators  # noqa: E402
from test_gpu_gated import BF16, Case  # noqa: E402

E = 0.735 * 2.0 ** -24 / 3 ** 0.5
LISTED = {c["name"]: c for c in operators.listed() if c["dtype"] == operators.F32}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def cd():
    from paper_2505_17701_amd import binding

    return binding


def S(n):
    return (n / 16) ** 0.5 * E


def limits(T, m, f):
    d = 2.3 * S(m) + 8 * E
    return {"h": 3.2 * S(m) + 8 * E, "dx": d + S(6 * f), "dW_gate": d + S(3 * T), "dW_up": d + S(3 * T)}


def off(got, ref):
    return float((got.double() - ref).norm() / ref.norm())


@pytest.mark.parametrize("name", LISTED)
def test_listed_case(monkeypatch, name):
    case = {k: v for k, v in LISTED[name].items() if k != "name"}
    monkeypatch.setattr(operators, "own", True)
    got = operators.run(operators.prepare(case, 6))
    ref = operators.exact(case, 6)
    if case["op"] == "backward":
        most = limits(case["tokens"], case["d_model"], case["d_ff"])
        for k in got:
            assert off(got[k], ref[k]) <= most[k], k
    elif case["op"] == "forward":
        assert off(got, ref) <= limits(case["tokens"], case["d_model"], case["d_ff"])["h"]
    else:
        groups = -(-case["cols"] // case["group"])  # (codes of rms 3)
        assert off(got, ref) <= (9 * (case["group"] + 8) ** 0.5 / 3 + groups ** 0.5) * E


def two_terms(d):
    """d in two bf16 terms, both to nearest: the least that is lost without the third"""
    first = d.to(BF16).double()
    return first + (d - first).to(BF16).double()


# dx and the weights' gradients in 256 x 256 tiles; in 64 x 128 and 128 x 128; in 64 x 64; in one launch
@pytest.mark.parametrize("shape", [(520, 2048, 2816), (777, 1024, 8008), (300, 1024, 2816), (1000, 64, 512),
                                   (300, 128, 512)], ids=str)
def test_gradients(cd, shape):
    c = Case(*shape, seed=4, sigma=shape[1] ** -0.5)
    with cd.Gated(c.m, c.f, c.T, train=True, fp32_grads=True) as p:
        got = cd.countdown_gated_backward(p, c.x, c.dh, c.Wg, c.Wu)
    x, Wg, Wu, dh = c.x.double(), c.Wg.double(), c.Wu.double(), c.dh.double()
    g, u = x @ Wg.t(), x @ Wu.t()
    s = torch.sigmoid(g)
    dg, du = dh * u * s * (1 + g * (1 - s)), dh * g * s
    most = limits(*shape)
    for name, out, of in (("dx", got[0], lambda a, b: a @ Wg + b @ Wu), ("dW_gate", got[1], lambda a, b: a.t() @ x),
                          ("dW_up", got[2], lambda a, b: b.t() @ x)):
        ref = of(dg, du)
        assert off(out, ref) <= most[name], name
        assert off(of(two_terms(dg), two_terms(du)), ref) > most[name], f"{name}: the limit would not see it"
