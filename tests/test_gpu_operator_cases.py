"""The framework's calls on the listed performance cases of the adapters and clipping, at their own
sizes, against exact() in 64 bits.

Tolerances are those of test_gpu_adapters.py and test_gpu_clip.py. The magnitudes that they
refer to (the same sums over absolute values) are exact() of the inputs' absolute values."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from perf import operators  # noqa: E402

U = 2.0 ** -23
CASES = {c["name"]: {k: v for k, v in c.items() if k != "name"} for c in operators.listed()}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def close(got, ref, mag, adds):
    off = (adds + 8) * U * mag
    tol = off + torch.finfo(got.dtype).eps / 2 * (ref.abs() + off)
    assert int(((got.double() - ref).abs() > tol).sum()) == 0


@pytest.mark.parametrize("name", CASES)
def test_listed_case(monkeypatch, name):
    case, seed = CASES[name], 5
    monkeypatch.setattr(operators, "own", True)
    got = operators.run(operators.prepare(case, seed))
    ref = operators.exact(case, seed)
    if case["op"] == "clip":
        n = sum(r * c for r, c in operators._grad_shapes(case))
        assert abs(float(got["norm"]) - float(ref["norm"])) <= 2.0 ** -52 * (n / 2 + 2) * float(ref["norm"])
        assert (got["grads"] is None) == (not math.isfinite(case["max_norm"]))
        for o, t in zip(got["grads"] or (), ref["grads"] or ()):
            tol = (2.0 ** -23 + torch.finfo(o.dtype).eps / 2) * t.abs() + 1e-45
            assert int(((o.double() - t).abs() > tol).sum()) == 0
        return
    inputs = operators._inputs
    monkeypatch.setattr(operators, "_inputs", lambda *a: {
        k: v if k == "ids" else v.abs() for k, v in inputs(*a).items()})
    mag = operators.exact(case, seed)
    T, di, do, r = (case[k] for k in ("tokens", "d_in", "d_out", "rank"))
    if case["op"] == "backward":
        for k, adds in (("dx", do + r), ("dA", do + T), ("dB", di + T)):
            close(got[k], ref[k], mag[k], adds)
    else:
        close(got, ref, mag, di + r)
